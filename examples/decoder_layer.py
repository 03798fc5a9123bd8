"""Decoder layers with quantised linears, a paged key / value cache and ragged batches: prompts in chunks, then one token per
sequence and step.

    python examples/decoder_layer.py [--linears w4a16|mx] [--activations e2m1|e4m3] [--cache fp16|int8|e4m3|e2m1] [--layers 4] [--hidden 4096]
                                     [--heads 32] [--kv-heads 8] [--steps 32]

Linears: 4-bit integers with fp16 steps per group (w4a16), or microscaled numbers (mx: weights e2m1 in blocks of 32, activations e2m1 or e4m3
in such blocks).  Synthetic weights; prints the time of the prompts' steps and of a decode step, eager and replayed as a graph.
"""
import argparse
import math
import os
import sys
import time

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2312_03788_amd as sqp  # noqa: E402

EPS = 1e-5
CACHE_TYPES = {"fp16": torch.float16, "int8": torch.int8, "e4m3": torch.float8_e4m3fn, "e2m1": torch.uint8}  # (two e2m1 codes to a byte)
BLOCK_TYPES = {"e2m1": torch.uint8, "e4m3": torch.float8_e4m3fn}


def rotary_table(positions, head_dim, theta=1e6, device="cuda"):
    """[positions, head_dim] fp32: cosines, sines."""
    inv = theta ** (-torch.arange(head_dim // 2, dtype=torch.float64) / (head_dim // 2))
    angle = torch.arange(positions, dtype=torch.float64)[:, None] * inv
    return torch.cat([angle.cos(), angle.sin()], 1).float().to(device)


class PagedCache:
    """Keys and values of all layers in pages of `page` tokens; a sequence's pages are handed out as it grows."""

    def __init__(self, layers, pages, kv_heads, page, head_dim, dtype, sequences, max_len):
        shape = (pages, kv_heads, page, head_dim)
        self.page, self.max_len = page, max_len
        blocks = dtype == torch.uint8
        codes = shape[:3] + (head_dim // 2,) if blocks else shape
        self.k = [torch.zeros(codes, dtype=torch.float16, device="cuda").to(dtype) for _ in range(layers)]
        self.v = [torch.zeros(codes, dtype=torch.float16, device="cuda").to(dtype) for _ in range(layers)]
        block_scales = lambda: torch.zeros(shape[:3] + (head_dim // 32,), dtype=torch.uint8, device="cuda")
        scales = lambda: None if dtype == torch.float16 else block_scales() if blocks else torch.zeros(shape[:3], dtype=torch.float32, device="cuda")
        self.ks, self.vs = [scales() for _ in range(layers)], [scales() for _ in range(layers)]
        self.free = list(range(pages))[::-1]
        self.pages = [[] for _ in range(sequences)]
        self.lens = [0] * sequences

    def grow(self, news):
        """Room for `news` more tokens of every sequence: (slots, positions) of the new tokens, sequence by sequence."""
        slots, positions = [], []
        for b, n in enumerate(news):
            first, self.lens[b] = self.lens[b], self.lens[b] + n
            while len(self.pages[b]) * self.page < self.lens[b]:
                self.pages[b].append(self.free.pop())
            positions += range(first, first + n)
            slots += [self.pages[b][t // self.page] * self.page + t % self.page for t in range(first, first + n)]
        return slots, positions

    def table(self):
        width = -(-self.max_len // self.page)
        return [p + [-1] * (width - len(p)) for p in self.pages]


class Step:
    """What a step's layers share: the new tokens' places, and the sequences' page table, lengths and starts."""

    def __init__(self, cache, news):
        slots, positions = cache.grow(news)
        t = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")
        self.slots, self.positions, self.table, self.lens = t(slots), t(positions), t(cache.table()), t(cache.lens)
        self.max_q, self.max_len = max(news), cache.max_len
        self.starts = None if self.max_q == 1 and min(news) == 1 else t([sum(news[:b]) for b in range(len(news) + 1)])


class Layer:
    def __init__(self, hidden, heads, kv_heads, head_dim, intermediate, group, gen):
        self.heads, self.kv_heads, self.head_dim, self.group = heads, kv_heads, head_dim, group
        w = lambda k, n: (torch.randn((k, n), generator=gen, device="cuda") / math.sqrt(k)).half()
        self.gamma1, self.gamma2 = [(1 + 0.1 * torch.randn(hidden, generator=gen, device="cuda")).half() for _ in range(2)]
        q = lambda m: sqp.quantize_pack(m, group)
        self.qkv = q(w(hidden, (heads + 2 * kv_heads) * head_dim))
        self.o = q(w(heads * head_dim, hidden))
        self.gate_up = q(sqp.interleave_gate_up(w(hidden, intermediate), w(hidden, intermediate)))
        self.down = q(w(intermediate, hidden))

    def __call__(self, x, residual, cache, at, step, cos_sin, note=lambda name, *tensors: None):
        """x: the previous layer's output, not added to the residual yet (the first layer: the embedding, residual None).
        Returns this layer's (output, residual); note(name, inputs..., outputs...) sees every stage."""
        if residual is None:
            y, r = sqp.rmsnorm(x, self.gamma1, EPS), x
            note("norm", x, y)
        else:
            y, r = sqp.add_rmsnorm(x, residual, self.gamma1, EPS)
            note("add_norm", self.gamma1, x, residual, y, r)
        n, D = x.shape[0], self.head_dim
        qkv = sqp.w4a16_gemm(y, *self.qkv, self.group)
        note("gemm", self.qkv, y, qkv)
        q, k, v = [p.view(n, -1, D) for p in qkv.split([self.heads * D, self.kv_heads * D, self.kv_heads * D], 1)]
        c = (cache.k[at], cache.v[at])
        scales = (cache.ks[at], cache.vs[at])
        qr = sqp.kv_cache_write(k, v, step.slots, *c, *scales, q=q, cos_sin=cos_sin, positions=step.positions)
        note("cache", q, k, v, qr, at)
        a = sqp.paged_attention(qr, *c, step.table, step.lens, step.starts, *scales, max_q=step.max_q, max_len=step.max_len)
        note("attention", qr, a, at)
        o = sqp.w4a16_gemm(a.view(n, -1), *self.o, self.group)
        note("gemm", self.o, a.view(n, -1), o)
        y, r2 = sqp.add_rmsnorm(o, r, self.gamma2, EPS)
        note("add_norm", self.gamma2, o, r, y, r2)
        h = sqp.w4a16_gemm_silu_mul(y, *self.gate_up, self.group)
        note("silu", self.gate_up, y, h)
        down = sqp.w4a16_gemm(h, *self.down, self.group)
        note("gemm", self.down, h, down)
        return down, r2


class MxLayer:
    """Layer with its linears on microscaled numbers: every activation that a linear takes is in blocks of `dtype`, from the norm or from
    mx_quantize."""

    def __init__(self, hidden, heads, kv_heads, head_dim, intermediate, dtype, gen):
        self.heads, self.kv_heads, self.head_dim, self.dtype = heads, kv_heads, head_dim, dtype
        w = lambda k, n: (torch.randn((k, n), generator=gen, device="cuda") / math.sqrt(k)).half()
        self.gamma1, self.gamma2 = [(1 + 0.1 * torch.randn(hidden, generator=gen, device="cuda")).half() for _ in range(2)]
        self.qkv = sqp.mx_quantize_weight(w(hidden, (heads + 2 * kv_heads) * head_dim))
        self.o = sqp.mx_quantize_weight(w(heads * head_dim, hidden))
        self.gate_up = sqp.mx_quantize_weight(sqp.interleave_gate_up(w(hidden, intermediate), w(hidden, intermediate)))
        self.down = sqp.mx_quantize_weight(w(intermediate, hidden))

    def __call__(self, x, residual, cache, at, step, cos_sin, note=lambda name, *tensors: None):
        def blocks(t):
            b = sqp.mx_quantize(t, self.dtype)
            note("blocks", t, *b)
            return b

        def norm(gamma, x, residual):
            *y, r = sqp.add_rmsnorm_mx(x, residual, gamma, EPS, self.dtype)
            note("add_norm_mx", gamma, x, residual, *y, r)
            return y, r

        if residual is None:
            y, r = sqp.rmsnorm(x, self.gamma1, EPS), x
            note("norm", x, y)
            y = blocks(y)
        else:
            y, r = norm(self.gamma1, x, residual)
        n, D = x.shape[0], self.head_dim
        qkv = sqp.mx_gemm(*y, *self.qkv)
        note("mx_gemm", *self.qkv, *y, qkv)
        q, k, v = [p.view(n, -1, D) for p in qkv.split([self.heads * D, self.kv_heads * D, self.kv_heads * D], 1)]
        c = (cache.k[at], cache.v[at])
        scales = (cache.ks[at], cache.vs[at])
        qr = sqp.kv_cache_write(k, v, step.slots, *c, *scales, q=q, cos_sin=cos_sin, positions=step.positions)
        note("cache", q, k, v, qr, at)
        a = sqp.paged_attention(qr, *c, step.table, step.lens, step.starts, *scales, max_q=step.max_q, max_len=step.max_len)
        note("attention", qr, a, at)
        y = blocks(a.view(n, -1))
        o = sqp.mx_gemm(*y, *self.o)
        note("mx_gemm", *self.o, *y, o)
        y, r2 = norm(self.gamma2, o, r)
        h = sqp.mx_gemm_silu_mul(*y, *self.gate_up)
        note("mx_silu", *self.gate_up, *y, h)
        y = blocks(h)
        down = sqp.mx_gemm(*y, *self.down)
        note("mx_gemm", *self.down, *y, down)
        return down, r2


def run(layers, x, cache, step, cos_sin, note=lambda name, *tensors: None):
    """All layers on the new tokens' embeddings x [tokens, hidden]; returns the last residual, everything added."""
    residual = None
    for at, layer in enumerate(layers):
        x, residual = layer(x, residual, cache, at, step, cos_sin, note)
    return x + residual


def main():
    ap = argparse.ArgumentParser()
    ap.add_argument("--linears", choices=["w4a16", "mx"], default="w4a16")
    ap.add_argument("--activations", choices=list(BLOCK_TYPES), default="e2m1", help="of the mx linears")
    ap.add_argument("--cache", choices=list(CACHE_TYPES), default="e4m3")
    for name, default in (("layers", 4), ("hidden", 4096), ("heads", 32), ("kv-heads", 8), ("intermediate", 11008), ("steps", 32)):
        ap.add_argument("--" + name, type=int, default=default)
    a = ap.parse_args()
    gen = torch.Generator(device="cuda")
    gen.manual_seed(1)
    D, prompts = 128, [1500, 37, 800, 1, 311, 64, 2048, 129]
    kind, how = (Layer, 128) if a.linears == "w4a16" else (MxLayer, BLOCK_TYPES[a.activations])
    layers = [kind(a.hidden, a.heads, a.kv_heads, D, a.intermediate, how, gen) for _ in range(a.layers)]
    max_len = max(prompts) + a.steps + 2
    cache = PagedCache(a.layers, sum(-(-(n + a.steps + 2) // 64) for n in prompts), a.kv_heads, 64, D, CACHE_TYPES[a.cache], len(prompts), max_len)
    cos_sin = rotary_table(max_len, D)
    embed = lambda n: torch.randn((n, a.hidden), generator=gen, device="cuda").half()
    done = [0] * len(prompts)
    while done != prompts:  # prompts in chunks of up to 512 tokens; a sequence whose prompt has ended waits
        news = [min(512, n - d) for n, d in zip(prompts, done)]
        x, step = embed(sum(news)), Step(cache, news)
        torch.cuda.synchronize()
        t = time.perf_counter()
        run(layers, x, cache, step, cos_sin)
        torch.cuda.synchronize()
        print("prompt step: %5d new tokens, %8.2f ms" % (sum(news), (time.perf_counter() - t) * 1e3), flush=True)
        done = [d + n for d, n in zip(done, news)]
    for i in range(a.steps):
        x, step = embed(len(prompts)), Step(cache, [1] * len(prompts))
        torch.cuda.synchronize()
        t = time.perf_counter()
        run(layers, x, cache, step, cos_sin)
        torch.cuda.synchronize()
        if i == a.steps - 1:
            print("decode step: %d sequences, %.1f us" % (len(prompts), (time.perf_counter() - t) * 1e6), flush=True)
    graph = torch.cuda.CUDAGraph()  # the step's index tensors are the graph's inputs: a server writes the next step's into them
    with torch.cuda.graph(graph):
        run(layers, x, cache, step, cos_sin)
    torch.cuda.synchronize()
    t = time.perf_counter()
    for _ in range(20):
        graph.replay()
    torch.cuda.synchronize()
    print("decode step as a graph: %.1f us" % ((time.perf_counter() - t) / 20 * 1e6), flush=True)


if __name__ == "__main__":
    main()
