"""Operators on microscaled numbers (blocks of 32 values with one power-of-two scale, elements e2m1 or e4m3), as cases that can be
timed and compared.

Five kinds, with the shapes of Code Llama 7B / 13B / 34B and generic ones drawn over the same ranges:
  quant   fp16 activations [M, K] or a weight [K, N] into blocks along K, and back to fp16
  linear  the product of activations and a weight held in such blocks, plain or as SiLU(gate) * up of alternating columns;
          the activations come as codes, or as fp16 that the call quantises first
  norm    the residual's addition, the RMS norm behind it, its output in blocks, and that output back as fp16
  cache   new tokens' keys and values into a paged cache of e2m1 blocks, queries and keys rotated on the way, and the same slots
          read back as fp16
  attn    attention of each sequence's new tokens over such a cache
Where `own` is false, run() computes them in elementary torch operations in 32 bits (the norm in 64: its outputs lie next to
the borders between codes).
"""
import math
import random

import torch

own = False

EPS = 1e-5
BLOCK = 32
# of an element: the largest value, the exponent of the largest power of two, mantissa bits, the least normal exponent, and from where
# on a magnitude would round to more than the largest value (None: beyond this itself is the first)
TYPES = {"e2m1": (6.0, 2, 1, 0, 7.0), "e4m3": (448.0, 8, 3, -6, 464.0)}


def listed():
    return [
        # a ragged batch of prompts of 13B whose next product takes 8-bit activations
        {"name": "quant_13b_m1001_e4m3", "kind": "quant", "what": "rows", "M": 1001, "K": 5120, "type": "e4m3"},
        # the merged qkv weight of 34B, once per model
        {"name": "quant_34b_weight_qkv", "kind": "quant", "what": "weight", "M": 10240, "K": 8192, "type": "e2m1"},
        # one token of single-stream decoding through a 7B layer: nothing but latency
        {"name": "linear_7b_m1", "kind": "linear", "M": 1, "N": 4096, "K": 4096, "type": "e2m1", "given": "codes", "silu": False},
        # a decode batch of 34B through gate and up
        {"name": "linear_34b_m16_gate_up", "kind": "linear", "M": 16, "N": 44032, "K": 8192, "type": "e2m1", "given": "codes", "silu": True},
        # ragged prompts of 13B through the down projection, 8-bit activations quantised in front of it
        {"name": "linear_13b_m333_down_e4m3", "kind": "linear", "M": 333, "N": 5120, "K": 13824, "type": "e4m3", "given": "fp16", "silu": False},
        # a prompt chunk of 34B: the most arithmetic
        {"name": "linear_34b_m2048_qkv", "kind": "linear", "M": 2048, "N": 10240, "K": 8192, "type": "e2m1", "given": "codes", "silu": False},
        # one token of 7B
        {"name": "norm_7b_m1_e2m1", "kind": "norm", "M": 1, "H": 4096, "type": "e2m1"},
        # a prompt chunk of 34B
        {"name": "norm_34b_m2048_e2m1", "kind": "norm", "M": 2048, "H": 8192, "type": "e2m1"},
        # a decode batch of 34B (64 query heads on 8 cached ones)
        {"name": "cache_34b_m16", "kind": "cache", "T": 16, "heads": 64, "kv_heads": 8, "D": 128, "page": 16},
        # a ragged prompt chunk of 13B (every head has its own cache)
        {"name": "cache_13b_m1001", "kind": "cache", "T": 1001, "heads": 40, "kv_heads": 40, "D": 128, "page": 64},
        # a decode batch of 34B at ragged lengths up to 8192
        {"name": "attn_34b_b16_len8192", "kind": "attn", "B": 16, "new": 1, "L": 8192, "heads": 64, "kv_heads": 8, "D": 128, "page": 16},
        # the last chunk of a long prompt of 34B
        {"name": "attn_34b_chunk_1024_of_8192", "kind": "attn", "B": 1, "new": 1024, "L": 8192, "heads": 64, "kv_heads": 8, "D": 128, "page": 64},
    ]


def _log_int(rng, lo, hi, step=1):
    v = math.exp(rng.uniform(math.log(lo), math.log(hi)))
    return min(max(int(round(v / step)), -(-lo // step)), hi // step) * step


def _heads(rng):
    kv, group = rng.choice([(32, 1), (40, 1), (8, 8), (8, 4), (2, 7), (4, 6), (1, 16), (5, 3), (1, 1)])
    return {"heads": kv * group, "kv_heads": kv, "D": rng.choice([128, 128, 64]), "page": rng.choice([16, 16, 32, 64, 128, 256])}


def draw(rng):
    kind = rng.choice(["quant", "linear", "linear", "linear", "norm", "cache", "attn", "attn"])
    if kind == "quant":
        what = rng.choice(["rows", "weight"])
        if what == "rows":
            return {"kind": kind, "what": what, "M": _log_int(rng, 1, 4096), "K": _log_int(rng, 512, 22016, 32), "type": rng.choice(["e2m1", "e4m3"])}
        return {"kind": kind, "what": what, "M": _log_int(rng, 512, 10240, 8), "K": _log_int(rng, 512, 8192, 32), "type": "e2m1"}
    if kind == "linear":
        while True:
            c = {"kind": kind, "M": _log_int(rng, 1, 4096), "N": _log_int(rng, 512, 44032, 16), "K": _log_int(rng, 512, 22016, 32),
                 "type": rng.choice(["e2m1", "e4m3"]), "given": rng.choice(["codes", "codes", "fp16"]), "silu": rng.random() < 0.3}
            if c["N"] * c["K"] <= 44032 * 8192 and c["M"] * c["N"] * c["K"] <= 2048 * 10240 * 8192:
                return c
    if kind == "norm":
        return {"kind": kind, "M": _log_int(rng, 1, 2048), "H": _log_int(rng, 512, 8192, 32), "type": rng.choice(["e2m1", "e4m3"])}
    if kind == "cache":
        return {"kind": kind, "T": _log_int(rng, 1, 4096), **_heads(rng)}
    while True:
        c = {"kind": kind, "B": _log_int(rng, 1, 64), "new": 1 if rng.random() < 0.5 else _log_int(rng, 2, 1024), "L": _log_int(rng, 1, 32768), **_heads(rng)}
        if c["new"] <= c["L"] and c["B"] * c["L"] * c["kv_heads"] * c["D"] <= 16 * 8192 * 8 * 128 and c["B"] * c["new"] * c["L"] * c["heads"] <= 1024 * 8192 * 64:
            return c


def _lengths(case):
    """(cached tokens, new tokens) of every sequence, which the case alone decides.  The first sequence has the full
    lengths; of the others some are single tokens, and one in 16 is an unused place of the batch (no tokens cached)."""
    rng = random.Random(case["B"] * 1000003 + case["L"] * 31 + case["new"])
    lens, news = [case["L"]], [case["new"]]
    for _ in range(case["B"] - 1):
        n = rng.choice([1, rng.randint(1, case["new"])])
        news.append(n)
        lens.append(0 if n == 1 and rng.random() < 1 / 16 else rng.randint(max(n, case["L"] // 4), case["L"]))
    return lens, news


# ---------------------------------------------------------------- blocks in elementary operations

def _two(e, dtype):
    """2^e for whole numbers e, from the bits (torch's own powers of two are not exact everywhere)."""
    if dtype == torch.float64:
        return (e.long() + 1023 << 52).view(dtype)
    return (e.int() + 127 << 23).view(dtype)


def _blocks(z, kind):
    """Elements (the values that codes stand for, unscaled) and exponents of the blocks along the last axis: [..., n] and
    [..., n / 32].  The scale is the least power of two with which the block's largest magnitude rounds to a value of the type."""
    _, top, bits, least, over = TYPES[kind]
    b = z.unflatten(-1, (-1, BLOCK))
    most = b.abs().amax(-1, keepdim=True)
    m, x = torch.frexp(most)
    m = m * 2.0 ** (top + 1)  # the magnitude as the scale 2^(x - top - 1) leaves it
    e = x - top - 1 + ((m >= over) if kind == "e2m1" else (m > over)).to(x.dtype)
    some = most >= 2.0 ** -100
    y = torch.where(some, b * _two(-e, z.dtype), 0.0)
    _, place = torch.frexp(y)
    step = torch.clamp(place - 1, min=least) - bits
    y = torch.round(y * _two(-step, z.dtype)) * _two(step, z.dtype)
    return y.flatten(-2), torch.where(some, e, -127)[..., 0]


def _pack(y, kind):
    """The codes of elements: two e2m1 to a byte, the first in the low half, or e4m3."""
    if kind == "e4m3":
        return y.to(torch.float8_e4m3fn)
    a = y.abs()
    c = torch.where(a < 2, 2 * a, torch.where(a < 4, a + 2, a / 2 + 4)) + 8 * torch.signbit(y)
    c = c.to(torch.uint8).unflatten(-1, (-1, 2))
    return c[..., 0] | c[..., 1] << 4


def _codes(z, kind):
    """(codes, scales) of rows: the scales are the exponents plus 127 in a byte."""
    y, e = _blocks(z, kind)
    return _pack(y, kind), (e + 127).to(torch.uint8)


def _values(codes, scales):
    """What codes and scales stand for, in 32 bits."""
    if codes.dtype == torch.uint8:
        table = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0, -0.0, -0.5, -1.0, -1.5, -2.0, -3.0, -4.0, -6.0], device=codes.device)
        y = table[torch.stack([codes & 15, codes >> 4], -1).flatten(-2).int()]
    else:
        y = codes.float()
    return (y.unflatten(-1, (-1, BLOCK)) * _two(scales.int() - 127, torch.float32)[..., None]).flatten(-2)


# ---------------------------------------------------------------- inputs (from the seed alone)

def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _randn(g, *shape):
    return torch.randn(shape, generator=g, device="cuda", dtype=torch.float32)


def _activations(g, M, K):
    """fp16 rows with a few channels 30 times as large, as they come out of a norm."""
    gain = torch.ones(K, device="cuda")
    gain[torch.randperm(K, generator=g, device="cuda")[: max(1, K // 200)]] = 30.0
    return (_randn(g, M, K) * gain).half()


def _cached(g, pages, case):
    """One of the two caches as earlier steps have left it: values N(0, 1) with a few larger channels."""
    x = torch.randn((pages, case["kv_heads"], case["page"], case["D"]), generator=g, device="cuda", dtype=torch.float32)
    x[..., ::37] *= 3.0
    return _codes(x, "e2m1")


def prepare(case, seed):
    g = _gen(seed)
    s = dict(case)
    if case["kind"] == "quant":
        M, K = case["M"], case["K"]
        s["x"] = _activations(g, M, K) if case["what"] == "rows" else (_randn(g, K, M) / math.sqrt(K)).half()
        return s
    if case["kind"] == "linear":
        x = _activations(g, case["M"], case["K"])
        s["x"] = x if case["given"] == "fp16" else _codes(x.float(), case["type"])
        s["w"] = _codes(_randn(g, case["N"], case["K"]) / math.sqrt(case["K"]), "e2m1")
        return s
    if case["kind"] == "norm":
        M, H = case["M"], case["H"]
        s["x"] = _randn(g, M, H).half()
        s["residual"] = _activations(g, M, H)
        s["gamma"] = (1.0 + 0.1 * _randn(g, H)).half()
        return s
    heads, kv, D, page = case["heads"], case["kv_heads"], case["D"], case["page"]
    if case["kind"] == "cache":
        T = case["T"]
        pages = -(-T // page) + 3
        # what the merged qkv projection gives, and its three parts as views
        s["qkv"] = _randn(g, T, (heads + 2 * kv) * D).half()
        s["q"] = s["qkv"][:, : heads * D].view(T, heads, D)
        s["k"] = s["qkv"][:, heads * D: (heads + kv) * D].view(T, kv, D)
        s["v"] = s["qkv"][:, (heads + kv) * D:].view(T, kv, D)
        s["slots"] = torch.randperm(pages * page, generator=g, device="cuda")[:T].int()
        s["positions"] = torch.randint(0, 16384, (T,), generator=g, device="cuda", dtype=torch.int32)
        angle = torch.arange(16384, device="cuda", dtype=torch.float64)[:, None] * 1e6 ** (-torch.arange(D // 2, device="cuda", dtype=torch.float64) / (D // 2))
        s["cos_sin"] = torch.cat([angle.cos(), angle.sin()], 1).float()
        s["k_cache"], s["k_scales"] = _cached(g, pages, case)
        s["v_cache"], s["v_scales"] = _cached(g, pages, case)
        return s
    lens, news = _lengths(case)
    T, s["most_new"] = sum(news), max(news)
    need = [-(-n // page) for n in lens]
    pages = sum(need) + 1
    s["q"] = (2.0 * _randn(g, T, heads, D)).half()
    order = torch.randperm(pages, generator=g, device="cuda").int()
    table = torch.zeros((case["B"], max(1, -(-case["L"] // page))), dtype=torch.int32, device="cuda")
    at = 0
    for b, n in enumerate(need):
        table[b, :n] = order[at: at + n]
        at += n
    s["page_table"] = table
    s["seq_lens"] = torch.tensor(lens, dtype=torch.int32, device="cuda")
    s["q_starts"] = torch.tensor([sum(news[:b]) for b in range(case["B"] + 1)], dtype=torch.int32, device="cuda")
    s["k_cache"], s["k_scales"] = _cached(g, pages, case)
    s["v_cache"], s["v_scales"] = _cached(g, pages, case)
    return s


# ---------------------------------------------------------------- the framework's operators

def _run_own(s):
    import paper_2312_03788_amd as sqp
    dtype = {"e2m1": torch.uint8, "e4m3": torch.float8_e4m3fn}[s.get("type", "e2m1")]
    if s["kind"] == "quant":
        return sqp.mx_dequantize(*(sqp.mx_quantize(s["x"], dtype) if s["what"] == "rows" else sqp.mx_quantize_weight(s["x"])))
    if s["kind"] == "linear":
        x = sqp.mx_quantize(s["x"], dtype) if s["given"] == "fp16" else s["x"]
        return (sqp.mx_gemm_silu_mul if s["silu"] else sqp.mx_gemm)(*x, *s["w"])
    if s["kind"] == "norm":
        codes, scales, r = sqp.add_rmsnorm_mx(s["x"], s["residual"], s["gamma"], EPS, dtype)
        return sqp.mx_dequantize(codes, scales), r
    if s["kind"] == "cache":
        q = sqp.kv_cache_write(s["k"], s["v"], s["slots"], s["k_cache"], s["v_cache"], s["k_scales"], s["v_scales"],
                               q=s["q"], cos_sin=s["cos_sin"], positions=s["positions"])
        return (q,) + tuple(sqp.kv_cache_read(s["slots"], s["k_cache"], s["v_cache"], s["k_scales"], s["v_scales"]))
    return sqp.paged_attention(s["q"], s["k_cache"], s["v_cache"], s["page_table"], s["seq_lens"], s["q_starts"] if s["most_new"] > 1 else None,
                               s["k_scales"], s["v_scales"], max_q=s["most_new"], max_len=s["L"])


# ---------------------------------------------------------------- the plain forms

def _quant(s):
    x = s["x"].float()
    return _values(*_codes(x if s["what"] == "rows" else x.t().contiguous(), s["type"])).half()


def _linear(s):
    x = _values(*(_codes(s["x"].float(), s["type"]) if s["given"] == "fp16" else s["x"]))
    y = torch.matmul(x, _values(*s["w"]).t())
    if s["silu"]:
        gate, up = y[:, ::2], y[:, 1::2]
        y = gate / (1.0 + torch.exp(-gate)) * up
    return y.half()


def _norm(s):
    r = (s["x"].float() + s["residual"].float()).half()
    v = r.double()
    z = v * s["gamma"].double() * (1.0 / torch.sqrt((v * v).mean(1, keepdim=True) + EPS))
    return _values(*_codes(z, s["type"])).half(), r


def _rotate(x, c, sn):
    a, b = x.float().chunk(2, -1)
    return torch.cat([a * c - b * sn, b * c + a * sn], -1)


def _cache(s):
    c, sn = s["cos_sin"][s["positions"].long()][:, None].chunk(2, -1)
    page, row = s["slots"].long() // s["page"], s["slots"].long() % s["page"]
    out = [_rotate(s["q"], c, sn).half()]
    for x, cache, scales in ((_rotate(s["k"], c, sn), s["k_cache"], s["k_scales"]), (s["v"].float(), s["v_cache"], s["v_scales"])):
        cache[page, :, row], scales[page, :, row] = _codes(x, "e2m1")
        out.append(_values(cache[page, :, row], scales[page, :, row]).half())
    return tuple(out)


def _gathered(s, cache, scales):
    """All sequences' tokens [B, heads, L, D] in 32 bits (what lies past a sequence's length is masked later)."""
    t = torch.arange(s["L"], device="cuda")
    page, row = s["page_table"].long()[:, t // s["page"]], t % s["page"]
    return _values(cache[page, :, row], scales[page, :, row]).transpose(1, 2).contiguous()


def _attend(s):
    T, heads, D = s["q"].shape
    kv, B = s["kv_heads"], s["B"]
    starts, lens = s["q_starts"].long(), s["seq_lens"].long()
    n = starts[1:] - starts[:-1]
    token = torch.arange(T, device="cuda")
    seq = torch.searchsorted(starts[1:].contiguous(), token, right=True)
    place = token - starts[seq]
    most = s["most_new"]
    q = torch.zeros((B, most, heads, D), device="cuda")
    q[seq, place] = s["q"].float()
    q = q.view(B, most, kv, heads // kv, D).permute(0, 2, 3, 1, 4).reshape(B, kv, heads // kv * most, D)
    k, v = _gathered(s, s["k_cache"], s["k_scales"]), _gathered(s, s["v_cache"], s["v_scales"])
    scores = torch.matmul(q * D ** -0.5, k.transpose(2, 3).contiguous()).view(B, heads, most, s["L"])
    last = (lens - n)[:, None] + torch.arange(most, device="cuda")
    hidden = torch.arange(s["L"], device="cuda") > last[:, None, :, None]
    scores.masked_fill_(hidden, float("-inf"))
    top = scores.amax(-1, keepdim=True).clamp_(min=-3e38)
    p = torch.exp(scores.sub_(top))
    total = p.sum(-1, keepdim=True)
    o = torch.matmul(p.view(B, kv, -1, s["L"]), v).view(B, heads, most, D)
    o = torch.where(total > 0, o / total, 0.0)
    return o.transpose(1, 2)[seq, place].half()


def run(s):
    if own:
        return _run_own(s)
    return {"quant": _quant, "linear": _linear, "norm": _norm, "cache": _cache, "attn": _attend}[s["kind"]](s)


# ---------------------------------------------------------------- what a pass cannot do without

def _held(n, kind):
    """Bytes of n values in blocks."""
    return n // (2 if kind == "e2m1" else 1) + n // BLOCK


def work(case):
    if case["kind"] == "quant":
        n = case["M"] * case["K"]
        return {"bytes": 4 * n + 2 * _held(n, case["type"]), "flops": 3 * n}
    if case["kind"] == "linear":
        M, N, K = case["M"], case["N"], case["K"]
        x = 2 * M * K if case["given"] == "fp16" else _held(M * K, case["type"])
        return {"bytes": x + _held(N * K, "e2m1") + M * N * (1 if case["silu"] else 2), "flops": 2 * M * N * K}
    if case["kind"] == "norm":
        M, H = case["M"], case["H"]
        return {"bytes": 2 * H + 8 * M * H + 2 * _held(M * H, case["type"]), "flops": 7 * M * H}
    heads, kv, D = case["heads"], case["kv_heads"], case["D"]
    entry = 2 * kv * _held(D, "e2m1")  # keys and values of one cached token
    if case["kind"] == "cache":
        T = case["T"]
        return {"bytes": 2 * T * (2 * heads + 2 * kv) * D + 4 * T * D + 12 * T + 2 * T * entry + 4 * T * kv * D, "flops": 6 * T * (heads + 2 * kv) * D}
    lens, news = _lengths(case)
    pairs = sum(n * l - n * (n - 1) // 2 for l, n in zip(lens, news) if l)
    return {"bytes": 4 * sum(news) * heads * D + sum(lens) * entry + 4 * sum(-(-l // case["page"]) for l in lens) + 8 * case["B"],
            "flops": 4 * D * heads * pairs}


# ---------------------------------------------------------------- 64-bit values

def _nearest64(z, kind):
    """Rows in 64 bits as their blocks hold them, found on the list of the type's values."""
    grid = {"e2m1": [0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0, 8.0],
            "e4m3": [i / 512 for i in range(8)] + [(8 + i) / 8 * 2.0 ** e for e in range(-6, 9) for i in range(8)]}[kind]
    grid = torch.tensor(grid, dtype=torch.float64, device=z.device)  # (an even place is an even code; the last one is no value of the type)
    middle = (grid[1:] + grid[:-1]) / 2
    shape, z = z.shape, z.reshape(-1, BLOCK)

    def place(a):
        below, above = torch.searchsorted(middle, a), torch.searchsorted(middle, a, right=True)
        return torch.where(below % 2 == 0, below, above)  # the two differ in the middle between two values

    most = z.abs().max(1, keepdim=True).values
    most = most.clamp(min=2.0 ** -100)
    scale = most / torch.frexp(most).mantissa * 2.0 ** -(TYPES[kind][1] + 2)  # (a power of two over itself: exact)
    for _ in range(2):
        scale = torch.where(place(most / scale) == len(grid) - 1, 2 * scale, scale)
        scale = torch.where(most / scale > grid[-1], 2 * scale, scale)
    return (torch.sign(z) * grid[place(z.abs() / scale)] * scale).view(shape)


def _held64(codes, scales):
    """What codes and scales stand for, from the bits."""
    if codes.dtype == torch.uint8:
        c = torch.empty(codes.shape[:-1] + (2 * codes.shape[-1],), dtype=torch.int64, device=codes.device)
        c[..., 0::2], c[..., 1::2] = codes % 16, codes // 16
        bits, bias, sign = 1, 1, c // 8
        c = c % 8
    else:
        c = codes.view(torch.uint8).long()
        bits, bias, sign = 3, 7, c // 128
        c = c % 128
    e, m = c // 2 ** bits, c % 2 ** bits
    powers = torch.tensor([2.0 ** i for i in range(-127, 129)], dtype=torch.float64, device=codes.device)
    y = (m + 2 ** bits * (e > 0)).double() * powers[e.clamp(min=1) - bias - bits + 127] * (1 - 2 * sign)
    return y * powers[scales.long()].repeat_interleave(BLOCK, -1)


def _exact_linear(s):
    x = _nearest64(s["x"].double(), s["type"]) if s["given"] == "fp16" else _held64(*s["x"])
    out = []
    for first in range(0, s["N"], 8192):
        y = x @ _held64(*(t[first: first + 8192] for t in s["w"])).t()
        out.append(y if not s["silu"] else y[:, 0::2] * torch.sigmoid(y[:, 0::2]) * y[:, 1::2])
    return torch.cat(out, 1)


def _exact_cache(s):
    T, heads, D = s["q"].shape
    angles = s["cos_sin"].double().index_select(0, s["positions"].long()).view(T, 1, D)
    turn = torch.complex(angles[..., : D // 2], angles[..., D // 2:])
    out = []
    for x in (s["q"], s["k"]):
        z = torch.complex(x[..., : D // 2].double(), x[..., D // 2:].double()) * turn
        out.append(torch.cat([z.real, z.imag], 2))
    return out[0], _nearest64(out[1], "e2m1"), _nearest64(s["v"].double(), "e2m1")


def _exact_attend(s):
    lens, news = _lengths(s)
    D, kv = s["D"], s["kv_heads"]
    group = s["heads"] // kv
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
    first = 0
    for b, (length, n) in enumerate(zip(lens, news)):
        if length:
            pages = s["page_table"][b, : -(-length // s["page"])].long()
            visible = torch.ones((n, length), device="cuda", dtype=torch.bool).tril(length - n)
            for h in range(kv):
                k, v = (_held64(c[pages, h], z[pages, h]).reshape(-1, D)[:length] for c, z in ((s["k_cache"], s["k_scales"]), (s["v_cache"], s["v_scales"])))
                for j in range(h * group, (h + 1) * group):
                    a = (s["q"][first: first + n, j].double() @ k.t()) / math.sqrt(D)
                    out[first: first + n, j] = torch.softmax(a.masked_fill(~visible, -math.inf), 1) @ v
        first += n
    return out


def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"] == "quant":
        return _nearest64(s["x"].double() if case["what"] == "rows" else s["x"].double().t().contiguous(), case["type"])
    if case["kind"] == "linear":
        return _exact_linear(s)
    if case["kind"] == "norm":
        r = s["x"].double() + s["residual"].double()
        v = r.half().double()
        return _nearest64(v * s["gamma"].double() / torch.sqrt(v.pow(2).sum(1, keepdim=True) / case["H"] + EPS), case["type"]), r
    return _exact_cache(s) if case["kind"] == "cache" else _exact_attend(s)
