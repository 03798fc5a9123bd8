"""The operators between the linears together with the linears, as examples/decoder_layer.py runs them: prompts in chunks, then
single tokens, every stage of every layer against its definition in 64 bits on the stage's own inputs."""
import importlib.util
import os

import pytest
import torch

import layer_ref as ref

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def ex():
    spec = importlib.util.spec_from_file_location("decoder_layer", os.path.join(ROOT, "examples", "decoder_layer.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


class Check:
    """note() of a run: compares each stage.  Tolerances: those of the operators' own tests (test_gpu_layer_ops.py) and of the
    linears (1e-3 of the sum of magnitudes and an fp16 step)."""

    def __init__(self, cache, step, cos_sin, news):
        self.cache, self.step, self.cos_sin, self.news, self.seen = cache, step, cos_sin, news, []

    def close(self, name, got, want, tol):
        err = (got.cpu().double() - want).abs()
        assert bool((err <= tol).all()), "%s: worst error / tolerance %.3f" % (name, float((err / tol).max()))
        self.seen.append(name)

    def product(self, weight, x, group=128):
        import paper_2312_03788_amd as sqp
        w = sqp.dequantize(*weight, group).cpu().double()
        x = x.cpu().double()
        return x @ w, x.abs() @ w.abs()

    def __call__(self, name, *t):
        if name == "gemm":
            want, size = self.product(t[0], t[1])
            self.close(name, t[2], want, 1e-3 * size + 2.0 ** -10 * want.abs() + 2.0 ** -24)
        elif name == "silu":
            s, size = self.product(t[0], t[1])
            g, u, dg, du = s[:, 0::2], s[:, 1::2], 1e-3 * size[:, 0::2], 1e-3 * size[:, 1::2]
            silu = g / (1 + torch.exp(-g))
            want = silu * u
            self.close(name, t[2], want, 1.1 * u.abs() * dg + silu.abs() * du + 1.1 * dg * du + 1e-6 * want.abs() + 2.0 ** -10 * want.abs() + 2.0 ** -24)
        elif name == "add_norm":
            gamma, x, residual, y, r = [a.cpu() for a in t]
            y0, r0 = ref.add_rmsnorm(x, residual, gamma, 1e-5)
            H = x.shape[1]
            self.close(name, r, r0, 2.0 ** -11 * r0.abs() + 2.0 ** -25)
            self.close(name, y, y0, (2.0 ** -11 + H * 2.0 ** -25 + 2.0 ** -22) * y0.abs() + 2.0 ** -25)
        elif name == "cache":
            q, k, v, qr, at = t
            c, pos, slots = self.cache, self.step.positions.cpu(), self.step.slots.cpu().long()
            D = q.shape[-1]
            rot = lambda x: ref.rotate(x.cpu(), self.cos_sin.cpu(), pos)
            err = lambda x: 2.0 ** -22 * (x.cpu().double().abs() + x.cpu().double().abs().roll(D // 2, -1))
            want = rot(q)
            self.close(name, qr, want, 2.0 ** -11 * want.abs() + 2.0 ** -25 + err(q))
            for x, want, e, codes, scales in ((k, rot(k), err(k), c.k[at], c.ks[at]), (v, v.cpu().double(), 0 * v.cpu().double(), c.v[at], c.vs[at])):
                raw = codes.cpu()
                got = ref.dequantised(raw.float() if scales is not None else raw, None if scales is None else scales.cpu())
                got = got[slots // c.page, :, slots % c.page]
                if scales is None:
                    tol = 2.0 ** -11 * want.abs() + 2.0 ** -25 + e
                else:  # half a step of the codes around the value, in units of the row's scale
                    kind = "int8" if codes.dtype == torch.int8 else "e4m3"
                    unit = want.abs().amax(-1, keepdim=True) / ref.QMAX[kind]
                    tol = torch.maximum(ref.code_gap(got / unit, kind), ref.code_gap(want / unit, kind)) * unit / 2 + 2.0 ** -20 * want.abs() + e
                self.close(name, got, want, tol)
        elif name == "attention":
            qr, out, at = t
            s = ref.Step.__new__(ref.Step)
            c = self.cache
            s.lens, s.news, s.page = list(c.lens), self.news, c.page
            s.heads, s.kv_heads, s.D = qr.shape[1], c.k[at].shape[1], qr.shape[2]
            s.q, s.table = qr.cpu(), self.step.table.cpu()
            s.starts = torch.tensor([sum(self.news[:b]) for b in range(len(self.news) + 1)])
            cpu = lambda x: None if x is None else x.cpu()
            s.k, s.v, s.ks, s.vs = cpu(c.k[at]), cpu(c.v[at]), cpu(c.ks[at]), cpu(c.vs[at])
            want, tol = s.expected()
            self.close(name, out, want, tol)
        else:
            self.seen.append(name)


@pytest.mark.parametrize("kind", ["fp16", "int8", "e4m3"])
def test_prompts_and_tokens_through_two_layers(ex, kind):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(3)
    hidden, heads, kv, D = 512, 8, 2, 64
    layers = [ex.Layer(hidden, heads, kv, D, 1024, 128, gen) for _ in range(2)]
    cache = ex.PagedCache(2, 24, kv, 16, D, ex.CACHE_TYPES[kind], 3, 96)
    cos_sin = ex.rotary_table(96, D)
    for news in ([37, 5, 40], [3, 0, 24], [1, 1, 1], [1, 1, 1]):
        print("case decoder", kind, news, flush=True)
        x = torch.randn((sum(news), hidden), generator=gen, device="cuda").half()
        step = ex.Step(cache, news)
        check = Check(cache, step, cos_sin, news)
        out = ex.run(layers, x, cache, step, cos_sin, check)
        assert bool(out.isfinite().all()) and out.shape == (sum(news), hidden)
        assert set(check.seen) == {"norm", "add_norm", "gemm", "cache", "attention", "silu"}


@pytest.mark.parametrize("kind", ["fp16", "int8", "e4m3"])
def test_a_prompt_in_chunks_is_the_prompt(ex, kind):
    """Tokens written in three calls leave the bits of one call in the cache, and their attention chunk by chunk is held to the same
    64-bit values as that of the whole prompt."""
    import paper_2312_03788_amd as sqp
    gen = torch.Generator(device="cuda")
    gen.manual_seed(4)
    heads, kv, D = 8, 2, 64
    qkv = torch.randn((50, (heads + 2 * kv) * D), generator=gen, device="cuda").half()
    q, k, v = [p.view(50, -1, D) for p in qkv.split([heads * D, kv * D, kv * D], 1)]
    cos_sin = ex.rotary_table(96, D)
    kept = []
    for chunks in ([50], [20, 1, 29]):
        cache, at, rotated = ex.PagedCache(1, 4, kv, 16, D, ex.CACHE_TYPES[kind], 1, 64), 0, []
        c, scales = (cache.k[0], cache.v[0]), (cache.ks[0], cache.vs[0])
        for n in chunks:
            step = ex.Step(cache, [n])
            part = slice(at, at + n)
            qr = sqp.kv_cache_write(k[part], v[part], step.slots, *c, *scales, q=q[part], cos_sin=cos_sin, positions=step.positions)
            out = sqp.paged_attention(qr, *c, step.table, step.lens, step.starts, *scales, max_q=n, max_len=64)
            Check(cache, step, cos_sin, [n])("attention", qr, out, 0)
            rotated.append(qr)
            at += n
        kept.append([torch.cat(rotated)] + [t.view(torch.uint8) for t in c] + [t for t in scales if t is not None])
    assert all(torch.equal(a, b) for a, b in zip(*kept))
