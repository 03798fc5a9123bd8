"""The operators on microscaled numbers together, as examples/decoder_layer.py runs them (its layers with such linears and an e2m1 cache,
and each of the two alone), every stage against its definition in 64 bits on the stage's own inputs; whole steps in graphs; calls on two streams; the
largest sizes, and caches beyond 2^32 bytes."""
import pytest
import torch

import layer_ref as ref
import mx_ref as mx
from test_gpu_decoder_layer import Check, ex  # noqa: F401  (a fixture)

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def sqp():
    import paper_2312_03788_amd as m
    m.lib()
    return m


def _kind(codes):
    return "e2m1" if codes.dtype == torch.uint8 else "e4m3"


def _same(got, scales, want, kind):
    codes, bytes_ = mx.quantise(want, kind)
    assert torch.equal(mx.raw(got), mx.pack(codes, kind)) and torch.equal(scales.cpu(), bytes_)


class MxCheck(Check):
    """The stages on blocks: codes and scales are those of the definition bit for bit, products within the tolerance of mx_ref."""

    def __call__(self, name, *t):
        c = self.cache
        if name in ("mx_gemm", "mx_silu"):
            w, ws, x, xs, y = t
            want, tol = mx.product(mx.raw(x), xs.cpu(), _kind(x), mx.raw(w), ws.cpu(), name == "mx_silu")
            self.close(name, y, want, tol)
        elif name == "blocks":
            x, codes, scales = t
            _same(codes, scales, x.cpu().double(), _kind(codes))
            self.seen.append(name)
        elif name == "add_norm_mx":
            gamma, x, residual, codes, scales, r = t
            y0, r0 = ref.add_rmsnorm(x.cpu(), residual.cpu(), gamma.cpu(), 1e-5)
            self.close(name, r, r0, 2.0 ** -11 * r0.abs() + 2.0 ** -25)
            _same(codes, scales, y0, _kind(codes))
        elif name == "cache" and c.k[0].dtype == torch.uint8:
            q, k, v, qr, at = [a.cpu() if isinstance(a, torch.Tensor) else a for a in t]
            pos, slots, D = self.step.positions.cpu().long(), self.step.slots.cpu().long(), q.shape[-1]
            cs = self.cos_sin.cpu()[pos][:, None]
            a, b = k.float().chunk(2, -1)
            turned = torch.cat([a * cs[..., : D // 2] - b * cs[..., D // 2:], b * cs[..., : D // 2] + a * cs[..., D // 2:]], -1)
            want = ref.rotate(q, self.cos_sin.cpu(), self.step.positions.cpu())
            self.close(name, qr, want, 2.0 ** -11 * want.abs() + 2.0 ** -25 + 2.0 ** -22 * (q.double().abs() + q.double().abs().roll(D // 2, -1)))
            rows = lambda x: x.cpu()[slots // c.page, :, slots % c.page].flatten(0, 1)
            for want, codes, scales in ((turned, c.k[at], c.ks[at]), (v, c.v[at], c.vs[at])):
                _same(rows(codes), rows(scales), want.flatten(0, 1).double(), "e2m1")
        elif name == "attention" and c.k[0].dtype == torch.uint8:
            qr, out, at = t
            s = mx.Step.__new__(mx.Step)
            s.lens, s.news, s.page = list(c.lens), self.news, c.page
            s.heads, s.kv_heads, s.D = qr.shape[1], c.k[at].shape[1], qr.shape[2]
            s.q, s.table = qr.cpu(), self.step.table.cpu()
            s.starts = torch.tensor([sum(self.news[:b]) for b in range(len(self.news) + 1)])
            s.k, s.v, s.ks, s.vs = c.k[at].cpu(), c.v[at].cpu(), c.ks[at].cpu(), c.vs[at].cpu()
            want, tol = s.expected()
            self.close(name, out, want, tol)
        else:
            super().__call__(name, *t)


def _layers(ex, linears, gen, n=2, hidden=512, heads=8, kv=2, D=64, intermediate=1024):
    if linears == "w4a16":
        return [ex.Layer(hidden, heads, kv, D, intermediate, 128, gen) for _ in range(n)]
    return [ex.MxLayer(hidden, heads, kv, D, intermediate, ex.BLOCK_TYPES[linears], gen) for _ in range(n)]


@pytest.mark.parametrize("linears,cached", [("e2m1", "e2m1"), ("e4m3", "e2m1"), ("e4m3", "e4m3"), ("w4a16", "e2m1")])
def test_prompts_and_tokens_through_two_layers(ex, linears, cached):  # noqa: F811
    gen = torch.Generator(device="cuda")
    gen.manual_seed(5)
    hidden, kv, D = 512, 2, 64
    layers = _layers(ex, linears, gen)
    cache = ex.PagedCache(2, 24, kv, 16, D, ex.CACHE_TYPES[cached], 3, 96)
    cos_sin = ex.rotary_table(96, D)
    for news in ([37, 5, 40], [3, 0, 24], [1, 1, 1], [1, 1, 1]):
        print("case blocks", linears, cached, news, flush=True)
        x = torch.randn((sum(news), hidden), generator=gen, device="cuda").half()
        step = ex.Step(cache, news)
        check = MxCheck(cache, step, cos_sin, news)
        out = ex.run(layers, x, cache, step, cos_sin, check)
        assert bool(out.isfinite().all()) and out.shape == (sum(news), hidden)
        stages = {"norm", "add_norm", "gemm", "cache", "attention", "silu"}
        assert set(check.seen) == (stages if linears == "w4a16" else {"norm", "blocks", "add_norm_mx", "mx_gemm", "mx_silu", "cache", "attention"})


def test_a_prompt_in_chunks_is_the_prompt(ex, sqp):  # noqa: F811
    """Tokens written in three calls leave the bits of one call in the cache, and their attention chunk by chunk is held to the same
    64-bit values as that of the whole prompt."""
    gen = torch.Generator(device="cuda")
    gen.manual_seed(6)
    heads, kv, D = 8, 2, 128
    qkv = torch.randn((50, (heads + 2 * kv) * D), generator=gen, device="cuda").half()
    q, k, v = [p.view(50, -1, D) for p in qkv.split([heads * D, kv * D, kv * D], 1)]
    cos_sin = ex.rotary_table(96, D)
    kept = []
    for chunks in ([50], [20, 1, 29]):
        cache, at, rotated = ex.PagedCache(1, 4, kv, 16, D, ex.CACHE_TYPES["e2m1"], 1, 64), 0, []
        c, scales = (cache.k[0], cache.v[0]), (cache.ks[0], cache.vs[0])
        for n in chunks:
            step = ex.Step(cache, [n])
            part = slice(at, at + n)
            qr = sqp.kv_cache_write(k[part], v[part], step.slots, *c, *scales, q=q[part], cos_sin=cos_sin, positions=step.positions)
            out = sqp.paged_attention(qr, *c, step.table, step.lens, step.starts, *scales, max_q=n, max_len=64)
            MxCheck(cache, step, cos_sin, [n])("attention", qr, out, 0)
            rotated.append(qr)
            at += n
        kept.append([torch.cat(rotated), *c, *scales])
    assert all(torch.equal(a, b) for a, b in zip(*kept))


@pytest.mark.parametrize("activations", ["e2m1", "e4m3"])
def test_steps_in_two_graphs(ex, sqp, activations):  # noqa: F811
    """Two graphs, each of a whole step (a decode step, and a chunk whose products split K over workgroups), replayed in turn with
    eager work between: every replay gives the bits of the eager step."""
    gen = torch.Generator(device="cuda")
    gen.manual_seed(7)
    hidden, kv, D = 512, 2, 64
    layers = _layers(ex, activations, gen, intermediate=8192)
    assert sqp.lib().sqp_mx_gemm_scratch_bytes(120, hidden, 8192, 4 if activations == "e2m1" else 2) > 0
    cos_sin = ex.rotary_table(300, D)
    runs = []
    for news in ([1, 1, 1], [50, 40, 30]):
        cache = ex.PagedCache(2, 60, kv, 16, D, torch.uint8, 3, 300)
        first = ex.Step(cache, [200, 130, 17])
        ex.run(layers, torch.randn((347, hidden), generator=gen, device="cuda").half(), cache, first, cos_sin)
        x, step = torch.zeros((sum(news), hidden), dtype=torch.float16, device="cuda"), ex.Step(cache, news)
        ex.run(layers, x, cache, step, cos_sin)  # (everything is set up before the capture)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            out = ex.run(layers, x, cache, step, cos_sin)
        runs.append((x, cache, step, graph, out))
    for turn in range(4):
        want = []
        for x, cache, step, graph, out in runs:
            x.copy_(torch.randn(x.shape, generator=gen, device="cuda"))
            want.append(ex.run(layers, x, cache, step, cos_sin))
        for x, cache, step, graph, out in runs:
            out.zero_()
            graph.replay()
        torch.cuda.synchronize()
        for w, (x, cache, step, graph, out) in zip(want, runs):
            assert torch.equal(w, out), (turn, activations)


@pytest.mark.parametrize("kind", ["e2m1", "e4m3"])
def test_products_on_two_streams(sqp, kind):
    """Calls that split K, on two streams at once (each has scratch of its own): the bits of calls one after the other."""
    M, N, K = 120, 512, 8192
    assert sqp.lib().sqp_mx_gemm_scratch_bytes(M, N, K, 4 if kind == "e2m1" else 2) > 0
    g = ref.gen(8)
    data = [(*sqp.mx_quantize(mx.random_rows(g, M, K, 2).cuda(), mx.DTYPES[kind]), *sqp.mx_quantize(mx.random_rows(g, N, K, 2).cuda())) for _ in range(2)]
    want = [sqp.mx_gemm(*d) for d in data]
    torch.cuda.synchronize()
    streams, got = [torch.cuda.Stream() for _ in data], [[], []]
    for _ in range(8):
        for s, d, o in zip(streams, data, got):
            with torch.cuda.stream(s):
                o.append(sqp.mx_gemm(*d))
    torch.cuda.synchronize()
    assert all(torch.equal(y, w) for w, o in zip(want, got) for y in o)


def _random_codes(R, K, kind, gen):
    codes = torch.randint(0, 256, (R, K // 2 if kind == "e2m1" else K), generator=gen, device="cuda", dtype=torch.uint8)
    if kind == "e4m3":
        codes &= 0xf7  # (0x7f and 0xff are NaN)
    scales = torch.randint(120, 131, (R, K // 32), generator=gen, device="cuda", dtype=torch.uint8)
    return (codes if kind == "e2m1" else codes.view(torch.float8_e4m3fn)), scales


@pytest.mark.parametrize("M,N,K,kind", [(262000, 8184, 64, "e2m1"), (262000, 24, 8192, "e4m3"), (262000, 16, 8160, "e4m3"), (262000, 8, 8192, "e2m1"),
                                        (16, 262000, 8192, "e2m1"), (40, 262000, 8192, "e4m3"), (300, 262000, 8192, "e2m1"), (1, 8, 1 << 20, "e2m1"), (1, 8, 1 << 17, "e4m3")])
def test_largest_products(sqp, M, N, K, kind):
    """Near 2^31 elements in one of the operands or in the product: the first, the last and some other rows and columns."""
    print("case largest product", M, N, K, kind, flush=True)
    gen = torch.Generator(device="cuda")
    gen.manual_seed(M + N)
    x, xs = _random_codes(M, K, kind, gen)
    w, ws = _random_codes(N, K, "e2m1", gen)
    ws -= 8
    y = sqp.mx_gemm(x, xs, w, ws)
    some = lambda n: torch.tensor(sorted({i for i in (0, 1, n // 3, n // 2, n - 9, n - 2, n - 1) if 0 <= i < n}), device="cuda")
    m, n = some(M), some(N)
    want, tol = mx.product(x.view(torch.uint8)[m].cpu(), xs[m].cpu(), kind, w[n].cpu(), ws[n].cpu())
    # (results beyond fp16 are infinite; one within the tolerance of the border may be either)
    err = (y[m][:, n].cpu().double().clamp(-65504, 65504) - want.clamp(-65504, 65504)).abs()
    assert bool((err <= tol).all()), float((err / tol).max())


@pytest.mark.parametrize("kind", ["e2m1", "e4m3"])
def test_largest_rows(sqp, kind):
    """Near 2^31 values: into blocks and back, and the norm."""
    R, K = 262000, 8192
    gen = torch.Generator(device="cuda")
    gen.manual_seed(9)
    x = torch.randn((R, K), generator=gen, device="cuda", dtype=torch.float16)
    rows = torch.tensor([0, R // 2, R - 2, R - 1], device="cuda")
    codes, scales = sqp.mx_quantize(x, mx.DTYPES[kind])
    _same(codes.view(torch.uint8)[rows], scales[rows], x[rows].cpu().double(), kind)
    want = mx.values(codes.view(torch.uint8)[rows].cpu(), scales[rows].cpu(), kind).half()
    back = sqp.mx_dequantize(codes, scales)
    assert torch.equal(back[rows].cpu(), want)
    del codes, scales
    gamma = torch.ones(K, dtype=torch.float16, device="cuda")
    before = x[rows].cpu(), back[rows].cpu()
    codes, scales, r = sqp.add_rmsnorm_mx(x, back, gamma, 1e-5, mx.DTYPES[kind], sum_out=back)
    y0, r0 = ref.add_rmsnorm(*before, gamma.cpu(), 1e-5)
    assert bool(((r[rows].cpu().double() - r0).abs() <= 2.0 ** -11 * r0.abs() + 2.0 ** -25).all())
    _same(codes.view(torch.uint8)[rows], scales[rows], y0, kind)


@pytest.mark.parametrize("kind", ["e2m1", "e4m3"])
def test_most_rows(sqp, kind):
    """More short rows than one launch has threads for."""
    M, H = (1 << 24) + 37, 32
    gen = torch.Generator(device="cuda")
    gen.manual_seed(13)
    x, res = [torch.randn((M, H), generator=gen, device="cuda", dtype=torch.float16) for _ in range(2)]
    gamma = torch.randn(H, generator=gen, device="cuda", dtype=torch.float16)
    codes, scales, r = sqp.add_rmsnorm_mx(x, res, gamma, 1e-5, mx.DTYPES[kind])
    rows = torch.tensor([0, 1, (1 << 21) - 1, 1 << 21, (1 << 23) + 5, (1 << 24) - 1, 1 << 24, M - 1], device="cuda")
    y0, r0 = ref.add_rmsnorm(x[rows].cpu(), res[rows].cpu(), gamma.cpu(), 1e-5)
    assert bool(((r[rows].cpu().double() - r0).abs() <= 2.0 ** -11 * r0.abs() + 2.0 ** -25).all())
    _same(codes.view(torch.uint8)[rows], scales[rows], y0, kind)
    codes, scales = sqp.mx_quantize(x, mx.DTYPES[kind])
    _same(codes.view(torch.uint8)[rows], scales[rows], x[rows].cpu().double(), kind)
    y = sqp.mx_gemm(codes, scales, *sqp.mx_quantize(x[:8]))
    want, tol = mx.product(codes.view(torch.uint8)[rows].cpu(), scales[rows].cpu(), kind, *[t.cpu() for t in sqp.mx_quantize(x[:8])])
    assert bool(((y[rows].cpu().double() - want).abs() <= tol).all())


def test_largest_weight(sqp):
    K, N = 8192, 262000
    gen = torch.Generator(device="cuda")
    gen.manual_seed(10)
    w = torch.randn((K, N), generator=gen, device="cuda", dtype=torch.float16)
    codes, scales = sqp.mx_quantize_weight(w)
    cols = torch.tensor([0, 1, N // 2, N - 130, N - 1], device="cuda")
    _same(codes[cols], scales[cols], w[:, cols].cpu().double().t().contiguous(), "e2m1")


@pytest.mark.parametrize("new", [1, 40])
def test_cache_beyond_32_bits(sqp, new):
    """A cache whose codes take more than 2^32 bytes: its last pages are written, read and attended."""
    heads, kv, D, page, n = 8, 8, 128, 16, 100
    pages = (1 << 32) // (kv * page * D // 2) + 500
    g = ref.gen(11)
    qkv = mx.random_rows(g, n, (heads + 2 * kv) * D, 1).cuda()
    q, k, v = [t.view(n, -1, D) for t in qkv.split([heads * D, kv * D, kv * D], 1)]
    c = [torch.empty((pages, kv, page, e), dtype=torch.uint8, device="cuda") for e in (D // 2, D // 2, D // 32, D // 32)]
    small = [torch.empty((7, kv, page, e), dtype=torch.uint8, device="cuda") for e in (D // 2, D // 2, D // 32, D // 32)]
    table = torch.arange(pages - 7, pages, dtype=torch.int32, device="cuda")[None]
    at = torch.arange(n, dtype=torch.int32, device="cuda")
    lens, starts = torch.tensor([n], dtype=torch.int32, device="cuda"), torch.tensor([0, new], dtype=torch.int32, device="cuda")
    sqp.kv_cache_write(k, v, at + (pages - 7) * page, *c)
    sqp.kv_cache_write(k, v, at, *small)
    for a, b in zip(sqp.kv_cache_read(at + (pages - 7) * page, *c), sqp.kv_cache_read(at, *small)):
        assert torch.equal(a, b) and bool(a.any())
    far = sqp.paged_attention(q[-new:].contiguous(), c[0], c[1], table, lens, starts, c[2], c[3], max_q=new, max_len=n)
    near = sqp.paged_attention(q[-new:].contiguous(), small[0], small[1], table - (pages - 7), lens, starts, small[2], small[3], max_q=new, max_len=n)
    assert torch.equal(far, near) and bool(far.any())


@pytest.mark.parametrize("lens,news", [([3, 40, 0], [5, 2, 2]), ([17, 0, 90], [40, 3, 33])])
def test_rows_that_see_nothing_and_rows_of_no_sequence(sqp, lens, news):
    """More new tokens than the length has: those in front see nothing and are zeros, as rows of no sequence are."""
    s = mx.Step(lens, news, 8, 2, 128, 16, seed=12)
    T = sum(news)
    g = s.gpu()
    g["q"] = torch.cat([g["q"], torch.ones_like(g["q"][:3])])
    out = torch.full(g["q"].shape, 7.0, dtype=torch.float16, device="cuda")
    sqp.paged_attention(**g, max_q=max(news), max_len=max(lens), out=out)
    assert not bool(out[T:].any())
    want, tol = s.expected()
    assert bool(((out[:T].cpu().double() - want).abs() <= tol).all())
    blind = torch.cat([torch.arange(n) < n - length for length, n in zip(lens, news)])
    assert bool(blind.any()) and not bool(out[:T].cpu()[blind].any())


def test_pages_that_no_cache_has(sqp):
    """Page numbers outside the cache, lengths beyond the table and starts outside the batch give some values, and no access outside."""
    heads, kv, D, page = 8, 2, 128, 16
    c = [torch.zeros((4, kv, page, e), dtype=torch.uint8, device="cuda") for e in (D // 2, D // 2, D // 32, D // 32)]
    i = lambda *x: torch.tensor(x, dtype=torch.int32, device="cuda")
    for new in (1, 30):
        q = torch.randn((2 * new, heads, D), device="cuda").half()
        for table in (i(-1, 1 << 30, 4, 3).repeat(2, 1), i(0, 1, 2, 3).repeat(2, 1)):
            for lens in (i(64, 60), i(1 << 30, -5)):
                for starts in (i(0, new, 2 * new), i(-7, new, 1 << 30)):
                    print("case no such page", new, lens.tolist(), starts.tolist(), flush=True)
                    o = sqp.paged_attention(q, c[0], c[1], table, lens, starts, c[2], c[3], max_q=new, max_len=64)
                    assert o.shape == q.shape
                    torch.cuda.synchronize()
