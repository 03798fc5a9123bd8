"""GPU parity of the operators on microscaled numbers (blocks of 32, a power-of-two scale each): quantisation bit for bit, the product,
the norm with its output in blocks, the paged cache of blocks and the attention over it, each against its definition in 64 bits."""
import ctypes

import pytest
import torch

import layer_ref as ref
import mx_ref as mx

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def sqp():
    import paper_2312_03788_amd as m
    m.lib()
    return m


@pytest.fixture
def plan(sqp):
    """Sets the product's plan, automatic again afterwards."""
    f = sqp.lib().sqp_debug_set_mx_plan
    yield f
    f(0, 0, 0, 0)


# ---------------------------------------------------------------- rows and weights into blocks

def _edges(kind):
    """Blocks with every border between codes, both sides of it, at several scales; maxima around every change of the scale; zeros,
    fp16's smallest and largest numbers, infinities and NaN."""
    rows = []
    g = mx.grid(kind)
    middle = ((g[1:] + g[:-1]) / 2)
    pick = middle if kind == "e2m1" else middle[::5]
    for e in (-12, -3, 0, 4):
        for top in (GRID_TOP[kind], GRID_TOP[kind] / 2):
            for m in pick:
                for step in (0, 1, -1):
                    h = (m * 2.0 ** e).half()
                    v = (h.view(torch.int16) + step).view(torch.float16).float()
                    rows.append([top * 2.0 ** e, float(v), -float(v)] + [0.0] * 29)
    for e in (-14, 0, 6):
        for m in (1.0, 1.5, 1.7490234375, 1.75, 1.7509765625, 1.8115234375, 1.8125, 1.8134765625, 1.9990234375):
            rows.append([-m * 2.0 ** e, 0.3 * 2.0 ** e, -0.0] + [0.01 * 2.0 ** e] * 29)
    rows.append([0.0] * 16 + [-0.0] * 16)
    rows.append([2.0 ** -24, -2.0 ** -24] + [0.0] * 30)
    rows.append([65504.0, -65504.0, 1.0] + [60000.0] * 29)
    rows.append([float("inf")] + [1.0] * 31)
    rows.append([1.0] * 31 + [float("nan")])
    rows.append([float("-inf"), float("nan")] + [0.0] * 30)
    return torch.tensor(rows, dtype=torch.float64).half()


GRID_TOP = {"e2m1": 6.0, "e4m3": 448.0}


def _check_quantised(codes, scales, x, kind):
    c0, s0 = mx.quantise(x.double(), kind)
    assert torch.equal(scales.cpu(), s0)
    assert torch.equal(mx.raw(codes), mx.pack(c0, kind))


@pytest.mark.parametrize("kind", ["e2m1", "e4m3"])
def test_quantise_edges(sqp, kind):
    x = _edges(kind)
    codes, scales = sqp.mx_quantize(x.cuda(), mx.DTYPES[kind])
    _check_quantised(codes, scales, x, kind)


@pytest.mark.parametrize("kind", ["e2m1", "e4m3"])
@pytest.mark.parametrize("R,K", [(1, 32), (1, 4096), (3, 96), (17, 4128), (333, 1024), (1001, 5120)])
def test_quantise_and_back(sqp, R, K, kind):
    print("case quantise", R, K, kind, flush=True)
    x = mx.random_rows(ref.gen(R + K), R, K)
    codes, scales = sqp.mx_quantize(x.cuda(), mx.DTYPES[kind])
    assert codes.dtype == mx.DTYPES[kind] and tuple(codes.shape) == (R, K // 2 if kind == "e2m1" else K) and tuple(scales.shape) == (R, K // 32)
    _check_quantised(codes, scales, x, kind)
    back = sqp.mx_dequantize(codes, scales)
    want = mx.values(mx.raw(codes), scales.cpu(), kind)
    assert back.dtype == torch.float16 and torch.equal(back.cpu(), want.half())
    # into given tensors
    c2, s2 = torch.empty_like(codes), torch.empty_like(scales)
    o = sqp.mx_quantize(x.cuda(), mx.DTYPES[kind], out=(c2, s2))
    assert o[0] is c2 and o[1] is s2 and torch.equal(mx.raw(c2), mx.raw(codes)) and torch.equal(s2, scales)
    b2 = torch.empty_like(back)
    assert sqp.mx_dequantize(codes, scales, out=b2) is b2 and torch.equal(b2, back)


@pytest.mark.parametrize("kind", ["e2m1", "e4m3"])
def test_dequantise_any_bits(sqp, kind):
    """Every code under every scale byte, as another program may have written them."""
    n = 16 if kind == "e2m1" else 256
    codes = torch.arange(n).repeat(32 * 8 // n if kind == "e2m1" else 1).to(torch.uint8)
    if kind == "e4m3":
        codes[127], codes[255] = 0, 128  # (the type's two NaN)
    codes = codes.reshape(1, 256).repeat(256, 1)
    packed = mx.pack(codes, kind)
    scales = torch.arange(256).to(torch.uint8)[:, None].repeat(1, 8)
    back = sqp.mx_dequantize(mx.typed(packed, kind).cuda(), scales.cuda()).cpu()
    want = mx.values(packed, scales, kind).half()
    assert torch.equal(back.isnan(), want.isnan())
    assert torch.equal(back[:255], want[:255])


@pytest.mark.parametrize("K,N", [(32, 8), (96, 24), (256, 64), (288, 72), (4096, 136), (512, 1000)])
def test_quantise_weight(sqp, K, N):
    print("case weight", K, N, flush=True)
    w = mx.random_rows(ref.gen(N + K), N, K).t().contiguous()
    codes, scales = sqp.mx_quantize_weight(w.cuda())
    assert tuple(codes.shape) == (N, K // 2) and tuple(scales.shape) == (N, K // 32)
    _check_quantised(codes, scales, w.t().contiguous(), "e2m1")
    o = sqp.mx_quantize_weight(w.cuda(), out=(torch.empty_like(codes), torch.empty_like(scales)))
    assert torch.equal(o[0], codes) and torch.equal(o[1], scales)


def test_quantise_weight_edges(sqp):
    x = _edges("e2m1")
    x = x[: x.shape[0] // 8 * 8] if x.shape[0] % 8 else x
    bad = torch.zeros((8, 32), dtype=torch.float16)
    bad[1, 3], bad[2, 31], bad[5, 0] = float("inf"), float("nan"), 65504.0
    x = torch.cat([x, bad])
    codes, scales = sqp.mx_quantize_weight(x.t().contiguous().cuda())
    _check_quantised(codes, scales, x, "e2m1")


# ---------------------------------------------------------------- product

def _operands(M, N, K, kind, seed=3):
    g = ref.gen(seed)
    cx, sx = mx.quantise(mx.random_rows(g, M, K, 2).double(), kind)
    cw, sw = mx.quantise(mx.random_rows(g, N, K, 2).double() / K ** 0.5, "e2m1")
    return mx.pack(cx, kind), sx, mx.pack(cw, "e2m1"), sw


def _on_gpu(x, xs, w, ws, kind):
    return mx.typed(x, kind).cuda(), xs.cuda(), w.contiguous().cuda(), ws.cuda()


def _check_product(y, x, xs, w, ws, kind, silu):
    y0, tol = mx.product(x, xs, kind, w, ws, silu)
    err = (y.cpu().double() - y0).abs()
    assert bool((err <= tol).all()), float((err / tol).max())
    return float((err / tol).max())


SIZES = [  # M, N, K
    (1, 8, 32), (1, 64, 512), (2, 24, 544), (16, 48, 1056), (17, 40, 96), (33, 136, 2048), (64, 72, 4128), (65, 264, 800), (130, 520, 1312), (300, 144, 736)]


@pytest.mark.parametrize("silu", [False, True])
@pytest.mark.parametrize("kind", ["e2m1", "e4m3"])
@pytest.mark.parametrize("M,N,K", SIZES)
def test_product(sqp, M, N, K, kind, silu):
    if silu and N % 16:
        N += 8
    print("case product", M, N, K, kind, silu, flush=True)
    ops = _operands(M, N, K, kind)
    f = sqp.mx_gemm_silu_mul if silu else sqp.mx_gemm
    dev = _on_gpu(*ops, kind)
    y = f(*dev)
    assert y.dtype == torch.float16 and tuple(y.shape) == (M, N // 2 if silu else N)
    print("worst", _check_product(y, *ops, kind, silu), flush=True)
    out = torch.empty_like(y)
    assert f(*dev, out=out) is out and torch.equal(out, y)


FEW = [(1, 1, 8), (1, 2, 8), (2, 1, 8), (2, 2, 4), (4, 1, 8)]


@pytest.mark.parametrize("kind", ["e2m1", "e4m3"])
@pytest.mark.parametrize("M,N,K", [(5, 88, 1568), (70, 40, 9248)])
def test_product_few_rows_plans(sqp, plan, M, N, K, kind):
    """Every built form of the few-rows kernel, rows and columns past the last whole tile, a last round that is not whole."""
    ops = _operands(M, N, K, kind, 5)
    dev = _on_gpu(*ops, kind)
    for mt, nt, kw in FEW:
        print("case few", M, N, K, kind, mt, nt, kw, flush=True)
        plan(1, mt, nt, kw)
        _check_product(sqp.mx_gemm(*dev), *ops, kind, False)


TILES = {t: t not in (7, 8, 9) for t in range(10)}  # whether it is for K of whole 128 alone, 512 at least


@pytest.mark.parametrize("kind", ["e2m1", "e4m3"])
@pytest.mark.parametrize("M,N,K", [(40, 72, 32), (70, 136, 256), (300, 336, 1568), (270, 272, 4224), (20, 272, 512), (140, 528, 1920)])
def test_product_tile_plans(sqp, plan, M, N, K, kind):
    """Every tile, whole and in K parts, the parts' borders inside a chunk of 16 scales too."""
    ops = _operands(M, N, K, kind, 6)
    dev = _on_gpu(*ops, kind)
    for tile, direct in TILES.items():
        if direct and (K % 128 or K < 512):
            plan(2, tile, 1, 0)
            with pytest.raises(sqp.SqpError):
                sqp.mx_gemm(*dev)
            continue
        for parts in (1, 2, 3, 5):
            print("case tiles", M, N, K, kind, tile, parts, flush=True)
            plan(2, tile, parts, 0)
            y = sqp.mx_gemm(*dev)
            _check_product(y, *ops, kind, False)
            if parts in (1, 3):
                _check_product(sqp.mx_gemm_silu_mul(*dev), *ops, kind, True) if N % 16 == 0 else None
            assert torch.equal(sqp.mx_gemm(*dev), y)


@pytest.mark.parametrize("kind", ["e2m1", "e4m3"])
@pytest.mark.parametrize("silu", [False, True])
def test_product_columns_in_two_launches(sqp, plan, kind, silu):
    """The first columns in tiles of one shape, the others in another's: every column once, the same values as in one launch."""
    M, N, K = 200, 656, 1152
    ops = _operands(M, N, K, kind, 9)
    dev = _on_gpu(*ops, kind)
    f = sqp.mx_gemm_silu_mul if silu else sqp.mx_gemm
    for first, other, cols in ((0, 1, 1), (0, 3, 2), (1, 4, 2), (2, 4, 4), (1, 2, 1), (0, 2, 5)):
        print("case two launches", kind, silu, first, other, cols, flush=True)
        plan(3, first, other, cols)
        _check_product(f(*dev), *ops, kind, silu)


@pytest.mark.parametrize("M,N,K,kind", [(1, 1024, 4096, "e2m1"), (16, 4096, 2048, "e4m3"), (40, 8192, 1024, "e2m1"), (100, 2048, 8192, "e2m1"), (260, 16640, 512, "e4m3"),
                                        (520, 10240, 512, "e2m1"), (48, 512, 8320, "e4m3"), (70, 264, 4128, "e2m1")])
def test_product_automatic_plans(sqp, M, N, K, kind):
    """What the library chooses by itself, over sizes that lead to each kernel, K parts and two launches: two rows against 64 bits, all of them
    against another plan within the tolerance of both."""
    print("case automatic", M, N, K, kind, flush=True)
    ops = _operands(M, N, K, kind, 10)
    dev = _on_gpu(*ops, kind)
    y = sqp.mx_gemm(*dev)
    rows = sorted({0, M // 2, M - 1})
    _check_product(y[rows], ops[0][rows], ops[1][rows], ops[2], ops[3], kind, False)
    assert torch.equal(sqp.mx_gemm(*dev), y)


@pytest.mark.parametrize("kind", ["e2m1", "e4m3"])
@pytest.mark.parametrize("M", [3, 200])
def test_product_rows_that_are_nan(sqp, M, kind):
    """A block that is NaN makes NaN of its row or column and leaves the others; memory behind the operands does not matter."""
    N, K = 136, 1312
    x, xs, w, ws = _operands(M, N, K, kind, 7)
    xs[1, 40], ws[5, 3], ws[N - 1, 0] = 255, 255, 255
    x[2], xs[2] = 0, 0  # a row of zeros
    y = sqp.mx_gemm(*_on_gpu(x, xs, w, ws, kind)).cpu()
    assert bool(y[1].isnan().all()) and bool(y[:, 5].isnan().all()) and bool(y[:, N - 1].isnan().all())
    rows, cols = [i for i in range(M) if i != 1], [j for j in range(N) if j not in (5, N - 1)]
    y0, tol = mx.product(x[rows], xs[rows], kind, w[cols], ws[cols])
    assert bool(((y[rows][:, cols].double() - y0).abs() <= tol).all())
    assert not bool(y[2][cols].any())


def test_product_given_no_scratch(sqp, plan):
    """K parts need scratch: without it, or with too little, a plan that fits gives the same within the sums' order; under capture with
    `out` nothing is allocated."""
    M, N, K = 200, 264, 8192
    ops = _operands(M, N, K, "e2m1", 8)
    dev = _on_gpu(*ops, "e2m1")
    plan(2, 1, 4, 0)
    L, y = sqp.lib(), torch.empty((M, N), dtype=torch.float16, device="cuda")
    p = lambda t: ctypes.c_void_p(t.data_ptr())
    need = L.sqp_mx_gemm_scratch_bytes(M, N, K, 4)
    assert need == 4 * M * N * 4
    room = torch.empty(need, dtype=torch.uint8, device="cuda")
    for nbytes in (0, 100, need // 2, need - 1, need):
        y.zero_()
        rc = L.sqp_mx_gemm(M, N, K, 4, 0, p(dev[0]), p(dev[1]), p(dev[2]), p(dev[3]), p(y), p(room) if nbytes else None, nbytes,
                           ctypes.c_void_p(torch.cuda.current_stream().cuda_stream))
        assert rc == 0
        _check_product(y, *ops, "e2m1", False)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        sqp.mx_gemm(*dev, out=y)
    for _ in range(3):
        y.zero_()
        graph.replay()
        torch.cuda.synchronize()
        _check_product(y, *ops, "e2m1", False)


# ---------------------------------------------------------------- residual and norm

NORM_SIZES = [(1, 32), (1, 2048), (3, 2080), (5, 4096), (2, 4128), (33, 8192), (2, 8224), (3, 16384), (2, 16416), (2, 32768), (2, 32800), (700, 544)]


def _norm_inputs(M, H, seed):
    g = ref.gen(seed)
    gain = torch.ones(H)
    gain[torch.randperm(H, generator=g)[: max(1, H // 100)]] = 50.0
    return ref.randn(g, M, H).half(), (ref.randn(g, M, H) * gain).half(), (1 + 0.1 * ref.randn(g, H)).half()


@pytest.mark.parametrize("kind", ["e2m1", "e4m3"])
@pytest.mark.parametrize("M,H", NORM_SIZES)
def test_add_rmsnorm_mx(sqp, M, H, kind):
    """Codes and scales are those of the formula in 64 bits (whose own sums are off by 2^-50, so that a value on a border's other side
    would need to lie as near to it)."""
    print("case add_rmsnorm_mx", M, H, kind, flush=True)
    x, res, gamma = _norm_inputs(M, H, 4)
    codes, scales, r = sqp.add_rmsnorm_mx(x.cuda(), res.cuda(), gamma.cuda(), 1e-5, mx.DTYPES[kind])
    y0, r0 = ref.add_rmsnorm(x, res, gamma, 1e-5)
    assert bool(((r.cpu().double() - r0).abs() <= 2.0 ** -11 * r0.abs() + 2.0 ** -25).all())
    _check_quantised(codes, scales, y0, kind)
    # in place, and into given tensors
    rx, out = res.cuda(), (torch.empty_like(codes), torch.empty_like(scales))
    c2, s2, r2 = sqp.add_rmsnorm_mx(x.cuda(), rx, gamma.cuda(), 1e-5, mx.DTYPES[kind], out=out, sum_out=rx)
    assert c2 is out[0] and s2 is out[1] and r2 is rx
    assert torch.equal(mx.raw(c2), mx.raw(codes)) and torch.equal(s2, scales) and torch.equal(r2, r)
    xx = x.cuda()
    c3, s3, r3 = sqp.add_rmsnorm_mx(xx, res.cuda(), gamma.cuda(), 1e-5, mx.DTYPES[kind], sum_out=xx)
    assert r3 is xx and torch.equal(mx.raw(c3), mx.raw(codes)) and torch.equal(s3, scales) and torch.equal(r3, r)


@pytest.mark.parametrize("kind", ["e2m1", "e4m3"])
def test_add_rmsnorm_mx_on_the_borders(sqp, kind):
    """Rows whose norm is exactly 1 or 2 (values +-1 and +-2), so that y = gamma and gamma / 2 x 2: every border is met exactly."""
    edge = _edges(kind)
    edge = edge[edge.isfinite().all(1)]
    H = 32 * edge.shape[0]
    gamma = edge.reshape(-1)
    g = ref.gen(2)
    x = (torch.randint(0, 2, (4, H), generator=g) * 2 - 1).half()
    x[2:] *= 2
    zero = torch.zeros_like(x)
    codes, scales, _ = sqp.add_rmsnorm_mx(x.cuda(), zero.cuda(), gamma.cuda(), 0.0, mx.DTYPES[kind])
    y0, _ = ref.add_rmsnorm(x, zero, gamma, 0.0)
    assert torch.equal(y0.abs(), gamma.double().abs().expand(4, H))
    _check_quantised(codes, scales, y0, kind)


def test_add_rmsnorm_mx_rows_that_are_not_numbers(sqp):
    """Blocks that hold a value which is NaN by the formula are NaN as a whole; a row of zeros is zeros; neighbours are untouched."""
    x, res, gamma = _norm_inputs(6, 1024, 5)
    x[1, 7], x[2, 9] = float("inf"), float("nan")
    x[3], res[3] = 0, 0
    x[4] = x[4] * 1e-3
    res[4] = res[4] * 0 + 2.0 ** -24
    for kind in ("e2m1", "e4m3"):
        for eps in (1e-5, 0.0):
            codes, scales, _ = sqp.add_rmsnorm_mx(x.cuda(), res.cuda(), gamma.cuda(), eps, mx.DTYPES[kind])
            y0, _ = ref.add_rmsnorm(x, res, gamma, eps)
            _check_quantised(codes, scales, y0, kind)
            assert bool((scales[2] == 255).all()) and int((scales[1] == 255).sum()) == 1
            if eps:
                assert not bool(scales[3].any())


# ---------------------------------------------------------------- cache

CACHE_CASES = [  # tokens, heads, kv_heads, D, page
    (1, 64, 8, 128, 16), (1, 1, 1, 64, 16), (7, 32, 32, 128, 64), (37, 14, 2, 128, 32), (5, 16, 1, 64, 256), (130, 40, 40, 128, 16), (33, 15, 5, 64, 128)]


def _rotate32(x, cos_sin, positions):
    """Every product and sum in 32 bits, rounded for itself."""
    cs = cos_sin[positions.long()][:, None]
    h = x.shape[-1] // 2
    a, b, c, s = x[..., :h].float(), x[..., h:].float(), cs[..., :h], cs[..., h:]
    return torch.cat([a * c - b * s, b * c + a * s], -1)


def _rows_of(t, slots, page):
    return t[slots.long() // page, :, slots.long() % page]


@pytest.mark.parametrize("rotated", [True, False])
@pytest.mark.parametrize("T,heads,kv,D,page", CACHE_CASES)
def test_cache_write_and_read(sqp, T, heads, kv, D, page, rotated):
    """Codes and scales are those of the rotation in plain 32-bit arithmetic, bit for bit; other tokens' places keep their bits, tokens
    without a slot are not written; reading back is one rounding of code times scale."""
    print("case cache", T, heads, kv, D, page, rotated, flush=True)
    g = ref.gen(6)
    pages = -(-T // page) + 2
    qkv = mx.random_rows(g, T, (heads + 2 * kv) * D)
    slots = torch.randperm(pages * page, generator=g)[:T].int()
    if T > 4:
        slots[2], slots[4] = -1, pages * page
    positions = torch.randint(0, 5000, (T,), generator=g, dtype=torch.int32)
    table = ref.cos_sin_table(5000, D)
    k0, v0 = [torch.randint(0, 256, (pages, kv, page, D // 2), generator=g, dtype=torch.uint8) for _ in range(2)]
    ks0, vs0 = [torch.randint(100, 140, (pages, kv, page, D // 32), generator=g, dtype=torch.uint8) for _ in range(2)]
    gk, gv, gks, gvs = [t.cuda() for t in (k0, v0, ks0, vs0)]
    d = qkv.cuda()
    q, k, v = d[:, : heads * D].view(T, heads, D), d[:, heads * D: (heads + kv) * D].view(T, kv, D), d[:, (heads + kv) * D:].view(T, kv, D)
    turn = dict(cos_sin=table.cuda(), positions=positions.cuda()) if rotated else {}
    qr = sqp.kv_cache_write(k, v, slots.cuda(), gk, gv, gks, gvs, q=q, **turn)
    hk, hv, hq = k.cpu(), v.cpu(), q.cpu()
    if rotated:
        want_k, want_q = _rotate32(hk, table, positions), _rotate32(hq, table, positions)
    else:
        want_k, want_q = hk.float(), hq.float()
    assert torch.equal(qr.cpu(), want_q.half())
    ok = (slots >= 0) & (slots < pages * page)
    for x, got, scales, before, scales_before in ((want_k, gk, gks, k0, ks0), (hv.float(), gv, gvs, v0, vs0)):
        codes, bytes_ = mx.quantise(x[ok].reshape(-1, D).double(), "e2m1")
        n = int(ok.sum())
        before[slots[ok].long() // page, :, slots[ok].long() % page] = mx.pack(codes, "e2m1").reshape(n, kv, D // 2)
        scales_before[slots[ok].long() // page, :, slots[ok].long() % page] = bytes_.reshape(n, kv, D // 32)
        assert torch.equal(got.cpu(), before) and torch.equal(scales.cpu(), scales_before)
    rk, rv = sqp.kv_cache_read(slots.cuda(), gk, gv, gks, gvs)
    for got, c, s in ((rk, k0, ks0), (rv, v0, vs0)):
        want = torch.zeros((T, kv, D), dtype=torch.float16)
        want[ok] = mx.values(_rows_of(c, slots[ok], page), _rows_of(s, slots[ok], page), "e2m1").half()
        assert torch.equal(got.cpu(), want)


def test_cache_positions_outside_the_table(sqp):
    """Such a token's keys and queries are NaN: its blocks have the scale 255, its values are kept."""
    T, kv, D, page = 3, 2, 64, 16
    g = ref.gen(8)
    qkv = ref.randn(g, T, 3 * kv, D).half().cuda()
    c = [torch.zeros((1, kv, page, n), dtype=torch.uint8, device="cuda") for n in (D // 2, D // 2, D // 32, D // 32)]
    slots, positions = torch.arange(T).int().cuda(), torch.tensor([0, 7, -1], dtype=torch.int32).cuda()
    q = sqp.kv_cache_write(qkv[:, kv: 2 * kv], qkv[:, 2 * kv:], slots, *c, q=qkv[:, :kv], cos_sin=ref.cos_sin_table(7, D).cuda(), positions=positions)
    assert bool(q[1:].isnan().all()) and bool(q[0].isfinite().all())
    assert bool((c[2][0, :, 1:3] == 255).all()) and not bool((c[2][0, :, 0] == 255).any()) and not bool((c[3] == 255).any())


# ---------------------------------------------------------------- attention

def _attend(sqp, s, **kw):
    g = s.gpu()
    if all(n == 1 for n in s.news):
        g["q_starts"] = None
    return sqp.paged_attention(**g, max_q=max(s.news), max_len=max(s.lens), **kw)


ATTENTION = [  # lengths, new tokens, heads, kv_heads, D, page
    ([1], [1], 1, 1, 128, 16), ([1], [1], 4, 1, 64, 16), ([17], [1], 8, 8, 128, 16), ([64, 65, 0, 129], [1, 1, 1, 1], 14, 2, 128, 32),
    ([700, 33], [1, 1], 16, 1, 64, 16), ([2100], [1], 8, 1, 128, 64), ([40, 300], [3, 2], 8, 2, 128, 16), ([5], [5], 2, 2, 64, 16),
    ([129, 64], [100, 64], 6, 2, 128, 16), ([130, 1, 500], [97, 1, 33], 8, 1, 64, 32), ([1100], [40], 16, 2, 128, 128), ([333, 20, 257], [333, 1, 200], 4, 4, 128, 16),
    ([900], [300], 64, 8, 128, 64), ([700], [400], 32, 2, 64, 64)]


@pytest.mark.parametrize("lens,news,heads,kv,D,page", ATTENTION)
def test_attention(sqp, lens, news, heads, kv, D, page):
    print("case attention", lens, news, heads, kv, D, page, flush=True)
    s = mx.Step(lens, news, heads, kv, D, page)
    o = _attend(sqp, s).cpu().double()
    want, tol = s.expected()
    assert bool(((o - want).abs() <= tol).all()), float(((o - want).abs() / tol).max())


@pytest.mark.parametrize("heads,kv,D,new", [(8, 2, 128, 1), (8, 2, 64, 1), (8, 2, 128, 40), (8, 2, 64, 40), (64, 2, 128, 300), (64, 2, 64, 300)])
def test_attention_blocks_too_large_for_fp16(sqp, heads, kv, D, new):
    """Values and keys beyond fp16 (codes of 4 and 6 times 2^14 and more, as another program may have written them), tokens that are
    NaN: the rows that see them follow the formula, the others do not know of them."""
    L = 600
    s = mx.Step([L, 70], [new, min(new, 20)], heads, kv, D, 16, seed=3)
    t = s.table[0].long()
    at = lambda j: (t[j // 16], slice(None), j % 16)
    s.vs[at(100)] = 127 + 14          # 6 x 2^14 does not fit fp16
    s.k[at(200)] = 0x77
    s.ks[at(200)] = 127 + 14          # the largest key that fp16 pairs make
    s.k[at(201)] = 0xff
    s.ks[at(201)] = 127 + 17
    s.q = (s.q.float() * 1e-4).half()
    o = _attend(sqp, s).cpu().double()
    want, tol = s.expected()
    # the output itself may not fit fp16
    want = torch.where(want.abs() >= 65520, want.sign() * float("inf"), want)
    fine = want.isfinite()
    assert torch.equal(o.isfinite(), fine)
    assert bool(((o - want).abs() <= tol)[fine].all()), float(((o - want).abs() / tol)[fine].max())
    s.vs[at(L - 1)] = 255             # the last token: only the last row sees it (the others of its tile go another way now: to the same values)
    o2 = _attend(sqp, s).cpu().double()
    assert bool(o2[new - 1].isnan().all())
    others = torch.arange(o.shape[0]) != new - 1
    assert torch.equal(o2.isfinite()[others], fine[others])
    assert bool(((o2 - want).abs() <= tol)[others][fine[others]].all())


def test_attention_from_written_cache(sqp):
    """What write leaves is what attention reads: the output equals that over the same cache read back as fp16 (exact: no value is
    beyond fp16 or below its steps)."""
    T, heads, kv, D, page = 150, 8, 2, 128, 16
    g = ref.gen(11)
    qkv = ref.randn(g, T, heads + 2 * kv, D).half().cuda()
    pages = 12
    c = [torch.zeros((pages, kv, page, n), dtype=torch.uint8, device="cuda") for n in (D // 2, D // 2, D // 32, D // 32)]
    order = torch.randperm(pages, generator=g).int()
    slots = (order.long()[torch.arange(T) // page] * page + torch.arange(T) % page).int().cuda()
    turn = dict(cos_sin=ref.cos_sin_table(T, D).cuda(), positions=torch.arange(T).int().cuda())
    q = sqp.kv_cache_write(qkv[:, heads: heads + kv], qkv[:, heads + kv:], slots, *c, q=qkv[:, :heads], **turn)
    k, v = sqp.kv_cache_read(slots, *c)
    half = [torch.zeros((pages, kv, page, D), dtype=torch.float16, device="cuda") for _ in range(2)]
    sqp.kv_cache_write(k, v, slots, *half)
    lens, starts = torch.tensor([T], dtype=torch.int32).cuda(), torch.tensor([0, T], dtype=torch.int32).cuda()
    a = sqp.paged_attention(q, c[0], c[1], order[None].cuda(), lens, starts, c[2], c[3], max_q=T, max_len=T)
    b = sqp.paged_attention(q, *half, order[None].cuda(), lens, starts, max_q=T, max_len=T)
    assert torch.equal(a, b)
    # one token, the last.  Over blocks p is rounded to fp16 once (2^-11 of sum p |v|), over fp16 taken in two parts (2^-22 of it); both
    # outputs are rounded (half a step each), and the sum p |v| itself is an output over the values' magnitudes (half a step more).
    a1 = sqp.paged_attention(q[-1:], c[0], c[1], order[None].cuda(), lens, None, c[2], c[3], max_len=T)
    b1 = sqp.paged_attention(q[-1:], *half, order[None].cuda(), lens, max_len=T)
    size = sqp.paged_attention(q[-1:], half[0], half[1].abs(), order[None].cuda(), lens, max_len=T).double()
    assert bool(((a1.double() - b1.double()).abs() <= 2.0 ** -10 * b1.double().abs() + 1.01 * 2.0 ** -11 * size + 2.0 ** -24).all())
