"""GPU parity of the operators between the linears: residual and norm (fp16 and 8-bit output), the paged cache, the attention
over it -- each against its definition in 64 bits, at the sizes, masks and contents where it can go wrong."""
import pytest
import torch

import layer_ref as ref

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def sqp():
    import paper_2312_03788_amd as m
    m.lib()
    return m


# ---------------------------------------------------------------- residual and norm

NORM_SIZES = [(1, 8), (1, 2048), (3, 2056), (5, 4096), (2, 4104), (33, 8192), (2, 8200), (3, 16384), (2, 16392), (2, 32768), (2, 32776), (700, 520)]


def _norm_inputs(M, H, seed):
    g = ref.gen(seed)
    gain = torch.ones(H)
    gain[torch.randperm(H, generator=g)[: max(1, H // 100)]] = 50.0
    return ref.randn(g, M, H).half(), (ref.randn(g, M, H) * gain).half(), (1 + 0.1 * ref.randn(g, H)).half()


@pytest.mark.parametrize("M,H", NORM_SIZES)
def test_add_rmsnorm(sqp, M, H):
    """r: one rounding of the exact sum.  y: the fp32 sum of H squares (each thread's, then a tree) is off by far less than
    H 2^-24 relative, of which the root takes half, the four fp32 operations behind it by 2^-22; then the rounding to fp16."""
    print("case add_rmsnorm", M, H, flush=True)
    x, res, gamma = _norm_inputs(M, H, 3)
    y, r = sqp.add_rmsnorm(x.cuda(), res.cuda(), gamma.cuda(), 1e-5)
    y0, r0 = ref.add_rmsnorm(x, res, gamma, 1e-5)
    assert bool(((r.cpu().double() - r0).abs() <= 2.0 ** -11 * r0.abs() + 2.0 ** -25).all())
    tol = (2.0 ** -11 + H * 2.0 ** -25 + 2.0 ** -22) * y0.abs() + 2.0 ** -25
    assert bool(((y.cpu().double() - y0).abs() <= tol).all())
    # in place, and into given tensors
    rx, out = res.cuda(), torch.empty_like(y)
    y2, r2 = sqp.add_rmsnorm(x.cuda(), rx, gamma.cuda(), 1e-5, out=out, sum_out=rx)
    assert y2 is out and r2 is rx and torch.equal(y2, y) and torch.equal(r2, r)
    # the norm alone gives the same values of the same rows
    assert bool(((sqp.rmsnorm(r, gamma.cuda(), 1e-5).cpu().double() - y0).abs() <= tol).all())


@pytest.mark.parametrize("kind", ["int8", "e4m3"])
@pytest.mark.parametrize("M,H", NORM_SIZES)
def test_add_rmsnorm_quant(sqp, M, H, kind):
    """The scale follows the row's largest |y| (relative error as above, twice for the division); a code is the nearest of
    y / scale, so what it stands for is off by half a step of the codes there and by the errors of y and the scale."""
    print("case add_rmsnorm_quant", M, H, kind, flush=True)
    x, res, gamma = _norm_inputs(M, H, 4)
    codes, scales, r = sqp.add_rmsnorm_quant(x.cuda(), res.cuda(), gamma.cuda(), 1e-5, ref.TYPES[kind])
    assert codes.dtype == ref.TYPES[kind] and tuple(scales.shape) == (M,)
    y0, r0 = ref.add_rmsnorm(x, res, gamma, 1e-5)
    assert bool(((r.cpu().double() - r0).abs() <= 2.0 ** -11 * r0.abs() + 2.0 ** -25).all())
    e = H * 2.0 ** -25 + 2.0 ** -21
    s0 = y0.abs().amax(1) / ref.QMAX[kind]
    assert bool(((scales.cpu().double() - s0).abs() <= e * s0).all())
    back = codes.cpu().float().double()
    want = y0 / s0[:, None]
    tol = torch.maximum(ref.code_gap(back, kind), ref.code_gap(want, kind)) / 2 + 2 * e * want.abs()
    assert bool(((back - want).abs() <= tol).all())
    assert bool((back.abs().amax(1) == ref.QMAX[kind]).all())


def test_add_rmsnorm_rows_that_are_not_numbers(sqp):
    """A row with an infinity or NaN is NaN where the formula is, in the 8-bit form all of it; its neighbours are untouched,
    and a row of zeros is zeros."""
    x, res, gamma = _norm_inputs(5, 1024, 5)
    x[1, 7], x[2, 9] = float("inf"), float("nan")
    x[3], res[3] = 0, 0
    y, r = sqp.add_rmsnorm(x.cuda(), res.cuda(), gamma.cuda(), 1e-5)
    c, s, _ = sqp.add_rmsnorm_quant(x.cuda(), res.cuda(), gamma.cuda(), 1e-5, torch.int8)
    c8, s8, _ = sqp.add_rmsnorm_quant(x.cuda(), res.cuda(), gamma.cuda(), 1e-5, torch.float8_e4m3fn)
    ok = [0, 4]
    y1, _ = sqp.add_rmsnorm(x[ok].cuda(), res[ok].cuda(), gamma.cuda(), 1e-5)
    assert torch.equal(y[ok], y1)
    assert bool(y[2].isnan().all()) and bool(y[1, 7].isnan()) and not bool(y[3].any())
    assert bool(s[1:3].isnan().all()) and bool(s8[1:3].isnan().all()) and float(s[3]) == 0 and float(s8[3]) == 0
    assert not bool(c[3].any()) and not bool(c8[3].float().any())
    assert bool(s[ok].isfinite().all())


# ---------------------------------------------------------------- cache

CACHE_CASES = [  # tokens, heads, kv_heads, D, page
    (1, 64, 8, 128, 16), (1, 1, 1, 64, 16), (7, 32, 32, 128, 64), (37, 14, 2, 128, 32), (5, 16, 1, 64, 256), (130, 40, 40, 128, 16), (33, 15, 5, 64, 128)]


def _cache_inputs(T, heads, kv, D, page, kind, seed=6):
    g = ref.gen(seed)
    pages = -(-T // page) + 2
    qkv = ref.randn(g, T, (heads + 2 * kv) * D).half()
    slots = torch.randperm(pages * page, generator=g)[:T].int()
    positions = torch.randint(0, 5000, (T,), generator=g, dtype=torch.int32)
    k, ks = ref.make_cache(g, pages, kv, page, D, kind)
    v, vs = ref.make_cache(g, pages, kv, page, D, kind)
    return qkv, slots, positions, k, ks, v, vs


def _parts(qkv, heads, kv, D):
    T = qkv.shape[0]
    return (qkv[:, : heads * D].view(T, heads, D), qkv[:, heads * D: (heads + kv) * D].view(T, kv, D), qkv[:, (heads + kv) * D:].view(T, kv, D))


def _raw(t):
    return t.cpu().view(torch.uint8) if t.dtype == torch.float8_e4m3fn else t.cpu()


@pytest.mark.parametrize("rotated", [True, False])
@pytest.mark.parametrize("kind", ["fp16", "int8", "e4m3"])
@pytest.mark.parametrize("T,heads,kv,D,page", CACHE_CASES)
def test_cache_write_and_read(sqp, T, heads, kv, D, page, kind, rotated):
    """Rotation: two fp32 products and a sum, off by 2^-22 (|x| + |y|); then fp16's half step, or the codes' (the scale's
    error 2^-22 relative beside it).  Reading back adds one rounding to fp16.  Slots of other tokens keep their bits."""
    print("case cache", T, heads, kv, D, page, kind, rotated, flush=True)
    qkv, slots, positions, k0, ks0, v0, vs0 = _cache_inputs(T, heads, kv, D, page, kind)
    d = qkv.cuda()
    q, k, v = _parts(d, heads, kv, D)
    kc, vc, ks, vs = [None if t is None else t.cuda() for t in (k0, v0, ks0, vs0)]
    table = ref.cos_sin_table(5000, D)
    args = dict(cos_sin=table.cuda(), positions=positions.cuda()) if rotated else {}
    qr = sqp.kv_cache_write(k, v, slots.cuda(), kc, vc, ks, vs, q=q, **args)
    kb, vb = sqp.kv_cache_read(slots.cuda(), kc, vc, ks, vs)
    hq, hk, hv = _parts(qkv, heads, kv, D)
    want_q, want_k = [ref.rotate(x, table, positions) if rotated else x.double() for x in (hq, hk)]
    err_rot = lambda x: 2.0 ** -22 * (x.double().abs() + x.double().abs().roll(D // 2, -1)) * (1 if rotated else 0)
    tq = 2.0 ** -11 * want_q.abs() + 2.0 ** -25 + err_rot(hq)
    assert bool(((qr.cpu().double() - want_q).abs() <= tq).all())
    at, place = (slots // page).long(), (slots % page).long()
    for name, x, want, err, got_c, got_s, old_c, old_s, back in (("k", hk, want_k, err_rot(hk), kc, ks, k0, ks0, kb),
                                                                 ("v", hv, hv.double(), 0 * hv.double(), vc, vs, v0, vs0, vb)):
        stored = _raw(got_c)[at, :, place]
        untouched = torch.ones((k0.shape[0], page), dtype=torch.bool)
        untouched[at, place] = False
        same = untouched[:, None, :].expand(k0.shape[:3])
        assert torch.equal(_raw(got_c)[same], _raw(old_c)[same]), name
        if kind == "fp16":
            assert bool(((stored.double() - want).abs() <= 2.0 ** -11 * want.abs() + 2.0 ** -25 + err).all()), name
            assert torch.equal(back.cpu(), stored), name
            continue
        assert torch.equal(got_s.cpu()[same], old_s[same]), name
        scale = got_s.cpu()[at, :, place].double()
        codes = stored.view(torch.float8_e4m3fn).float().double() if kind == "e4m3" else stored.double()
        amax = want.abs().amax(-1)
        assert bool(((scale * ref.QMAX[kind] - amax).abs() <= 2.0 ** -22 * amax + err.amax(-1)).all()), name
        value = codes * scale[..., None]
        gap = torch.maximum(ref.code_gap(codes, kind), ref.code_gap(want / scale[..., None], kind)) * scale[..., None]
        assert bool(((value - want).abs() <= gap / 2 + 2.0 ** -21 * want.abs() + err).all()), name
        assert bool(((back.cpu().double() - value).abs() <= 2.0 ** -11 * value.abs() + 2.0 ** -25).all()), name


@pytest.mark.parametrize("kind", ["fp16", "int8", "e4m3"])
def test_cache_slots_and_positions_outside(sqp, kind):
    """Slots outside the cache: nothing is written, zeros are read; the queries come all the same.  A position outside the table
    makes its token NaN and no other.  Rows that are not finite read back as NaN (8-bit), rows of zeros as zeros."""
    T, heads, kv, D, page = 9, 8, 2, 128, 16
    qkv, _, positions, k0, ks0, v0, vs0 = _cache_inputs(T, heads, kv, D, page, kind)
    total = k0.shape[0] * page
    slots = torch.tensor([3, -1, total, total - 1, 1 << 30, 0, 17, 20, 21], dtype=torch.int32)
    positions[6], positions[5] = 5000, -1
    qkv[7, :], qkv[8, heads * D + 3] = 0, float("inf")
    q, k, v = _parts(qkv.cuda(), heads, kv, D)
    kc, vc, ks, vs = [None if t is None else t.cuda() for t in (k0, v0, ks0, vs0)]
    table = ref.cos_sin_table(5000, D)
    qr = sqp.kv_cache_write(k, v, slots.cuda(), kc, vc, ks, vs, q=q, cos_sin=table.cuda(), positions=positions.cuda())
    kb, vb = [t.cpu() for t in sqp.kv_cache_read(slots.cuda(), kc, vc, ks, vs)]
    inside = [0, 3, 5, 6, 7, 8]
    for i in (1, 2, 4):
        assert not bool(kb[i].any()) and not bool(vb[i].any()) and bool(qr[i].isfinite().all())
    free = torch.ones(total, dtype=torch.bool)
    free[slots[inside].long()] = False
    same = free.view(-1, 1, page).expand(k0.shape[:3])
    assert torch.equal(_raw(kc)[same], _raw(k0)[same]) and torch.equal(_raw(vc)[same], _raw(v0)[same])
    for i in (5, 6):
        assert bool(qr[i].isnan().all()) and bool(kb[i].isnan().all()) and bool(vb[i].isfinite().all())
    assert not bool(kb[7].any()) and not bool(vb[7].any())
    assert bool(kb[8, 0].isnan().all()) if kind != "fp16" else bool((~kb[8, 0].isfinite()).any())
    assert bool(kb[8, 1].isfinite().all()) and bool(kb[0].isfinite().all())


def test_cache_without_queries_and_empty(sqp):
    qkv, slots, positions, k0, ks0, v0, vs0 = _cache_inputs(3, 8, 2, 64, 16, "int8")
    q, k, v = _parts(qkv.cuda(), 8, 2, 64)
    a = [t.cuda() for t in (k0, v0, ks0, vs0)]
    b = [t.cuda() for t in (k0, v0, ks0, vs0)]
    sl = slots.cuda()
    assert sqp.kv_cache_write(k, v, sl, *a) is None
    out = torch.empty((3, 8, 64), dtype=torch.float16, device="cuda")
    assert sqp.kv_cache_write(k.contiguous(), v.contiguous(), sl, *b, q=q, out=out) is out
    assert torch.equal(out, q) and all(torch.equal(x, y) for x, y in zip(a, b))
    e = torch.empty((0, 2, 64), dtype=torch.float16, device="cuda")
    assert sqp.kv_cache_write(e, e, sl[:0], *b) is None
    kb, vb = sqp.kv_cache_read(sl[:0], *b)
    assert kb.shape == vb.shape == (0, 2, 64) and all(torch.equal(x, y) for x, y in zip(a, b))


def test_cache_larger_than_31_bits(sqp):
    """Slots at both ends of a cache of more than 2^31 elements: reads and writes go where they should, and the attention over
    those pages gives what it gives over the same tokens in a small cache."""
    kv, D, page, pages = 2, 128, 16, (1 << 31) // (2 * 128 * 16) + 40
    cache = [torch.empty((pages, kv, page, D), dtype=torch.int8, device="cuda") for _ in range(2)]
    scales = [torch.empty((pages, kv, page), dtype=torch.float32, device="cuda") for _ in range(2)]
    g = ref.gen(8)
    T = 48
    k, v = ref.randn(g, T, kv, D).half().cuda(), ref.randn(g, T, kv, D).half().cuda()
    use = torch.tensor([pages - 1, 1, pages - 20], dtype=torch.int32)
    t = torch.arange(T)
    slots = (use[t // page] * page + t % page).int().cuda()
    sqp.kv_cache_write(k, v, slots, *cache, *scales)
    small = [torch.empty((3, kv, page, D), dtype=torch.int8, device="cuda") for _ in range(2)]
    small_s = [torch.empty((3, kv, page), dtype=torch.float32, device="cuda") for _ in range(2)]
    sqp.kv_cache_write(k, v, t.int().cuda(), *small, *small_s)
    for a, b in zip(sqp.kv_cache_read(slots, *cache, *scales), sqp.kv_cache_read(t.int().cuda(), *small, *small_s)):
        assert torch.equal(a, b)
    for n in (1, 20):
        q = ref.randn(g, n, 8, D).half().cuda()
        lens, starts = torch.tensor([T - 3], dtype=torch.int32, device="cuda"), torch.tensor([0, n], dtype=torch.int32, device="cuda")
        o1 = sqp.paged_attention(q, *cache, use[None].cuda(), lens, starts, *scales, max_q=n, max_len=T)
        o2 = sqp.paged_attention(q, *small, torch.arange(3, dtype=torch.int32, device="cuda")[None], lens, starts, *small_s, max_q=n, max_len=T)
        assert torch.equal(o1, o2)


# ---------------------------------------------------------------- attention

def _compare(step, got, scale=None):
    want, tol = step.expected(scale)
    err = (got.cpu().double() - want).abs()
    assert bool((err <= tol).all()), "worst error / tolerance %.3f" % float((err / tol).nan_to_num(nan=1e9).max())


ATTENTION_CASES = [  # cached tokens, new tokens, heads, kv_heads, D, page
    ([1], [1], 32, 32, 128, 16),
    ([129], [1], 32, 32, 128, 16),
    ([0, 5, 17, 16, 15, 64, 65, 33], [1] * 8, 64, 8, 128, 16),
    ([1000, 1, 0, 31, 700, 257], [1] * 6, 14, 2, 64, 32),
    ([3001], [1], 16, 1, 128, 256),
    ([2200, 40], [1, 1], 40, 40, 128, 64),
    ([300, 301], [1, 1], 34, 2, 64, 16),                # 17 query heads on a cached one
    ([70, 9, 200], [2, 1, 3], 8, 2, 128, 16),           # a few new tokens each
    ([5, 5], [5, 5], 3, 1, 64, 16),                     # a prompt and nothing before it
    ([64], [64], 4, 4, 128, 64),
    ([200], [200], 6, 2, 64, 16),
    ([333, 50, 128], [129, 50, 1], 8, 1, 128, 16),
    ([517, 65, 64, 0, 90], [33, 1, 64, 1, 32], 20, 4, 128, 32),
    ([1300], [70], 16, 2, 64, 128),
    ([400, 3], [1, 3], 2, 2, 128, 16),
    ([2600], [17], 5, 5, 128, 64),
]


@pytest.mark.parametrize("kind", ["fp16", "int8", "e4m3"])
@pytest.mark.parametrize("case", range(len(ATTENTION_CASES)))
def test_attention(sqp, case, kind):
    lens, news, heads, kv, D, page = ATTENTION_CASES[case]
    print("case attention", lens, news, heads, kv, D, page, kind, flush=True)
    step = ref.Step(lens, news, heads, kv, D, page, kind, seed=20 + case)
    a = step.gpu()
    got = sqp.paged_attention(**a, max_q=max(news), max_len=max(lens))
    _compare(step, got)
    assert torch.equal(got, sqp.paged_attention(**a, max_q=max(news), max_len=max(lens))), "not the same bits twice"
    # without the hints, and into a given tensor
    out = torch.full_like(got, float("nan"))
    assert sqp.paged_attention(**a, out=out) is out
    _compare(step, out)
    if max(news) == 1:
        a["q_starts"] = None
        assert torch.equal(got, sqp.paged_attention(**a, max_q=1, max_len=max(lens)))


@pytest.mark.parametrize("kind", ["fp16", "int8", "e4m3"])
@pytest.mark.parametrize("heads,kv,D,lens,news", [
    (8, 2, 128, [1, 7, 40, 300], [1] * 4), (16, 1, 64, [2, 90, 33], [1] * 3), (4, 2, 128, [90, 8], [3, 8]), (8, 8, 64, [1500], [1])])
def test_attention_of_few_rows_rounds_once(sqp, heads, kv, D, lens, news, kind):
    """Up to 16 rows per cached head take p in two parts of 11 bits (2^-22 of it), so that the output's rounding is the only one to fp16.
    With x what is rounded and w the formula's value, fp16(x) is nearest to x: |fp16(x) - w| <= |fp16(w) - w| + 2 |x - w|.  Scores
    are small here, so that their own errors are."""
    print("case rounds once", heads, kv, D, lens, news, kind, flush=True)
    step = ref.Step(lens, news, heads, kv, D, 16, kind, seed=33, q_scale=0.01)
    got = sqp.paged_attention(**step.gpu(), max_q=max(news), max_len=max(lens)).cpu().double()
    want, tol = step.expected(p_error=2.0 ** -22, rounded=False)
    assert bool(((got - want).abs() <= (want.half().double() - want).abs() + 2 * tol).all())


@pytest.mark.parametrize("kind", ["fp16", "int8", "e4m3"])
@pytest.mark.parametrize("lens,news", [([40], [1]), ([40, 600, 9], [1, 1, 1]), ([40, 60], [2, 1]), ([60, 700], [40, 50]), ([300], [150])])
def test_attention_of_infinite_values(sqp, lens, news, kind):
    """A value (in 8 bits: its scale) that is infinite gives the outputs that the formula gives: infinities of its signs, NaN where a
    code of zero is scaled by it, and what is beside it is untouched."""
    print("case infinite values", lens, news, kind, flush=True)
    step = ref.Step(lens, news, 8, 2, 128, 16, kind, seed=34, q_scale=0.1)
    tol = step.expected()[1]                        # (as without the infinities, which are in dimensions of their own)
    page, place = int(step.table[0, 1]), 3          # token 19 of the first sequence, which all of its new tokens see
    if kind == "fp16":
        step.v[page, 1, place, ::5] = float("inf")
        step.v[page, 1, place, 1::5] = float("-inf")
    else:
        step.vs[page, 1, place] = float("inf")
    got = sqp.paged_attention(**step.gpu(), max_q=max(news), max_len=max(lens)).cpu().double()
    want, _ = step.expected()
    fine = want.isfinite()
    assert bool((~fine).any()) and bool(fine.any())
    assert bool(((got[fine] - want[fine]).abs() <= tol[fine]).all())
    assert torch.equal(got[~fine].nan_to_num(nan=0.0, posinf=1.0, neginf=-1.0), want[~fine].nan_to_num(nan=0.0, posinf=1.0, neginf=-1.0))


@pytest.mark.parametrize("lens,news", [([40, 9], [1, 1]), ([40], [3]), ([300, 70], [150, 9])])
def test_attention_of_codes_that_are_not_numbers(sqp, lens, news):
    """A NaN among e4m3's codes makes NaN of its dimension (a value) or its token's score (a key), of the rows that see it."""
    print("case codes not numbers", lens, news, flush=True)
    for what, at in (("v", 20), ("v", lens[0] - 1), ("k", lens[0] - 1)):
        step = ref.Step(lens, news, 8, 2, 128, 16, "e4m3", seed=36)
        tol = step.expected()[1]  # (as without the NaN, which is in one dimension, or in all of a lost row)
        getattr(step, what).view(torch.uint8)[int(step.table[0, at // 16]), 1, at % 16, 77] = 0x7f
        got = sqp.paged_attention(**step.gpu(), max_q=max(news), max_len=max(lens)).cpu().double()
        want, _ = step.expected()
        lost = want.isnan()
        rows = news[0] if at == 20 else 1
        assert int(lost.sum()) == rows * 4 * (1 if what == "v" else 128)
        assert torch.equal(got.isnan(), lost)
        assert bool(((got - want).abs() <= tol)[~lost].all())


@pytest.mark.parametrize("kind", ["int8", "e4m3"])
@pytest.mark.parametrize("lens,news", [([40, 600], [1, 1]), ([300, 70], [150, 9])])
def test_attention_of_scales_of_either_sign_and_not_a_number(sqp, lens, news, kind):
    """A scale is a factor like any other: negative ones (which the write does not make), zero, and NaN where a token is seen."""
    print("case scales", lens, news, kind, flush=True)
    step = ref.Step(lens, news, 8, 2, 128, 16, kind, seed=35)
    for scales in (step.ks, step.vs):
        scales[..., 1::3] *= -1.0
        scales[..., 5::7] = 0.0
    step.vs[int(step.table[0, 1]), 1, 4] = float("nan")  # token 20 of the first sequence, second cached head
    got = sqp.paged_attention(**step.gpu(), max_q=max(news), max_len=max(lens)).cpu().double()
    want, tol = step.expected()
    lost = want.isnan()
    assert torch.equal(got.isnan(), lost) and bool(lost[: news[0], 4:].all()) and int(lost.sum()) == news[0] * 4 * 128
    assert bool(((got - want).abs() <= tol)[~lost].all())


@pytest.mark.parametrize("kind", ["fp16", "int8", "e4m3"])
@pytest.mark.parametrize("heads,kv,D,lens,news", [
    (32, 32, 64, [4096], [4096]),                       # as many tiles as take the 256-row form, one sequence
    (64, 8, 128, [2300, 1500], [1100, 1029]),           # and two
    (64, 16, 128, [600, 2111, 33, 700], [600, 1, 33, 500]),
    (8, 8, 128, [1025], [1025])])
def test_attention_many_rows(sqp, heads, kv, D, lens, news, kind):
    """Long prompts: sampled rows (the first and last of every tile edge's neighbourhood among them) of sampled heads."""
    print("case many rows", heads, kv, D, lens, news, kind, flush=True)
    step = ref.Step(lens, news, heads, kv, D, 64, kind, seed=30)
    got = sqp.paged_attention(**step.gpu(), max_q=max(news), max_len=max(lens)).cpu()
    assert bool(got.isfinite().all())
    rows = [(b, i, h) for b, n in enumerate(news) for i in sorted({0, 1, n // 3, n // 2, n - 2, n - 1, *range(31, n, max(32, n // 8)), *range(32, n, max(32, n // 8))})
            if 0 <= i < n for h in (0, heads // 2 + 1, heads - 1)]
    want, tol = step.expected(rows=rows)
    at = [(int(step.starts[b]) + i, h) for b, i, h in rows]
    t, h = torch.tensor([a[0] for a in at]), torch.tensor([a[1] for a in at])
    err = (got[t, h].double() - want[t, h]).abs()
    assert bool((err <= tol[t, h]).all()), "worst error / tolerance %.3f" % float((err / tol[t, h]).max())


@pytest.mark.parametrize("kind", ["fp16", "int8"])
def test_attention_many_rows_later_token_not_a_number(sqp, kind):
    """The slow way of the 256-row form."""
    step = ref.Step([900], [900], 160, 160, 64, 16, kind, seed=31)
    free = torch.zeros((step.k.shape[0], 16), dtype=torch.bool)
    free[step.table[0, 899 // 16].long(), 899 % 16] = True
    ref.spoil(step.v, step.vs, free)
    got = sqp.paged_attention(**step.gpu(), max_q=900, max_len=900).cpu()
    assert bool(got[899].isnan().all()) and bool(got[:899].isfinite().all())
    rows = [(0, i, h) for i in (0, 255, 256, 511, 640, 767, 768, 897, 898) for h in (0, 77, 159)]
    want, tol = step.expected(rows=rows)
    for b, i, h in rows:
        assert bool(((got[i, h].double() - want[i, h]).abs() <= tol[i, h]).all()), (i, h)


@pytest.mark.parametrize("kind", ["fp16", "e4m3"])
@pytest.mark.parametrize("B", [9, 64, 65, 150])
def test_attention_many_sequences(sqp, B, kind):
    """Ragged batches of more sequences than a wave has lanes, single tokens beside short prompts, some of them unused."""
    print("case many sequences", B, kind, flush=True)
    lens = [(37 * b * b + 11 * b) % 190 for b in range(B)]
    news = [1 if b % 3 or lens[b] < 30 else 17 + b % 13 for b in range(B)]
    step = ref.Step(lens, news, 6, 2, 64, 16, kind, seed=32)
    got = sqp.paged_attention(**step.gpu(), max_q=max(news), max_len=max(lens))
    _compare(step, got)
    _compare(step, sqp.paged_attention(**step.gpu(), max_q=1, max_len=16))


@pytest.mark.parametrize("kind", ["fp16", "e4m3"])
@pytest.mark.parametrize("lens,news", [([700, 90], [1, 1]), ([700, 300], [40, 130])])
def test_attention_hints_that_are_too_small(sqp, lens, news, kind):
    """Arrays that hold more than max_q and max_len say give the same values."""
    step = ref.Step(lens, news, 8, 2, 128, 16, kind, seed=9)
    for max_q, max_len in ((1, 1), (5, 100), (64, 128), (1 << 20, 1 << 20)):
        print("case hints", lens, news, kind, max_q, max_len, flush=True)
        _compare(step, sqp.paged_attention(**step.gpu(), max_q=max_q, max_len=max_len))


@pytest.mark.parametrize("kind", ["fp16", "int8", "e4m3"])
@pytest.mark.parametrize("heads,kv,D,lens,news", [(8, 2, 128, [100, 90], [3, 2]), (4, 4, 64, [300, 20], [150, 20]), (16, 2, 128, [260], [40])])
def test_attention_later_tokens_that_are_not_numbers(sqp, heads, kv, D, lens, news, kind):
    """Keys and values of the newest token are NaN: the tokens before it do not depend on them, the newest itself is NaN."""
    print("case later tokens", heads, kv, D, lens, news, kind, flush=True)
    step = ref.Step(lens, news, heads, kv, D, 16, kind, seed=10)
    for b, n in enumerate(lens):
        free = torch.zeros((step.k.shape[0], 16), dtype=torch.bool)
        free[step.table[b, (n - 1) // 16].long(), (n - 1) % 16] = True
        ref.spoil(step.v, step.vs, free)
        if b == 0:
            ref.spoil(step.k, step.ks, free)
    got = sqp.paged_attention(**step.gpu(), max_q=max(news), max_len=max(lens)).cpu()
    want, tol = step.expected()
    last = (step.starts[1:] - 1).long()
    assert bool(got[last].isnan().all())
    keep = torch.ones(got.shape[0], dtype=torch.bool)
    keep[last] = False
    assert bool(((got[keep].double() - want[keep]).abs() <= tol[keep]).all())


def test_attention_infinite_scores_and_tokens_that_see_nothing(sqp):
    """Scores of minus infinity and of the lowest values weigh nothing; a token all of whose scores are minus infinity, or that
    sees no token (more new tokens than cached ones), gets zeros."""
    for n, heads, kv in ((1, 8, 2), (6, 8, 1), (40, 8, 2)):
        print("case scores", n, heads, kv, flush=True)
        step = ref.Step([90], [n], heads, kv, 128, 16, "fp16", seed=11)
        step.q[..., 0] = 1.0
        a = step.gpu()
        rows = lambda t: (step.table[0, t // 16].long(), t % 16)
        k = step.k.clone()
        for t in range(90):
            pg, pl = rows(t)
            if t % 3 == 1:
                k[pg, :, pl, :] = 0
                k[pg, :, pl, 0] = float("-inf")
            elif t % 3 == 2:
                k[pg, :, pl, :] = 0
                k[pg, :, pl, 0] = -65504.0
        a["k_cache"] = k.cuda()
        got = sqp.paged_attention(**a, max_q=n, max_len=90)
        step.k = k.clone()
        for t in range(90):  # (a score of minus infinity: the lowest finite one stands for it in the 64-bit form)
            pg, pl = rows(t)
            step.k[pg, :, pl, 0] = torch.where(step.k[pg, :, pl, 0].isinf(), torch.tensor(-65504.0).half(), step.k[pg, :, pl, 0])
        _compare(step, got)
        for t in range(90):
            pg, pl = rows(t)
            k[pg, :, pl, :] = 0
            k[pg, :, pl, 0] = float("-inf")
        a["k_cache"] = k.cuda()
        assert not bool(sqp.paged_attention(**a, max_q=n, max_len=90).any())
    for n, length in ((3, 2), (50, 20)):
        step = ref.Step([length], [n], 4, 2, 64, 16, "fp16", seed=12)
        got = sqp.paged_attention(**step.gpu(), max_q=n, max_len=length)
        _compare(step, got)
        assert not bool(got[: n - length].any())


@pytest.mark.parametrize("kind", ["int8", "e4m3"])
def test_attention_scales_of_all_sizes(sqp, kind):
    """Value scales from 2^-60 to 2^60 and zeros: tokens of any size beside each other, and all of them tiny."""
    for n in (1, 40):
        step = ref.Step([300], [n], 8, 2, 128, 16, kind, seed=13)
        g = ref.gen(14)
        step.vs.copy_(torch.exp2(torch.randint(-60, 10, step.vs.shape, generator=g).float()))
        step.vs[:, :, 3] = 0
        _compare_wide(step, sqp.paged_attention(**step.gpu(), max_q=n, max_len=300))
        step.vs.fill_(2.0 ** -13)
        _compare(step, sqp.paged_attention(**step.gpu(), max_q=n, max_len=300))
        step.ks.mul_(30.0)
        _compare(step, sqp.paged_attention(**step.gpu(), max_q=n, max_len=300))


def _compare_wide(step, got):
    """Where values of very different size meet, p times the value's scale is rounded against the largest of them: the term per
    token of the tolerance has the largest |v| of the row in it already; outputs past fp16's range are infinite."""
    want, tol = step.expected()
    got, top = got.cpu().double(), 65504.0
    assert bool((((got - want).abs() <= tol) | (want.abs() >= top - tol)).all())


def test_attention_scale_and_views(sqp):
    """A scale of the caller's, queries that are a view of a merged projection, a page table with longer rows."""
    step = ref.Step([150, 60], [40, 1], 8, 2, 128, 16, "fp16", seed=15)
    a = step.gpu()
    merged = torch.full((41, 8 * 128 + 512), float("nan"), dtype=torch.float16, device="cuda")
    merged[:, : 8 * 128] = a["q"].reshape(41, -1)
    a["q"] = merged[:, : 8 * 128].view(41, 8, 128)
    wide = torch.full((2, 40), 1 << 29, dtype=torch.int32, device="cuda")
    wide[:, : a["page_table"].shape[1]] = a["page_table"]
    a["page_table"] = wide[:, : a["page_table"].shape[1]]
    _compare(step, sqp.paged_attention(**a, scale=0.02, max_q=40, max_len=150), 0.02)


def test_attention_rows_of_no_sequence(sqp):
    """Rows in front of the first start and behind the last one get zeros; starts beyond T and lengths beyond the table are
    taken as the nearest inside."""
    step = ref.Step([50, 80], [3, 30], 8, 2, 64, 16, "fp16", seed=16)
    a = step.gpu()
    q = torch.cat([torch.ones_like(a["q"][:2]), a["q"], torch.ones_like(a["q"][:5])])
    a["q"], a["q_starts"] = q, a["q_starts"] + 2
    got = sqp.paged_attention(**a, max_q=30, max_len=80)
    assert not bool(got[:2].any()) and not bool(got[-5:].any())
    _compare(step, got[2:-5])
    one = ref.Step([64], [2], 8, 2, 64, 16, "fp16", seed=17)
    b = one.gpu()
    b["seq_lens"] = torch.tensor([1 << 30], dtype=torch.int32, device="cuda")
    b["q_starts"] = torch.tensor([0, 1 << 30], dtype=torch.int32, device="cuda")
    _compare(one, sqp.paged_attention(**b, max_q=2, max_len=64))


def test_attention_streams_and_graphs(sqp):
    """On a side stream, and recorded into graphs that are replayed with eager work and new inputs between the replays."""
    steps = [ref.Step([1500, 40], [1, 1], 8, 2, 128, 16, "e4m3", seed=18), ref.Step([700, 64], [40, 3], 8, 2, 128, 16, "int8", seed=19)]
    for step in steps:
        a, n, most = step.gpu(), max(step.news), max(step.lens)
        eager = sqp.paged_attention(**a, max_q=n, max_len=most)
        _compare(step, eager)
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            on_side = sqp.paged_attention(**a, max_q=n, max_len=most)
        torch.cuda.current_stream().wait_stream(side)
        assert torch.equal(on_side, eager)
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            held = sqp.paged_attention(**a, max_q=n, max_len=most)
        g2 = torch.cuda.CUDAGraph()
        given = torch.empty_like(eager)
        with torch.cuda.graph(g2):
            sqp.paged_attention(**a, max_q=n, max_len=most, out=given)
        for i in range(3):
            a["q"].mul_(0.5 if i else 1.0)
            now = sqp.paged_attention(**a, max_q=n, max_len=most)
            g.replay()
            g2.replay()
            torch.cuda.synchronize()
            assert torch.equal(held, now)
            step.q = a["q"].cpu()
            _compare(step, given)


# ---------------------------------------------------------------- bounds

def _guarded(nbytes, front=256, back=256):
    """A device buffer with guard bytes on both sides: (whole, the part in between)."""
    whole = torch.full((front + nbytes + back,), 0xA5, dtype=torch.uint8, device="cuda")
    return whole, whole[front: front + nbytes]


def _intact(whole, nbytes, front=256):
    return bool((whole[:front] == 0xA5).all()) and bool((whole[front + nbytes:] == 0xA5).all())


@pytest.mark.parametrize("kind", ["fp16", "e4m3"])
@pytest.mark.parametrize("lens,news,heads,kv,D", [([3000, 5, 700], [1, 1, 1], 8, 2, 128), ([2500], [17], 5, 5, 64), ([1500, 900], [33, 900], 8, 2, 128)])
def test_attention_scratch_of_any_size_and_guards(sqp, lens, news, heads, kv, D, kind):
    """The output and the scratch stay inside their buffers, and with less scratch than the preferred plan's, or none, the
    values are still right."""
    import ctypes
    L = sqp.lib()
    step = ref.Step(lens, news, heads, kv, D, 16, kind, seed=40)
    a, T, B, page, width = step.gpu(), sum(news), len(lens), 16, step.table.shape[1]
    need = int(L.sqp_paged_attention_scratch_bytes(T, B, heads, kv, D, max(news), max(lens)))
    P = lambda t: ctypes.c_void_p(t.data_ptr()) if t is not None else None
    st = ctypes.c_void_p(torch.cuda.current_stream().cuda_stream)
    kind_at = {"fp16": 0, "int8": 1, "e4m3": 2}[kind]
    for nbytes in sorted({0, need // 3 & ~15, need}):
        print("case scratch", lens, news, kind, nbytes, need, flush=True)
        out_w, out = _guarded(T * heads * D * 2)
        scr_w, scr = _guarded(max(nbytes, 16))
        rc = L.sqp_paged_attention(T, B, heads, kv, D, kind_at, page, step.k.shape[0], width, max(news), max(lens), D ** -0.5, P(a["q"]), heads * D,
                                   P(a["k_cache"]), P(a["v_cache"]), P(a["k_scales"]), P(a["v_scales"]), P(a["page_table"]), width, P(a["seq_lens"]),
                                   P(a["q_starts"]), P(out), P(scr) if nbytes else None, nbytes, st)
        assert rc == 0
        torch.cuda.synchronize()
        assert _intact(out_w, T * heads * D * 2) and _intact(scr_w, max(nbytes, 16))
        _compare(step, out.view(torch.float16).view(T, heads, D))


@pytest.mark.parametrize("kind", ["fp16", "int8", "e4m3"])
def test_cache_and_norm_guards(sqp, kind):
    """Writes stay inside the outputs on odd sizes."""
    T, heads, kv, D, page, pages = 7, 3, 1, 64, 16, 2
    qkv, slots, positions, *_ = _cache_inputs(T, heads, kv, D, page, kind)
    q, k, v = _parts(qkv.cuda(), heads, kv, D)
    dt = ref.TYPES[kind]
    size = pages * kv * page * D * (2 if kind == "fp16" else 1)
    bufs = [_guarded(size), _guarded(size), _guarded(pages * kv * page * 4), _guarded(pages * kv * page * 4), _guarded(T * heads * D * 2)]
    kc, vc = [b[1].view(dt).view(pages, kv, page, D) for b in bufs[:2]]
    ks, vs = [b[1].view(torch.float32).view(pages, kv, page) if kind != "fp16" else None for b in bufs[2:4]]
    slots = torch.tensor([0, 31, 15, 16, 40, -3, 7], dtype=torch.int32).cuda()
    sqp.kv_cache_write(k, v, slots, kc, vc, ks, vs, q=q, cos_sin=ref.cos_sin_table(5000, D).cuda(), positions=positions.cuda(),
                       out=bufs[4][1].view(torch.float16).view(T, heads, D))
    rk, rv = _guarded(T * kv * D * 2), _guarded(T * kv * D * 2)
    sqp.kv_cache_read(slots, kc, vc, ks, vs, out=[b[1].view(torch.float16).view(T, kv, D) for b in (rk, rv)])
    torch.cuda.synchronize()
    for whole, part in bufs + [rk, rv]:
        assert _intact(whole, part.numel())
    M, H = 3, 2056
    x, res, gamma = _norm_inputs(M, H, 50)
    y, r, c, s = _guarded(M * H * 2), _guarded(M * H * 2), _guarded(M * H), _guarded(16)
    half = lambda b: b[1].view(torch.float16).view(M, H)
    sqp.add_rmsnorm(x.cuda(), res.cuda(), gamma.cuda(), 1e-5, out=half(y), sum_out=half(r))
    if kind != "fp16":
        sqp.add_rmsnorm_quant(x.cuda(), res.cuda(), gamma.cuda(), 1e-5, dt, out=(c[1].view(dt).view(M, H), s[1].view(torch.float32)[:M]), sum_out=half(r))
    torch.cuda.synchronize()
    for whole, part in (y, r, c, s):
        assert _intact(whole, part.numel())
