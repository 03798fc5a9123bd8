"""GPU parity of the attention over the paged cache where weights and values span a wide range: against 64 bits, with a bound
in which a token's share is that of its own weight."""
import pytest
import torch

import layer_ref as ref

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def sqp():
    import paper_2312_03788_amd as m
    m.lib()
    return m


def expected(step, floor, alone=True):
    """(out, tolerance) [T, heads, D] in 64 bits.  With w_j what is rounded for the matrix cores (p_j, for codes p_j times the value's
    scale), c_j the value over that scale and A = sum_j p_j |v_j|, the outputs are off by at most
      output's rounding   2^-11 |o| + 2^-25
      w's rounding        sum_j max(eps w_j, floor max_i w_i) |c_j|: eps = 2^-22 up to 16 rows per cached head, 2^-11 above and beside
                          sequences of more (alone=False), where fp16 caches sum the rounded p, so that |o| is added to |c_j|;
                          floor: half of fp16's smallest step, 2^-25, over the least that the largest w is held at
      scores              (D + 8) 2^-24 sum_d |q_d k_d| scale, the power of two 2^-21, in tiles of codes 2^-16 for the logarithm
                          of the value's scale (2^-18 of up to 40 each way) and its inverse: of each p, in numerator and denominator
      sums                len 2^-24 each."""
    scale, group = step.D ** -0.5, step.heads // step.kv_heads
    T = step.q.shape[0]
    out, tol = torch.zeros((T, step.heads, step.D), dtype=torch.float64), torch.full((T, step.heads, step.D), 2.0 ** -25, dtype=torch.float64)
    codes = step.v.float()
    for b, (length, n) in enumerate(zip(step.lens, step.news)):
        if length == 0:
            continue
        few = n * group <= 16 and alone
        k, c = step.rows(b, step.k, step.ks), step.rows(b, codes, None)
        size = step.rows(b, torch.ones_like(codes[..., :1]), step.vs)[..., 0]
        for i in range(max(0, n - length), n):
            m, t = length - n + i + 1, int(step.starts[b]) + i
            for h in range(step.kv_heads):
                at = slice(h * group, (h + 1) * group)
                kh, ch, vs, q = k[h, :m], c[h, :m], size[h, :m], step.q[t, at].double()
                p = torch.softmax(q @ kh.T * scale, 1)
                w = p * vs
                o, A = w @ ch, w @ ch.abs()
                d = torch.maximum((2.0 ** -22 if few else 2.0 ** -11) * w, floor * w.amax(1, keepdim=True))
                e = (step.D + 8) * 2.0 ** -24 * scale * (q.abs() @ kh.abs().T) + 2.0 ** -21 + (0 if few or step.kind == "fp16" else 2.0 ** -16)
                out[t, at] = o
                tol[t, at] += 2.0 ** -11 * o.abs() + d @ ch.abs() + (d.sum(1, keepdim=True) * o.abs() if not few and step.kind == "fp16" else 0) \
                    + (e * w) @ ch.abs() + (e * p).sum(1, keepdim=True) * o.abs() + m * 2.0 ** -23 * A
    return out, tol


def compare(step, got, floor, alone=True):
    want, tol = expected(step, floor, alone)
    err = (got.cpu().double() - want).abs()
    assert bool((err <= tol).all()), "worst error / tolerance %.3f" % float((err / tol).nan_to_num(nan=1e9).max())


def attend(sqp, step, **more):
    return sqp.paged_attention(**step.gpu(), max_q=max(step.news), max_len=max(step.lens), **more)


def set_scores(step, of):
    """Queries and keys whose score of token t, of every sequence and head, is near of(t) as a power of two: the first dimension alone
    of the keys, the first of the queries 8."""
    step.q[..., 0] = 8.0
    raw = step.k if step.kind == "fp16" else step.k.view(torch.int8)
    for b, length in enumerate(step.lens):
        for t in range(length):
            page, place = int(step.table[b, t // step.page]), t % step.page
            x = of(t) * 0.6931471805599453 * step.D ** 0.5 / 8.0
            raw[page, :, place] = 0
            if step.kind == "fp16":
                step.k[page, :, place, 0] = x
            else:
                raw[page, :, place, 0] = 64 if step.kind == "int8" else 0x38  # (0x38: 1.0)
                step.ks[page, :, place] = x / (64.0 if step.kind == "int8" else 1.0)


@pytest.mark.parametrize("kind", ["int8", "e4m3"])
@pytest.mark.parametrize("r", [12, 16, 20, 24, 30])
@pytest.mark.parametrize("lens,news", [([40], [1]), ([40, 1024], [1, 1]), ([90, 33], [2, 3]), ([300], [40])])
def test_large_values_that_weigh_nothing(sqp, lens, news, r, kind):
    """Two tokens' value rows, one seen by all and the newest, lie 2^r above the others while their scores leave them nothing
    (2^-(r + 24)): the other tokens' weights lose no bits to them."""
    print("case large values", lens, news, r, kind, flush=True)
    step = ref.Step(lens, news, 8, 2, 128, 16, kind, seed=60)
    loud = lambda t: t == 5 or t + 1 in lens
    set_scores(step, lambda t: -(r + 24.0) if loud(t) else (t * 7 % 5) * 0.25)
    for b, length in enumerate(lens):
        for t in range(length):
            if loud(t):
                step.vs[int(step.table[b, t // 16]), :, t % 16] *= 2.0 ** r
    compare(step, attend(sqp, step), 2.0 ** -25)


@pytest.mark.parametrize("kind", ["fp16", "int8", "e4m3"])
@pytest.mark.parametrize("down", [14, 20, 26])
@pytest.mark.parametrize("lens,news", [([3000], [1]), ([700, 5000], [1, 2]), ([2500], [20])])
def test_a_first_token_that_outweighs_a_long_tail(sqp, lens, news, down, kind):
    """The first token has a score `down` powers of two above all the others and values of zero: the output is the tail's, whose
    weights are held to 2^-11 (few rows: 2^-22) of themselves or 2^-35 of the largest."""
    print("case long tail", lens, news, down, kind, flush=True)
    step = ref.Step(lens, news, 4, 2, 128, 16, kind, seed=61)
    set_scores(step, lambda t: 0.0 if t == 0 else -down + (t * 7 % 5) * 0.25)
    if kind == "fp16":
        step.v.abs_().mul_(50.0)
    else:
        step.v.view(torch.uint8).copy_(step.v.float().abs().to(step.v.dtype).view(torch.uint8))
        step.vs.mul_(50.0)
    for b in range(len(lens)):
        step.v.view(torch.int16 if kind == "fp16" else torch.uint8)[int(step.table[b, 0]), :, 0] = 0
    compare(step, attend(sqp, step), 2.0 ** -35)


@pytest.mark.parametrize("lens,news,heads", [([33, 0], [32, 1], 512), ([40, 40], [40, 40], 1024), ([9, 1, 5], [9, 1, 3], 600), ([70, 3], [64, 3], 300)])
def test_many_query_heads_on_one_cached_head(sqp, lens, news, heads):
    """More query heads per cached one than a tile has rows, so that a token takes several tiles: every row of several sequences is
    written (the output holds NaN before)."""
    print("case many heads", lens, news, heads, flush=True)
    step = ref.Step(lens, news, heads, 1, 64, 16, "fp16", seed=62)
    out = torch.full(step.q.shape, float("nan"), dtype=torch.float16, device="cuda")
    compare(step, attend(sqp, step, out=out), 2.0 ** -35)


@pytest.mark.parametrize("lens,news", [([150], [1]), ([150, 900], [1, 1]), ([300], [40])])
def test_not_a_number_among_scores_of_minus_infinity(sqp, lens, news):
    """The first 70 tokens have scores of minus infinity, one of them a value row of NaN: zero times it is NaN, for every row that sees it,
    whether or not anything has a weight before it."""
    print("case NaN behind minus infinity", lens, news, flush=True)
    step = ref.Step(lens, news, 8, 2, 128, 16, "fp16", seed=63)
    set_scores(step, lambda t: 0.0)
    for b in range(len(lens)):
        for t in range(70):
            step.k[int(step.table[b, t // 16]), :, t % 16, 0] = float("-inf")
        step.v[int(step.table[b, 1]), :, 3] = float("nan")
    assert bool(attend(sqp, step).isnan().all())


@pytest.mark.parametrize("kind", ["int8", "e4m3"])
@pytest.mark.parametrize("lens,news", [([12000], [1]), ([12000], [20]), ([90, 12000], [33, 20])])
def test_tokens_of_zero_values_keep_their_weight(sqp, lens, news, kind):
    """One token with a weight 2^20 above the others' and large values, thousands of zero values (scale 0): these have 1 % of the
    sum, in whatever part of the sequence they are."""
    print("case zero values", lens, news, kind, flush=True)
    step = ref.Step(lens, news, 4, 2, 128, 16, kind, seed=64)
    set_scores(step, lambda t: 20.0 if t == 5 else 0.0)
    for b, length in enumerate(lens):
        for t in range(length):
            step.vs[int(step.table[b, t // 16]), :, t % 16] = (2.0 ** 9 if kind == "int8" else 2.0 ** 7) if t == 5 else 0.0
    compare(step, attend(sqp, step), 2.0 ** -35)


@pytest.mark.parametrize("kind", ["int8", "e4m3"])
@pytest.mark.parametrize("n", [1, 40])
def test_value_scales_up_to_large_powers(sqp, n, kind):
    """Value scales of 2^-60 to 2^60 beside each other, with scores that leave the large ones a share of the output or more: outputs inside
    fp16's range are to 64 bits, the others are infinite with the right sign."""
    print("case large scales", n, kind, flush=True)
    step = ref.Step([300], [n], 8, 2, 128, 16, kind, seed=65)
    power = lambda t: t * 41 % 121 - 60
    set_scores(step, lambda t: -1.0 * max(power(t) - (16 if t % 7 == 0 else 0), 0))
    for t in range(300):
        step.vs[int(step.table[0, t // 16]), :, t % 16] = 2.0 ** power(t)
    got = attend(sqp, step).cpu().double()
    want, tol = expected(step, 2.0 ** -35)
    top = 65520.0  # (from here on rounding gives an infinity)
    inside, outside = want.abs() < 65504.0 - tol, want.abs() > top + tol
    assert bool(inside.any()) and bool(((got - want).abs() <= tol)[inside].all())
    assert bool((got == torch.sign(want) * float("inf"))[outside].all())


@pytest.mark.parametrize("kind", ["fp16", "e4m3"])
@pytest.mark.parametrize("lens,news,heads,kv,D,max_len", [
    ([3000, 17, 2600, 0, 1500, 700, 2049, 1, 2048, 900, 1800, 64], [1, 1, 40, 1, 2, 17, 1, 1, 4, 3, 33, 5], 8, 2, 128, 3000),    # parts of tiles
    ([2500, 2600, 1100, 513, 512, 2700, 256, 257, 1600, 40], [2090] + [1] * 9, 16, 1, 64, 8192),             # of the single tokens beside whole tiles
    ([1100, 900, 1100, 513, 512, 700, 256, 257, 600, 0], [1050, 850] + [1] * 8, 24, 24, 64, 1100)])          # a cache for every head
def test_single_tokens_and_chunks_in_parts(sqp, lens, news, heads, kv, D, max_len, kind):
    """Single tokens and chunks in one call, long enough for parts, with one kernel and with two: the partial results stay inside the scratch,
    with any amount of it, and the output is whole."""
    import ctypes
    print("case parts", lens, news, heads, kv, D, kind, flush=True)
    L = sqp.lib()
    step = ref.Step(lens, news, heads, kv, D, 16, kind, seed=66)
    want, tol = expected(step, 2.0 ** -35, alone=False)
    T, B, a = sum(news), len(lens), step.gpu()
    need = int(L.sqp_paged_attention_scratch_bytes(T, B, heads, kv, D, max(news), max_len))
    assert need > 0
    P = lambda t: ctypes.c_void_p(t.data_ptr()) if t is not None else None
    for nbytes in (need, need - 16, need // 3 & ~15, 16, 0):
        out = torch.full((T + 2, heads, D), float("nan"), dtype=torch.float16, device="cuda")
        scratch = torch.full((need + 512,), 0xFF, dtype=torch.uint8, device="cuda")  # (NaN where it is read without having been written)
        rc = L.sqp_paged_attention(T, B, heads, kv, D, {"fp16": 0, "e4m3": 2}[kind], 16, step.k.shape[0], step.table.shape[1], max(news), max_len, D ** -0.5,
                                   P(a["q"]), heads * D, P(a["k_cache"]), P(a["v_cache"]), P(a["k_scales"]), P(a["v_scales"]), P(a["page_table"]),
                                   step.table.shape[1], P(a["seq_lens"]), P(a["q_starts"]), P(out[1:]), P(scratch[256:]) if nbytes else None, nbytes,
                                   ctypes.c_void_p(torch.cuda.current_stream().cuda_stream))
        assert rc == 0
        torch.cuda.synchronize()
        assert bool((scratch[:256] == 0xFF).all()) and bool((scratch[256 + nbytes:] == 0xFF).all())
        assert bool(out[0].isnan().all()) and bool(out[-1].isnan().all())
        err = (out[1:-1].cpu().double() - want).abs()
        assert bool((err <= tol).all()), "scratch %d of %d: worst error / tolerance %.3f" % (nbytes, need, float((err / tol).nan_to_num(nan=1e9).max()))
    # hints that are too small: sequences of more rows, and longer ones, than there are places for
    compare(step, sqp.paged_attention(**a, max_q=2, max_len=1000), 2.0 ** -35, alone=False)
