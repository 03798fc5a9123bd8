"""How the operators on microscaled numbers add: what is rounded, and what is not."""
import pytest
import torch

import layer_ref as ref
import mx_ref as mx
import mx_sums

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def sqp():
    import paper_2312_03788_amd as m
    m.lib()
    return m


# ---------------------------------------------------------------- attention

@pytest.mark.parametrize("heads,kv,D,lens,news", [
    (8, 2, 128, [1, 7, 40, 300], [1] * 4), (16, 1, 64, [2, 90, 33], [1] * 3), (4, 2, 128, [90, 8], [3, 8]), (8, 8, 64, [1500], [1]), (64, 8, 128, [2100, 700], [1, 1])])
def test_attention_of_few_rows_rounds_once(sqp, heads, kv, D, lens, news):
    """Over e2m1 blocks as over the other caches, up to 16 rows per cached head take p in two parts of 11 bits (2^-22 of it), so that the
    output's rounding is the only one to fp16.  With x what is rounded and w the formula's value, fp16(x) is nearest to x:
    |fp16(x) - w| <= |fp16(w) - w| + 2 |x - w|.  Scores are small here, so that their own errors are."""
    print("case rounds once", heads, kv, D, lens, news, flush=True)
    s = mx.Step(lens, news, heads, kv, D, 16, seed=33, q_scale=0.01)
    got = sqp.paged_attention(**s.gpu(), max_q=max(news), max_len=max(lens)).cpu().double()
    want, tol = s.expected(p_error=2.0 ** -22, rounded=False)
    assert bool(((got - want).abs() <= (want.half().double() - want).abs() + 2 * tol).all())


# ---------------------------------------------------------------- product

FEW = [(1, mt, nt, kw) for mt, nt, kw in ((1, 1, 8), (1, 2, 8), (2, 1, 8), (2, 2, 4), (4, 1, 8))]
TILES = [(2, tile, parts, 0) for tile in range(8) for parts in (1, 2, 3)]  # (tile 7: any K, the others: whole 128, 512 at least)
TWO = [(3, 0, 1, 1), (3, 0, 3, 2), (3, 1, 4, 2), (3, 2, 4, 4)]


def _fits(p, K):
    return p[0] == 1 or (p[1] == 7 if K % 128 or K < 512 else True)


@pytest.fixture
def plan(sqp):
    """Sets the product's plan, automatic again afterwards."""
    f = sqp.lib().sqp_debug_set_mx_plan
    yield f
    f(0, 0, 0, 0)


def _gpu(x, xs, w, ws, kind):
    return mx.typed(x, kind).cuda(), xs.cuda(), w.contiguous().cuda(), ws.cuda()


def _e4m3(v):
    return torch.tensor(v, dtype=torch.float32).to(torch.float8_e4m3fn).view(torch.uint8)


@pytest.mark.parametrize("p", [(1, 1, 1, 8), (1, 4, 1, 8), (2, 0, 1, 0), (2, 3, 1, 0), (2, 5, 1, 0), (2, 7, 1, 0)])
def test_product_cuts_beside_the_largest_of_eight(sqp, plan, p):
    """Two large products that cancel, and a small one somewhere: where it is one of their eight it is cut, to the bit as mx_sums has it, by no more
    than the documented bound; anywhere else in the block, and in other blocks that fp32 tells from the large ones, it is kept whole."""
    K, N = 512, 64
    rows = []
    for a, b in ((0, 1), (5, 6), (66, 70), (511, 504)):
        for j in (2, 3, 7, 8, 15, 31, 32, 67, 72, 95, 505, 507):
            if j in (a, b) or (j // 8 != a // 8 and j // 32 == a // 32 and j < a):
                continue
            for small in (1.875, -1.375, 0.203125, 2.0 ** -5, -2.0 ** -9):
                rows.append((a, b, j, small))
    x = torch.zeros((len(rows), K), dtype=torch.uint8)
    for r, (a, b, j, small) in enumerate(rows):
        x[r, a], x[r, b], x[r, j] = _e4m3(448.0), _e4m3(-448.0), _e4m3(small)
    xs = torch.full((len(rows), K // 32), 127, dtype=torch.uint8)
    big = torch.full((N, K), 2, dtype=torch.uint8)                 # ones
    big[:, [0, 1, 5, 6, 66, 70, 511, 504]] = 7                     # sixes under the large ones
    w = mx.pack(big, "e2m1")
    ws = torch.full((N, K // 32), 127, dtype=torch.uint8)
    print("case cut", p, len(rows), flush=True)
    plan(*p)
    y = sqp.mx_gemm(*_gpu(x, xs, w, ws, "e4m3")).cpu().double()
    cut, _, _, largest = mx_sums.cut_product(x, xs, w, ws)
    exact = mx.values(x, xs, "e4m3") @ mx.values(w, ws, "e2m1").t()
    assert torch.equal(y, cut.half().double())
    assert bool(((y - exact).abs() <= 7 * 2.0 ** -12 * largest).all())
    apart = torch.tensor([a // 8 != j // 8 for a, b, j, small in rows])
    assert torch.equal(y[apart], exact[apart].half().double())
    assert bool((y != exact.half())[~apart].any())


@pytest.mark.parametrize("M,N,K", [(3, 40, 64), (17, 72, 800), (64, 136, 1376), (70, 136, 1920), (300, 200, 2176), (40, 264, 4224)])
def test_product_e4m3_is_that_of_cut_products(sqp, plan, M, N, K):
    """Random codes of every exponent, through the automatic plan and every kernel: within fp32's additions and fp16's rounding of the sum of
    the cut products; K / 32 + 16 additions, each off by 2^-23 at most of what is added so far."""
    g = ref.gen(M + K)
    x = torch.randint(0, 256, (M, K), generator=g).to(torch.uint8)
    x[(x & 127) == 127] = 0  # (the type's two NaN)
    xs = torch.randint(124, 131, (M, K // 32), generator=g).to(torch.uint8)
    w, ws = torch.randint(0, 256, (N, K // 2), generator=g).to(torch.uint8), torch.randint(110, 116, (N, K // 32), generator=g).to(torch.uint8)
    dev = _gpu(x, xs, w, ws, "e4m3")
    want, size, lost, largest = mx_sums.cut_product(x, xs, w, ws, "cuda")
    exact = mx.values(x, xs, "e4m3") @ mx.values(w, ws, "e2m1").t()
    assert bool(((want.cpu() - exact).abs() <= lost.cpu() + 2.0 ** -40 * size.cpu()).all()) and bool((lost <= 7 * 2.0 ** -12 * largest).all())
    sums = K / 32 + 16
    tol = sums * 2.0 ** -23 * size
    tol = tol + 2.0 ** -11 * (want.abs() + tol) + 2.0 ** -25
    for p in [(0, 0, 0, 0)] + FEW + TILES + TWO:
        if not _fits(p, K):
            continue
        print("case cut products", M, N, K, p, flush=True)
        plan(*p)
        err = sqp.mx_gemm(*dev).double() - want
        assert bool((err.abs() <= tol).all()), float((err.abs() / tol).max())
        # the whole: half a step of fp16 each, and independent additions
        assert float(err.norm()) <= 2.0 ** -11 * float(want.norm()) + sums ** 0.5 * 2.0 ** -24 * float(size.norm()) + 2.0 ** -25 * err.numel() ** 0.5


@pytest.mark.parametrize("kind", ["e2m1", "e4m3"])
@pytest.mark.parametrize("M,N,K", [(1, 8, 32), (5, 88, 1376), (33, 136, 96), (64, 1000, 2048), (70, 136, 4128), (140, 528, 4224), (300, 336, 1920), (257, 264, 512)])
def test_product_of_whole_numbers(sqp, plan, M, N, K, kind):
    """Operands whose products and sums fp32 holds exactly in any order (whole numbers up to 15, scales a power of two apart, so that no product is cut):
    the automatic plan and every kernel give the sum rounded once, bit for bit and everywhere."""
    g = ref.gen(M + N + K)
    if kind == "e4m3":
        n = torch.randint(-15, 16, (M, K), generator=g)
        x = n.float().to(torch.float8_e4m3fn).view(torch.uint8)
    else:
        x = torch.randint(0, 256, (M, K // 2), generator=g).to(torch.uint8)
    w = torch.randint(0, 256, (N, K // 2), generator=g).to(torch.uint8)
    xs, ws = [torch.randint(126, 129, (R, K // 32), generator=g).to(torch.uint8) for R in (M, N)]
    X, W = mx.values(x, xs, kind), mx.values(w, ws, "e2m1")
    # multiples of 2^-1 2^-1 2^-1 (e4m3: whole x), sums below 2^24 of them
    assert float((X.abs() @ W.abs().t()).max()) * (16 if kind == "e2m1" else 8) < 2 ** 24
    want = (X @ W.t()).half()
    dev = _gpu(x, xs, w, ws, kind)
    for p in [(0, 0, 0, 0)] + FEW + TILES + TWO:
        if not _fits(p, K):
            continue
        print("case whole numbers", M, N, K, kind, p, flush=True)
        plan(*p)
        y = sqp.mx_gemm(*dev).cpu()
        assert torch.equal(y, want), (p, (y != want).nonzero()[:4].tolist())
