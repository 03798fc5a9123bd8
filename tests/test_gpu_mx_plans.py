"""The microscaled product through the plans that the library chooses by itself, every output of every call."""
import pytest
import torch

import layer_ref as ref
import mx_plans
import mx_ref as mx

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def sqp():
    import paper_2312_03788_amd as m
    m.lib()
    return m


def _whole(g, M, N, K, kind):
    """Operands whose products and sums fp32 holds exactly in any order: x whole numbers up to 7 (e4m3) or any e2m1 code, scales of 1 or 2."""
    if kind == "e4m3":
        x = torch.randint(-7, 8, (M, K), generator=g).float().to(torch.float8_e4m3fn).view(torch.uint8)
    else:
        x = torch.randint(0, 256, (M, K // 2), generator=g).to(torch.uint8)
    w = torch.randint(0, 256, (N, K // 2), generator=g).to(torch.uint8)
    xs, ws = [torch.randint(127, 129, (R, K // 32), generator=g).to(torch.uint8) for R in (M, N)]
    assert 7 * 6 * 4 * K * 4 < 2 ** 24  # magnitudes, in multiples of 2^-2
    return x, xs, w, ws


def _sums(x, xs, w, ws, kind):
    """The product in 64 bits, on the GPU, in pieces of columns."""
    X = mx.values(x, xs, kind).cuda()
    return torch.cat([X @ mx.values(w[n: n + 8192], ws[n: n + 8192], "e2m1").cuda().t().contiguous() for n in range(0, w.shape[0], 8192)], 1)


@pytest.mark.parametrize("silu", [False, True])
@pytest.mark.parametrize("M,N,K,kind,want", mx_plans.CHOSEN)
def test_every_chosen_plan(sqp, M, N, K, kind, want, silu):
    """The plan is the one that the size stands for; the sums are exact, so that every output is the definition's rounded once, and what another plan
    gives, bit for bit; with SiLU(gate) * up, within that function's own error of it (as in mx_ref.product) and the other plan's bits."""
    print("case chosen", M, N, K, kind, want, silu, flush=True)
    L = sqp.lib()
    N += N % 16 if silu else 0  # (pairs of gate and up)
    plan, cols = mx_plans.chosen(L, M, N, K, kind)
    assert plan == want
    ops = _whole(ref.gen(M + N + K), M, N, K, kind)
    x, xs, w, ws = ops
    dev = mx.typed(x, kind).cuda(), xs.cuda(), w.cuda(), ws.cuda()
    f = sqp.mx_gemm_silu_mul if silu else sqp.mx_gemm
    y = f(*dev)
    s = _sums(*ops, kind)
    if silu:
        gate, up = s[:, 0::2], s[:, 1::2]
        v = gate * torch.sigmoid(gate) * up
        big = v.abs() > 65504
        # (the exponential's argument is a product rounded in fp32, times a rounded constant: |gate| 2^-23)
        off = (2.0 ** -20 + 2.0 ** -23 * gate.abs()) * v.abs()
        tol = off + 2.0 ** -11 * (v.abs() + off) + 2.0 ** -25
        assert bool(((y.double() - v).abs() <= tol)[~big].all()) and bool((y[big].abs() >= 65472).all())
    else:
        assert torch.equal(y, s.half())
    other = (2, 7, 1, 0) if want[:2] != ("tiles", 7) else (1, 4, 1, 8)
    try:
        L.sqp_debug_set_mx_plan(*other)
        assert torch.equal(f(*dev), y)
    finally:
        L.sqp_debug_set_mx_plan(0, 0, 0, 0)


@pytest.mark.parametrize("kind", ["e2m1", "e4m3"])
@pytest.mark.parametrize("silu", [False, True])
def test_columns_in_two_launches_are_those_of_one(sqp, kind, silu):
    """Whatever tiles the first columns and the others take: the bits of one launch of either (all tiles add a row's k in the same order only
    for some types, so the sums are exact ones)."""
    M, N, K = 200, 656, 1152
    L = sqp.lib()
    x, xs, w, ws = _whole(ref.gen(9), M, N, K, kind)
    dev = mx.typed(x, kind).cuda(), xs.cuda(), w.cuda(), ws.cuda()
    f = sqp.mx_gemm_silu_mul if silu else sqp.mx_gemm
    try:
        for first, other, cols in ((0, 1, 1), (0, 3, 2), (1, 4, 2), (2, 4, 4), (1, 2, 1), (0, 2, 5)):
            print("case two launches", kind, silu, first, other, cols, flush=True)
            got = []
            for p in ((3, first, other, cols), (2, first, 1, 0), (2, other, 1, 0)):
                L.sqp_debug_set_mx_plan(*p)
                got.append(f(*dev))
            assert torch.equal(got[0], got[1]) and torch.equal(got[0], got[2])
    finally:
        L.sqp_debug_set_mx_plan(0, 0, 0, 0)
