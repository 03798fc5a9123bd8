"""Operators on microscaled numbers where inputs are as other programs may have written them, and forms that only long prompts take."""
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
    f = sqp.lib().sqp_debug_set_mx_plan
    yield f
    f(0, 0, 0, 0)


def test_dequantise_codes_that_are_nan(sqp):
    """The two e4m3 codes that are NaN: themselves alone, not their block."""
    codes, scales = torch.full((2, 96), 0x38, dtype=torch.uint8), torch.full((2, 3), 127, dtype=torch.uint8)
    codes[0, 3], codes[1, 40] = 0x7f, 0xff
    back = sqp.mx_dequantize(codes.cuda().view(torch.float8_e4m3fn), scales.cuda()).cpu()
    assert torch.equal(back.isnan().nonzero(), torch.tensor([[0, 3], [1, 40]])) and bool((back.nan_to_num(1.0) == 1).all())


PLANS = [(0, 0, 0, 0), (1, 1, 1, 8), (1, 4, 1, 8), (2, 0, 1, 0), (2, 3, 2, 0), (2, 6, 1, 0), (2, 7, 1, 0)]


def _fits(p, K):
    return p[0] != 2 or p[1] == 7 or (K % 128 == 0 and K >= 512)  # (tile 7 alone takes any K)


@pytest.mark.parametrize("M,K,p", [(M, K, p) for M, K in ((3, 64), (3, 1312), (200, 544), (200, 1152)) for p in PLANS if _fits(p, K)])
def test_product_of_codes_that_are_nan(sqp, plan, M, K, p):
    """An e4m3 code that is NaN, the last of its row (which is read again for k past the end): its row is NaN, no other is."""
    N = 72
    g = ref.gen(K)
    x = torch.randint(-7, 8, (M, K), generator=g).float().to(torch.float8_e4m3fn).view(torch.uint8)
    w = torch.randint(0, 256, (N, K // 2), generator=g).to(torch.uint8)
    w[5] = 0  # (zeros by NaN are NaN)
    xs, ws = [torch.full((R, K // 32), 127, dtype=torch.uint8) for R in (M, N)]
    want = (mx.values(x, xs, "e4m3") @ mx.values(w, ws, "e2m1").t()).half()
    for code in (0x7f, 0xff):
        x[1, K - 1] = code
        plan(*p)
        print("case NaN code", M, K, p, code, flush=True)
        y = sqp.mx_gemm(mx.typed(x, "e4m3").cuda(), xs.cuda(), w.cuda(), ws.cuda()).cpu()
        others = torch.arange(M) != 1
        assert bool(y[1].isnan().all()) and torch.equal(y[others], want[others])


@pytest.mark.parametrize("kind", ["e2m1", "e4m3"])
@pytest.mark.parametrize("M,N,K", [(4, 40, 1056), (40, 72, 4096), (150, 136, 2048)])
def test_product_of_far_scales(sqp, plan, M, N, K, kind):
    """Scale bytes over their whole range, 2^-127 to 2^127, where a block's two make up for each other: sums that fp32 holds exactly, bit for bit."""
    g = ref.gen(K + M)
    x = torch.randint(-15, 16, (M, K), generator=g).float().to(torch.float8_e4m3fn).view(torch.uint8) if kind == "e4m3" else torch.randint(0, 256, (M, K // 2), generator=g).to(torch.uint8)
    w = torch.randint(0, 256, (N, K // 2), generator=g).to(torch.uint8)
    middle = torch.randint(1, 254, (1, K // 32), generator=g)
    middle[0, :2] = torch.tensor([1, 253])
    xs = (middle + torch.randint(-1, 2, (M, K // 32), generator=g)).to(torch.uint8)
    ws = (254 - middle + torch.randint(-1, 2, (N, K // 32), generator=g)).to(torch.uint8)
    assert int(xs.min()) == 0 and int(xs.max()) == 254
    X, W = mx.values(x, xs, kind), mx.values(w, ws, "e2m1")
    assert float((X.abs() @ W.abs().t()).max()) * 16 < 2 ** 24  # (multiples of 2^-4 at least)
    want = (X @ W.t()).half()
    for p in [(0, 0, 0, 0), (1, 1, 1, 8), (1, 4, 1, 8)] + [(2, t, n, 0) for t in range(8) for n in (1, 2)]:
        if not _fits(p, K):
            continue
        print("case far scales", M, N, K, kind, p, flush=True)
        plan(*p)
        assert torch.equal(sqp.mx_gemm(mx.typed(x, kind).cuda(), xs.cuda(), w.cuda(), ws.cuda()).cpu(), want), p


@pytest.mark.parametrize("D", [128, 64])
@pytest.mark.parametrize("T,length", [(2050, 2050), (2047, 3001)])
def test_attention_of_long_prompts(sqp, T, length, D):
    """Enough rows for tiles of 256 of them (twice as many as compute units): the bits of the same attention over an fp16 cache that holds what the blocks
    stand for (exact: no value is beyond fp16 or below its steps), whose own tests hold it to the formula."""
    heads, kv, page = 64, 8, 64
    assert -(-T * (heads // kv) // 256) * kv >= 2 * 256
    g = ref.gen(T)
    pages = -(-length // page) + 2
    qkv = mx.random_rows(g, length, (heads + 2 * kv) * D, 2).view(length, -1, D).cuda()
    c = [torch.zeros((pages, kv, page, n), dtype=torch.uint8, device="cuda") for n in (D // 2, D // 2, D // 32, D // 32)]
    order = torch.randperm(pages, generator=g).int()
    slots = (order.long()[torch.arange(length) // page] * page + torch.arange(length) % page).int().cuda()
    q = sqp.kv_cache_write(qkv[:, heads: heads + kv], qkv[:, heads + kv:], slots, *c, q=qkv[:, :heads])[-T:] * 0.25
    half = [torch.zeros((pages, kv, page, D), dtype=torch.float16, device="cuda") for _ in range(2)]
    sqp.kv_cache_write(*sqp.kv_cache_read(slots, *c), slots, *half)
    table, lens, starts = order[None].cuda(), torch.tensor([length], dtype=torch.int32).cuda(), torch.tensor([0, T], dtype=torch.int32).cuda()
    a = sqp.paged_attention(q, c[0], c[1], table, lens, starts, c[2], c[3], max_q=T, max_len=length)
    b = sqp.paged_attention(q, *half, table, lens, starts, max_q=T, max_len=length)
    assert bool(a.isfinite().all()) and torch.equal(a, b)
