"""Refusals of the operators on microscaled numbers, without a GPU: the C entries turn bad arguments into errors before anything is
enqueued, the binding names what is wrong."""
import ctypes

import pytest
import torch


@pytest.fixture(scope="module")
def L():
    import paper_2312_03788_amd as sqp
    return sqp.lib()


P = ctypes.c_void_p
good, odd, null = P(0x1000), P(0x1008), P(0)
NULL, SHAPE, ALIGN, ARG = -1, -2, -3, -4
E4M3, E2M1 = 2, 4


@pytest.mark.parametrize("name", ["sqp_mx_quantize", "sqp_mx_dequantize"])
def test_rows_refusals(L, name):
    f = getattr(L, name)
    for at in range(3):
        a = [good] * 3
        a[at] = null
        assert f(4, 64, E2M1, *a, null) == NULL
        a[at] = odd
        assert f(4, 64, E2M1, *a, null) == ALIGN
    for R, K in ((0, 64), (-1, 64), (4, 0), (4, 48), (4, 8), (1 << 16, 1 << 15)):
        assert f(R, K, E4M3, good, good, good, null) == SHAPE
    for t in (0, 1, 3, 5, -1):
        assert f(4, 64, t, good, good, good, null) == ARG


def test_weight_refusals(L):
    f = L.sqp_mx_quantize_weight
    for at in range(3):
        a = [good] * 3
        a[at] = null
        assert f(64, 64, *a, null) == NULL
        a[at] = odd
        assert f(64, 64, *a, null) == ALIGN
    for N, K in ((0, 64), (64, 0), (64, 40), (12, 64), (1 << 16, 1 << 15)):
        assert f(N, K, good, good, good, null) == SHAPE


def test_norm_refusals(L):
    f = L.sqp_add_rmsnorm_mx
    eps = ctypes.c_float(1e-5)
    for at in range(6):
        a = [good] * 6
        a[at] = null
        assert f(4, 1024, E2M1, a[0], a[1], a[2], eps, a[3], a[4], a[5], null) == NULL
        a[at] = odd
        assert f(4, 1024, E2M1, a[0], a[1], a[2], eps, a[3], a[4], a[5], null) == ALIGN
    for M, H in ((0, 1024), (4, 0), (4, 1032), (1 << 16, 1 << 15)):
        assert f(M, H, E4M3, good, good, good, eps, good, good, good, null) == SHAPE
    for t in (0, 1, 3):
        assert f(4, 1024, t, good, good, good, eps, good, good, good, null) == ARG
    for e in (-1e-5, 1.0, float("nan"), float("inf")):
        assert f(4, 1024, E2M1, good, good, good, ctypes.c_float(e), good, good, good, null) == ARG


def _product(L, **kw):
    a = dict(M=4, N=64, K=64, type=E2M1, silu=0, x=good, xs=good, w=good, ws=good, y=good, scratch=null, bytes=0, stream=null)
    a.update(kw)
    return L.sqp_mx_gemm(*a.values())


def test_product_refusals(L):
    for name in ("x", "xs", "w", "ws", "y"):
        assert _product(L, **{name: null}) == NULL and _product(L, **{name: odd}) == ALIGN
    assert _product(L, scratch=odd, bytes=64) == ALIGN
    for bad in (dict(M=0), dict(N=0), dict(K=0), dict(M=-1), dict(N=60), dict(K=48), dict(N=72, silu=1), dict(M=1 << 16, K=1 << 15), dict(N=1 << 16, K=1 << 15),
                dict(M=1 << 16, N=1 << 15)):
        assert _product(L, **bad) == SHAPE, bad
    for t in (0, 1, 3):
        assert _product(L, type=t) == ARG


def test_product_scratch_size(L):
    """Host arithmetic: nothing for bad shapes, whole sums per part otherwise, and never more than 64 MB more than a small output needs."""
    f = L.sqp_mx_gemm_scratch_bytes
    for bad in ((0, 64, 64, E2M1), (4, 60, 64, E2M1), (4, 64, 40, E2M1), (4, 64, 64, 1)):
        assert f(*bad) == 0
    for M in (1, 16, 33, 100, 333, 1000, 4096):
        for N, K in ((512, 512), (4096, 4096), (5120, 13824), (44032, 8192), (8192, 22016)):
            for t in (E2M1, E4M3):
                n = f(M, N, K, t)
                assert n % (4 * M * N) == 0 and n <= 16 * 4 * M * N


def test_cache_refusals(L):
    def write(**kw):
        a = dict(T=4, heads=8, kv=2, D=128, type=E2M1, page=16, pages=4, q=good, qs=1024, k=good, ks=256, v=good, vs=256, slots=good, cs=good, pos=good, n=100,
                 kc=good, vc=good, ksc=good, vsc=good, out=good, stream=null)
        a.update(kw)
        return L.sqp_kv_cache_write(*a.values())
    assert write(T=0) == 0
    assert write(ksc=null) == NULL and write(vsc=null) == NULL and write(ksc=odd) == ALIGN and write(D=96) == SHAPE and write(type=3) == ARG


def test_binding_refusals():
    import paper_2312_03788_amd as sqp
    x = torch.zeros((2, 64), dtype=torch.float16)
    c, s = torch.zeros((2, 32), dtype=torch.uint8), torch.zeros((2, 2), dtype=torch.uint8)
    kc, ks = torch.zeros((2, 1, 16, 32), dtype=torch.uint8), torch.zeros((2, 1, 16, 2), dtype=torch.uint8)
    i = torch.zeros(2, dtype=torch.int32)
    t = x.view(2, 1, 64)
    for call, what in ((lambda: sqp.mx_quantize(x), "GPU tensor"),
                       (lambda: sqp.mx_quantize(x, torch.int8), "dtype must be"),
                       (lambda: sqp.mx_quantize(x[:, :40]), "blocks of 32"),
                       (lambda: sqp.mx_quantize(x, out=(c[:1], s)), "codes must have shape"),
                       (lambda: sqp.mx_quantize_weight(x[:, :8]), "blocks of 32"),
                       (lambda: sqp.mx_dequantize(c, s[:, :1]), "scales must have shape"),
                       (lambda: sqp.mx_dequantize(x, s), "must be"),
                       (lambda: sqp.mx_gemm(c, s, c, s), "GPU tensor"),
                       (lambda: sqp.mx_gemm(c, s, c[:, :16], s[:, :1]), "disagree on K"),
                       (lambda: sqp.mx_gemm(c, s, c.repeat(1, 2).view(torch.float8_e4m3fn), s), "must be e2m1"),
                       (lambda: sqp.mx_gemm(c, s, c, s, out=x), "out must have shape"),
                       (lambda: sqp.mx_gemm_silu_mul(c, s, c, s, out=x[:, :2].contiguous()), "out must have shape"),
                       (lambda: sqp.add_rmsnorm_mx(x, x[:1], x[0], 1e-5), "residual must have shape"),
                       (lambda: sqp.add_rmsnorm_mx(x, x, x[0], 1e-5, torch.float16), "dtype must be"),
                       (lambda: sqp.kv_cache_write(t, t, i, kc, kc), "GPU tensor"),
                       (lambda: sqp.kv_cache_read(i, kc, kc, ks), "GPU tensor"),
                       (lambda: sqp.paged_attention(t, kc, kc, i[None], i[:1]), "GPU tensor")):
        with pytest.raises(sqp.SqpError, match=what):
            call()


def test_tensors_of_another_device(monkeypatch):
    """Every tensor of a call has to be on the current device: the one that is not is named."""
    import types

    import paper_2312_03788_amd as sqp
    from paper_2312_03788_amd import binding
    monkeypatch.setattr(binding.torch.cuda, "current_device", lambda: 1)
    on = lambda i: types.SimpleNamespace(device=torch.device("cuda", i))
    binding._on_current(x=on(1), out=None, w=on(1))
    with pytest.raises(sqp.SqpError, match="w must be on the current device \\(1\\), not on cuda:0"):
        binding._on_current(x=on(1), out=None, w=on(0))
