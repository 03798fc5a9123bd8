"""Refusals of the operators between the linears, without a GPU: the C entries turn bad arguments into errors before anything
is enqueued, the binding names what is wrong."""
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


def test_norm_refusals(L):
    f = L.sqp_add_rmsnorm
    eps = ctypes.c_float(1e-5)
    for at in range(5):
        a = [good] * 5
        a[at] = null
        assert f(4, 1024, a[0], a[1], a[2], eps, a[3], a[4], null) == NULL
        a[at] = odd
        assert f(4, 1024, a[0], a[1], a[2], eps, a[3], a[4], null) == ALIGN
    for M, H in ((0, 1024), (-1, 1024), (4, 0), (4, 1020), (1 << 16, 1 << 15)):
        assert f(M, H, good, good, good, eps, good, good, null) == SHAPE
    for e in (-1e-5, 1.0, float("nan"), float("inf")):
        assert f(4, 1024, good, good, good, ctypes.c_float(e), good, good, null) == ARG
    q = L.sqp_add_rmsnorm_quant
    assert q(4, 1024, 0, good, good, good, eps, good, good, good, null) == ARG
    assert q(4, 1024, 3, good, good, good, eps, good, good, good, null) == ARG
    assert q(4, 1024, 1, good, good, good, eps, good, null, good, null) == NULL
    assert q(4, 1024, 1, good, good, good, eps, good, odd, good, null) == ALIGN


def _write(L, **kw):
    a = dict(T=4, heads=8, kv=2, D=128, type=1, page=16, pages=4, q=good, qs=1024, k=good, ks=256, v=good, vs=256, slots=good, cs=good, pos=good, n=100,
             kc=good, vc=good, ksc=good, vsc=good, out=good, stream=null)
    a.update(kw)
    return L.sqp_kv_cache_write(*a.values())


def _read(L, **kw):
    a = dict(T=4, kv=2, D=128, type=1, page=16, pages=4, slots=good, kc=good, vc=good, ksc=good, vsc=good, k=good, v=good, stream=null)
    a.update(kw)
    return L.sqp_kv_cache_read(*a.values())


def _attend(L, **kw):
    a = dict(T=4, B=2, heads=8, kv=2, D=128, type=1, page=16, pages=4, width=3, max_q=3, max_len=40, scale=0.1, q=good, qs=1024, kc=good, vc=good, ksc=good,
             vsc=good, table=good, ts=3, lens=good, starts=good, out=good, scratch=null, bytes=0, stream=null)
    a.update(kw)
    return L.sqp_paged_attention(*a.values())


def test_cache_refusals(L):
    for f in (_write, _read, _attend):
        for bad in (dict(D=96), dict(D=0), dict(kv=0), dict(page=8), dict(page=24), dict(page=0), dict(page=1 << 17), dict(pages=0), dict(pages=1 << 27),
                    dict(T=-1), dict(kv=1 << 15, page=1 << 9)):
            if f is _attend and "kv" in bad:
                bad = dict(bad, heads=bad["kv"])
            assert f(L, **bad) == SHAPE, (f, bad)
        for bad in (dict(type=3), dict(type=-1)):
            assert f(L, **bad) == ARG
        for bad in (dict(kc=null), dict(vc=null), dict(ksc=null), dict(vsc=null)):
            assert f(L, **bad) == NULL
        for bad in (dict(kc=odd), dict(vc=odd), dict(ksc=odd), dict(vsc=odd)):
            assert f(L, **bad) == ALIGN
    for bad in (dict(k=null), dict(v=null), dict(slots=null), dict(q=null), dict(out=null), dict(pos=null)):
        assert _write(L, **bad) == NULL
    for bad in (dict(k=odd), dict(v=odd), dict(slots=P(0x1002)), dict(q=odd), dict(out=odd), dict(pos=P(0x1001)), dict(cs=odd), dict(qs=1028), dict(ks=260), dict(vs=260)):
        assert _write(L, **bad) == ALIGN
    for bad in (dict(qs=1016), dict(ks=248), dict(vs=248), dict(n=0), dict(heads=-1)):
        assert _write(L, **bad) == SHAPE
    for bad in (dict(slots=null), dict(k=null), dict(v=null)):
        assert _read(L, **bad) == NULL
    for bad in (dict(slots=P(0x1002)), dict(k=odd), dict(v=odd)):
        assert _read(L, **bad) == ALIGN
    assert _write(L, T=0) == 0 and _read(L, T=0) == 0      # nothing is enqueued


def test_attention_refusals(L):
    for bad in (dict(q=null), dict(table=null), dict(lens=null), dict(out=null)):
        assert _attend(L, **bad) == NULL
    for bad in (dict(heads=7), dict(heads=0), dict(B=-1), dict(B=1 << 16), dict(B=0), dict(max_q=-1), dict(max_len=-1), dict(starts=null), dict(width=0), dict(width=1 << 27), dict(width=(1 << 26) + 1, ts=1 << 27),
                dict(ts=2), dict(qs=1016), dict(T=1 << 22)):
        assert _attend(L, **bad) == SHAPE, bad
    for bad in (dict(scale=0.0), dict(scale=-1.0), dict(scale=float("nan")), dict(scale=float("inf"))):
        assert _attend(L, **bad) == ARG
    for bad in (dict(q=odd), dict(out=odd), dict(scratch=odd), dict(qs=1028), dict(table=P(0x1001)), dict(lens=P(0x1002)), dict(starts=P(0x1003))):
        assert _attend(L, **bad) == ALIGN
    assert _attend(L, T=0, B=0) == 0 and _attend(L, T=0) == 0


def test_attention_scratch_size(L):
    """Host arithmetic: nothing for calls without work or with bad arguments, and never more than the partial results of
    every row and part."""
    f = L.sqp_paged_attention_scratch_bytes
    assert f(0, 0, 8, 2, 128, 1, 100) == 0 and f(4, 4, 8, 0, 128, 1, 100) == 0 and f(4, 4, 7, 2, 128, 1, 100) == 0 and f(-4, 4, 8, 2, 128, 1, 100) == 0
    assert f(1, 1, 32, 32, 128, 1, 64) == 0                # too short for parts
    assert f(1 << 20, 1 << 10, 64, 8, 128, 1 << 20, 1 << 30) < 1 << 33


def test_binding_refusals():
    import paper_2312_03788_amd as sqp
    x = torch.zeros((2, 64), dtype=torch.float16)
    c = torch.zeros((2, 1, 16, 64), dtype=torch.float16)
    i = torch.zeros(2, dtype=torch.int32)
    for call, what in ((lambda: sqp.add_rmsnorm(x, x, x[0], 1e-5), "GPU tensor"),
                       (lambda: sqp.add_rmsnorm(x, x[:1], x[0], 1e-5), "residual must have shape"),
                       (lambda: sqp.add_rmsnorm(x, x, x[0, :8], 1e-5), "gamma must have shape"),
                       (lambda: sqp.add_rmsnorm_quant(x, x, x[0], 1e-5, torch.float16), "dtype must be"),
                       (lambda: sqp.kv_cache_write(x.view(2, 1, 64), x.view(2, 1, 64), i, c, c), "GPU tensor"),
                       (lambda: sqp.kv_cache_read(i, c, c[:1]), "v_cache must have shape"),
                       (lambda: sqp.kv_cache_read(i, c.float(), c), "k_cache must be"),
                       (lambda: sqp.paged_attention(x.view(2, 1, 64), c, c, i[None], i[:1]), "GPU tensor")):
        with pytest.raises(sqp.SqpError, match=what):
            call()
