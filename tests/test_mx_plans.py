"""What the library chooses for the microscaled product, by host arithmetic: no GPU."""
import ctypes

import pytest

import mx_plans


@pytest.fixture(scope="module")
def L():
    import paper_2312_03788_amd as m
    return m.lib()


def test_sizes_lead_to_every_form(L):
    """Each of the sizes that test_gpu_mx_plans.py runs leads to the form it stands for: together every form of the few-rows kernel, every tile, K
    parts, and columns left over for a second launch."""
    for M, N, K, kind, want in mx_plans.CHOSEN:
        plan, cols = mx_plans.chosen(L, M, N, K, kind)
        assert plan == want, (M, N, K, kind)
        assert cols == N if plan[0] == "few" or plan[3] is None else 0 < cols < N and cols % 128 == 0
    plans = [c[4] for c in mx_plans.CHOSEN]
    assert {p[1:] for p in plans if p[0] == "few"} == {(1, 1, 8), (1, 2, 8), (2, 1, 8), (2, 2, 4), (4, 1, 8)}
    assert {p[1] for p in plans if p[0] == "tiles"} == set(range(8))
    assert {p[1] for p in plans if p[0] == "tiles" and p[2] > 1} == {2, 3, 4, 5, 6, 7}  # (tiles 0 and 1: no size asks for parts of them)
    assert {p[1] for p in plans if p[0] == "tiles" and p[3] is not None} == {0, 1}


def test_no_such_plan(L):
    p = (ctypes.c_int * 5)()
    for bad in ((0, 64, 64, 4), (4, 60, 64, 4), (4, 64, 40, 2), (4, 64, 64, 1), (1 << 16, 64, 1 << 15, 4)):
        assert L.sqp_debug_mx_plan(*bad, p) != 0
    assert L.sqp_debug_mx_plan(4, 64, 64, 4, None) != 0


def test_scratch_never_grows_large(L):
    """Partial sums are M N floats for each of up to 8 parts, and 96 MiB at most: K is split while the workgroups are no more than one and a half
    times those that run at once, 256 of 256 x 256 sums in the largest tile (1.5 * 256 * 256 * 256 floats), 256 to 1024 of fewer sums in the others."""
    p, most = (ctypes.c_int * 5)(), 0
    sizes = [int(2 ** (i / 2)) for i in range(23)] + [33, 65, 100, 129, 333, 1001]
    for t in (4, 2):
        for M in sizes:
            for N in (8, 64, 136, 512, 1000, 1024, 4096, 5120, 8192, 10240, 16384, 22016, 32768, 44032):
                for K in (32, 96, 512, 1024, 1376, 2048, 4096, 4128, 8192, 11008, 13824, 19712, 22016, 131072):
                    if M * N >= 1 << 31 or M * K >= 1 << 31 or N * K >= 1 << 31:
                        continue
                    n = L.sqp_mx_gemm_scratch_bytes(M, N, K, t)
                    assert L.sqp_debug_mx_plan(M, N, K, t, p) == 0
                    parts = p[2] if p[0] == 2 else 1
                    assert 1 <= parts <= 8 and n == (4 * M * N * parts if parts > 1 else 0) and n <= 96 << 20, (M, N, K, t)
                    most = max(most, n)
    assert most >= 32 << 20  # (the sizes do reach for it)
