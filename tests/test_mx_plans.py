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
