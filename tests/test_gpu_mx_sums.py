"""How the operators on microscaled numbers add: what is rounded, and what is not."""
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
