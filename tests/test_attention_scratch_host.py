"""Scratch of the attention over the paged cache (CPU: host arithmetic alone)."""
import pytest


@pytest.fixture(scope="module")
def scratch():
    import paper_2312_03788_amd as sqp
    return sqp.lib().sqp_paged_attention_scratch_bytes


@pytest.mark.parametrize("T,B,heads,kv,D,max_q,max_len", [
    (16, 16, 64, 8, 128, 1, 8192), (1, 1, 32, 32, 128, 1, 32768), (4, 4, 32, 8, 64, 1, 1 << 20), (3, 1, 5, 5, 64, 3, 5000), (40, 1, 8, 1, 128, 40, 1 << 30),
    (2063, 16, 64, 8, 128, 2048, 16384), (2056, 9, 8, 1, 128, 2048, 16384), (16385, 9, 16, 1, 128, 2048, 32768), (60, 12, 8, 2, 128, 40, 3000)])
def test_scratch_that_splits(scratch, T, B, heads, kv, D, max_q, max_len):
    """Calls that are split: at most 64 partial results, of D + 4 floats, for every row; and where single tokens lie beside chunks, at most
    what the places of the chip can be given: 512 parts of 16 rows (two workgroups per compute unit), and 512 of 128."""
    n = scratch(T, B, heads, kv, D, max_q, max_len)
    partial = (D + 4) * 4
    assert 0 < n and n % partial == 0
    assert n <= (512 * 16 + 512 * 128) * partial
    if max_q == 1:
        assert n <= T * heads * 64 * partial


@pytest.mark.parametrize("T,B,heads,kv,max_q,max_len,most", [(2063, 16, 64, 8, 2048, 16384, 5 << 20), (16385, 9, 16, 1, 2048, 32768, 5 << 20)])
def test_scratch_of_single_tokens_beside_chunks(scratch, T, B, heads, kv, max_q, max_len, most):
    """Chunks that are not split have no partial results: the call takes what its single tokens need."""
    assert 0 < scratch(T, B, heads, kv, 128, max_q, max_len) <= most
