"""Scratch of the feed-forward blocks' backward passes: host arithmetic."""
import pytest

from paper_2305_02299_amd import binding as B_


@pytest.mark.parametrize("dtype,elem", [(B_.F32, 4), (B_.BF16, 2)])
@pytest.mark.parametrize("ablated", [0, 1])
@pytest.mark.parametrize("n", [768, 3072, 4096, 16384])
def test_whole_numbers_of_stages_take_no_more_chunks_of_rows(n, ablated, dtype, elem):
    """Widths that need no padding are cut into as many chunks of rows as the widths beside them: a column more of the sums, four bytes a chunk, is all that they take.  B is where a pass over fewer columns would take fewer
    rows to a chunk, d_in beyond what cuts K into parts, whose sums would stand beside these."""
    B, d_in = 2048 * 16384 // n, 65536
    at, below = (B_.srigl_structured_bwd_workspace_bytes(B, d_in, k, k + ablated, dtype) for k in (n, n - 1))
    chunks = -(-B // 16)   # (two rows to a thread at least, eight side by side)
    assert 0 <= at - below <= 4 * chunks + 256
    assert B * n * elem < at < B * n * elem + 4 * (n + 1) * chunks + 512
