"""Size limits of the row-wise calls that the host can see: refused with the documented status before anything is launched (no
GPU needed)."""
import pytest

from test_rows_refusals import UNSUPPORTED, linear, qlinear


@pytest.mark.parametrize("N", [2 ** 31 - 511, 2 ** 31 - 200, 2 ** 31 - 1])
def test_output_channels_whose_tile_count_leaves_32_bits(N):
    """N + 255 wraps near 2^31; such a weight matrix (16 bytes a row) would fit the memory."""
    assert qlinear(N=N, ldy=N, K=16, lda=16, ldw=16) == UNSUPPORTED
    assert linear(N=N, ldy=N, C=16, ldx=16, ldw=16, ws_bytes=1 << 40) == UNSUPPORTED
