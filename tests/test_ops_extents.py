"""CPU tests of the largest extents of the int8 products: what does not fit is refused before any CUDA call."""
import pytest

from paper_2609_11562_b200 import build as B

B.build()
from paper_2609_11562_b200 import entwine as E  # noqa: E402

P = 1 << 20  # an aligned address that is never followed


@pytest.mark.parametrize("M,N", [(2147418112, 32), (4, 2147483393), (4, 2147483647)])
def test_rows_and_channels_that_pass_32_bits_with_their_tiles_are_refused(M, N):
    """The number of a tile's last channel (of 256) must fit: N + 255 < 2^31."""
    assert E._lib.entwine_gemm_i8(P, 64, P, P, 64, P, None, P, E.DTYPE_BF16, N, M, N, 64, None) == E.ERR_INVALID
    assert E._lib.entwine_gemm_i8_grouped(P, 64, P, P, 64, 64 * N, P, None, P, P, E.DTYPE_BF16, N, M, N, 64, 1, None) == E.ERR_INVALID
    # without rows there is nothing to refuse but the extents themselves
    assert E._lib.entwine_gemm_i8(P, 64, P, P, 64, P, None, P, E.DTYPE_BF16, N, 0, min(N, 2147483392), 64, None) == E.OK
