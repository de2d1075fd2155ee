"""Sizes of the gated projections whose tiles a launch cannot count, refused on the host."""
import os

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
LIB = os.path.join(ROOT, "paper_2507_03312_amd", "libmpx.so")
pytestmark = pytest.mark.skipif(not os.path.exists(LIB), reason="libmpx.so not built")

p = 256  # never dereferenced


# direct tiles, register-staged ones, those of any rows
@pytest.mark.parametrize("M, N, K", [((1 << 31) - 1, 1 << 24, 64), (1 << 30, 1 << 12, 64), ((1 << 31) - 1, 128, 64),
                                     ((1 << 31) - 1, 1 << 10, 72), ((1 << 31) - 1, 33, 1), ((1 << 31) - 1, 1, 1)])
def test_sizes_past_a_launch(M, N, K):
    from paper_2507_03312_amd import binding as mx
    with pytest.raises(mx.MPXError, match="too large"):
        mx.mpx_gated_fwd(p, p, None, p, None, M, N, K, mx.MPX_BF16, mx.MPX_ACT_SILU, 0)
    with pytest.raises(mx.MPXError, match="too large"):   # N x K in the backward's terms: K x N
        mx.mpx_linear_bwd_gated(None, p, p, p, mx.MPX_ACT_SILU, p, None, None, M, K, 2 * N, mx.MPX_BF16, None, 0, None,
                                0)
