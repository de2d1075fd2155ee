"""Workspaces of the linear cross entropy, on the host."""
import os

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
LIB = os.path.join(ROOT, "paper_2507_03312_amd", "libmpx.so")
pytestmark = pytest.mark.skipif(not os.path.exists(LIB), reason="libmpx.so not built")

SIZES = [(10, 64), (16, 224), (40, 7), (128, 3), (170, 64), (1000, 384), (1003, 320), (4099, 75), (20011, 64), (65537, 768),
         (131072, 768), (131072, 183), (530003, 40), (1 << 20, 1024), (50257, 2048), (1 << 24, 64)]


@pytest.mark.parametrize("V, K", SIZES, ids=lambda v: str(v))
def test_workspaces_never_fall_as_rows_grow(V, K):
    """A buffer for the largest batch serves a smaller last one, which other tiles and splits
    may take."""
    from paper_2507_03312_amd import binding as mx
    most = min(1 << 20, (1 << 36) // V, (1 << 33) // K - V)
    rows = sorted({m for m in [*range(1, 1600), *range(1600, 20000, 61), *(1 << i for i in range(21)),
                               *((1 << i) + 1 for i in range(20))] if m <= most})
    for f in (mx.mpx_linear_ce_fwd_workspace, mx.mpx_linear_ce_bwd_workspace):
        sizes = [f(m, V, K) for m in rows]
        falls = [(a, b) for a, b, x, y in zip(rows, rows[1:], sizes, sizes[1:]) if y < x]
        assert not falls, (f.__name__, falls[:3])


@pytest.mark.parametrize("M, V, K", [(128, 131072, 768), (4096, 131072, 768), (65536, 65536, 768), (65536, 1280, 64),
                                     (1 << 20, 65536, 64), (1 << 20, 512, 64)])
def test_a_piece_is_what_the_workspace_holds_of_the_logits(M, V, K):
    """dz of 128 MiB or 256 columns, 256 columns more in the last piece; beside it dX's sums
    (float32) and the bounded ones of splits."""
    from paper_2507_03312_amd import binding as mx
    rows = max(M, 256)   # up to 128 rows two sets of them
    columns = max((64 << 20) // rows, 256) + 256
    splits = 4 * (3 * 768 * 64 + 3 * 512 * 128) * 128 + (64 << 20)   # of dX and dW; db's
    assert mx.mpx_linear_ce_bwd_workspace(M, V, K) <= 2 * rows * min(V, columns) + 4 * rows * K + splits + (1 << 20)
