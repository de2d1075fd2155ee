"""Statistics of the linear cross entropy at their edges: rows with a NaN, among others or
alone."""
import numpy as np
import pytest

from tests.gpu_util import HAVE_GPU, to_host

pytestmark = [pytest.mark.gpu, pytest.mark.skipif(not HAVE_GPU, reason="no GPU")]

if HAVE_GPU:
    import torch
    from paper_2507_03312_amd import binding as mx
    TYPES = {"f16": torch.float16, "bf16": torch.bfloat16}

FMTS = ["f16", "bf16"]
SCALE = 2.0 ** 11


def _s():
    return torch.cuda.current_stream().cuda_stream


def _dev(a, fmt):
    return torch.from_numpy(np.ascontiguousarray(a, np.float32)).to(TYPES[fmt]).cuda()


def _run(x, w, b, t, fmt, g=None, loss=True):
    """loss, stats and, with cotangents, dX, dW, db and the count of the non-finite ones."""
    (M, K), V = x.shape, len(w)
    xt, wt, bt = _dev(x, fmt), _dev(w, fmt), None if b is None else _dev(b, fmt)
    tt = torch.from_numpy(np.asarray(t, np.int32)).cuda()
    lo, st = torch.full((M,), -7.0, device="cuda"), torch.full((M, 2), -7.0, device="cuda")
    ws = torch.empty(max(mx.mpx_linear_ce_fwd_workspace(M, V, K), mx.mpx_linear_ce_bwd_workspace(M, V, K)),
                     dtype=torch.uint8, device="cuda")
    at = None if bt is None else bt.data_ptr()
    mx.mpx_linear_ce_fwd(xt.data_ptr(), wt.data_ptr(), at, tt.data_ptr(), M, V, K,
                         lo.data_ptr() if loss else None, st.data_ptr(), None, mx.DTYPES[fmt], ws.data_ptr(),
                         ws.numel(), _s())
    if g is None:
        return to_host(lo), to_host(st)
    outs = [torch.full(s, -7.0, dtype=TYPES[fmt], device="cuda") for s in ((M, K), (V, K), (V,))]
    gt = torch.from_numpy(np.asarray(g, np.float32)).cuda()
    state = torch.tensor([SCALE, 0.0, 0.0, 2.0, 1.0, 2.0 ** 100], device="cuda")
    n = torch.zeros(1, dtype=torch.int32, device="cuda")
    mx.mpx_linear_ce_bwd(xt.data_ptr(), wt.data_ptr(), at, tt.data_ptr(), M, V, K, st.data_ptr(), gt.data_ptr(),
                         state.data_ptr(), *(o.data_ptr() for o in outs), mx.DTYPES[fmt], ws.data_ptr(), ws.numel(),
                         n.data_ptr(), _s())
    return (to_host(lo), to_host(st), *map(to_host, outs), int(n))


# tiles of 32 and 64 rows and more; whole and ragged ones, direct, register-staged and of < 8
NAN_SHAPES = [(5, 128, 64), (5, 200, 64), (40, 256, 64), (40, 201, 64), (150, 1000, 64), (9, 130, 40), (70, 65, 40),
              (40, 100, 5), (600, 4100, 72)]


@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("shape", NAN_SHAPES, ids=lambda s: "x".join(map(str, s)))
def test_a_row_of_nan_logits(fmt, shape):
    """A NaN in a row of X makes all its logits NaN: its statistics and loss are NaN, not
    those of a row that is masked whole, and no other row's change."""
    M, V, K = shape
    rng = np.random.default_rng(M + V)
    x, w = rng.normal(0, 1, (M, K)), rng.normal(0, K ** -0.5, (V, K))
    t = rng.integers(0, V, M).astype(np.int32)
    lo, st = _run(x, w, None, t, fmt)
    assert np.isfinite(lo).all() and np.isfinite(st).all()
    bad = [2, M - 1]
    x[2, 3] = x[M - 1, 0] = np.nan
    lo2, st2, dx, dw, db, n = _run(x, w, None, t, fmt, np.full(M, 1.0 / M))
    for a, b in ((lo, lo2), (st, st2)):
        assert np.isnan(b[bad]).all()
        assert np.array_equal(np.delete(a, bad, axis=0), np.delete(b, bad, axis=0))
    only = _run(x, w, None, t, fmt, loss=False)
    assert (only[0] == -7.0).all() and np.array_equal(only[1], st2, equal_nan=True)
    assert np.isnan(dx[bad]).all() and np.isfinite(np.delete(dx, bad, axis=0)).all()
    assert np.isnan(dw).all() and np.isnan(db).all() and n == dw.size + db.size


@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("shape", [(5, 128, 64), (40, 201, 64), (9, 130, 40)], ids=lambda s: "x".join(map(str, s)))
def test_one_nan_logit_among_masked_ones(fmt, shape):
    """Every column masked but one whose bias is NaN: NaN, whatever the targets, not the
    infinite loss of a masked target; rows without a target have a loss of 0."""
    M, V, K = shape
    rng = np.random.default_rng(V)
    x, w = rng.normal(0, 1, (M, K)), rng.normal(0, K ** -0.5, (V, K))
    b = np.full(V, -np.inf)
    b[V - 2] = np.nan
    t = np.arange(M, dtype=np.int32) % (V - 2)
    t[0], t[1] = V - 2, -1
    lo, st, dx, dw, db, _ = _run(x, w, b, t, fmt, np.full(M, 1.0 / M))
    assert lo[1] == 0 and np.isnan(np.delete(lo, 1)).all() and np.isnan(st).all()
    assert np.isnan(dx).all() and np.isnan(dw).all() and np.isnan(db).all()
