"""Statistics of the linear cross entropy at their edges: rows with a NaN, among others or
alone, and rows whose largest logit is nearly all of the sum."""
import numpy as np
import pytest

from oracle import linear_ce
from tests.gpu_util import HAVE_GPU, assert_within, to_host, ulp

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


# logits of the largest column: whole products of two half values
TOPS = [0.0, 0.40625, 10.25, 20.5, 31.75, 40.25, 55.5, 81.0, 127.0, 250.0, 1000.0]


@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("bias", [False, True], ids=["", "bias"])
@pytest.mark.parametrize("shape", [(11, 128, 64), (11, 201, 64), (33, 1000, 64), (44, 130, 40), (22, 100, 5),
                                   (550, 4100, 72)], ids=lambda s: "x".join(map(str, s)))
def test_confident_rows_are_exact(fmt, bias, shape):
    """Rows whose other logits lie 32 below the largest: 4100 e^-32 is 5e-11, less than half a
    float32 step of 1, so S is 1, ln S and the target's loss exactly 0, wherever
    the largest lies; the other columns' losses are their exact distance, and the target's
    gradient is that of p = 1: nothing."""
    M, V, K = shape
    x, w = np.zeros((M, K)), np.zeros((V, K))
    x[:, 0] = np.resize(TOPS, M)
    x[:, 1] = 32.0
    w[:, 0] = 1.0
    w[:, 1] = -1.0
    top = V // 3
    w[top, 1] = 0.0
    b = np.full(V, 0.5) if bias else None
    m = x[:, 0] + (0.5 if bias else 0.0)
    lo, st, dx, dw, db, n = _run(x, w, b, np.full(M, top), fmt, np.full(M, 1.0))
    assert np.array_equal(st[:, 0], m.astype(np.float32))
    assert (st[:, 1] == 0).all() and (lo == 0).all() and n == 0
    # p of the others, f e^-32 each, is all there is: 0 for float16, whose dz 2^14 e^-32 is below its
    # least value
    p = SCALE * np.exp(-32.0)
    if fmt == "f16":
        assert (db == 0).all() and (dx == 0).all()
    else:
        assert db[top] == 0
        other = np.delete(db, top)
        # one rounding of each dz and one of the sum (their product 2^-16), the exponent's of
        # 46 2^-24, two of its constant and exp2: below 2^-17, and the sum's M
        assert (np.abs(other - M * p) <= M * p * (2.0 ** -7 + 2.0 ** -16 + 2.0 ** -17 + M * 2.0 ** -24)).all()
    lo, _ = _run(x, w, b, np.full(M, (top + 1) % V), fmt)
    assert (lo == 32).all()


@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("gap", [1.0, 4.0, 8.0, 12.0])
def test_nearly_certain_targets(fmt, gap):
    """Two columns, all others masked, the target's logit `gap` above the other's: S is one float32
    sum, 1 + e^-gap.  Its exponential is off by gap 2^-22 + 2^-22 of itself, the sum by half a
    step, ln S by that and 2^-22 of itself; p by its exponent, exp2 and one rounding: 2^-22.
    Neither ln S, the loss nor 1 - p is ever below 0."""
    M, V, K = len(TOPS), 150, 64
    x, w = np.zeros((M, K)), np.zeros((V, K))
    x[:, 0], x[:, 1] = TOPS, gap
    w[:, 0] = 1.0
    w[9, 1] = -1.0
    b = np.full(V, -np.inf)
    b[3] = b[9] = 0.0
    want = np.log1p(np.exp(-gap))
    off = np.exp(-gap) * (gap + 1) * 2.0 ** -22 + 2.0 ** -24 * 1.37 + want * 2.0 ** -22
    for row in range(M):
        lo, st, dx, dw, db, n = _run(x[row:row + 1], w, b, [3], fmt, [1.0])
        assert st[0, 0] == TOPS[row] and 0 <= st[0, 1] == lo[0]
        assert abs(st[0, 1] - want) <= off
        p, err = np.exp(-want), off + 2.0 ** -22
        ref = SCALE * np.array([p - 1, 1 - p])
        got = db[[3, 9]]
        assert got[0] <= 0 <= got[1]
        # dW holds dz x: 2^11 times 0.27 times 250 and more is past float16's 65504
        assert n == ((np.abs(ref[:, None] * x[row]) > 65520).sum() if fmt == "f16" else 0)
        # dz and what rounding it leaves are kept, so db has one rounding
        assert_within(got, ref, SCALE * err + 0.5 * (1 + 2.0 ** -7) * ulp(ref, fmt), "db")
        assert (np.delete(db, [3, 9]) == 0).all()


@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("shape", [(31, 300, 64), (700, 5000, 128), (300, 70, 24)], ids=lambda s: "x".join(map(str, s)))
def test_no_loss_below_zero(fmt, shape):
    """Large logits (of some tens) leave ln S within the roundings of z - m, not of m: the
    oracle gets the logits that the sums are exact for (whole numbers times 2^-2)."""
    M, V, K = shape
    rng = np.random.default_rng(M)
    x = rng.integers(-3, 4, (M, K)) * 0.5
    w = rng.integers(-3, 4, (V, K)) * 0.5
    z = x @ w.T + 64.0          # exact in float32: fewer than 24 bits
    b = np.full(V, 64.0)
    t = z.argmax(axis=1).astype(np.int32)
    lo, st = _run(x, w, b, t, fmt)
    stats, loss = linear_ce.forward(z, t)
    assert np.array_equal(st[:, 0], stats[:, 0].astype(np.float32))
    p = np.exp(z - stats[:, :1] - stats[:, 1:])
    # exponents (z - m) log2 e: 2^-22 |z - m| on the average over p, exp2, a chain of sums and joins
    bound = ((p * np.abs(z - stats[:, :1])).sum(axis=1) + 48 + V / 64) * 2.0 ** -22 + 2.0 ** -22 * stats[:, 1]
    assert (st[:, 1] >= 0).all() and (lo >= 0).all()
    assert_within(st[:, 1], stats[:, 1], bound, "ln S")
    assert_within(lo, loss, bound, "loss")
