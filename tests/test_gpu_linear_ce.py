"""Cross entropy of a linear layer, without its logits, on the GPU against the float64 oracle."""
import numpy as np
import pytest

from oracle import linear_ce
from oracle.numfmt import round_to
from tests.gpu_util import HAVE_GPU, assert_within, to_host, ulp

pytestmark = [pytest.mark.gpu, pytest.mark.skipif(not HAVE_GPU, reason="no GPU")]

if HAVE_GPU:
    import torch
    from paper_2507_03312_amd import binding as mx
    TYPES = {"f16": torch.float16, "bf16": torch.bfloat16}

FMTS = ["f16", "bf16"]
HALF = {"f16": 2.0 ** -11, "bf16": 2.0 ** -8}   # the largest relative rounding
SCALE = 2.0 ** 11


def _s():
    return torch.cuda.current_stream().cuda_stream


def _dev(a, fmt, off=0):
    buf = torch.empty(a.size + off, dtype=TYPES[fmt], device="cuda")
    t = buf[off:].view(a.shape)
    t.copy_(torch.from_numpy(np.ascontiguousarray(a, np.float32)))
    return t


def _ptr(t):
    return None if t is None else t.data_ptr()


def _state(scale=SCALE):
    return torch.tensor([scale, 0.0, 0.0, 2.0, 1.0, 2.0 ** 100], device="cuda")


def _guarded(shape, dtype, off=0):
    n = int(np.prod(shape))
    buf = torch.full((n + 256 + off,), -7.0, dtype=dtype, device="cuda")
    return buf, buf[128 + off:128 + off + n].view(shape)


def _untouched(buf, out):
    lo = (out.data_ptr() - buf.data_ptr()) // buf.element_size()
    assert (buf[:lo] == -7.0).all() and (buf[lo + out.numel():] == -7.0).all()


def _inputs(M, V, K, fmt, bias, seed=0):
    rng = np.random.default_rng(M * 31 + V * 7 + K + seed)
    x = round_to(rng.normal(0, 1, (M, K)), fmt)
    w = round_to(rng.normal(0, 2.0 * K ** -0.5, (V, K)), fmt)
    b = round_to(rng.normal(0, 0.5, V), fmt) if bias else None
    t = rng.integers(0, V, M).astype(np.int32)
    t[rng.random(M) < 0.1] = -1
    g = rng.uniform(0.5, 1.5, M).astype(np.float32) / M
    return x, w, b, t, g


def _logits(x, w, b):
    z = x.astype(np.float64) @ w.astype(np.float64).T
    return z if b is None else z + b


def _logit_error(x, w, b):
    """Two float32 orders of the sums."""
    e = np.abs(x.astype(np.float64)) @ np.abs(w.astype(np.float64)).T
    return 2.0 * (x.shape[1] + 1) * 2.0 ** -24 * (e if b is None else e + np.where(np.isfinite(b), np.abs(b), 0))


def _stat_errors(z, dz, stats):
    """m is off by the worst logit's error; ln S by that twice, by the exponentials'
    arguments ((z - m) log2 e and m log2 e rounded: (|z - m| + |m|) 2^-22 on the average over
    p), exp2, and a chain of sums: 32 values and at most V / 64 + 12 joins."""
    m, ln = stats[:, 0], stats[:, 1]
    worst = dz.max(axis=1)
    with np.errstate(all="ignore"):
        p = np.exp(z - m[:, None] - ln[:, None])
        d = np.where(p > 0, np.abs(z - m[:, None]), 0.0)
        args = (p * d).sum(axis=1) + np.abs(m)
    e = 2.0 * worst + (args + 48 + z.shape[1] / 64) * 2.0 ** -22 + 2.0 ** -22 * np.abs(ln)
    return worst + 2.0 ** -23 * np.abs(m), e


def _forward(x, w, b, t, fmt, off=0, loss=True, stats=True, mean=True):
    M, K = x.shape
    V = len(w)
    xt, wt = _dev(x, fmt, off), _dev(w, fmt, off)
    bt = None if b is None else _dev(b, fmt, off)
    tt = torch.from_numpy(t).cuda()
    bufs = [_guarded(s, torch.float32) for s in ((M,), (M, 2), (1,))]
    ws = torch.empty(mx.mpx_linear_ce_fwd_workspace(M, V, K), dtype=torch.uint8, device="cuda")
    outs = [o if use else None for (_, o), use in zip(bufs, (loss, stats, mean))]
    mx.mpx_linear_ce_fwd(xt.data_ptr(), wt.data_ptr(), _ptr(bt), tt.data_ptr(), M, V, K, *map(_ptr, outs),
                         mx.DTYPES[fmt], ws.data_ptr(), ws.numel(), _s())
    for (buf, o), use in zip(bufs, (loss, stats, mean)):
        if use:
            _untouched(buf, o)
        else:
            assert (buf == -7.0).all()
    return (xt, wt, bt, tt), outs


# one and few rows; every direct tile; ragged edges; register-staged; rows of < 8
SHAPES = [(1, 1, 1), (1, 10, 64), (2, 1000, 64), (8, 4099, 128), (32, 300, 192), (33, 129, 64), (3, 7, 5),
          (65, 40, 7), (64, 257, 100), (130, 1003, 320), (300, 515, 72), (520, 2050, 64), (1030, 6500, 64),
          (2100, 16500, 64), (2050, 70, 64), (700, 3001, 75),
          (1100, 4130, 70), (1027, 4099, 200), (256, 64, 1)]


@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("bias", [False, True], ids=["", "bias"])
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "x".join(map(str, s)))
def test_forward(fmt, bias, shape):
    x, w, b, t, _ = _inputs(*shape, fmt, bias)
    z, dz = _logits(x, w, b), _logit_error(x, w, b)
    stats, loss = linear_ce.forward(z, t)
    em, el = _stat_errors(z, dz, stats)
    zt = np.where(t < 0, 0.0, np.abs(stats[:, 0] - z[np.arange(len(t)), np.maximum(t, 0)]))
    eloss = np.where(t < 0, 0.0, 2.0 * dz.max(axis=1) + el + 2.0 ** -22 * (zt + np.abs(loss)))
    for off in (0, 1):
        _, (lo, st, mean) = _forward(x, w, b, t, fmt, off)
        assert_within(to_host(st)[:, 0], stats[:, 0], em, f"m, {off} past alignment")
        assert_within(to_host(st)[:, 1], stats[:, 1], el, f"ln S, {off} past alignment")
        assert_within(to_host(lo), loss, eloss, f"loss, {off} past alignment")
        n = max(1, (t >= 0).sum())
        got = to_host(lo).astype(np.float64)
        assert abs(float(mean) - got.sum() / n) <= (len(t) / 1024 + 12) * 2.0 ** -23 * np.abs(got).sum() / n
    _, (_, st2, _) = _forward(x, w, b, t, fmt, 1, loss=False, mean=False)
    assert torch.equal(st, st2)


def _backward(dev, st, g, fmt, M, V, K, off=0, dx=True, dw=True, db=True, state=True, count=None):
    xt, wt, bt, tt = dev
    bufs = [_guarded(s, TYPES[fmt], off) for s in ((M, K), (V, K), (V,))]
    outs = [o if use else None for (_, o), use in zip(bufs, (dx, dw, db))]
    ws = torch.empty(mx.mpx_linear_ce_bwd_workspace(M, V, K), dtype=torch.uint8, device="cuda")
    gt = None if g is None else torch.from_numpy(np.asarray(g, np.float32)).cuda()
    mx.mpx_linear_ce_bwd(xt.data_ptr(), wt.data_ptr(), _ptr(bt), tt.data_ptr(), M, V, K, st.data_ptr(), _ptr(gt),
                         _state().data_ptr() if state else None, *map(_ptr, outs), mx.DTYPES[fmt], ws.data_ptr(),
                         ws.numel(), _ptr(count), _s())
    torch.cuda.synchronize()
    for (buf, o), use in zip(bufs, (dx, dw, db)):
        if use:
            _untouched(buf, o)
        else:
            assert (buf == -7.0).all()
    return outs


def _gradient_bounds(x, w, z, dz, d, f, stats, fmt):
    """dz = f (p - 1[target]): p is off by its logit's and ln S's errors and its own
    exponent's rounding (z log2 e against the rounded (m + ln S) log2 e), then dz is rounded once (float16: in units of 2^-25 of 2^13
    to 2^14 for the largest f, at worst); float32 sums of two orders, half a step at the
    end, and 2^-20 of itself for an error that moves a value over a rounding border."""
    em, el = _stat_errors(z, dz, stats)
    with np.errstate(all="ignore"):
        p = np.exp(z - stats[:, :1] - stats[:, 1:])
        arg = np.where(p > 0, np.abs(z) + np.abs(stats[:, :1]) + np.abs(stats[:, 1:]) + 8, 0.0)
    fa = np.abs(f)[:, None]
    # up to 128 rows what the rounding of dz leaves is kept, and rounded itself
    step = HALF[fmt] ** 2 if len(x) <= 128 else HALF[fmt]
    e = fa * p * 1.01 * (dz + (em + el)[:, None] + arg * 2.0 ** -22) + np.abs(d) * (step + 2.0 ** -22)
    if fmt == "f16":
        e = e + 2.0 ** -38 * fa.max()

    def of(a, b, ref, n):
        size = (np.abs(a) + e) if a is d else (np.abs(a) + e.T)
        ee = e if a is d else e.T
        err = ee @ np.abs(b) + 2.0 * (n + 16) * 2.0 ** -24 * (size @ np.abs(b))
        return 0.5 * (1 + 2.0 ** -10) * ulp(ref, fmt) + err
    x64, w64 = x.astype(np.float64), w.astype(np.float64)
    dx, dw, db = d @ w64, d.T @ x64, d.sum(0)
    ones = np.ones((len(x), 1))
    return (dx, of(d, w64, dx, len(w))), (dw, of(d.T, x64, dw, len(x))), \
        (db, of(d.T, ones, db[:, None], len(x))[:, 0])


@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("bias", [False, True], ids=["", "bias"])
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "x".join(map(str, s)))
def test_backward(fmt, bias, shape):
    M, V, K = shape
    x, w, b, t, g = _inputs(M, V, K, fmt, bias)
    z, dz = _logits(x, w, b), _logit_error(x, w, b)
    stats, _ = linear_ce.forward(z, t)
    for off, weights in ((0, g), (1, None)):
        dev, (_, st, _) = _forward(x, w, b, t, fmt, off)
        gw = linear_ce.mean_weights(t) if weights is None else weights
        d = linear_ce.dlogits(z, t, stats, gw, SCALE)
        f = np.where(t < 0, 0.0, SCALE * gw)
        outs = _backward(dev, st, weights, fmt, M, V, K, off)
        for name, o, (ref, bound) in zip(("dX", "dW", "db"), outs, _gradient_bounds(x, w, z, dz, d, f, stats, fmt)):
            assert_within(to_host(o), ref, bound, f"{name}, {off} past alignment")
        # any subset: dX and dW the same bits, db by its own sums
        only = _backward(dev, st, weights, fmt, M, V, K, off, dw=False, db=False)
        assert torch.equal(only[0], outs[0])
        only = _backward(dev, st, weights, fmt, M, V, K, off, dx=False, db=False)
        assert torch.equal(only[1], outs[1])
        only = _backward(dev, st, weights, fmt, M, V, K, off, dx=False, dw=False)
        ref, bound = _gradient_bounds(x, w, z, dz, d, f, stats, fmt)[2]
        assert_within(to_host(only[2]), ref, bound, "db alone")


@pytest.mark.parametrize("fmt", FMTS)
def test_several_pieces(fmt):
    """A vocabulary of several pieces, the last one ragged, against the exact gradient of
    some rows and columns."""
    M, V, K = 6000, 20011, 64
    g = torch.Generator(device="cuda").manual_seed(4)
    x = torch.empty(M, K, device="cuda").normal_(generator=g).to(TYPES[fmt])
    w = (0.3 * torch.empty(V, K, device="cuda").normal_(generator=g)).to(TYPES[fmt])
    t = torch.randint(-1, V, (M,), generator=g, device="cuda", dtype=torch.int32)
    assert mx.mpx_linear_ce_bwd_workspace(M, V, K) < 2 * M * V   # the logits never exist whole
    loss, st = torch.empty(M, device="cuda"), torch.empty(M, 2, device="cuda")
    ws = torch.empty(max(mx.mpx_linear_ce_fwd_workspace(M, V, K), mx.mpx_linear_ce_bwd_workspace(M, V, K)),
                     dtype=torch.uint8, device="cuda")
    mx.mpx_linear_ce_fwd(x.data_ptr(), w.data_ptr(), None, t.data_ptr(), M, V, K, loss.data_ptr(), st.data_ptr(),
                         None, mx.DTYPES[fmt], ws.data_ptr(), ws.numel(), _s())
    dx, dw = torch.empty_like(x), torch.empty_like(w)
    db = torch.empty(V, dtype=TYPES[fmt], device="cuda")
    wt = (torch.rand(M, generator=g, device="cuda") + 0.5) / M
    mx.mpx_linear_ce_bwd(x.data_ptr(), w.data_ptr(), None, t.data_ptr(), M, V, K, st.data_ptr(), wt.data_ptr(),
                         _state().data_ptr(), dx.data_ptr(), dw.data_ptr(), db.data_ptr(), mx.DTYPES[fmt],
                         ws.data_ptr(), ws.numel(), None, _s())
    z = x.double() @ w.double().t()
    d = torch.softmax(z, 1)
    at = torch.arange(M, device="cuda")
    d[at, t.long().clamp(min=0)] -= 1.0
    d *= (torch.where(t < 0, 0.0, wt.double()) * SCALE)[:, None]
    # each dz is off by half a step and 2^-12 of itself and of f p (float32 logits and
    # exponents: below 64 * 64 * 2^-24 + 40 * 2^-22), sums by two orders, the result by half a step
    for got, a, b, n in ((dx, d, w.double(), V), (dw, d.t(), x.double(), M), (db[:, None], d.t(), None, M)):
        mm = lambda p, q: p.sum(1, keepdim=True) if q is None else p @ q
        ref = mm(a, b)
        size = mm(a.abs(), None if b is None else b.abs())
        bound = (HALF[fmt] + 2.0 ** -12 + 2.0 * n * 2.0 ** -24) * size + 0.5 * torch.from_numpy(
            ulp(ref.cpu().numpy(), fmt)).cuda() * (1 + 2.0 ** -10)
        assert ((got.double() - ref).abs() <= bound).all()


@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("M, V, K", [(20, 1049001, 64), (50, 530003, 40), (100, 262500, 72), (129, 350001, 36),
                                     (300, 210011, 72)])
def test_few_rows_over_several_pieces(fmt, M, V, K):
    """Few rows, with what the rounding of dz leaves, over a vocabulary of more than one piece:
    dW and db element by element, dX in norm (half a step of every element, 2^-12 for its
    float32 logits, exponents and sums; past 128 rows half a step of every dz more); subsets
    and the padded rows of the reduction."""
    g = torch.Generator(device="cuda").manual_seed(M)
    x = torch.empty(M, K, device="cuda").normal_(generator=g).to(TYPES[fmt])
    w = (2.0 * K ** -0.5 * torch.empty(V, K, device="cuda").normal_(generator=g)).to(TYPES[fmt])
    b = (0.5 * torch.empty(V, device="cuda").normal_(generator=g)).to(TYPES[fmt])
    t = torch.randint(-1, V, (M,), generator=g, device="cuda", dtype=torch.int32)
    t[0], t[1] = V - 1, 0   # the first and the last piece's own
    st = torch.empty(M, 2, device="cuda")
    ws = torch.empty(mx.mpx_linear_ce_fwd_workspace(M, V, K), dtype=torch.uint8, device="cuda")
    mx.mpx_linear_ce_fwd(x.data_ptr(), w.data_ptr(), b.data_ptr(), None, M, V, K, None, st.data_ptr(), None,
                         mx.DTYPES[fmt], ws.data_ptr(), ws.numel(), _s())
    wt = (torch.rand(M, generator=g, device="cuda") + 0.5) / M
    got = _backward((x, w, b, t), st, wt.cpu().numpy(), fmt, M, V, K)
    z = x.double() @ w.double().t() + b.double()
    d = torch.softmax(z, 1)
    d[torch.arange(M, device="cuda"), t.long().clamp(min=0)] -= (t >= 0).double()
    d *= (torch.where(t < 0, 0.0, wt.double()) * SCALE)[:, None]
    ref = d @ w.double()
    left = 0.0 if M <= 128 else HALF[fmt] * float((d.abs() @ w.double().abs()).norm() / ref.norm())
    assert float((got[0].double() - ref).norm() / ref.norm()) <= HALF[fmt] + 2.0 ** -12 + left
    step = 2.0 ** -12 + (HALF[fmt] ** 2 if M <= 128 else HALF[fmt])
    least = 2.0 ** -38 * float(wt.max()) * SCALE if fmt == "f16" else 0.0   # float16's smallest dz
    for o, q in ((got[1], x.double()), (got[2][:, None], torch.ones(M, 1, dtype=torch.float64, device="cuda"))):
        ref, size = d.t() @ q, d.t().abs() @ q.abs()
        bound = (step + 2.0 * M * 2.0 ** -24) * size + least * q.abs().sum(0) + 0.5 * torch.from_numpy(
            ulp(ref.cpu().numpy(), fmt)).cuda() * (1 + 2.0 ** -10)
        assert ((o.double() - ref).abs() <= bound).all()
    for use in ({"dw": False, "db": False}, {"dx": False, "db": False}):
        only = _backward((x, w, b, t), st, wt.cpu().numpy(), fmt, M, V, K, **use)
        assert all(o is None or torch.equal(o, p) for o, p in zip(only, got))


@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("M", [5, 40])
def test_masks_targets_and_not_finite_rows(fmt, M):
    """A bias of -inf masks its column; a target outside the vocabulary, a masked one,
    rows without one; a row with an infinity."""
    V, K = 200, 64
    x, w, b, t, g = _inputs(M, V, K, fmt, True)
    t[:] = np.arange(M) % V
    b[3] = -np.inf
    b[150:] = -np.inf
    t[0], t[1], t[2], t[3], t[4] = -5, V, 2 ** 31 - 1, 3, 7
    dev, (lo, st, mean) = _forward(x, w, b, t, fmt)
    z = _logits(x, w, b)
    stats, loss = linear_ce.forward(z, t)
    got = to_host(lo)
    assert np.array_equal(np.isnan(got), np.isnan(loss)) and np.isnan(got[1]) and np.isnan(got[2])
    assert got[0] == 0 and got[3] == np.inf and np.isnan(float(mean))
    fin = np.isfinite(loss)
    assert np.allclose(got[fin], loss[fin], rtol=1e-4, atol=1e-4)
    dx, dw, db = map(to_host, _backward(dev, st, g, fmt, M, V, K))
    assert np.isnan(dx[[1, 2]]).all() and np.isfinite(np.delete(dx, [1, 2], axis=0)).all() and (dx[0] == 0).all()
    assert np.isnan(dw).all() and np.isnan(db).all()
    t[1] = t[2] = 4
    masked = np.isinf(b)
    dev, (lo, st, _) = _forward(x, w, b, t, fmt)
    dx, dw, db = map(to_host, _backward(dev, st, g, fmt, M, V, K))
    assert np.isfinite(dx).all() and (dw[masked] == 0).all() and (db[masked] == 0).all()
    assert np.isfinite(dw).all() and (dw[~masked] != 0).any(axis=1).all()
    # everything masked
    b[:] = -np.inf
    dev, (lo, st, _) = _forward(x, w, b, t, fmt)
    assert (to_host(st)[:, 0] == -np.inf).all() and (to_host(st)[:, 1] == 0).all()
    assert to_host(lo)[0] == 0 and (to_host(lo)[1:] == np.inf).all()
    for o in _backward(dev, st, g, fmt, M, V, K):
        assert (o == 0).all()
    # an infinity in one row
    x[4, 9] = np.inf
    dev, (lo, st, _) = _forward(x, w, None, t, fmt)
    assert np.isnan(to_host(lo)[4]) and np.isfinite(np.delete(to_host(lo), 4)).all()
    n = torch.zeros(1, dtype=torch.int32, device="cuda")
    dx, dw, db = map(to_host, _backward(dev, st, g, fmt, M, V, K, count=n))
    assert np.isnan(dx[4]).all() and np.isfinite(np.delete(dx, 4, axis=0)).all() and not np.isfinite(dw).any()
    assert int(n) == (~np.isfinite(dw)).sum() + (~np.isfinite(db)).sum()


def test_small_probabilities_survive_float16():
    """Rows whose probabilities times scale g lie below float16's smallest value keep
    their share of dW: dz is held in the middle of the type's range."""
    M, V, K = 64, 512, 64
    rng = np.random.default_rng(7)
    x = round_to(rng.normal(0, 1, (M, K)), "f16")
    w = round_to(rng.normal(0, 1, (V, K)) * 1e-3, "f16")
    b = round_to(np.where(np.arange(V) == 0, 12.0, 0.0), "f16")   # column 0 has all but 0.3%
    t = np.zeros(M, np.int32)
    g = np.full(M, 1e-4, np.float32)                              # scale g p about 6e-9 for the others
    dev, (_, st, _) = _forward(x, w, b, t, "f16")
    xt, wt, bt, tt = dev
    state = _state(2.0 ** 4)
    dw = torch.empty(V, K, dtype=torch.float16, device="cuda")
    ws = torch.empty(mx.mpx_linear_ce_bwd_workspace(M, V, K), dtype=torch.uint8, device="cuda")
    gt = torch.from_numpy(g).cuda()
    mx.mpx_linear_ce_bwd(xt.data_ptr(), wt.data_ptr(), bt.data_ptr(), tt.data_ptr(), M, V, K, st.data_ptr(),
                         gt.data_ptr(), state.data_ptr(), None, dw.data_ptr(), None, mx.MPX_F16, ws.data_ptr(),
                         ws.numel(), None, _s())
    z = _logits(x, w, b)
    d = linear_ce.dlogits(z, t, linear_ce.forward(z, t)[0], g, 16.0)
    assert np.abs(d[:, 1:]).max() < 2.0 ** -25   # nothing of it is a float16 value
    ref = d.T @ x.astype(np.float64)
    # half a step of dz and of the result's subnormal range, and float32 terms
    bound = (2.0 ** -11 + 2.0 ** -12) * (np.abs(d).T @ np.abs(x)) + 2.0 ** -25
    assert_within(to_host(dw), ref, bound, "dW")
    assert np.linalg.norm(ref[1:]) > 64 * 2.0 ** -25   # and the rounding to 0 would show


def test_side_stream_and_graph():
    """Forward and backward captured and replayed with the program's own eager calls
    between, each with a workspace of its own."""
    M, V, K = 200, 1500, 64
    x, w, _, t, g = _inputs(M, V, K, "bf16", False)
    dev, _ = _forward(x, w, None, t, "bf16")
    xt, wt, _, tt = dev
    gt, state = torch.from_numpy(g).cuda(), _state()
    sets = []
    for _ in range(2):
        sets.append({"loss": torch.empty(M, device="cuda"), "st": torch.empty(M, 2, device="cuda"),
                     "mean": torch.empty(1, device="cuda"), "dx": torch.empty_like(xt), "dw": torch.empty_like(wt),
                     "ws": torch.empty(max(mx.mpx_linear_ce_fwd_workspace(M, V, K),
                                           mx.mpx_linear_ce_bwd_workspace(M, V, K)), dtype=torch.uint8,
                                       device="cuda")})

    def call(o, s):
        mx.mpx_linear_ce_fwd(xt.data_ptr(), wt.data_ptr(), None, tt.data_ptr(), M, V, K, o["loss"].data_ptr(),
                             o["st"].data_ptr(), o["mean"].data_ptr(), mx.MPX_BF16, o["ws"].data_ptr(),
                             o["ws"].numel(), s)
        mx.mpx_linear_ce_bwd(xt.data_ptr(), wt.data_ptr(), None, tt.data_ptr(), M, V, K, o["st"].data_ptr(),
                             gt.data_ptr(), state.data_ptr(), o["dx"].data_ptr(), o["dw"].data_ptr(), None,
                             mx.MPX_BF16, o["ws"].data_ptr(), o["ws"].numel(), None, s)
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        call(sets[0], _s())
    side = torch.cuda.Stream()
    for i in range(4):
        xt.copy_(torch.randn(M, K, device="cuda"))
        tt.copy_(torch.randint(-1, V, (M,), device="cuda", dtype=torch.int32))
        torch.cuda.synchronize()
        with torch.cuda.stream(side):
            call(sets[1], side.cuda_stream)
        graph.replay()
        torch.cuda.synchronize()
        for k in ("loss", "st", "mean", "dx", "dw"):
            assert torch.equal(sets[0][k], sets[1][k]), (i, k)


def test_gradient_by_differences():
    """<dX, D> and <dW, E> against central differences of the mean loss that the forward
    itself computes.  Along a direction that moves a row's logits by u the loss's third
    derivative is the third central moment of u under some p, at most (max u - min u)^3,
    so the difference is off by a sixth of its mean; each loss by its statistics' bound,
    (args + 48 + 1) 2^-22 with args below 16, hence 2^-16; the gradient's elements by half a step."""
    M, V, K = 24, 50, 64
    x, w, _, t, _ = _inputs(M, V, K, "f16", False)
    rng = np.random.default_rng(8)
    dev, (_, st, _) = _forward(x, w, None, t, "f16")
    dx, dw, _ = _backward(dev, st, None, "f16", M, V, K, db=False)
    for arg, grad, h in ((0, dx, 2.0 ** -8), (1, dw, 2.0 ** -10)):
        a = (x, w)[arg]
        # uphill, each element by a random share of h (sums of random signs say little)
        d = (np.sign(to_host(grad)) * rng.uniform(0.5, 1, a.shape)).astype(np.float32)
        moved = [round_to(a + s * h * d, "f16") for s in (1, -1)]
        step = (moved[0].astype(np.float64) - moved[1]) / 2   # what the rounding left of h d
        losses = []
        for m in moved:
            xs = [x, w]
            xs[arg] = m
            losses.append(float(_forward(xs[0], xs[1], None, t, "f16")[1][2]))
        u = step @ w.astype(np.float64).T if arg == 0 else x.astype(np.float64) @ step.T
        third = ((u.max(axis=1) - u.min(axis=1)) ** 3).mean() / 6
        middle = (moved[0].astype(np.float64) + moved[1]) / 2 - a   # not quite 0 after rounding
        second = np.abs(middle).max() * K * np.abs(step).max() * (np.abs(w).max() if arg == 0 else np.abs(x).max()) ** 2
        g = to_host(grad).astype(np.float64) / SCALE
        want = (losses[0] - losses[1]) / 2
        assert abs(want - (g * step).sum()) <= 2.0 ** -11 * np.abs(g * step).sum() + third + second + 2.0 ** -16, arg
        assert third + second + 2.0 ** -16 < 0.5 * abs(want)   # the comparison says something
