"""Log probabilities, entropy, top alternatives and their gradient on the GPU
against the float64 oracle."""
import numpy as np
import pytest

from oracle import logprob
from oracle.numfmt import round_to
from tests.gpu_util import HAVE_GPU, ulp

pytestmark = [pytest.mark.gpu, pytest.mark.skipif(not HAVE_GPU, reason="no GPU")]

if HAVE_GPU:
    import torch
    from paper_2507_03312_amd import binding as mx
    HALF = {"f16": torch.float16, "bf16": torch.bfloat16, "f32": torch.float32}

FMTS = ["f16", "bf16", "f32"]
U = 2.0 ** -24


def _s():
    return torch.cuda.current_stream().cuda_stream


def _upload(z, fmt, pad=0, off=0):
    """Logits [rows, V] at row stride V + pad, the first at element `off`, NaN in
    the padding (it must not be read)."""
    rows, V = z.shape
    buf = torch.full((off + rows * (V + pad),), float("nan"), dtype=HALF[fmt], device="cuda")
    t = buf[off:].view(rows, V + pad)
    t[:, :V] = torch.from_numpy(np.ascontiguousarray(z)).to(HALF[fmt]).cuda()
    return t


def _fwd(t, targets, V, k, fmt, stream=None, ws=None):
    rows, ld = t.shape[0], t.stride(0)
    f = torch.full((4, rows + 1), -7.0, device="cuda")   # logp, entropy, stats (2 rows' worth)
    top = torch.full((rows * k + 1,), -7.0, device="cuda")
    idx = torch.full((rows * k + 1,), -7, dtype=torch.int32, device="cuda")
    need = mx.mpx_logprob_workspace(rows, V, k)
    ws = torch.full((need + 64,), 0xA5, dtype=torch.uint8, device="cuda") if ws is None else ws
    mx.mpx_logprob_fwd(t.data_ptr(), ld, targets.data_ptr(), rows, V, k, f[0].data_ptr(), f[1].data_ptr(),
                       f[2].data_ptr(), top.data_ptr() if k else None, idx.data_ptr() if k else None,
                       mx.DTYPES[fmt], ws.data_ptr(), need, _s() if stream is None else stream)
    return f, top, idx, ws, need


def _np(t):
    return t.double().cpu().numpy()


def _stats(f, rows):
    return _np(f[2:].reshape(-1)[:2 * rows].view(rows, 2))


def _check_forward(z, t, targets, k, fmt):
    rows, V = z.shape
    f, top, idx, ws, need = _fwd(t, targets, V, k, fmt)
    torch.cuda.synchronize()
    assert (f[:2, rows:] == -7.0).all() and (f[2:].reshape(-1)[2 * rows:] == -7.0).all() and top[rows * k:] == -7.0 and idx[rows * k:] == -7
    assert (ws[need:] == 0xA5).all()
    rstats, logp, ent, rtop, ridx = logprob.forward(z, targets.cpu().numpy(), k)
    with np.errstate(over="ignore"):     # -6e38 of logits 3e38 apart is -inf in float32
        logp, rtop = (np.where(np.isinf(a.astype(np.float32)), -np.inf, a) for a in (logp, rtop))
    stats = _stats(f, rows)
    fin = np.isfinite(rstats).all(axis=1)
    zf = z[fin]
    if len(zf):
        # relative error of S: each exponential (|d| + 4) 2 U (rounded argument and
        # function), sums in chains of at most V / 64 + 64 terms
        m = zf.max(axis=1)
        d = zf - m[:, None]
        p = np.exp(np.where(np.isfinite(d), d, -1e9))
        p /= p.sum(axis=1, keepdims=True)
        ad = np.where(p > 0, np.abs(np.where(np.isfinite(d), d, 0.0)), 0.0)
        chain = (V / 64 + 64) * U
        dS = (p * (ad + 4) * 2 * U).sum(axis=1) + chain
        lnS = rstats[fin, 1]
        dln = dS + 4 * U * (1 + np.abs(lnS))
        assert np.array_equal(stats[fin, 0], m) and np.all(np.abs(stats[fin, 1] - lnS) <= dln)
        pw = (p * ad).sum(axis=1)
        dW = (p * ad * (ad + 4) * 2 * U).sum(axis=1) + pw * (chain + dS + 4 * U)
        assert np.all(np.abs(_np(f[1, :rows])[fin] - ent[fin]) <= dln + dW + 2 * U * (np.abs(lnS) + pw))
        tol = dln + 2 * U * np.abs(lnS)
        g, r = _np(f[0, :rows])[fin], logp[fin]
        ok = np.isfinite(r)
        assert np.array_equal(g[~ok], r[~ok], equal_nan=True)
        assert np.all(np.abs(g[ok] - r[ok]) <= (tol + 4 * U * (np.abs(np.where(ok, r, 0)) + np.abs(lnS)))[ok])
        if k:
            g, r = _np(top[:rows * k]).reshape(rows, k)[fin], rtop[fin]
            ok = np.isfinite(r)
            assert np.array_equal(g[~ok], r[~ok])
            lim = tol[:, None] + 4 * U * (np.abs(np.where(ok, r, 0)) + np.abs(lnS)[:, None])
            assert np.all(np.abs(g[ok] - r[ok]) <= lim[ok])
    rest = ~fin
    assert np.array_equal(stats[rest], rstats[rest], equal_nan=True)
    for i, r in enumerate((logp, ent)):
        assert np.array_equal(_np(f[i, :rows])[rest], r[rest], equal_nan=True), i
    if k:
        assert np.array_equal(_np(top[:rows * k]).reshape(rows, k)[rest], rtop[rest], equal_nan=True)
        assert np.array_equal(idx[:rows * k].view(rows, k).cpu().numpy(), ridx)
    return f, idx


def _check_backward(z, t, targets, k, fmt, f, idx, which="les", scale=None, in_place=False, seed=0):
    rows, V = z.shape
    rng = np.random.default_rng(seed)
    gl, ge = (rng.normal(0, 1, rows).astype(np.float32) for _ in range(2))
    gt = rng.normal(0, 1, (rows, k)).astype(np.float32)
    dev = [torch.from_numpy(a).cuda() for a in (gl, ge, gt)]
    use = ["l" in which, "e" in which, "s" in which and k > 0]
    st = torch.tensor([scale or 1.0, 0, 0, 2, 1, 2.0 ** 100], device="cuda")
    out = t.clone() if in_place else torch.full((rows + 1, V + 3), -7.0, dtype=HALF[fmt], device="cuda")
    src = out if in_place else t
    ldo = out.stride(0)
    keep = out.clone()
    mx.mpx_logprob_bwd(src.data_ptr(), src.stride(0), targets.data_ptr(), rows, V, k, f[2].data_ptr(),
                       f[1].data_ptr(), idx.data_ptr() if k else None,
                       *[d.data_ptr() if u else None for d, u in zip(dev, use)],
                       st.data_ptr() if scale else None, out.data_ptr(), ldo, mx.DTYPES[fmt], _s())
    torch.cuda.synchronize()
    same = lambda a, b: torch.equal(a.contiguous().view(torch.uint8), b.contiguous().view(torch.uint8))
    assert same(out[:, V:], keep[:, V:]) and same(out[rows:], keep[rows:])
    stats, ent = _stats(f, rows), _np(f[1, :rows])
    ridx = idx[:rows * k].view(rows, k).cpu().numpy() if k else None
    ref, mag = logprob.backward(z, targets.cpu().numpy(), stats, ent, ridx, gl if use[0] else None,
                                ge if use[1] else None, gt if use[2] else None, scale or 1.0)
    got = _np(out[:rows, :V])
    with np.errstate(all="ignore"):
        lp = np.abs(z - stats[:, :1]) + np.abs(stats[:, 1:])
        # float32 terms: p to (2 |lp| + 8) U, the sum of k + 1 cotangents and the
        # products around it (k + 8) U; then half a step of the output; and a
        # probability below 2^-126, float32's least normal value, may come out of
        # the exponential as 0: off by up to 2^-126 times what it is multiplied by
        tol = mag * (2 * np.where(np.isfinite(lp), lp, 0) + 16 + k) * U * 2
        want = round_to(ref, fmt).astype(np.float64)
        bound = tol + 0.5 * ulp(np.where(np.isfinite(ref), np.abs(ref) + tol, 0), fmt) * (1 + 2.0 ** -10)
        factor = (np.abs(gl) * use[0] + np.abs(gt).sum(axis=1) * use[2])[:, None] + (
            np.abs(ge)[:, None] * use[1] * (np.minimum(lp, 200) + np.abs(ent)[:, None]))
        bound = bound + 2.0 ** -126 * (1 + (scale or 1.0) * np.nan_to_num(factor))
    fin = np.isfinite(want)
    assert np.array_equal(np.isnan(got), np.isnan(want))
    edge = ~np.isfinite(got) ^ ~fin      # an overflow on one side only: at the border
    if edge.any():
        big = {"f16": 65504.0, "bf16": 3.38e38, "f32": 3.4e38}[fmt]
        assert np.all(np.abs(ref[edge]) > big * (1 - 2.0 ** -8))
    bad = np.argwhere(fin & ~edge & ~(np.abs(got - ref) <= bound))
    assert not len(bad), [(tuple(i), got[tuple(i)], ref[tuple(i)], bound[tuple(i)], z[tuple(i)]) for i in bad[:4]]
    return out


SHAPES = [(1, 1, 1), (1, 2, 2), (3, 7, 7), (5, 10, 0), (4, 63, 3), (2, 64, 16), (7, 65, 16), (64, 100, 5),
          (9, 511, 2), (6, 513, 8), (256, 1000, 5), (33, 1024, 1), (5, 2049, 4), (3, 4099, 16), (2, 8192, 8),
          (17, 10007, 6), (1, 65537, 16), (3, 131072, 8), (1, 262144, 1), (300, 5003, 4), (2048, 1501, 5),
          (4097, 1031, 3)]


@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("case", SHAPES, ids=lambda c: "x".join(map(str, c)))
def test_logprob(fmt, case):
    rows, V, k = case
    rng = np.random.default_rng(rows + V)
    z = round_to(rng.normal(0, 3, (rows, V)), fmt).astype(np.float64)
    targets = torch.from_numpy(rng.integers(0, V, rows).astype(np.int32)).cuda()
    for pad, off in ((0, 0), (3, 1)):
        t = _upload(z, fmt, pad, off)
        f, idx = _check_forward(z, t, targets, k, fmt)
        _check_backward(z, t, targets, k, fmt, f, idx, scale=2.0 ** 10 if pad else None, seed=V)
    _check_backward(z, t, targets, k, fmt, f, idx, in_place=True, seed=V + 1)


@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("V", [5, 300, 3000, 70000])
def test_masked_rows_and_special_values(fmt, V):
    """Masks of -inf and of the type's lowest value, rows with nothing left, with
    one value left, with NaN and +inf, far from zero, all equal."""
    rng = np.random.default_rng(V)
    low = {"f16": -65504.0, "bf16": -3.3895313892515355e38, "f32": -3.4028234663852886e38}[fmt]
    far = {"f16": 6.0e4, "bf16": 3.0e38, "f32": 3.0e38}[fmt]
    z = round_to(rng.normal(0, 2, (16, V)), fmt).astype(np.float64)
    z[0] = -np.inf
    z[1, :] = -np.inf
    z[1, V - 1] = 1.5
    z[2, ::2] = -np.inf
    z[3] = low
    z[4, 1:] = low
    z[5, V // 2] = np.nan
    z[6, V // 3] = np.inf
    z[7] = np.inf
    z[8] = np.nan
    z[9] = 0.25
    z[10] = round_to(z[10] + far / 2, fmt)
    z[11, 0], z[11, 1] = far, -far
    z[12, : V // 2] = 0.0
    z[12, V // 2:] = -0.0
    z[13, V - 1] = 100.0                       # all but one hopeless
    z[14] = round_to(np.linspace(-5, 5, V), fmt)
    z[15] = z[14][::-1]
    k = min(16, V)
    tg = rng.integers(0, V, 16).astype(np.int32)
    tg[1], tg[2], tg[13], tg[14], tg[15] = V - 1, 0, V - 1, -1, V
    targets = torch.from_numpy(tg).cuda()
    t = _upload(z, fmt, 2)
    z = _np(t[:, :V])    # 3e38 is no bfloat16 or float32 value: the oracle gets what was uploaded
    f, idx = _check_forward(z, t, targets, k, fmt)
    for which in ("les", "l", "e", "s", "le"):
        _check_backward(z, t, targets, k, fmt, f, idx, which, seed=V)
    assert (f[0, 14] == 0.0) and torch.isnan(f[0, 15])
    out = _check_backward(z, t, targets, k, fmt, f, idx, "les", in_place=True)
    assert (out[0, :V] == 0).all()


@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("V", [40, 1000, 20000])
def test_ties_go_to_the_lowest_column(fmt, V):
    rng = np.random.default_rng(V)
    z = rng.integers(-2, 3, (12, V)).astype(np.float64)    # five values, thousands of ties
    z[0] = np.arange(V)[::-1] // 3 * 0.125 if V < 2000 else z[0]
    z = round_to(z, fmt).astype(np.float64)
    targets = torch.zeros(12, dtype=torch.int32, device="cuda")
    _check_forward(z, _upload(z, fmt), targets, 16, fmt)
    up = round_to(np.sort(rng.normal(0, 3, (12, V)), axis=1), fmt).astype(np.float64)
    _check_forward(up, _upload(up, fmt, 1, 1), targets, 16, fmt)           # every value beats the last
    _check_forward(up[:, ::-1], _upload(up[:, ::-1], fmt), targets, 16, fmt)


@pytest.mark.parametrize("fmt", FMTS)
def test_any_subset_of_the_results(fmt):
    rows, V, k = 3, 9000, 4
    rng = np.random.default_rng(8)
    z = round_to(rng.normal(0, 3, (rows, V)), fmt).astype(np.float64)
    t = _upload(z, fmt)
    targets = torch.from_numpy(rng.integers(0, V, rows).astype(np.int32)).cuda()
    f, top, idx, ws, need = _fwd(t, targets, V, k, fmt)
    for keep in range(1, 16):
        g = torch.full((4, rows), -7.0, device="cuda")
        tp, ix = torch.full((rows * k,), -7.0, device="cuda"), torch.full((rows * k,), -7, dtype=torch.int32, device="cuda")
        kk = k if keep & 8 else 0
        ptr = [g[i].data_ptr() if keep >> i & 1 else None for i in range(3)]
        mx.mpx_logprob_fwd(t.data_ptr(), V, targets.data_ptr() if keep & 1 else None, rows, V, kk, *ptr,
                           tp.data_ptr() if kk else None, ix.data_ptr() if kk else None, mx.DTYPES[fmt],
                           ws.data_ptr(), need, _s())
        for i in range(3):
            got, want = (g[i], f[i, :rows]) if i < 2 else (g[2:].reshape(-1), f[2:].reshape(-1)[:2 * rows])
            assert torch.equal(got, want) if keep >> i & 1 else (got == -7.0).all()
        assert torch.equal(ix, idx[:rows * k]) and torch.equal(tp, top[:rows * k]) if kk else (ix == -7).all()


def test_gradient_against_differences():
    """The float32 kernels alone: directional differences of the forward's
    results against the backward.  Truncation h^2 |f'''| / 6 and rounding
    (|f| 2^-22 / h for the summed results) at h = 2^-6, for results of size 10."""
    rows, V, k = 4, 50, 3
    rng = np.random.default_rng(2)
    z = rng.normal(0, 2, (rows, V)).astype(np.float32).astype(np.float64)
    targets = torch.from_numpy(rng.integers(0, V, rows).astype(np.int32)).cuda()
    f, top, idx, _, _ = _fwd(_upload(z, "f32"), targets, V, k, "f32")
    g = [torch.from_numpy(a.astype(np.float32)).cuda() for a in (rng.normal(size=rows), rng.normal(size=rows), rng.normal(size=(rows, k)))]
    dz = torch.empty(rows, V, device="cuda")
    t = _upload(z, "f32")
    mx.mpx_logprob_bwd(t.data_ptr(), V, targets.data_ptr(), rows, V, k, f[2].data_ptr(), f[1].data_ptr(),
                       idx.data_ptr(), g[0].data_ptr(), g[1].data_ptr(), g[2].data_ptr(), None, dz.data_ptr(),
                       V, mx.MPX_F32, _s())
    h = 2.0 ** -6

    def value(zz):
        a, tp, _, _, _ = _fwd(_upload(zz, "f32"), targets, V, k, "f32")
        return float((a[0, :rows].double() * g[0].double()).sum() + (a[1, :rows].double() * g[1].double()).sum()
                     + (tp[:rows * k].view(rows, k).double() * g[2].double()).sum())
    for i in range(6):
        d = rng.choice([-1.0, 1.0], (rows, V)) / np.sqrt(rows * V)   # |d z| <= h / 14: the top order stays
        num = (value(z + h * d) - value(z - h * d)) / (2 * h)
        want = float((_np(dz) * d).sum())
        # |g| sums to about 16; f''' along d is below 10 of it times |d|_inf^2
        assert abs(num - want) <= 16 * (10 * h * h / 6 / 14 ** 2 + 40 * 2.0 ** -22 / (2 * h)) + 1e-5


def test_graph_side_stream_and_two_calls_at_once():
    rows, V, k = 6, 40000, 5
    t = torch.zeros(rows, V, dtype=torch.bfloat16, device="cuda")
    targets = torch.zeros(rows, dtype=torch.int32, device="cuda")
    g = torch.cuda.CUDAGraph()
    _fwd(t, targets, V, k, "bf16")
    torch.cuda.synchronize()
    with torch.cuda.graph(g):
        cap = _fwd(t, targets, V, k, "bf16")
    side = torch.cuda.Stream()
    for i in range(4):
        t.copy_(torch.randn(rows, V, device="cuda") * 3)
        targets.copy_(torch.randint(0, V, (rows,), device="cuda"))
        torch.cuda.synchronize()
        with torch.cuda.stream(side):
            a = _fwd(t, targets, V, k, "bf16", side.cuda_stream)
        b = _fwd(t, targets, V, k, "bf16")
        g.replay()
        torch.cuda.synchronize()
        for x, y, w in zip(cap[:3], a[:3], b[:3]):
            assert torch.equal(x, y) and torch.equal(y, w), i


def test_offsets_past_32_bits():
    """Rows 2^30 + 8 elements apart: the third starts past 2^31 elements."""
    rows, V, ld = 3, 5000, (1 << 30) + 8
    buf = torch.zeros(2 * ld + V, dtype=torch.bfloat16, device="cuda")
    rng = np.random.default_rng(4)
    z = round_to(rng.normal(0, 3, (rows, V)), "bf16").astype(np.float64)
    t = buf.as_strided((rows, V), (ld, 1))
    t.copy_(torch.from_numpy(z).bfloat16().cuda())
    targets = torch.tensor([1, 4999, 77], dtype=torch.int32, device="cuda")
    f, idx = _check_forward(z, t, targets, 4, "bf16")
    small = _upload(z, "bf16")
    want = _check_backward(z, small, targets, 4, "bf16", f, idx, seed=3)[:rows, :V]
    gl, ge = (torch.from_numpy(a).cuda() for a in [np.random.default_rng(3).normal(0, 1, (2, rows)).astype(np.float32)][0])
    gt = None
    st = torch.tensor([1.0, 0, 0, 2, 1, 1e30], device="cuda")
    one = torch.empty(rows, V, dtype=torch.bfloat16, device="cuda")
    for src, out, lo in ((small, one, V), (t, t, ld)):
        mx.mpx_logprob_bwd(src.data_ptr(), src.stride(0), targets.data_ptr(), rows, V, 0, f[2].data_ptr(),
                           f[1].data_ptr(), None, gl.data_ptr(), ge.data_ptr(), gt, st.data_ptr(),
                           out.data_ptr(), lo, mx.MPX_BF16, _s())
    assert torch.equal(t, one) and want.shape == one.shape


@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("k", [0, 1, 16])
def test_rows_do_not_depend_on_how_many_there_are(fmt, k):
    """Thousands of rows (a wave each), hundreds (a workgroup each) and single ones
    (several workgroups each): the same alternatives, and float results that
    differ by their summation orders only (chains of at most V / 64 + 64 terms on
    either side, relative to sums of positive terms)."""
    rows, V = 4096, 20011
    g = torch.Generator(device="cuda").manual_seed(k)
    t = torch.empty(rows, V, device="cuda").normal_(0, 2.5, generator=g).to(HALF[fmt])
    t[5] = float("-inf")
    t[9, ::3] = float("-inf")
    t[11, 77] = float("nan")
    targets = torch.randint(0, V, (rows,), generator=g, device="cuda").int()
    f, top, idx, _, _ = _fwd(t, targets, V, k, fmt)
    stats = f[2:].reshape(-1)[:2 * rows].view(rows, 2)
    tol = 2 * (V / 64 + 64 + 40) * U
    for lo, n in ((0, 700), (3000, 700), (5, 1), (9, 4), (4095, 1), (100, 33)):
        pf, ptop, pidx, _, _ = _fwd(t[lo:lo + n], targets[lo:lo + n], V, k, fmt)
        assert torch.equal(pidx[:n * k], idx[lo * k:(lo + n) * k])
        for a, b, size in ((pf[0, :n], f[0, lo:lo + n], 30.0), (pf[1, :n], f[1, lo:lo + n], 30.0),
                           (ptop[:n * k], top[lo * k:(lo + n) * k], 30.0),
                           (pf[2:].reshape(-1)[:2 * n].view(n, 2)[:, 1], stats[lo:lo + n, 1], 30.0)):
            assert torch.equal(torch.isfinite(a), torch.isfinite(b))
            ok = torch.isfinite(a)
            assert torch.equal(a[~ok].isnan(), b[~ok].isnan())
            assert ok.sum() == 0 or float((a[ok] - b[ok]).abs().max()) <= tol * size


@pytest.mark.parametrize("fmt, rows, V", [("bf16", 4100, 33001), ("f16", 16400, 8200), ("f32", 2100, 32777)])
def test_logits_past_the_cache(fmt, rows, V):
    """Logits whose size sends them around the last-level cache, against calls on
    few of their rows: the alternatives and, from the same statistics, the
    gradients are the same bits, in place too."""
    k = 3
    g = torch.Generator(device="cuda").manual_seed(rows)
    t = torch.empty(rows, V, device="cuda").normal_(0, 2.5, generator=g).to(HALF[fmt])
    targets = torch.randint(0, V, (rows,), generator=g, device="cuda").int()
    f, top, idx, _, _ = _fwd(t, targets, V, k, fmt)
    stats = f[2:].reshape(-1)[:2 * rows].view(rows, 2)
    gl, ge = (torch.empty(rows, device="cuda").normal_(generator=g) for _ in range(2))
    gt = torch.empty(rows, k, device="cuda").normal_(generator=g)
    ent, ix = f[1, :rows].contiguous(), idx[:rows * k].view(rows, k)

    def bwd(z, out, lo, n):
        s = slice(lo, lo + n)
        args = [a[s].contiguous() for a in (targets, stats, ent, ix, gl, ge, gt)]
        tg, st, en, i, a, b, c = (x.data_ptr() for x in args)
        mx.mpx_logprob_bwd(z.data_ptr(), V, tg, n, V, k, st, en, i, a, b, c, None, out.data_ptr(), V,
                           mx.DTYPES[fmt], _s())
        torch.cuda.synchronize()
    dz = torch.full((rows + 1, V), -7.0, dtype=HALF[fmt], device="cuda")
    bwd(t, dz, 0, rows)
    assert (dz[rows] == -7.0).all()
    for lo, n in ((0, 3), (1000, 17), (rows - 4, 4)):
        pf, ptop, pidx, _, _ = _fwd(t[lo:lo + n], targets[lo:lo + n], V, k, fmt)
        assert torch.equal(pidx[:n * k], idx[lo * k:(lo + n) * k])
        tol = 2 * (V / 64 + 64 + 40) * U * 30.0
        assert float((pf[:2, :n] - f[:2, lo:lo + n]).abs().max()) <= tol
        part = torch.empty(n, V, dtype=HALF[fmt], device="cuda")
        bwd(t[lo:lo + n], part, lo, n)
        assert torch.equal(part, dz[lo:lo + n])
    bwd(t, t, 0, rows)
    assert torch.equal(t, dz[:rows])


@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("V", [300, 5000, 100001])
def test_spoilt_rows_without_a_target(fmt, V):
    """NaN or +inf in a row that has no target: logp stays 0, every other float
    result is NaN (one wave, one workgroup and several per row)."""
    rows, k = 4, 3
    rng = np.random.default_rng(V)
    z = round_to(rng.normal(0, 2, (rows, V)), fmt).astype(np.float64)
    z[0, 7], z[1, V - 1], z[2, 0] = np.nan, np.inf, np.nan
    z[2, 5] = np.inf
    targets = torch.tensor([-1, -5, 2, -1], dtype=torch.int32, device="cuda")
    f, _ = _check_forward(z, _upload(z, fmt), targets, k, fmt)
    logp = _np(f[0, :rows])
    assert logp[0] == logp[1] == logp[3] == 0.0 and np.isnan(logp[2])
    assert np.isnan(_np(f[1, :3])).all() and np.isnan(_stats(f, rows)[:3]).all()
