"""Gated feed-forward projections on the GPU against the float64 oracle."""
import numpy as np
import pytest

from oracle import gated
from oracle.numfmt import round_to
from tests.gpu_util import HAVE_GPU, assert_within, gemm_bound, to_host, ulp

pytestmark = [pytest.mark.gpu, pytest.mark.skipif(not HAVE_GPU, reason="no GPU")]

if HAVE_GPU:
    import torch
    from paper_2507_03312_amd import binding as mx
    TYPES = {"f16": torch.float16, "bf16": torch.bfloat16, "f32": torch.float32}
    ACTS = {"silu": mx.MPX_ACT_SILU, "gelu": mx.MPX_ACT_GELU_TANH}

FMTS = ["f16", "bf16"]


def _s():
    return torch.cuda.current_stream().cuda_stream


def _dev(a, fmt, off=0):
    """On the GPU, `off` elements past a 256-byte boundary."""
    buf = torch.empty(a.size + off, dtype=TYPES[fmt], device="cuda")
    t = buf[off:].view(a.shape)
    t.copy_(torch.from_numpy(np.ascontiguousarray(a, np.float32)))
    return t


def _ptr(t):
    return None if t is None else t.data_ptr()


def _guarded(shape, fmt, off=0):
    """An output with 64 marked values on each side, `off` elements past a 256-byte boundary."""
    n = int(np.prod(shape))
    buf = torch.full((n + 256 + off,), -7.0, dtype=TYPES[fmt], device="cuda")
    return buf, buf[128 + off:128 + off + n].view(shape)


def _untouched(buf, out):
    lo = (out.data_ptr() - buf.data_ptr()) // buf.element_size()
    assert (buf[:lo] == -7.0).all() and (buf[lo + out.numel():] == -7.0).all()


def _act_error(act, x):
    """Errors of act and act' in float32 on the hardware exp2 and reciprocal: sigma's
    argument is rounded to 2^-22 of itself, exp2, the sum and the reciprocal to 2^-22
    each, so sigma to (|arg| + 8) 2^-22; act' adds up sigma and x sigma (1 - sigma) arg',
    three more roundings."""
    s = gated.sigma(act, x)
    arg, darg = gated.argument(act, x)
    rel = (np.abs(arg) + 8.0) * 2.0 ** -22
    return np.abs(x) * s * rel, (s + np.abs(x * darg) * s) * 2.0 * rel


def _forward_bounds(x, w, b, ref, pre, act, fmt):
    """The sums are off by two float32 orders; H by the sums' errors times its slopes
    (|act'| <= 1.13), act's own and the product's rounding, and half a step."""
    K = x.shape[1]
    d = 2.0 * (K + 1) * 2.0 ** -24 * (np.abs(x.astype(np.float64)) @ np.abs(w.astype(np.float64)).T
                                      + (0 if b is None else np.abs(b)))
    (g, u), (dg, du) = np.split(pre, 2, axis=1), np.split(d, 2, axis=1)
    a, _ = gated.activation(act, g)
    ea, _ = _act_error(act, g)
    e = 1.13 * dg * (np.abs(u) + du) + (np.abs(a) + ea) * du + ea * np.abs(u) + 2.0 ** -22 * np.abs(ref)
    half = 0.5 * (1 + 2.0 ** -10)
    return half * ulp(ref, fmt) + e, half * ulp(pre, fmt) + d


def _inputs(M, N, K, fmt, bias, seed=0):
    rng = np.random.default_rng(M * 31 + N * 7 + K + seed)
    x = round_to(rng.normal(0, 1, (M, K)), fmt)
    w = round_to(rng.normal(0, K ** -0.5, (2 * N, K)), fmt)
    b = round_to(rng.normal(0, 0.3, 2 * N), fmt) if bias else None
    return x, w, b


# few rows; direct tiles of each size; ragged edges; register-staged ones; rows of < 8
SHAPES = [(1, 1, 1), (1, 17, 40), (3, 64, 5), (4, 96, 768), (32, 130, 200), (33, 64, 64), (31, 33, 7),
          (64, 5, 3), (65, 31, 128), (100, 77, 192), (130, 257, 64), (257, 129, 320), (300, 40, 75),
          (1030, 100, 588), (2100, 1100, 128), (1500, 320, 76), (4200, 2050, 64)]


@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("act, bias, keep", [("silu", False, True), ("gelu", True, True), ("silu", True, False)])
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "x".join(map(str, s)))
def test_gated_fwd(fmt, act, bias, keep, shape):
    M, N, K = shape
    x, w, b = _inputs(M, N, K, fmt, bias)
    ref, pre = gated.forward(x, w, b, act)
    bh, bp = _forward_bounds(x, w, b, ref, pre, act, fmt)
    for off in (0, 1):
        xt, wt = _dev(x, fmt, off), _dev(w, fmt, off)
        bt = None if b is None else _dev(b, fmt, off)
        hb, h = _guarded((M, N), fmt, off)
        pb, p = _guarded((M, 2 * N), fmt, off) if keep else (None, None)
        mx.mpx_gated_fwd(xt.data_ptr(), wt.data_ptr(), _ptr(bt), h.data_ptr(), _ptr(p), M, N, K,
                         mx.DTYPES[fmt], ACTS[act], _s())
        assert_within(to_host(h), ref, bh, f"H, {off} past alignment")
        _untouched(hb, h)
        if keep:
            assert_within(to_host(p), pre, bp, f"Pre, {off} past alignment")
            _untouched(pb, p)


# M, N (out), K (the hidden width)
BWD = [(1, 1, 1), (3, 5, 6), (40, 64, 64), (65, 128, 100), (129, 70, 131), (257, 192, 264), (1000, 64, 72),
       (2100, 128, 1100), (4200, 64, 2050), (700, 588, 320)]


@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("act", ["silu", "gelu"])
@pytest.mark.parametrize("shape", BWD, ids=lambda s: "x".join(map(str, s)))
def test_linear_bwd_gated(fmt, act, shape):
    M, N, K = shape
    rng = np.random.default_rng(M + N + K)
    pre = round_to(rng.normal(0, 1.5, (M, 2 * K)), fmt)
    h = round_to(rng.normal(0, 1, (M, K)), fmt)
    w = round_to(rng.normal(0, K ** -0.5, (N, K)), fmt)
    dy = round_to(rng.normal(0, 1, (M, N)), fmt)
    dh = dy.astype(np.float64) @ w.astype(np.float64)
    ref = gated.backward(dh, pre, act)
    g, u = np.split(pre.astype(np.float64), 2, axis=1)
    a, d = gated.activation(act, g)
    ea, ed = _act_error(act, g)
    e = 2.0 * N * 2.0 ** -24 * (np.abs(dy.astype(np.float64)) @ np.abs(w.astype(np.float64)))
    err = np.concatenate([np.abs(u) * (e * (np.abs(d) + ed) + np.abs(dh) * ed), e * (np.abs(a) + ea) + np.abs(dh) * ea],
                         axis=1)
    bound = 0.5 * (1 + 2.0 ** -10) * ulp(ref, fmt) + err + 2.0 ** -22 * np.abs(ref)
    for off in (0, 1):
        ht, wt, yt, pt = (_dev(v, fmt, off) for v in (h, w, dy, pre))
        buf, dpre = _guarded((M, 2 * K), fmt, off)
        dw, db = (torch.full(s, -7.0, dtype=TYPES[fmt], device="cuda") for s in ((N, K), (N,)))
        ws = torch.empty(mx.mpx_linear_bwd_gated_workspace(M, N, K), dtype=torch.uint8, device="cuda")
        mx.mpx_linear_bwd_gated(ht.data_ptr(), wt.data_ptr(), yt.data_ptr(), pt.data_ptr(), ACTS[act],
                                dpre.data_ptr(), dw.data_ptr(), db.data_ptr(), M, N, K, mx.DTYPES[fmt],
                                ws.data_ptr(), ws.numel(), None, _s())
        assert_within(to_host(dpre), ref, bound, f"dPre, {off} past alignment")
        _untouched(buf, dpre)
        assert_within(to_host(dw), dy.astype(np.float64).T @ h,
                      gemm_bound(dy.T, h, dy.astype(np.float64).T @ h, fmt, M), "dW")
        assert_within(to_host(db), dy.astype(np.float64).sum(0),
                      gemm_bound(dy.T, np.ones((M, 1)), dy.astype(np.float64).sum(0)[:, None], fmt, M)[:, 0], "db")
        only = torch.empty_like(dpre)   # each output alone: the same bits
        mx.mpx_linear_bwd_gated(None, wt.data_ptr(), yt.data_ptr(), pt.data_ptr(), ACTS[act], only.data_ptr(),
                                None, None, M, N, K, mx.DTYPES[fmt], None, 0, None, _s())
        assert torch.equal(only, dpre)


@pytest.mark.parametrize("act", ["silu", "gelu"])
def test_float32(act):
    """Full precision: sums of two float32 orders, act to its error, nothing rounded."""
    M, N, K = 70, 45, 33
    x, w, b = _inputs(M, N, K, "f32", True)
    ref, pre = gated.forward(x, w, b, act)
    xt, wt, bt = (_dev(v, "f32") for v in (x, w, b))
    h, p = torch.empty(M, N, device="cuda"), torch.empty(M, 2 * N, device="cuda")
    mx.mpx_gated_fwd(xt.data_ptr(), wt.data_ptr(), bt.data_ptr(), h.data_ptr(), p.data_ptr(), M, N, K, mx.MPX_F32,
                     ACTS[act], _s())
    bh, bp = _forward_bounds(x, w, b, ref, pre, act, "f32")
    assert_within(to_host(h), ref, bh, "H")
    assert_within(to_host(p), pre, bp, "Pre")
    pre32 = to_host(p)
    rng = np.random.default_rng(5)
    dy, w2 = (rng.normal(0, 1, s).astype(np.float32) for s in ((M, K), (K, N)))
    dh = dy.astype(np.float64) @ w2
    want = gated.backward(dh, pre32, act)
    dp, dw, db = torch.empty(M, 2 * N, device="cuda"), torch.empty(K, N, device="cuda"), torch.empty(K, device="cuda")
    ws = torch.empty(mx.mpx_linear_bwd_gated_workspace(M, K, N), dtype=torch.uint8, device="cuda")
    w2t, dyt = _dev(w2, "f32"), _dev(dy, "f32")
    mx.mpx_linear_bwd_gated(h.data_ptr(), w2t.data_ptr(), dyt.data_ptr(), p.data_ptr(),
                            ACTS[act], dp.data_ptr(), dw.data_ptr(), db.data_ptr(), M, K, N, mx.MPX_F32,
                            ws.data_ptr(), ws.numel(), None, _s())
    g, u = np.split(pre32.astype(np.float64), 2, axis=1)
    (a, d), (ea, ed) = gated.activation(act, g), _act_error(act, g)
    e = 2.0 * K * 2.0 ** -24 * (np.abs(dy) @ np.abs(w2).astype(np.float64))
    err = np.concatenate([np.abs(u) * (e * (np.abs(d) + ed) + np.abs(dh) * ed), e * (np.abs(a) + ea) + np.abs(dh) * ea],
                         axis=1) + 2.0 ** -22 * np.abs(want)
    assert_within(to_host(dp), want, err, "dPre")
    assert_within(to_host(dw), dy.astype(np.float64).T @ to_host(h),
                  gemm_bound(dy.T, to_host(h), dy.astype(np.float64).T @ to_host(h), "f32", M), "dW")


@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("M", [5, 70])
def test_not_finite_values_stay_in_their_rows(fmt, M):
    """A NaN or infinity of X reaches its own row of H only; one of a W row its column."""
    N, K = 40, 64
    x, w, _ = _inputs(M, N, K, fmt, False)
    x[2, 3], w[N + 7, 5] = np.inf, np.nan
    xt, wt = _dev(x, fmt), _dev(w, fmt)
    h = torch.empty(M, N, dtype=TYPES[fmt], device="cuda")
    mx.mpx_gated_fwd(xt.data_ptr(), wt.data_ptr(), None, h.data_ptr(), None, M, N, K, mx.DTYPES[fmt], ACTS["silu"],
                     _s())
    bad = ~np.isfinite(to_host(h))
    want = np.zeros((M, N), bool)
    want[:, 7] = True
    assert np.array_equal(np.delete(bad, 2, axis=0), np.delete(want, 2, axis=0)) and bad[2].mean() > 0.9


def test_side_stream_and_graph():
    """A captured call, replayed on new inputs, beside the same call on another stream."""
    M, N, K = 300, 200, 128
    x, w, _ = _inputs(M, N, K, "bf16", False)
    xt, wt = _dev(x, "bf16"), _dev(w, "bf16")
    hs = [torch.empty(M, N, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    ps = [torch.empty(M, 2 * N, dtype=torch.bfloat16, device="cuda") for _ in range(2)]

    def call(i, stream):
        mx.mpx_gated_fwd(xt.data_ptr(), wt.data_ptr(), None, hs[i].data_ptr(), ps[i].data_ptr(), M, N, K,
                         mx.MPX_BF16, mx.MPX_ACT_SILU, stream)
    g = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(g):
        call(0, _s())
    side = torch.cuda.Stream()
    for i in range(4):
        xt.copy_(torch.randn(M, K, device="cuda"))
        torch.cuda.synchronize()
        with torch.cuda.stream(side):
            call(1, side.cuda_stream)
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(hs[0], hs[1]) and torch.equal(ps[0], ps[1]), i


def test_rows_past_32_bits():
    """Outputs and inputs whose last rows lie past 2^31 elements equal those of the same
    rows in a call of their own."""
    M, N, K = 262400, 4096, 64     # Pre: 2.15e9 elements
    g = torch.Generator(device="cuda").manual_seed(1)
    x = torch.empty(M, K, dtype=torch.bfloat16, device="cuda").normal_(generator=g)
    w = torch.empty(2 * N, K, dtype=torch.bfloat16, device="cuda").normal_(0, 0.1, generator=g)
    h, p = (torch.empty(M, n, dtype=torch.bfloat16, device="cuda") for n in (N, 2 * N))
    mx.mpx_gated_fwd(x.data_ptr(), w.data_ptr(), None, h.data_ptr(), p.data_ptr(), M, N, K, mx.MPX_BF16,
                     mx.MPX_ACT_SILU, _s())
    lo, n = M - 300, 300
    h1, p1 = torch.empty(n, N, dtype=h.dtype, device="cuda"), torch.empty(n, 2 * N, dtype=h.dtype, device="cuda")
    mx.mpx_gated_fwd(x[lo:].data_ptr(), w.data_ptr(), None, h1.data_ptr(), p1.data_ptr(), n, N, K, mx.MPX_BF16,
                     mx.MPX_ACT_SILU, _s())
    assert torch.equal(h[lo:], h1) and torch.equal(p[lo:], p1)
