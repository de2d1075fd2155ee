"""8-bit activation checkpoints on the GPU against the float64 oracle: packing
byte for byte over every half value, widening bit for bit, and the linear
backward that reads checkpoints against float64 products."""
import numpy as np
import pytest

from oracle import act8, ops
from oracle.numfmt import round_to
from oracle.policy import Policy
from tests.gpu_util import HAVE_GPU, assert_within, gemm_bound, to_dev_half, to_host, ulp

pytestmark = [pytest.mark.gpu, pytest.mark.skipif(not HAVE_GPU, reason="no GPU")]

if HAVE_GPU:
    import torch
    from paper_2507_03312_amd import binding as mx
    from tests.gpu_util import TORCH_HALF

FMTS = ["f16", "bf16"]
FILL = 0xA5


def _s():
    return torch.cuda.current_stream().cuda_stream


def _bytes(n):
    return torch.full((n,), FILL, dtype=torch.uint8, device="cuda")


def _pack(x, fmt, ldx=None, off=0):
    """Packed codes and scales of the half tensor x (row stride ldx), with 64
    bytes behind each that must stay as they were; codes start at byte `off`."""
    M, K = x.shape
    ldx = ldx or x.stride(0)
    nc, ns = M * K, -(-M // 32) * K
    c, s = _bytes(off + nc + 64), _bytes(off + ns + 64)
    mx.mpx_act8_pack(x.data_ptr(), ldx, c.data_ptr() + off, s.data_ptr() + off, M, K, mx.DTYPES[fmt], _s())
    torch.cuda.synchronize()
    for t, n in ((c, nc), (s, ns)):
        assert (t[:off] == FILL).all() and (t[off + n:] == FILL).all()
    return c[off:off + nc].view(M, K), s[off:off + ns].view(-1, K)


def _check_pack(x, fmt, c, s):
    rc, re = act8.pack(to_host(x), fmt)
    assert np.array_equal(s.cpu().numpy(), (re + 127).astype(np.uint8))
    assert np.array_equal(c.cpu().numpy() & 0x7F, act8.code_bytes(rc) & 0x7F)
    signs = ~np.isnan(rc)   # the sign of a NaN code says nothing
    assert np.array_equal(c.cpu().numpy()[signs], act8.code_bytes(rc)[signs])
    return rc, re


@pytest.mark.parametrize("fmt", FMTS)
def test_pack_every_half_value(fmt):
    """All 65536 patterns, each in a group whose largest value is 0, 1 (the
    pattern scales the group itself where it is larger), about 450 (both sides
    of a power of two's last code) or the format's largest value."""
    bits = torch.arange(65536, dtype=torch.int32).to(torch.int16).view(TORCH_HALF[fmt])
    for amax in (0.0, 1.0, 448.0, 452.0, 3.0e-5, 65504.0 if fmt == "f16" else 3.0e38):
        x = torch.zeros(32, 65536, dtype=TORCH_HALF[fmt])
        x[7] = bits
        x[19] = amax
        x = x.cuda()
        c, s = _pack(x, fmt)
        rc, re = act8.pack(to_host(x)[[7, 19]], fmt)
        assert np.array_equal(s.cpu().numpy()[0], (re[0] + 127).astype(np.uint8))
        got, want = c.cpu().numpy()[7], act8.code_bytes(rc)[0]
        nan = np.isnan(rc[0])
        assert np.array_equal(got[~nan], want[~nan]) and np.all((got[nan] & 0x7F) == 0x7F)


@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("mk", [(1, 1), (1, 7), (31, 3), (32, 8), (33, 16), (64, 256), (95, 257), (200, 588),
                                (129, 1024), (1000, 72), (7, 4096), (4099, 33)],
                         ids=lambda s: "x".join(map(str, s)))
def test_pack_and_unpack(fmt, mk):
    M, K = mk
    rng = np.random.default_rng(M * 1000 + K)
    mag = np.exp2(rng.integers(-20, 10, (1, K)))
    x = round_to(rng.normal(0, 1, (M, K)) * mag, fmt)
    x[rng.random((M, K)) < 0.01] = 0.0
    if M > 3:
        x[1, 0], x[2, K // 2], x[M - 1, K - 1] = np.inf, np.nan, -np.inf
    for extra, off in ((0, 0), (5, 3)):   # dense; a strided x and odd byte addresses
        buf = torch.zeros(M * (K + extra) + 1, dtype=TORCH_HALF[fmt], device="cuda")
        xt = buf[(1 if extra else 0):][:M * (K + extra)].view(M, K + extra)[:, :K]
        xt.copy_(to_dev_half(x, fmt))
        c, s = _pack(xt, fmt, K + extra, off)
        rc, re = _check_pack(xt, fmt, c, s)
        ref = act8.values(rc, re)
        y = torch.full((M + 1, K + extra), -7.0, dtype=TORCH_HALF[fmt], device="cuda")
        mx.mpx_act8_unpack(c.data_ptr(), s.data_ptr(), y.data_ptr(), K + extra, M, K, mx.DTYPES[fmt], _s())
        assert np.array_equal(to_host(y[:M, :K]), ref.astype(np.float32), equal_nan=True)
        assert (y[M:] == -7.0).all() and (y[:, K:] == -7.0).all()


def _problem(fmt, M, N, K, seed=0):
    rng = np.random.default_rng(seed + M + 7 * N + 13 * K)
    pre = round_to(rng.normal(0, 1.5, (M, K)) * np.where(rng.random((1, K)) < 0.05, 20.0, 1.0), fmt)
    x = round_to(rng.normal(0, 1, (M, K)), fmt)
    w = round_to(rng.normal(0, 0.05, (N, K)), fmt)
    dy = round_to(rng.normal(0, 1, (M, N)), fmt)
    return x, pre, w, dy


def _run(fmt, M, N, K, x, pre, w, dy, act, want="xwb", off=0, counter=True):
    """mpx_linear_bwd_act8 on packed x and pre; the outputs' neighbours and the
    workspace's end are checked to be left alone."""
    dt, h = mx.DTYPES[fmt], TORCH_HALF[fmt]
    xc, xs = _pack(to_dev_half(x, fmt), fmt, off=off)
    pc, ps = _pack(to_dev_half(pre, fmt), fmt, off=off)
    tw, tdy = to_dev_half(w, fmt), to_dev_half(dy, fmt)
    dx, dw, db = (torch.full((n + 8,), -7.0, dtype=h, device="cuda") for n in (M * K, N * K, N))
    need = mx.mpx_linear_bwd_act8_workspace(M, N, K)
    ws = _bytes(need + 256)
    nf = torch.zeros(1, dtype=torch.int32, device="cuda")
    mx.mpx_linear_bwd_act8(xc.data_ptr(), xs.data_ptr(), tw.data_ptr(), tdy.data_ptr(), pc.data_ptr(),
                           ps.data_ptr(), act, dx.data_ptr() if "x" in want else None,
                           dw.data_ptr() if "w" in want else None, db.data_ptr() if "b" in want else None,
                           M, N, K, dt, ws.data_ptr(), need, nf.data_ptr() if counter else None, _s())
    torch.cuda.synchronize()
    assert (ws[need:] == FILL).all()
    for t, n, c in ((dx, M * K, "x"), (dw, N * K, "w"), (db, N, "b")):
        assert (t[n if c in want else 0:] == -7.0).all()
    xv = act8.values(act8.byte_values(xc.cpu().numpy()), xs.cpu().numpy().astype(np.int64) - 127)
    pv = act8.values(act8.byte_values(pc.cpu().numpy()), ps.cpu().numpy().astype(np.int64) - 127)
    return dx[:M * K].view(M, K), dw[:N * K].view(N, K), db[:N], int(nf.item()), xv, pv


SHAPES = [(1, 1, 1), (1, 64, 128), (5, 3, 9), (31, 64, 64), (33, 128, 128), (64, 512, 1024), (65, 40, 24),
          (128, 10, 384), (257, 136, 144), (1000, 96, 588), (2048, 768, 384), (2500, 200, 136),
          (4097, 72, 264), (8320, 384, 256), (63, 64, 128), (65, 72, 144), (97, 8, 16), (2049, 64, 16),
          (1537, 136, 400), (4099, 200, 272), (5000, 1032, 48), (2056, 2056, 1040), (700, 2568, 2576),
          (3300, 2056, 1040)]


@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("mnk", SHAPES, ids=lambda s: "x".join(map(str, s)))
def test_linear_bwd_act8(fmt, mnk):
    """Against float64 products of the checkpoints' values: one rounding of each
    output plus two float32 summation orders; dX through GELU' adds its own
    rounding, with the product's bound scaled by |gelu'| <= 1.13."""
    M, N, K = mnk
    pol = Policy(fmt)
    x, pre, w, dy = _problem(fmt, M, N, K)
    for act in (mx.MPX_ACT_NONE, mx.MPX_ACT_GELU_TANH):
        dx, dw, db, bad, xv, pv = _run(fmt, M, N, K, x, pre, w, dy, act, off=0 if act else 3)
        rdx, rdw, rdb = ops.linear_bwd(pol, xv, w, dy)
        bound = gemm_bound(dy, w, rdx, fmt, N)
        if act:
            rdx = ops.gelu_bwd(pol, pv, rdx)
            bound = 1.13 * bound + ulp(rdx, fmt)
        assert_within(to_host(dx), rdx, bound, "dX")
        assert_within(to_host(dw), rdw, gemm_bound(dy.T, xv, rdw, fmt, M), "dW")
        colb = ulp(rdb, fmt) + 2.0 * M * 2.0 ** -24 * np.abs(dy.astype(np.float64)).sum(axis=0)
        assert_within(to_host(db), rdb, colb, "db")
        assert bad == 0


@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("off", [0, 3], ids=["aligned", "any"])
@pytest.mark.parametrize("mnk", [(100, 72, 65), (70, 33, 131), (2100, 136, 133), (2049, 79, 135), (130, 65, 260),
                                 (4223, 79, 131)], ids=lambda s: "x".join(map(str, s)))
def test_fewer_than_8_columns_in_the_last_tile(fmt, mnk, off):
    """Vectors that reach back from the last column over the tile's first one: dW
    and db against float64 products, one rounding and two float32 orders."""
    M, N, K = mnk
    x, pre, w, dy = _problem(fmt, M, N, K, 6)
    _, dw, db, bad, xv, _ = _run(fmt, M, N, K, x, pre, w, dy, mx.MPX_ACT_NONE, "wb", off=off)
    _, rdw, rdb = ops.linear_bwd(Policy(fmt), xv, w, dy)
    assert_within(to_host(dw), rdw, gemm_bound(dy.T, xv, rdw, fmt, M), "dW")
    colb = ulp(rdb, fmt) + 2.0 * M * 2.0 ** -24 * np.abs(dy.astype(np.float64)).sum(axis=0)
    assert_within(to_host(db), rdb, colb, "db")
    assert bad == 0


@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("off", [0, 3], ids=["aligned", "any"])
@pytest.mark.parametrize("mnk", [(449, 64, 128), (1672, 320, 192), (2050, 64, 16), (3089, 8, 8), (4223, 79, 131),
                                 (2471, 287, 267), (4161, 64, 61), (3000, 6, 9)],
                         ids=lambda s: "x".join(map(str, s)))
def test_short_splits(fmt, mnk, off):
    """Reductions of a few k tiles each in many splits, the last one shorter: dW
    and db against float64 products, one rounding and two float32 orders."""
    M, N, K = mnk
    x, pre, w, dy = _problem(fmt, M, N, K, 4)
    _, dw, db, bad, xv, _ = _run(fmt, M, N, K, x, pre, w, dy, mx.MPX_ACT_NONE, "wb", off=off)
    _, rdw, rdb = ops.linear_bwd(Policy(fmt), xv, w, dy)
    assert_within(to_host(dw), rdw, gemm_bound(dy.T, xv, rdw, fmt, M), "dW")
    colb = ulp(rdb, fmt) + 2.0 * M * 2.0 ** -24 * np.abs(dy.astype(np.float64)).sum(axis=0)
    assert_within(to_host(db), rdb, colb, "db")
    assert bad == 0


@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("wide", ["N", "K"])
def test_every_width(fmt, wide):
    """dX through GELU', dW and db at every width up to past the widest tile, with
    bounds as in test_linear_bwd_act8."""
    for n in range(1, 150):
        M, (N, K) = (33, 70)[n % 2], (n, 41) if wide == "N" else (24, n)
        x, pre, w, dy = _problem(fmt, M, N, K, 7)
        dx, dw, db, bad, xv, pv = _run(fmt, M, N, K, x, pre, w, dy, mx.MPX_ACT_GELU_TANH, off=n % 3)
        pol = Policy(fmt)
        rdx, rdw, rdb = ops.linear_bwd(pol, xv, w, dy)
        bound = 1.13 * gemm_bound(dy, w, rdx, fmt, N)
        rdx = ops.gelu_bwd(pol, pv, rdx)
        assert_within(to_host(dx), rdx, bound + ulp(rdx, fmt), f"dX {n}")
        assert_within(to_host(dw), rdw, gemm_bound(dy.T, xv, rdw, fmt, M), f"dW {n}")
        colb = ulp(rdb, fmt) + 2.0 * M * 2.0 ** -24 * np.abs(dy.astype(np.float64)).sum(axis=0)
        assert_within(to_host(db), rdb, colb, f"db {n}")
        assert bad == 0


@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("mnk", [(1100, 128, 256), (333, 72, 40), (64, 64, 128)],
                         ids=lambda s: "x".join(map(str, s)))
def test_subsets_are_the_full_call(fmt, mnk):
    M, N, K = mnk
    prob = _problem(fmt, M, N, K, 1)
    full = _run(fmt, M, N, K, *prob, mx.MPX_ACT_GELU_TANH)
    for want in ("x", "w", "b", "wb", "xb"):
        part = _run(fmt, M, N, K, *prob, mx.MPX_ACT_GELU_TANH, want, counter=False)
        for i, c in enumerate("xw"):
            if c in want:
                assert torch.equal(part[i].view(torch.int16), full[i].view(torch.int16)), (want, c)
        if "b" in want:   # alone, the column sums take another order: one rounding apart at most
            a, b = to_host(part[2]), to_host(full[2])
            order = 2.0 * M * 2.0 ** -24 * np.abs(prob[3].astype(np.float64)).sum(axis=0)
            assert np.all(np.abs(a - b) <= ulp(b, fmt) + order)


@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("mnk", [(2048, 128, 128), (100, 64, 128), (77, 33, 50)],
                         ids=lambda s: "x".join(map(str, s)))
def test_overflow_reaches_the_finite_check(fmt, mnk):
    """inf and NaN activations come out of the checkpoint as NaN in exactly their
    column of dW, and the counter adds what the separate check counts."""
    M, N, K = mnk
    x, pre, w, dy = _problem(fmt, M, N, K, 2)
    x[3, 5], x[M - 1, K - 1] = np.inf, np.nan
    dx, dw, db, bad, _, _ = _run(fmt, M, N, K, x, pre, w, dy, mx.MPX_ACT_NONE)
    g = to_host(dw)
    cols = np.flatnonzero(np.isnan(g).all(axis=0))
    assert cols.tolist() == [5, K - 1] and np.isfinite(np.delete(g, [5, K - 1], axis=1)).all()
    ref = torch.zeros(1, dtype=torch.int32, device="cuda")
    mx.mpx_unscale_check(mx.TensorList([dw.contiguous(), db.contiguous()]), mx.DTYPES[fmt], 0, ref.data_ptr(),
                         None, _s())
    assert bad == int(ref.item()) == 2 * N
    assert np.isfinite(to_host(dx)).all()


@pytest.mark.parametrize("fmt", FMTS)
def test_extreme_scales_in_the_product(fmt):
    """Groups at the least and the largest exponent widen exactly on the way to
    the matrix cores: dW against float64 products of the checkpoint's values."""
    M, N, K = 192, 64, 128
    rng = np.random.default_rng(9)
    x = rng.normal(0, 1, (M, K))
    tiny, big = (2.0 ** -18, 2.0 ** 14) if fmt == "f16" else (2.0 ** -112, 2.0 ** 100)
    x[:, :32] *= tiny
    x[:, 32:64] *= big / 4
    x[0, 40] = 65504.0 if fmt == "f16" else 3.3e38   # the largest exponent; held as 240 codes
    x = round_to(x, fmt)
    _, pre, w, dy = _problem(fmt, M, N, K, 3)
    dy = round_to(dy * 2.0 ** -7, fmt)
    _, dw, _, _, xv, _ = _run(fmt, M, N, K, x, pre, w, dy, mx.MPX_ACT_NONE)
    ref64 = dy.astype(np.float64).T @ xv
    rdw = round_to(ref64, fmt)
    ok = np.isfinite(rdw)
    bound = gemm_bound(dy.T, xv, np.where(ok, rdw, 0), fmt, M)
    got = to_host(dw).astype(np.float64)
    near_max = np.abs(ref64) > (60000.0 if fmt == "f16" else 3.0e38)
    assert np.all((np.abs(got - rdw.astype(np.float64)) <= bound)[ok & ~near_max])


@pytest.mark.parametrize("fmt", FMTS)
def test_graph_replays_with_fresh_data(fmt):
    """Pack and backward captured on a side stream and replayed on new data,
    with eager calls in between: every replay is the eager result."""
    M, N, K = 520, 128, 256
    dt, h = mx.DTYPES[fmt], TORCH_HALF[fmt]
    x = torch.zeros(M, K, dtype=h, device="cuda")
    dy = torch.zeros(M, N, dtype=h, device="cuda")
    w = (torch.randn(N, K, device="cuda") * 0.05).to(h)
    c, s = _bytes(M * K), _bytes(-(-M // 32) * K)
    out = [torch.zeros(n, dtype=h, device="cuda") for n in (M * K, N * K, N)]
    need = mx.mpx_linear_bwd_act8_workspace(M, N, K)

    def call(o, ws, st):
        mx.mpx_act8_pack(x.data_ptr(), K, c.data_ptr(), s.data_ptr(), M, K, dt, st)
        mx.mpx_linear_bwd_act8(c.data_ptr(), s.data_ptr(), w.data_ptr(), dy.data_ptr(), c.data_ptr(),
                               s.data_ptr(), mx.MPX_ACT_GELU_TANH, o[0].data_ptr(), o[1].data_ptr(),
                               o[2].data_ptr(), M, N, K, dt, ws.data_ptr(), need, None, st)
    ws = [_bytes(need) for _ in range(2)]
    g = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(g):
        call(out, ws[0], _s())
    for i in range(4):
        x.copy_(torch.randn(M, K, device="cuda") * (i + 1))
        dy.copy_(torch.randn(M, N, device="cuda"))
        eager = [torch.zeros_like(o) for o in out]
        call(eager, ws[1], _s())
        g.replay()
        torch.cuda.synchronize()
        for a, b in zip(out, eager):
            assert torch.equal(a.view(torch.int16), b.view(torch.int16)), i


@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("config", [1, 2, 3, 5, 7, 9])
@pytest.mark.parametrize("mnk", [(512, 128, 768), (300, 192, 392), (65, 64, 72), (257, 128, 999)],
                         ids=lambda s: "x".join(map(str, s)))
def test_gelu_backward_on_every_tile(fmt, config, mnk):
    """dX through GELU' from a checkpoint against mpx_linear_bwd on its widened
    values, on each tile shape (whole tiles, edges, partial vectors): the same
    roundings, so the same values up to one last place (the compiler may form
    the float16 product in one rounding or two)."""
    M, N, K = mnk
    x, pre, w, dy = _problem(fmt, M, N, K, config)
    pre[3, 5], pre[M - 1, K - 1], pre[:, 7] = 0.0, -30.0, 0.0
    dt, h = mx.DTYPES[fmt], TORCH_HALF[fmt]
    pc, ps = _pack(to_dev_half(pre, fmt), fmt)
    P = torch.empty(M, K, dtype=h, device="cuda")
    mx.mpx_act8_unpack(pc.data_ptr(), ps.data_ptr(), P.data_ptr(), K, M, K, dt, _s())
    tw, tdy = to_dev_half(w, fmt), to_dev_half(dy, fmt)
    a, b = (torch.full((M + 1, K), -7.0, dtype=h, device="cuda") for _ in range(2))
    mx.mpx_gemm_set_config(config)
    try:
        mx.mpx_linear_bwd_act8(None, None, tw.data_ptr(), tdy.data_ptr(), pc.data_ptr(), ps.data_ptr(),
                               mx.MPX_ACT_GELU_TANH, a.data_ptr(), None, None, M, N, K, dt, None, 0, None, _s())
        mx.mpx_linear_bwd(None, tw.data_ptr(), tdy.data_ptr(), P.data_ptr(), mx.MPX_ACT_GELU_TANH, b.data_ptr(),
                          None, None, M, N, K, dt, None, 0, None, _s())
    finally:
        mx.mpx_gemm_set_config(0)
    assert (a[M] == -7.0).all()
    ga, gb = to_host(a[:M]).astype(np.float64), to_host(b[:M]).astype(np.float64)
    assert np.all(np.abs(ga - gb) <= ulp(np.maximum(np.abs(ga), np.abs(gb)), fmt))


@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("dy_off, x_off, s_off", [(1, 0, 0), (0, 8, 0), (0, 0, 2), (8, 16, 4), (3, 5, 7)])
def test_any_address_of_the_operands(fmt, dy_off, x_off, s_off):
    """dY, codes and scales at addresses that the direct copies take and at others:
    the same sums, in one of two orders."""
    M, N, K = 1700, 136, 272
    x, pre, w, dy = _problem(fmt, M, N, K, 5)
    dt, h = mx.DTYPES[fmt], TORCH_HALF[fmt]
    xc, xs = _pack(to_dev_half(x, fmt), fmt)
    put = lambda t, off: torch.cat([torch.zeros(off, dtype=t.dtype, device="cuda"), t.reshape(-1)])
    tdy, c, s = put(to_dev_half(dy, fmt), dy_off), put(xc, x_off), put(xs, s_off)
    dw, db = torch.zeros(N, K, dtype=h, device="cuda"), torch.zeros(N, dtype=h, device="cuda")
    need = mx.mpx_linear_bwd_act8_workspace(M, N, K)
    ws = _bytes(need)
    mx.mpx_linear_bwd_act8(c.data_ptr() + x_off, s.data_ptr() + s_off, None, tdy.data_ptr() + 2 * dy_off, None, None,
                           0, None, dw.data_ptr(), db.data_ptr(), M, N, K, dt, ws.data_ptr(), need, None, _s())
    xv = act8.values(*act8.pack(x, fmt))
    _, rdw, rdb = ops.linear_bwd(Policy(fmt), xv, w, dy)
    assert_within(to_host(dw), rdw, gemm_bound(dy.T, xv, rdw, fmt, M), "dW")
    colb = ulp(rdb, fmt) + 2.0 * M * 2.0 ** -24 * np.abs(dy.astype(np.float64)).sum(axis=0)
    assert_within(to_host(db), rdb, colb, "db")


def test_offsets_past_32_bits():
    """1,100,005 rows of 2048: codes past 2^31 bytes, halves past 2^32."""
    M, N, K, h, dt = 1_100_005, 16, 2048, torch.bfloat16, mx.MPX_BF16
    g = torch.Generator(device="cuda").manual_seed(1)
    x = torch.empty(M, K, dtype=h, device="cuda").normal_(generator=g)
    dy = torch.empty(M, N, dtype=h, device="cuda").normal_(generator=g)
    w = torch.empty(N, K, dtype=h, device="cuda").normal_(generator=g)
    c, s = torch.empty(M, K, dtype=torch.uint8, device="cuda"), torch.empty(-(-M // 32), K, dtype=torch.uint8, device="cuda")
    mx.mpx_act8_pack(x.data_ptr(), K, c.data_ptr(), s.data_ptr(), M, K, dt, _s())
    r0 = (M - 70) // 32 * 32   # the last groups on their own
    ec, es = _pack(x[r0:].contiguous(), "bf16")
    assert torch.equal(c[r0:], ec) and torch.equal(s[r0 // 32:], es)
    y = torch.empty(M, K, dtype=h, device="cuda")
    mx.mpx_act8_unpack(c.data_ptr(), s.data_ptr(), y.data_ptr(), K, M, K, dt, _s())
    dx, dw, db = torch.empty(M, K, dtype=h, device="cuda"), torch.empty(N, K, dtype=h, device="cuda"), torch.empty(N, dtype=h, device="cuda")
    need = mx.mpx_linear_bwd_act8_workspace(M, N, K)
    ws = _bytes(need)
    mx.mpx_linear_bwd_act8(c.data_ptr(), s.data_ptr(), w.data_ptr(), dy.data_ptr(), c.data_ptr(), s.data_ptr(),
                           mx.MPX_ACT_GELU_TANH, dx.data_ptr(), dw.data_ptr(), db.data_ptr(), M, N, K, dt,
                           ws.data_ptr(), need, None, _s())
    ref, mag = torch.zeros(N, K, dtype=torch.float64, device="cuda"), torch.zeros(N, K, dtype=torch.float64, device="cuda")
    for r in range(0, M, 1 << 17):
        a, b = dy[r:r + (1 << 17)].double(), y[r:r + (1 << 17)].double()
        ref += a.t() @ b
        mag += a.abs().t() @ b.abs()
    # two float32 summation orders of M products, one rounding
    ref, mag = ref.cpu().numpy(), mag.cpu().numpy()
    assert np.all(np.abs(to_host(dw) - ref) <= ulp(ref, "bf16") + 2.0 * M * 2.0 ** -24 * mag)
    assert np.linalg.norm(to_host(dw) - ref) <= 2.0 ** -8 * np.linalg.norm(ref)
    # the last rows of dX, and rows across 2^31 codes, alone
    for lo in (r0, (1 << 31) // K // 32 * 32 - 64):
        n = min(128, M - lo)
        part = torch.empty(n, K, dtype=h, device="cuda")
        mx.mpx_linear_bwd(None, w.data_ptr(), dy[lo:lo + n].contiguous().data_ptr(), y[lo:lo + n].contiguous().data_ptr(),
                          mx.MPX_ACT_GELU_TANH, part.data_ptr(), None, None, n, N, K, dt, None, 0, None, _s())
        d = (dx[lo:lo + n].double() - part.double()).abs().cpu().numpy()
        assert np.all(d <= ulp(to_host(part), "bf16"))
