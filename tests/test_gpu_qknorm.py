"""Norms of queries and keys with rotary positions on the GPU against the float64 oracle."""
import numpy as np
import pytest

from oracle import qknorm, rotary
from oracle.numfmt import round_to
from tests.gpu_util import HAVE_GPU, assert_within, to_host, ulp

pytestmark = [pytest.mark.gpu, pytest.mark.skipif(not HAVE_GPU, reason="no GPU")]

if HAVE_GPU:
    import torch
    from paper_2507_03312_amd import binding as mx
    TYPES = {"f16": torch.float16, "bf16": torch.bfloat16, "f32": torch.float32}

FMTS = ["f16", "bf16", "f32"]
EPS = 1e-5


def _s():
    return torch.cuda.current_stream().cuda_stream


def _dev(a, fmt):
    return torch.from_numpy(np.ascontiguousarray(a, np.float32)).to(TYPES[fmt]).cuda()


def _ptr(t):
    return None if t is None else t.data_ptr()


def _partner_sums(m, pairs, interleaved, rot, hd):
    """|x0| + |x1| of every turned value's pair, |x| of the others."""
    m = np.abs(m).reshape(len(m), -1, hd)
    out = m.copy()
    for _, _, a, b in rotary.pair_columns(pairs, interleaved):
        out[:, :rot, a] = out[:, :rot, b] = m[:, :rot, a] + m[:, :rot, b]
    return out


def _half(ref, fmt):
    return 0.5 * (1 + 2.0 ** -10) * ulp(ref, fmt)


CASES = [
    # rows, pos_rows, queries, keys, copied, hd, pairs, far
    (1, 1, 1, 0, 0, 2, [1], 5),
    (1, 1, 32, 8, 8, 128, [16, 24, 24], 1 << 24),
    (3, 3, 2, 1, 1, 64, [16, 16], 14),
    (16, 16, 12, 4, 4, 128, [16, 24, 24], 1000000),
    (65 * 3, 65, 5, 5, 3, 80, [20, 20], 9),
    (77, 7, 3, 2, 0, 96, [8, 40], 4000),
    (50, 50, 4, 1, 2, 64, [11, 4, 1, 16], 2000000),
    (50, 25, 4, 1, 2, 64, [3, 4], 100),          # values behind the sections
    (50, 25, 4, 3, 2, 64, [8, 12], 100),
    (33, 11, 7, 2, 5, 10, [1, 1, 1, 1], 50),
    (20, 20, 2, 2, 1, 512, [256], 300),
    (1030, 1030, 2, 1, 1, 256, [64, 64], 300),
    (2600, 1300, 12, 12, 12, 64, [16, 16], 14),
    (4097, 4097, 2, 1, 1, 32, [8, 8], 64),
    (20, 10, 3, 1, 1, 130, [33, 30], 50),
    (2050, 2050, 2, 1, 1, 65, [8, 8], 9),        # an odd one
    (1030, 515, 3, 1, 2, 24, [4, 8], 9),
]


@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("interleaved", [False, True], ids=["halves", "interleaved"])
@pytest.mark.parametrize("case", CASES, ids=lambda c: "-".join(str(v).replace(" ", "") for v in c))
def test_qknorm_rope(fmt, interleaved, case):
    """Both directions, out of place and in place, dense and strided; the columns past the
    heads and the rows behind the last stay as they were.

    Bounds: r is off by hd + 8 roundings of a sum of squares, halved by the root, and
    one of its own: (hd + 16) 2^-24 of itself; a turn by 2^-20 (|n0| + |n1|); the
    products by three roundings.  Backward, the mean of w dn x likewise from the
    magnitudes it adds up.  A gain's sum has rows x heads terms."""
    rows, pos_rows, hq, hk, copy, hd, pairs, far = case
    rng = np.random.default_rng(rows + hd)
    rot = hq + hk
    base = [10000.0, 100.0, 37.5, 2.0][:len(pairs)]
    width = (rot + copy) * hd
    x, dy = (round_to(rng.normal(0, s, (rows, width)), fmt) for s in (1.5, 0.7))
    x[rows // 2, :hd] = 0.0                     # a head of nothing but zeros
    gains = [round_to(1 + rng.normal(0, 0.3, hd), fmt) for _ in range(2)]
    pos = rng.integers(0, far, (pos_rows, len(pairs))).astype(np.float32)
    pos[0] = 0.0
    plan = mx.RopePlan(pairs, base, interleaved)
    tp = torch.from_numpy(pos).cuda()
    rel = (hd + 16) * 2.0 ** -24 + 2.0 ** -20
    for wq, wk in (gains, (gains[0], None), (None, None)):
        rest = (EPS, pos, pairs, base, interleaved, hq, hk, hd)
        ref, n = qknorm.forward(x, wq, wk, *rest)
        bound = _half(ref, fmt).reshape(rows, -1, hd)
        bound[:, :rot] += rel * _partner_sums(n, pairs, interleaved, rot, hd)[:, :rot]
        bound[:, rot:] = 0.0
        dx, dwq, dwk, dn = qknorm.backward(x, dy, wq, wk, *rest)
        h, d = (v.astype(np.float64).reshape(rows, -1, hd)[:, :rot] for v in (x, dn))
        r = qknorm._root(h, EPS)
        w = np.abs(qknorm._gains(wq, wk, hq, hk, hd))
        ed = rel * _partner_sums(dy, pairs, interleaved, rot, hd)[:, :rot]
        size = np.abs(w * d * h)
        bdx = _half(dx, fmt).reshape(rows, -1, hd)
        bdx[:, :rot] += r * w * (ed + rel * np.abs(d)) + np.abs(h) * r ** 3 * (
            (w * np.abs(h) * ed).mean(-1, keepdims=True) + 3 * rel * size.mean(-1, keepdims=True))
        bdx[:, rot:] = 0.0
        terms = np.abs(d * h * r)
        chain = (rows * rot + 8) * 2.0 ** -24
        bdw = (np.abs(h) * r * ed + terms * (2 * rel + chain))
        bdw = [_half(dwq, fmt) + bdw[:, :hq].sum((0, 1)), _half(dwk, fmt) + bdw[:, hq:].sum((0, 1))]

        tq, tk = (None if g is None else _dev(g, fmt) for g in (wq, wk))
        ws = torch.empty(mx.mpx_qknorm_rope_bwd_workspace(rows, hd), dtype=torch.uint8, device="cuda")
        fwd, bwd = [], []
        for pad, off in ((0, 0), (5, 1)):
            ld = width + pad

            def strided(a):
                buf = torch.full((off + (rows + 1) * ld,), -7.0, dtype=TYPES[fmt], device="cuda")
                t = buf[off:].view(rows + 1, ld)
                t[:rows, :width] = _dev(a, fmt)
                return t

            def marked():
                return torch.full((rows + 1, width + 3), -7.0, dtype=TYPES[fmt], device="cuda")

            xt, yt, y, g = strided(x), strided(dy), marked(), marked()
            heads = (rows, hq, hk, copy, hd, plan)
            mx.mpx_qknorm_rope_fwd(xt.data_ptr(), ld, y.data_ptr(), width + 3, _ptr(tq), _ptr(tk), EPS,
                                   tp.data_ptr(), pos_rows, *heads, mx.DTYPES[fmt], _s())
            gq, gk = (torch.full((hd,), -7.0, dtype=TYPES[fmt], device="cuda") for _ in range(2))
            back = lambda o, ldo: mx.mpx_qknorm_rope_bwd(
                xt.data_ptr(), ld, yt.data_ptr(), ld, o.data_ptr(), ldo, _ptr(tq), _ptr(tk), EPS, tp.data_ptr(),
                pos_rows, *heads, gq.data_ptr(), gk.data_ptr(), mx.DTYPES[fmt], ws.data_ptr(), ws.numel(), None,
                _s())
            back(g, width + 3)
            for o in (y, g):
                assert (o[rows:] == -7.0).all() and (o[:, width:] == -7.0).all()
            fwd.append(y[:rows, :width])
            bwd.append((g[:rows, :width], gq.clone(), gk.clone()))
            before = yt.clone()
            back(yt, ld)                          # in place
            assert torch.equal(yt[rows:], before[rows:]) and torch.equal(yt[:, width:], before[:, width:])
            bwd.append((yt[:rows, :width], gq, gk))
            mx.mpx_qknorm_rope_fwd(xt.data_ptr(), ld, xt.data_ptr(), ld, _ptr(tq), _ptr(tk), EPS, tp.data_ptr(),
                                   pos_rows, *heads, mx.DTYPES[fmt], _s())
            assert (xt[rows:] == -7.0).all() and (xt[:, width:] == -7.0).all()
            fwd.append(xt[:rows, :width])
        assert all(torch.equal(o, fwd[0]) for o in fwd)
        assert all(torch.equal(a, b) for o in bwd for a, b in zip(o, bwd[0]))
        assert_within(to_host(fwd[0]), ref, bound.reshape(rows, -1), "Y")
        for name, o, want, b in zip(("dX", "dwq", "dwk"), bwd[0], (dx, dwq, dwk),
                                    (bdx.reshape(rows, -1), *bdw)):
            assert_within(to_host(o), want, b, name)


@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("pairs", [[16, 16], [11, 4, 1, 16]], ids=["runs", "any"])
def test_not_finite_values_stay_in_their_heads(fmt, pairs):
    rows, hq, hk, copy, hd = 6, 3, 2, 1, 64
    x = torch.randn(rows, (hq + hk + copy) * hd, device="cuda").to(TYPES[fmt])
    dy = torch.randn(x.shape, device="cuda").to(TYPES[fmt])
    x[1, 2 * hd + 5], x[4, 4 * hd + 63], x[5, 5 * hd] = float("nan"), float("inf"), float("nan")
    pos = torch.ones(rows, len(pairs), device="cuda")
    plan, ld = mx.RopePlan(pairs), x.shape[1]
    y = torch.empty_like(x)
    mx.mpx_qknorm_rope_fwd(x.data_ptr(), ld, y.data_ptr(), ld, None, None, EPS, pos.data_ptr(), rows, rows, hq, hk,
                           copy, hd, plan, mx.DTYPES[fmt], _s())
    fine = torch.isfinite(y).view(rows, -1, hd).all(2).cpu().numpy()
    want = np.ones((rows, hq + hk + copy), bool)
    want[1, 2] = want[4, 4] = want[5, 5] = False
    assert np.array_equal(fine, want)
    g = [torch.empty(hd, dtype=x.dtype, device="cuda") for _ in range(2)]
    ws = torch.empty(mx.mpx_qknorm_rope_bwd_workspace(rows, hd), dtype=torch.uint8, device="cuda")
    n = torch.zeros(1, dtype=torch.int32, device="cuda")
    mx.mpx_qknorm_rope_bwd(x.data_ptr(), ld, dy.data_ptr(), ld, y.data_ptr(), ld, None, None, EPS, pos.data_ptr(),
                           rows, rows, hq, hk, copy, hd, plan, g[0].data_ptr(), g[1].data_ptr(), mx.DTYPES[fmt],
                           ws.data_ptr(), ws.numel(), None if fmt == "f32" else n.data_ptr(), _s())
    fine = torch.isfinite(y).view(rows, -1, hd).all(2).cpu().numpy()
    want[5, 5] = True    # its cotangent is finite
    assert np.array_equal(fine, want)
    if fmt != "f32":
        assert int(n) == sum(int((~torch.isfinite(v)).sum()) for v in g) > 0


@pytest.mark.parametrize("fmt", FMTS)
def test_gradient_by_differences(fmt):
    """<dX, d> and <dw, e> against differences of <dY, Y> over the kernel's own float32
    outputs.  With s the head's root mean square along unit steps d, |s'| <= 1,
    |s''| <= 1 / s and |s'| <= 3 / s^2, so the third derivative of n = x / s is at most
    (15 |n| + 9) / s^3, and the difference off by h^2 / 6 of that (s taken a step
    smaller, eps adds to it); Y is linear in the gains.  Y itself by the forward's bound.
    """
    rows, hq, hk, hd, pairs, h = 4, 2, 1, 32, [6, 10], 2.0 ** -6
    rng = np.random.default_rng(2)
    width = (hq + hk) * hd
    v = {"x": rng.normal(0, 1.5, (rows, width)), "wq": 1 + rng.normal(0, 0.3, hd), "wk": 1 + rng.normal(0, 0.3, hd)}
    v = {k: round_to(a, fmt) for k, a in v.items()}
    dy = round_to(rng.normal(0, 1, (rows, width)), fmt)
    at = rng.integers(0, 30, (rows, 2)).astype(np.float32)
    pos = torch.from_numpy(at).cuda()
    plan = mx.RopePlan(pairs)
    rest = (EPS, at, pairs, [10000.0] * 2, False, hq, hk, hd)

    def y(a):
        t = {k: _dev(b, "f32") for k, b in a.items()}
        o = torch.empty_like(t["x"])
        mx.mpx_qknorm_rope_fwd(t["x"].data_ptr(), width, o.data_ptr(), width, t["wq"].data_ptr(),
                               t["wk"].data_ptr(), EPS, pos.data_ptr(), rows, rows, hq, hk, 0, hd, plan,
                               mx.MPX_F32, _s())
        return (to_host(o).astype(np.float64) * dy)
    t = {k: _dev(b, fmt) for k, b in {**v, "dy": dy}.items()}
    out = [torch.empty_like(t[k]) for k in ("x", "wq", "wk")]
    ws = torch.empty(mx.mpx_qknorm_rope_bwd_workspace(rows, hd), dtype=torch.uint8, device="cuda")
    mx.mpx_qknorm_rope_bwd(t["x"].data_ptr(), width, t["dy"].data_ptr(), width, out[0].data_ptr(), width,
                           t["wq"].data_ptr(), t["wk"].data_ptr(), EPS, pos.data_ptr(), rows, rows, hq, hk, 0, hd,
                           plan, out[1].data_ptr(), out[2].data_ptr(), mx.DTYPES[fmt], ws.data_ptr(), ws.numel(),
                           None, _s())
    half = {"f16": 2.0 ** -11, "bf16": 2.0 ** -8, "f32": 2.0 ** -24}[fmt]
    for key, grad in zip(("x", "wq", "wk"), out):
        d = np.sign(rng.normal(0, 1, v[key].shape))
        up, down = (y({**v, key: (v[key] + s * h * d).astype(np.float32)}) for s in (1, -1))
        want = (up - down).sum() / (2 * h)
        g = to_host(grad).astype(np.float64) * d
        _, n = qknorm.forward(v["x"], v["wq"], v["wk"], *rest)
        dn = np.abs(qknorm.backward(v["x"], dy, v["wq"], v["wk"], *rest)[3]).reshape(rows, -1, hd)
        heads = v["x"].astype(np.float64).reshape(rows, -1, hd)
        w = np.abs(qknorm._gains(v["wq"], v["wk"], hq, hk, hd))
        low = np.sqrt((heads ** 2).mean(-1, keepdims=True)) - h
        assert (low > 0.5).all()
        third = (dn * w * (15 * (np.abs(heads) + h) / low + 9) / low ** 3).sum() * h * h / 6
        rel = (hd + 16) * 2.0 ** -24 + 2.0 ** -20
        near = _partner_sums(n, pairs, False, hq + hk, hd) * 1.1     # n a step away
        own = rel * (near.reshape(rows, -1) * np.abs(dy)).sum() / h
        assert abs(want - g.sum()) <= half * np.abs(g).sum() + (third if key == "x" else 0.0) + own, key


def test_side_stream_and_graph():
    rows, hq, hk, copy, hd = 2100, 6, 3, 3, 64
    plan = mx.RopePlan([16, 16])
    ld = (hq + hk + copy) * hd
    x, dy = (torch.zeros(rows, ld, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    w = torch.rand(2, hd, device="cuda").bfloat16()
    pos = torch.zeros(rows, 2, device="cuda")
    sets = [[torch.empty_like(x), torch.empty_like(x), torch.empty_like(w),
             torch.empty(mx.mpx_qknorm_rope_bwd_workspace(rows, hd), dtype=torch.uint8, device="cuda")]
            for _ in range(2)]

    def call(o, s):
        mx.mpx_qknorm_rope_fwd(x.data_ptr(), ld, o[0].data_ptr(), ld, w[0].data_ptr(), w[1].data_ptr(), EPS,
                               pos.data_ptr(), rows, rows, hq, hk, copy, hd, plan, mx.MPX_BF16, s)
        mx.mpx_qknorm_rope_bwd(x.data_ptr(), ld, dy.data_ptr(), ld, o[1].data_ptr(), ld, w[0].data_ptr(),
                               w[1].data_ptr(), EPS, pos.data_ptr(), rows, rows, hq, hk, copy, hd, plan,
                               o[2][0].data_ptr(), o[2][1].data_ptr(), mx.MPX_BF16, o[3].data_ptr(), o[3].numel(),
                               None, s)
    g = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(g):
        call(sets[0], _s())
    side = torch.cuda.Stream()
    for i in range(4):
        x.copy_(torch.randn(x.shape, device="cuda"))
        dy.copy_(torch.randn(x.shape, device="cuda"))
        pos.copy_(torch.randint(0, 50, pos.shape, device="cuda").float())
        torch.cuda.synchronize()
        with torch.cuda.stream(side):
            call(sets[1], side.cuda_stream)
        g.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(sets[0][:3], sets[1][:3])), i


def test_long_strides_pass_32_bits():
    """Rows 2^27 + 8 elements apart: the last row's offset is past 2^31 elements."""
    rows, ld, hd = 20, (1 << 27) + 8, 64
    x = torch.zeros(rows * ld, dtype=torch.bfloat16, device="cuda").view(rows, ld)
    plan = mx.RopePlan([16, 16])
    v, dy = (torch.randn(rows, 3 * hd, device="cuda").bfloat16() for _ in range(2))
    pos = torch.arange(2 * rows, device="cuda", dtype=torch.float32).view(rows, 2)
    ws = torch.empty(mx.mpx_qknorm_rope_bwd_workspace(rows, hd), dtype=torch.uint8, device="cuda")
    x[:, :3 * hd] = v
    outs = []
    for t, l in ((v, 3 * hd), (x, ld)):
        y, d = torch.empty_like(v), torch.empty_like(v)
        mx.mpx_qknorm_rope_fwd(t.data_ptr(), l, y.data_ptr(), 3 * hd, None, None, EPS, pos.data_ptr(), rows, rows,
                               1, 1, 1, hd, plan, mx.MPX_BF16, _s())
        mx.mpx_qknorm_rope_bwd(t.data_ptr(), l, dy.data_ptr(), 3 * hd, d.data_ptr(), 3 * hd, None, None, EPS,
                               pos.data_ptr(), rows, rows, 1, 1, 1, hd, plan, None, None, mx.MPX_BF16,
                               ws.data_ptr(), ws.numel(), None, _s())
        outs.append((y, d))
    assert torch.equal(outs[0][0], outs[1][0]) and torch.equal(outs[0][1], outs[1][1])
