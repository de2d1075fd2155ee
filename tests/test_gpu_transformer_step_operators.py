"""The norms of queries and keys with rotary positions, dropout, the gated projections
and the linear cross entropy in one training pass of a transformer block, as a step uses
them beside the library's linear layers and attention: forward, backward, finite check,
generator advance, eagerly and as a replayed graph, against the same pass in float64 with
the same masks.

Bounds: those of the train steps' own end-to-end comparison.  A gradient is within 2e-2 of
the exact one in norm, and every element within 2e-2 max(max |ref|, S), S = |dY|^T |X| the
magnitude of the summands of a weight gradient."""
import numpy as np
import pytest

from oracle import dropout, gated, linear_ce, qknorm
from oracle.numfmt import round_to
from tests.gpu_util import HAVE_GPU, rel_norm_err, to_host

pytestmark = [pytest.mark.gpu, pytest.mark.skipif(not HAVE_GPU, reason="no GPU")]

if HAVE_GPU:
    import torch
    from paper_2507_03312_amd import binding as mx
    from tests.gpu_util import TORCH_HALF

B, H, HD, N, V = 4, 2, 64, 192, 1003
D = H * HD
PAIRS, EPS, P, SEED = [12, 20], 1e-6, 0.2, 2 ** 40 + 7
SCALE = 2.0 ** 12


def _reference(v, pos, targets, g, T, step, act):
    """Float64 pass: loss per row, gradients, and (dY, X) of every product."""
    M = B * T
    rest = (EPS, pos, PAIRS, [10000.0] * 2, False, H, H, HD)
    keeps = []
    for site in (0, 1):
        k, s = dropout.kept(M * D, P, SEED, step, site)
        keeps.append(k.reshape(M, D) * s)
    qkv = v["x"] @ v["wqkv"].T
    turned, _ = qknorm.forward(qkv, v["gq"], v["gk"], *rest)
    heads = lambda a, i: a.reshape(B, T, 3, H, HD)[:, :, i].transpose(0, 2, 1, 3)
    q, k, val = (heads(turned, i) for i in range(3))
    s = q @ k.transpose(0, 1, 3, 2) / np.sqrt(HD)
    p = np.exp(s - s.max(-1, keepdims=True))
    p /= p.sum(-1, keepdims=True)
    o = (p @ val).transpose(0, 2, 1, 3).reshape(M, D)
    x1 = v["x"] + keeps[0] * (o @ v["wo"].T)
    h, pre = gated.forward(x1, v["w1"], v["b1"], act)
    x2 = x1 + keeps[1] * (h @ v["w2"].T)
    z = x2 @ v["wv"].T
    stats, loss = linear_ce.forward(z, targets)
    dz = linear_ce.dlogits(z, targets, stats, g, SCALE)
    dx2 = dz @ v["wv"]
    dy = keeps[1] * dx2
    dpre = gated.backward(dy @ v["w2"], pre, act)
    dx1 = dx2 + dpre @ v["w1"]
    da = keeps[0] * dx1
    do = (da @ v["wo"]).reshape(B, T, H, HD).transpose(0, 2, 1, 3)
    dv = p.transpose(0, 1, 3, 2) @ do
    dp = do @ val.transpose(0, 1, 3, 2)
    ds = p * (dp - (dp * p).sum(-1, keepdims=True)) / np.sqrt(HD)
    dt = np.stack([a.transpose(0, 2, 1, 3) for a in (ds @ k, ds.transpose(0, 1, 3, 2) @ q, dv)], axis=2)
    dqkv, dgq, dgk, _ = qknorm.backward(qkv, dt.reshape(M, 3 * D), v["gq"], v["gk"], *rest)
    products = {"wqkv": (dqkv, v["x"]), "wo": (da, o), "w1": (dpre, x1), "w2": (dy, h), "wv": (dz, x2)}
    other = {"b1": dpre.sum(0), "gq": dgq, "gk": dgk, "x": dx1 + dqkv @ v["wqkv"]}
    return loss, products, other


class _Pass:
    """The same pass on the library's calls, buffers made once."""

    def __init__(self, v, pos, fmt, T, act):
        half = TORCH_HALF[fmt]
        self.M, self.T, self.dt = B * T, T, mx.DTYPES[fmt]
        self.act = {"silu": mx.MPX_ACT_SILU, "gelu": mx.MPX_ACT_GELU_TANH}[act]
        self.w = {k: torch.from_numpy(a).to(half).cuda() for k, a in v.items()}
        self.pos = torch.from_numpy(pos).cuda()
        self.targets = torch.zeros(self.M, dtype=torch.int32, device="cuda")
        self.g = torch.zeros(self.M, device="cuda")
        self.rng = torch.tensor([SEED, 0], dtype=torch.int64, device="cuda")
        self.state = torch.tensor([SCALE, 0.0, 0.0, 2.0, 1.0, 2.0 ** 100], device="cuda")
        self.count = torch.zeros(1, dtype=torch.int32, device="cuda")
        self.plan = mx.RopePlan(PAIRS)
        e = lambda *s: torch.empty(*s, dtype=half, device="cuda")
        M = self.M
        ld = -(-T // 8) * 8
        self.b = {"qkv": e(M, 3 * D), "turned": e(M, 3 * D), "o": e(M, D), "p": e(B * H, T, ld), "a": e(M, D),
                  "x1": e(M, D), "h": e(M, N), "pre": e(M, 2 * N), "y": e(M, D), "x2": e(M, D),
                  "dx2": e(M, D), "dy": e(M, D), "dpre": e(M, 2 * N), "dx1": e(M, D), "da": e(M, D), "do": e(M, D),
                  "dturned": e(M, 3 * D), "dqkv": e(M, 3 * D)}
        self.grad = {k: torch.empty_like(t) for k, t in self.w.items()}
        self.loss, self.stats = torch.empty(M, device="cuda"), torch.empty(M, 2, device="cuda")
        self.mean = torch.empty(1, device="cuda")
        need = max(mx.mpx_linear_ce_fwd_workspace(M, V, D), mx.mpx_linear_ce_bwd_workspace(M, V, D),
                   mx.mpx_linear_bwd_gated_workspace(M, D, N), mx.mpx_linear_bwd_workspace(M, 2 * N, D),
                   mx.mpx_linear_bwd_workspace(M, D, D), mx.mpx_linear_bwd_workspace(M, 3 * D, D),
                   mx.mpx_qknorm_rope_bwd_workspace(M, HD))
        self.ws = torch.empty(need, dtype=torch.uint8, device="cuda")

    def run(self):
        s = torch.cuda.current_stream().cuda_stream
        M, T, dt = self.M, self.T, self.dt
        w, b, g = ({k: t.data_ptr() for k, t in d.items()} for d in (self.w, self.b, self.grad))
        ws, n, cnt = self.ws.data_ptr(), self.ws.numel(), self.count.data_ptr()
        rng, pos = self.rng.data_ptr(), self.pos.data_ptr()
        heads = (T, M, H, H, H, HD, self.plan)
        none = mx.MPX_ACT_NONE
        mx.mpx_zero(cnt, 4, s)
        mx.mpx_linear_fwd(w["x"], w["wqkv"], None, None, b["qkv"], None, M, 3 * D, D, dt, none, s)
        mx.mpx_qknorm_rope_fwd(b["qkv"], 3 * D, b["turned"], 3 * D, w["gq"], w["gk"], EPS, pos, *heads, dt, s)
        mx.mpx_attention_fwd(b["turned"], b["o"], b["p"], B, T, H, HD, dt, s)
        mx.mpx_linear_fwd(b["o"], w["wo"], None, None, b["a"], None, M, D, D, dt, none, s)
        mx.mpx_dropout_fwd(b["a"], w["x"], b["x1"], M * D, P, rng, 0, dt, s)
        mx.mpx_gated_fwd(b["x1"], w["w1"], w["b1"], b["h"], b["pre"], M, N, D, dt, self.act, s)
        mx.mpx_linear_fwd(b["h"], w["w2"], None, None, b["y"], None, M, D, N, dt, none, s)
        mx.mpx_dropout_fwd(b["y"], b["x1"], b["x2"], M * D, P, rng, 1, dt, s)
        mx.mpx_linear_ce_fwd(b["x2"], w["wv"], None, self.targets.data_ptr(), M, V, D, self.loss.data_ptr(),
                             self.stats.data_ptr(), self.mean.data_ptr(), dt, ws, n, s)
        mx.mpx_linear_ce_bwd(b["x2"], w["wv"], None, self.targets.data_ptr(), M, V, D, self.stats.data_ptr(),
                             self.g.data_ptr(), self.state.data_ptr(), b["dx2"], g["wv"], None, dt, ws, n, cnt, s)
        mx.mpx_dropout_bwd(b["dx2"], b["dy"], M * D, P, rng, 1, dt, s)
        mx.mpx_linear_bwd_gated(b["h"], w["w2"], b["dy"], b["pre"], self.act, b["dpre"], g["w2"], None, M, D, N, dt,
                                ws, n, cnt, s)
        mx.mpx_linear_bwd(b["x1"], w["w1"], b["dpre"], None, none, b["dx1"], g["w1"], g["b1"], M, 2 * N, D, dt, ws,
                          n, cnt, s)
        # the residual branch's cotangent: dropout of nothing adds
        mx.mpx_dropout_fwd(b["dx1"], b["dx2"], b["dx1"], M * D, 0.0, rng, 2, dt, s)
        mx.mpx_dropout_bwd(b["dx1"], b["da"], M * D, P, rng, 0, dt, s)
        mx.mpx_linear_bwd(b["o"], w["wo"], b["da"], None, none, b["do"], g["wo"], None, M, D, D, dt, ws, n, cnt, s)
        mx.mpx_attention_bwd(b["turned"], b["p"], b["do"], b["dturned"], B, T, H, HD, dt, None, 0, s)
        mx.mpx_qknorm_rope_bwd(b["qkv"], 3 * D, b["dturned"], 3 * D, b["dqkv"], 3 * D, w["gq"], w["gk"], EPS, pos,
                               *heads, g["gq"], g["gk"], dt, ws, n, cnt, s)
        mx.mpx_linear_bwd(w["x"], w["wqkv"], b["dqkv"], None, none, g["x"], g["wqkv"], None, M, 3 * D, D, dt, ws, n,
                          cnt, s)
        mx.mpx_dropout_fwd(g["x"], b["dx1"], g["x"], M * D, 0.0, rng, 2, dt, s)
        mx.mpx_rng_advance(rng, s)

    def results(self):
        torch.cuda.synchronize()
        return {"loss": self.loss.clone(), "mean": self.mean.clone(), **{k: t.clone() for k, t in self.grad.items()}}


def _inputs(fmt, T, seed):
    rng = np.random.default_rng(seed)
    M = B * T
    v = {"x": rng.normal(0, 1, (M, D)), "wqkv": rng.normal(0, D ** -0.5, (3 * D, D)),
         "wo": rng.normal(0, D ** -0.5, (D, D)), "w1": rng.normal(0, D ** -0.5, (2 * N, D)),
         "b1": rng.normal(0, 0.1, 2 * N), "w2": rng.normal(0, N ** -0.5, (D, N)),
         "wv": rng.normal(0, 2.0 * D ** -0.5, (V, D)), "gq": rng.normal(1, 0.2, HD), "gk": rng.normal(1, 0.2, HD)}
    v = {k: round_to(a, fmt) for k, a in v.items()}
    pos = rng.integers(0, 14, (T, 2)).astype(np.float32)
    t = rng.integers(0, V, M).astype(np.int32)
    t[rng.random(M) < 0.1] = -1
    return v, pos, t, (rng.uniform(0.5, 1.5, M) / M).astype(np.float32)


@pytest.mark.parametrize("fmt", ["f16", "bf16"])
@pytest.mark.parametrize("T, act", [(9, "silu"), (65, "gelu"), (197, "silu")])
def test_training_pass(fmt, T, act):
    v, pos, t, g = _inputs(fmt, T, T)
    run = _Pass(v, pos, fmt, T, act)
    run.targets.copy_(torch.from_numpy(t))
    run.g.copy_(torch.from_numpy(g))
    run.run()
    eager = [run.results()]
    assert int(run.count) == 0 and run.rng.tolist() == [SEED, 1]
    v64 = {k: a.astype(np.float64) for k, a in v.items()}
    loss, products, other = _reference(v64, pos, t, g, T, 0, act)
    got = {k: to_host(a).astype(np.float64) for k, a in eager[0].items()}
    assert np.abs(got["loss"] - loss).max() <= 2e-2 * np.abs(loss).max()
    assert abs(got["mean"][0] - loss.sum() / (t >= 0).sum()) <= 2e-2 * loss.max()
    for name, (dy, x) in products.items():
        ref, size = dy.T @ x, np.abs(dy).T @ np.abs(x)
        assert rel_norm_err(got[name], ref) <= 2e-2, name
        assert (np.abs(got[name] - ref) <= 2e-2 * np.maximum(np.abs(ref).max(), size)).all(), name
    for name, ref in other.items():
        assert rel_norm_err(got[name], ref) <= 2e-2, name
    # a captured pass: every replay draws the masks of its own step, as the eager pass does
    run.rng[1] = 0
    run.run()
    run.run()
    eager.append(run.results())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run.run()
    run.rng[1] = 0
    for i in range(4):
        graph.replay()
        again = run.results()
        if i < 2:
            for k in again:
                assert torch.equal(again[k], eager[i][k]), (i, k)
        else:
            assert not torch.equal(again["wv"], eager[1]["wv"])   # other masks
        torch.empty(1 << 20, device="cuda").normal_()   # the program's own work between replays
    assert run.rng.tolist() == [SEED, 4] and int(run.count) == 0


def test_overflow_shows_in_the_finite_check():
    """A scale that overflows float16's gradients: every operator's share of the count is that
    of its written gradients."""
    T = 65
    v, pos, t, g = _inputs("f16", T, 3)
    run = _Pass(v, pos, "f16", T, "silu")
    run.targets.copy_(torch.from_numpy(t))
    run.g.copy_(torch.from_numpy(g))
    run.state[0] = 2.0 ** 40
    run.run()
    out = run.results()
    want = sum(int((~torch.isfinite(out[k])).sum()) for k in out if k not in ("loss", "mean", "x"))
    assert int(run.count) == want > 0
    assert torch.isfinite(out["loss"]).all()
