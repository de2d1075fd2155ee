"""The 8-bit checkpoints, rotary positions and log probabilities in one training
pass of an attention layer with a token head, as a step uses them: forward,
backward, finite check, eagerly and as a replayed graph, against the same pass in
float64.

Bounds: a gradient is a sum over tokens of products dY * X.  X from a checkpoint
is off by at most 2^-4 |X| (normal codes), and the operands of an end-to-end half
pass by up to 2e-2 of theirs (the bar of the train steps' own comparison), so
every element of a weight gradient is within (2^-4 + 2e-2) S of the exact one,
S = |dY|^T |X|; a bias gradient within 2e-2 sum |dY|."""
import numpy as np
import pytest

from oracle import act8, logprob, ops, rotary
from oracle.numfmt import round_to
from oracle.policy import Policy
from tests.gpu_util import HAVE_GPU, assert_within, gemm_bound, to_host, ulp

pytestmark = [pytest.mark.gpu, pytest.mark.skipif(not HAVE_GPU, reason="no GPU")]

if HAVE_GPU:
    import torch
    from paper_2507_03312_amd import binding as mx
    from tests.gpu_util import TORCH_HALF

B, H, HD, V, K = 3, 2, 64, 1003, 4
D = H * HD
PAIRS, BASES = [12, 20], [100.0, 10000.0]
SCALE = 2.0 ** 10


def _reference(x, pos, wq, wo, wv, bv, tg, gl, ge, gt, T, chosen):
    """Float64 pass: per-row results, and (dY, X) of every product, biases' dY.
    chosen: the alternatives whose log probabilities the loss uses (logits that
    lie closer than the half pass is exact may come in another order there)."""
    M = B * T
    turn = lambda a, back: rotary.turn(a, pos, PAIRS, BASES, False, 2 * H, HD, back)
    qkv = turn(x @ wq.T, False)
    heads = lambda a, i: a.reshape(B, T, 3, H, HD)[:, :, i].transpose(0, 2, 1, 3)
    q, k, v = (heads(qkv, i) for i in range(3))
    s = q @ k.transpose(0, 1, 3, 2) / np.sqrt(HD)
    p = np.exp(s - s.max(-1, keepdims=True))
    p /= p.sum(-1, keepdims=True)
    o = (p @ v).transpose(0, 2, 1, 3).reshape(M, D)
    a = o @ wo.T
    z = a @ wv.T + bv
    stats, logp, ent, top, idx = logprob.forward(z, tg, K)
    dz, _ = logprob.backward(z, tg, stats, ent, chosen, gl, ge, gt, SCALE)
    da = dz @ wv
    do = (da @ wo).reshape(B, T, H, HD).transpose(0, 2, 1, 3)
    dv = p.transpose(0, 1, 3, 2) @ do
    dp = do @ v.transpose(0, 1, 3, 2)
    ds = p * (dp - (dp * p).sum(-1, keepdims=True)) / np.sqrt(HD)
    dq, dk = ds @ k, ds.transpose(0, 1, 3, 2) @ q
    dqkv = np.stack([g.transpose(0, 2, 1, 3) for g in (dq, dk, dv)], axis=2).reshape(M, 3 * D)
    dqkv = turn(dqkv, True)
    lp = (z - stats[:, :1]) - stats[:, 1:]
    return logp, ent, top, np.take_along_axis(lp, chosen, axis=1), {"wv": (dz, a), "wo": (da, o), "wq": (dqkv, x)}, dz


class Pass:
    """Device buffers and the calls of one pass."""

    def __init__(self, fmt, T, arrays):
        self.fmt, self.T, self.M = fmt, T, B * T
        h, M = TORCH_HALF[fmt], B * T
        up = lambda a: torch.from_numpy(np.ascontiguousarray(a, np.float32)).cuda()
        self.x, self.wq, self.wo, self.wv, self.bv = (up(a).to(h) for a in arrays[:5])
        self.pos, self.gl, self.ge, self.gt = (up(a) for a in arrays[5:9])
        self.tg = torch.from_numpy(arrays[9].astype(np.int32)).cuda()
        e = lambda *s, dtype=h: torch.zeros(*s, dtype=dtype, device="cuda")
        ck = lambda n: (e(M, n, dtype=torch.uint8), e(-(-M // 32), n, dtype=torch.uint8))
        self.xc, self.oc, self.ac = ck(D), ck(D), ck(D)
        self.qkv, self.dqkv = e(M, 3 * D), e(M, 3 * D)
        self.o, self.a, self.z, self.dz, self.da, self.do = e(M, D), e(M, D), e(M, V), e(M, V), e(M, D), e(M, D)
        self.P = e(B * H * T, -(-T // 8) * 8)
        self.g = {"wv": e(V, D), "wo": e(D, D), "wq": e(3 * D, D), "bv": e(V)}
        f = lambda *s: e(*s, dtype=torch.float32)
        self.logp, self.ent, self.stats, self.top = f(M), f(M), f(M, 2), f(M, K)
        self.idx = e(M, K, dtype=torch.int32)
        self.state = torch.tensor([SCALE, 0, 0, 2, 1, 2.0 ** 100], device="cuda")
        self.nf = e(1, dtype=torch.int32)
        n = max(mx.mpx_logprob_workspace(M, V, K), *(mx.mpx_linear_bwd_act8_workspace(M, *s) for s in
                                                     ((V, D), (D, D), (3 * D, D))))
        self.ws = e(n, dtype=torch.uint8)
        self.plan = mx.RopePlan(PAIRS, BASES)

    def run(self, s):
        M, T, dt = self.M, self.T, mx.DTYPES[self.fmt]
        p = lambda t: None if t is None else t.data_ptr()
        none, nb = mx.MPX_ACT_NONE, self.ws.numel()
        mx.mpx_zero(p(self.nf), 4, s)
        pack = lambda a, c: mx.mpx_act8_pack(p(a), D, p(c[0]), p(c[1]), M, D, dt, s)
        pack(self.x, self.xc)
        mx.mpx_linear_fwd(p(self.x), p(self.wq), None, None, p(self.qkv), None, M, 3 * D, D, dt, none, s)
        mx.mpx_rope_fwd(p(self.qkv), 3 * D, p(self.qkv), 3 * D, p(self.pos), T, M, 2 * H, H, HD, self.plan, dt, s)
        mx.mpx_attention_fwd(p(self.qkv), p(self.o), p(self.P), B, T, H, HD, dt, s)
        pack(self.o, self.oc)
        mx.mpx_linear_fwd(p(self.o), p(self.wo), None, None, p(self.a), None, M, D, D, dt, none, s)
        pack(self.a, self.ac)
        mx.mpx_linear_fwd(p(self.a), p(self.wv), p(self.bv), None, p(self.z), None, M, V, D, dt, none, s)
        mx.mpx_logprob_fwd(p(self.z), V, p(self.tg), M, V, K, p(self.logp), p(self.ent), p(self.stats),
                           p(self.top), p(self.idx), dt, p(self.ws), nb, s)
        mx.mpx_logprob_bwd(p(self.z), V, p(self.tg), M, V, K, p(self.stats), p(self.ent), p(self.idx),
                           p(self.gl), p(self.ge), p(self.gt), p(self.state), p(self.dz), V, dt, s)
        bwd = lambda c, w, dy, dx, dw, db, n: mx.mpx_linear_bwd_act8(
            p(c[0]), p(c[1]), p(w), p(dy), None, None, none, p(dx), p(dw), p(db), M, n, D, dt, p(self.ws), nb,
            p(self.nf), s)
        bwd(self.ac, self.wv, self.dz, self.da, self.g["wv"], self.g["bv"], V)
        bwd(self.oc, self.wo, self.da, self.do, self.g["wo"], None, D)
        mx.mpx_attention_bwd(p(self.qkv), p(self.P), p(self.do), p(self.dqkv), B, T, H, HD, dt, None, 0, s)
        mx.mpx_rope_bwd(p(self.dqkv), 3 * D, p(self.dqkv), 3 * D, p(self.pos), T, M, 2 * H, H, HD, self.plan, dt, s)
        bwd(self.xc, self.wq, self.dqkv, None, self.g["wq"], None, 3 * D)


def _arrays(fmt, T, seed=0):
    rng = np.random.default_rng(seed)
    M = B * T
    r = lambda *s, std=1.0: round_to(rng.normal(0, std, s), fmt).astype(np.float64)
    x = r(M, D)
    x[:, 5] *= 16.0
    pos = np.stack([np.arange(T) // 8, np.arange(T) % 8], axis=1).astype(np.float64)
    pos[0] = 0.0
    tg = rng.integers(0, V, M)
    tg[3] = -1
    f = lambda *s: rng.normal(0, 1, s).astype(np.float32).astype(np.float64)
    return [x, r(3 * D, D, std=0.06), r(D, D, std=0.09), r(V, D, std=0.15), r(V, std=0.1), pos,
            f(M) / M, f(M) / M, f(M, K) / M, tg]


@pytest.mark.parametrize("fmt", ["f16", "bf16"])
@pytest.mark.parametrize("T", [65, 130])
def test_one_training_pass(fmt, T):
    arrays = _arrays(fmt, T)
    x, wq, wo, wv, bv, pos, gl, ge, gt, tg = arrays
    step = Pass(fmt, T, arrays)
    step.run(torch.cuda.current_stream().cuda_stream)
    torch.cuda.synchronize()
    chosen = step.idx.cpu().numpy().astype(np.int64)
    logp, ent, best, taken, products, dz = _reference(x, pos, wq, wo, wv, bv, tg, gl, ge, gt, T, chosen)
    got = step.logp.double().cpu().numpy()
    # logits of size up to about 10 off by 2e-2 of theirs
    assert np.abs(got - logp).max() <= 2e-2 * 10 and got[3] == 0.0
    assert np.abs(step.ent.double().cpu().numpy() - ent).max() <= 2e-2 * 10
    # the alternatives taken are the best ones, up to that difference either way
    assert np.abs(taken - best).max() <= 2 * 2e-2 * 10
    assert all(len(set(r)) == K for r in chosen)
    for name, (dy, a) in products.items():
        g = step.g[name].double().cpu().numpy()
        S = np.abs(dy).T @ np.abs(a)
        ref = dy.T @ a
        assert np.all(np.abs(g - ref) <= (2.0 ** -4 + 2e-2) * np.maximum(S, np.abs(ref).max())), name
        # the errors are not systematic: far smaller in norm
        assert np.linalg.norm(g - ref) <= (2.0 ** -4 + 2e-2) * np.linalg.norm(ref), name
    db = step.g["bv"].double().cpu().numpy()
    S = np.abs(dz).sum(axis=0)
    assert np.all(np.abs(db - dz.sum(axis=0)) <= 2e-2 * np.maximum(S, np.abs(dz.sum(axis=0)).max()))
    assert int(step.nf.item()) == 0


@pytest.mark.parametrize("fmt", ["f16", "bf16"])
@pytest.mark.parametrize("T", [65, 130])
def test_products_of_the_pass(fmt, T):
    """Every checkpoint and every linear gradient of the pass from the operands that
    the pass itself left: codes byte for byte, each element of dW, dX and db within
    one rounding and two float32 summation orders of the float64 product."""
    arrays = _arrays(fmt, T, 1)
    step, pol = Pass(fmt, T, arrays), Policy(fmt)
    step.run(torch.cuda.current_stream().cuda_stream)
    torch.cuda.synchronize()
    M = step.M
    for name, dy, x, ck, w, dx, db in (("wv", step.dz, step.a, step.ac, step.wv, step.da, step.g["bv"]),
                                       ("wo", step.da, step.o, step.oc, step.wo, step.do, None),
                                       ("wq", step.dqkv, step.x, step.xc, step.wq, None, None)):
        values, e = act8.pack(to_host(x), fmt)
        assert np.array_equal(ck[0].cpu().numpy(), act8.code_bytes(values)), name
        assert np.array_equal(ck[1].cpu().numpy(), (e + 127).astype(np.uint8)), name
        xv, dy, w = act8.values(values, e), to_host(dy), to_host(w)
        assert np.isfinite(dy).all() and np.abs(dy).max() > 0.0, name
        rdx, rdw, rdb = ops.linear_bwd(pol, xv, w, dy)
        assert_within(to_host(step.g[name]), rdw, gemm_bound(dy.T, xv, rdw, fmt, M), "d" + name)
        if dx is not None:
            assert_within(to_host(dx), rdx, gemm_bound(dy, w, rdx, fmt, len(w)), "dX of " + name)
        if db is not None:
            colb = ulp(rdb, fmt) + 2.0 * M * 2.0 ** -24 * np.abs(dy.astype(np.float64)).sum(axis=0)
            assert_within(to_host(db), rdb, colb, "db")


@pytest.mark.parametrize("fmt", ["f16", "bf16"])
def test_one_training_pass_replayed(fmt):
    """Captured once, replayed on new tokens with eager passes of another instance
    between: the same bits.  An infinite activation raises the finite count."""
    T = 65
    a, b = Pass(fmt, T, _arrays(fmt, T)), Pass(fmt, T, _arrays(fmt, T))
    stream = lambda: torch.cuda.current_stream().cuda_stream
    b.run(stream())
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        a.run(stream())
    for i in range(4):
        x = torch.randn(B * T, D, device="cuda")
        if i == 3:
            x[7, 9] = float("inf")
        a.x.copy_(x)
        b.x.copy_(x)
        b.run(stream())
        g.replay()
        torch.cuda.synchronize()
        for n in a.g:
            assert torch.equal(a.g[n].view(torch.int16), b.g[n].view(torch.int16)), (i, n)
        assert torch.equal(a.idx, b.idx) and torch.equal(a.nf, b.nf)
        assert (int(a.nf.item()) > 0) == (i == 3)
