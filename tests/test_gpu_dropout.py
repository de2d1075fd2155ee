"""Counter-based dropout on the GPU: the mask bit for bit against the oracle's generator,
values to one rounding."""
import numpy as np
import pytest

from oracle import dropout
from oracle.numfmt import round_to
from tests.gpu_util import HAVE_GPU, assert_within, to_host, ulp

pytestmark = [pytest.mark.gpu, pytest.mark.skipif(not HAVE_GPU, reason="no GPU")]

if HAVE_GPU:
    import torch
    from paper_2507_03312_amd import binding as mx
    TYPES = {"f16": torch.float16, "bf16": torch.bfloat16, "f32": torch.float32}

FMTS = ["f16", "bf16", "f32"]


def _s():
    return torch.cuda.current_stream().cuda_stream


def _dev(a, fmt, off=0):
    buf = torch.empty(a.size + off, dtype=TYPES[fmt], device="cuda")
    buf[off:].copy_(torch.from_numpy(np.ascontiguousarray(a, np.float32)))
    return buf[off:]


def _state(seed, step):
    as_signed = lambda v: v - 2 ** 64 if v >= 2 ** 63 else v
    return torch.tensor([as_signed(seed), as_signed(step)], dtype=torch.int64, device="cuda")


@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("n", [1, 7, 8, 9, 2047, 2048, 4101, 100003])
@pytest.mark.parametrize("p, seed, step, site", [(0.1, 1, 0, 0), (0.5, 2 ** 64 - 1, 2 ** 63 + 5, 2 ** 32 - 1),
                                                 (0.0, 5, 5, 5), (0.9999, 12345678901234567, 7, 3)])
def test_dropout(fmt, n, p, seed, step, site):
    """Forward with and without a residual, backward, out of place and in place, any
    alignment.  A kept value is rounded once in float32 with the factor, its sum with
    the residual once more, and once to the type."""
    rng = np.random.default_rng(n)
    x, r = (round_to(rng.normal(0, 1, n) + 3, fmt) for _ in range(2))   # none is 0
    keep, scale = dropout.kept(n, p, seed, step, site)
    y = np.where(keep, x.astype(np.float64) * scale, 0.0)
    state, dt = _state(seed, step), mx.DTYPES[fmt]
    for off in (0, 1):
        for res in (False, True):
            want = y + r if res else y
            xt, rt = _dev(x, fmt, off), _dev(r, fmt, off)
            buf = torch.full((n + 128,), -7.0, dtype=TYPES[fmt], device="cuda")
            out = buf[64 + off:64 + off + n]
            mx.mpx_dropout_fwd(xt.data_ptr(), rt.data_ptr() if res else None, out.data_ptr(), n, p,
                               state.data_ptr(), site, dt, _s())
            assert (buf[:64 + off] == -7.0).all() and (buf[64 + off + n:] == -7.0).all()
            got = to_host(out)
            bound = 0.5 * (1 + 2.0 ** -10) * ulp(want, fmt) + 2.0 ** -23 * (np.abs(y) + np.abs(want))
            assert_within(got, want, bound)
            if res:
                mx.mpx_dropout_fwd(xt.data_ptr(), rt.data_ptr(), rt.data_ptr(), n, p, state.data_ptr(), site, dt,
                                   _s())
                assert torch.equal(rt, out)
            else:
                assert np.array_equal(got != 0, keep)
                dx = torch.empty_like(out)
                mx.mpx_dropout_bwd(xt.data_ptr(), dx.data_ptr(), n, p, state.data_ptr(), site, dt, _s())
                assert torch.equal(dx, out)
                mx.mpx_dropout_bwd(xt.data_ptr(), xt.data_ptr(), n, p, state.data_ptr(), site, dt, _s())
                assert torch.equal(xt, out)


@pytest.mark.parametrize("fmt", FMTS)
def test_dropped_values_are_zero_whatever_they_hold(fmt):
    n = 5000
    x = torch.full((n,), float("nan"), dtype=TYPES[fmt], device="cuda")
    x[1::2] = float("inf")
    y, state = torch.empty_like(x), _state(3, 4)
    keep, _ = dropout.kept(n, 0.5, 3, 4, 1)
    mx.mpx_dropout_fwd(x.data_ptr(), None, y.data_ptr(), n, 0.5, state.data_ptr(), 1, mx.DTYPES[fmt], _s())
    got = to_host(y)
    assert (got[~keep] == 0).all() and not np.isfinite(got[keep]).any()


def test_advance_in_a_graph_draws_anew():
    """A captured step of two sites and an advance: every replay's masks are its step's,
    forward and backward alike."""
    n, seed = 30011, 77
    x = torch.ones(n, dtype=torch.float32, device="cuda")
    y, z, d = (torch.empty_like(x) for _ in range(3))
    state = _state(seed, 2 ** 32 - 2)   # the step's lower word wraps during the replays
    g = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(g):
        s = _s()
        for out, site in ((y, 0), (z, 1)):
            mx.mpx_dropout_fwd(x.data_ptr(), None, out.data_ptr(), n, 0.25, state.data_ptr(), site, 0, s)
        mx.mpx_dropout_bwd(x.data_ptr(), d.data_ptr(), n, 0.25, state.data_ptr(), 1, 0, s)
        mx.mpx_rng_advance(state.data_ptr(), s)
    for i in range(4):
        g.replay()
        torch.cuda.synchronize()
        masks = [dropout.kept(n, 0.25, seed, 2 ** 32 - 2 + i, site)[0] for site in (0, 1)]
        assert np.array_equal(to_host(y) != 0, masks[0]) and np.array_equal(to_host(z) != 0, masks[1])
        assert torch.equal(d, z)
    assert state.tolist() == [seed, 2 ** 32 + 2]


def test_many_values():
    """More than 2^31 values: the last ones' draws come from their own blocks."""
    n = (1 << 31) + 1003
    x = torch.ones(n, dtype=torch.bfloat16, device="cuda")
    state = _state(9, 1)
    mx.mpx_dropout_fwd(x.data_ptr(), None, x.data_ptr(), n, 0.5, state.data_ptr(), 0, mx.MPX_BF16, _s())
    first = (n - 5000) // 8 * 8
    keep, _ = dropout.kept(n - first, 0.5, 9, 1, 0, first=first)
    assert np.array_equal(to_host(x[first:]) != 0, keep)
