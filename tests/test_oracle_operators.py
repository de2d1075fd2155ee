"""CPU pins of the oracles of the 8-bit checkpoints, the rotary positions and
the log probabilities: the formats' defining properties, brute force, and
central differences in float64."""
import numpy as np
import pytest

from oracle import act8, logprob, rotary
from oracle.numfmt import round_to


def test_e4m3_bytes_and_values_are_inverse():
    b = np.arange(256)
    v = act8.byte_values(b)
    fin = ~np.isnan(v)
    assert fin.sum() == 254 and np.nanmax(v) == 448.0
    assert np.array_equal(act8.code_bytes(v[fin]), b[fin].astype(np.uint8))
    assert np.array_equal(act8.e4m3(v[fin]), v[fin])
    torch = pytest.importorskip("torch")
    t = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).float().numpy()
    assert np.array_equal(v, t.astype(np.float64), equal_nan=True)


def test_e4m3_rounds_to_nearest_even():
    v = np.sort(act8.byte_values(np.arange(0x7F)))
    for lo, hi, blo in zip(v[:-1], v[1:], range(0x7E)):
        mid = (lo + hi) / 2
        assert act8.e4m3(mid) == (lo if blo % 2 == 0 else hi)
        assert act8.e4m3(np.nextafter(mid, 0)) == lo and act8.e4m3(np.nextafter(mid, 1e9)) == hi


@pytest.mark.parametrize("fmt", ["f16", "bf16"])
def test_checkpoint_values_are_half_values_and_near(fmt):
    """Every value of a checkpoint is exactly a half value, within 2^-4 of x or
    within half the code's smallest step; groups use the least exponent."""
    rng = np.random.default_rng(3)
    mag = np.ldexp(1.0, rng.integers(-24, 15, (97, 60)) if fmt == "f16" else rng.integers(-126, 127, (97, 60)))
    x = round_to(rng.normal(0, 1, (97, 60)) * mag, fmt).astype(np.float64)
    x[:, 0], x[:, 1] = 0.0, (65504.0 if fmt == "f16" else float(np.ldexp(2 - 2 ** -7, 127)))
    c, e = act8.pack(x, fmt)
    v = act8.values(c, e)
    assert np.all(np.isfinite(v)) and np.array_equal(round_to(v, fmt).astype(np.float64), v)
    rows = np.repeat(e, 32, axis=0)[:97]
    assert np.all(np.abs(v - x) <= np.maximum(2.0 ** -4 * np.abs(x), np.ldexp(2.0 ** -10, rows)))
    a = np.stack([np.abs(x[g * 32:(g + 1) * 32]).max(axis=0) for g in range(4)])
    assert np.all((a <= 448 * np.exp2(e)) | (e == act8.EMAX[fmt]))
    assert np.all((a > 448 * np.exp2(e - 1.0)) | (e == act8.EMIN[fmt]))


def test_checkpoint_keeps_nonfinite_values_apart():
    x = np.ones((40, 3))
    x[5, 1], x[33, 2] = np.inf, np.nan
    c, e = act8.pack(x, "f16")
    v = act8.values(c, e)
    assert np.isnan(v[5, 1]) and np.isnan(v[33, 2]) and np.isnan(v).sum() == 2
    assert np.all(v[~np.isnan(v)] == 1.0)


@pytest.mark.parametrize("interleaved", [False, True])
def test_rotary_gradient_and_norms(interleaved):
    rng = np.random.default_rng(4)
    pairs, base, hd, rot = [3, 1, 2], [10000.0, 100.0, 7.5], 14, 2
    x, g = rng.normal(size=(6, 3 * hd)), rng.normal(size=(6, 3 * hd))
    pos = rng.integers(0, 50, (3, 3)).astype(np.float64)
    args = (pos, pairs, base, interleaved, rot, hd)
    y, dx = rotary.turn(x, *args), rotary.turn(g, *args, back=True)
    assert np.allclose(rotary.turn(y, *args, back=True), x, atol=1e-12)
    assert np.array_equal(y[:, rot * hd:], x[:, rot * hd:])
    assert np.array_equal(y.reshape(6, 3, hd)[..., 12:], x.reshape(6, 3, hd)[..., 12:])
    num, h = np.zeros_like(x), 1e-6
    for i in np.ndindex(*x.shape):
        d = np.zeros_like(x)
        d[i] = h
        num[i] = ((rotary.turn(x + d, *args) - rotary.turn(x - d, *args)) * g).sum() / (2 * h)
    assert np.allclose(num, dx, atol=1e-8)


def test_rotary_scores_depend_on_position_differences():
    """The property the rotation is for: q . k is the same when both tokens'
    positions move by the same vector."""
    rng = np.random.default_rng(5)
    q, k = rng.normal(size=(1, 16)), rng.normal(size=(1, 16))
    f = lambda v, p: rotary.turn(v, np.array([p]), [5, 3], [100.0, 50.0], False, 1, 16)
    a = (f(q, (3, 7)) * f(k, (1, 2))).sum()
    b = (f(q, (13, 27)) * f(k, (11, 22))).sum()
    assert abs(a - b) < 1e-12


def test_logprob_gradient_by_differences():
    rng = np.random.default_rng(6)
    z = rng.normal(0, 2, (4, 9))
    z[1, 3] = -np.inf
    t = np.array([2, 0, -1, 8])
    gl, ge, gt = rng.normal(size=4), rng.normal(size=4), rng.normal(size=(4, 3))
    stats, logp, ent, top, idx = logprob.forward(z, t, 3)
    assert logp[2] == 0.0

    def loss(zz):
        l, lp, en, tp, ix = logprob.forward(zz, t, 3)
        return (gl * lp).sum() + (ge * en).sum() + (gt * tp).sum()
    dz, _ = logprob.backward(z, t, stats, ent, idx, gl, ge, gt, 3.0)
    h = 1e-6
    for i in np.ndindex(*z.shape):
        if not np.isfinite(z[i]):
            assert dz[i] == 0.0
            continue
        d = np.zeros_like(z)
        d[i] = h
        assert abs((loss(z + d) - loss(z - d)) / (2 * h) * 3.0 - dz[i]) < 1e-7


def test_logprob_special_rows():
    inf, nan = np.inf, np.nan
    z = np.array([[-inf, -inf, -inf, -inf], [1.0, nan, 2.0, -inf], [0.0, inf, 1.0, inf], [1.0, 1.0, 1.0, -inf]])
    stats, logp, ent, top, idx = logprob.forward(z, np.array([1, 0, 0, 4]), 3)
    assert stats[0].tolist() == [-inf, 0.0] and logp[0] == -inf and ent[0] == 0.0 and idx[0].tolist() == [0, 1, 2]
    assert np.isnan(stats[1:3]).all() and np.isnan(ent[1:3]).all() and np.isnan(top[1:3]).all()
    assert idx[1].tolist() == [1, 2, 0] and idx[2].tolist() == [1, 3, 2]
    assert np.isnan(logp[3]) and idx[3].tolist() == [0, 1, 2] and abs(ent[3] - np.log(3)) < 1e-15
    dz, _ = logprob.backward(z, np.array([1, 0, 0, 0]), stats, ent, idx, np.ones(4), None, None, 1.0)
    low = np.full((1, 5), -3.4028234663852886e38)   # masked by the lowest value: evenly spread
    stats, _, ent, _, _ = logprob.forward(low, np.array([0]), 0)
    assert ent[0] == pytest.approx(np.log(5)) and stats[0, 1] == pytest.approx(np.log(5))
    assert np.all(dz[0] == 0) and np.isnan(dz[1:3]).all() and dz[3, 3] == 0 and np.isfinite(dz[3]).all()
