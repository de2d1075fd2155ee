"""Host-side argument checks of the 8-bit checkpoints, the rotary positions and
the log probabilities: every refusal comes before anything is launched or
dereferenced (the pointers here are placeholders)."""
import os

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
LIB = os.path.join(ROOT, "paper_2507_03312_amd", "libmpx.so")
pytestmark = pytest.mark.skipif(not os.path.exists(LIB), reason="libmpx.so not built")

p = 256  # never dereferenced


@pytest.fixture(scope="module")
def mx():
    from paper_2507_03312_amd import binding
    return binding


def refused(mx, match, fn, *args):
    with pytest.raises(mx.MPXError, match=match):
        fn(*args)


@pytest.mark.parametrize("change, match", [
    ({0: None}, "NULL"), ({2: None}, "NULL"), ({3: None}, "NULL"), ({4: 0}, ">= 1"), ({5: 0}, ">= 1"),
    ({4: -3}, ">= 1"), ({1: 63}, "stride"), ({6: 0}, "MPX_F16 or MPX_BF16"), ({6: 7}, "MPX_F16 or MPX_BF16"),
    ({0: 257}, "aligned"), ({4: 1 << 45}, "too large"), ({5: 1 << 40, 1: 1 << 40}, "too large")])
def test_pack_refusals(mx, change, match):
    args = [p, 64, p, p, 33, 64, mx.MPX_BF16, 0]
    for i, v in change.items():
        args[i] = v
    refused(mx, match, mx.mpx_act8_pack, *args)


@pytest.mark.parametrize("change, match", [
    ({0: None}, "NULL"), ({1: None}, "NULL"), ({2: None}, "NULL"), ({3: 10}, "stride"), ({4: 0}, ">= 1"),
    ({6: 0}, "MPX_F16 or MPX_BF16"), ({2: 255}, "aligned"), ({4: 1 << 45}, "too large")])
def test_unpack_refusals(mx, change, match):
    args = [p, p, p, 64, 33, 64, mx.MPX_F16, 0]
    for i, v in change.items():
        args[i] = v
    refused(mx, match, mx.mpx_act8_unpack, *args)


# Xc Xs W dY Pc Ps x_act dX dW db M N K dt ws bytes nonfinite stream
@pytest.mark.parametrize("change, match", [
    ({3: None}, "NULL dY"), ({7: None, 8: None, 9: None}, "nothing to compute"), ({2: None}, "W is required"),
    ({0: None}, "Xc and Xs"), ({1: None}, "Xc and Xs"), ({4: None}, "Pc and Ps"), ({5: None}, "Pc and Ps"),
    ({10: 0}, ">= 1"), ({11: 0}, ">= 1"), ({12: -1}, ">= 1"), ({13: 0}, "MPX_F16 or MPX_BF16"),
    ({6: 2}, "unknown activation"), ({14: None}, "workspace"), ({15: 0}, "workspace")])
def test_linear_bwd_act8_refusals(mx, change, match):
    need = mx.mpx_linear_bwd_act8_workspace(64, 32, 48)
    args = [p, p, p, p, p, p, 1, p, p, p, 64, 32, 48, mx.MPX_BF16, p, need, None, 0]
    for i, v in change.items():
        args[i] = v
    refused(mx, match, mx.mpx_linear_bwd_act8, *args)


@pytest.mark.parametrize("nk", [(2304, 768), (1000, 768), (64, 64), (640, 588)],
                         ids=lambda s: "x".join(map(str, s)))
def test_linear_bwd_act8_workspace_never_falls_with_the_batch(mx, nk):
    sizes = [mx.mpx_linear_bwd_act8_workspace(M, *nk) for M in range(1, 40001, 13)]
    assert sizes == sorted(sizes) and sizes[0] > 0
    assert mx.mpx_linear_bwd_act8_workspace(0, *nk) == 0


# X ldx Y ldy pos pos_rows rows rot copy hd plan dt stream
@pytest.mark.parametrize("change, match", [
    ({0: None}, "NULL"), ({2: None}, "NULL"), ({4: None}, "NULL"), ({5: 0}, "multiple"), ({5: 7}, "multiple"),
    ({6: 0}, "multiple"), ({6: -12}, "multiple"), ({7: 0}, "heads_rot"), ({8: -1}, "heads_copy"),
    ({9: 1}, "hd"), ({9: 513, 1: 9999, 3: 9999}, "hd"), ({1: 191}, "stride"), ({3: 191}, "stride"),
    ({2: p, 3: 200}, "in place"), ({11: 3}, "MPX_F16"), ({0: 257}, "aligned"), ({4: 258}, "aligned"),
    ({6: 1 << 40, 5: 1}, "rows"), ({7: 1 << 62}, "heads_rot")])
@pytest.mark.parametrize("back", [False, True])
def test_rope_refusals(mx, change, match, back):
    args = [p, 192, 4096, 192, p, 6, 12, 2, 1, 64, mx.RopePlan([16, 16]), mx.MPX_BF16, 0]
    for i, v in change.items():
        args[i] = v
    refused(mx, match, mx.mpx_rope_bwd if back else mx.mpx_rope_fwd, *args)


@pytest.mark.parametrize("field, value, match", [
    ("axes", 0, "axes"), ("axes", 5, "axes"), ("axes", -1, "axes"), ("pairs", (0, 16), "pairs"),
    ("pairs", (16, 17), "pairs"), ("pairs", (-4, 16), "pairs"), ("pairs", (2 ** 31 - 1, 1), "pairs"),
    ("base", (1.0, 10.0), "base"), ("base", (0.0, 10.0), "base"), ("base", (10.0, float("inf")), "base"),
    ("base", (10.0, float("nan")), "base"), ("interleaved", 2, "interleaved")])
def test_rope_plan_refusals(mx, field, value, match):
    plan = mx.RopePlan([16, 16])
    if isinstance(value, tuple):
        for i, v in enumerate(value):
            getattr(plan, field)[i] = v
    else:
        setattr(plan, field, value)
    refused(mx, match, mx.mpx_rope_fwd, p, 192, 4096, 192, p, 6, 12, 2, 1, 64, plan, mx.MPX_BF16, 0)
    refused(mx, "NULL", mx.mpx_rope_fwd, p, 192, 4096, 192, p, 6, 12, 2, 1, 64, None, mx.MPX_BF16, 0)


def test_rope_plan_of_the_binding(mx):
    plan = mx.RopePlan([3, 5], base=[10.0, 20.0], interleaved=True)
    assert plan.axes == 2 and list(plan.pairs) == [3, 5, 0, 0] and list(plan.base)[:2] == [10.0, 20.0]
    assert plan.interleaved == 1
    for bad in ([], [1] * 5):
        with pytest.raises(ValueError):
            mx.RopePlan(bad)
    with pytest.raises(ValueError):
        mx.RopePlan([3, 5], base=[10.0])


@pytest.mark.parametrize("pairs", [[2 ** 32 + 8, 3], [8, 2 ** 31], [-2 ** 32 + 4], [-2 ** 31 - 1]])
def test_rope_plan_keeps_no_part_of_a_number(mx, pairs):
    """Counts that do not fit the plan's fields are refused, not cut to 32 bits."""
    with pytest.raises(ValueError, match="pairs"):
        mx.RopePlan(pairs)
    plan = mx.RopePlan([2 ** 31 - 1, -2 ** 31])   # they fit: the calls refuse them
    assert list(plan.pairs)[:2] == [2 ** 31 - 1, -2 ** 31]
    refused(mx, "pairs", mx.mpx_rope_fwd, p, 192, 4096, 192, p, 6, 12, 2, 1, 64, plan, mx.MPX_BF16, 0)


# Z ldz targets rows V k logp entropy stats top idx dt ws bytes stream
@pytest.mark.parametrize("change, match", [
    ({0: None}, "NULL"), ({2: None}, "targets"), ({3: 0}, "sizes"), ({4: 0}, "sizes"), ({4: 1 << 31}, "sizes"),
    ({3: 1 << 40}, "sizes"), ({1: 99}, "stride"), ({5: 17}, "k must"), ({5: -1}, "k must"),
    ({4: 3, 5: 4}, "k must"), ({9: None}, "top_logp"), ({10: None}, "top_logp"), ({5: 0}, "top_logp"),
    ({6: None, 7: None, 8: None, 5: 0, 9: None, 10: None}, "nothing to compute"), ({11: 5}, "MPX_F16"),
    ({0: 257}, "misaligned"), ({6: 258}, "misaligned"), ({10: 258}, "misaligned")])
def test_logprob_fwd_refusals(mx, change, match):
    args = [p, 100, p, 4, 100, 4, p, p, p, p, p, mx.MPX_F16, p, 1 << 40, 0]
    for i, v in change.items():
        args[i] = v
    refused(mx, match, mx.mpx_logprob_fwd, *args)


def test_logprob_workspace_is_checked(mx):
    for rows, V, k in [(1, 1 << 20, 8), (4, 262144, 0), (2, 100000, 16)]:
        need = mx.mpx_logprob_workspace(rows, V, k)
        if need:
            refused(mx, "workspace", mx.mpx_logprob_fwd, p, V, p, rows, V, k, p, p, p, p if k else None,
                    p if k else None, mx.MPX_F16, p, need - 1, 0)
            refused(mx, "workspace", mx.mpx_logprob_fwd, p, V, p, rows, V, k, p, p, p, p if k else None,
                    p if k else None, mx.MPX_F16, None, need, 0)


@pytest.mark.parametrize("rows, V, k", [(1, 1 << 20, 8), (4, 262144, 0), (2, 100000, 16), (1023, 65536, 4)])
def test_logprob_workspace_of_split_rows(mx, rows, V, k):
    """Few long rows are split: they need a workspace, and a call without it, or
    with a byte less, is refused.  Rows that fill the chip need none."""
    need = mx.mpx_logprob_workspace(rows, V, k)
    assert need >= rows * 2 * (12 + 8 * k)   # at least two splits
    top = p if k else None
    for ws, n in ((p, need - 1), (None, need), (p, 0)):
        refused(mx, "workspace", mx.mpx_logprob_fwd, p, V, p, rows, V, k, p, p, p, top, top, mx.MPX_F16, ws, n, 0)
    assert mx.mpx_logprob_workspace(4096, V, k) == 0


# Z ldz targets rows V k stats entropy idx g_logp g_entropy g_top state dZ ldo dt stream
@pytest.mark.parametrize("change, match", [
    ({0: None}, "NULL"), ({6: None}, "NULL"), ({13: None}, "NULL"), ({3: 0}, "sizes"), ({4: 0}, "sizes"),
    ({1: 99}, "stride"), ({14: 99}, "stride"), ({13: p, 14: 101}, "in place"), ({5: 17}, "k must"),
    ({9: None, 10: None, 11: None}, "nothing to compute"), ({2: None}, "targets"), ({7: None}, "entropy"),
    ({8: None}, "top_idx"), ({5: 0}, "top_idx"), ({15: 9}, "MPX_F16"), ({0: 257}, "misaligned"),
    ({13: 257}, "misaligned"), ({6: 258}, "misaligned"), ({11: 258}, "misaligned"),
    ({3: 1 << 23, 4: 1 << 30, 1: 1 << 30, 14: 1 << 30}, "too large")])
def test_logprob_bwd_refusals(mx, change, match):
    args = [p, 100, p, 4, 100, 4, p, p, p, p, p, p, p, 4096, 100, mx.MPX_F16, 0]
    for i, v in change.items():
        args[i] = v
    refused(mx, match, mx.mpx_logprob_bwd, *args)
