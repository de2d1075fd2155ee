"""Host-side argument checks of the gated projections, the linear cross entropy, the norms
of queries and keys, and dropout: every refusal comes before anything is launched or
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


def refused(mx, match, fn, args, change):
    args = list(args)
    for i, v in change.items():
        args[i] = v
    with pytest.raises(mx.MPXError, match=match):
        fn(*args)


# X W b H Pre M N K dt act stream
@pytest.mark.parametrize("change, match", [
    ({0: None}, "NULL"), ({1: None}, "NULL"), ({3: None}, "NULL"), ({5: 0}, ">= 1"), ({6: 0}, ">= 1"),
    ({7: -1}, ">= 1"), ({5: 1 << 31}, "too large"), ({6: (1 << 24) + 1}, "too large"),
    ({7: (1 << 24) + 1}, "too large"), ({8: 3}, "MPX_F16"), ({9: 0}, "activation"), ({9: 3}, "activation"),
    ({8: 0, 4: None}, "Pre is required"), ({0: 257}, "aligned"), ({2: 257}, "aligned"), ({4: 257}, "aligned"),
    ({8: 0, 3: 258}, "aligned")])
def test_gated_fwd_refusals(mx, change, match):
    refused(mx, match, mx.mpx_gated_fwd, [p, p, p, p, p, 8, 16, 32, mx.MPX_BF16, mx.MPX_ACT_SILU, 0], change)


# X W dY Pre act dPre dW db M N K dt ws bytes nonfinite stream
@pytest.mark.parametrize("change, match", [
    ({2: None}, "NULL dY"), ({5: None, 6: None, 7: None}, "nothing to compute"), ({1: None}, "W and Pre"),
    ({3: None}, "W and Pre"), ({0: None}, "X is required"), ({8: 0}, ">= 1"), ({9: -2}, ">= 1"), ({10: 0}, ">= 1"),
    ({8: 1 << 31}, "too large"), ({11: 5}, "MPX_F16"), ({4: 0}, "activation"), ({4: 7}, "activation"),
    ({11: 0, 14: p}, "half gradients only"), ({5: 257}, "aligned"), ({12: None}, "workspace"), ({13: 0}, "workspace")])
def test_linear_bwd_gated_refusals(mx, change, match):
    need = mx.mpx_linear_bwd_gated_workspace(64, 32, 48)
    refused(mx, match, mx.mpx_linear_bwd_gated,
            [p, p, p, p, mx.MPX_ACT_SILU, p, p, p, 64, 32, 48, mx.MPX_BF16, p, need, None, 0], change)


def test_silu_is_no_activation_of_plain_layers(mx):
    """Only the gated calls know it; the linear ones refuse it as before."""
    refused(mx, "unknown activation", mx.mpx_linear_fwd,
            [p, p, None, None, p, p, 8, 8, 8, mx.MPX_BF16, mx.MPX_ACT_SILU, 0], {})
    refused(mx, "unknown activation", mx.mpx_linear_bwd,
            [p, p, p, p, mx.MPX_ACT_SILU, p, None, None, 8, 8, 8, mx.MPX_BF16, None, 0, None, 0], {})


# X W b targets M V K loss stats mean dt ws bytes stream
@pytest.mark.parametrize("change, match", [
    ({0: None}, "NULL"), ({1: None}, "NULL"), ({3: None}, "targets"), ({4: 0}, ">= 1"), ({5: 0}, ">= 1"),
    ({6: 0}, ">= 1"), ({4: (1 << 20) + 1}, "too large"), ({5: (1 << 24) + 1}, "too large"),
    ({6: (1 << 16) + 1}, "too large"), ({4: 1 << 20, 5: (1 << 16) + 1}, "too large"),
    ({5: 1 << 20, 6: 1 << 13}, "too large"), ({7: None, 8: None}, "nothing to compute"), ({7: None}, "its mean"),
    ({10: 0}, "MPX_F16"), ({10: 9}, "MPX_F16"), ({0: 257}, "aligned"), ({2: 257}, "aligned"), ({3: 258}, "aligned"),
    ({7: 258}, "aligned"), ({8: 260}, "aligned"), ({11: None}, "workspace"), ({12: 10}, "workspace"),
    ({11: 264}, "workspace")])
def test_linear_ce_fwd_refusals(mx, change, match):
    need = mx.mpx_linear_ce_fwd_workspace(64, 1000, 128)
    refused(mx, match, mx.mpx_linear_ce_fwd, [p, p, p, p, 64, 1000, 128, p, p, p, mx.MPX_F16, p, need, 0], change)


# X W b targets M V K stats g state dX dW db dt ws bytes nonfinite stream
@pytest.mark.parametrize("change, match", [
    ({0: None}, "NULL"), ({1: None}, "NULL"), ({3: None}, "NULL"), ({7: None}, "NULL"), ({4: 0}, ">= 1"),
    ({5: -1}, ">= 1"), ({6: 0}, ">= 1"), ({5: (1 << 24) + 1}, "too large"), ({10: None, 11: None, 12: None}, "nothing"),
    ({13: 0}, "MPX_F16"), ({7: 260}, "aligned"), ({8: 258}, "aligned"), ({11: 257}, "aligned"),
    ({14: None}, "workspace"), ({15: 10}, "workspace"), ({14: 264}, "workspace")])
def test_linear_ce_bwd_refusals(mx, change, match):
    need = mx.mpx_linear_ce_bwd_workspace(64, 1000, 128)
    refused(mx, match, mx.mpx_linear_ce_bwd,
            [p, p, p, p, 64, 1000, 128, p, p, p, p, p, p, mx.MPX_F16, p, need, None, 0], change)


def test_linear_ce_workspace_stays_below_the_logits(mx):
    """A large vocabulary's workspace is a piece of its logits, and does not grow with it."""
    sizes = [mx.mpx_linear_ce_bwd_workspace(4096, V, 768) for V in (32768, 65537, 131072, 1 << 20)]
    assert max(sizes) < 4096 * 65537 * 2 and max(sizes) < 1.5 * min(sizes)
    assert mx.mpx_linear_ce_fwd_workspace(4096, 131072, 768) < 4096 * 131072 * 2 / 16
    for f in (mx.mpx_linear_ce_fwd_workspace, mx.mpx_linear_ce_bwd_workspace):
        assert f(0, 5, 5) == f(5, 0, 5) == f(5, 5, -1) == 0 < f(1, 1, 1)


# X ldx Y ldy wq wk eps pos pos_rows rows hq hk copy hd plan dt stream
@pytest.mark.parametrize("change, match", [
    ({0: None}, "NULL"), ({2: None}, "NULL"), ({7: None}, "NULL"), ({14: None}, "NULL"), ({8: 0}, "multiple"),
    ({8: 7}, "multiple"), ({9: 0}, "multiple"), ({9: 1 << 24, 8: 1}, "rows"), ({10: 0}, "heads_q"),
    ({11: -1}, "heads_k"), ({12: -1}, "heads_copy"), ({10: 1 << 62}, "heads_q"), ({13: 1}, "hd"),
    ({13: 513, 1: 9999, 3: 9999}, "hd"), ({1: 255}, "stride"), ({3: 255}, "stride"), ({2: p, 3: 300}, "in place"),
    ({6: -1e-9}, "eps"), ({6: float("nan")}, "eps"), ({6: float("inf")}, "eps"), ({15: 3}, "MPX_F16"),
    ({0: 257}, "aligned"), ({4: 257}, "aligned"), ({7: 258}, "aligned")])
def test_qknorm_fwd_refusals(mx, change, match):
    refused(mx, match, mx.mpx_qknorm_rope_fwd,
            [p, 256, 4096, 256, p, p, 1e-6, p, 6, 12, 2, 1, 1, 64, mx.RopePlan([16, 16]), mx.MPX_BF16, 0], change)


# X ldx dY ldy dX ldo wq wk eps pos pos_rows rows hq hk copy hd plan dwq dwk dt ws bytes nonfinite stream
@pytest.mark.parametrize("change, match", [
    ({0: None}, "NULL"), ({2: None}, "NULL"), ({4: None}, "NULL"), ({1: 191}, "stride"), ({3: 255}, "stride"),
    ({5: 255}, "stride"), ({4: 8192, 5: 300}, "in place"), ({4: p}, "dX must not be X"), ({8: -1.0}, "eps"),
    ({19: 4}, "MPX_F16"), ({19: 0, 22: p}, "half gradients only"), ({17: 257}, "aligned"), ({20: None}, "workspace"),
    ({21: 12 * 2 * 64 * 4 - 1}, "workspace"), ({20: 258}, "workspace")])
def test_qknorm_bwd_refusals(mx, change, match):
    need = mx.mpx_qknorm_rope_bwd_workspace(12, 64)
    refused(mx, match, mx.mpx_qknorm_rope_bwd,
            [p, 256, 8192, 256, 4096, 256, p, p, 1e-6, p, 6, 12, 2, 1, 1, 64, mx.RopePlan([16, 16]), p, p,
             mx.MPX_BF16, p, need, None, 0], change)


def test_qknorm_plan_and_workspace(mx):
    plan = mx.RopePlan([16, 17])
    refused(mx, "pairs", mx.mpx_qknorm_rope_fwd,
            [p, 256, 4096, 256, p, p, 1e-6, p, 6, 12, 2, 1, 1, 64, plan, mx.MPX_BF16, 0], {})
    sizes = [mx.mpx_qknorm_rope_bwd_workspace(r, 128) for r in range(1, 5000, 7)]
    assert sizes == sorted(sizes) and sizes[0] > 0 == mx.mpx_qknorm_rope_bwd_workspace(0, 128)


# X R Y n p rng site dt stream
@pytest.mark.parametrize("change, match", [
    ({0: None}, "NULL"), ({2: None}, "NULL"), ({5: None}, "NULL"), ({3: 0}, "n must"), ({3: -5}, "n must"),
    ({3: (1 << 34) + 1}, "n must"), ({4: -0.1}, "p must"), ({4: 1.0}, "p must"), ({4: float("nan")}, "p must"),
    ({4: 1 - 2.0 ** -18}, "p must"), ({7: 3}, "MPX_F16"), ({0: 257}, "aligned"), ({1: 257}, "aligned"),
    ({5: 260}, "aligned"), ({7: 0, 2: 258}, "aligned")])
def test_dropout_refusals(mx, change, match):
    refused(mx, match, mx.mpx_dropout_fwd, [p, p, p, 100, 0.1, p, 0, mx.MPX_BF16, 0], change)
    if not {1} & set(change):
        back = {0: 0, 2: 1, 3: 2, 4: 3, 5: 4, 6: 5, 7: 6}
        refused(mx, match, mx.mpx_dropout_bwd, [p, p, 100, 0.1, p, 0, mx.MPX_BF16, 0],
                {back[i]: v for i, v in change.items()})


def test_dropout_sites_and_state(mx):
    for site in (-1, 2 ** 32, 2 ** 40):   # not cut to 32 bits
        with pytest.raises(ValueError, match="site"):
            mx.mpx_dropout_fwd(p, None, p, 100, 0.1, p, site, mx.MPX_BF16, 0)
        with pytest.raises(ValueError, match="site"):
            mx.mpx_dropout_bwd(p, p, 100, 0.1, p, site, mx.MPX_BF16, 0)
    refused(mx, "NULL", mx.mpx_rng_advance, [None, 0], {})
    refused(mx, "misaligned", mx.mpx_rng_advance, [260, 0], {})
