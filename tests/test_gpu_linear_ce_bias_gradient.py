"""The linear cross entropy's bias gradient over many rows, alone and beside dW."""
import numpy as np
import pytest

from tests.gpu_util import HAVE_GPU, to_host, ulp

pytestmark = [pytest.mark.gpu, pytest.mark.skipif(not HAVE_GPU, reason="no GPU")]

if HAVE_GPU:
    import torch
    from paper_2507_03312_amd import binding as mx
    TYPES = {"f16": torch.float16, "bf16": torch.bfloat16}


@pytest.mark.parametrize("fmt", ["f16", "bf16"])
@pytest.mark.parametrize("M", [5, 4096, 4097, 70001, 1 << 18, 1 << 20])
@pytest.mark.parametrize("dw", [False, True], ids=["alone", "beside dW"])
def test_equal_rows_add_up(fmt, M, dw):
    """Rows of 16 equal logits with one target for all: every other column's dz is the same
    value v of the half type in every row (f / 16, and p = 1 / 16 is off by 2^-22 at most), the
    hardest case for a long float32 chain, whose every step is rounded the same way.  v has 8 or
    11 bits; of n of them a sum below 2^(24 - bits) n is exact, and no chain of these sums is longer
    than 2^12: what is left are joins, 16 + 6 roundings of 2^-24 at most, and the result's half step."""
    V, K, scale = 16, 8, 2.0 ** 11
    v = {"bf16": 181 / 128, "f16": 1447 / 1024}[fmt] * 2.0 ** -10
    x, w = (torch.zeros(n, K, dtype=TYPES[fmt], device="cuda") for n in (M, V))
    t = torch.full((M,), 3, dtype=torch.int32, device="cuda")
    st = torch.tensor([0.0, np.log(16.0)], dtype=torch.float32, device="cuda").repeat(M, 1)
    g = torch.full((M,), 16 * v / scale, device="cuda")
    state = torch.tensor([scale, 0.0, 0.0, 2.0, 1.0, 2.0 ** 100], device="cuda")
    db = torch.full((V,), -7.0, dtype=TYPES[fmt], device="cuda")
    grad = torch.empty_like(w)
    ws = torch.empty(mx.mpx_linear_ce_bwd_workspace(M, V, K), dtype=torch.uint8, device="cuda")
    mx.mpx_linear_ce_bwd(x.data_ptr(), w.data_ptr(), None, t.data_ptr(), M, V, K, st.data_ptr(), g.data_ptr(),
                         state.data_ptr(), None, grad.data_ptr() if dw else None, db.data_ptr(), mx.DTYPES[fmt],
                         ws.data_ptr(), ws.numel(), None, torch.cuda.current_stream().cuda_stream)
    got, want = np.delete(to_host(db), 3).astype(np.float64), M * v
    # up to 128 rows what rounding left of f p is added too
    bound = 0.5 * (1 + 2.0 ** -10) * ulp(np.float64(want), fmt) + want * (22 * 2.0 ** -24 + 2.0 ** -22)
    assert (np.abs(got - want) <= bound).all(), (got, want)
