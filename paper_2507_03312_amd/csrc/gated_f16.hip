// Gated feed-forward products for f16 operands (see gemm_gated.h).
#include "gemm_gated.h"

namespace mpx {

hipError_t run_gated_fwd_f16(const GemmArgs& g, int64_t pair, RowTile t, hipStream_t s) {
  return g.act == MPX_ACT_SILU ? run_gated_fwd<MPX_F16, MPX_ACT_SILU>(g, pair, t, s)
                               : run_gated_fwd<MPX_F16, MPX_ACT_GELU_TANH>(g, pair, t, s);
}
hipError_t run_gated_bwd_f16(const GemmArgs& g, RowTile t, hipStream_t s) {
  return g.act == MPX_ACT_SILU ? run_gated_bwd<MPX_F16, MPX_ACT_SILU>(g, t, s)
                               : run_gated_bwd<MPX_F16, MPX_ACT_GELU_TANH>(g, t, s);
}

}  // namespace mpx
