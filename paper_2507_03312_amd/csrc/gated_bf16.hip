// Gated feed-forward products for bf16 operands (see gemm_gated.h).
#include "gemm_gated.h"

namespace mpx {

hipError_t run_gated_fwd_bf16(const GemmArgs& g, int64_t pair, hipStream_t s) {
  return g.act == MPX_ACT_SILU ? run_gated_fwd<MPX_BF16, MPX_ACT_SILU>(g, pair, s)
                               : run_gated_fwd<MPX_BF16, MPX_ACT_GELU_TANH>(g, pair, s);
}
hipError_t run_gated_bwd_bf16(const GemmArgs& g, hipStream_t s) {
  return g.act == MPX_ACT_SILU ? run_gated_bwd<MPX_BF16, MPX_ACT_SILU>(g, s)
                               : run_gated_bwd<MPX_BF16, MPX_ACT_GELU_TANH>(g, s);
}

}  // namespace mpx
