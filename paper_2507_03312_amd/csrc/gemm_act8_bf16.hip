// Weight gradients from 8-bit checkpoints for bf16 (see gemm_act8.h).
#include "gemm_act8.h"

namespace mpx {

hipError_t run_gemm_act8_bf16(const GemmArgs& g, hipStream_t s, bool* db_fused) {
  return run_gemm_act8<MPX_BF16>(g, s, db_fused);
}

}  // namespace mpx
