// Linear cross entropy for f16 operands: dW and dX in one launch (see linear_ce.h).
#include "linear_ce.h"

namespace mpx {

hipError_t run_ce_out_pair_f16(const CeOutArgs& w, RowTile tw, const CeOutArgs& x, RowTile tx, hipStream_t s) {
  return launch_ce_out_pair<MPX_F16>(w, tw, x, tx, s);
}

}  // namespace mpx
