// Linear cross entropy for f16 operands (see linear_ce.h).
#include "linear_ce.h"

namespace mpx {

hipError_t run_ce_fwd_f16(const CeFwdArgs& g, RowTile t, hipStream_t s) {
  return launch_rows<MPX_F16, CeFwdArgs, true, true, false>(g, t, s);
}
hipError_t run_ce_grad_f16(const CeGradArgs& g, RowTile t, hipStream_t s) {
  return launch_rows<MPX_F16, CeGradArgs, true, true, false>(g, t, s);
}
hipError_t run_ce_out_f16(const CeOutArgs& g, bool ak, RowTile t, hipStream_t s) {
  if (ak) return launch_rows<MPX_F16, CeOutArgs, true, false, false>(g, t, s);
  return g.dbp || g.db ? launch_rows<MPX_F16, CeOutArgs, false, false, true>(g, t, s)
               : launch_rows<MPX_F16, CeOutArgs, false, false, false>(g, t, s);
}

}  // namespace mpx
