// Launchers of the 8-bit activation checkpoints (act8.hip), for the linear
// backward that reads them.  Internal; not part of the ABI.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "mpx.h"

namespace mpx {

hipError_t launch_act8_unpack(const uint8_t* codes, const uint8_t* scales, uint16_t* Y, int64_t ldy,
                              int64_t M, int64_t K, mpx_dtype dt, hipStream_t s);

}  // namespace mpx
