// Ends of the tile kernels of gemm_kernels.h that work on float32 rows: accumulators
// through LDS, 8 halves at any address.  Internal; not part of the ABI.
#pragma once

#include "gemm_kernels.h"

namespace mpx {

// A wave's accumulators, 32 rows of 64 columns at a time, through its own LDS region
// into the row layout, in float32.
constexpr int kRowsPitch = 68;  // a column of 32 rows spreads over all banks
constexpr int kRowsBytes = 32 * kRowsPitch * 4;
__device__ __forceinline__ void rows_put(const f32x16& a, float* lds, int lane, int col0) {
#pragma unroll
  for (int q = 0; q < 4; ++q)
    *reinterpret_cast<f32x4*>(lds + (lane & 31) * kRowsPitch + col0 + 8 * q + 4 * (lane >> 5)) =
        f32x4{a[4 * q], a[4 * q + 1], a[4 * q + 2], a[4 * q + 3]};
}
__device__ __forceinline__ void rows_get8(const float* p, float (&v)[8]) {
  const f32x4 lo = *reinterpret_cast<const f32x4*>(p), hi = *reinterpret_cast<const f32x4*>(p + 4);
#pragma unroll
  for (int c = 0; c < 4; ++c) {
    v[c] = lo[c];
    v[4 + c] = hi[c];
  }
}
template <int DT>
__device__ __forceinline__ u32x4 pack8(const float (&v)[8]) {
  u32x4 w;
#pragma unroll
  for (int k = 0; k < 4; ++k) w[k] = f2h<DT>(v[2 * k]) | ((uint32_t)f2h<DT>(v[2 * k + 1]) << 16);
  return w;
}
template <int DT>
__device__ __forceinline__ void unpack8(u32x4 w, float (&v)[8]) {
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    v[2 * k] = h2f<DT>((uint16_t)(w[k] & 0xFFFFu));
    v[2 * k + 1] = h2f<DT>((uint16_t)(w[k] >> 16));
  }
}
// 8 halves at p, or the first nc of them
__device__ __forceinline__ void store8(uint16_t* p, u32x4 w, int nc) {
  if (nc >= 8) {
    *reinterpret_cast<u32x4_any*>(p) = w;
  } else {
#pragma unroll
    for (int c = 0; c < 8; ++c)
      if (c < nc) p[c] = (uint16_t)(w[c / 2] >> (16 * (c & 1)));
  }
}
__device__ __forceinline__ u32x4 load8(const uint16_t* p, int nc) {
  if (nc >= 8) return *reinterpret_cast<const u32x4_any*>(p);
  u32x4 w = {0u, 0u, 0u, 0u};
#pragma unroll
  for (int c = 0; c < 8; ++c)
    if (c < nc) w[c / 2] |= (uint32_t)p[c] << (16 * (c & 1));
  return w;
}

}  // namespace mpx
