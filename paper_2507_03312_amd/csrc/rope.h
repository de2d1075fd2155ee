// Rotary positions: what the kernels of mpx_rope_* and mpx_qknorm_rope_* share.
// Internal; not part of the ABI.
#pragma once

#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>

#include "common.h"

namespace mpx {

constexpr int kRopeMaxHd = 512;
constexpr int kRopeTable = 1024;  // turns (cosine, sine) that a workgroup holds in LDS

struct RopeArgs {
  const void* X;
  void* Y;
  const float* pos;
  int64_t ldx, ldy;
  uint32_t pos_rows, rows, heads_rot, copy;  // copy: values copied behind the turned heads
  int32_t hd, axes, npairs, interleaved, back, in_place;
  int32_t stream;  // more than the last-level cache holds
  // a workgroup's rows, and the threads that share a row's heads: thread
  // (slot, chunk) takes heads slot % head_slots, + head_slots, ... of row
  // slot / head_slots, with the pairs of `chunk` of each
  int32_t wg_rows, head_slots, chunks;
  int32_t first_pair[MPX_ROPE_MAX_AXES + 1];  // axis a owns pairs [first_pair[a], first_pair[a + 1])
  double step[MPX_ROPE_MAX_AXES];             // log2(base) / pairs
};

template <int DT> struct RopeValue { typedef uint16_t type; };
template <> struct RopeValue<MPX_F32> { typedef float type; };

typedef uint32_t rope_u32x4 __attribute__((ext_vector_type(4)));
typedef rope_u32x4 rope_u32x4_any __attribute__((aligned(2)));

// N values at any alignment of theirs (global accesses need no more on gfx950)
template <int DT, int N> struct RopeVec {
  typedef typename RopeValue<DT>::type T;
  T v[N];
  // NT (16-byte vectors): around the caches
  template <bool NT = false>
  __device__ __forceinline__ void load(const T* p) {
    if constexpr (NT) {
      const rope_u32x4 w = __builtin_nontemporal_load(reinterpret_cast<const rope_u32x4_any*>(p));
      __builtin_memcpy(v, &w, sizeof(v));
    } else {
      __builtin_memcpy(v, p, sizeof(v));
    }
  }
  template <bool NT = false>
  __device__ __forceinline__ void store(T* p) const {
    if constexpr (NT) {
      rope_u32x4 w;
      __builtin_memcpy(&w, v, sizeof(v));
      __builtin_nontemporal_store(w, reinterpret_cast<rope_u32x4_any*>(p));
    } else {
      __builtin_memcpy(p, v, sizeof(v));
    }
  }
  // the same vector of another lane
  __device__ __forceinline__ RopeVec from_lane(int l) const {
    constexpr int W = (sizeof(v) + 3) / 4;
    int w[W] = {};
    __builtin_memcpy(w, v, sizeof(v));
#pragma unroll
    for (int i = 0; i < W; ++i) w[i] = __builtin_amdgcn_ds_bpermute(4 * l, w[i]);
    RopeVec o;
    __builtin_memcpy(o.v, w, sizeof(v));
    return o;
  }
  __device__ __forceinline__ float get(int i) const {
    if constexpr (DT == MPX_F32) return v[i];
    else return h2f<DT>(v[i]);
  }
  __device__ __forceinline__ void set(int i, float f) {
    if constexpr (DT == MPX_F32) v[i] = f;
    else v[i] = f2h<DT>(f);
  }
};

// The turns of the workgroup's rows into LDS; ends with a barrier.
__device__ __forceinline__ void rope_turns(const RopeArgs& a, uint32_t row0, uint32_t nrows, float2* turns) {
  for (uint32_t i = threadIdx.x; i < nrows * a.npairs; i += 256) {
    const uint32_t r = i / a.npairs, p = i % a.npairs;
    int ax = 0;
#pragma unroll
    for (int k = 1; k < MPX_ROPE_MAX_AXES; ++k) ax += (int)p >= a.first_pair[k] ? 1 : 0;
    const double turn = exp2(-(double)((int)p - a.first_pair[ax]) * a.step[ax]) * 0.15915494309189533577;
    double t = (double)a.pos[(int64_t)((row0 + r) % a.pos_rows) * a.axes + ax] * turn;
    t -= rint(t);  // exact: what is left is at most half a turn
    float s, c;
    sincospif(2.0f * (float)t, &s, &c);
    turns[i] = make_float2(c, a.back ? -s : s);
  }
  __syncthreads();
}

// The copied heads of the workgroup's rows, from rows of ldx.
template <int DT>
__device__ __forceinline__ void rope_copies(const RopeArgs& a, const typename RopeValue<DT>::type* X, int64_t ldx,
                                            typename RopeValue<DT>::type* Y, uint32_t nrows) {
  typedef typename RopeValue<DT>::type T;
  if (!a.in_place && a.copy) {
    constexpr uint32_t VE = 16 / sizeof(T);
    const int64_t w0 = (int64_t)a.heads_rot * a.hd;
    const uint32_t nv = a.copy / VE, rest = a.copy % VE;
    for (uint32_t i = threadIdx.x; i < nrows * nv; i += 256) {
      const uint32_t r = i / nv, c = (i % nv) * VE;
      RopeVec<DT, VE> v;
      v.load(X + r * ldx + w0 + c);
      v.store(Y + r * a.ldy + w0 + c);
    }
    for (uint32_t i = threadIdx.x; i < nrows * rest; i += 256) {
      const int64_t r = i / rest, c = w0 + nv * VE + i % rest;
      Y[r * a.ldy + c] = X[r * ldx + c];
    }
  }
}

// A plan's checks and its places in `a`.  vw: values of one run, a power of two of at most
// 16 bytes that divides every section's halves (interleaved: twice the pairs) and what is
// not turned; vp: the same of pairs of runs.  NULL, or why it is refused.
inline const char* rope_plan(const mpx_rope_plan* plan, int64_t hd, mpx_dtype dt, RopeArgs& a, int& vw, int& vp) {
  if (plan->axes < 1 || plan->axes > MPX_ROPE_MAX_AXES) return "axes must be in [1, 4]";
  if (plan->interleaved != 0 && plan->interleaved != 1) return "interleaved must be 0 or 1";
  int64_t n = 0;
  const bool inter = plan->interleaved != 0;
  const int wide = dt == MPX_F32 ? 4 : 8;
  vw = wide;
  vp = hd % 2 ? 1 : wide;
  for (int ax = 0; ax < plan->axes; ++ax) {
    const int64_t p = plan->pairs[ax];
    const double base = plan->base[ax];
    if (p < 1 || 2 * (n + p) > hd) return "pairs must be >= 1 and 2 * their sum <= hd";
    if (!std::isfinite(base) || base <= 1.0) return "base must be finite and > 1";
    a.step[ax] = std::log2(base) / (double)p;
    a.first_pair[ax] = (int32_t)n;
    n += p;
    while (!inter && p % vw) vw /= 2;
    while (!inter && p % vp) vp /= 2;
  }
  while (2 * n % vw || (hd - 2 * n) % vw) vw /= 2;
  while (n % vp || (hd / 2 - n) % vp) vp /= 2;
  for (int ax = plan->axes; ax <= MPX_ROPE_MAX_AXES; ++ax) a.first_pair[ax] = (int32_t)n;
  a.axes = plan->axes;
  a.npairs = (int32_t)n;
  a.interleaved = plan->interleaved;
  a.hd = (int32_t)hd;
  return nullptr;
}

}  // namespace mpx
