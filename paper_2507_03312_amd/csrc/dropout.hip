// Dropout from a counter-based generator (mpx_dropout_fwd, mpx_dropout_bwd,
// mpx_rng_advance): the mask is a function of (seed, step, site, element), made again
// wherever it is needed and never stored.
#include <cmath>

#include "mfma.h"

namespace mpx {

// Philox4x32-10 (Salmon, Moraes, Dror and Shaw, "Parallel random numbers: as easy as 1, 2,
// 3", SC 2011): ten rounds of two 32 x 32 -> 64 products over a counter of four words.
__device__ __forceinline__ u32x4 philox(uint32_t c0, uint32_t c1, uint32_t c2, uint32_t c3, uint32_t k0,
                                        uint32_t k1) {
#pragma unroll
  for (int r = 0; r < 10; ++r) {
    const uint64_t a = (uint64_t)0xD2511F53u * c0, b = (uint64_t)0xCD9E8D57u * c2;
    c0 = (uint32_t)(b >> 32) ^ c1 ^ k0;
    c1 = (uint32_t)b;
    c2 = (uint32_t)(a >> 32) ^ c3 ^ k1;
    c3 = (uint32_t)a;
    k0 += 0x9E3779B9u;
    k1 += 0xBB67AE85u;
  }
  return u32x4{c0, c1, c2, c3};
}

template <int DT> struct DropValue { typedef uint16_t type; };
template <> struct DropValue<MPX_F32> { typedef float type; };

typedef u32x4 drop_u32x4 __attribute__((aligned(2)));

// 8 values, or the first n of them, at any alignment of theirs
template <int DT>
__device__ __forceinline__ void drop_load(const typename DropValue<DT>::type* p, int n, float (&v)[8]) {
  typedef typename DropValue<DT>::type T;
  constexpr int W = 8 * sizeof(T) / 16;
  T t[8];
  if (n >= 8) {
    drop_u32x4 w[W];
#pragma unroll
    for (int i = 0; i < W; ++i) w[i] = reinterpret_cast<const drop_u32x4*>(p)[i];
    __builtin_memcpy(t, w, sizeof(t));
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e) t[e] = e < n ? p[e] : T(0);
  }
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    if constexpr (DT == MPX_F32) v[e] = t[e];
    else v[e] = h2f<DT>(t[e]);
  }
}
template <int DT>
__device__ __forceinline__ void drop_store(typename DropValue<DT>::type* p, int n, const float (&v)[8]) {
  typedef typename DropValue<DT>::type T;
  constexpr int W = 8 * sizeof(T) / 16;
  T t[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    if constexpr (DT == MPX_F32) t[e] = v[e];
    else t[e] = f2h<DT>(v[e]);
  }
  if (n >= 8) {
    drop_u32x4 w[W];
    __builtin_memcpy(w, t, sizeof(t));
#pragma unroll
    for (int i = 0; i < W; ++i) reinterpret_cast<drop_u32x4*>(p)[i] = w[i];
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if (e < n) p[e] = t[e];
  }
}

// One counter block for 8 values, a 16-bit draw each (so p counts in steps of 2^-16):
// word e / 2, the lower half for even e.  Kept when the draw is `least` or more.  Bound by HBM:
// the 20 products of a block hide behind its loads (9.7 M values bf16 with a residual and
// back 19 us for 97 MB, 5.0 TB/s, what a large copy reaches); no mask is written or read.
template <int DT, bool RES>
__global__ __launch_bounds__(256) void dropout_kernel(const typename DropValue<DT>::type* X,
                                                      const typename DropValue<DT>::type* R,
                                                      typename DropValue<DT>::type* Y, int64_t n, uint32_t least,
                                                      float scale, const mpx_rng_state* rng, uint32_t site) {
  const uint64_t seed = rng->seed, step = rng->step;
  const int64_t block = (int64_t)blockIdx.x * 256 + threadIdx.x;
  const int64_t at = block * 8;
  if (at >= n) return;
  const int left = (int)min<int64_t>(8, n - at);
  float x[8], r[8];
  drop_load<DT>(X + at, left, x);
  if constexpr (RES) drop_load<DT>(R + at, left, r);
  const u32x4 w = philox((uint32_t)block, site, (uint32_t)step, (uint32_t)(step >> 32), (uint32_t)seed,
                         (uint32_t)(seed >> 32));
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const uint32_t draw = (w[e / 2] >> (16 * (e & 1))) & 0xFFFFu;
    x[e] = draw >= least ? x[e] * scale : 0.0f;  // a dropped NaN or infinity is 0 as well
    if constexpr (RES) x[e] += r[e];
  }
  drop_store<DT>(Y + at, left, x);
}

__global__ void rng_advance_kernel(mpx_rng_state* rng) { rng->step += 1; }

static int dropout(const char* fn, const void* X, const void* R, void* Y, int64_t n, double p,
                   const mpx_rng_state* rng, uint32_t site, mpx_dtype dt, void* stream) {
  const char* why = nullptr;
  const int size = dt == MPX_F32 ? 4 : 2;
  const auto mis = [&](const void* q) { return reinterpret_cast<uintptr_t>(q) % size != 0; };
  if (!X || !Y || !rng) why = "NULL operand";
  else if (!is_half(dt) && dt != MPX_F32) why = "dt must be MPX_F16, MPX_BF16 or MPX_F32";
  else if (n < 1 || n > ((int64_t)1 << 34)) why = "n must be in [1, 2^34]";
  else if (!(p >= 0.0 && p < 1.0)) why = "p must be in [0, 1)";
  else if (std::nearbyint(p * 65536.0) > 65535.0) why = "p must be below 1 - 2^-17";
  else if (mis(X) || mis(R) || mis(Y) || reinterpret_cast<uintptr_t>(rng) % 8 != 0)
    why = "pointers must be aligned to their element";
  if (why) {
    set_error(std::string(fn) + ": " + why);
    return MPX_ERR_INVALID;
  }
  const uint32_t least = (uint32_t)std::nearbyint(p * 65536.0);
  const float scale = (float)(65536.0 / (65536.0 - least));
  const unsigned blocks = (unsigned)cdiv(n, 2048);
  hipStream_t s = (hipStream_t)stream;
#define MPX_DROP(DTv)                                                                                       \
  do {                                                                                                      \
    typedef DropValue<DTv>::type T;                                                                         \
    const T *x = (const T*)X, *r = (const T*)R;                                                             \
    if (R) dropout_kernel<DTv, true><<<blocks, 256, 0, s>>>(x, r, (T*)Y, n, least, scale, rng, site);       \
    else dropout_kernel<DTv, false><<<blocks, 256, 0, s>>>(x, r, (T*)Y, n, least, scale, rng, site);        \
  } while (0)
  if (dt == MPX_F32) MPX_DROP(MPX_F32);
  else if (dt == MPX_F16) MPX_DROP(MPX_F16);
  else MPX_DROP(MPX_BF16);
#undef MPX_DROP
  MPX_LAUNCHED();
  return MPX_OK;
}

}  // namespace mpx

extern "C" int mpx_dropout_fwd(const void* X, const void* R, void* Y, int64_t n, double p,
                               const mpx_rng_state* d_rng, uint32_t site, mpx_dtype dt, void* stream) {
  mpx::clear_error();
  return mpx::dropout("mpx_dropout_fwd", X, R, Y, n, p, d_rng, site, dt, stream);
}

extern "C" int mpx_dropout_bwd(const void* dY, void* dX, int64_t n, double p, const mpx_rng_state* d_rng,
                               uint32_t site, mpx_dtype dt, void* stream) {
  mpx::clear_error();
  return mpx::dropout("mpx_dropout_bwd", dY, nullptr, dX, n, p, d_rng, site, dt, stream);
}

extern "C" int mpx_rng_advance(mpx_rng_state* d_rng, void* stream) {
  using namespace mpx;
  clear_error();
  MPX_REQUIRE(d_rng && reinterpret_cast<uintptr_t>(d_rng) % 8 == 0, "NULL or misaligned state");
  rng_advance_kernel<<<1, 1, 0, (hipStream_t)stream>>>(d_rng);
  MPX_LAUNCHED();
  return MPX_OK;
}
