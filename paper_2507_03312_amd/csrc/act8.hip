// Activation checkpoints in 8 bits: e4m3 codes with one power-of-two scale per
// 32 rows of a column (the format is documented at mpx_act8_pack).
#include <hip/hip_runtime.h>

#include "act8.h"
#include "common.h"

namespace mpx {

// Least and largest scale exponent: the code's smallest step (2^-9) times the
// least scale is the half type's smallest value (float16) or smallest normal
// value (bfloat16); the largest scale is the one its largest finite value needs.
template <int DT> constexpr int kAct8Emin = DT == MPX_F16 ? -15 : -117;
template <int DT> constexpr int kAct8Emax = DT == MPX_F16 ? 8 : 120;

// Scale exponent of a group whose largest finite magnitude has float32 bits a:
// the smallest e with a <= 448 2^e = 1.75 2^(e + 8).  Adding all mantissa bits
// up to that of 1.75 carries into the exponent exactly when a's mantissa exceeds
// 1.75.
template <int DT>
__device__ __forceinline__ int act8_exponent(uint32_t a) {
  const int e = (int)((a + 0x001FFFFFu) >> 23) - 127 - 8;
  return min(max(e, kAct8Emin<DT>), kAct8Emax<DT>);
}

// float32 bits of |h| of a finite half value, 0 for +-inf and NaN
template <int DT>
__device__ __forceinline__ uint32_t finite_bits(uint16_t h) {
  return h_nonfinite<DT>(h) ? 0u : __builtin_bit_cast(uint32_t, h2f<DT>(h)) & 0x7FFFFFFFu;
}

// Code of one half value: the scaling is exact (a power of two; float32 holds
// every scaled half value), the conversion rounds once, to nearest even.
template <int DT>
__device__ __forceinline__ uint8_t act8_code(uint16_t h, int e) {
  if (h_nonfinite<DT>(h)) return 0x7F;
  const float y = __builtin_ldexpf(h2f<DT>(h), -e);
  uint32_t c = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(y, y, 0, false) & 0xFFu;
  // 256 at the largest scale is infinite in the half type: held as 240
  if (e == kAct8Emax<DT> && (c & 0x7Fu) > 0x77u) c = (c & 0x80u) | 0x77u;
  return (uint8_t)c;
}

// One thread per column and group.
template <int DT>
__global__ __launch_bounds__(256) void act8_pack_kernel(const uint16_t* __restrict__ X, int64_t ldx,
                                                        uint8_t* __restrict__ codes,
                                                        uint8_t* __restrict__ scales, int64_t M,
                                                        int64_t K, int64_t col_blocks) {
  const int64_t g = blockIdx.x / col_blocks;
  const int64_t c = (blockIdx.x % col_blocks) * 256 + threadIdx.x;
  if (c >= K) return;
  const int64_t r0 = g * MPX_ACT8_GROUP, r1 = min(M, r0 + MPX_ACT8_GROUP);
  uint32_t a = 0;
  for (int64_t r = r0; r < r1; ++r) a = max(a, finite_bits<DT>(X[r * ldx + c]));
  const int e = act8_exponent<DT>(a);
  scales[g * K + c] = (uint8_t)(e + 127);
  for (int64_t r = r0; r < r1; ++r) codes[r * K + c] = act8_code<DT>(X[r * ldx + c], e);
}

template <int DT>
__global__ __launch_bounds__(256) void act8_unpack_kernel(const uint8_t* __restrict__ codes,
                                                          const uint8_t* __restrict__ scales,
                                                          uint16_t* __restrict__ Y, int64_t ldy,
                                                          int64_t M, int64_t K, int64_t col_blocks) {
  const int64_t g = blockIdx.x / col_blocks;
  const int64_t c = (blockIdx.x % col_blocks) * 256 + threadIdx.x;
  if (c >= K) return;
  const int64_t r0 = g * MPX_ACT8_GROUP, r1 = min(M, r0 + MPX_ACT8_GROUP);
  const int e = (int)scales[g * K + c] - 127;
  for (int64_t r = r0; r < r1; ++r) {
    const float v = __builtin_amdgcn_cvt_f32_fp8((int)codes[r * K + c], 0);
    Y[r * ldy + c] = f2h<DT>(__builtin_ldexpf(v, e));
  }
}

hipError_t launch_act8_unpack(const uint8_t* codes, const uint8_t* scales, uint16_t* Y, int64_t ldy,
                              int64_t M, int64_t K, mpx_dtype dt, hipStream_t s) {
  const int64_t cb = cdiv(K, 256);
  const unsigned blocks = (unsigned)(cdiv(M, MPX_ACT8_GROUP) * cb);
  if (dt == MPX_F16)
    act8_unpack_kernel<MPX_F16><<<blocks, 256, 0, s>>>(codes, scales, Y, ldy, M, K, cb);
  else
    act8_unpack_kernel<MPX_BF16><<<blocks, 256, 0, s>>>(codes, scales, Y, ldy, M, K, cb);
  return hipGetLastError();
}

}  // namespace mpx

using namespace mpx;

// workgroups of 32 rows x 256 columns that one launch holds (2^32 work-items)
static bool act8_fits(int64_t M, int64_t K) {
  return K <= INT32_MAX && cdiv(M, MPX_ACT8_GROUP) <= ((int64_t)1 << 23) / cdiv(K, 256);
}

extern "C" int mpx_act8_pack(const void* X, int64_t ldx, uint8_t* codes, uint8_t* scales, int64_t M,
                             int64_t K, mpx_dtype dt, void* stream) {
  clear_error();
  MPX_REQUIRE(X && codes && scales, "NULL operand");
  MPX_REQUIRE(M >= 1 && K >= 1, "M, K must be >= 1");
  MPX_REQUIRE(ldx >= K, "row stride below K");
  MPX_REQUIRE(is_half(dt), "dt must be MPX_F16 or MPX_BF16");
  MPX_REQUIRE((reinterpret_cast<uintptr_t>(X) & 1u) == 0, "X must be 2-byte aligned");
  MPX_REQUIRE(act8_fits(M, K), "M * K too large for one call");
  hipStream_t s = (hipStream_t)stream;
  const int64_t cb = cdiv(K, 256);
  const unsigned blocks = (unsigned)(cdiv(M, MPX_ACT8_GROUP) * cb);
  if (dt == MPX_F16)
    act8_pack_kernel<MPX_F16><<<blocks, 256, 0, s>>>((const uint16_t*)X, ldx, codes, scales, M, K, cb);
  else
    act8_pack_kernel<MPX_BF16><<<blocks, 256, 0, s>>>((const uint16_t*)X, ldx, codes, scales, M, K, cb);
  MPX_LAUNCHED();
  return MPX_OK;
}

extern "C" int mpx_act8_unpack(const uint8_t* codes, const uint8_t* scales, void* Y, int64_t ldy,
                               int64_t M, int64_t K, mpx_dtype dt, void* stream) {
  clear_error();
  MPX_REQUIRE(codes && scales && Y, "NULL operand");
  MPX_REQUIRE(M >= 1 && K >= 1, "M, K must be >= 1");
  MPX_REQUIRE(ldy >= K, "row stride below K");
  MPX_REQUIRE(is_half(dt), "dt must be MPX_F16 or MPX_BF16");
  MPX_REQUIRE((reinterpret_cast<uintptr_t>(Y) & 1u) == 0, "Y must be 2-byte aligned");
  MPX_REQUIRE(act8_fits(M, K), "M * K too large for one call");
  MPX_HIP(launch_act8_unpack(codes, scales, (uint16_t*)Y, ldy, M, K, dt, (hipStream_t)stream));
  return MPX_OK;
}
