// Activation checkpoints in 8 bits: e4m3 codes with one power-of-two scale per
// 32 rows of a column (the format is documented at mpx_act8_pack).
#include <hip/hip_runtime.h>

#include "common.h"
#include "mfma.h"

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

// Byte- and halfword-aligned vectors (global accesses need no alignment on gfx950)
typedef uint16_t act8_u16x2 __attribute__((ext_vector_type(2)));
typedef u32x4 act8_u32x4_any __attribute__((aligned(2)));
typedef u32x2 act8_u32x2_any __attribute__((aligned(1)));

__device__ __forceinline__ uint32_t pk_max_u16(uint32_t a, uint32_t b) {
  return __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(act8_u16x2, a),
                                                                __builtin_bit_cast(act8_u16x2, b)));
}

// Rows a thread takes of its group, 8 threads apart; 32 columns of 8 values (the
// threads of half a wave) and 8 threads down the rows make a workgroup.
constexpr int kAct8Rows = 4;

// This thread's 8 columns and group: chunks of 8 columns are numbered group by
// group, so a workgroup's 32 columns of threads are always taken (588 columns
// would leave 44% of 256-column tiles idle).  The last chunk of a row ends at
// its last column: where K is no multiple of 8 some columns are done twice, with
// the same result.
struct Act8Place {
  int64_t group, col;
  bool valid;
  __device__ __forceinline__ Act8Place(int64_t M, int64_t K) {
    const uint32_t per = (uint32_t)((K + 7) / 8);
    const uint32_t id = blockIdx.x * 32 + (threadIdx.x & 31);
    const uint32_t g = id / per;
    valid = g < (uint32_t)((M + MPX_ACT8_GROUP - 1) / MPX_ACT8_GROUP);
    group = g;
    col = min((int64_t)(id % per) * 8, K - 8);
  }
};

// Bound by HBM: 2 bytes in and 1 out per value (12608 x 2304 bf16 15.4 us, 5.7 TB/s;
// one thread per column and group 23.5 us at 12608 x 768, this 7.7).  One workgroup reads its rows
// once, 4 vectors of 16 bytes in flight per thread, finds the groups' largest
// magnitudes in the packed halves (as integers; a thread that sees +-inf or NaN,
// or the largest scale, takes a slower path of its own) and through LDS across
// its 8 rows of threads, and converts from registers.
template <int DT>
__global__ __launch_bounds__(256) void act8_pack_kernel(const uint16_t* __restrict__ X, int64_t ldx,
                                                        uint8_t* __restrict__ codes,
                                                        uint8_t* __restrict__ scales, int64_t M,
                                                        int64_t K) {
  constexpr uint32_t kInf = DT == MPX_F16 ? 0x7C00u : 0x7F80u;
  __shared__ u32x4 red[8][32];
  const int ct = threadIdx.x & 31, rt = threadIdx.x >> 5;
  const Act8Place at(M, K);
  const int64_t r0 = at.group * MPX_ACT8_GROUP + rt;
  u32x4 v[kAct8Rows];
  if (at.valid) {
#pragma unroll
    for (int i = 0; i < kAct8Rows; ++i)  // rows behind the last one read it again
      v[i] = *reinterpret_cast<const act8_u32x4_any*>(X + min(r0 + 8 * i, M - 1) * ldx + at.col);
  }
  bool special = false;
  u32x4 amax = {0u, 0u, 0u, 0u};
  if (at.valid) {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
#pragma unroll
      for (int i = 0; i < kAct8Rows; ++i) amax[j] = pk_max_u16(amax[j], v[i][j] & 0x7FFF7FFFu);
      special |= (amax[j] & 0xFFFFu) >= kInf || (amax[j] >> 16) >= kInf;
    }
    if (special) {
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        amax[j] = 0;
#pragma unroll
        for (int i = 0; i < kAct8Rows; ++i) {
          const uint32_t lo = v[i][j] & 0x7FFFu, hi = (v[i][j] >> 16) & 0x7FFFu;
          amax[j] = pk_max_u16(amax[j], (lo < kInf ? lo : 0u) | ((hi < kInf ? hi : 0u) << 16));
        }
      }
    }
  }
  red[rt][ct] = amax;
  __syncthreads();
  if (!at.valid) return;
  amax = red[0][ct];
#pragma unroll
  for (int i = 1; i < 8; ++i) {
    const u32x4 o = red[i][ct];
#pragma unroll
    for (int j = 0; j < 4; ++j) amax[j] = pk_max_u16(amax[j], o[j]);
  }
  int e[8];
  float inv[8];
  u32x2 sc = {0u, 0u};
#pragma unroll
  for (int c = 0; c < 8; ++c) {
    const uint16_t h = (uint16_t)(amax[c / 2] >> (16 * (c & 1)));
    e[c] = act8_exponent<DT>(__builtin_bit_cast(uint32_t, h2f<DT>(h)));
    inv[c] = __builtin_bit_cast(float, (uint32_t)(127 - e[c]) << 23);  // 2^-e
    sc[c / 4] |= (uint32_t)(e[c] + 127) << (8 * (c & 3));
    special |= e[c] == kAct8Emax<DT>;
  }
  if (rt == 0) *reinterpret_cast<act8_u32x2_any*>(scales + at.group * K + at.col) = sc;
#pragma unroll
  for (int i = 0; i < kAct8Rows; ++i) {
    if (r0 + 8 * i >= M) break;
    u32x2 q = {0u, 0u};
    if (special) {
#pragma unroll
      for (int c = 0; c < 8; ++c)
        q[c / 4] |= (uint32_t)act8_code<DT>((uint16_t)(v[i][c / 2] >> (16 * (c & 1))), e[c]) << (8 * (c & 3));
    } else {
      float y[8];
#pragma unroll
      for (int c = 0; c < 8; ++c) y[c] = h2f<DT>((uint16_t)(v[i][c / 2] >> (16 * (c & 1)))) * inv[c];
#pragma unroll
      for (int w = 0; w < 2; ++w) {
        const int lo = __builtin_amdgcn_cvt_pk_fp8_f32(y[4 * w], y[4 * w + 1], 0, false);
        q[w] = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(y[4 * w + 2], y[4 * w + 3], lo, true);
      }
    }
    *reinterpret_cast<act8_u32x2_any*>(codes + (r0 + 8 * i) * K + at.col) = q;
  }
}

// The same places the other way round (16640 x 1536 f16 13.5 to 15 us, 5.1 to 5.7 TB/s;
// one thread per column and group 43).
template <int DT>
__global__ __launch_bounds__(256) void act8_unpack_kernel(const uint8_t* __restrict__ codes,
                                                          const uint8_t* __restrict__ scales,
                                                          uint16_t* __restrict__ Y, int64_t ldy,
                                                          int64_t M, int64_t K) {
  const int rt = threadIdx.x >> 5;
  const Act8Place at(M, K);
  if (!at.valid) return;
  const int64_t r0 = at.group * MPX_ACT8_GROUP + rt;
  const u32x2 sc = *reinterpret_cast<const act8_u32x2_any*>(scales + at.group * K + at.col);
  u32x2 q[kAct8Rows];
#pragma unroll
  for (int i = 0; i < kAct8Rows; ++i)
    q[i] = *reinterpret_cast<const act8_u32x2_any*>(codes + min(r0 + 8 * i, M - 1) * K + at.col);
  float s[8];
#pragma unroll
  for (int c = 0; c < 8; ++c)
    s[c] = __builtin_bit_cast(float, ((sc[c / 4] >> (8 * (c & 3))) & 0xFFu) << 23);
#pragma unroll
  for (int i = 0; i < kAct8Rows; ++i) {
    if (r0 + 8 * i >= M) break;
    u32x4 y;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const auto p = j & 1 ? __builtin_amdgcn_cvt_pk_f32_fp8((int)q[i][j / 2], true)
                           : __builtin_amdgcn_cvt_pk_f32_fp8((int)q[i][j / 2], false);
      y[j] = f2h<DT>(p[0] * s[2 * j]) | ((uint32_t)f2h<DT>(p[1] * s[2 * j + 1]) << 16);
    }
    *reinterpret_cast<act8_u32x4_any*>(Y + (r0 + 8 * i) * ldy + at.col) = y;
  }
}

// Fewer than 8 columns: one thread per column and group.
template <int DT>
__global__ __launch_bounds__(256) void act8_pack_narrow_kernel(const uint16_t* __restrict__ X, int64_t ldx,
                                                               uint8_t* __restrict__ codes,
                                                               uint8_t* __restrict__ scales, int64_t M,
                                                               int64_t K) {
  const int64_t id = (int64_t)blockIdx.x * 256 + threadIdx.x, g = id / K, c = id % K;
  const int64_t r0 = g * MPX_ACT8_GROUP, r1 = min(M, r0 + MPX_ACT8_GROUP);
  if (r0 >= M) return;
  uint32_t a = 0;
  for (int64_t r = r0; r < r1; ++r) a = max(a, finite_bits<DT>(X[r * ldx + c]));
  const int e = act8_exponent<DT>(a);
  scales[g * K + c] = (uint8_t)(e + 127);
  for (int64_t r = r0; r < r1; ++r) codes[r * K + c] = act8_code<DT>(X[r * ldx + c], e);
}

template <int DT>
__global__ __launch_bounds__(256) void act8_unpack_narrow_kernel(const uint8_t* __restrict__ codes,
                                                                 const uint8_t* __restrict__ scales,
                                                                 uint16_t* __restrict__ Y, int64_t ldy,
                                                                 int64_t M, int64_t K) {
  const int64_t id = (int64_t)blockIdx.x * 256 + threadIdx.x, r = id / K, c = id % K;
  if (r >= M) return;
  const float s = __builtin_bit_cast(float, (uint32_t)scales[r / MPX_ACT8_GROUP * K + c] << 23);
  Y[r * ldy + c] = f2h<DT>(__builtin_amdgcn_cvt_f32_fp8((int)codes[r * K + c], 0) * s);
}

static unsigned act8_blocks(int64_t M, int64_t K) {
  return (unsigned)cdiv(cdiv(M, MPX_ACT8_GROUP) * cdiv(K, 8), 32);
}

template <int DT>
static hipError_t launch_pack(const uint16_t* X, int64_t ldx, uint8_t* codes, uint8_t* scales, int64_t M,
                              int64_t K, hipStream_t s) {
  if (K < 8)
    act8_pack_narrow_kernel<DT>
        <<<(unsigned)cdiv(cdiv(M, MPX_ACT8_GROUP) * K, 256), 256, 0, s>>>(X, ldx, codes, scales, M, K);
  else
    act8_pack_kernel<DT><<<act8_blocks(M, K), 256, 0, s>>>(X, ldx, codes, scales, M, K);
  return hipGetLastError();
}

template <int DT>
static hipError_t launch_unpack(const uint8_t* codes, const uint8_t* scales, uint16_t* Y, int64_t ldy,
                                int64_t M, int64_t K, hipStream_t s) {
  if (K < 8)
    act8_unpack_narrow_kernel<DT><<<(unsigned)cdiv(M * K, 256), 256, 0, s>>>(codes, scales, Y, ldy, M, K);
  else
    act8_unpack_kernel<DT><<<act8_blocks(M, K), 256, 0, s>>>(codes, scales, Y, ldy, M, K);
  return hipGetLastError();
}

static hipError_t launch_act8_unpack(const uint8_t* codes, const uint8_t* scales, uint16_t* Y, int64_t ldy,
                              int64_t M, int64_t K, mpx_dtype dt, hipStream_t s) {
  return dt == MPX_F16 ? launch_unpack<MPX_F16>(codes, scales, Y, ldy, M, K, s)
                       : launch_unpack<MPX_BF16>(codes, scales, Y, ldy, M, K, s);
}

}  // namespace mpx

using namespace mpx;

// One launch holds fewer than 2^32 work-items.  Each takes 32 values, so 2^36 values
// make 2^31, and less than twice that where the last group of rows is short (33 rows
// are two groups); in narrow matrices each takes one value, up to 2^31.
static bool act8_fits(int64_t M, int64_t K) {
  return K <= INT32_MAX && M <= ((int64_t)1 << (K < 8 ? 31 : 36)) / (K < 8 ? K : 8 * cdiv(K, 8));
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
  MPX_HIP(dt == MPX_F16 ? launch_pack<MPX_F16>((const uint16_t*)X, ldx, codes, scales, M, K, s)
                        : launch_pack<MPX_BF16>((const uint16_t*)X, ldx, codes, scales, M, K, s));
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
