// Log probabilities of given tokens with entropy and top alternatives, and the
// gradient at the logits (mpx_logprob_fwd, mpx_logprob_bwd).
#include <hip/hip_runtime.h>

#include <initializer_list>

#include "common.h"

namespace mpx {

template <int DT> struct LogitOf { typedef uint16_t type; };
template <> struct LogitOf<MPX_F32> { typedef float type; };

template <int DT>
__device__ __forceinline__ float logit(const typename LogitOf<DT>::type* z) {
  if constexpr (DT == MPX_F32) return *z;
  else return h2f<DT>(*z);
}

// Order of the alternatives as unsigned keys: by value (-0 as 0, NaN above
// all), then by the lower column.
__device__ __forceinline__ uint64_t rank_key(float v, uint32_t col) {
  const uint32_t b = __builtin_bit_cast(uint32_t, v + 0.0f);
  const uint32_t o = v != v ? 0xFFFFFFFFu : (b & 0x80000000u) ? ~b : b | 0x80000000u;
  return ((uint64_t)o << 32) | (uint32_t)~col;
}
__device__ __forceinline__ float rank_value(uint64_t key) {
  const uint32_t o = (uint32_t)(key >> 32);
  return __builtin_bit_cast(float, o == 0xFFFFFFFFu ? 0x7FC00000u : (o & 0x80000000u) ? o & 0x7FFFFFFFu : ~o);
}

struct LogprobOut {
  float *logp, *entropy, *stats, *top_logp;
  int32_t* top_idx;
};

// One workgroup per row.
template <int DT>
__global__ __launch_bounds__(256) void logprob_fwd_kernel(const void* Z, int64_t ldz,
                                                          const int32_t* targets, int64_t V, int k,
                                                          LogprobOut out) {
  typedef typename LogitOf<DT>::type T;
  __shared__ float fred[4];
  __shared__ uint64_t kred[4];
  const int64_t r = blockIdx.x;
  const T* z = (const T*)Z + r * ldz;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  float m = -INFINITY;
  for (int64_t j = threadIdx.x; j < V; j += 256) m = fmaxf(m, logit<DT>(z + j));
  m = wave_max(m);
  if (lane == 0) fred[wave] = m;
  __syncthreads();
  m = fmaxf(fmaxf(fred[0], fred[1]), fmaxf(fred[2], fred[3]));
  if (m == -INFINITY) m = 0.0f;  // nothing but masked logits (or NaN)
  __syncthreads();
  float s = 0.0f, w = 0.0f;
  for (int64_t j = threadIdx.x; j < V; j += 256) {
    const float d = logit<DT>(z + j) - m, e = expf(d);
    s += e;
    if (e > 0.0f) w = __builtin_fmaf(e, d, w);
  }
  s = wave_sum(s);
  w = wave_sum(w);
  if (lane == 0) fred[wave] = s;
  __syncthreads();
  s = (fred[0] + fred[1]) + (fred[2] + fred[3]);
  __syncthreads();
  if (lane == 0) fred[wave] = w;
  __syncthreads();
  w = (fred[0] + fred[1]) + (fred[2] + fred[3]);
  const bool empty = s == 0.0f;
  const float ln = logf(s);
  if (threadIdx.x == 0) {
    if (out.stats) {
      out.stats[2 * r] = empty ? -INFINITY : s != s ? NAN : m;
      out.stats[2 * r + 1] = empty ? 0.0f : ln;
    }
    if (out.entropy) out.entropy[r] = empty ? 0.0f : ln - w / s;
    if (out.logp) {
      const int32_t t = targets[r];
      out.logp[r] = t < 0 ? 0.0f : t >= V ? NAN : empty ? -INFINITY : (logit<DT>(z + t) - m) - ln;
    }
  }
  uint64_t last = ~0ull;
  for (int i = 0; i < k; ++i) {
    uint64_t best = 0;
    for (int64_t j = threadIdx.x; j < V; j += 256) {
      const uint64_t key = rank_key(logit<DT>(z + j), (uint32_t)j);
      if (key < last || i == 0) best = max(best, key);
    }
    for (int o = 32; o >= 1; o >>= 1) best = max(best, (uint64_t)__shfl_xor((unsigned long long)best, o));
    __syncthreads();
    if (lane == 0) kred[wave] = best;
    __syncthreads();
    last = max(max(kred[0], kred[1]), max(kred[2], kred[3]));
    if (threadIdx.x == 0) {
      out.top_idx[r * k + i] = (int32_t)~(uint32_t)last;
      out.top_logp[r * k + i] = empty ? -INFINITY : (rank_value(last) - m) - ln;
    }
  }
}

struct LogprobGrad {
  const int32_t *targets, *top_idx;
  const float *stats, *entropy, *g_logp, *g_entropy, *g_top;
  const mpx_scale_state* state;
};

template <int DT>
__global__ __launch_bounds__(256) void logprob_bwd_kernel(const void* Z, int64_t ldz, int64_t V, int k,
                                                          LogprobGrad g, void* dZ, int64_t ldo,
                                                          int64_t col_blocks) {
  typedef typename LogitOf<DT>::type T;
  const int64_t r = blockIdx.x / col_blocks;
  const int64_t j = (blockIdx.x % col_blocks) * 256 + threadIdx.x;
  if (j >= V) return;
  const float scale = g.state ? g.state->scale : 1.0f;
  const float m = g.stats[2 * r], ln = g.stats[2 * r + 1];
  const bool empty = m == -INFINITY;
  const int32_t t = g.g_logp ? g.targets[r] : -1;
  float up = 0.0f, own = 0.0f;  // cotangents of all log probabilities, and of column j's
  if (t >= 0) {
    const float gl = g.g_logp[r];
    up += t < V ? gl : NAN;
    if (t == j) own += gl;
  }
  if (g.g_top) {
    for (int i = 0; i < k; ++i) {
      const float gt = g.g_top[r * k + i];
      const int32_t c = g.top_idx[r * k + i];
      up += c >= 0 && c < V ? gt : NAN;
      if (c == j) own += gt;
    }
  }
  const float z = logit<DT>((const T*)Z + r * ldz + j);
  const float lp = (z - m) - ln, p = expf(lp);
  float d = own - p * up;
  if (g.g_entropy && p > 0.0f) d -= g.g_entropy[r] * p * (lp + g.entropy[r]);
  if (empty || z == -INFINITY) d = ln != ln ? NAN : 0.0f;
  T* o = (T*)dZ + r * ldo + j;
  if constexpr (DT == MPX_F32) *o = scale * d;
  else *o = f2h<DT>(scale * d);
}

}  // namespace mpx

using namespace mpx;

static bool aligned4(std::initializer_list<const void*> ps) {
  for (const void* p : ps)
    if (reinterpret_cast<uintptr_t>(p) % 4 != 0) return false;
  return true;
}

#define MPX_BY_TYPE(dt, CALL)                   \
  do {                                          \
    if (dt == MPX_F16) CALL(MPX_F16);           \
    else if (dt == MPX_BF16) CALL(MPX_BF16);    \
    else CALL(MPX_F32);                         \
  } while (0)

extern "C" size_t mpx_logprob_workspace(int64_t rows, int64_t V, int32_t k) {
  (void)rows;
  (void)V;
  (void)k;
  return 0;
}

extern "C" int mpx_logprob_fwd(const void* Z, int64_t ldz, const int32_t* targets, int64_t rows,
                               int64_t V, int32_t k, float* logp, float* entropy, float* stats,
                               float* top_logp, int32_t* top_idx, mpx_dtype dt, void* workspace,
                               size_t ws_bytes, void* stream) {
  clear_error();
  (void)workspace;
  (void)ws_bytes;
  MPX_REQUIRE(Z, "NULL logits");
  MPX_REQUIRE(is_half(dt) || dt == MPX_F32, "dt must be MPX_F16, MPX_BF16 or MPX_F32");
  MPX_REQUIRE(rows >= 1 && V >= 1 && V <= INT32_MAX && rows <= ((int64_t)1 << 23), "bad sizes");
  MPX_REQUIRE(ldz >= V, "row stride below V");
  MPX_REQUIRE(k >= 0 && k <= MPX_LOGPROB_MAX_K && k <= V, "k must be in [0, 16] and at most V");
  MPX_REQUIRE((top_logp != nullptr) == (k > 0) && (top_idx != nullptr) == (k > 0),
              "top_logp and top_idx go with k >= 1");
  MPX_REQUIRE(!logp || targets, "logp needs targets");
  MPX_REQUIRE(logp || entropy || stats || k > 0, "nothing to compute");
  MPX_REQUIRE(reinterpret_cast<uintptr_t>(Z) % (dt == MPX_F32 ? 4 : 2) == 0, "misaligned logits");
  MPX_REQUIRE(aligned4({targets, logp, entropy, stats, top_logp, top_idx}), "misaligned operand");
  const LogprobOut out = {logp, entropy, stats, top_logp, top_idx};
#define MPX_LP(DTv) \
  logprob_fwd_kernel<DTv><<<(unsigned)rows, 256, 0, (hipStream_t)stream>>>(Z, ldz, targets, V, k, out)
  MPX_BY_TYPE(dt, MPX_LP);
#undef MPX_LP
  MPX_LAUNCHED();
  return MPX_OK;
}

extern "C" int mpx_logprob_bwd(const void* Z, int64_t ldz, const int32_t* targets, int64_t rows,
                               int64_t V, int32_t k, const float* stats, const float* entropy,
                               const int32_t* top_idx, const float* g_logp, const float* g_entropy,
                               const float* g_top, const mpx_scale_state* d_state, void* dZ,
                               int64_t ldo, mpx_dtype dt, void* stream) {
  clear_error();
  MPX_REQUIRE(Z && dZ && stats, "NULL operand");
  MPX_REQUIRE(is_half(dt) || dt == MPX_F32, "dt must be MPX_F16, MPX_BF16 or MPX_F32");
  MPX_REQUIRE(rows >= 1 && V >= 1 && V <= INT32_MAX && rows <= ((int64_t)1 << 23), "bad sizes");
  MPX_REQUIRE(ldz >= V && ldo >= V, "row stride below V");
  MPX_REQUIRE(Z != dZ || ldz == ldo, "in place needs equal row strides");
  MPX_REQUIRE(k >= 0 && k <= MPX_LOGPROB_MAX_K && k <= V, "k must be in [0, 16] and at most V");
  MPX_REQUIRE(g_logp || g_entropy || g_top, "nothing to compute: no cotangent given");
  MPX_REQUIRE(!g_logp || targets, "g_logp needs targets");
  MPX_REQUIRE(!g_entropy || entropy, "g_entropy needs entropy");
  MPX_REQUIRE(!g_top || (top_idx && k > 0), "g_top needs top_idx and k >= 1");
  const uintptr_t mis = reinterpret_cast<uintptr_t>(Z) | reinterpret_cast<uintptr_t>(dZ);
  MPX_REQUIRE(mis % (dt == MPX_F32 ? 4 : 2) == 0, "misaligned logits");
  MPX_REQUIRE(aligned4({targets, stats, entropy, top_idx, g_logp, g_entropy, g_top, d_state}),
              "misaligned operand");
  const LogprobGrad g = {targets, top_idx, stats, entropy, g_logp, g_entropy, g_top, d_state};
  const int64_t cb = cdiv(V, 256);
  MPX_REQUIRE(rows <= ((int64_t)1 << 23) / cb, "rows * V too large for one call");
#define MPX_LP(DTv)                                                                                \
  logprob_bwd_kernel<DTv><<<(unsigned)(rows * cb), 256, 0, (hipStream_t)stream>>>(Z, ldz, V, k, g, dZ, \
                                                                                  ldo, cb)
  MPX_BY_TYPE(dt, MPX_LP);
#undef MPX_LP
  MPX_LAUNCHED();
  return MPX_OK;
}
