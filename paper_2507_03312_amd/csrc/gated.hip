// Gated feed-forward block (mpx_gated_fwd, mpx_linear_bwd_gated): argument checks, the
// kernel of few rows, the elementwise halves of the float32 form.
#include "gemm_f32.h"
#include "gemm_gated.h"

namespace mpx {

// Few rows (single tokens of some sequences), bound by one read of W: a workgroup makes
// 16 columns of H for up to 32 rows of X, its four waves a quarter of the reduction
// each, with as many loads in flight as that has steps.  A = 16 gate rows of W and the
// 16 other ones, B = X: lane l has row l % 32 of X, accumulators i and 8 + i are G and U of
// the same column.  The waves' sums are added in wave order.  4 x 2048 x 768 bf16 about 6 us
// for 6.3 MB: latency, of a launch and of one round of loads (128 workgroups).
template <int DT, int ACT>
__global__ __launch_bounds__(256) void gated_few_kernel(GemmArgs g) {
  __shared__ float part[4][16][64];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, r32 = lane & 31, hi = lane >> 5;
  const int64_t n0 = (int64_t)blockIdx.x * 16, m0 = (int64_t)blockIdx.y * 32;
  const int64_t wrow = min(n0 + (r32 & 15), g.N - 1) + (r32 >= 16 ? g.N : 0);
  const uint16_t* w = g.B + wrow * g.K;
  const uint16_t* x = g.A + min(m0 + r32, g.M - 1) * g.K;
  // the wave's k steps of 16: a quarter of them, rounded up
  const int steps = (int)((g.K + 15) / 16), per = (steps + 3) / 4;
  const int s0 = wave * per, s1 = min(steps, s0 + per);
  f32x16 acc;
#pragma unroll
  for (int e = 0; e < 16; ++e) acc[e] = 0.0f;
  constexpr int U = 12;
  for (int s = s0; s < s1; s += U) {
    u32x4 a[U], b[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int64_t k = 16 * (int64_t)min(s + u, s1 - 1) + 8 * hi;
      const int64_t kc = max((int64_t)0, min(k, g.K - 8));  // the loads end with the row
      if (g.K >= 8) {
        a[u] = *reinterpret_cast<const u32x4_any*>(w + kc);
        b[u] = *reinterpret_cast<const u32x4_any*>(x + kc);
      } else {
        a[u] = load8(w, hi ? 0 : (int)g.K);
        b[u] = load8(x, hi ? 0 : (int)g.K);
      }
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (s + u >= s1) break;  // uniform
      const int64_t k = 16 * (int64_t)(s + u) + 8 * hi;
      const int sh = g.K >= 8 ? (int)min<int64_t>(8, max((int64_t)0, k - (g.K - 8))) : 0;
      if (16 * (int64_t)(s + u) + 16 > g.K) {  // uniform: the last step, what is past the row dropped
        a[u] = StagedOperand<64, true, 4, false>::shr_halves(a[u], sh);
        b[u] = StagedOperand<64, true, 4, false>::shr_halves(b[u], sh);
      }
      acc = mfma32<DT>(__builtin_bit_cast(uint4, a[u]), __builtin_bit_cast(uint4, b[u]), acc);
    }
  }
#pragma unroll
  for (int e = 0; e < 16; ++e) part[wave][e][lane] = acc[e];
  __syncthreads();
  // wave w ends accumulators 2 w and 2 w + 1, two neighbouring columns
  const int64_t m = m0 + r32;
#pragma unroll
  for (int j = 0; j < 2; ++j) {
    const int i = 2 * wave + j;
    const int64_t n = n0 + 8 * (i / 4) + 4 * hi + i % 4;
    float a = part[0][i][lane], b = part[0][8 + i][lane];
#pragma unroll
    for (int w2 = 1; w2 < 4; ++w2) {
      a += part[w2][i][lane];
      b += part[w2][8 + i][lane];
    }
    if (m < g.M && n < g.N) {
      if (g.bias) {
        a += h2f<DT>(g.bias[n]);
        b += h2f<DT>(g.bias[g.N + n]);
      }
      g.C[m * g.N + n] = f2h<DT>(gate_act<ACT>(a) * b);
      if (g.pre) {
        g.pre[m * 2 * g.N + n] = f2h<DT>(a);
        g.pre[(m * 2 + 1) * g.N + n] = f2h<DT>(b);
      }
    }
  }
}

template <int DT>
static hipError_t launch_few(const GemmArgs& g, hipStream_t s) {
  const dim3 grid((unsigned)cdiv(g.N, 16), (unsigned)cdiv(g.M, 32));
  if (g.act == MPX_ACT_SILU) gated_few_kernel<DT, MPX_ACT_SILU><<<grid, 256, 0, s>>>(g);
  else gated_few_kernel<DT, MPX_ACT_GELU_TANH><<<grid, 256, 0, s>>>(g);
  return hipGetLastError();
}

// Float32: the product is the library's float32 one, into Pre (forward) or into dG's
// place (backward), and these end it.  BWD: P = Pre, D holds dH in its left half.
template <int ACT, bool BWD>
__global__ __launch_bounds__(256) void gated_f32_kernel(const float* P, float* D, float* H, int64_t M, int64_t N) {
  const int64_t stride = (int64_t)gridDim.x * 256;
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < M * N; i += stride) {
    const int64_t m = i / N, n = i - m * N, at = m * 2 * N + n;
    if constexpr (BWD) {
      float a, da;
      gate_act_grad<ACT>(P[at], a, da);
      const float d = D[at];
      D[at] = d * P[at + N] * da;
      D[at + N] = d * a;
    } else {
      H[i] = gate_act<ACT>(P[at]) * P[at + N];
    }
  }
}

template <bool BWD>
static hipError_t launch_f32(int32_t act, const float* P, float* D, float* H, int64_t M, int64_t N, hipStream_t s) {
  const unsigned blocks = (unsigned)std::min<int64_t>(cdiv(M * N, 256), 4096);
  if (act == MPX_ACT_SILU) gated_f32_kernel<MPX_ACT_SILU, BWD><<<blocks, 256, 0, s>>>(P, D, H, M, N);
  else gated_f32_kernel<MPX_ACT_GELU_TANH, BWD><<<blocks, 256, 0, s>>>(P, D, H, M, N);
  return hipGetLastError();
}

static GemmF32Args gated_f32_args(const void* A, const void* B, float* C, int64_t M, int64_t N, int64_t K,
                                  int64_t ldb, int64_t ldc) {
  GemmF32Args g{};
  g.nb1 = 1;
  g.splits = 1;
  g.k_split = INT64_MAX / 4;
  g.A = (const float*)A;
  g.B = (const float*)B;
  g.C = C;
  g.M = M; g.N = N; g.K = K;
  g.lda = K; g.ldb = ldb; g.ldc = ldc;
  return g;
}

static GemmArgs gated_args(const void* A, const void* B, void* C, int64_t M, int64_t N, int64_t K, int64_t ldb,
                           int64_t ldc, int32_t act) {
  GemmArgs g{};
  g.nb1 = 1;
  g.splits = 1;
  g.k_split = INT64_MAX / 4;
  g.A = (const uint16_t*)A;
  g.B = (const uint16_t*)B;
  g.C = (uint16_t*)C;
  g.M = M; g.N = N; g.K = K;
  g.lda = K; g.ldb = ldb; g.ldc = ldc;
  g.act = act;
  return g;
}

static bool misaligned(const void* p, mpx_dtype dt) {
  return reinterpret_cast<uintptr_t>(p) % (dt == MPX_F32 ? 4 : 2) != 0;
}

}  // namespace mpx

using namespace mpx;

// sizes past these would not fit an element count's 63 bits (tiles_fit: a launch)
static constexpr int64_t kMostRows = (int64_t)1 << 31, kMostCols = (int64_t)1 << 24;

extern "C" int mpx_gated_fwd(const void* X, const void* W, const void* b, void* H, void* Pre, int64_t M,
                             int64_t N, int64_t K, mpx_dtype dt, int32_t act, void* stream) {
  clear_error();
  MPX_REQUIRE(X && W && H, "NULL operand");
  MPX_REQUIRE(M >= 1 && N >= 1 && K >= 1, "M, N, K must be >= 1");
  MPX_REQUIRE(M < kMostRows && N <= kMostCols && K <= kMostCols, "too large");
  MPX_REQUIRE(is_half(dt) || dt == MPX_F32, "dt must be MPX_F16, MPX_BF16 or MPX_F32");
  MPX_REQUIRE(act == MPX_ACT_GELU_TANH || act == MPX_ACT_SILU, "unknown activation");
  MPX_REQUIRE(dt != MPX_F32 || Pre, "Pre is required with MPX_F32");
  MPX_REQUIRE(!misaligned(X, dt) && !misaligned(W, dt) && !misaligned(b, dt) && !misaligned(H, dt) &&
                  !misaligned(Pre, dt),
              "pointers must be aligned to their element");
  hipStream_t s = (hipStream_t)stream;
  if (dt == MPX_F32) {
    GemmF32Args g = gated_f32_args(X, W, (float*)Pre, M, 2 * N, K, K, 2 * N);
    g.bias = (const float*)b;
    MPX_HIP(launch_gemm_f32(g, true, true, 1, s));
    MPX_HIP(launch_f32<false>(act, (const float*)Pre, nullptr, (float*)H, M, N, s));
    return MPX_OK;
  }
  GemmArgs g = gated_args(X, W, H, M, N, K, K, N, act);
  g.bias = (const uint16_t*)b;
  g.pre = (uint16_t*)Pre;
  if (M <= 32) {
    MPX_HIP(dt == MPX_F16 ? launch_few<MPX_F16>(g, s) : launch_few<MPX_BF16>(g, s));
    return MPX_OK;
  }
  const RowTile t = gated_tile(g, true);
  MPX_REQUIRE(tiles_fit(t, M, 2 * N), "too large");
  MPX_HIP(dt == MPX_F16 ? run_gated_fwd_f16(g, N * K, t, s) : run_gated_fwd_bf16(g, N * K, t, s));
  return MPX_OK;
}

extern "C" size_t mpx_linear_bwd_gated_workspace(int64_t M, int64_t N, int64_t K) {
  return mpx_linear_bwd_workspace(M, N, K);
}

extern "C" int mpx_linear_bwd_gated(const void* X, const void* W, const void* dY, const void* Pre, int32_t act,
                                    void* dPre, void* dW, void* db, int64_t M, int64_t N, int64_t K,
                                    mpx_dtype dt, void* workspace, size_t ws_bytes, int32_t* d_nonfinite,
                                    void* stream) {
  clear_error();
  MPX_REQUIRE(dY, "NULL dY");
  MPX_REQUIRE(dPre || dW || db, "nothing to compute: dPre, dW and db are all NULL");
  MPX_REQUIRE(!dPre || (W && Pre), "W and Pre are required for dPre");
  MPX_REQUIRE(!dW || X, "X is required for dW");
  MPX_REQUIRE(M >= 1 && N >= 1 && K >= 1, "M, N, K must be >= 1");
  MPX_REQUIRE(M < kMostRows && N <= kMostCols && K <= kMostCols, "too large");
  MPX_REQUIRE(is_half(dt) || dt == MPX_F32, "dt must be MPX_F16, MPX_BF16 or MPX_F32");
  MPX_REQUIRE(act == MPX_ACT_GELU_TANH || act == MPX_ACT_SILU, "unknown activation");
  MPX_REQUIRE(dt != MPX_F32 || !d_nonfinite, "d_nonfinite is counted for half gradients only");
  MPX_REQUIRE(!misaligned(X, dt) && !misaligned(W, dt) && !misaligned(dY, dt) && !misaligned(Pre, dt) &&
                  !misaligned(dPre, dt) && !misaligned(dW, dt) && !misaligned(db, dt),
              "pointers must be aligned to their element");
  if (dW || db) {
    const size_t need = mpx_linear_bwd_gated_workspace(M, N, K);
    if (ws_bytes < need || !workspace) {
      set_error("mpx_linear_bwd_gated: workspace of " + std::to_string(need) + " bytes required");
      return MPX_ERR_WORKSPACE;
    }
  }
  hipStream_t s = (hipStream_t)stream;
  if (dPre) {
    if (dt == MPX_F32) {
      MPX_HIP(launch_gemm_f32(gated_f32_args(dY, W, (float*)dPre, M, K, N, K, 2 * K), true, false, 1, s));
      MPX_HIP(launch_f32<true>(act, (const float*)Pre, (float*)dPre, nullptr, M, K, s));
    } else {
      GemmArgs g = gated_args(dY, W, dPre, M, K, N, K, 2 * K, act);
      g.dact = (const uint16_t*)Pre;
      const RowTile t = gated_tile(g, false);
      MPX_REQUIRE(tiles_fit(t, M, K), "too large");
      MPX_HIP(dt == MPX_F16 ? run_gated_bwd_f16(g, t, s) : run_gated_bwd_bf16(g, t, s));
    }
  }
  if (dW || db)
    return mpx_linear_bwd(X, nullptr, dY, nullptr, MPX_ACT_NONE, nullptr, dW, db, M, N, K, dt, workspace,
                          ws_bytes, d_nonfinite, stream);
  return MPX_OK;
}
