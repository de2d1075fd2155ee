// Cross entropy of a linear layer's outputs without the logits (mpx_linear_ce_fwd,
// mpx_linear_ce_bwd): argument checks, the plan of pieces and splits, and the kernels
// around the products of linear_ce.h.
#include "linear_ce.h"

namespace mpx {

// (m, S) of two sets of logits together; m = -inf: all masked, S = 0.
__device__ __forceinline__ float2 ce_join(float2 a, float2 b) {
  const float m = fmaxf(a.x, b.x), at = m == -__builtin_inff() ? 0.0f : m;
  return make_float2(m, a.y * __builtin_amdgcn_exp2f((a.x - at) * kLog2e) +
                            b.y * __builtin_amdgcn_exp2f((b.x - at) * kLog2e));
}

// Joins the tile columns' (m, S) of R rows, 1024 / R threads to a row; a fixed order.
template <int R>
__global__ __launch_bounds__(1024) void ce_join_kernel(const float2* part, const float* zt, const int32_t* targets,
                                                       int64_t M, int32_t V, int parts, float* loss, float2* stats) {
  constexpr int G = 1024 / R;
  __shared__ float2 lds[G][R];
  const int r = threadIdx.x % R, g = threadIdx.x / R;
  const int64_t row = (int64_t)blockIdx.x * R + r, rc = min(row, M - 1);
  float2 a = make_float2(-__builtin_inff(), 0.0f);
  constexpr int U = 4;
  for (int c = g; c < parts; c += U * G) {
    float2 b[U];
#pragma unroll
    for (int u = 0; u < U; ++u) b[u] = part[(int64_t)min(c + u * G, parts - 1) * M + rc];
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (c + u * G < parts) a = ce_join(a, b[u]);
  }
  lds[g][r] = a;
  for (int h = G / 2; h >= 1; h /= 2) {
    __syncthreads();
    if (g < h) lds[g][r] = a = ce_join(a, lds[g + h][r]);
  }
  if (g != 0 || row >= M) return;
  const float ln = a.x == -__builtin_inff() ? 0.0f : logf(a.y);
  if (stats) stats[row] = make_float2(a.x, ln);
  if (loss) {
    const int32_t t = targets[row];
    float l = 0.0f;
    if (t >= V) {
      l = __builtin_nanf("");
    } else if (t >= 0) {
      const float z = zt[row];
      l = ln != ln ? ln : z == -__builtin_inff() ? __builtin_inff() : (a.x - z) + ln;
    }
    loss[row] = l;
  }
}

// Sum of v over a workgroup of 1024, in a fixed order.
template <typename T>
__device__ __forceinline__ T ce_sum1024(T v, T* lds) {
  lds[threadIdx.x] = v;
  for (int h = 512; h >= 1; h /= 2) {
    __syncthreads();
    if (threadIdx.x < h) lds[threadIdx.x] += lds[threadIdx.x + h];
  }
  __syncthreads();
  return lds[0];
}

// The mean over the rows that have a target (0 if none has).
__global__ __launch_bounds__(1024) void ce_mean_kernel(const float* loss, const int32_t* targets, int64_t M,
                                                       float* mean) {
  __shared__ float sums[1024];
  __shared__ int counts[1024];
  float s = 0.0f;
  int n = 0;
  for (int64_t i = threadIdx.x; i < M; i += 1024) {
    s += loss[i];
    n += targets[i] >= 0 ? 1 : 0;
  }
  s = ce_sum1024(s, sums);
  n = ce_sum1024(n, counts);
  if (threadIdx.x == 0) *mean = n ? s / (float)n : 0.0f;
}

// The backward's scalars: c (see linear_ce.h) from the largest |scale g|, and
// without g_loss the number of rows with a target.  C16: float16.
template <bool C16>
__global__ __launch_bounds__(1024) void ce_scalars_kernel(const float* g_loss, const int32_t* targets, int64_t M,
                                                          const mpx_scale_state* state, float* scalars) {
  __shared__ float most[1024];
  __shared__ int counts[1024];
  const float scale = state ? state->scale : 1.0f;
  float a = 0.0f, unit = scale;
  if (!g_loss) {
    int n = 0;
    for (int64_t i = threadIdx.x; i < M; i += 1024) n += targets[i] >= 0 ? 1 : 0;
    n = ce_sum1024(n, counts);
    unit = n ? scale / (float)n : 0.0f;
    a = fabsf(unit);
  } else if (C16) {
    for (int64_t i = threadIdx.x; i < M; i += 1024) a = fmaxf(a, targets[i] < 0 ? 0.0f : fabsf(g_loss[i] * scale));
    most[threadIdx.x] = a;
    for (int h = 512; h >= 1; h /= 2) {
      __syncthreads();
      if (threadIdx.x < h) most[threadIdx.x] = fmaxf(most[threadIdx.x], most[threadIdx.x + h]);
    }
    __syncthreads();
    a = most[0];
  }
  if (threadIdx.x != 0) return;
  int e = 0;  // c = 2^e
  if (C16 && a > 0.0f && a < __builtin_inff()) {
    e = 140 - (int)(__builtin_bit_cast(uint32_t, a) >> 23);  // a c in [2^13, 2^14)
    const int u = (int)(__builtin_bit_cast(uint32_t, fabsf(unit)) >> 23);
    e = min(min(100, 250 - u), max(-100, e));  // c scale stays finite
  }
  scalars[0] = __builtin_bit_cast(float, (uint32_t)(127 - e) << 23);
  scalars[1] = unit * __builtin_bit_cast(float, (uint32_t)(127 + e) << 23);
}

// out[i] = half(alpha sum over splits of part[s][i]); workgroups past those: db[r] = half(alpha
// sum over p of dbp[r][p]), one wave a row, lanes p = l, l + 64, ..., then wave_sum.
template <int DT>
__global__ __launch_bounds__(256) void ce_reduce_kernel(const float* part, int splits, int64_t n, uint16_t* out,
                                                        const float* dbp, int dbparts, int64_t nrows, uint16_t* db,
                                                        const float* alpha, int32_t* nonfinite) {
  const int64_t blocks = (n + 1023) / 1024;
  const float scale = *alpha;
  int bad = 0;
  if (blockIdx.x < blocks) {
    const int64_t i = ((int64_t)blockIdx.x * 256 + threadIdx.x) * 4;
    if (i >= n) return;
    if (n % 4 == 0) {
      f32x4 s = *reinterpret_cast<const f32x4*>(part + i);
      for (int k = 1; k < splits; ++k) {
        const f32x4 t = *reinterpret_cast<const f32x4*>(part + (int64_t)k * n + i);
#pragma unroll
        for (int e = 0; e < 4; ++e) s[e] += t[e];
      }
      uint16_t h[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        h[e] = f2h<DT>(s[e] * scale);
        bad += h_nonfinite<DT>(h[e]) ? 1 : 0;
      }
      __builtin_memcpy(out + i, h, 8);
    } else {
      for (int64_t j = i; j < min(i + 4, n); ++j) {
        float s = part[j];
        for (int k = 1; k < splits; ++k) s += part[(int64_t)k * n + j];
        const uint16_t h = f2h<DT>(s * scale);
        out[j] = h;
        bad += h_nonfinite<DT>(h) ? 1 : 0;
      }
    }
  } else {
    const int64_t row = ((int64_t)blockIdx.x - blocks) * 4 + (threadIdx.x >> 6);
    if (row >= nrows) return;  // uniform over the wave
    const int lane = threadIdx.x & 63;
    float s = 0.0f;
    for (int k = lane; k < dbparts; k += 64) s += dbp[row * dbparts + k];
    s = wave_sum(s);
    if (lane == 0) {
      const uint16_t h = f2h<DT>(s * scale);
      db[row] = h;
      bad = h_nonfinite<DT>(h) ? 1 : 0;
    }
  }
  if (nonfinite) add_nonfinite(nonfinite, bad);
}

// db of a piece where dW is not asked for: four groups of rows a workgroup, 64 columns.
template <int DT>
__global__ __launch_bounds__(256) void ce_colsum_kernel(const uint16_t* dz, int64_t ld, int64_t M, int64_t cols,
                                                        uint16_t* db, const float* alpha, int32_t* nonfinite) {
  __shared__ float lds[4][64];
  const int lane = threadIdx.x & 63, g = threadIdx.x >> 6;
  const int64_t c = (int64_t)blockIdx.x * 64 + lane;  // < ld, a multiple of 64
  float s = 0.0f;
  for (int64_t m = g; m < M; m += 4) s += h2f<DT>(dz[m * ld + c]);
  lds[g][lane] = s;
  __syncthreads();
  if (g != 0 || c >= cols) return;
  const uint16_t h = f2h<DT>((lds[0][lane] + lds[1][lane] + lds[2][lane] + lds[3][lane]) * *alpha);
  db[c] = h;
  if (nonfinite) add_nonfinite(nonfinite, h_nonfinite<DT>(h) ? 1 : 0);
}

// ------------------------------------------------------------------ plans --

// Tile of a product of two k-major operands (forward and dz).
static CeTile ce_tile(int64_t M, int64_t N, bool dma, bool any, bool forward) {
  if (any) return CE_STAGED_ANY;
  if (!dma) return cdiv(M, 64) * cdiv(N, 64) <= 512 ? CE_STAGED_64 : CE_STAGED_128;
  if (forward && M <= 32) return CE_32x128;
  if (cdiv(M, 256) * cdiv(N, 256) >= 512) return CE_256x256;
  return cdiv(M, 128) * cdiv(N, 128) >= 384 ? CE_128x128 : CE_64x128;
}

static size_t align256(size_t n) { return (n + 255) / 256 * 256; }

// Forward workspace: (m, S) of every tile column, whatever the operands' alignment,
// and the targets' logits.
static int64_t ce_parts(int64_t M, int64_t V, int64_t K) {
  return std::max(cdiv(V, ce_tile_cols(ce_tile(M, V, true, false, true))),
                  cdiv(V, ce_tile_cols(ce_tile(M, V, false, K < 8, true))));
}

// The backward's pieces of the vocabulary and splits of its two reductions.
struct CePlan {
  int64_t cols, pieces;  // columns of a piece (a multiple of 256)
  int dx_splits, dw_splits;
  int64_t dx_k, dw_k;  // reduction length of a split
  bool dx_parts;
  size_t dz, dxp, dwp, dbp, total;  // workspace offsets, scalars first
};

// Splits of a reduction of length len over tiles of 128 x 128: two workgroups per CU,
// 512 values a split at least.
static int ce_splits(int64_t M, int64_t N, int64_t len, int64_t& k_split) {
  const int64_t tiles = cdiv(M, 128) * cdiv(N, 128);
  const int64_t s = std::max<int64_t>(1, std::min<int64_t>({512 / tiles, 16, len / 512}));
  k_split = cdiv(cdiv(len, s), 64) * 64;
  return (int)cdiv(len, k_split);
}

static CePlan ce_plan(int64_t M, int64_t V, int64_t K) {
  CePlan p{};
  const int64_t rows = cdiv(M, 64) * 64;
  const int64_t most = std::max<int64_t>(256, ((int64_t)96 << 20) / (2 * rows) / 256 * 256);
  p.pieces = cdiv(V, most);
  p.cols = cdiv(cdiv(V, p.pieces), 256) * 256;
  p.pieces = cdiv(V, p.cols);
  const int64_t cols = std::min(p.cols, V);
  p.dx_splits = ce_splits(M, K, cols, p.dx_k);
  p.dw_splits = ce_splits(cols, K, M, p.dw_k);
  p.dx_parts = p.pieces > 1 || p.dx_splits > 1;
  p.dz = 256;
  p.dxp = p.dz + align256((size_t)rows * cdiv(cols, 64) * 64 * 2);
  p.dwp = p.dxp + (p.dx_parts ? align256((size_t)p.dx_splits * M * K * 4) : 0);
  p.dbp = p.dwp + (p.dw_splits > 1 ? align256((size_t)p.dw_splits * cols * K * 4) : 0);
  p.total = p.dbp + align256((size_t)p.dw_splits * cdiv(K, 64) * cols * 4);
  return p;
}

static GemmArgs ce_args(const void* A, const void* B, int64_t M, int64_t N, int64_t K, int64_t lda, int64_t ldb) {
  GemmArgs g{};
  g.nb1 = 1;
  g.splits = 1;
  g.k_split = INT64_MAX / 4;
  g.A = (const uint16_t*)A;
  g.B = (const uint16_t*)B;
  g.M = M; g.N = N; g.K = K;
  g.lda = lda; g.ldb = ldb;
  return g;
}

static bool ce_misaligned(const void* p, int n) { return reinterpret_cast<uintptr_t>(p) % n != 0; }

static int ce_check(const char* fn, const void* X, const void* W, const void* b, const int32_t* targets, int64_t M,
                    int64_t V, int64_t K, mpx_dtype dt) {
  const char* why = nullptr;
  if (!X || !W) why = "NULL operand";
  else if (M < 1 || V < 1 || K < 1) why = "M, V, K must be >= 1";
  else if (M > (1 << 20) || V > (1 << 24) || K > (1 << 16)) why = "too large";
  else if (!is_half(dt)) why = "dt must be MPX_F16 or MPX_BF16";
  else if (ce_misaligned(X, 2) || ce_misaligned(W, 2) || ce_misaligned(b, 2) || ce_misaligned(targets, 4))
    why = "pointers must be aligned to their element";
  if (!why) return MPX_OK;
  set_error(std::string(fn) + ": " + why);
  return MPX_ERR_INVALID;
}

template <class F>
static hipError_t by_type(mpx_dtype dt, F f) {
  return dt == MPX_F16 ? f(std::integral_constant<int, MPX_F16>{}) : f(std::integral_constant<int, MPX_BF16>{});
}

}  // namespace mpx

using namespace mpx;

extern "C" size_t mpx_linear_ce_fwd_workspace(int64_t M, int64_t V, int64_t K) {
  if (M < 1 || V < 1 || K < 1) return 0;
  return align256((size_t)ce_parts(M, V, K) * M * 8) + align256((size_t)M * 4);
}

extern "C" int mpx_linear_ce_fwd(const void* X, const void* W, const void* b, const int32_t* targets, int64_t M,
                                 int64_t V, int64_t K, float* loss, float* stats, float* d_mean, mpx_dtype dt,
                                 void* workspace, size_t ws_bytes, void* stream) {
  clear_error();
  if (const int rc = ce_check("mpx_linear_ce_fwd", X, W, b, targets, M, V, K, dt)) return rc;
  MPX_REQUIRE(loss || stats, "nothing to compute: loss and stats are both NULL");
  MPX_REQUIRE(!loss || targets, "targets are required for the loss");
  MPX_REQUIRE(!d_mean || loss, "loss is required for its mean");
  MPX_REQUIRE(!ce_misaligned(loss, 4) && !ce_misaligned(stats, 8) && !ce_misaligned(d_mean, 4),
              "pointers must be aligned to their element (stats to 8 bytes)");
  const size_t need = mpx_linear_ce_fwd_workspace(M, V, K);
  if (!workspace || ws_bytes < need || ce_misaligned(workspace, 16)) {
    set_error("mpx_linear_ce_fwd: workspace of " + std::to_string(need) + " bytes, 16-byte aligned, required");
    return MPX_ERR_WORKSPACE;
  }
  hipStream_t s = (hipStream_t)stream;
  CeFwdArgs g;
  static_cast<GemmArgs&>(g) = ce_args(X, W, M, V, K, K, K);
  g.bias = (const uint16_t*)b;
  g.part = (float2*)workspace;
  g.zt = (float*)((char*)workspace + align256((size_t)ce_parts(M, V, K) * M * 8));
  g.targets = loss ? targets : nullptr;
  const CeTile t = ce_tile(M, V, dma_ok(g, operands_aligned(g), true, true), false, true);
  const bool any = (t == CE_STAGED_64 || t == CE_STAGED_128) && staged_any(g, true, true);
  const CeTile tile = any ? CE_STAGED_ANY : t;
  MPX_HIP(dt == MPX_F16 ? run_ce_fwd_f16(g, tile, s) : run_ce_fwd_bf16(g, tile, s));
  const int parts = (int)cdiv(V, ce_tile_cols(tile));
  if (M >= 2048)
    ce_join_kernel<32><<<(unsigned)cdiv(M, 32), 1024, 0, s>>>(g.part, g.zt, targets, M, (int32_t)V, parts, loss,
                                                              (float2*)stats);
  else
    ce_join_kernel<4><<<(unsigned)cdiv(M, 4), 1024, 0, s>>>(g.part, g.zt, targets, M, (int32_t)V, parts, loss,
                                                            (float2*)stats);
  MPX_LAUNCHED();
  if (d_mean) {
    ce_mean_kernel<<<1, 1024, 0, s>>>(loss, targets, M, d_mean);
    MPX_LAUNCHED();
  }
  return MPX_OK;
}

extern "C" size_t mpx_linear_ce_bwd_workspace(int64_t M, int64_t V, int64_t K) {
  if (M < 1 || V < 1 || K < 1) return 0;
  return ce_plan(M, V, K).total;
}

extern "C" int mpx_linear_ce_bwd(const void* X, const void* W, const void* b, const int32_t* targets, int64_t M,
                                 int64_t V, int64_t K, const float* stats, const float* g_loss,
                                 const mpx_scale_state* d_state, void* dX, void* dW, void* db, mpx_dtype dt,
                                 void* workspace, size_t ws_bytes, int32_t* d_nonfinite, void* stream) {
  clear_error();
  if (const int rc = ce_check("mpx_linear_ce_bwd", X, W, b, targets, M, V, K, dt)) return rc;
  MPX_REQUIRE(targets && stats, "NULL targets or stats");
  MPX_REQUIRE(dX || dW || db, "nothing to compute: dX, dW and db are all NULL");
  MPX_REQUIRE(!ce_misaligned(stats, 8) && !ce_misaligned(g_loss, 4) && !ce_misaligned(d_state, 4) &&
                  !ce_misaligned(dX, 2) && !ce_misaligned(dW, 2) && !ce_misaligned(db, 2),
              "pointers must be aligned to their element (stats to 8 bytes)");
  const CePlan p = ce_plan(M, V, K);
  if (!workspace || ws_bytes < p.total || ce_misaligned(workspace, 16)) {
    set_error("mpx_linear_ce_bwd: workspace of " + std::to_string(p.total) + " bytes, 16-byte aligned, required");
    return MPX_ERR_WORKSPACE;
  }
  hipStream_t s = (hipStream_t)stream;
  char* ws = (char*)workspace;
  float* scalars = (float*)ws;
  uint16_t* dz = (uint16_t*)(ws + p.dz);
  if (dt == MPX_F16) ce_scalars_kernel<true><<<1, 1024, 0, s>>>(g_loss, targets, M, d_state, scalars);
  else ce_scalars_kernel<false><<<1, 1024, 0, s>>>(g_loss, targets, M, d_state, scalars);
  MPX_LAUNCHED();
  // the reductions' own operands: dz is aligned, X and W as they come
  const auto out_tile = [&](const GemmArgs& g, bool ak) {
    if ((reinterpret_cast<uintptr_t>(g.B) & 15u) == 0 && g.ldb % 8 == 0) return CE_128x128;
    return staged_any(g, ak, false) ? CE_STAGED_ANY
           : cdiv(g.M, 64) * cdiv(g.N, 64) * g.splits <= 512 ? CE_STAGED_64 : CE_STAGED_128;
  };
  const auto run_out = [&](const CeOutArgs& g, bool ak, CeTile t) {
    return dt == MPX_F16 ? run_ce_out_f16(g, ak, t, s) : run_ce_out_bf16(g, ak, t, s);
  };
  const auto reduce = [&](const float* part, int splits, int64_t n, void* out, const float* dbp, int dbparts,
                          int64_t nrows, void* dbo, int32_t* count) {
    return by_type(dt, [&](auto type) {
      ce_reduce_kernel<type><<<(unsigned)(cdiv(n, 1024) + cdiv(nrows, 4)), 256, 0, s>>>(
          part, splits, n, (uint16_t*)out, dbp, dbparts, nrows, (uint16_t*)dbo, scalars, count);
      return hipGetLastError();
    });
  };
  for (int64_t v0 = 0; v0 < V; v0 += p.cols) {
    const int64_t cols = std::min(p.cols, V - v0), ldz = cdiv(cols, 64) * 64;
    const uint16_t* Wp = (const uint16_t*)W + v0 * K;
    CeGradArgs z;
    static_cast<GemmArgs&>(z) = ce_args(X, Wp, M, cols, K, K, K);
    z.bias = b ? (const uint16_t*)b + v0 : nullptr;
    z.C = dz;
    z.ldc = ldz;
    z.stats = (const float2*)stats;
    z.scalars = scalars;
    z.g_loss = g_loss;
    z.targets = targets;
    z.v0 = (int32_t)v0;
    z.vocabulary = (int32_t)V;
    const bool dma = dma_ok(z, operands_aligned(z), true, true);
    const CeTile t = ce_tile(M, cols, dma, !dma && staged_any(z, true, true), false);
    MPX_HIP(dt == MPX_F16 ? run_ce_grad_f16(z, t, s) : run_ce_grad_bf16(z, t, s));
    if (dX) {
      CeOutArgs g;
      static_cast<GemmArgs&>(g) = ce_args(dz, Wp, M, K, cols, ldz, K);
      g.C = (uint16_t*)dX;
      g.splits = (int)cdiv(cols, p.dx_k);  // the last piece may need fewer
      g.k_split = p.dx_k;
      g.part = p.dx_parts ? (float*)(ws + p.dxp) : nullptr;
      g.alpha = scalars;
      g.add = v0 > 0;
      MPX_HIP(run_out(g, true, out_tile(g, true)));
    }
    if (dW) {
      CeOutArgs g;
      static_cast<GemmArgs&>(g) = ce_args(dz, X, cols, K, M, ldz, K);
      g.C = (uint16_t*)dW + v0 * K;
      g.splits = p.dw_splits;
      g.k_split = p.dw_k;
      g.part = p.dw_splits > 1 ? (float*)(ws + p.dwp) : nullptr;
      g.alpha = scalars;
      g.add = 0;
      g.nonfinite = d_nonfinite;
      g.dbp = db ? (float*)(ws + p.dbp) : nullptr;
      const CeTile tw = out_tile(g, false);
      MPX_HIP(run_out(g, false, tw));
      const int dbparts = (int)(p.dw_splits * cdiv(K, ce_tile_cols(tw)));
      if (g.part || db)
        MPX_HIP(reduce(g.part, p.dw_splits, g.part ? cols * K : 0, g.C, g.dbp, dbparts, db ? cols : 0,
                       db ? (uint16_t*)db + v0 : nullptr, d_nonfinite));
    } else if (db) {
      MPX_HIP(by_type(dt, [&](auto type) {
        ce_colsum_kernel<type><<<(unsigned)(ldz / 64), 256, 0, s>>>(dz, ldz, M, cols, (uint16_t*)db + v0, scalars,
                                                                   d_nonfinite);
        return hipGetLastError();
      }));
    }
  }
  if (dX && p.dx_parts)
    MPX_HIP(reduce((const float*)(ws + p.dxp), p.dx_splits, M * K, dX, nullptr, 0, 0, nullptr, nullptr));
  return MPX_OK;
}
