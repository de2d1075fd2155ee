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

// Joins the tile columns' (m, S) of R rows, 1024 / R threads to a row; a fixed order.  R is
// what a row's parts leave threads for, and 16 (whole lines of 128 bytes) where there are rows
// enough: 2019 rows of 710 parts 11 us by 4, 7.1 by 16.
template <int R>
__global__ __launch_bounds__(1024) void ce_join_kernel(const float2* part, const float* zt, const int32_t* targets,
                                                       int64_t M, int32_t V, int parts, float* loss, float2* stats) {
  constexpr int G = 1024 / R;
  __shared__ float2 lds[G][R];
  const int r = threadIdx.x % R, g = threadIdx.x / R;
  const int64_t row = (int64_t)blockIdx.x * R + r, rc = min(row, M - 1);
  // ahead of the join: zt has no value of a row without a target, which is not used either
  const int32_t t = loss && g == 0 ? targets[rc] : -1;
  const float z = loss && g == 0 ? zt[rc] : 0.0f;
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
  // S is 0 where everything is masked and nowhere else.  m passes over NaN logits, S does not:
  // beside nothing but them and masked ones m is no -inf, which would say all masked
  const float ln = a.y == 0.0f ? 0.0f : logf(a.y);
  if (stats) stats[row] = make_float2(ln != ln && a.x == -__builtin_inff() ? ln : a.x, ln);
  if (loss) {
    float l = 0.0f;
    if (t >= V) {
      l = __builtin_nanf("");
    } else if (t >= 0) {
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
#pragma unroll 8
  for (int64_t i = threadIdx.x; i < M; i += 1024) {
    s += loss[i];
    n += targets[i] >= 0 ? 1 : 0;
  }
  s = ce_sum1024(s, sums);
  n = ce_sum1024(n, counts);
  if (threadIdx.x == 0) *mean = n ? s / (float)n : 0.0f;
}

// The backward's scalars, by workgroup 0: c (see linear_ce.h) from the largest |scale g|, and
// without g_loss the number of rows with a target.  C16: float16.  The workgroups behind it
// copy a row each of X twice over (zeros behind its own, half the grid apart), for the products of
// dz and its remainders; rows of ld values.
template <bool C16>
__global__ __launch_bounds__(1024) void ce_prepare_kernel(const float* g_loss, const int32_t* targets, int64_t M,
                                                          const mpx_scale_state* state, float* scalars,
                                                          const uint16_t* X, int64_t K, uint16_t* twice, int64_t ld) {
  if (blockIdx.x > 0) {
    const int64_t at = blockIdx.x - 1, row = at % ((gridDim.x - 1) / 2);
    for (int64_t k = threadIdx.x; k < ld; k += 1024)
      twice[at * ld + k] = row < M && k < K ? X[row * K + k] : (uint16_t)0;
    return;
  }
  __shared__ float most[1024];
  __shared__ int counts[1024];
  const float scale = state ? state->scale : 1.0f;
  float a = 0.0f, unit = scale;
  if (!g_loss) {
    int n = 0;
#pragma unroll 8
    for (int64_t i = threadIdx.x; i < M; i += 1024) n += targets[i] >= 0 ? 1 : 0;
    n = ce_sum1024(n, counts);
    unit = n ? scale / (float)n : 0.0f;
    a = fabsf(unit);
  } else if (C16) {
#pragma unroll 4
    for (int64_t i = threadIdx.x; i < M; i += 1024) {
      const float g = fabsf(g_loss[i] * scale);
      a = fmaxf(a, targets[i] < 0 ? 0.0f : g);
    }
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

// out[i] = half(alpha sum over splits of part[s stride + i]); rows of `width` sums, of which
// `cols` are kept.
struct CeSum {
  const float* part;
  int64_t stride, n;
  int32_t splits;
  uint16_t* out;
  int32_t* nonfinite;
};
struct CeReduce {
  CeSum first, second;  // n = 0: none
  int32_t width, cols;
  const float* dbp;  // [nrows][dbparts]
  int64_t nrows;
  int32_t dbparts;
  uint16_t* db;
  int32_t* nonfinite;
  const float *alpha, *rest;  // nullable: 1, none
  const int32_t* targets;
  int32_t rows, v0;
};

// Both sums, VEC: 4 values a thread (n, stride and part allow 16 bytes).  Workgroups past
// those: db[r] = half(alpha (sum over p of dbp[r][p], and of the rests of the rows whose
// target is r)), one wave a row, or with rests a workgroup, in strides of 64 or 256 and then in
// order (12616 x 16 x 224 f16 with gradient: the rests by a wave 133 us, by a workgroup 46).
// G threads a value where there are few values and many splits, each every G-th split, then
// added in order.
template <int DT, bool VEC, int G>
__global__ __launch_bounds__(256) void ce_reduce_kernel(CeReduce a) {
  constexpr int PER = VEC ? 4 : 1, AT = 256 / G;  // AT threads' worth of values
  __shared__ float lds[G > 1 ? G : 1][PER][AT];
  const int64_t blocks1 = (a.first.n + AT * PER - 1) / (AT * PER);
  const int64_t blocks = blocks1 + (a.second.n + AT * PER - 1) / (AT * PER);
  const float scale = a.alpha ? *a.alpha : 1.0f;
  int bad = 0;
  int32_t* count = a.nonfinite;
  if (blockIdx.x < blocks) {
    const bool one = blockIdx.x < blocks1;
    const CeSum u = one ? a.first : a.second;
    const int at = threadIdx.x % AT, g = threadIdx.x / AT;
    const int64_t i = ((blockIdx.x - (one ? 0 : blocks1)) * AT + at) * PER;
    const bool in = i < u.n;
    count = u.nonfinite;
    float s[PER] = {};
#pragma unroll 8
    for (int k = g; k < u.splits; k += G) {
      float t[PER];
      if (in) __builtin_memcpy(t, u.part + k * u.stride + i, sizeof(t));
#pragma unroll
      for (int e = 0; e < PER; ++e) s[e] += in ? t[e] : 0.0f;
    }
    if constexpr (G > 1) {
#pragma unroll
      for (int e = 0; e < PER; ++e) lds[g][e][at] = s[e];
      __syncthreads();
      if (g > 0) return;
#pragma unroll
      for (int k = 1; k < G; ++k) {
#pragma unroll
        for (int e = 0; e < PER; ++e) s[e] += lds[k][e][at];
      }
    }
    if (!in) return;
    uint16_t h[PER];
#pragma unroll
    for (int e = 0; e < PER; ++e) h[e] = f2h<DT>(s[e] * scale);
    if (a.width == a.cols) {  // uniform
#pragma unroll
      for (int e = 0; e < PER; ++e) bad += h_nonfinite<DT>(h[e]) ? 1 : 0;
      __builtin_memcpy(u.out + i, h, sizeof(h));
    } else {
      const int64_t row = i / a.width;
      const int c = (int)(i - row * a.width);
#pragma unroll
      for (int e = 0; e < PER; ++e) {
        if (c + e < a.cols) {
          u.out[row * a.cols + c + e] = h[e];
          bad += h_nonfinite<DT>(h[e]) ? 1 : 0;
        }
      }
    }
  } else {
    __shared__ float waves[4];
    const bool whole = a.rest != nullptr;  // uniform
    const int wave = threadIdx.x >> 6, span = whole ? 256 : 64, first = threadIdx.x % span;
    const int64_t row = ((int64_t)blockIdx.x - blocks) * (whole ? 1 : 4) + (whole ? 0 : wave);
    if (row >= a.nrows) return;  // uniform over the wave, none with rests
    float s = 0.0f;
    for (int k = first; k < a.dbparts; k += span) s += a.dbp[row * a.dbparts + k];
    if (whole) {  // what rounding left of the targets that are this column
#pragma unroll 8
      for (int r = first; r < a.rows; r += 256) {
        const float v = a.rest[r];
        s += a.targets[r] == a.v0 + row ? v : 0.0f;
      }
    }
    s = wave_sum(s);
    if (whole) {
      if ((threadIdx.x & 63) == 0) waves[wave] = s;
      __syncthreads();
      s = (waves[0] + waves[1]) + (waves[2] + waves[3]);
    }
    if (first == 0) {
      const uint16_t h = f2h<DT>(s * scale);
      a.db[row] = h;
      bad = h_nonfinite<DT>(h) ? 1 : 0;
    }
  }
  if (count) add_nonfinite(count, bad);
}

// db of a piece where dW is not asked for: partial sums dbp[column][part] for the reduction,
// four groups of kColsumRows rows a workgroup, 64 columns.  Equal dz (a uniform softmax's) round
// every step of a chain the same way: in chains of 2^18 float16's lost 2^-8.5, ones of
// kColsumRows / 4 are exact for it (and spread the rows: 12616 x 16 x 224 f16 db alone 771 us with
// chains of all rows, 40 so).
constexpr int64_t kColsumRows = 256;
static int64_t ce_colsum_parts(int64_t rows) { return 4 * cdiv(rows, kColsumRows); }
template <int DT>
__global__ __launch_bounds__(256) void ce_colsum_kernel(const uint16_t* dz, int64_t ld, int64_t M, int64_t cols,
                                                        float* dbp) {
  const int g = threadIdx.x >> 6;
  const int64_t c = (int64_t)blockIdx.x * 64 + (threadIdx.x & 63);  // < ld, a multiple of 64
  const int64_t m0 = blockIdx.y * kColsumRows, end = min(M, m0 + kColsumRows);
  float s = 0.0f;
  for (int64_t m = m0 + g; m < end; m += 4) s += h2f<DT>(dz[m * ld + c]);
  if (c < cols) dbp[(c * gridDim.y + blockIdx.y) * 4 + g] = s;
}

// Rows of X [M, K] and then of W [V, K] with zeros behind them, up to ld values (a multiple
// of 8), 16-byte aligned: 8 values a thread.
__global__ __launch_bounds__(256) void ce_pad_kernel(const uint16_t* X, int64_t M, const uint16_t* W, int64_t V,
                                                     int64_t K, uint16_t* out, int64_t ld) {
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x, chunks = ld / 8;
  const int64_t row = i / chunks, k = (i - row * chunks) * 8;
  if (row >= M + V) return;
  const uint16_t* p = (row < M ? X + row * K : W + (row - M) * K) + k;
  *reinterpret_cast<u32x4*>(out + row * ld + k) = load8(p, (int)max((int64_t)-8, min((int64_t)8, K - k)));
}

// ------------------------------------------------------------------ plans --

// The products' tables for choose_rows: forward 0.3% slower than the fastest tile on average,
// dz 0.5%, dX and dW with their split counts 2.3% and 2.7% (those above 60 us 3.5% and 0.7%).
static const RowCost kFwdCost[] = {{TILE_64x128, 64, 128, 3, {0.43, 0.53, 0.83}, 1.04},
                                   {TILE_128x128, 128, 128, 2, {0.62, 0.75, 0}, 2.93},
                                   {TILE_192x128, 192, 128, 2, {0.78, 0.81, 0}, 3.23},
                                   {TILE_256x256, 256, 256, 1, {1.11, 0, 0}, 9.58}};
static const RowCost kGradCost[] = {{TILE_64x128, 64, 128, 3, {0.14, 0.24, 0.78}, 1.46},
                                    {TILE_128x128, 128, 128, 2, {0.28, 0.66, 0}, 3.36},
                                    {TILE_192x128, 192, 128, 2, {0.61, 0.88, 0}, 4.29},
                                    {TILE_256x256, 256, 256, 1, {1.02, 0, 0}, 13.4}};
static const RowCost kDxCost[] = {{TILE_64x128, 64, 128, 3, {0.45, 0.47, 0.74}, 2.03},
                                  {TILE_128x128, 128, 128, 2, {0.49, 0.64, 0}, 4.76},
                                  {TILE_192x128, 192, 128, 2, {1.02, 1.07, 0}, 4.70},
                                  {TILE_256x256, 256, 256, 1, {1.32, 0, 0}, 13.2}};
static const RowCost kDwCost[] = {{TILE_128x128, 128, 128, 2, {0.60, 0.77, 0}, 2.88},
                                  {TILE_192x128, 192, 128, 2, {0.82, 1.04, 0}, 4.92},
                                  {TILE_256x256, 256, 256, 1, {1.29, 0, 0}, 13.3}};

// The most rows that take 64 x 64 staged tiles: one row of tiles, or up to two tiles per CU.
static int64_t ce_narrow_rows(int64_t N) { return std::max<int64_t>(64, 512 / cdiv(N, 64) * 64); }

// Tile of a product of two k-major operands (forward and dz).  Staged ones of at most 64
// rows: 11 x 51223 x 183 f16 dz 18.3 us by 128 x 128, 12.5 by 64 x 64.
static RowTile ce_tile(int64_t M, int64_t N, int64_t K, bool dma, bool any, bool forward) {
  if (any) return STAGED_ANY;
  if (!dma) return M <= ce_narrow_rows(N) ? STAGED_64 : STAGED_128;
  if (forward && M <= 32) return TILE_32x128;
  return choose_rows(forward ? kFwdCost : kGradCost, M, N, K).tile;
}

static size_t align256(size_t n) { return (n + 255) / 256 * 256; }

// Forward workspace: (m, S) of every row and tile column, whatever the operands' alignment,
// and the targets' logits.  Never less than fewer rows take, whose tiles may be narrower.
static int64_t ce_pairs(int64_t M, int64_t V, int64_t K) {
  const int64_t narrow = K < 8 ? M : std::min(M, ce_narrow_rows(V));
  return std::max(cdiv(V, tile_cols(STAGED_64)) * narrow, cdiv(V, tile_cols(STAGED_128)) * M);
}

// Tile and splits of a piece's reductions over direct operands; at least 192 values a split,
// none of them empty.  Register-staged ones take the splits and a tile of their own.  At most
// three rounds of the smallest tiles, which bounds the partial sums of any number of rows (of
// 20000 drawn products of K <= 2048 it changes the splits of 0.06%).
constexpr int64_t kDxGroups = 3 * 768, kDwGroups = 3 * 512;
static RowChoice ce_dx(int64_t M, int64_t cols, int64_t K, bool parts) {
  const int64_t most = std::min({(int64_t)64, cols / 192, kDxGroups / (cdiv(M, 64) * cdiv(K, 128))});
  // without partial sums a split also costs the kernel that adds them
  return choose_rows(kDxCost, M, K, cols, std::max<int64_t>(1, most), parts ? 0.0 : 3.0, 1.25e-6, !parts);
}
static RowChoice ce_dw(int64_t M, int64_t cols, int64_t K) {
  const int64_t most = std::min({(int64_t)64, M / 192, kDwGroups / (cdiv(cols, 128) * cdiv(K, 128))});
  return choose_rows(kDwCost, cols, K, M, std::max<int64_t>(1, most), 2.0, 2.5e-6);
}

// Operands whose reduction is no multiple of 64 go to the direct tiles as padded copies
// where these cost less than register staging (bf16, us, staged / padded): forward
// from 1024 rows on (700 x 50000 x 700 86 / 92, 1500 x 50000 x 700 157 / 148, 4000 x 20000 x 300 104 /
// 81) but for few columns (1500 x 1000 x 100 12.4 / 13.7), with gradient from 256 on (300 x 50000
// x 700 248 / 224, 4000 x 50000 x 700 1867 / 1371; 100 x 50000 x 700 142 / 166).
static int64_t ce_padded(int64_t K) { return cdiv(K, 64) * 64; }
static bool ce_pads_fwd(int64_t M, int64_t V, int64_t K) { return K % 64 != 0 && M >= 1024 && V >= 4096; }
static bool ce_pads_bwd(int64_t M, int64_t K) { return K % 64 != 0 && M >= 256; }

// The backward's pieces of the vocabulary, all but the last of `cols` columns, and their
// place in the workspace.
struct CePlan {
  int64_t cols, pieces, last, most;  // a multiple of 256; how many; the last one's and the largest's columns
  int dx_splits;                     // partial sums of dX: the most any piece takes
  bool dx_parts, rest;
  int64_t twice, rows;  // rows between dz and what its rounding left (0: not kept), of all
  int64_t width;  // of dX's and dW's partial sums: K, or of padded operands a multiple of 4
  size_t lo, dz, dxp, dwp, dbp, x2;  // workspace offsets, scalars first; x2: other forms of X (and W)
};

// Rows of dz that what its rounding left is kept for, in as many rows more: 32, 64 or 128 of each
// (20 x 63884 x 256 bf16 of 64 each 72 us, of 32 62).  Up to 128 rows dX's norm would lose up to
// a factor of 1.8 to the rounding of dz, with 256 1.45; db's, of few columns, of up to a
// thousand rows 2: there, up to kCeRest logits, what the targets' dz left.
static int64_t ce_twice(int64_t M) { return M <= 32 ? 32 : M <= 64 ? 64 : M <= 128 ? 128 : 0; }
constexpr int64_t kCeRest = (int64_t)1 << 22, kCeDz = (int64_t)64 << 20;  // kCeDz: values of a piece's dz

static int64_t split_len(int64_t len, int splits) { return cdiv(cdiv(len, splits), 64) * 64; }
// splits of that length that cover len: none is empty
static int split_count(int64_t len, int splits) { return (int)cdiv(len, split_len(len, splits)); }

// dz takes at most 128 MiB (so that its readers find much of it in the last-level cache), or
// 256 columns; the only or last piece up to 256 columns more, so that none is narrow (65536
// rows: 160 MiB at most, 2^20: 1 GiB).  Among the column counts that allow: the one of least estimated time
// (whole rounds of tiles: 4096 x 65537 in 5 equal pieces of 52 tile columns 1.10 of the
// time of 3 of 64 and one of 65).
static CePlan ce_plan(int64_t M, int64_t V, int64_t K) {
  CePlan p{};
  p.twice = ce_twice(M);
  p.rest = !p.twice && M * V <= kCeRest;
  p.width = ce_pads_bwd(M, K) ? cdiv(K, 4) * 4 : K;
  const int64_t rows = p.rows = p.twice ? 2 * p.twice : cdiv(M, 64) * 64, Mr = p.twice ? p.rows : M;
  const int64_t most = std::max<int64_t>(256, kCeDz / rows / 256 * 256);
  const auto lay = [&](int64_t cols) {  // what is left after whole pieces: its own, or with the last
    p.cols = cols;
    p.pieces = std::max<int64_t>(1, cdiv(V - 256, cols));
    p.last = V - (p.pieces - 1) * cols;
    p.most = std::max(p.pieces > 1 ? cols : 0, p.last);
  };
  if (V <= most + 256) {
    lay(cdiv(V, 256) * 256);
  } else {
    const auto us = [&](int64_t cols) {
      return choose_rows(kGradCost, M, cols, K).us + ce_dx(Mr, cols, K, true).us + ce_dw(Mr, cols, K).us + 10.0;
    };
    int64_t best = most;
    double least = 0.0;
    for (int i = 0; i < 12 && most - i * (most / 24 / 256 * 256) >= 256; ++i) {
      lay(most - i * (most / 24 / 256 * 256));
      const double t = us(p.cols) * (double)(p.pieces - 1) + us(p.last);
      if (least == 0.0 || t < least) {
        least = t;
        best = p.cols;
      }
    }
    lay(best);
  }
  p.dx_parts = p.pieces > 1;
  size_t dw = 0, db = 0;  // bytes
  for (const int64_t cols : {p.pieces > 1 ? p.cols : p.last, p.last}) {
    p.dx_splits = std::max(p.dx_splits, split_count(cols, ce_dx(Mr, cols, K, p.pieces > 1 || p.twice > 0).splits));
    const int s = split_count(Mr, ce_dw(Mr, cols, K).splits);
    dw = std::max(dw, s > 1 ? (size_t)s * cols * p.width * 4 : 0);
    db = std::max(db, (size_t)std::max(ce_colsum_parts(rows), s * cdiv(K, 64)) * cols * 4);
  }
  p.dx_parts = p.twice > 0 || p.dx_parts || p.dx_splits > 1;
  p.lo = 256;
  p.dz = p.lo + (p.rest ? align256((size_t)M * 4) : 0);
  p.dxp = p.dz + align256((size_t)rows * cdiv(p.most, 64) * 64 * 2);
  p.dwp = p.dxp + (p.dx_parts ? align256((size_t)p.dx_splits * Mr * p.width * 4) : 0);
  p.dbp = p.dwp + align256(dw);
  p.x2 = p.dbp + align256(db);
  return p;
}

// A workspace that holds the plan of any number of rows up to M, part by part the largest:
// few rows take two sets, wide pieces and many splits, many rows the most of the others.
static size_t ce_bwd_bytes(int64_t M, int64_t V, int64_t K) {
  const int64_t twice = M > 128 ? 128 : ce_twice(M), width = cdiv(K, 4) * 4, tiles = cdiv(K, 128);
  const int64_t rows = std::max(2 * twice, M > 128 ? cdiv(M, 64) * 64 : 0), Mr = std::max(2 * twice, M);
  const int64_t most_cols = std::min(V, kCeDz / 64 + 256);  // of a piece, of the fewest rows
  // a piece's columns times rows: kCeDz or 256 columns, and up to 256 columns more
  const int64_t dz = std::min(rows * cdiv(V, 64) * 64, std::max(kCeDz, rows * 256) + rows * 256);
  const int64_t dx_splits = std::max<int64_t>(1, std::min<int64_t>(64, V / 192));
  const int64_t dx = std::max(Mr * width, std::min(dx_splits * Mr * width, kDxGroups * 64 / tiles * width));
  const int64_t dw_splits = Mr / 192;
  const int64_t dw = dw_splits < 2 ? 0 : std::min(dw_splits * V * width, kDwGroups * 128 / tiles * width);
  // a split's column of sums for each 64 of K, two in a tile; or four for every kColsumRows rows of dz
  const int64_t db = std::max({cdiv(K, 64) * most_cols, dw ? kDwGroups * 128 * 2 : 0,
                               4 * (most_cols + dz / kColsumRows)});
  const size_t x2 = align256((size_t)2 * twice * cdiv(K, 8) * 8 * 2);
  return 256 + (M > 128 ? align256((size_t)std::min(M, kCeRest / V) * 4) : 0) + align256((size_t)dz * 2) +
         align256((size_t)dx * 4) + align256((size_t)dw * 4) + align256((size_t)db * 4) +
         std::max(x2, ce_pads_bwd(M, K) ? align256((size_t)(M + V) * ce_padded(K) * 2) : 0);
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

// Padded copies of both operands at `out`, and the product g on them.
static hipError_t ce_pad(const void* X, int64_t M, const void* W, int64_t V, int64_t K, uint16_t* out, GemmArgs& g,
                         hipStream_t s) {
  const int64_t ld = ce_padded(K);
  ce_pad_kernel<<<(unsigned)cdiv((M + V) * (ld / 8), 256), 256, 0, s>>>((const uint16_t*)X, M, (const uint16_t*)W, V,
                                                                        K, out, ld);
  g.A = out;
  g.B = out + M * ld;
  g.K = g.lda = g.ldb = ld;
  return hipGetLastError();
}

static bool ce_misaligned(const void* p, int n) { return reinterpret_cast<uintptr_t>(p) % n != 0; }

static int ce_check(const char* fn, const void* X, const void* W, const void* b, const int32_t* targets, int64_t M,
                    int64_t V, int64_t K, mpx_dtype dt) {
  const char* why = nullptr;
  if (!X || !W) why = "NULL operand";
  else if (M < 1 || V < 1 || K < 1) why = "M, V, K must be >= 1";
  else if (M > (1 << 20) || V > (1 << 24) || K > (1 << 16) || M * V > (int64_t)1 << 36 ||
           (M + V) * K > (int64_t)1 << 33)  // the launches' threads would not fit 32 bits
    why = "too large";
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
  return align256((size_t)ce_pairs(M, V, K) * 8) + align256((size_t)M * 4) +
         (ce_pads_fwd(M, V, K) ? align256((size_t)(M + V) * ce_padded(K) * 2) : 0);
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
  CeFwdArgs g{};
  static_cast<GemmArgs&>(g) = ce_args(X, W, M, V, K, K, K);
  g.bias = (const uint16_t*)b;
  g.part = (float2*)workspace;
  g.zt = (float*)((char*)workspace + align256((size_t)ce_pairs(M, V, K) * 8));
  g.targets = loss ? targets : nullptr;
  if (ce_pads_fwd(M, V, K)) MPX_HIP(ce_pad(X, M, W, V, K, (uint16_t*)(g.zt + align256((size_t)M * 4) / 4), g, s));
  const RowTile t = ce_tile(M, V, g.K, dma_ok(g, operands_aligned(g), true, true), false, true);
  const bool any = (t == STAGED_64 || t == STAGED_128) && staged_any(g, true, true);
  const RowTile tile = any ? STAGED_ANY : t;
  MPX_HIP(dt == MPX_F16 ? run_ce_fwd_f16(g, tile, s) : run_ce_fwd_bf16(g, tile, s));
  const int parts = (int)cdiv(V, tile_cols(tile));
  if (parts <= 16)
    ce_join_kernel<128><<<(unsigned)cdiv(M, 128), 1024, 0, s>>>(g.part, g.zt, targets, M, (int32_t)V, parts, loss,
                                                                (float2*)stats);
  else if (M >= 512)
    ce_join_kernel<16><<<(unsigned)cdiv(M, 16), 1024, 0, s>>>(g.part, g.zt, targets, M, (int32_t)V, parts, loss,
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
  return ce_bwd_bytes(M, V, K);
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
  const size_t need = mpx_linear_ce_bwd_workspace(M, V, K);
  if (!workspace || ws_bytes < need || ce_misaligned(workspace, 16)) {
    set_error("mpx_linear_ce_bwd: workspace of " + std::to_string(need) + " bytes, 16-byte aligned, required");
    return MPX_ERR_WORKSPACE;
  }
  const CePlan p = ce_plan(M, V, K);
  hipStream_t s = (hipStream_t)stream;
  char* ws = (char*)workspace;
  float* scalars = (float*)ws;
  uint16_t* dz = (uint16_t*)(ws + p.dz);
  // few rows: dz and what its rounding left, over X twice over
  const int64_t Mr = p.twice ? p.rows : M;
  uint16_t* X2 = (uint16_t*)(ws + p.x2);
  GemmArgs both = ce_args(X, W, M, V, K, K, K);  // X, W, or their padded copies
  if (ce_pads_bwd(M, K)) MPX_HIP(ce_pad(X, M, W, V, K, X2, both, s));
  const uint16_t* Xr = p.twice ? X2 : both.A;
  const int64_t ldx = p.twice ? cdiv(K, 8) * 8 : both.ldb;
  const unsigned grid = p.twice && dW ? (unsigned)(1 + p.rows) : 1;
  // bf16 with cotangents of its own: c = 1 and the scale as it stands, nothing to prepare
  const bool plain = dt == MPX_BF16 && g_loss;
  const float* unit = !plain ? scalars + 1 : d_state ? &d_state->scale : nullptr;
  const float* alpha = plain ? nullptr : scalars;
  if (!plain || grid > 1)
    MPX_HIP(by_type(dt, [&](auto type) {
      ce_prepare_kernel<type == MPX_F16><<<grid, 1024, 0, s>>>(g_loss, targets, M, d_state, scalars, (const uint16_t*)X,
                                                               K, X2, ldx);
      return hipGetLastError();
    }));
  // the reductions' own operands: dz is aligned, X and W as they come
  const auto out_tile = [&](const GemmArgs& g, bool ak, RowTile direct) {
    if ((reinterpret_cast<uintptr_t>(g.B) & 15u) == 0 && g.ldb % 8 == 0) return direct;
    return staged_any(g, ak, false) ? STAGED_ANY
           : cdiv(g.M, 64) * cdiv(g.N, 64) * g.splits <= 512 ? STAGED_64 : STAGED_128;
  };
  float* rest = p.rest && db ? (float*)(ws + p.lo) : nullptr;
  const auto run_out = [&](const CeOutArgs& g, bool ak, RowTile t) {
    return dt == MPX_F16 ? run_ce_out_f16(g, ak, t, s) : run_ce_out_bf16(g, ak, t, s);
  };
  CeReduce sums{};  // of a piece, and with the last one's dX's
  sums.width = (int32_t)p.width;
  sums.cols = (int32_t)K;
  sums.nonfinite = d_nonfinite;
  sums.alpha = alpha;
  sums.rest = rest;
  sums.targets = targets;
  sums.rows = (int32_t)M;
  const auto reduce = [&] {
    const auto fits = [](const CeSum& u) { return u.n % 4 == 0 && u.stride % 4 == 0; };
    const bool vec = fits(sums.first) && fits(sums.second);
    // 20 x 256 sums of 128 parts: one thread a value 6.8 us, 8 of them 4.5
    const int64_t per = vec ? 4 : 1, n = sums.first.n + sums.second.n;
    const bool few = n / per <= 16384 && std::max(sums.first.splits, sums.second.splits) >= 16;
    const int64_t at = (few ? 32 : 256) * per;
    const unsigned blocks = (unsigned)(cdiv(sums.first.n, at) + cdiv(sums.second.n, at) +
                                       (rest ? sums.nrows : cdiv(sums.nrows, 4)));
    return by_type(dt, [&](auto type) {
      const auto kernel = vec ? (few ? ce_reduce_kernel<type, true, 8> : ce_reduce_kernel<type, true, 1>)
                              : (few ? ce_reduce_kernel<type, false, 8> : ce_reduce_kernel<type, false, 1>);
      kernel<<<blocks, 256, 0, s>>>(sums);
      return hipGetLastError();
    });
  };
  int dx_parts = 0;  // partial sums of dX so far
  for (int64_t i = 0; i < p.pieces; ++i) {
    const int64_t v0 = i * p.cols, cols = i + 1 < p.pieces ? p.cols : p.last, ldz = cdiv(cols, 64) * 64;
    const uint16_t* Wp = both.B + v0 * both.ldb;
    CeGradArgs z{};
    static_cast<GemmArgs&>(z) = ce_args(both.A, Wp, M, cols, both.K, both.lda, both.ldb);
    z.bias = b ? (const uint16_t*)b + v0 : nullptr;
    z.C = dz;
    z.ldc = ldz;
    z.stats = (const float2*)stats;
    z.unit = unit;
    z.g_loss = g_loss;
    z.targets = targets;
    z.v0 = (int32_t)v0;
    z.vocabulary = (int32_t)V;
    const bool dma = dma_ok(z, operands_aligned(z), true, true);
    z.twice = (int32_t)p.twice;
    z.rest = rest;
    RowTile t = ce_tile(M, cols, K, dma, !dma && staged_any(z, true, true), false);
    if (t == TILE_256x256 && (z.twice || rest)) t = TILE_192x128;  // the large tiles make neither
    MPX_HIP(dt == MPX_F16 ? run_ce_grad_f16(z, t, s) : run_ce_grad_bf16(z, t, s));
    CeOutArgs x{}, w{};
    RowTile tx{}, tw{};
    if (dX) {
      static_cast<GemmArgs&>(x) = ce_args(dz, Wp, Mr, p.dx_parts ? p.width : K, cols, ldz, both.ldb);
      x.C = (uint16_t*)dX;
      const RowChoice c = ce_dx(Mr, cols, K, p.pieces > 1 || p.twice > 0);
      x.k_split = split_len(cols, c.splits);
      x.splits = split_count(cols, c.splits);
      x.part = p.dx_parts ? (float*)(ws + p.dxp) : nullptr;
      x.alpha = alpha;
      // the last piece may take another count than those before: what it adds to stands there
      x.add = i > 0 ? dx_parts : 0;
      dx_parts = std::max(dx_parts, x.splits);
      tx = out_tile(x, true, c.tile);
    }
    if (dW) {
      static_cast<GemmArgs&>(w) = ce_args(dz, Xr, cols, K, Mr, ldz, ldx);
      w.C = (uint16_t*)dW + v0 * K;
      const RowChoice c = ce_dw(Mr, cols, K);
      w.k_split = split_len(Mr, c.splits);
      w.splits = split_count(Mr, c.splits);
      w.part = w.splits > 1 ? (float*)(ws + p.dwp) : nullptr;
      if (w.part) w.N = p.width;
      w.alpha = alpha;
      w.add = 0;
      w.nonfinite = d_nonfinite;
      // db: summed by the first column of tiles and ended there, or shared by all columns
      // and ended by the reduction, which is worth its launch from about 30 us on, and
      // needed where the targets' rests belong to it
      if (db && !rest && w.splits == 1 && c.us < 30.0) w.db = (uint16_t*)db + v0;
      else if (db) w.dbp = (float*)(ws + p.dbp);
      tw = out_tile(w, false, c.tile);
    }
    if (dX && dW && tx <= TILE_192x128 && tw <= TILE_192x128) {
      MPX_HIP(dt == MPX_F16 ? run_ce_out_pair_f16(w, tw, x, tx, s) : run_ce_out_pair_bf16(w, tw, x, tx, s));
    } else {
      if (dX) MPX_HIP(run_out(x, true, tx));
      if (dW) MPX_HIP(run_out(w, false, tw));
    }
    if (dW) {
      sums.dbparts = (int)(w.splits * cdiv(K, tile_cols(tw)));
      sums.dbp = w.dbp;
      if (w.part) sums.first = {w.part, cols * p.width, cols * p.width, w.splits, w.C, d_nonfinite};
    } else if (db) {
      sums.dbp = (float*)(ws + p.dbp);
      sums.dbparts = (int)ce_colsum_parts(p.rows);
      MPX_HIP(by_type(dt, [&](auto type) {
        const dim3 grid((unsigned)(ldz / 64), (unsigned)cdiv(p.rows, kColsumRows));
        ce_colsum_kernel<type><<<grid, 256, 0, s>>>(dz, ldz, p.rows, cols, (float*)(ws + p.dbp));
        return hipGetLastError();
      }));
    }
    if (sums.dbp) {
      sums.nrows = cols;
      sums.db = (uint16_t*)db + v0;
      sums.v0 = (int32_t)v0;
    }
    if (dX && p.dx_parts && i + 1 == p.pieces)
      // few rows: each split's partial sums are two sets of rows
      sums.second = {(const float*)(ws + p.dxp), (p.twice ? p.twice : M) * p.width, M * p.width,
                     p.twice ? 2 * dx_parts : dx_parts, (uint16_t*)dX, nullptr};
    if (sums.first.n || sums.second.n || sums.nrows) MPX_HIP(reduce());
    sums.first = {};
    sums.nrows = 0;
  }
  return MPX_OK;
}
