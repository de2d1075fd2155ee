// Cross entropy straight from the last hidden states, on the tile kernels of
// gemm_kernels.h: the logits z = X W^T + b exist only as a tile's accumulators.
//   forward   per row m = max z, S = sum e^(z - m): a tile leaves its own (m, S) per row,
//             and the target's logit; a second kernel joins them.
//   backward  in pieces of the vocabulary: z again, dz = f (p - [target]) to a workspace of
//             one piece in the half type, dX += dz W (float32), dW = dz^T X.
// f = c scale g of the row.  c is a power of two, taken out of the results again: it
// brings float16's dz into the middle of its range (a probability of 2^-28 still has
// all its bits), and is 1 for bf16.
// Internal; not part of the ABI.
#pragma once

#include "gemm_rows.h"

namespace mpx {

constexpr float kLog2e = 1.4426950408889634f;

// The value of the other half wave's lane.
__device__ __forceinline__ float other_half(float v) { return __shfl_xor(v, 32); }

// Forward.  A = X, B = W; lane l of a 32 x 32 block has row l % 32 and 16 of its 32
// columns, so a row's maximum and sum take one exchange beside the lane's own values.
// The matrix units bound the large ones: 4096 x 65537 x 768 bf16 400 to 416 us, 0.99 to 1.03 PFLOP/s
// (the exponentials of 2.7e8 logits are what keeps it off the 387 us of the bare
// product); W's 201 MB the few rows: 2 x 131072 x 768 42 us, 4.8 TB/s.
struct CeFwdArgs : GemmArgs {
  static constexpr bool kPair = false, kRagged = false;
  static constexpr unsigned kTiles = bit(TILE_32x128) | bit(TILE_256x256);
  static constexpr int lds_bytes(int bm, int bn, int wm, int wn) { return bm * (bn / wn) * 8; }
  float2* part;  // [tile column][M]
  float* zt;     // [M]: the target's logit
  const int32_t* targets;
  template <int TM>
  struct Rows {
    int32_t target[TM];
  };
  template <int DT, int TM, int STG>
  __device__ __forceinline__ Rows<TM> prefetch(int64_t mw, int64_t, int lane) const {
    Rows<TM> r;
#pragma unroll
    for (int i = 0; i < TM; ++i) {
      const int64_t row = mw + 32 * i + (lane & 31);
      r.target[i] = targets && row < M ? targets[row] : -1;
    }
    return r;
  }
  template <int DT, int BM, int BN, int WM, int WN, int TM, int TN>
  __device__ __forceinline__ void epilogue(f32x16 (&acc)[TM][TN], const Rows<TM>& early, int64_t m0, int64_t n0,
                                           int64_t mw, int64_t nw, int lane, int wave, int, uint8_t* smem) const {
    __syncthreads();  // every wave is done reading the stage buffers
    float2* rows = reinterpret_cast<float2*>(smem);  // [wave column][BM]
    const int hi = lane >> 5, wc = wave % (BN / WN), wr = wave / (BN / WN);
    const int nv = (int)min<int64_t>(WN, N - nw);  // may be <= 0
    if (bias && nv > 0) add_bias<DT>(acc, bias + nw, nv, lane);
    if (nv < WN) {  // uniform: columns behind the vocabulary have probability 0
      static_for<TN>([&](auto j) {
#pragma unroll
        for (int e = 0; e < 16; ++e) {
          const bool in = 32 * j + 8 * (e / 4) + 4 * hi + e % 4 < nv;
          static_for<TM>([&](auto i) { acc[i][j][e] = in ? acc[i][j][e] : -__builtin_inff(); });
        }
      });
    }
    static_for<TM>([&](auto i) {
      const int64_t row = mw + 32 * i + (lane & 31);
      const int64_t t = early.target[i] < 0 ? -1 : early.target[i] - nw;
      if (__ballot(t >= 0 && t < nv)) {  // few tiles hold a target
        static_for<TN>([&](auto j) {
#pragma unroll
          for (int e = 0; e < 16; ++e)
            if (t == 32 * j + 8 * (e / 4) + 4 * hi + e % 4 && t < nv) zt[row] = acc[i][j][e];
        });
      }
      float m = acc[i][0][0];
      static_for<TN>([&](auto j) {
#pragma unroll
        for (int e = 0; e < 16; ++e) m = fmaxf(m, acc[i][j][e]);
      });
      m = fmaxf(m, other_half(m));
      const float at = m == -__builtin_inff() ? 0.0f : m;  // nothing but masked ones: S = 0
      // m first, which is exact near it: the largest one's own term is 1 and ln S never below 0,
      // while z log2 e - m log2 e in one rounding would leave m log2 e's (2^-24 m in ln S)
      float s = 0.0f;
      static_for<TN>([&](auto j) {
#pragma unroll
        for (int e = 0; e < 16; ++e) s += __builtin_amdgcn_exp2f((acc[i][j][e] - at) * kLog2e);
      });
      s += other_half(s);
      if (hi == 0) rows[wc * BM + wr * WM + 32 * i + lane] = make_float2(m, s);
    });
    __syncthreads();
    float2* out = part + n0 / BN * M + m0;
    for (int r = threadIdx.x; r < BM && m0 + r < M; r += BM / WM * (BN / WN) * 64) {
      float2 a = rows[r];
#pragma unroll
      for (int w = 1; w < BN / WN; ++w) {
        const float2 b = rows[w * BM + r];
        const float m = fmaxf(a.x, b.x), at = m == -__builtin_inff() ? 0.0f : m;
        a = make_float2(m, a.y * __builtin_amdgcn_exp2f((a.x - at) * kLog2e) +
                               b.y * __builtin_amdgcn_exp2f((b.x - at) * kLog2e));
      }
      out[r] = a;
    }
  }
};

// Backward, dz of a piece (bound as the forward: 4096 x 15872 x 768 bf16 115 us, 0.87 PFLOP/s,
// the 130 MB of dz go out while it runs): the same product, C = dz [M rounded up to 64][ldc], with
// zeros in rows behind M and columns behind N (up to ldc), as the products that reduce
// over them need.  A masked logit (-inf) has no gradient, but in a row that is NaN.
// twice (few rows): row twice + r holds what rounding row r to half left, and the products
// take both.  Few rows have few large dz (their targets'), whose roundings do not average
// out: 4 rows of 170 columns bf16 3.3e-3 of dX's norm against 1.8e-3 for one rounding of
// the result, while the second rows cost little beside the reading of W.  rest (nullable):
// the same of the rows' targets alone, for db, whose sums of few rows cancel.
struct CeGradArgs : GemmArgs {
  static constexpr bool kPair = false, kRagged = false;
  static constexpr unsigned kTiles = bit(TILE_256x256);
  static constexpr int lds_bytes(int bm, int bn, int wm, int wn) { return bm / wm * (bn / wn) * kHalfBytes; }
  const float2* stats;
  const float* unit;  // c scale, or c scale / rows with a target when g_loss is NULL (nullable: 1)
  const float* g_loss;
  const int32_t* targets;
  int32_t v0, vocabulary;  // the piece's first column, and the columns of all
  int32_t twice;
  float* rest;  // [M]
  template <int TM>
  struct Rows {
    float2 stats[TM];
    float g[TM];
    int32_t target[TM];
    float unit;
  };
  template <int DT, int TM, int STG>
  __device__ __forceinline__ Rows<TM> prefetch(int64_t mw, int64_t, int lane) const {
    Rows<TM> r;
    r.unit = unit ? *unit : 1.0f;
#pragma unroll
    for (int i = 0; i < TM; ++i) {
      const int64_t row = min(mw + 32 * i + (lane & 31), M - 1);
      r.stats[i] = stats[row];
      r.target[i] = targets[row];
      r.g[i] = g_loss ? g_loss[row] : 1.0f;
    }
    return r;
  }
  template <int DT, int BM, int BN, int WM, int WN, int TM, int TN>
  __device__ __forceinline__ void epilogue(f32x16 (&acc)[TM][TN], const Rows<TM>& early, int64_t, int64_t, int64_t mw,
                                           int64_t nw, int lane, int wave, int, uint8_t* smem) const {
    static_assert(TN == 2, "64 columns of a wave");
    // neither of twice and rest comes with tiles of 256: there they spilled (118 -> 164 us)
    constexpr bool kExact = BM < 256;
    __syncthreads();
    const int64_t rows64 = twice ? twice : (M + 63) / 64 * 64;
    if (mw >= rows64 || nw >= ldc) return;  // uniform over the wave
    uint16_t* lds = reinterpret_cast<uint16_t*>(smem + wave * kHalfBytes);
    const int hi = lane >> 5, nv = (int)min<int64_t>(64, N - nw);  // >= 1: ldc is N rounded up to 64
    if (bias) add_bias<DT>(acc, bias + nw, nv, lane);
    static_for<TM>([&](auto i) {
      const int64_t row = mw + 32 * i + (lane & 31);
      const float2 st = early.stats[i];
      const int32_t target = early.target[i];
      const int64_t t = (int64_t)target - v0 - nw;
      const float f = row >= M || target < 0 ? 0.0f
                      : target >= vocabulary ? __builtin_nanf("") : early.g[i] * early.unit;
      // f p = f 2^((z - m) log2 e + c), m first as in the forward (a certain target's p - 1 is never
      // above 0): a masked z gives 0, a NaN in m, ln S or f a NaN row.  All masked: m = 0
      const float at = st.x == -__builtin_inff() ? 0.0f : st.x;
      const float c = row >= M ? -__builtin_inff() : -(st.y * kLog2e);
      const bool plain = nv == 64 && !__ballot(t >= 0 && t < 64);  // uniform: no target, no edge
      for (int low = 0; low <= (kExact && twice ? 1 : 0); ++low) {
        asm volatile("" ::: "memory");  // the wave's reads of the block before come first
        static_for<2>([&](auto j) {
#pragma unroll
          for (int q = 0; q < 4; ++q) {
            float p[4];
            if (plain) {
#pragma unroll
              for (int k = 0; k < 4; ++k)
                p[k] = f * __builtin_amdgcn_exp2f(__builtin_fmaf(acc[i][j][4 * q + k] - at, kLog2e, c));
            } else {
#pragma unroll
              for (int k = 0; k < 4; ++k) {
                const int col = 32 * j + 8 * q + 4 * hi + k;
                const float z = acc[i][j][4 * q + k];
                p[k] = __builtin_amdgcn_exp2f(__builtin_fmaf(z - at, kLog2e, c));
                p[k] = f * (p[k] - (col == t && z != -__builtin_inff() ? 1.0f : 0.0f));
                p[k] = col < nv ? p[k] : 0.0f;
                if (kExact && rest && col == t && row < M) rest[row] = p[k] - h2f<DT>(f2h<DT>(p[k]));
              }
            }
            if (low) {
#pragma unroll
              for (int k = 0; k < 4; ++k) p[k] -= h2f<DT>(f2h<DT>(p[k]));
            }
            half_put<DT, kHalfPitch>(p[0], p[1], p[2], p[3], lds, lane, 32 * j + 8 * q);
          }
        });
        asm volatile("" ::: "memory");  // the lanes' writes come before the wave's reads
#pragma unroll
        for (int t4 = 0; t4 < 4; ++t4) {
          const int r = (lane >> 3) + 8 * t4;
          const u32x4 w = *reinterpret_cast<const u32x4*>(lds + r * kHalfPitch + 8 * (lane & 7));
          if (mw + 32 * i + r < rows64)
            *reinterpret_cast<u32x4*>(C + (mw + 32 * i + r + (low ? twice : 0)) * ldc + nw + 8 * (lane & 7)) = w;
        }
      }
    });
  }
};

// Backward, products of a piece: C = half(alpha acc), or (part set) float32 partial
// sums per split, on top of an earlier piece's in the first `add` of them.  Of pieces of
// 4096 x 16384 x 768 bf16 dX 110 us and dW 98 alone (0.94 and 1.05 PFLOP/s; the bare product 91).
struct CeOutArgs : GemmArgs {
  static constexpr bool kPair = false, kRagged = true;
  static constexpr unsigned kTiles = bit(TILE_256x256);
  static constexpr int lds_bytes(int bm, int bn, int wm, int wn) { return bm / wm * (bn / wn) * kRowsBytes; }
  float* part;         // [splits][M][N]
  const float* alpha;  // 1 / c (nullable: 1)
  int32_t add;
  __device__ __forceinline__ float db_end(float sum, int64_t) const { return alpha ? sum * *alpha : sum; }
  template <int DT, int TM, int STG>
  __device__ __forceinline__ NoPrefetch prefetch(int64_t, int64_t, int) const { return {}; }
  template <int DT, int BM, int BN, int WM, int WN, int TM, int TN>
  __device__ __forceinline__ void epilogue(const f32x16 (&acc)[TM][TN], const NoPrefetch&, int64_t, int64_t,
                                           int64_t mw, int64_t nw, int lane, int wave, int split,
                                           uint8_t* smem) const {
    static_assert(TN == 2, "64 columns of a wave");
    __syncthreads();
    const int mv = (int)min<int64_t>(WM, M - mw), c8 = 8 * (lane & 7);
    const int nc = (int)min<int64_t>(8, N - nw - c8);
    if (mv <= 0 || N - nw <= 0) return;  // uniform over the wave
    float* lds = reinterpret_cast<float*>(smem + wave * kRowsBytes);
    const float scale = part || !alpha ? 1.0f : *alpha;
    const bool whole = nc == 8 && N % 4 == 0, more = split < add;
    int bad = 0;
    static_for<TM>([&](auto i) {
      rows_put(acc[i][0], lds, lane, 0);
      rows_put(acc[i][1], lds, lane, 32);
      asm volatile("" ::: "memory");
      f32x4 old[8];
      if (part && more && whole) {  // all in flight before the first is used
#pragma unroll
        for (int t = 0; t < 4; ++t) {
          const int row = min(32 * i + (lane >> 3) + 8 * t, mv - 1);
          const float* p = part + ((int64_t)split * M + mw + row) * N + nw + c8;
          old[2 * t] = *reinterpret_cast<const f32x4*>(p);
          old[2 * t + 1] = *reinterpret_cast<const f32x4*>(p + 4);
        }
      }
#pragma unroll
      for (int t = 0; t < 4; ++t) {
        const int r = (lane >> 3) + 8 * t, row = 32 * i + r;
        float v[8];
        rows_get8(lds + r * kRowsPitch + c8, v);
        if (row >= mv || nc <= 0) continue;
        if (part) {
          float* p = part + ((int64_t)split * M + mw + row) * N + nw + c8;
          if (whole) {
#pragma unroll
            for (int c = 0; c < 8; ++c) v[c] += more ? old[2 * t + c / 4][c % 4] : 0.0f;
            *reinterpret_cast<f32x4*>(p) = f32x4{v[0], v[1], v[2], v[3]};
            *reinterpret_cast<f32x4*>(p + 4) = f32x4{v[4], v[5], v[6], v[7]};
          } else {
#pragma unroll
            for (int c = 0; c < 8; ++c)
              if (c < nc) p[c] = more ? p[c] + v[c] : v[c];
          }
        } else {
#pragma unroll
          for (int c = 0; c < 8; ++c) v[c] *= scale;
          const u32x4 w = pack8<DT>(v);
          store8(C + (mw + row) * N + nw + c8, w, nc);
          if (nonfinite) {
#pragma unroll
            for (int c = 0; c < 8; ++c)
              bad += c < nc && h_nonfinite<DT>((uint16_t)(w[c / 2] >> (16 * (c & 1)))) ? 1 : 0;
          }
        }
      }
      asm volatile("" ::: "memory");
    });
    if (nonfinite && !part) add_nonfinite(nonfinite, bad);
  }
};

// dW and dX of a piece in one launch, 128 columns and four waves a tile each: small ones leave
// most of the chip empty while they wait for memory (509 x 1000 x 384 f16 5.9 + 10.5 us alone,
// 12.0 together), large ones share their last rounds.  Over 40 passes with gradient 0.91 of the
// time of two launches, none slower.
struct CePairPlace {
  uint32_t group, in_row;  // of a product's workgroups, its tiles
  __device__ __forceinline__ uint32_t tile() const { return group % in_row; }
  __device__ __forceinline__ uint32_t tiles() const { return in_row; }
  __device__ __forceinline__ uint32_t batch() const { return group / in_row; }
};
template <int DT, bool DBS, int BMW, int BMX>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(2, 2)))
void ce_out_pair_kernel(CeOutArgs w, uint32_t wtiles, uint32_t wgroups, CeOutArgs x, uint32_t xtiles) {
  __shared__ __attribute__((aligned(1024))) uint8_t smem[std::max(
      gemm_tile_lds<BMW, 128, BMW / 2, 64, CeOutArgs>(), gemm_tile_lds<BMX, 128, BMX / 2, 64, CeOutArgs>())];
  const uint32_t b = blockIdx.x;
  if (b < wgroups)
    gemm_tile<DT, BMW, 128, BMW / 2, 64, false, false, 0, DBS, 0, false>(w, smem, CePairPlace{b, wtiles});
  else
    gemm_tile<DT, BMX, 128, BMX / 2, 64, true, false, 0, false, 0, false>(x, smem, CePairPlace{b - wgroups, xtiles});
}
template <int DT, int BMW, int BMX>
hipError_t launch_ce_out_pair(const CeOutArgs& w, const CeOutArgs& x, hipStream_t s) {
  const uint32_t wt = (uint32_t)(cdiv(w.M, BMW) * cdiv(w.N, 128)), xt = (uint32_t)(cdiv(x.M, BMX) * cdiv(x.N, 128));
  const uint32_t wg = wt * w.splits, groups = wg + xt * x.splits;
  if (w.dbp || w.db) ce_out_pair_kernel<DT, true, BMW, BMX><<<groups, 256, 0, s>>>(w, wt, wg, x, xt);
  else ce_out_pair_kernel<DT, false, BMW, BMX><<<groups, 256, 0, s>>>(w, wt, wg, x, xt);
  return hipGetLastError();
}
template <int DT>
hipError_t launch_ce_out_pair(const CeOutArgs& w, RowTile tw, const CeOutArgs& x, RowTile tx, hipStream_t s) {
  if (tw == TILE_128x128) {
    if (tx == TILE_64x128) return launch_ce_out_pair<DT, 128, 64>(w, x, s);
    if (tx == TILE_128x128) return launch_ce_out_pair<DT, 128, 128>(w, x, s);
    return launch_ce_out_pair<DT, 128, 192>(w, x, s);
  }
  if (tx == TILE_64x128) return launch_ce_out_pair<DT, 192, 64>(w, x, s);
  if (tx == TILE_128x128) return launch_ce_out_pair<DT, 192, 128>(w, x, s);
  return launch_ce_out_pair<DT, 192, 192>(w, x, s);
}

// Launchers, compiled once per half type.  The layouts: forward and dz k-major operands,
// dX a k-major A, dW neither.
hipError_t run_ce_fwd_f16(const CeFwdArgs& g, RowTile t, hipStream_t s);
hipError_t run_ce_fwd_bf16(const CeFwdArgs& g, RowTile t, hipStream_t s);
hipError_t run_ce_grad_f16(const CeGradArgs& g, RowTile t, hipStream_t s);
hipError_t run_ce_grad_bf16(const CeGradArgs& g, RowTile t, hipStream_t s);
hipError_t run_ce_out_f16(const CeOutArgs& g, bool ak, RowTile t, hipStream_t s);
hipError_t run_ce_out_bf16(const CeOutArgs& g, bool ak, RowTile t, hipStream_t s);
hipError_t run_ce_out_pair_f16(const CeOutArgs& w, RowTile tw, const CeOutArgs& x, RowTile tx, hipStream_t s);
hipError_t run_ce_out_pair_bf16(const CeOutArgs& w, RowTile tw, const CeOutArgs& x, RowTile tx, hipStream_t s);

}  // namespace mpx
