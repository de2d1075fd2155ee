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
// The same of results that need nothing from the row layout: rounded to half first, which
// halves the LDS traffic.  Rows of PITCH halves, a multiple of 8 for 16-byte reads.
template <int DT, int PITCH>
__device__ __forceinline__ void half_put(float a, float b, float c, float d, uint16_t* lds, int lane, int col) {
  *reinterpret_cast<u32x2*>(lds + (lane & 31) * PITCH + col + 4 * (lane >> 5)) =
      u32x2{f2h<DT>(a) | ((uint32_t)f2h<DT>(b) << 16), f2h<DT>(c) | ((uint32_t)f2h<DT>(d) << 16)};
}
constexpr int kHalfPitch = 72;  // 64 columns
constexpr int kHalfBytes = 32 * kHalfPitch * 2;
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

// Values p[0 .. 3] of a vector, the last `left` (>= 1) of its ones from p on at most; what is
// past them repeats the last one.
template <int DT>
__device__ __forceinline__ f32x4 load4(const uint16_t* p, int left) {
  typedef u32x2 u32x2_half __attribute__((aligned(2)));
  f32x4 v;
  if (left >= 4) {
    const u32x2 w = *reinterpret_cast<const u32x2_half*>(p);
#pragma unroll
    for (int c = 0; c < 4; ++c) v[c] = h2f<DT>((uint16_t)(w[c / 2] >> (16 * (c & 1))));
  } else {
#pragma unroll
    for (int c = 0; c < 4; ++c) v[c] = h2f<DT>(p[min(c, left - 1)]);
  }
  return v;
}
// acc += bias of its columns, from b on, nv (>= 1) of them in the output
template <int DT, int TM, int TN>
__device__ __forceinline__ void add_bias(f32x16 (&acc)[TM][TN], const uint16_t* b, int nv, int lane) {
  static_for<TN>([&](auto j) {
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const int col = 32 * j + 8 * q + 4 * (lane >> 5);
      const int at = min(col, nv - 1);
      const f32x4 v = load4<DT>(b + at, nv - at);
      static_for<TM>([&](auto i) {
#pragma unroll
        for (int k = 0; k < 4; ++k) acc[i][j][4 * q + k] += v[k];
      });
    }
  });
}

struct NoPrefetch {};

// Which tile a product with an end of its own takes: direct-to-LDS ones by size, or
// register-staged ones (any alignment; STAGED_ANY: also rows of fewer than 8 values).
enum RowTile { TILE_32x128, TILE_64x128, TILE_128x128, TILE_192x128, TILE_256x256, STAGED_64, STAGED_128, STAGED_ANY };
constexpr unsigned bit(RowTile t) { return 1u << t; }
constexpr int tile_cols(RowTile t) {
  return t == TILE_256x256 ? 256 : t == STAGED_64 || t == STAGED_ANY ? 64 : 128;
}
constexpr int tile_rows(RowTile t) {
  return t == TILE_32x128 ? 32 : t == TILE_192x128 ? 192 : t == TILE_256x256 ? 256
         : t == TILE_128x128 || t == STAGED_128 ? 128 : 64;
}
// Whether the threads of a launch of these tiles fit its 32 bits.
constexpr bool tiles_fit(RowTile t, int64_t M, int64_t cols) {
  const int64_t threads = t == STAGED_64 || t == STAGED_ANY ? 128 : t == TILE_256x256 ? 512 : 256;
  return cdiv(M, tile_rows(t)) * cdiv(cols, tile_cols(t)) < ((int64_t)1 << 32) / threads;
}

// Direct-to-LDS tiles by estimated time: a chip of 256 CUs runs 256 x per_cu workgroups at
// a time; a round of o per CU takes its k tiles of 64 x k_us[o - 1] plus o x tile_us for what
// surrounds the k loops, and the last round has the workgroups that are left.  The
// constants are set for the choice, not for the times: those of least loss on 70% of
// 520 products of each kind (33 to 16640 rows, 128 to 32768 columns, reductions of 64 to
// 1536, a quarter of them large), operands from HBM; what they lose on the other 30%
// stands at each table.
struct RowCost {
  RowTile tile;
  int bm, bn, per_cu;
  double k_us[3], tile_us;
};
struct RowChoice {
  RowTile tile;
  int splits;
  double us;
};
// cols: columns of operand B's tiles; splits 1 .. most, each with `len` / splits of the
// reduction.  join_us, part_us: what a second split costs, and every output of a split.
template <int N>
inline RowChoice choose_rows(const RowCost (&costs)[N], int64_t M, int64_t cols, int64_t len, int64_t most = 1,
                             double join_us = 0.0, double part_us = 0.0, bool one_is_free = true) {
  RowChoice best{costs[0].tile, 1, 0.0};
  for (const RowCost& c : costs) {
    const int64_t tiles = cdiv(M, c.bm) * cdiv(cols, c.bn), slots = 256 * c.per_cu;
    for (int64_t s = 1; s <= most; s += s < 6 ? 1 : s < 16 ? 2 : s / 4) {
      const double nk = (double)cdiv(len, 64 * s);
      auto round = [&](int64_t o) { return o ? nk * c.k_us[o - 1] + c.tile_us * (double)o : 0.0; };
      const double t = (double)(tiles * s / slots) * round(c.per_cu) + round(cdiv(tiles * s % slots, 256)) +
                       (s > 1 ? join_us : 0.0) +
                       (s > 1 || !one_is_free ? part_us * (double)s * (double)M * (double)cols : 0.0);
      if (best.us == 0.0 || t < best.us) best = {c.tile, (int)s, t};
    }
  }
  return best;
}

template <int DT, class Args, bool AK, bool BKM, bool DBS, int BM, int BN, int WM, int WN, int OCC, int STG>
hipError_t launch_row_tiles(const Args& g, hipStream_t s) {
  const dim3 grid((unsigned)(cdiv(g.M, BM) * cdiv(g.N, Args::kPair ? BN / 2 : BN)), (unsigned)g.splits);
  gemm_tile_kernel<DT, BM, BN, WM, WN, OCC, AK, BKM, 0, DBS, STG, false, Args>
      <<<grid, BM / WM * (BN / WN) * 64, 0, s>>>(g);
  return hipGetLastError();
}

// AK, BKM: the operands' layouts; DBS: with the sums of A's rows.  Tiles of 32
// rows and of 256 are compiled where Args::kTiles has them, of 64 for a k-major A.
template <int DT, class Args, bool AK, bool BKM, bool DBS>
hipError_t launch_rows(const Args& g, RowTile t, hipStream_t s) {
  constexpr unsigned tiles = Args::kTiles;
  switch (t) {
    case TILE_32x128:
      if constexpr (tiles & bit(TILE_32x128))
        return launch_row_tiles<DT, Args, AK, BKM, DBS, 32, 128, 32, 32, 4, 0>(g, s);
      break;
    case TILE_64x128:
      if constexpr (AK) return launch_row_tiles<DT, Args, AK, BKM, DBS, 64, 128, 32, 64, 3, 0>(g, s);
      break;
    case TILE_128x128: return launch_row_tiles<DT, Args, AK, BKM, DBS, 128, 128, 64, 64, 2, 0>(g, s);
    case TILE_192x128: return launch_row_tiles<DT, Args, AK, BKM, DBS, 192, 128, 96, 64, 2, 0>(g, s);
    case TILE_256x256:
      if constexpr (tiles & bit(TILE_256x256))
        return launch_row_tiles<DT, Args, AK, BKM, DBS, 256, 256, 128, 64, 2, 0>(g, s);
      break;
    case STAGED_64: return launch_row_tiles<DT, Args, AK, BKM, DBS, 64, 64, 32, 64, 2, 1>(g, s);
    case STAGED_128: return launch_row_tiles<DT, Args, AK, BKM, DBS, 128, 128, 64, 64, 2, 1>(g, s);
    case STAGED_ANY: return launch_row_tiles<DT, Args, AK, BKM, DBS, 64, 64, 32, 64, 2, 2>(g, s);
  }
  return hipErrorInvalidValue;
}

}  // namespace mpx
