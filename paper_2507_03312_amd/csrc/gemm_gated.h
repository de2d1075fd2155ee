// Gated feed-forward products on the tile kernels of gemm_kernels.h: forward
//   G = X Wg^T + bg,  U = X Wu^T + bu,  H = half(act(G) U)
// and, on the dX side of the down projection, dH = dY W,
//   dG = half(dH U act'(G)),  dU = half(dH act(G)).
// Sums, activation and products stay in float32: each result is rounded once.
// Internal; not part of the ABI.
#pragma once

#include "gemm_rows.h"

namespace mpx {

// silu(x) = x sigma(x) and its derivative sigma + x sigma (1 - sigma), on the
// hardware exp2 and reciprocal as gelu_sigma.
__device__ __forceinline__ float silu_sigma(float x) {
  return __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(-1.4426950408889634f * x));
}
template <int ACT>
__device__ __forceinline__ float gate_act(float x) {
  return x * (ACT == MPX_ACT_SILU ? silu_sigma(x) : gelu_sigma(x));
}
// act(x) and act'(x)
template <int ACT>
__device__ __forceinline__ void gate_act_grad(float x, float& a, float& d) {
  if constexpr (ACT == MPX_ACT_SILU) {
    const float s = silu_sigma(x);
    a = x * s;
    d = __builtin_fmaf(a, 1.0f - s, s);
  } else {
    a = gelu_tanh(x);
    d = gelu_tanh_grad(x);
  }
}

// Forward: operand B is the pair of W's gate and other rows, so a wave's two
// accumulator columns are G and U of the same 32 columns of H.  The matrix units and the
// stores behind them share the time: 12608 x 2048 x 768 bf16 with Pre 97 to 112 us, 0.73 PFLOP/s
// (the bare product of 4096 columns 91), without it 85; 8320 x 1024 x 384 f16 28 us, 59 MB, without
// 23.5.  Rounded before they pass LDS, at half its traffic: the first 5 us less.
template <int ACT>
struct GatedArgs : GemmArgs {  // C = H, pre = [G | U] or NULL, bias [2 N] or NULL
  static constexpr bool kPair = true, kRagged = false;
  static constexpr unsigned kTiles = 0;
  static constexpr int kPitch = 104, kBytes = 32 * kPitch * 2;  // 32 rows of H, G and U
  static constexpr int lds_bytes(int bm, int bn, int wm, int wn) { return bm / wm * (bn / wn) * kBytes; }
  int64_t pair;
  template <int DT, int TM, int STG>
  __device__ __forceinline__ NoPrefetch prefetch(int64_t, int64_t, int) const { return {}; }
  template <int DT, int BM, int BN, int WM, int WN, int TM, int TN>
  __device__ __forceinline__ void epilogue(const f32x16 (&acc)[TM][TN], const NoPrefetch&, int64_t, int64_t, int64_t mw,
                                           int64_t nw, int lane, int wave, int, uint8_t* smem) const {
    __syncthreads();  // every wave is done reading the stage buffers
    const int mv = (int)min<int64_t>(WM, M - mw), c8 = 8 * (lane & 3);
    const int nc = (int)min<int64_t>(8, N - nw - c8);
    if (mv <= 0 || N - nw <= 0) return;  // uniform over the wave
    const int nv = (int)min<int64_t>(32, N - nw);
    uint16_t* lds = reinterpret_cast<uint16_t*>(smem + wave * kBytes);
    f32x4 bg[4] = {}, bu[4] = {};
    if (bias) {  // uniform
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const int at = min(8 * q + 4 * (lane >> 5), nv - 1);
        bg[q] = load4<DT>(bias + nw + at, nv - at);
        bu[q] = load4<DT>(bias + N + nw + at, nv - at);
      }
    }
    static_for<TM>([&](auto i) {
      asm volatile("" ::: "memory");  // the wave's reads of the block before come first
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        float g[4], u[4], h[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          g[k] = acc[i][0][4 * q + k] + bg[q][k];
          u[k] = acc[i][1][4 * q + k] + bu[q][k];
          h[k] = gate_act<ACT>(g[k]) * u[k];
        }
        half_put<DT, kPitch>(h[0], h[1], h[2], h[3], lds, lane, 8 * q);
        if (pre) {
          half_put<DT, kPitch>(g[0], g[1], g[2], g[3], lds, lane, 32 + 8 * q);
          half_put<DT, kPitch>(u[0], u[1], u[2], u[3], lds, lane, 64 + 8 * q);
        }
      }
      asm volatile("" ::: "memory");  // the lanes' writes come before the wave's reads
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        const int r = (lane >> 2) + 16 * t, row = 32 * i + r;
        const uint16_t* p = lds + r * kPitch + c8;
        if (row < mv && nc > 0) {
          store8(C + (mw + row) * N + nw + c8, *reinterpret_cast<const u32x4*>(p), nc);
          if (pre) {
            uint16_t* o = pre + (mw + row) * 2 * N + nw + c8;
            store8(o, *reinterpret_cast<const u32x4*>(p + 32), nc);
            store8(o + N, *reinterpret_cast<const u32x4*>(p + 64), nc);
          }
        }
      }
    });
  }
};

// Backward: an ordinary dX product, whose float32 results meet G and U in the row
// layout (dact = [G | U], C = [dG | dU], rows of 2 N).  12608 x 2048 x 768 bf16 85 to 93 us,
// the matrix units busy 19% of them; repeated on one set of operands (in the last-level cache) 75
// to 78, of which the bare product 44.  The 207 MB of G, U and their gradients take the rest.
template <int ACT>
struct GatedBwdArgs : GemmArgs {
  static constexpr bool kPair = false, kRagged = false;
  static constexpr unsigned kTiles = 0;
  static constexpr int lds_bytes(int bm, int bn, int wm, int wn) { return bm / wm * (bn / wn) * kRowsBytes; }
  template <int DT, int TM, int STG>
  __device__ __forceinline__ NoPrefetch prefetch(int64_t, int64_t, int) const { return {}; }
  template <int DT, int BM, int BN, int WM, int WN, int TM, int TN>
  __device__ __forceinline__ void epilogue(const f32x16 (&acc)[TM][TN], const NoPrefetch&, int64_t, int64_t, int64_t mw,
                                           int64_t nw, int lane, int wave, int, uint8_t* smem) const {
    static_assert(TN == 2, "64 columns of a wave");
    __syncthreads();
    const int mv = (int)min<int64_t>(WM, M - mw), c8 = 8 * (lane & 7);
    const int nc = (int)min<int64_t>(8, N - nw - c8);
    if (mv <= 0 || N - nw <= 0) return;
    float* lds = reinterpret_cast<float*>(smem + wave * kRowsBytes);
    static_for<TM>([&](auto i) {
      // all in flight before the first is used.  (Loaded ahead of the main loop they cost
      // more than they hide: 12608 x 2048 x 768, one set, 74.5 -> 77.9 us, 8320 x 1024 x 384 21.5 -> 23.6)
      u32x4 gw[4], uw[4];
#pragma unroll
      for (int t = 0; t < 4; ++t) {
        const int row = min(32 * i + (lane >> 3) + 8 * t, mv - 1);
        const uint16_t* p = dact + (mw + row) * 2 * N + nw + c8;
        gw[t] = load8(p, nc);
        uw[t] = load8(p + N, nc);
      }
      rows_put(acc[i][0], lds, lane, 0);
      rows_put(acc[i][1], lds, lane, 32);
      asm volatile("" ::: "memory");
#pragma unroll
      for (int t = 0; t < 4; ++t) {
        const int r = (lane >> 3) + 8 * t, row = 32 * i + r;
        float d[8], x[8], u[8];
        rows_get8(lds + r * kRowsPitch + c8, d);
        unpack8<DT>(gw[t], x);
        unpack8<DT>(uw[t], u);
#pragma unroll
        for (int c = 0; c < 8; ++c) {
          float a, da;
          gate_act_grad<ACT>(x[c], a, da);
          x[c] = d[c] * u[c] * da;
          u[c] = d[c] * a;
        }
        if (row < mv && nc > 0) {
          uint16_t* p = C + (mw + row) * 2 * N + nw + c8;
          store8(p, pack8<DT>(x), nc);
          store8(p + N, pack8<DT>(u), nc);
        }
      }
      asm volatile("" ::: "memory");
    });
  }
};

// Tile of either product; pair: W's halves side by side, two columns for each of H.  Direct
// tiles: forward without and with Pre 1.1% and 0.9% slower than the fastest on average
// (64 x 128 alone 2.1 and 1.5, where the largest lose 20), backward 0.3%.  256 x 256 tiles
// were never more than 0.1% better a choice.
inline RowTile gated_tile(const GemmArgs& g, bool pair) {
  const int64_t cols = pair ? 2 * g.N : g.N;
  if (!dma_ok(g, operands_aligned(g), true, pair)) {
    if (staged_any(g, true, pair)) return STAGED_ANY;
    return cdiv(g.M, 64) * cdiv(cols, 64) <= 512 ? STAGED_64 : STAGED_128;
  }
  static const RowCost fwd[] = {{TILE_64x128, 64, 128, 3, {0.21, 0.60, 0.87}, 2.07},
                                {TILE_128x128, 128, 128, 2, {0.62, 0.62, 0}, 4.58},
                                {TILE_192x128, 192, 128, 2, {0.63, 1.00, 0}, 5.62}};
  static const RowCost keep[] = {{TILE_64x128, 64, 128, 3, {0.35, 0.62, 0.84}, 1.68},
                                 {TILE_128x128, 128, 128, 2, {0.73, 0.73, 0}, 3.82},
                                 {TILE_192x128, 192, 128, 2, {0.76, 0.80, 0}, 5.86}};
  static const RowCost bwd[] = {{TILE_64x128, 64, 128, 3, {0.92, 0.95, 1.02}, 2.33},
                                {TILE_128x128, 128, 128, 2, {0.83, 0.83, 0}, 6.84},
                                {TILE_192x128, 192, 128, 2, {1.12, 1.12, 0}, 10.0}};
  return choose_rows(!pair ? bwd : g.pre ? keep : fwd, g.M, cols, g.K).tile;
}

// Launchers, compiled once per half type
hipError_t run_gated_fwd_f16(const GemmArgs& g, int64_t pair, RowTile t, hipStream_t s);
hipError_t run_gated_fwd_bf16(const GemmArgs& g, int64_t pair, RowTile t, hipStream_t s);
hipError_t run_gated_bwd_f16(const GemmArgs& g, RowTile t, hipStream_t s);
hipError_t run_gated_bwd_bf16(const GemmArgs& g, RowTile t, hipStream_t s);

template <int DT, int ACT>
hipError_t run_gated_fwd(const GemmArgs& g, int64_t pair, RowTile t, hipStream_t s) {
  GatedArgs<ACT> a{};
  static_cast<GemmArgs&>(a) = g;
  a.pair = pair;
  return launch_rows<DT, GatedArgs<ACT>, true, true, false>(a, t, s);
}
template <int DT, int ACT>
hipError_t run_gated_bwd(const GemmArgs& g, RowTile t, hipStream_t s) {
  GatedBwdArgs<ACT> a{};
  static_cast<GemmArgs&>(a) = g;
  return launch_rows<DT, GatedBwdArgs<ACT>, true, false, false>(a, t, s);
}

}  // namespace mpx
