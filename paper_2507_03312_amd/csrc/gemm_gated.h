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
// accumulator columns are G and U of the same 32 columns of H.
template <int ACT>
struct GatedArgs : GemmArgs {  // C = H, pre = [G | U] or NULL, bias [2 N] or NULL
  static constexpr bool kPair = true, kRagged = false;
  static constexpr int lds_bytes(int bm, int bn, int wm, int wn) { return bm / wm * (bn / wn) * kRowsBytes; }
  int64_t pair;
  template <int DT, int BM, int BN, int WM, int WN, int TM, int TN>
  __device__ __forceinline__ void epilogue(const f32x16 (&acc)[TM][TN], int64_t, int64_t, int64_t mw, int64_t nw,
                                           int lane, int wave, int, uint8_t* smem) const {
    __syncthreads();  // every wave is done reading the stage buffers
    const int mv = (int)min<int64_t>(WM, M - mw), c8 = 8 * (lane & 3);
    const int nc = (int)min<int64_t>(8, N - nw - c8);
    if (mv <= 0 || N - nw <= 0) return;  // uniform over the wave
    float* lds = reinterpret_cast<float*>(smem + wave * kRowsBytes);
    float bg[8] = {}, bu[8] = {};
    if (bias && nc > 0) {
      unpack8<DT>(load8(bias + nw + c8, nc), bg);
      unpack8<DT>(load8(bias + N + nw + c8, nc), bu);
    }
    static_for<TM>([&](auto i) {
      rows_put(acc[i][0], lds, lane, 0);
      rows_put(acc[i][1], lds, lane, 32);
      asm volatile("" ::: "memory");  // the lanes' writes come before the wave's reads
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        const int r = (lane >> 2) + 16 * t, row = 32 * i + r;
        float a[8], b[8], h[8];
        rows_get8(lds + r * kRowsPitch + c8, a);
        rows_get8(lds + r * kRowsPitch + 32 + c8, b);
#pragma unroll
        for (int c = 0; c < 8; ++c) {
          a[c] += bg[c];
          b[c] += bu[c];
          h[c] = gate_act<ACT>(a[c]) * b[c];
        }
        if (row < mv && nc > 0) {
          store8(C + (mw + row) * N + nw + c8, pack8<DT>(h), nc);
          if (pre) {
            uint16_t* p = pre + (mw + row) * 2 * N + nw + c8;
            store8(p, pack8<DT>(a), nc);
            store8(p + N, pack8<DT>(b), nc);
          }
        }
      }
      asm volatile("" ::: "memory");  // and its reads before the next block's writes
    });
  }
};

// Backward: an ordinary dX product, whose float32 results meet G and U in the row
// layout (dact = [G | U], C = [dG | dU], rows of 2 N).
template <int ACT>
struct GatedBwdArgs : GemmArgs {
  static constexpr bool kPair = false, kRagged = false;
  static constexpr int lds_bytes(int bm, int bn, int wm, int wn) { return bm / wm * (bn / wn) * kRowsBytes; }
  template <int DT, int BM, int BN, int WM, int WN, int TM, int TN>
  __device__ __forceinline__ void epilogue(const f32x16 (&acc)[TM][TN], int64_t, int64_t, int64_t mw, int64_t nw,
                                           int lane, int wave, int, uint8_t* smem) const {
    static_assert(TN == 2, "64 columns of a wave");
    __syncthreads();
    const int mv = (int)min<int64_t>(WM, M - mw), c8 = 8 * (lane & 7);
    const int nc = (int)min<int64_t>(8, N - nw - c8);
    if (mv <= 0 || N - nw <= 0) return;
    float* lds = reinterpret_cast<float*>(smem + wave * kRowsBytes);
    static_for<TM>([&](auto i) {
      u32x4 gw[4], uw[4];  // all in flight before the first is used
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

// Tile launches.  Both products have a k-major A and no splits; BKM: the layout of B.
template <int DT, class Args, bool BKM, int BM, int BN, int WM, int OCC, int STG>
hipError_t launch_gated_tiles(const Args& g, hipStream_t s) {
  constexpr int BC = Args::kPair ? BN / 2 : BN;
  const int64_t tiles = cdiv(g.M, BM) * cdiv(g.N, BC);
  gemm_tile_kernel<DT, BM, BN, WM, 64, OCC, true, BKM, 0, false, STG, false, Args>
      <<<(unsigned)tiles, BM / WM * (BN / 64) * 64, 0, s>>>(g);
  return hipGetLastError();
}

template <int DT, class Args, bool BKM>
hipError_t launch_gated(const Args& g, hipStream_t s) {
  const bool dma = dma_ok(g, operands_aligned(g), true, BKM);
  const int64_t cols = Args::kPair ? 2 * g.N : g.N;
  if (!dma) {
    if (staged_any(g, true, BKM)) return launch_gated_tiles<DT, Args, BKM, 64, 64, 32, 2, 2>(g, s);
    if (cdiv(g.M, 64) * cdiv(cols, 64) <= 512) return launch_gated_tiles<DT, Args, BKM, 64, 64, 32, 2, 1>(g, s);
    return launch_gated_tiles<DT, Args, BKM, 128, 128, 64, 2, 1>(g, s);
  }
  if (cdiv(g.M, 256) * cdiv(cols, 256) >= 512) return launch_gated_tiles<DT, Args, BKM, 256, 256, 128, 2, 0>(g, s);
  if (cdiv(g.M, 128) * cdiv(cols, 128) >= 384) return launch_gated_tiles<DT, Args, BKM, 128, 128, 64, 2, 0>(g, s);
  return launch_gated_tiles<DT, Args, BKM, 64, 128, 32, 3, 0>(g, s);
}

hipError_t run_gated_fwd_f16(const GemmArgs& g, int64_t pair, hipStream_t s);
hipError_t run_gated_fwd_bf16(const GemmArgs& g, int64_t pair, hipStream_t s);
hipError_t run_gated_bwd_f16(const GemmArgs& g, hipStream_t s);
hipError_t run_gated_bwd_bf16(const GemmArgs& g, hipStream_t s);

template <int DT, int ACT>
hipError_t run_gated_fwd(const GemmArgs& g, int64_t pair, hipStream_t s) {
  GatedArgs<ACT> a;
  static_cast<GemmArgs&>(a) = g;
  a.pair = pair;
  return launch_gated<DT, GatedArgs<ACT>, true>(a, s);
}
template <int DT, int ACT>
hipError_t run_gated_bwd(const GemmArgs& g, hipStream_t s) {
  GatedBwdArgs<ACT> a;
  static_cast<GemmArgs&>(a) = g;
  return launch_gated<DT, GatedBwdArgs<ACT>, false>(a, s);
}

}  // namespace mpx
