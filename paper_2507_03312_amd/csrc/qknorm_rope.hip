// Norms of queries and keys for each head with the rotary positions in the same pass
// (mpx_qknorm_rope_fwd, mpx_qknorm_rope_bwd).  Per head x of hd values, with the gain w:
//   r = 1 / sqrt(mean(x^2) + eps),  n = x r w,  y = turn(n)
// backward, dn = turn^-1(dy):
//   dx = r (w dn - x r^2 mean(w dn x)),   dw = sum over rows and heads of dn x r
#include "rope.h"

namespace mpx {

struct QkArgs : RopeArgs {  // heads_rot: queries and keys together
  const void *dY, *wq, *wk;  // backward: X, dY in; Y is dX
  int64_t ldy_in;            // row stride of dY
  float* part;               // backward: [workgroup][2][hd] sums of dw
  float eps;
  uint32_t hq;
  uint32_t tiles;  // workgroups' worth of rows
};

// Sum over the lanes of a head: `n` neighbouring lanes, the first of them a multiple of
// n.  The same on every lane.  U values at once.
template <int U>
__device__ __forceinline__ void head_sum(float (&v)[U], int n, int lane) {
  auto add = [&](auto f) {
#pragma unroll
    for (int u = 0; u < U; ++u) v[u] += __builtin_bit_cast(float, f(__builtin_bit_cast(int, v[u])));
  };
  if ((n & (n - 1)) == 0) {  // uniform
    if (n >= 2) add([](int x) { return __builtin_amdgcn_mov_dpp(x, 0xB1, 0xF, 0xF, false); });    // lane ^ 1
    if (n >= 4) add([](int x) { return __builtin_amdgcn_mov_dpp(x, 0x4E, 0xF, 0xF, false); });    // lane ^ 2
    if (n >= 8) add([](int x) { return __builtin_amdgcn_mov_dpp(x, 0x141, 0xF, 0xF, false); });   // 7 - lane
    if (n >= 16) add([](int x) { return __builtin_amdgcn_mov_dpp(x, 0x140, 0xF, 0xF, false); });  // 15 - lane
    if (n >= 32) add([&](int x) { return __builtin_amdgcn_ds_bpermute(4 * (lane ^ 16), x); });
    if (n >= 64) add([&](int x) { return __builtin_amdgcn_ds_bpermute(4 * (lane ^ 32), x); });
    return;
  }
  const int i = lane % n;
  for (int s = 1; s < n; s *= 2)  // lane i: the sum of i .. i + 2 s - 1
    add([&](int x) {
      const int o = __builtin_amdgcn_ds_bpermute(4 * min(lane + s, 63), x);
      return i + s < n ? o : 0;
    });
#pragma unroll
  for (int u = 0; u < U; ++u)
    v[u] = __builtin_bit_cast(float, __builtin_amdgcn_ds_bpermute(4 * (lane - i), __builtin_bit_cast(int, v[u])));
}

// A thread's part in its heads: VW values from v0 on, their pairs' first turn p0 and the lane
// of their partners (halves; interleaved ones are its own).
template <int VW, bool INTER>
struct QkRun {
  int v0, p0, partner;
  bool turned, second;
  __device__ __forceinline__ void init(const RopeArgs& a, int chunk, int lane) {
    v0 = chunk * VW;
    turned = v0 < 2 * a.npairs;
    p0 = v0 / 2;
    partner = lane;
    second = false;
    if (!INTER && turned) {
      int first = 0, n = a.first_pair[1];
#pragma unroll
      for (int k = 1; k < MPX_ROPE_MAX_AXES; ++k) {
        if (v0 >= 2 * a.first_pair[k]) {
          first = a.first_pair[k];
          n = a.first_pair[k + 1] - first;
        }
      }
      second = v0 - 2 * first >= n;
      p0 = v0 - first - (second ? n : 0);
      partner = lane + (second ? -n : n) / VW;
    }
  }
  // y_i = own_i c_i + other_i s_i for a row's turns: the sign is in s
  __device__ __forceinline__ void factors(const float2* t, float (&c)[VW], float (&s)[VW]) const {
#pragma unroll
    for (int i = 0; i < VW; ++i) {
      const float2 f = turned ? t[p0 + (INTER ? i / 2 : i)] : make_float2(1.0f, 0.0f);
      c[i] = f.x;
      s[i] = (INTER ? (i & 1) != 0 : second) ? f.y : -f.y;
    }
  }
};

// The values' partners, and those of a gain in registers.
template <int VW, bool INTER>
__device__ __forceinline__ void partners(const float (&x)[VW], int lane, float (&o)[VW]) {
#pragma unroll
  for (int i = 0; i < VW; ++i) {
    if constexpr (INTER) o[i] = x[i ^ 1];
    else o[i] = __builtin_bit_cast(float, __builtin_amdgcn_ds_bpermute(4 * lane, __builtin_bit_cast(int, x[i])));
  }
}

// Bound by HBM: every value is read and written once.  As rope_kernel: a row's turns once
// into LDS, a thread keeps one run of VW values of every head it takes, U heads in
// flight; the lanes of a head lie in one wave and share its sum of squares.
template <int DT, int VW, bool INTER>
__global__ __launch_bounds__(256) void qknorm_rope_kernel(QkArgs a) {
  typedef typename RopeValue<DT>::type T;
  __shared__ float2 turns[kRopeTable];
  const uint32_t row0 = blockIdx.x * a.wg_rows;
  const T* X = (const T*)a.X + (int64_t)row0 * a.ldx;
  T* Y = (T*)a.Y + (int64_t)row0 * a.ldy;
  const uint32_t nrows = min((uint32_t)a.wg_rows, a.rows - row0);
  rope_copies<DT>(a, X, a.ldx, Y, nrows);
  rope_turns(a, row0, nrows, turns);

  const int lane = threadIdx.x & 63;
  const uint32_t chunk = lane % a.chunks, wave_slots = 64 / a.chunks;
  const uint32_t slot = (threadIdx.x >> 6) * wave_slots + lane / a.chunks;
  const uint32_t r = slot / a.head_slots, h0 = slot % a.head_slots;
  if ((uint32_t)lane >= wave_slots * a.chunks || r >= nrows) return;  // all lanes of a head or none
  QkRun<VW, INTER> run;
  run.init(a, chunk, lane);
  float c[VW], s[VW];
  run.factors(turns + r * a.npairs, c, s);
  const T* x = X + r * a.ldx + run.v0;
  T* y = Y + r * a.ldy + run.v0;
  const float over = 1.0f / (float)a.hd;
  constexpr int U = 4;
  for (int part = 0; part < 2; ++part) {  // queries, keys
    const uint32_t lo = part ? a.hq : 0, hi = part ? a.heads_rot : a.hq;
    float wc[VW], ws[VW];  // the gains times the turn
    {
      RopeVec<DT, VW> w;
      float f[VW], o[VW];
      const T* g = (const T*)(part ? a.wk : a.wq);
      if (g) w.load(g + run.v0);
#pragma unroll
      for (int i = 0; i < VW; ++i) f[i] = g ? w.get(i) : 1.0f;
      partners<VW, INTER>(f, run.partner, o);
#pragma unroll
      for (int i = 0; i < VW; ++i) {
        wc[i] = f[i] * c[i];
        ws[i] = o[i] * s[i];
      }
    }
    for (uint32_t h = lo + h0; h < hi; h += U * a.head_slots) {
      RopeVec<DT, VW> v[U];
      float ss[U];
#pragma unroll
      for (int u = 0; u < U; ++u) v[u].load(x + (int64_t)min(h + u * a.head_slots, hi - 1) * a.hd);
#pragma unroll
      for (int u = 0; u < U; ++u) {
        ss[u] = 0.0f;
#pragma unroll
        for (int i = 0; i < VW; ++i) ss[u] = __builtin_fmaf(v[u].get(i), v[u].get(i), ss[u]);
      }
      head_sum<U>(ss, a.chunks, lane);
#pragma unroll
      for (int u = 0; u < U; ++u) {
        RopeVec<DT, VW> o;
        if constexpr (!INTER) o = v[u].from_lane(run.partner);
        if (h + u * a.head_slots >= hi) break;
        const float inv = rsqrtf(__builtin_fmaf(ss[u], over, a.eps));
        RopeVec<DT, VW> n;
#pragma unroll
        for (int i = 0; i < VW; ++i) {
          const float other = INTER ? v[u].get(i ^ 1) : o.get(i);
          // values that are not turned keep clear of their neighbours
          n.set(i, inv * (run.turned ? __builtin_fmaf(v[u].get(i), wc[i], other * ws[i]) : v[u].get(i) * wc[i]));
        }
        n.store(y + (int64_t)(h + u * a.head_slots) * a.hd);
      }
    }
  }
}

// Backward, likewise, over a grid that strides over the rows: a thread adds up dw for its own
// run of values, a workgroup its threads' sums in order, and qk_gains_kernel the
// workgroups'.
template <int DT, int VW, bool INTER>
__global__ __launch_bounds__(256) void qknorm_rope_bwd_kernel(QkArgs a) {
  typedef typename RopeValue<DT>::type T;
  __shared__ float2 turns[kRopeTable];
  __shared__ float sums[256 * VW];
  const int lane = threadIdx.x & 63;
  const uint32_t chunk = lane % a.chunks, wave_slots = 64 / a.chunks;
  const uint32_t slot = (threadIdx.x >> 6) * wave_slots + lane / a.chunks;
  const uint32_t r = slot / a.head_slots, h0 = slot % a.head_slots;
  const bool whole = (uint32_t)lane < wave_slots * a.chunks;
  QkRun<VW, INTER> run;
  run.init(a, chunk, lane);
  const float over = 1.0f / (float)a.hd;
  float dw[2][VW] = {};
  for (uint32_t tile = blockIdx.x; tile < a.tiles; tile += gridDim.x) {
    const uint32_t row0 = tile * a.wg_rows;
    const T* X = (const T*)a.X + (int64_t)row0 * a.ldx;
    const T* D = (const T*)a.dY + (int64_t)row0 * a.ldy_in;
    T* Y = (T*)a.Y + (int64_t)row0 * a.ldy;
    const uint32_t nrows = min((uint32_t)a.wg_rows, a.rows - row0);
    __syncthreads();  // the last tile's turns have been read
    rope_copies<DT>(a, D, a.ldy_in, Y, nrows);
    rope_turns(a, row0, nrows, turns);
    if (!whole || r >= nrows) continue;
    float c[VW], s[VW];
    run.factors(turns + r * a.npairs, c, s);
    const T* x = X + r * a.ldx + run.v0;
    const T* d = D + r * a.ldy_in + run.v0;
    T* y = Y + r * a.ldy + run.v0;
    constexpr int U = 2;
#pragma unroll
    for (int part = 0; part < 2; ++part) {
      const uint32_t lo = part ? a.hq : 0, hi = part ? a.heads_rot : a.hq;
      float w[VW];
      {
        RopeVec<DT, VW> g;
        const T* p = (const T*)(part ? a.wk : a.wq);
        if (p) g.load(p + run.v0);
#pragma unroll
        for (int i = 0; i < VW; ++i) w[i] = p ? g.get(i) : 1.0f;
      }
      for (uint32_t h = lo + h0; h < hi; h += U * a.head_slots) {
        RopeVec<DT, VW> v[U], g[U];
        float sum[2 * U], dn[U][VW];
#pragma unroll
        for (int u = 0; u < U; ++u) {
          const int64_t at = (int64_t)min(h + u * a.head_slots, hi - 1) * a.hd;
          v[u].load(x + at);
          g[u].load(d + at);
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
          RopeVec<DT, VW> o;
          if constexpr (!INTER) o = g[u].from_lane(run.partner);
          sum[2 * u] = sum[2 * u + 1] = 0.0f;
#pragma unroll
          for (int i = 0; i < VW; ++i) {
            const float other = INTER ? g[u].get(i ^ 1) : o.get(i);
            dn[u][i] = run.turned ? __builtin_fmaf(g[u].get(i), c[i], other * s[i]) : g[u].get(i);
            sum[2 * u] = __builtin_fmaf(v[u].get(i), v[u].get(i), sum[2 * u]);
            sum[2 * u + 1] = __builtin_fmaf(w[i] * dn[u][i], v[u].get(i), sum[2 * u + 1]);
          }
        }
        head_sum<2 * U>(sum, a.chunks, lane);
#pragma unroll
        for (int u = 0; u < U; ++u) {
          if (h + u * a.head_slots >= hi) break;
          const float inv = rsqrtf(__builtin_fmaf(sum[2 * u], over, a.eps));
          const float k = inv * inv * (sum[2 * u + 1] * over);
          RopeVec<DT, VW> n;
#pragma unroll
          for (int i = 0; i < VW; ++i) {
            const float xi = v[u].get(i);
            dw[part][i] = __builtin_fmaf(dn[u][i], xi * inv, dw[part][i]);
            n.set(i, inv * __builtin_fmaf(-xi, k, w[i] * dn[u][i]));
          }
          n.store(y + (int64_t)(h + u * a.head_slots) * a.hd);
        }
      }
    }
  }
  // the workgroup's sums: its slots in order
#pragma unroll
  for (int part = 0; part < 2; ++part) {
    __syncthreads();
    if (whole) {
#pragma unroll
      for (int i = 0; i < VW; ++i) sums[slot * a.hd + run.v0 + i] = dw[part][i];
    }
    __syncthreads();
    for (int j = threadIdx.x; j < a.hd; j += 256) {
      float t = 0.0f;
      for (uint32_t k = 0; k < 4 * wave_slots; ++k) t += sums[k * a.hd + j];
      a.part[((int64_t)blockIdx.x * 2 + part) * a.hd + j] = t;
    }
  }
}

// Heads whose sections allow no such runs: a wave takes a head at a time, lane l the values
// l, l + 64, ..., their partners straight from memory (the same lines).
constexpr int kQkPer = kRopeMaxHd / 64;
template <int DT, bool BACK>
__global__ __launch_bounds__(256) void qknorm_rope_any_kernel(QkArgs a) {
  typedef typename RopeValue<DT>::type T;
  __shared__ float2 turns[kRopeTable];
  __shared__ float sums[4][kRopeMaxHd];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const float over = 1.0f / (float)a.hd;
  auto get = [](T v) { if constexpr (DT == MPX_F32) return v; else return h2f<DT>(v); };
  auto put = [](float v) { if constexpr (DT == MPX_F32) return v; else return f2h<DT>(v); };
  // the lane's values' pairs (-1: not turned) and partners
  int pair[kQkPer], other[kQkPer];
  bool second[kQkPer];
  float dw[2][kQkPer];
#pragma unroll
  for (int i = 0; i < kQkPer; ++i) {
    const int j = lane + 64 * i;
    pair[i] = -1;
    other[i] = j;
    second[i] = false;
    dw[0][i] = dw[1][i] = 0.0f;
    if (j < 2 * a.npairs) {
      if (a.interleaved) {
        pair[i] = j / 2;
        other[i] = j ^ 1;
        second[i] = j & 1;
      } else {
        int first = 0, n = a.first_pair[1];
#pragma unroll
        for (int k = 1; k < MPX_ROPE_MAX_AXES; ++k) {
          if (j >= 2 * a.first_pair[k]) {
            first = a.first_pair[k];
            n = a.first_pair[k + 1] - first;
          }
        }
        second[i] = j - 2 * first >= n;
        pair[i] = j - first - (second[i] ? n : 0);
        other[i] = j + (second[i] ? -n : n);
      }
    }
  }
  for (uint32_t tile = blockIdx.x; tile < a.tiles; tile += gridDim.x) {
    const uint32_t row0 = tile * a.wg_rows, nrows = min((uint32_t)a.wg_rows, a.rows - row0);
    const T* X = (const T*)a.X + (int64_t)row0 * a.ldx;
    const T* D = BACK ? (const T*)a.dY + (int64_t)row0 * a.ldy_in : X;
    const int64_t ldd = BACK ? a.ldy_in : a.ldx;
    T* Y = (T*)a.Y + (int64_t)row0 * a.ldy;
    __syncthreads();
    rope_copies<DT>(a, D, ldd, Y, nrows);
    rope_turns(a, row0, nrows, turns);
    for (uint32_t item = wave; item < nrows * a.heads_rot; item += 4) {
      const uint32_t r = item / a.heads_rot, h = item % a.heads_rot;
      const T* x = X + r * a.ldx + (int64_t)h * a.hd;
      const T* d = D + r * ldd + (int64_t)h * a.hd;
      T* y = Y + r * a.ldy + (int64_t)h * a.hd;
      const int part = h >= a.hq ? 1 : 0;
      const T* g = (const T*)(part ? a.wk : a.wq);
      float xv[kQkPer], own[kQkPer], oth[kQkPer], ss = 0.0f, sp = 0.0f;
#pragma unroll
      for (int i = 0; i < kQkPer; ++i) {
        const int j = lane + 64 * i;
        const bool in = j < a.hd;
        xv[i] = in ? get(x[j]) : 0.0f;
        const float w = in && g ? get(g[j]) : 1.0f, wo = in && g ? get(g[other[i]]) : 1.0f;
        own[i] = in ? get(d[j]) : 0.0f;
        oth[i] = in ? get(d[other[i]]) : 0.0f;
        if (pair[i] >= 0) {
          float2 t = turns[r * a.npairs + pair[i]];
          if (!second[i]) t.y = -t.y;
          own[i] = BACK ? __builtin_fmaf(own[i], t.x, oth[i] * t.y)
                        : __builtin_fmaf(own[i], w * t.x, oth[i] * (wo * t.y));
        } else if (!BACK) {
          own[i] *= w;
        }
        ss = __builtin_fmaf(xv[i], xv[i], ss);
        if (BACK) {
          oth[i] = w * own[i];
          sp = __builtin_fmaf(oth[i], xv[i], sp);
        }
      }
      const float inv = rsqrtf(__builtin_fmaf(wave_sum(ss), over, a.eps));
      const float k = BACK ? inv * inv * (wave_sum(sp) * over) : 0.0f;
#pragma unroll
      for (int i = 0; i < kQkPer; ++i) {
        const int j = lane + 64 * i;
        if (j >= a.hd) continue;
        if (BACK) {
          const float t = own[i] * (xv[i] * inv);
          dw[0][i] += part ? 0.0f : t;
          dw[1][i] += part ? t : 0.0f;
          y[j] = put(inv * __builtin_fmaf(-xv[i], k, oth[i]));
        } else {
          y[j] = put(inv * own[i]);
        }
      }
    }
  }
  if constexpr (BACK) {
#pragma unroll
    for (int part = 0; part < 2; ++part) {
      __syncthreads();
#pragma unroll
      for (int i = 0; i < kQkPer; ++i) sums[wave][lane + 64 * i] = dw[part][i];
      __syncthreads();
      for (int j = threadIdx.x; j < a.hd; j += 256)
        a.part[((int64_t)blockIdx.x * 2 + part) * a.hd + j] = (sums[0][j] + sums[1][j]) + (sums[2][j] + sums[3][j]);
    }
  }
}

// dw: 16 columns a workgroup, 64 threads to each, the workgroups' sums in a fixed order.
template <int DT>
__global__ __launch_bounds__(1024) void qk_gains_kernel(const float* part, int parts, int hd, void* dwq, void* dwk,
                                                        int32_t* nonfinite) {
  typedef typename RopeValue<DT>::type T;
  __shared__ float lds[64][17];
  const int c = threadIdx.x % 16, g = threadIdx.x / 16, col = blockIdx.x * 16 + c;  // of [dwq | dwk]
  float s = 0.0f;
  if (col < 2 * hd)
    for (int p = g; p < parts; p += 64) s += part[(int64_t)p * 2 * hd + col];
  lds[g][c] = s;
  for (int h = 32; h >= 1; h /= 2) {
    __syncthreads();
    if (g < h) lds[g][c] += lds[g + h][c];
  }
  if (g != 0 || col >= 2 * hd) return;
  T* out = (T*)(col < hd ? dwq : dwk);
  if (!out) return;
  if constexpr (DT == MPX_F32) {
    out[col % hd] = lds[0][c];
  } else {
    const uint16_t v = f2h<DT>(lds[0][c]);
    out[col % hd] = v;
    if (nonfinite) add_nonfinite(nonfinite, h_nonfinite<DT>(v) ? 1 : 0);
  }
}

constexpr int64_t kQkWorkgroups = 1024;  // of the backward

template <int DT, int VW>
static void launch_qk(const QkArgs& a, bool back, unsigned blocks, hipStream_t s) {
  if (back) {
    if (a.interleaved) qknorm_rope_bwd_kernel<DT, VW, true><<<blocks, 256, 0, s>>>(a);
    else qknorm_rope_bwd_kernel<DT, VW, false><<<blocks, 256, 0, s>>>(a);
  } else {
    if (a.interleaved) qknorm_rope_kernel<DT, VW, true><<<blocks, 256, 0, s>>>(a);
    else qknorm_rope_kernel<DT, VW, false><<<blocks, 256, 0, s>>>(a);
  }
}

static int64_t qk_workgroups(int64_t rows) { return std::min(rows, kQkWorkgroups); }

static int qknorm_rope(const char* fn, const void* X, int64_t ldx, const void* dY, int64_t ldy_in, void* Y,
                       int64_t ldy, const void* wq, const void* wk, double eps, const float* pos, int64_t pos_rows,
                       int64_t rows, int64_t heads_q, int64_t heads_k, int64_t heads_copy, int64_t hd,
                       const mpx_rope_plan* plan, void* dwq, void* dwk, mpx_dtype dt, void* workspace,
                       size_t ws_bytes, int32_t* d_nonfinite, bool back, void* stream) {
#define MPX_REQUIRE_FN(cond, msg)                       \
  do {                                                  \
    if (!(cond)) {                                      \
      set_error(std::string(fn) + ": " + (msg));        \
      return MPX_ERR_INVALID;                           \
    }                                                   \
  } while (0)
  MPX_REQUIRE_FN(X && Y && pos && plan && (!back || dY), "NULL operand");
  MPX_REQUIRE_FN(is_half(dt) || dt == MPX_F32, "dt must be MPX_F16, MPX_BF16 or MPX_F32");
  MPX_REQUIRE_FN(rows >= 1 && pos_rows >= 1 && rows % pos_rows == 0,
                 "rows must be a positive multiple of pos_rows");
  MPX_REQUIRE_FN(rows < ((int64_t)1 << 24), "too many rows for one call");
  MPX_REQUIRE_FN(hd >= 2 && hd <= kRopeMaxHd, "hd must be in [2, 512]");
  const int64_t most = (int64_t)1 << 20;
  MPX_REQUIRE_FN(heads_q >= 1 && heads_q <= most && heads_k >= 0 && heads_k <= most && heads_copy >= 0 &&
                     heads_copy <= most,
                 "heads_q must be >= 1, heads_k and heads_copy >= 0, at most 2^20 each");
  const int64_t width = (heads_q + heads_k + heads_copy) * hd;
  MPX_REQUIRE_FN(ldx >= (back ? (heads_q + heads_k) * hd : width) && ldy >= width && (!back || ldy_in >= width),
                 "row stride below the heads' width");
  const void* in = back ? dY : X;
  MPX_REQUIRE_FN(in != Y || (back ? ldy_in : ldx) == ldy, "in place needs equal row strides");
  MPX_REQUIRE_FN(!back || X != Y, "dX must not be X");
  MPX_REQUIRE_FN(eps >= 0.0 && std::isfinite(eps), "eps must be finite and >= 0");
  MPX_REQUIRE_FN(!d_nonfinite || dt != MPX_F32, "d_nonfinite is counted for half gradients only");
  const int64_t mis = reinterpret_cast<uintptr_t>(X) | reinterpret_cast<uintptr_t>(Y) |
                      reinterpret_cast<uintptr_t>(dY) | reinterpret_cast<uintptr_t>(wq) |
                      reinterpret_cast<uintptr_t>(wk) | reinterpret_cast<uintptr_t>(dwq) |
                      reinterpret_cast<uintptr_t>(dwk);
  MPX_REQUIRE_FN(mis % (dt == MPX_F32 ? 4 : 2) == 0 && reinterpret_cast<uintptr_t>(pos) % 4 == 0,
                 "pointers must be aligned to their element");
  QkArgs a{};
  int vw, vp;
  if (const char* why = rope_plan(plan, hd, dt, a, vw, vp)) MPX_REQUIRE_FN(false, why);
#undef MPX_REQUIRE_FN
  const int64_t workgroups = qk_workgroups(rows);
  if (back) {
    const size_t need = mpx_qknorm_rope_bwd_workspace(rows, hd);
    if (!workspace || ws_bytes < need || reinterpret_cast<uintptr_t>(workspace) % 4 != 0) {
      set_error(std::string(fn) + ": workspace of " + std::to_string(need) + " bytes, 4-byte aligned, required");
      return MPX_ERR_WORKSPACE;
    }
  }
  a.X = X;
  a.Y = Y;
  a.dY = dY;
  a.wq = wq;
  a.wk = wk;
  a.pos = pos;
  a.ldx = ldx;
  a.ldy = ldy;
  a.ldy_in = ldy_in;
  a.hq = (uint32_t)heads_q;
  a.heads_rot = (uint32_t)(heads_q + heads_k);
  a.copy = (uint32_t)(heads_copy * hd);
  a.back = back ? 1 : 0;
  a.in_place = in == Y ? 1 : 0;
  a.rows = (uint32_t)rows;
  a.pos_rows = (uint32_t)pos_rows;
  a.part = (float*)workspace;
  a.eps = (float)eps;
  hipStream_t s = (hipStream_t)stream;
  const bool any = vw == 1 || hd / vw > 64;
  a.chunks = any ? 64 : (int32_t)(hd / vw);
  const int64_t slots = any ? 4 : 4 * (64 / a.chunks);
  int64_t wg_rows = std::min<int64_t>({4 * slots / a.heads_rot, slots, kRopeTable / a.npairs, rows / 1024});
  wg_rows = std::max<int64_t>(wg_rows, 1);
  a.wg_rows = (int32_t)wg_rows;
  a.head_slots = (int32_t)(slots / wg_rows);
  a.tiles = (uint32_t)cdiv(rows, wg_rows);
  const unsigned blocks = (unsigned)(back ? std::min<int64_t>(a.tiles, workgroups) : a.tiles);
#define MPX_QK(DTv, VWv) launch_qk<DTv, VWv>(a, back, blocks, s)
#define MPX_QK_ANY(DTv)                                                        \
  do {                                                                         \
    if (back) qknorm_rope_any_kernel<DTv, true><<<blocks, 256, 0, s>>>(a);     \
    else qknorm_rope_any_kernel<DTv, false><<<blocks, 256, 0, s>>>(a);         \
  } while (0)
  if (dt == MPX_F32) {
    if (any) MPX_QK_ANY(MPX_F32);
    else if (vw == 4) MPX_QK(MPX_F32, 4);
    else MPX_QK(MPX_F32, 2);
  } else if (dt == MPX_F16) {
    if (any) MPX_QK_ANY(MPX_F16);
    else if (vw == 8) MPX_QK(MPX_F16, 8);
    else if (vw == 4) MPX_QK(MPX_F16, 4);
    else MPX_QK(MPX_F16, 2);
  } else {
    if (any) MPX_QK_ANY(MPX_BF16);
    else if (vw == 8) MPX_QK(MPX_BF16, 8);
    else if (vw == 4) MPX_QK(MPX_BF16, 4);
    else MPX_QK(MPX_BF16, 2);
  }
#undef MPX_QK
#undef MPX_QK_ANY
  MPX_LAUNCHED();
  if (back && (dwq || dwk)) {
    const unsigned grid = (unsigned)cdiv(2 * hd, 16);
    if (dt == MPX_F32) qk_gains_kernel<MPX_F32><<<grid, 1024, 0, s>>>(a.part, (int)blocks, (int)hd, dwq, dwk, nullptr);
    else if (dt == MPX_F16) qk_gains_kernel<MPX_F16><<<grid, 1024, 0, s>>>(a.part, (int)blocks, (int)hd, dwq, dwk, d_nonfinite);
    else qk_gains_kernel<MPX_BF16><<<grid, 1024, 0, s>>>(a.part, (int)blocks, (int)hd, dwq, dwk, d_nonfinite);
    MPX_LAUNCHED();
  }
  return MPX_OK;
}

}  // namespace mpx

extern "C" int mpx_qknorm_rope_fwd(const void* X, int64_t ldx, void* Y, int64_t ldy, const void* wq, const void* wk,
                                   double eps, const float* pos, int64_t pos_rows, int64_t rows, int64_t heads_q,
                                   int64_t heads_k, int64_t heads_copy, int64_t hd, const mpx_rope_plan* plan,
                                   mpx_dtype dt, void* stream) {
  mpx::clear_error();
  return mpx::qknorm_rope("mpx_qknorm_rope_fwd", X, ldx, nullptr, 0, Y, ldy, wq, wk, eps, pos, pos_rows, rows,
                          heads_q, heads_k, heads_copy, hd, plan, nullptr, nullptr, dt, nullptr, 0, nullptr, false,
                          stream);
}

extern "C" size_t mpx_qknorm_rope_bwd_workspace(int64_t rows, int64_t hd) {
  if (rows < 1 || hd < 1) return 0;
  return (size_t)mpx::qk_workgroups(rows) * 2 * hd * sizeof(float);
}

extern "C" int mpx_qknorm_rope_bwd(const void* X, int64_t ldx, const void* dY, int64_t ldy, void* dX, int64_t ldo,
                                   const void* wq, const void* wk, double eps, const float* pos, int64_t pos_rows,
                                   int64_t rows, int64_t heads_q, int64_t heads_k, int64_t heads_copy, int64_t hd,
                                   const mpx_rope_plan* plan, void* dwq, void* dwk, mpx_dtype dt, void* workspace,
                                   size_t ws_bytes, int32_t* d_nonfinite, void* stream) {
  mpx::clear_error();
  return mpx::qknorm_rope("mpx_qknorm_rope_bwd", X, ldx, dY, ldy, dX, ldo, wq, wk, eps, pos, pos_rows, rows, heads_q,
                          heads_k, heads_copy, hd, plan, dwq, dwk, dt, workspace, ws_bytes, d_nonfinite, true,
                          stream);
}
