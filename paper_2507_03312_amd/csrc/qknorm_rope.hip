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

// A thread's run of both gains (ones where there is none).
template <int DT, int VW>
struct QkGains {
  RopeVec<DT, VW> w[2];
  __device__ __forceinline__ void load(const QkArgs& a, int v0) {
    typedef typename RopeValue<DT>::type T;
#pragma unroll
    for (int p = 0; p < 2; ++p) {
      const T* g = (const T*)(p ? a.wk : a.wq);
      if (g) {
        w[p].load(g + v0);
      } else {
#pragma unroll
        for (int i = 0; i < VW; ++i) w[p].set(i, 1.0f);
      }
    }
  }
  __device__ __forceinline__ float get(bool key, int i) const { return key ? w[1].get(i) : w[0].get(i); }
};

// Bound by HBM: every value is read and written once.  As rope_kernel: a row's turns once
// into LDS, a thread keeps one run of VW values of every head it takes, U heads in
// flight; the lanes of a head lie in one wave and share its sum of squares.  Queries, keys
// and (in runs of 16 bytes) the copied heads are one list, so that few heads of a kind
// leave no thread without one.  12608 rows of 3 x 12 heads of 64 bf16 29 us, 4.0 TB/s (a loop
// for each kind 31.5; the 116 MB at a large copy's rate 22.6).  NT: results past the last-level
// cache.
template <int DT, int VW, bool INTER, bool NT>
__global__ __launch_bounds__(256) void qknorm_rope_kernel(QkArgs a) {
  typedef typename RopeValue<DT>::type T;
  __shared__ float2 turns[kRopeTable];
  const uint32_t row0 = blockIdx.x * a.wg_rows;
  const T* X = (const T*)a.X + (int64_t)row0 * a.ldx;
  T* Y = (T*)a.Y + (int64_t)row0 * a.ldy;
  const uint32_t nrows = min((uint32_t)a.wg_rows, a.rows - row0);
  constexpr bool kWide = VW * sizeof(T) == 16;
  const int lane = threadIdx.x & 63;
  const uint32_t chunk = lane % a.chunks, wave_slots = 64 / a.chunks;
  const uint32_t slot = (threadIdx.x >> 6) * wave_slots + lane / a.chunks;
  const uint32_t r = slot / a.head_slots, h0 = slot % a.head_slots;
  const uint32_t heads = a.heads_rot + (kWide && !a.in_place ? a.copy / a.hd : 0);
  const bool mine = (uint32_t)lane < wave_slots * a.chunks && r < nrows;  // all lanes of a head or none
  const T* x = X + r * a.ldx + chunk * VW;
  T* y = Y + r * a.ldy + chunk * VW;
  // the first heads' values in flight while the turns are made
  constexpr int U = 4;
  RopeVec<DT, VW> v[U];
  auto load = [&](uint32_t h) {
#pragma unroll
    for (int u = 0; u < U; ++u) v[u].template load<NT>(x + (int64_t)min(h + u * a.head_slots, heads - 1) * a.hd);
  };
  if (mine) load(h0);
  if constexpr (!kWide) rope_copies<DT>(a, X, a.ldx, Y, nrows);
  rope_turns(a, row0, nrows, turns);
  if (!mine) return;
  QkRun<VW, INTER> run;
  run.init(a, chunk, lane);
  float c[VW], s[VW];
  run.factors(turns + r * a.npairs, c, s);
  QkGains<DT, VW> own, other;
  own.load(a, run.v0);
  if constexpr (!INTER) {
#pragma unroll
    for (int p = 0; p < 2; ++p) other.w[p] = own.w[p].from_lane(run.partner);
  }
  const float over = 1.0f / (float)a.hd;
  for (uint32_t h = h0; h < heads; h += U * a.head_slots) {
    float ss[U];
    if (h != h0) load(h);
#pragma unroll
    for (int u = 0; u < U; ++u) {
      ss[u] = 0.0f;
#pragma unroll
      for (int i = 0; i < VW; ++i) ss[u] = __builtin_fmaf(v[u].get(i), v[u].get(i), ss[u]);
    }
    head_sum<U>(ss, a.chunks, lane);
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const uint32_t at = h + u * a.head_slots;
      if (at >= heads) break;
      RopeVec<DT, VW> o;
      if constexpr (!INTER) o = v[u].from_lane(run.partner);
      if (!kWide || at < a.heads_rot) {
        const bool key = at >= a.hq;
        const float inv = rsqrtf(__builtin_fmaf(ss[u], over, a.eps));
        float n[VW];
#pragma unroll
        for (int i = 0; i < VW; ++i) {
          n[i] = v[u].get(i) * own.get(key, i) * c[i];
          if (run.turned) {  // values that are not turned keep clear of their neighbours
            if constexpr (INTER) n[i] = __builtin_fmaf(v[u].get(i ^ 1) * own.get(key, i ^ 1), s[i], n[i]);
            else n[i] = __builtin_fmaf(o.get(i) * other.get(key, i), s[i], n[i]);
          }
        }
#pragma unroll
        for (int i = 0; i < VW; ++i) v[u].set(i, inv * n[i]);
      }
      v[u].template store<NT>(y + (int64_t)at * a.hd);
    }
  }
}

// Backward, likewise, over a grid that strides over the rows.  A thread's sums of dw for its
// run of values stand in LDS (their 16 registers serve the loads in flight); a workgroup
// adds up its threads' in order, and qk_gains_kernel the workgroups'.  Bound by HBM as well:
// 29997 rows of 16 + 4 heads and 4 copied ones of 128 f16 113 to 119 us, 4.5 TB/s (sums in
// registers, no loads ahead: 185).  At four waves a SIMD four of the variants of 8 values
// (halves within the caches and, of bf16, past them; f16 interleaved within) spill 2 or 3 registers.
template <int DT, int VW, bool INTER, bool NT>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(4, 4)))
void qknorm_rope_bwd_kernel(QkArgs a) {
  typedef typename RopeValue<DT>::type T;
  __shared__ float2 turns[kRopeTable];
  __shared__ float sums[2][256 * VW];
  constexpr bool kWide = VW * sizeof(T) == 16;
  const int lane = threadIdx.x & 63;
  const uint32_t chunk = lane % a.chunks, wave_slots = 64 / a.chunks;
  const uint32_t slot = (threadIdx.x >> 6) * wave_slots + lane / a.chunks;
  const uint32_t r = slot / a.head_slots, h0 = slot % a.head_slots;
  const bool whole = (uint32_t)lane < wave_slots * a.chunks;
  QkRun<VW, INTER> run;
  run.init(a, chunk, lane);
  float* own = &sums[0][slot * a.hd + run.v0];
  QkGains<DT, VW> w;
  if (whole) {
    w.load(a, run.v0);
#pragma unroll
    for (int i = 0; i < VW; ++i) own[i] = own[256 * VW + i] = 0.0f;
  }
  const float over = 1.0f / (float)a.hd;
  const uint32_t heads = a.heads_rot + (kWide && !a.in_place ? a.copy / a.hd : 0);
  for (uint32_t tile = blockIdx.x; tile < a.tiles; tile += gridDim.x) {
    const uint32_t row0 = tile * a.wg_rows;
    const T* X = (const T*)a.X + (int64_t)row0 * a.ldx;
    const T* D = (const T*)a.dY + (int64_t)row0 * a.ldy_in;
    T* Y = (T*)a.Y + (int64_t)row0 * a.ldy;
    const uint32_t nrows = min((uint32_t)a.wg_rows, a.rows - row0);
    const bool mine = whole && r < nrows;
    const T* x = X + r * a.ldx + run.v0;
    const T* d = D + r * a.ldy_in + run.v0;
    T* y = Y + r * a.ldy + run.v0;
    // a head's values in flight while the one before is worked on, the first ones
    // while the turns are made
    RopeVec<DT, VW> nv, ng;
    auto load = [&](uint32_t h) {
      nv.template load<NT>(x + (int64_t)min(h, a.heads_rot - 1) * a.hd);  // X has no copied heads
      ng.template load<NT>(d + (int64_t)min(h, heads - 1) * a.hd);
    };
    if (mine) load(h0);
    __syncthreads();  // the last tile's turns have been read
    if constexpr (!kWide) rope_copies<DT>(a, D, a.ldy_in, Y, nrows);
    rope_turns(a, row0, nrows, turns);
    if (!mine) continue;
    float c[VW], s[VW];
    run.factors(turns + r * a.npairs, c, s);
    for (uint32_t h = h0; h < heads; h += a.head_slots) {
      const RopeVec<DT, VW> v = nv, g = ng;
      load(h + a.head_slots);
      const bool key = h >= a.hq;
      RopeVec<DT, VW> o;
      if constexpr (!INTER) o = g.from_lane(run.partner);
      float sum[2] = {0.0f, 0.0f}, dn[VW];
#pragma unroll
      for (int i = 0; i < VW; ++i) {
        const float other = INTER ? g.get(i ^ 1) : o.get(i);
        dn[i] = run.turned ? __builtin_fmaf(g.get(i), c[i], other * s[i]) : g.get(i);
        sum[0] = __builtin_fmaf(v.get(i), v.get(i), sum[0]);
        sum[1] = __builtin_fmaf(w.get(key, i) * dn[i], v.get(i), sum[1]);
      }
      head_sum<2>(sum, a.chunks, lane);
      RopeVec<DT, VW> out = g;
      if (!kWide || h < a.heads_rot) {
        const float inv = rsqrtf(__builtin_fmaf(sum[0], over, a.eps));
        const float k = inv * inv * (sum[1] * over);
        float* add = own + (key ? 256 * VW : 0);
#pragma unroll
        for (int i = 0; i < VW; ++i) {
          const float xi = v.get(i);
          add[i] = __builtin_fmaf(dn[i], xi * inv, add[i]);
          out.set(i, inv * __builtin_fmaf(-xi, k, w.get(key, i) * dn[i]));
        }
      }
      out.template store<NT>(y + (int64_t)h * a.hd);
    }
  }
  // the workgroup's sums: its slots in order
  __syncthreads();
  for (int j = threadIdx.x; j < 2 * a.hd; j += 256) {
    const int part = j >= a.hd ? 1 : 0, col = j - part * a.hd;
    float t = 0.0f;
    for (uint32_t k = 0; k < 4 * wave_slots; ++k) t += sums[part][k * a.hd + col];
    a.part[(int64_t)blockIdx.x * 2 * a.hd + j] = t;
  }
}

// Heads whose sections allow no such runs: a wave takes a head at a time, U heads in flight,
// lane l the values l, l + 64, ..., their partners straight from memory (the same lines).
// Bound by latency and narrow accesses: 6304 rows of 36 heads of 128 bf16, sections of 21 and
// 43, 65 us, backward 92 (one head in flight 113 and 157; whole runs 30 and 52).  PER: values
// of a lane.
template <int DT, bool BACK, int PER>
__global__ __launch_bounds__(256) void qknorm_rope_any_kernel(QkArgs a) {
  typedef typename RopeValue<DT>::type T;
  __shared__ float2 turns[kRopeTable];
  __shared__ float sums[4][64 * PER];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const float over = 1.0f / (float)a.hd;
  auto get = [](T v) { if constexpr (DT == MPX_F32) return v; else return h2f<DT>(v); };
  auto put = [](float v) { if constexpr (DT == MPX_F32) return v; else return f2h<DT>(v); };
  // the lane's values' pairs (-1: not turned) and partners
  int pair[PER], other[PER];
  bool second[PER];
  float dw[2][PER], gain[2][PER], gain_other[2][PER];
  constexpr int U = PER <= 2 ? 4 : PER == 4 ? 2 : 1;
#pragma unroll
  for (int i = 0; i < PER; ++i) {
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
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    const bool in = lane + 64 * i < a.hd;
#pragma unroll
    for (int part = 0; part < 2; ++part) {
      const T* g = (const T*)(part ? a.wk : a.wq);
      gain[part][i] = in && g ? get(g[lane + 64 * i]) : 1.0f;
      gain_other[part][i] = in && g ? get(g[other[i]]) : 1.0f;
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
    const uint32_t items = nrows * a.heads_rot;
    for (uint32_t item0 = wave; item0 < items; item0 += 4 * U) {
      float xv[U][PER], own[U][PER], oth[U][PER];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const uint32_t item = min(item0 + 4 * u, items - 1), r = item / a.heads_rot, h = item % a.heads_rot;
        const T* x = X + r * a.ldx + (int64_t)h * a.hd;
        const T* d = D + r * ldd + (int64_t)h * a.hd;
#pragma unroll
        for (int i = 0; i < PER; ++i) {
          const int j = lane + 64 * i;
          const bool in = j < a.hd;
          xv[u][i] = in ? get(x[j]) : 0.0f;
          if constexpr (BACK) own[u][i] = in ? get(d[j]) : 0.0f;
          else own[u][i] = xv[u][i];
          oth[u][i] = in ? get(d[other[i]]) : 0.0f;
        }
      }
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const uint32_t item = item0 + 4 * u, r = item / a.heads_rot, h = item % a.heads_rot;
        if (item >= items) break;  // uniform over the wave
        const int part = h >= a.hq ? 1 : 0;
        float ss = 0.0f, sp = 0.0f;
#pragma unroll
        for (int i = 0; i < PER; ++i) {
          const float w = part ? gain[1][i] : gain[0][i], wo = part ? gain_other[1][i] : gain_other[0][i];
          if (pair[i] >= 0) {
            float2 t = turns[r * a.npairs + pair[i]];
            if (!second[i]) t.y = -t.y;
            own[u][i] = BACK ? __builtin_fmaf(own[u][i], t.x, oth[u][i] * t.y)
                             : __builtin_fmaf(own[u][i], w * t.x, oth[u][i] * (wo * t.y));
          } else if (!BACK) {
            own[u][i] *= w;
          }
          ss = __builtin_fmaf(xv[u][i], xv[u][i], ss);
          if (BACK) {
            oth[u][i] = w * own[u][i];
            sp = __builtin_fmaf(oth[u][i], xv[u][i], sp);
          }
        }
        const float inv = rsqrtf(__builtin_fmaf(wave_sum(ss), over, a.eps));
        const float k = BACK ? inv * inv * (wave_sum(sp) * over) : 0.0f;
        T* y = Y + r * a.ldy + (int64_t)h * a.hd;
#pragma unroll
        for (int i = 0; i < PER; ++i) {
          const int j = lane + 64 * i;
          if (j >= a.hd) continue;
          if (BACK) {
            const float t = own[u][i] * (xv[u][i] * inv);
            dw[0][i] += part ? 0.0f : t;
            dw[1][i] += part ? t : 0.0f;
            y[j] = put(inv * __builtin_fmaf(-xv[u][i], k, oth[u][i]));
          } else {
            y[j] = put(inv * own[u][i]);
          }
        }
      }
    }
  }
  if constexpr (BACK) {
#pragma unroll
    for (int part = 0; part < 2; ++part) {
      __syncthreads();
#pragma unroll
      for (int i = 0; i < PER; ++i) sums[wave][lane + 64 * i] = dw[part][i];
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

template <int DT, int VW, bool INTER, bool NT>
static void launch_qk_kernel(const QkArgs& a, bool back, unsigned blocks, hipStream_t s) {
  if (back) qknorm_rope_bwd_kernel<DT, VW, INTER, NT><<<blocks, 256, 0, s>>>(a);
  else qknorm_rope_kernel<DT, VW, INTER, NT><<<blocks, 256, 0, s>>>(a);
}
template <int DT, int VW>
static void launch_qk(const QkArgs& a, bool back, unsigned blocks, hipStream_t s) {
  if constexpr (VW * sizeof(typename RopeValue<DT>::type) == 16) {
    if (a.stream) {
      if (a.interleaved) launch_qk_kernel<DT, VW, true, true>(a, back, blocks, s);
      else launch_qk_kernel<DT, VW, false, true>(a, back, blocks, s);
      return;
    }
  }
  if (a.interleaved) launch_qk_kernel<DT, VW, true, false>(a, back, blocks, s);
  else launch_qk_kernel<DT, VW, false, false>(a, back, blocks, s);
}

template <int DT, int PER>
static void launch_qk_any(const QkArgs& a, bool back, unsigned blocks, hipStream_t s) {
  if (back) qknorm_rope_any_kernel<DT, true, PER><<<blocks, 256, 0, s>>>(a);
  else qknorm_rope_any_kernel<DT, false, PER><<<blocks, 256, 0, s>>>(a);
}
template <int DT>
static void launch_qk_any(const QkArgs& a, bool back, unsigned blocks, hipStream_t s) {
  if (a.hd <= 64) launch_qk_any<DT, 1>(a, back, blocks, s);
  else if (a.hd <= 128) launch_qk_any<DT, 2>(a, back, blocks, s);
  else if (a.hd <= 256) launch_qk_any<DT, 4>(a, back, blocks, s);
  else launch_qk_any<DT, 8>(a, back, blocks, s);
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
  // past the last-level cache, around it
  const double values = (double)width * (in == Y ? 1.0 : 2.0) + (back ? (double)(heads_q + heads_k) * hd : 0.0);
  const double bytes = (double)rows * values * (dt == MPX_F32 ? 4.0 : 2.0);
  a.stream = bytes > 256.0 * (1 << 20) ? 1 : 0;
  const bool any = vw == 1 || hd / vw > 64;
  a.chunks = any ? 64 : (int32_t)(hd / vw);
  const int64_t slots = any ? 4 : 4 * (64 / a.chunks);
  const int64_t listed = a.heads_rot + (!any && !a.in_place && vw * (dt == MPX_F32 ? 4 : 2) == 16 ? heads_copy : 0);
  // a wave a head: forward small workgroups for whole rounds, backward one round of them
  int64_t wg_rows = any ? (back ? std::min<int64_t>(16, cdiv(rows, kQkWorkgroups)) : std::min<int64_t>(2, rows / 1024))
                        : std::min<int64_t>({8 * slots / listed, slots, rows / 1024});
  wg_rows = std::min<int64_t>(wg_rows, kRopeTable / a.npairs);
  wg_rows = std::max<int64_t>(wg_rows, 1);
  a.wg_rows = (int32_t)wg_rows;
  a.head_slots = (int32_t)std::max<int64_t>(1, slots / wg_rows);
  a.tiles = (uint32_t)cdiv(rows, wg_rows);
  const unsigned blocks = (unsigned)(back ? std::min<int64_t>(a.tiles, workgroups) : a.tiles);
#define MPX_QK(DTv, VWv) launch_qk<DTv, VWv>(a, back, blocks, s)
#define MPX_QK_ANY(DTv) launch_qk_any<DTv>(a, back, blocks, s)
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
    else if (dt == MPX_F16)
      qk_gains_kernel<MPX_F16><<<grid, 1024, 0, s>>>(a.part, (int)blocks, (int)hd, dwq, dwk, d_nonfinite);
    else
      qk_gains_kernel<MPX_BF16><<<grid, 1024, 0, s>>>(a.part, (int)blocks, (int)hd, dwq, dwk, d_nonfinite);
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
