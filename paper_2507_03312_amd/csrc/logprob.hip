// Log probabilities of given tokens with entropy and top alternatives, and the
// gradient at the logits (mpx_logprob_fwd, mpx_logprob_bwd).
#include <hip/hip_runtime.h>

#include <algorithm>
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

// 16 bytes of a row at any alignment of its elements (global accesses need none
// on gfx950), and the VE logits in them.
typedef uint32_t lp_u32x4 __attribute__((ext_vector_type(4)));
typedef lp_u32x4 lp_u32x4_any __attribute__((aligned(2)));
// Operands past the 256 MB last-level cache stream past it (the choice is the
// caller's, by their size: kStreamBytes).
template <bool NT>
__device__ __forceinline__ lp_u32x4 lp_load(const void* p) {
  const lp_u32x4_any* q = reinterpret_cast<const lp_u32x4_any*>(p);
  if constexpr (NT) return __builtin_nontemporal_load(q);
  else return *q;
}
template <bool NT>
__device__ __forceinline__ void lp_store(void* p, lp_u32x4 v) {
  lp_u32x4_any* q = reinterpret_cast<lp_u32x4_any*>(p);
  if constexpr (NT) __builtin_nontemporal_store(v, q);
  else *q = v;
}
template <int DT> constexpr int kVec = DT == MPX_F32 ? 4 : 8;

template <int DT>
__device__ __forceinline__ void lp_unpack(lp_u32x4 u, float (&x)[kVec<DT>]) {
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    if constexpr (DT == MPX_F32) {
      x[j] = __builtin_bit_cast(float, (uint32_t)u[j]);
    } else {
      x[2 * j] = h2f<DT>((uint16_t)(u[j] & 0xFFFFu));
      x[2 * j + 1] = h2f<DT>((uint16_t)(u[j] >> 16));
    }
  }
}

// The first n (0 .. VE - 1) of a lane's logits one by one, the rest masked.
template <int DT>
__device__ __forceinline__ void lp_load_tail(const typename LogitOf<DT>::type* z, int n, float (&x)[kVec<DT>]) {
#pragma unroll
  for (int e = 0; e < kVec<DT>; ++e) x[e] = e < n ? logit<DT>(z + e) : -INFINITY;
}

// Order of the alternatives as unsigned integers: by value, -0 as 0, NaN above
// all.  0 is below every logit and marks an empty place.
__device__ __forceinline__ uint32_t rank_of(float v) {
  const uint32_t b = __builtin_bit_cast(uint32_t, v + 0.0f);
  return v != v ? 0xFFFFFFFFu : (b & 0x80000000u) ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float rank_value(uint32_t o) {
  return __builtin_bit_cast(float, o == 0xFFFFFFFFu ? 0x7FC00000u : (o & 0x80000000u) ? o & 0x7FFFFFFFu : ~o);
}

constexpr float kLog2e = 1.4426950408889634f;
// differences below -200 are taken as -200: their exponential is 0 in float32,
// and a product with it stays 0 (0 * -inf would not)
constexpr float kFar = -200.0f;
__device__ __forceinline__ float lp_exp(float d) { return __builtin_amdgcn_exp2f(d * kLog2e); }

// Sum S of e^(z - m) and W of e^(z - m) (z - m) over some logits, m their
// largest.  Two of them are joined by moving both to the larger m: with
// f = e^(m - m'), S' = f S and W' = f (W + (m - m') S).
struct Moments {
  float m, s, w;
  __device__ __forceinline__ void move(float to) {
    const float del = m == -INFINITY ? kFar : fmaxf(m - to, kFar);  // -inf: S = W = 0 (or NaN)
    const float f = lp_exp(del);
    w = f * __builtin_fmaf(del, s, w);
    s *= f;
    m = to;
  }
};

// The k best logits a wave has seen, as keys that order them: rank above, the
// complement of the column below, so the lower column is the greater key and no
// two are equal; 0 is below every key.  Candidates are appended to a buffer in
// LDS, 64 lanes at once; when there are 2 k (and at the end) they are put in
// order, each key counting those above it, and all but k dropped.  (A list in
// order at all times, an insertion per candidate: 4096 x 65536 bf16 with k = 16
// 201 us against 102 without alternatives, 8 x 131072 with k = 8 19 against 5.5.)
constexpr int kBestCap = 128;
struct BestK {
  uint64_t* buf;  // [kBestCap], the wave's own
  int k, lane, count = 0;
  uint64_t lim = 0;    // candidates exceed it: the k-th best key at the last ordering, or a bound below it
  float thr_f = NAN;   // what a later column's logit must exceed; NaN: nothing is known yet

  __device__ __forceinline__ static uint64_t key(uint32_t o, uint32_t col) { return ((uint64_t)o << 32) | (uint32_t)~col; }

  // A bound from the lanes' own best ranks (0: none): the k-th largest of them is
  // not above the k-th largest of all.  Its upper 16 bits, found bit by bit, do.
  __device__ __forceinline__ void bound(uint32_t om) {
    uint32_t t = 0;
    for (int b = 31; b >= 16; --b) {
      const uint32_t c = t | (1u << b);
      if (__builtin_popcountll(__builtin_amdgcn_ballot_w64(om >= c)) >= k) t = c;
    }
    if (t) {
      lim = ((uint64_t)t << 32) - 1;
      thr_f = rank_value(t - 2);  // a value below the bound's (t - 1 may be -0, which 0 does not exceed)
    }
  }
  // Lanes read what others of their wave wrote.  LDS serves a wave in order; this
  // keeps the compiler from moving such accesses across each other (no instruction).
  __device__ __forceinline__ static void in_order() { __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront", "local"); }
  // one key per lane (0: none)
  __device__ __forceinline__ void offer(uint64_t key) {
    const uint64_t mask = __builtin_amdgcn_ballot_w64(key > lim);
    if (!mask) return;
    if (count > kBestCap - 64) {
      order();
      offer_in(key, __builtin_amdgcn_ballot_w64(key > lim));
    } else {
      offer_in(key, mask);
    }
  }
  __device__ __forceinline__ void offer_in(uint64_t key, uint64_t mask) {
    const int at = count + (int)__builtin_amdgcn_mbcnt_hi((uint32_t)(mask >> 32),
                                                          __builtin_amdgcn_mbcnt_lo((uint32_t)mask, 0));
    if (mask >> lane & 1) buf[at] = key;
    count += __builtin_popcountll(mask);
  }
  // puts the buffer in falling order, drops all but k; places without a key hold 0
  __device__ __forceinline__ void order() {
    in_order();
    const uint64_t a = lane < count ? buf[lane] : 0, b = 64 + lane < count ? buf[64 + lane] : 0;
    int ra = 0, rb = 0;
#pragma unroll 4
    for (int j = 0; j < count; ++j) ra += buf[j] > a ? 1 : 0;
    if (count > 64) {
#pragma unroll 4
      for (int j = 0; j < count; ++j) rb += buf[j] > b ? 1 : 0;
    }
    in_order();
    if (lane < k) buf[lane] = 0;
    in_order();
    if (a && ra < k) buf[ra] = a;
    if (b && rb < k) buf[rb] = b;
    in_order();
    if (count >= k) {
      count = k;
      lim = max(lim, buf[k - 1]);
      lim = ((uint64_t)__builtin_amdgcn_readfirstlane((int)(lim >> 32)) << 32) |
            (uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)lim);
      thr_f = rank_value((uint32_t)(lim >> 32));
    }
  }
};

// Bound by HBM where the logits are many and the alternatives few (4096 x 65536
// bf16, calls replayed from a graph: 90 us without entropy and alternatives, 6.0 TB/s;
// 105 to 115 with both and 4 of them, 129 with 16; 4096 x 65537 float32 with 4 183 us,
// 5.9 TB/s), by the latency of the best's ordering in a few rows (8 x 131072 with 8
// 12.2 us, both kernels).
// One wave's pass over a row: per lane the moments about `ref` (moved only when a
// logit exceeds it by 8, so nearly never after the first vectors; the sums are
// float32 and e^8 of them costs no accuracy), the largest logit, and over the wave
// the k best logits.
template <int DT, bool ENT, bool TOP>
struct RowScan {
  static constexpr int VE = kVec<DT>;
  float ref = -INFINITY, mx = -INFINITY, s = 0.0f, w = 0.0f;
  BestK best;
  int lane;

  __device__ __forceinline__ RowScan(uint64_t* buf, int k, int lane_) : best{buf, k, lane_}, lane(lane_) {}

  // a lane's VE logits from column col on; n of them exist, the others are -inf
  __device__ __forceinline__ void add(const float (&x)[VE], uint32_t col, int n, bool first) {
    float vm = x[0];
#pragma unroll
    for (int e = 1; e < VE; ++e) vm = fmaxf(vm, x[e]);
    if (__builtin_amdgcn_ballot_w64(vm > ref + 8.0f)) {
      if (vm > ref + 8.0f) {
        Moments a{ref, s, w};
        a.move(vm);
        ref = a.m;
        s = a.s;
        w = a.w;
      }
    }
    const float at = ref == -INFINITY ? 0.0f : ref;
    float es = 0.0f;
#pragma unroll
    for (int e = 0; e < VE; ++e) {
      const float d = x[e] - at, ex = lp_exp(d);
      es += ex;
      if constexpr (ENT) w = __builtin_fmaf(ex, fmaxf(d, kFar), w);
    }
    s += es;
    mx = fmaxf(mx, vm);
    if constexpr (TOP) {
      // a logit of this vector may be among the best (columns rise from vector to
      // vector, so one equal to the k-th best is not), or is NaN
      if (__builtin_amdgcn_ballot_w64(!(vm <= best.thr_f) || es != es)) {
        if (first) best.bound(n ? rank_of(vm) : 0);
        const float thr = best.thr_f;
#pragma unroll
        for (int e = 0; e < VE; ++e)
          if (__builtin_amdgcn_ballot_w64(!(x[e] <= thr)))
            best.offer(!(x[e] <= thr) && e < n ? BestK::key(rank_of(x[e]), col + e) : 0);
        if (best.count >= 2 * best.k) best.order();
      }
    }
  }

  // columns [c0, c1) of the row z, this wave's chunks of 64 VE of them (every
  // `waves`-th, from the wave-th on)
  template <bool NT>
  __device__ __forceinline__ void scan(const typename LogitOf<DT>::type* z, int64_t c0, int64_t c1, int wave,
                                       int waves) {
    constexpr int CH = 64 * VE, U = 2;  // U loads in flight per wave, eight waves a SIMD
    const int chunks = (int)((c1 - c0) / CH), rest = (int)((c1 - c0) % CH);
    const typename LogitOf<DT>::type* p = z + c0 + lane * VE;
    bool first = true;
    for (int i = wave; i < chunks; i += U * waves) {
      lp_u32x4 v[U];
#pragma unroll
      for (int u = 0; u < U; ++u)
        v[u] = lp_load<NT>(p + (int64_t)min(i + u * waves, chunks - 1) * CH);
#pragma unroll
      for (int u = 0; u < U; ++u) {
        if (i + u * waves >= chunks) break;
        float x[VE];
        lp_unpack<DT>(v[u], x);
        add(x, (uint32_t)(c0 + (int64_t)(i + u * waves) * CH + lane * VE), VE, first);
        first = false;
      }
    }
    if (rest && wave == chunks % waves) {
      const int n = min(max(rest - lane * VE, 0), VE);
      const int64_t at = c0 + (int64_t)chunks * CH + lane * VE;
      float x[VE];
      if (n == VE) lp_unpack<DT>(*reinterpret_cast<const lp_u32x4_any*>(z + at), x);
      else lp_load_tail<DT>(z + at, n, x);
      add(x, (uint32_t)at, n, first);
    }
  }
  // the wave's moments about its largest logit, the same on every lane
  __device__ __forceinline__ Moments moments() const {
    const float m = wave_max(mx), to = m == -INFINITY ? 0.0f : m;
    Moments a{ref, s, w};
    a.move(to);
    return {m, wave_sum(a.s), wave_sum(a.w)};
  }
};

struct LogprobOut {
  float *logp, *entropy, *stats, *top_logp;
  int32_t* top_idx;
};

// Partial results of a row's splits: moments, then the k best keys in order.
struct LogprobParts {
  float* moments;  // [rows * splits][3]
  uint32_t* list;  // [rows * splits][k][2]: lower and upper half of each key
};

// A row's results from its moments (uniform over the wave) and its best in order.
template <int DT>
__device__ __forceinline__ void lp_results(const typename LogitOf<DT>::type* z, int64_t r, int64_t V, int k,
                                           int lane, Moments a, const uint64_t* best, const int32_t* targets,
                                           const LogprobOut& out) {
  const bool empty = a.s == 0.0f;
  const float m = empty ? 0.0f : a.m, ln = logf(a.s);
  if (lane == 0) {
    if (out.stats) {
      out.stats[2 * r] = empty ? -INFINITY : a.s != a.s ? NAN : m;
      out.stats[2 * r + 1] = empty ? 0.0f : ln;
    }
    if (out.entropy) out.entropy[r] = empty ? 0.0f : ln - a.w / a.s;
    if (out.logp) {
      const int32_t t = targets[r];
      out.logp[r] = t < 0 ? 0.0f : t >= V ? NAN : empty ? -INFINITY : (logit<DT>(z + t) - m) - ln;
    }
  }
  if (lane < k) {
    const uint64_t b = best[lane];
    out.top_idx[r * k + lane] = (int32_t)~(uint32_t)b;
    out.top_logp[r * k + lane] = empty ? -INFINITY : (rank_value((uint32_t)(b >> 32)) - m) - ln;
  }
}

// WAVES == 1: one wave per row, four rows per workgroup.  WAVES == 4: a
// workgroup per row, or per split of seg columns of it, whose partial results
// logprob_join_kernel joins.
template <int DT, int WAVES, bool ENT, bool TOP, bool NT>
__global__ __launch_bounds__(256) void logprob_fwd_kernel(const void* Z, int64_t ldz,
                                                          const int32_t* targets, int64_t rows, int64_t V,
                                                          int k, int splits, int64_t seg, LogprobOut out,
                                                          LogprobParts parts) {
  typedef typename LogitOf<DT>::type T;
  __shared__ uint64_t bufs[TOP ? 4 : 1][TOP ? kBestCap : 1];
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  RowScan<DT, ENT, TOP> scan(bufs[TOP ? wave : 0], k, lane);
  if constexpr (WAVES == 1) {
    const int64_t r = (int64_t)blockIdx.x * 4 + wave;
    if (r >= rows) return;
    const T* z = (const T*)Z + r * ldz;
    scan.template scan<NT>(z, 0, V, 0, 1);
    if constexpr (TOP) scan.best.order();
    lp_results<DT>(z, r, V, k, lane, scan.moments(), scan.best.buf, targets, out);
  } else {
    __shared__ float mom[4][3];
    const int64_t r = blockIdx.x / splits, sp = blockIdx.x % splits;
    const T* z = (const T*)Z + r * ldz;
    scan.template scan<NT>(z, sp * seg, min(V, (sp + 1) * seg), wave, 4);
    if constexpr (TOP) scan.best.order();
    const Moments a = scan.moments();
    if (lane == 0) {
      mom[wave][0] = a.m;
      mom[wave][1] = a.s;
      mom[wave][2] = a.w;
    }
    __syncthreads();
    if (wave != 0) return;
    const float m = fmaxf(fmaxf(mom[0][0], mom[1][0]), fmaxf(mom[2][0], mom[3][0]));
    Moments all{m, 0.0f, 0.0f};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      Moments b{mom[i][0], mom[i][1], mom[i][2]};
      b.move(m == -INFINITY ? 0.0f : m);
      all.s += b.s;
      all.w += b.w;
    }
    uint64_t* best = bufs[0];
    if constexpr (TOP) {  // the four waves' best, at most 64, in the first one's buffer
      const uint64_t mine = lane < 4 * k ? bufs[lane / k][lane % k] : 0;
      BestK joined{best, k, lane};
      joined.offer(mine);
      joined.order();
    }
    if (splits == 1) {
      lp_results<DT>(z, r, V, k, lane, all, best, targets, out);
      return;
    }
    if (lane == 0) {
      float* p = parts.moments + (int64_t)blockIdx.x * 3;
      p[0] = all.m;
      p[1] = all.s;
      p[2] = all.w;
    }
    if (TOP && lane < k) {
      uint32_t* p = parts.list + ((int64_t)blockIdx.x * k + lane) * 2;
      p[0] = (uint32_t)best[lane];
      p[1] = (uint32_t)(best[lane] >> 32);
    }
  }
}

// One wave per row: the splits' moments (up to 64, one per lane) and keys.
template <int DT, bool TOP>
__global__ __launch_bounds__(256) void logprob_join_kernel(const void* Z, int64_t ldz, const int32_t* targets,
                                                           int64_t rows, int64_t V, int k, int splits,
                                                           LogprobOut out, LogprobParts parts) {
  typedef typename LogitOf<DT>::type T;
  __shared__ uint64_t bufs[TOP ? 4 : 1][TOP ? kBestCap : 1];
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int64_t r = (int64_t)blockIdx.x * 4 + wave;
  if (r >= rows) return;
  Moments a{-INFINITY, 0.0f, 0.0f};
  if (lane < splits) {
    const float* p = parts.moments + (r * splits + lane) * 3;
    a = {p[0], p[1], p[2]};
  }
  const float m = wave_max(a.m);
  a.move(m == -INFINITY ? 0.0f : m);
  const Moments all{m, wave_sum(a.s), wave_sum(a.w)};
  BestK best{bufs[TOP ? wave : 0], k, lane};
  if constexpr (TOP) {
    const uint32_t* p = parts.list + r * splits * k * 2;
    const int n = splits * k;  // up to 16 keys a lane
    uint32_t om = 0;
    for (int i = lane; i < n; i += 64) om = max(om, p[2 * i + 1]);
    best.bound(om);
    for (int i = 0; i < n; i += 64) {
      uint64_t key = 0;
      if (i + lane < n) key = p[2 * (i + lane)] | ((uint64_t)p[2 * (i + lane) + 1] << 32);
      best.offer(key);
    }
    best.order();
  }
  lp_results<DT>((const T*)Z + r * ldz, r, V, k, lane, all, best.buf, targets, out);
}

struct LogprobGrad {
  const int32_t *targets, *top_idx;
  const float *stats, *entropy, *g_logp, *g_entropy, *g_top;
  const mpx_scale_state* state;
};

// Bound by HBM (one read and one write of every logit: 4096 x 65536 bf16 173 us,
// 6.2 TB/s, x 65537 184, float32 368, 5.8 TB/s; replayed from a graph).  A wave's part of a row: up to U vectors per lane, all loaded before
// the first store.  With t = (z - m) - ln S and p = e^t the gradient is
//   p (c0 + c1 t),  c0 = -scale (sum of the upstream cotangents + g_H H),
//   c1 = -scale g_H,
// plus scale g at the target's and the alternatives' own columns: lane i <= k
// holds one of those columns and its cotangent, and a chunk that holds none of
// them, which one comparison tells, goes without.
template <int DT, bool NT>
__global__ __launch_bounds__(256) void logprob_bwd_kernel(const void* Z, int64_t ldz, int64_t rows, int64_t V,
                                                          int k, LogprobGrad g, void* dZ, int64_t ldo,
                                                          int64_t row_waves) {
  typedef typename LogitOf<DT>::type T;
  constexpr int VE = kVec<DT>, CH = 64 * VE, U = 4;
  const int lane = threadIdx.x & 63;
  const int64_t task = (int64_t)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int64_t r = task / row_waves;
  if (r >= rows) return;
  const int64_t c0 = (task % row_waves) * (U * CH);
  const T* z = (const T*)Z + r * ldz + c0;
  T* o = (T*)dZ + r * ldo + c0;
  const int64_t left = V - c0;  // >= 1
  float x[U][VE];
  lp_u32x4 v[U];
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const int64_t at = u * CH + lane * VE;
    if (at + VE <= left) v[u] = lp_load<NT>(z + at);
    else lp_load_tail<DT>(z + at, (int)max<int64_t>(left - at, 0), x[u]);
  }
  const float scale = g.state ? g.state->scale : 1.0f;
  const float ms = g.stats[2 * r], ln = g.stats[2 * r + 1], m = ms == -INFINITY ? 0.0f : ms;
  int64_t mine = -1;  // lane's special column and its cotangent
  float own = 0.0f;
  if (lane < k && g.g_top) {
    mine = g.top_idx[r * k + lane];
    own = g.g_top[r * k + lane];
    if (mine < 0 || mine >= V) own = NAN;
  } else if (lane == k && g.g_logp) {
    mine = g.targets[r];
    own = mine < 0 ? 0.0f : mine < V ? g.g_logp[r] : NAN;
  }
  const float up = wave_sum(own);
  const float ge = g.g_entropy ? g.g_entropy[r] : 0.0f, H = g.g_entropy ? g.entropy[r] : 0.0f;
  const float nan = ln != ln ? NAN : 0.0f;
  const float k1 = -scale * ge, k0 = __builtin_fmaf(k1, H, -scale * up) + nan;
  own *= scale;
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const int64_t at = u * CH + lane * VE;
    if (u * CH >= left) break;
    const int n = (int)min<int64_t>(max<int64_t>(left - at, 0), VE);
    if (n == VE) lp_unpack<DT>(v[u], x[u]);
    float d[VE];
#pragma unroll
    for (int e = 0; e < VE; ++e) {
      const float t = fmaxf((x[u][e] - m) - ln, kFar);
      d[e] = lp_exp(t) * __builtin_fmaf(k1, t, k0);
    }
    uint64_t mask = __builtin_amdgcn_ballot_w64(mine - c0 >= u * CH && mine - c0 < (u + 1) * CH);
    while (mask) {
      const int l = __builtin_ctzll(mask);
      mask &= mask - 1;
      const int off = __builtin_amdgcn_readlane((int)(mine - c0), l);
      const float add = __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, own), l));
#pragma unroll
      for (int e = 0; e < VE; ++e)
        if (at + e == off && x[u][e] != -INFINITY) d[e] += add;
    }
    if (n == VE) {
      lp_u32x4 w;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        if constexpr (DT == MPX_F32) w[j] = __builtin_bit_cast(uint32_t, d[j]);
        else w[j] = f2h<DT>(d[2 * j]) | ((uint32_t)f2h<DT>(d[2 * j + 1]) << 16);
      }
      lp_store<NT>(o + at, w);
    } else {
#pragma unroll
      for (int e = 0; e < VE; ++e) {
        if (e < n) {
          if constexpr (DT == MPX_F32) o[at + e] = d[e];
          else o[at + e] = f2h<DT>(d[e]);
        }
      }
    }
  }
}

// One wave per row where the rows alone fill the chip, or are so short that a
// workgroup's join costs more than its other waves gain; else a workgroup per row
// or, up to about 1024 workgroups, several, of at least kLeastSplit columns each and
// at most 64.  A wave keeps its own best, so fewer waves per row also order less.
// Measured (bf16, 4 alternatives; us, one wave / a workgroup): 64 rows x 500 4.9 /
// 5.2, x 1000 6.1 / 5.1; 2048 x 1000 6.7 / 7.6, x 4000 13.3 / 12.0; 4096 x 4000 16 /
// 19, x 32000 61 / 60 (with 16 75 / 82), x 65536 112 / 107; 16384 x 16000 109 / 129.
// Splits (us; workgroups aimed at 256, 512, 1024): 64 x 131072 24.4, 19.4, 17.8; 1 x
// 131072 in parts of at least 4096 columns 11.2, of 8192 12.8.
constexpr int64_t kLeastSplit = 4096;
// Logits (and, backward, gradients) that together pass the last-level cache are
// read and written around it; smaller ones may stay there for the next call
// (4096 x 65537 bf16 gradient 218 -> 183 us, 16384 x 32000 forward 199 -> 177;
// 1024 x 32000 forward 22.8, around the cache 23.6).
constexpr int64_t kStreamBytes = 256 << 20;
struct LogprobPlan {
  bool wave;
  int splits;
  int64_t seg;
};
static LogprobPlan logprob_plan(int64_t rows, int64_t V) {
  if (V <= (rows >= 4096 ? 32768 : rows >= 2048 ? 2048 : 512)) return {true, 1, V};
  const int64_t want = std::min<int64_t>({cdiv(1024, rows), cdiv(V, kLeastSplit), 64});
  const int64_t seg = cdiv(cdiv(V, want), kLeastSplit) * kLeastSplit;
  return {false, (int)cdiv(V, seg), seg};
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
  if (rows < 1 || V < 1 || k < 0 || k > MPX_LOGPROB_MAX_K) return 0;
  const int splits = logprob_plan(rows, V).splits;
  return splits == 1 ? 0 : (size_t)rows * splits * (3 * sizeof(float) + 2 * k * sizeof(uint32_t));
}

extern "C" int mpx_logprob_fwd(const void* Z, int64_t ldz, const int32_t* targets, int64_t rows,
                               int64_t V, int32_t k, float* logp, float* entropy, float* stats,
                               float* top_logp, int32_t* top_idx, mpx_dtype dt, void* workspace,
                               size_t ws_bytes, void* stream) {
  clear_error();
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
  MPX_REQUIRE(aligned4({targets, logp, entropy, stats, top_logp, top_idx, workspace}), "misaligned operand");
  const size_t need = mpx_logprob_workspace(rows, V, k);
  if (need && (!workspace || ws_bytes < need)) {
    set_error("mpx_logprob_fwd: workspace of " + std::to_string(need) + " bytes required");
    return MPX_ERR_WORKSPACE;
  }
  const LogprobPlan plan = logprob_plan(rows, V);
  const LogprobOut out = {logp, entropy, stats, top_logp, top_idx};
  const LogprobParts parts = {(float*)workspace, (uint32_t*)workspace + rows * plan.splits * 3};
  hipStream_t s = (hipStream_t)stream;
  const unsigned waves4 = (unsigned)cdiv(rows, 4), blocks = (unsigned)(rows * plan.splits);
  const bool nt = rows * V > kStreamBytes / (dt == MPX_F32 ? 4 : 2);
#define MPX_LP_KERNEL(DTv, WAVESv, ENTv, TOPv, NTv, grid)  \
  logprob_fwd_kernel<DTv, WAVESv, ENTv, TOPv, NTv>         \
      <<<grid, 256, 0, s>>>(Z, ldz, targets, rows, V, k, plan.splits, plan.seg, out, parts)
#define MPX_LP_FWD(DTv, ENTv, TOPv)                                                      \
  do {                                                                                   \
    if (plan.wave && nt) MPX_LP_KERNEL(DTv, 1, ENTv, TOPv, true, waves4);                \
    else if (plan.wave) MPX_LP_KERNEL(DTv, 1, ENTv, TOPv, false, waves4);                \
    else if (nt) MPX_LP_KERNEL(DTv, 4, ENTv, TOPv, true, blocks);                        \
    else MPX_LP_KERNEL(DTv, 4, ENTv, TOPv, false, blocks);                               \
    if (plan.splits > 1)                                                                 \
      logprob_join_kernel<DTv, TOPv>                                                     \
          <<<waves4, 256, 0, s>>>(Z, ldz, targets, rows, V, k, plan.splits, out, parts); \
  } while (0)
#define MPX_LP(DTv)                              \
  do {                                           \
    if (entropy && k) MPX_LP_FWD(DTv, true, true);   \
    else if (entropy) MPX_LP_FWD(DTv, true, false);  \
    else if (k) MPX_LP_FWD(DTv, false, true);        \
    else MPX_LP_FWD(DTv, false, false);              \
  } while (0)
  MPX_BY_TYPE(dt, MPX_LP);
#undef MPX_LP
#undef MPX_LP_FWD
#undef MPX_LP_KERNEL
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
  // tasks of up to 4 vectors per lane, four to a workgroup: up to 2^31 work-items
  const int64_t row_waves = cdiv(V, 4 * 64 * (dt == MPX_F32 ? 4 : 8));
  MPX_REQUIRE(rows <= ((int64_t)1 << 25) / row_waves, "rows * V too large for one call");
  const unsigned blocks = (unsigned)cdiv(rows * row_waves, 4);
  const bool nt = 2 * rows * V > kStreamBytes / (dt == MPX_F32 ? 4 : 2);
#define MPX_LP_KERNEL(DTv, NTv)    \
  logprob_bwd_kernel<DTv, NTv>     \
      <<<blocks, 256, 0, (hipStream_t)stream>>>(Z, ldz, rows, V, k, g, dZ, ldo, row_waves)
#define MPX_LP(DTv)                            \
  do {                                         \
    if (nt) MPX_LP_KERNEL(DTv, true);          \
    else MPX_LP_KERNEL(DTv, false);            \
  } while (0)
  MPX_BY_TYPE(dt, MPX_LP);
#undef MPX_LP
#undef MPX_LP_KERNEL
  MPX_LAUNCHED();
  return MPX_OK;
}
