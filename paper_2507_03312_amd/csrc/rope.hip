// Rotary positions with several axes (mpx_rope_fwd, mpx_rope_bwd).
#include "rope.h"

namespace mpx {

// Bound by HBM (every value read and written once).  The turns are as many as
// rows x pairs, far fewer than the values, but dear (float64 angles): a
// workgroup makes each of its rows' once, into LDS, while the copied heads
// stream; every thread then keeps the turns of its VW values in registers and goes
// through the heads, one run of VW values from each, four heads in flight.  A
// value's partner lies in the same run (interleaved) or comes from the lane that
// has it (halves): y = x c + partner s, s negative in a section's first half.
// Values behind the sections count as pairs that are not turned.  The lanes of a
// head lie in one wave (a.chunks <= 64 runs).  12608 rows of 36 heads of 64 bf16 (116
// MB) take 25 us, in place 16.5; 29997 of 48 heads of 128 f16 (737 MB) 119 us; in
// float32 45, 28 and 258.  Lanes that do not make up a whole head idle: 8192 rows of 12
// heads of 256, 264 (33 of 64 lanes) and 320 (40) bf16 21.6, 27.7 and 29.2 us, in place
// 18.8, 22.1 and 24.3; of 128, 160 (40) and 256 float32 20.3, 27.4 and 38.7.
template <int DT, int VW, bool INTER, bool NT>
__global__ __launch_bounds__(256) void rope_kernel(RopeArgs a) {
  typedef typename RopeValue<DT>::type T;
  __shared__ float2 turns[kRopeTable];
  const uint32_t row0 = blockIdx.x * a.wg_rows;
  const T* X = (const T*)a.X + (int64_t)row0 * a.ldx;
  T* Y = (T*)a.Y + (int64_t)row0 * a.ldy;
  const uint32_t nrows = min((uint32_t)a.wg_rows, a.rows - row0);
  // runs of 16 bytes also serve the copied heads, like turned ones (a loop of
  // their own: 12608 x 36 heads of 64 bf16 28.6 us)
  constexpr bool kWide = VW * sizeof(T) == 16;
  if constexpr (!kWide) rope_copies<DT>(a, X, a.ldx, Y, nrows);
  rope_turns(a, row0, nrows, turns);

  const int lane = threadIdx.x & 63;
  const uint32_t chunk = lane % a.chunks, wave_slots = 64 / a.chunks;
  const uint32_t slot = (threadIdx.x >> 6) * wave_slots + lane / a.chunks;
  const uint32_t r = slot / a.head_slots, h0 = slot % a.head_slots;
  if ((uint32_t)lane >= wave_slots * a.chunks || r >= nrows) return;  // all lanes of a head or none
  const int v0 = chunk * VW;  // the thread's first value
  const bool turned = v0 < 2 * a.npairs;
  int p0 = v0 / 2, partner = lane;  // its first pair, the lane of its partners
  bool second = false;
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
  constexpr int NP = INTER ? VW / 2 : VW;  // pairs the thread has a part in
  float c[NP], s[NP];
#pragma unroll
  for (int i = 0; i < NP; ++i) {
    const float2 t = turned ? turns[r * a.npairs + p0 + i] : make_float2(1.0f, 0.0f);
    c[i] = t.x;
    s[i] = INTER || second ? t.y : -t.y;
  }
  const T* x = X + r * a.ldx + v0;
  T* y = Y + r * a.ldy + v0;
  const uint32_t heads = a.heads_rot + (kWide && !a.in_place ? a.copy / a.hd : 0);
  constexpr int U = 4;
  for (uint32_t h = h0; h < heads; h += U * a.head_slots) {
    RopeVec<DT, VW> v[U];
#pragma unroll
    for (int u = 0; u < U; ++u) v[u].template load<NT>(x + (int64_t)min(h + u * a.head_slots, heads - 1) * a.hd);
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (h + u * a.head_slots >= heads) break;
      const bool turn = turned && (!kWide || h + u * a.head_slots < a.heads_rot);
      T* p = y + (int64_t)(h + u * a.head_slots) * a.hd;
      if constexpr (INTER) {
        if (turn) {
#pragma unroll
          for (int i = 0; i < NP; ++i) {
            const float x0 = v[u].get(2 * i), x1 = v[u].get(2 * i + 1);
            v[u].set(2 * i, __builtin_fmaf(x0, c[i], -(x1 * s[i])));
            v[u].set(2 * i + 1, __builtin_fmaf(x1, c[i], x0 * s[i]));
          }
        }
      } else {
        const RopeVec<DT, VW> o = v[u].from_lane(partner);
        if (turn) {
#pragma unroll
          for (int i = 0; i < NP; ++i) v[u].set(i, __builtin_fmaf(v[u].get(i), c[i], o.get(i) * s[i]));
        }
      }
      if (turn || !a.in_place) v[u].template store<NT>(p);
    }
  }
}

// Heads of more than 64 runs (long ones whose sections allow only short runs), or
// of runs of one value: a thread takes both runs of VW pairs, so that nothing
// passes between lanes (8192 rows of 36 heads of 64 bf16 in sections of 11, 4, 1
// and 16 pairs 19.6 us; values passed one by one 23.1).  A head of odd length has
// one value more (VW == 1 then).
template <int DT, int VW, bool INTER>
__global__ __launch_bounds__(256) void rope_pairs_kernel(RopeArgs a) {
  typedef typename RopeValue<DT>::type T;
  __shared__ float2 turns[kRopeTable];
  const uint32_t row0 = blockIdx.x * a.wg_rows;
  const T* X = (const T*)a.X + (int64_t)row0 * a.ldx;
  T* Y = (T*)a.Y + (int64_t)row0 * a.ldy;
  const uint32_t nrows = min((uint32_t)a.wg_rows, a.rows - row0);

  rope_copies<DT>(a, X, a.ldx, Y, nrows);
  rope_turns(a, row0, nrows, turns);

  const uint32_t chunk = threadIdx.x % a.chunks, slot = threadIdx.x / a.chunks;
  const uint32_t r = slot / a.head_slots, h0 = slot % a.head_slots;
  if (r >= nrows) return;
  const int p0 = chunk * VW;  // the thread's first pair
  const bool turned = p0 < a.npairs;
  float c[VW], s[VW];
  int at0, at1;  // its two runs of values
  if constexpr (INTER) {
    at0 = 2 * p0;
    at1 = at0 + VW;
  } else {
    // sections: the axes', then what is not turned
    int first = 0, n = a.hd / 2 - a.npairs;
#pragma unroll
    for (int k = 0; k < MPX_ROPE_MAX_AXES; ++k) {
      if (p0 >= a.first_pair[k]) {
        first = a.first_pair[k];
        n = a.first_pair[k + 1] - first;
      }
    }
    if (!turned) {
      first = a.npairs;
      n = a.hd / 2 - a.npairs;
    }
    at0 = 2 * first + (p0 - first);
    at1 = at0 + n;
  }
#pragma unroll
  for (int i = 0; i < VW; ++i) {
    const float2 t = turned ? turns[r * a.npairs + p0 + i] : make_float2(1.0f, 0.0f);
    c[i] = t.x;
    s[i] = t.y;
  }
  const T* x = X + r * a.ldx;
  T* y = Y + r * a.ldy;
  constexpr int U = 4;
  for (uint32_t h = h0; h < a.heads_rot; h += U * a.head_slots) {
    RopeVec<DT, VW> v0[U], v1[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const T* p = x + (int64_t)min(h + u * a.head_slots, a.heads_rot - 1) * a.hd;
      v0[u].load(p + at0);
      v1[u].load(p + at1);
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (h + u * a.head_slots >= a.heads_rot) break;
      T* p = y + (int64_t)(h + u * a.head_slots) * a.hd;
      if (turned) {
#pragma unroll
        for (int i = 0; i < VW; ++i) {
          if constexpr (INTER && VW > 1) {  // pair i at values 2 i and 2 i + 1 of both runs together
            RopeVec<DT, VW>& v = 2 * i < VW ? v0[u] : v1[u];
            const int j = (2 * i) % VW;
            const float x0 = v.get(j), x1 = v.get(j + 1);
            v.set(j, __builtin_fmaf(x0, c[i], -(x1 * s[i])));
            v.set(j + 1, __builtin_fmaf(x1, c[i], x0 * s[i]));
          } else {
            const float x0 = v0[u].get(i), x1 = v1[u].get(i);
            v0[u].set(i, __builtin_fmaf(x0, c[i], -(x1 * s[i])));
            v1[u].set(i, __builtin_fmaf(x1, c[i], x0 * s[i]));
          }
        }
      }
      if (turned || !a.in_place) {
        v0[u].store(p + at0);
        v1[u].store(p + at1);
      }
    }
  }
  if constexpr (VW == 1) {
    if ((a.hd & 1) && chunk == 0 && !a.in_place)
      for (uint32_t h = h0; h < a.heads_rot; h += a.head_slots)
        y[(int64_t)h * a.hd + a.hd - 1] = x[(int64_t)h * a.hd + a.hd - 1];
  }
}

template <int DT, int VW>
static void launch_rope(const RopeArgs& a, bool pairs, unsigned blocks, hipStream_t s) {
  if constexpr (VW <= 4) {  // 512 values make at most 64 runs of 8
    if (pairs) {
      if (a.interleaved) rope_pairs_kernel<DT, VW, true><<<blocks, 256, 0, s>>>(a);
      else rope_pairs_kernel<DT, VW, false><<<blocks, 256, 0, s>>>(a);
      return;
    }
  }
  if constexpr (VW > 1) {
    constexpr bool kWide = VW * sizeof(typename RopeValue<DT>::type) == 16;
    if constexpr (kWide) {
      if (a.stream) {
        if (a.interleaved) rope_kernel<DT, VW, true, true><<<blocks, 256, 0, s>>>(a);
        else rope_kernel<DT, VW, false, true><<<blocks, 256, 0, s>>>(a);
        return;
      }
    }
    if (a.interleaved) rope_kernel<DT, VW, true, false><<<blocks, 256, 0, s>>>(a);
    else rope_kernel<DT, VW, false, false><<<blocks, 256, 0, s>>>(a);
  }
}

static int rope(const char* fn, bool back, const void* X, int64_t ldx, void* Y, int64_t ldy,
                const float* pos, int64_t pos_rows, int64_t rows, int64_t heads_rot,
                int64_t heads_copy, int64_t hd, const mpx_rope_plan* plan, mpx_dtype dt, void* stream) {
#define MPX_REQUIRE_FN(cond, msg)                       \
  do {                                                  \
    if (!(cond)) {                                      \
      set_error(std::string(fn) + ": " + (msg));        \
      return MPX_ERR_INVALID;                           \
    }                                                   \
  } while (0)
  MPX_REQUIRE_FN(X && Y && pos && plan, "NULL operand");
  MPX_REQUIRE_FN(is_half(dt) || dt == MPX_F32, "dt must be MPX_F16, MPX_BF16 or MPX_F32");
  MPX_REQUIRE_FN(rows >= 1 && pos_rows >= 1 && rows % pos_rows == 0,
                 "rows must be a positive multiple of pos_rows");
  MPX_REQUIRE_FN(rows <= INT32_MAX, "too many rows for one call");
  MPX_REQUIRE_FN(hd >= 2 && hd <= kRopeMaxHd, "hd must be in [2, 512]");
  const int64_t most = (int64_t)1 << 20;
  MPX_REQUIRE_FN(heads_rot >= 1 && heads_rot <= most && heads_copy >= 0 && heads_copy <= most,
                 "heads_rot must be >= 1 and heads_copy >= 0, at most 2^20 each");
  const int64_t width = (heads_rot + heads_copy) * hd;
  MPX_REQUIRE_FN(ldx >= width && ldy >= width, "row stride below (heads_rot + heads_copy) * hd");
  MPX_REQUIRE_FN(X != Y || ldx == ldy, "in place needs equal row strides");
  const uintptr_t mis = reinterpret_cast<uintptr_t>(X) | reinterpret_cast<uintptr_t>(Y);
  MPX_REQUIRE_FN(mis % (dt == MPX_F32 ? 4 : 2) == 0 && reinterpret_cast<uintptr_t>(pos) % 4 == 0,
                 "pointers must be aligned to their element");
  RopeArgs a{};
  int vw, vp;  // of the kernel of runs, and of pairs of runs
  if (const char* why = rope_plan(plan, hd, dt, a, vw, vp)) MPX_REQUIRE_FN(false, why);
  const int64_t n = a.npairs;
  const bool pairs = hd / vw > 64 || vw == 1;
  if (pairs) vw = vp;
  a.X = X;
  a.Y = Y;
  a.pos = pos;
  a.ldx = ldx;
  a.ldy = ldy;
  a.heads_rot = (uint32_t)heads_rot;
  a.copy = (uint32_t)(heads_copy * hd);
  a.back = back ? 1 : 0;
  a.in_place = X == Y ? 1 : 0;
  // Values past the 256 MB last-level cache go around it (29997 rows of 48 heads of
  // 128 f16 129 -> 119 us, in place 117 -> 100); smaller ones may be in it, or be read
  // from it next (16640 rows of 18 heads of 64 15.6 us, around it 18.9).
  const double bytes = (double)rows * (double)width * (dt == MPX_F32 ? 4.0 : 2.0);
  a.stream = (X == Y ? bytes : 2.0 * bytes) > 256.0 * (1 << 20) ? 1 : 0;
  a.chunks = (int32_t)(pairs ? hd / 2 : hd) / vw;
  // Rows of a workgroup: about four heads to a thread where the rows suffice for
  // 1024 workgroups, never more turns than the table holds (12608 rows of 36 heads of
  // 64 bf16, two, four and eight heads: 32, 25.7, 27 us).
  const int64_t slots = pairs ? 256 / a.chunks : 4 * (64 / a.chunks);
  int64_t wg_rows = std::min<int64_t>({4 * slots / (heads_rot + (a.in_place ? 0 : heads_copy)), slots, kRopeTable / n, rows / 1024});
  wg_rows = std::max<int64_t>(wg_rows, 1);
  a.wg_rows = (int32_t)wg_rows;
  a.head_slots = (int32_t)(slots / wg_rows);
  const int64_t blocks = cdiv(rows, wg_rows);
  MPX_REQUIRE_FN(blocks < ((int64_t)1 << 24), "too many rows for one call");
#undef MPX_REQUIRE_FN
  a.rows = (uint32_t)rows;
  a.pos_rows = (uint32_t)pos_rows;
  hipStream_t s = (hipStream_t)stream;
#define MPX_ROPE(DTv)                                                    \
  do {                                                                   \
    if (vw == 4) launch_rope<DTv, 4>(a, pairs, (unsigned)blocks, s);     \
    else if (vw == 2) launch_rope<DTv, 2>(a, pairs, (unsigned)blocks, s); \
    else launch_rope<DTv, 1>(a, pairs, (unsigned)blocks, s);             \
  } while (0)
  if (dt == MPX_F32) {
    MPX_ROPE(MPX_F32);
  } else if (vw == 8) {
    if (dt == MPX_F16) launch_rope<MPX_F16, 8>(a, pairs, (unsigned)blocks, s);
    else launch_rope<MPX_BF16, 8>(a, pairs, (unsigned)blocks, s);
  } else if (dt == MPX_F16) {
    MPX_ROPE(MPX_F16);
  } else {
    MPX_ROPE(MPX_BF16);
  }
#undef MPX_ROPE
  MPX_LAUNCHED();
  return MPX_OK;
}

}  // namespace mpx

extern "C" int mpx_rope_fwd(const void* X, int64_t ldx, void* Y, int64_t ldy, const float* pos,
                            int64_t pos_rows, int64_t rows, int64_t heads_rot, int64_t heads_copy,
                            int64_t hd, const mpx_rope_plan* plan, mpx_dtype dt, void* stream) {
  mpx::clear_error();
  return mpx::rope("mpx_rope_fwd", false, X, ldx, Y, ldy, pos, pos_rows, rows, heads_rot, heads_copy, hd,
                   plan, dt, stream);
}

extern "C" int mpx_rope_bwd(const void* dY, int64_t ldy, void* dX, int64_t ldx, const float* pos,
                            int64_t pos_rows, int64_t rows, int64_t heads_rot, int64_t heads_copy,
                            int64_t hd, const mpx_rope_plan* plan, mpx_dtype dt, void* stream) {
  mpx::clear_error();
  return mpx::rope("mpx_rope_bwd", true, dY, ldy, dX, ldx, pos, pos_rows, rows, heads_rot, heads_copy, hd,
                   plan, dt, stream);
}
