// Rotary positions with several axes (mpx_rope_fwd, mpx_rope_bwd).
#include <hip/hip_runtime.h>

#include <cmath>

#include "common.h"

namespace mpx {

constexpr int kRopeMaxHd = 512;

// The turn of every pair of a head, in turns per unit of position, and where
// its two values lie.
struct RopeArgs {
  double rev[kRopeMaxHd / 2];
  const void* X;
  void* Y;
  const float* pos;
  int64_t ldx, ldy, pos_rows, rows, heads_rot, heads_copy;
  int32_t hd, axes, npairs, interleaved, back, in_place;
  int32_t first_pair[MPX_ROPE_MAX_AXES + 1];  // axis a owns pairs [first_pair[a], first_pair[a + 1])
};

template <int DT> struct RopeValue { typedef uint16_t type; };
template <> struct RopeValue<MPX_F32> { typedef float type; };
template <int DT>
__device__ __forceinline__ float rope_load(const typename RopeValue<DT>::type* p) {
  if constexpr (DT == MPX_F32) return *p;
  else return h2f<DT>(*p);
}
template <int DT>
__device__ __forceinline__ void rope_store(typename RopeValue<DT>::type* p, float v) {
  if constexpr (DT == MPX_F32) *p = v;
  else *p = f2h<DT>(v);
}

// One workgroup per row: a thread takes one pair (or one value that is not
// turned) of every head in turn.
template <int DT>
__global__ __launch_bounds__(256) void rope_kernel(RopeArgs a) {
  typedef typename RopeValue<DT>::type T;
  const int64_t r = blockIdx.x;
  const T* x = (const T*)a.X + r * a.ldx;
  T* y = (T*)a.Y + r * a.ldy;
  const float* pos = a.pos + (r % a.pos_rows) * a.axes;
  const int rest = a.hd - 2 * a.npairs;
  for (int i = threadIdx.x; i < a.npairs + rest; i += 256) {
    if (i < a.npairs) {
      int ax = 0;
      while (i >= a.first_pair[ax + 1]) ++ax;
      const int n = a.first_pair[ax + 1] - a.first_pair[ax], j = i - a.first_pair[ax];
      const int o = 2 * a.first_pair[ax];
      const int i0 = o + (a.interleaved ? 2 * j : j), i1 = o + (a.interleaved ? 2 * j + 1 : n + j);
      double t = (double)pos[ax] * a.rev[i];
      t -= rint(t);
      float s, c;
      sincospif(2.0f * (float)t, &s, &c);
      if (a.back) s = -s;
      for (int64_t h = 0; h < a.heads_rot; ++h) {
        const float x0 = rope_load<DT>(x + h * a.hd + i0), x1 = rope_load<DT>(x + h * a.hd + i1);
        rope_store<DT>(y + h * a.hd + i0, __builtin_fmaf(x0, c, -(x1 * s)));
        rope_store<DT>(y + h * a.hd + i1, __builtin_fmaf(x1, c, x0 * s));
      }
    } else if (!a.in_place) {
      const int v = a.npairs + i;  // values behind the pairs
      for (int64_t h = 0; h < a.heads_rot; ++h) y[h * a.hd + v] = x[h * a.hd + v];
    }
  }
  if (a.in_place) return;
  const int64_t w0 = a.heads_rot * a.hd, w1 = w0 + a.heads_copy * a.hd;
  for (int64_t v = w0 + threadIdx.x; v < w1; v += 256) y[v] = x[v];
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
  MPX_REQUIRE_FN(hd >= 2 && hd <= kRopeMaxHd, "hd must be in [2, 512]");
  const int64_t most = (int64_t)1 << 20;
  MPX_REQUIRE_FN(heads_rot >= 1 && heads_rot <= most && heads_copy >= 0 && heads_copy <= most,
                 "heads_rot must be >= 1 and heads_copy >= 0, at most 2^20 each");
  const int64_t width = (heads_rot + heads_copy) * hd;
  MPX_REQUIRE_FN(ldx >= width && ldy >= width, "row stride below (heads_rot + heads_copy) * hd");
  MPX_REQUIRE_FN(X != Y || ldx == ldy, "in place needs equal row strides");
  MPX_REQUIRE_FN(plan->axes >= 1 && plan->axes <= MPX_ROPE_MAX_AXES, "axes must be in [1, 4]");
  MPX_REQUIRE_FN(plan->interleaved == 0 || plan->interleaved == 1, "interleaved must be 0 or 1");
  const uintptr_t mis = reinterpret_cast<uintptr_t>(X) | reinterpret_cast<uintptr_t>(Y);
  MPX_REQUIRE_FN(mis % (dt == MPX_F32 ? 4 : 2) == 0 && reinterpret_cast<uintptr_t>(pos) % 4 == 0,
                 "pointers must be aligned to their element");
  RopeArgs a{};
  int64_t n = 0;
  for (int ax = 0; ax < plan->axes; ++ax) {
    const int64_t p = plan->pairs[ax];
    const double base = plan->base[ax];
    MPX_REQUIRE_FN(p >= 1 && 2 * (n + p) <= hd, "pairs must be >= 1 and 2 * their sum <= hd");
    MPX_REQUIRE_FN(std::isfinite(base) && base > 1.0, "base must be finite and > 1");
    for (int64_t i = 0; i < p; ++i)
      a.rev[n + i] = std::pow(base, -(double)i / (double)p) / 6.283185307179586476925286766559;
    a.first_pair[ax] = (int32_t)n;
    n += p;
  }
  for (int ax = plan->axes; ax <= MPX_ROPE_MAX_AXES; ++ax) a.first_pair[ax] = (int32_t)n;
  MPX_REQUIRE_FN(rows < ((int64_t)1 << 24), "at most 2^24 - 1 rows in one call");
#undef MPX_REQUIRE_FN
  a.X = X;
  a.Y = Y;
  a.pos = pos;
  a.ldx = ldx;
  a.ldy = ldy;
  a.pos_rows = pos_rows;
  a.rows = rows;
  a.heads_rot = heads_rot;
  a.heads_copy = heads_copy;
  a.hd = (int32_t)hd;
  a.axes = plan->axes;
  a.npairs = (int32_t)n;
  a.interleaved = plan->interleaved;
  a.back = back ? 1 : 0;
  a.in_place = X == Y ? 1 : 0;
  hipStream_t s = (hipStream_t)stream;
  const unsigned blocks = (unsigned)rows;
  switch (dt) {
    case MPX_F16: rope_kernel<MPX_F16><<<blocks, 256, 0, s>>>(a); break;
    case MPX_BF16: rope_kernel<MPX_BF16><<<blocks, 256, 0, s>>>(a); break;
    default: rope_kernel<MPX_F32><<<blocks, 256, 0, s>>>(a);
  }
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
