// Weight gradients C = A^T B whose B is an 8-bit checkpoint, both operands copied
// straight into LDS as they lie in memory (see gemm_kernels.h for the half form
// and the register-staged form of any alignment).  Internal; not part of the ABI.
#pragma once

#include "gemm_kernels.h"

namespace mpx {

// Codes [64 k][128] of one stage, 16-byte chunks permuted so that the 8 rows x 2
// chunks which 32 lanes of a transposing read touch lie in 16 different 16-byte
// columns of the 256 bytes of banks (a row spans half of them).
__device__ __forceinline__ int act8_chunk(int r, int c) { return c ^ (2 * ((r >> 1) & 3)); }

#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"
// 4 bytes per lane from base + off (bytes) into LDS at lds + 4 * lane
__device__ __forceinline__ void dma4(const void* base, uint32_t off, uint32_t lds) {
  asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dword %0, %1"
               :
               : "v"(off), "s"(base), "s"(lds)
               : "memory", "m0");
}
#pragma clang diagnostic pop

// Copies of a stage's codes, 16 bytes per lane, or 4 (NARROW) where rows are not
// whole 16-byte chunks or start between them (8415 x 768 x 588 bf16 27 us, 38 with
// the register-staged tiles; 12608 x 2304 x 764 68 and 108).
template <int NWAVES, bool NARROW>
struct Act8Dma {
  static constexpr int Q = (NARROW ? 32 : 8) / NWAVES;
  static_assert(8 % NWAVES == 0, "copies do not split evenly over the waves");
  uint32_t off[Q];
  // k row of this lane's copy q
  __device__ __forceinline__ static int row(int q, int wave, int lane) {
    return (wave + NWAVES * q) * (NARROW ? 2 : 8) + lane / (NARROW ? 32 : 8);
  }
  // rv: outputs (a multiple of 16, or 4) of the matrix from the tile's first on; ld: bytes
  __device__ __forceinline__ void init(int64_t ld, int rv, int wave, int lane) {
#pragma unroll
    for (int q = 0; q < Q; ++q) {
      const int kr = row(q, wave, lane);
      const int col = NARROW ? 16 * act8_chunk(kr, lane % 32 / 4) + 4 * (lane & 3) : 16 * act8_chunk(kr, lane % 8);
      off[q] = (uint32_t)(kr * ld + (col < rv ? col : 0));
    }
  }
  __device__ __forceinline__ void issue(const uint8_t* base, uint32_t lds, int wave) const {
    const uint64_t p = reinterpret_cast<uint64_t>(base);
    const uint64_t lo = (uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)p);
    const uint64_t hi = (uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)(p >> 32));
    const uint32_t slds = (uint32_t)__builtin_amdgcn_readfirstlane((int)lds);
#pragma unroll
    for (int q = 0; q < Q; ++q) {
      if constexpr (NARROW)
        dma4(reinterpret_cast<const void*>(lo | (hi << 32)), off[q], slds + 256u * (uint32_t)(wave + NWAVES * q));
      else
        dma16(reinterpret_cast<const void*>(lo | (hi << 32)), off[q], slds + 1024u * (uint32_t)(wave + NWAVES * q));
    }
  }
};

typedef int act8_v2i __attribute__((ext_vector_type(2)));

// 8 codes of one output (ds_read_b64_tr_b8 transposes bytes across 16 lanes: lane
// i passes the address of row i / 2, columns 8 (i % 2), and gets 8 rows of column i)
__device__ __forceinline__ u32x2 lds_tr8_b64(uint32_t addr) {
  const act8_v2i v =
      __builtin_amdgcn_ds_read_tr8_b64_v2i32((__attribute__((address_space(3))) act8_v2i*)(uintptr_t)addr);
  return u32x2{(uint32_t)v[0], (uint32_t)v[1]};
}

// an MFMA fragment: 8 codes of one group, times its scale, as half values (exact)
template <int DT>
__device__ __forceinline__ uint4 act8_widen(u32x2 q, float s) {
  if constexpr (DT == MPX_F16) {
    return make_uint4(__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(q.x, s, false)),
                      __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(q.x, s, true)),
                      __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(q.y, s, false)),
                      __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(q.y, s, true)));
  } else {
    return make_uint4(__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(q.x, s, false)),
                      __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(q.x, s, true)),
                      __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(q.y, s, false)),
                      __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(q.y, s, true)));
  }
}

// gemm_tile_kernel's loop (k tiles of 64 in two LDS stages, one barrier a tile
// ahead of its last k step) with B in 8 bits: B takes half the LDS and copies,
// its fragments one transposing read each instead of two, and are widened in
// registers by the instruction that takes a scale: a lane's 8 codes are 8 rows of
// one column, so one group.  A k tile's scales (2 groups of BN columns) come with
// its copies, by one wave, and from LDS into registers (loaded by each lane for its
// own columns they cost as many memory instructions as the codes: 65536 x 1024 x
// 1024 bf16 192 us, 180 without any).
//
// Any reduction length: in the last k tile, rows behind the matrix read its last
// row again, and A's are then zeroed in LDS by the wave that copied them (a code
// of that row can be NaN only where its column's sum is NaN anyway).
template <int DT, int BM, int BN, int WM, int WN, int E, bool DBS, bool NARROW>
__global__ __launch_bounds__((BM / WM) * (BN / WN) * 64)
__attribute__((amdgpu_waves_per_eu(BM == 64 ? 4 : 2, BM == 64 ? 4 : 2)))
void gemm_act8_kernel(GemmArgs g) {
  constexpr int NWAVES = (BM / WM) * (BN / WN);
  constexpr int TM = WM / 32, TN = WN / 32;
  constexpr int A_BYTES = BM * 64 * 2, B_BYTES = BN * 64;
  constexpr int STAGE = A_BYTES + B_BYTES, SCALES = 2 * BN;
  static_assert(BN == 128, "act8_chunk, and one copy of scales");
  constexpr int kReads = 2 * TM + TN;
  constexpr int EC = WN < 64 ? WN : 64;
  constexpr int EPI = NWAVES * WM * (EC + 4) * 2;
  __shared__ __attribute__((aligned(1024))) uint8_t smem[2 * (STAGE + SCALES) > EPI ? 2 * (STAGE + SCALES) : EPI];
  const uint32_t lds0 = lds_u32(smem);

  const int tid = threadIdx.x;
  const int lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int wm0 = (wave / (BN / WN)) * WM;
  const int wn0 = (wave % (BN / WN)) * WN;

  int64_t m0, n0;
  tile_origin<BM, BN>(g.M, g.N, m0, n0);
  const int split = g.splits > 1 ? (int)blockIdx.y : 0;
  const int64_t kbeg = (int64_t)split * g.k_split;
  const int64_t kend = min(g.K, kbeg + g.k_split);
  const int nk = (int)((kend - kbeg + 63) / 64);
  const int krest = (int)(kend - kbeg) - 64 * (nk - 1);  // rows of the last k tile

  const uint16_t* Ab = g.A + kbeg * g.lda + m0;
  const uint8_t* Bb = g.b8 + kbeg * g.ldb + n0;
  DmaOperand<BM, false, NWAVES> da;
  Act8Dma<NWAVES, NARROW> db;
  da.init(g.lda, (int)min<int64_t>(BM, g.M - m0), wave, lane);
  db.init(g.ldb, (int)min<int64_t>(BN, g.N - n0), wave, lane);

  // scales of k tile kt: 2 groups of BN columns, in LDS behind both stages
  const uint8_t* Sb = g.b8_scale + kbeg / MPX_ACT8_GROUP * g.ldb + n0;
  const int groups = (int)((kend - kbeg + MPX_ACT8_GROUP - 1) / MPX_ACT8_GROUP);
  const int scols = (int)min<int64_t>(BN, g.N - n0);
  auto issue_scales = [&](int kt) {
    const uint64_t p = reinterpret_cast<uint64_t>(Sb + (int64_t)2 * kt * g.ldb);
    const uint64_t lo = (uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)p);
    const uint64_t hi = (uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)(p >> 32));
    const int c = 4 * lane % BN, gr = min(4 * lane / BN, groups - 1 - 2 * kt);
    dma4(reinterpret_cast<const void*>(lo | (hi << 32)), (uint32_t)(gr * g.ldb + (c < scols ? c : 0)),
         (uint32_t)__builtin_amdgcn_readfirstlane((int)(lds0 + 2 * STAGE + (kt & 1) * SCALES)));
  };
  auto issue = [&](int kt) {
    const uint32_t st = lds0 + (uint32_t)((kt & 1) * STAGE);
    const uint16_t* a = reinterpret_cast<const uint16_t*>(reinterpret_cast<const uint8_t*>(Ab) + kt * da.step);
    const uint8_t* b = Bb + (int64_t)kt * 64 * g.ldb;
    if (wave == 0) issue_scales(kt);
    if (kt + 1 < nk || krest == 64) {  // uniform
      da.issue(a, st, wave);
      db.issue(b, st + A_BYTES, wave);
    } else {
      auto ca = da;
      auto cb = db;
#pragma unroll
      for (int q = 0; q < ca.Q; ++q) {
        const int kr = (64 * (wave + NWAVES * q) + lane) / (BM / 8);
        ca.off[q] -= (uint32_t)(max(0, kr - (krest - 1)) * g.lda * 2);
      }
#pragma unroll
      for (int q = 0; q < cb.Q; ++q) {
        cb.off[q] -= (uint32_t)(max(0, cb.row(q, wave, lane) - (krest - 1)) * g.ldb);
      }
      ca.issue(a, st, wave);
      cb.issue(b, st + A_BYTES, wave);
    }
  };
  // this wave's copies of k tile kt have landed: A's rows behind the matrix
  auto landed = [&](int kt) {
    if (kt + 1 < nk || krest == 64) return;
    uint8_t* st = smem + (kt & 1) * STAGE;
#pragma unroll
    for (int q = 0; q < da.Q; ++q) {
      const int kr = (64 * (wave + NWAVES * q) + lane) / (BM / 8);
      if (kr >= krest) *reinterpret_cast<u32x4*>(st + 1024 * (wave + NWAVES * q) + 16 * lane) = u32x4{0u, 0u, 0u, 0u};
    }
  };
  issue(0);
  if (nk > 1) issue(1);

  FragReader<BM, false, TM> fa;
  fa.init(wm0, lane);
  uint32_t fb[TN];
  {
    const int gq = lane >> 4, i = lane & 15;
    const int kr = 8 * (gq >> 1) + (i >> 1);
#pragma unroll
    for (int j = 0; j < TN; ++j) {
      const int c = (wn0 + 32 * j) / 16 + (gq & 1);
      fb[j] = (uint32_t)(kr * BN + act8_chunk(kr, c) * 16 + 8 * (i & 1));
    }
  }
  f32x16 acc[TM][TN];
  static_for<TM>([&](auto i) {
    static_for<TN>([&](auto j) {
#pragma unroll
      for (int e = 0; e < 16; ++e) acc[i][j][e] = 0.0f;
    });
  });
  const int db_cols = g.splits > 1 ? (int)((g.N + BN - 1) / BN) : 1;
  const int db_col = g.splits > 1 ? (int)(n0 / BN) : 0;
  const bool dbw = DBS && wn0 == 0 && (g.splits > 1 || n0 == 0);
  int db_next = db_col;
  float dbs[TM];
#pragma unroll
  for (int i = 0; i < TM; ++i) dbs[i] = 0.0f;

  float sc[2][TN];
  auto take_scales = [&](int kt) {
    const uint8_t* s = smem + 2 * STAGE + (kt & 1) * SCALES + wn0 + (lane & 31);
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
      for (int j = 0; j < TN; ++j) sc[i][j] = __builtin_bit_cast(float, (uint32_t)s[i * BN + 32 * j] << 23);
  };

  constexpr int L = (DmaOperand<BM, false, NWAVES>::Q + Act8Dma<NWAVES, NARROW>::Q);
  if (nk > 1) wait_vmcnt<L>();  // the first wave has its scales' copies too: it waits for the second tile's
  else wait_vmcnt<0>();
  landed(0);
  __syncthreads();
  take_scales(0);

  constexpr std::integral_constant<int, 0> I0{};
  constexpr std::integral_constant<int, 1> I1{};
  constexpr std::integral_constant<int, 2> I2{};
  constexpr std::integral_constant<int, 3> I3{};
  uint4 af[2][TM], bf[2][TN];
  u32x2 raw[TN];
  auto read = [&](auto set, auto kk, uint32_t sa) {
    static_for<TM>([&](auto i) { af[set][i] = fa.template read<i, kk>(sa); });
    static_for<TN>([&](auto j) { raw[j] = lds_tr8_b64(sa + A_BYTES + fb[j] + kk * 16 * BN); });
  };
  auto widen = [&](auto set, auto kk) {
    static_for<TN>([&](auto j) { bf[set][j] = act8_widen<DT>(raw[j], sc[kk / 2][j]); });
  };
  auto multiply = [&](auto set, bool db_now) {
    static_for<TM>([&](auto i) {
      static_for<TN>([&](auto j) { acc[i][j] = mfma32<DT>(bf[set][j], af[set][i], acc[i][j]); });
    });
    if constexpr (DBS) {
      if (db_now) static_for<TM>([&](auto i) { dbs[i] += frag_sum8<DT>(af[set][i]); });
    }
    static_for<TM * TN>([&](auto x) {  // each MFMA with its share of the reads
      __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
      constexpr int n = (x + 1) * kReads / (TM * TN) - x * kReads / (TM * TN);
      if constexpr (n > 0) __builtin_amdgcn_sched_group_barrier(0x100, n, 0);
    });
    __builtin_amdgcn_sched_barrier(0);
  };
  read(I0, I0, lds0);
  widen(I0, I0);
  for (int kt = 0; kt < nk; ++kt) {
    const uint32_t sa = lds0 + (uint32_t)((kt & 1) * STAGE);
    const uint32_t sn = lds0 + (uint32_t)(((kt + 1) & 1) * STAGE);
    const bool db_now = dbw && kt == db_next;
    if (db_now) db_next += db_cols;
    read(I1, I1, sa);
    multiply(I0, db_now);
    widen(I1, I1);
    read(I0, I2, sa);
    multiply(I1, db_now);
    widen(I0, I2);
    read(I1, I3, sa);
    multiply(I0, db_now);
    widen(I1, I3);
    if (kt + 1 < nk) {
      wait_vmcnt<0>();  // k tile kt + 1 has landed
      landed(kt + 1);
      __syncthreads();
      take_scales(kt + 1);
      if (kt + 2 < nk) issue(kt + 2);
      read(I0, I0, sn);
    }
    multiply(I1, db_now);
    if (kt + 1 < nk) widen(I0, I0);
  }

  const int64_t mw = m0 + wm0, nw = n0 + wn0;
  if constexpr (DBS) {
    if (dbw) {
      int bad = 0;
      static_for<TM>([&](auto i) {
        const float other = __shfl_xor(dbs[i], 32);  // the row's other 8 k of every step
        const int64_t row = mw + 32 * i + lane;
        if (lane < 32 && row < g.M) {
          const float v = dbs[i] + other;
          if (g.splits > 1) {
            g.dbp[row * ((int64_t)g.splits * db_cols) + (int64_t)split * db_cols + db_col] = v;
          } else {
            const uint16_t h = f2h<DT>(v);
            g.db[row] = h;
            bad += h_nonfinite<DT>(h) ? 1 : 0;
          }
        }
      });
      if (g.nonfinite) add_nonfinite(g.nonfinite, bad);
    }
  }
  if (g.splits > 1) {
    gemm_partials<TM, TN>(g, acc, mw, nw, lane, split);
    return;
  }
  __syncthreads();  // every wave is done reading the stage buffers
  const bool whole = g.full_epi && m0 + BM <= g.M && n0 + BN <= g.N;
  uint16_t* lds = reinterpret_cast<uint16_t*>(smem) + wave * (WM * (EC + 4));
  static_for<(TN + 1) / 2>([&](auto c) {
    constexpr int J0 = 2 * c, TC = TN - J0 < 2 ? TN - J0 : 2;
    if (whole)
      gemm_epilogue_lds<DT, TM, TC, E, false, J0>(g, acc, mw, nw + 32 * J0, lane, 0, lds);
    else
      gemm_epilogue_lds<DT, TM, TC, E, true, J0>(g, acc, mw, nw + 32 * J0, lane, 0, lds, nullptr,
                                                 (int)min<int64_t>(WM, g.M - mw),
                                                 (int)min<int64_t>(32 * TC, g.N - nw - 32 * J0));
  });
}

// C = A^T B of a weight gradient whose B is an 8-bit checkpoint (g.b8): direct
// tiles of g.act8_rows x 128 (chosen with the splits, act8_plan), or, where that is
// 0, register-staged ones of 64 x 64 or 128 x 128 by choose_config's rule for such
// operands.
template <int DT>
static hipError_t run_gemm_act8(GemmArgs g, hipStream_t s, bool* db_fused) {
  if (!g.b8 || !g.b8_scale || g.dact8) return hipErrorInvalidValue;  // no kernel here has GELU'
  const int64_t lim = ((int64_t)1 << 31) - 4096;
  const bool any = g.M < 8 || g.N < 8 || g.lda * 256 >= lim || g.ldb * 64 >= lim;
  const int64_t t64 = ((g.M + 63) / 64) * ((g.N + 63) / 64);
  const bool small = !g.act8_rows && (any || g.M <= 64 || g.N <= 64 || (g.splits == 1 && t64 <= 512));
  *db_fused = g.db && (!small || g.splits == 1);  // split partials are laid out for 128-wide tile columns
  if (!*db_fused) {
    g.db = nullptr;
    g.dbp = nullptr;
  }
  const int bm = g.act8_rows ? g.act8_rows : small ? 64 : 128, bn = small ? 64 : 128;
  const dim3 grid((unsigned)(((g.M + bm - 1) / bm) * ((g.N + bn - 1) / bn)), (unsigned)g.splits);
  g.full_epi = full_epilogue_ok(g, bm) ? 1 : 0;
#define MPX_K8_STAGED(B, W, STGv, Ev, DBv) \
  gemm_tile_kernel<DT, B, B, W, W, 2, false, false, Ev, DBv, STGv, true><<<grid, 256, 0, s>>>(g)
#define MPX_K8_DIRECT(B, W, NARv, Ev, DBv) \
  gemm_act8_kernel<DT, B, 128, W, 64, Ev, DBv, NARv><<<grid, 256, 0, s>>>(g)
#define MPX_K8_EPI(KERNEL, B, W, STGv)                     \
  do {                                                     \
    const bool plain = epilogue_mask(g) == 0;              \
    if (g.db) {                                            \
      if (plain) KERNEL(B, W, STGv, 0, true);              \
      else KERNEL(B, W, STGv, EPI_GENERIC, true);          \
    } else {                                               \
      if (plain) KERNEL(B, W, STGv, 0, false);             \
      else KERNEL(B, W, STGv, EPI_GENERIC, false);         \
    }                                                      \
  } while (0)
  const bool narrow = g.ldb % 16 != 0 || (reinterpret_cast<uintptr_t>(g.b8) & 15u) != 0;
  if (g.act8_rows == 64 && narrow) MPX_K8_EPI(MPX_K8_DIRECT, 64, 32, true);
  else if (g.act8_rows == 64) MPX_K8_EPI(MPX_K8_DIRECT, 64, 32, false);
  else if (g.act8_rows && narrow) MPX_K8_EPI(MPX_K8_DIRECT, 128, 64, true);
  else if (g.act8_rows) MPX_K8_EPI(MPX_K8_DIRECT, 128, 64, false);
  else if (any) MPX_K8_EPI(MPX_K8_STAGED, 64, 32, 2);
  else if (small) MPX_K8_EPI(MPX_K8_STAGED, 64, 32, 1);
  else MPX_K8_EPI(MPX_K8_STAGED, 128, 64, 1);
#undef MPX_K8_EPI
#undef MPX_K8_DIRECT
#undef MPX_K8_STAGED
  return hipGetLastError();
}

}  // namespace mpx
