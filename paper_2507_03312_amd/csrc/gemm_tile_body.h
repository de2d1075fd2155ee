// A workgroup's work in a product, the text of gemm_tile_kernel and of gemm_tile (one function
// that both call changes the order of the kernels' scalar loads).  In scope: their template
// parameters, the product g, the tile's LDS smem, the workgroup's place `at`.
  constexpr bool kOwn = !std::is_same_v<Args, GemmArgs>, kPair = pair_operand<Args>();
  constexpr bool kRagged = ragged_reduction<Args>() && STG == 0;
  static_assert(!kOwn || (E == 0 && !B8), "an epilogue of its own has no other");
  static_assert(!kPair || (BKM && WN == 64), "a pair's fragments: 32 columns of each");
  constexpr int NWAVES = (BM / WM) * (BN / WN);
  constexpr int TM = WM / 32, TN = WN / 32;
  constexpr int A_BYTES = BM * 64 * 2, B_BYTES = BN * 64 * 2;
  constexpr int STAGE = A_BYTES + B_BYTES;
  constexpr int L = (BM + BN) / 8 / NWAVES;  // copies per lane per k tile
  // LDS read instructions per k step (a k-major fragment is one 16-byte
  // read, an mn-major one two transposing 8-byte reads)
  constexpr int kReads = TM * (AK ? 1 : 2) + TN * (BKM ? 1 : 2);
  // the epilogue works on 64 columns of a wave at a time
  constexpr int EC = WN < 64 ? WN : 64;
  const uint32_t lds0 = lds_u32(smem);

  const int tid = threadIdx.x;
  const int lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int wm0 = (wave / (BN / WN)) * WM;
  const int wn0 = (wave % (BN / WN)) * (kPair ? 32 : WN);

  int64_t m0, n0;
  tile_origin_of<BM, kPair ? BN / 2 : BN>(at.tile(), at.tiles(), g.M, g.N, m0, n0);
  int64_t z = at.batch();
  int split = 0;
  int64_t offA = 0, offB = 0, offC = 0;
  if (g.splits > 1) {
    split = (int)z;
  } else {
    const int64_t i0 = (uint32_t)z / (uint32_t)g.nb1, i1 = (uint32_t)z % (uint32_t)g.nb1;
    offA = i0 * g.sA0 + i1 * g.sA1;
    offB = i0 * g.sB0 + i1 * g.sB1;
    offC = i0 * g.sC0 + i1 * g.sC1;
  }
  const int64_t kbeg = (int64_t)split * g.k_split;
  const int64_t kend = min(g.K, kbeg + g.k_split);
  const int nk = (int)((kend - kbeg + (STG || kRagged ? 63 : 0)) / 64);

  const uint16_t* Ab = g.A + offA + (AK ? m0 * g.lda + kbeg : kbeg * g.lda + m0);
  const uint16_t* Bb = g.B + offB + (BKM ? n0 * g.ldb + kbeg : kbeg * g.ldb + n0);
  std::conditional_t<STG != 0, StagedOperand<BM, AK, NWAVES, STG == 2>, DmaOperand<BM, AK, NWAVES>> da;
  static_assert(!B8 || (STG != 0 && !BKM), "an 8-bit operand is staged, mn-major");
  std::conditional_t<kPair, PairOperand<BN, NWAVES, STG>,
                     std::conditional_t<B8, StagedAct8<DT, BN, NWAVES, STG == 2>,
                                        std::conditional_t<STG != 0, StagedOperand<BN, BKM, NWAVES, STG == 2>,
                                                           DmaOperand<BN, BKM, NWAVES>>>> db;
  if constexpr (STG != 0) {
    da.init(g.lda, g.M - m0, wave, lane);
    db.init(g.ldb, g.N - n0, wave, lane);
  } else {
    da.init(g.lda, (int)min<int64_t>(BM, g.M - m0), wave, lane);
    db.init(g.ldb, (int)min<int64_t>(BN, g.N - n0), wave, lane);
  }

  const bool whole = g.full_epi && m0 + BM <= g.M && n0 + BN <= g.N;  // uniform over the workgroup
  const int64_t mw = m0 + wm0, nw = n0 + wn0;
  // A whole tile's GELU' or residual operand is loaded into registers before
  // the first copies where they fit (the oldest loads, so the first tile's
  // wait covers them): the epilogue then starts without a memory round trip.
  constexpr bool kPF = STG == 0 && E != EPI_GENERIC && (E & (EPI_DACT | EPI_RESID)) != 0 && TN == 2 && TM <= 2;
  u32x4 pf[kPF ? 4 * TM : 1];
  if constexpr (kPF) {
    if (whole) {
      const int64_t ldp = (E & EPI_DACT) ? g.ldc : g.ldr;
      const uint16_t* src = ((E & EPI_DACT) ? g.dact : g.resid) + (mw * ldp + nw);
#pragma unroll
      for (int t = 0; t < 4 * TM; ++t)
        pf[t] = *reinterpret_cast<const u32x4*>(src + (uint32_t)(((lane >> 3) + 8 * t) * ldp + 8 * (lane & 7)));
    }
  }

  // likewise what an own epilogue reads
  const auto early = [&] {
    if constexpr (kOwn) return g.template prefetch<DT, TM, STG>(mw, nw, lane);
    else return 0;
  }();
  auto issue = [&](int kt, auto par) {  // par: STG's register set, kt & 1
    if constexpr (STG != 0) {
      const bool past = kt >= nk;
      kt = min(kt, nk - 1);
      const int krem = (int)min<int64_t>(kend - kbeg - 64 * (int64_t)kt, 1 << 20);
      da.template load<par>(Ab + (int64_t)kt * (AK ? 64 : 64 * g.lda), krem, past);
      if constexpr (B8)
        db.template load<par>(g.b8 + ((kbeg + 64 * (int64_t)kt) * g.ldb + n0),
                              g.b8_scale + ((kbeg + 64 * (int64_t)kt) / MPX_ACT8_GROUP * g.ldb + n0), krem, past);
      else if constexpr (kPair) db.template load<par>(Bb + (int64_t)kt * 64, g.pair, krem, past);
      else db.template load<par>(Bb + (int64_t)kt * (BKM ? 64 : 64 * g.ldb), krem, past);
    } else {
      const uint32_t st = lds0 + (uint32_t)((kt & 1) * STAGE);
      da.issue(reinterpret_cast<const uint16_t*>(reinterpret_cast<const uint8_t*>(Ab) + kt * da.step), st, wave);
      const uint16_t* b = reinterpret_cast<const uint16_t*>(reinterpret_cast<const uint8_t*>(Bb) + kt * db.step);
      if constexpr (kPair) {
        db.issue(b, g.pair, st + A_BYTES, wave);
      } else if constexpr (kRagged) {
        const int krem = (int)(kend - kbeg - 64 * (int64_t)kt);
        if (krem >= 64) db.issue(b, st + A_BYTES, wave);  // uniform
        else db.until(krem, g.ldb, wave, lane).issue(b, st + A_BYTES, wave);
      } else {
        db.issue(b, st + A_BYTES, wave);
      }
    }
  };
  auto put = [&](auto par) {  // STG: a loaded k tile (register set par) into stage par
    if constexpr (STG != 0) {
      da.template store<par>(smem + par * STAGE, wave, lane);
      db.template store<par>(smem + par * STAGE + A_BYTES, wave, lane);
    }
  };
  constexpr std::integral_constant<int, 0> I0{};
  constexpr std::integral_constant<int, 1> I1{};
  constexpr std::integral_constant<int, 2> I2{};
  constexpr std::integral_constant<int, 3> I3{};
  // a single k tile of one-value loads: nothing to prefetch
  const bool one = STG == 2 && nk == 1;
  if constexpr (STG != 0) {
    // no branch around a load in the loop (one would make the waits count the
    // later loads too): past the last k tile something is loaded and not used
    issue(0, I0);
    if (!one) issue(1, I1);
  } else {
    issue(0, I0);
    if (nk > 1) issue(1, I0);
  }

  FragReader<BM, AK, TM> fa;
  std::conditional_t<kPair, PairFragReader<BN>, FragReader<BN, BKM, TN>> fb;
  fa.init(wm0, lane);
  fb.init(wn0, lane);
  f32x16 acc[TM][TN];
  static_for<TM>([&](auto i) {
    static_for<TN>([&](auto j) {
#pragma unroll
      for (int e = 0; e < 16; ++e) acc[i][j][e] = 0.0f;
    });
  });
  // bias-gradient sums: tile columns sharing the A rows, this one's index,
  // and the next k tile this wave adds up (uniform over the wave)
  const bool db_parts = (kOwn && !g.db) || g.splits > 1;
  const int db_cols = db_parts ? (int)((g.N + BN - 1) / BN) : 1;
  const int db_col = db_parts ? (int)(n0 / BN) : 0;
  const bool dbw = DBS && wn0 == 0 && (db_parts || n0 == 0);
  int db_next = db_col;
  float dbs[TM];
#pragma unroll
  for (int i = 0; i < TM; ++i) dbs[i] = 0.0f;

  if constexpr (STG != 0) {
    put(I0);
    if (!one) issue(2, I0);
  } else {
    if (nk > 1) wait_vmcnt<L>();
    else wait_vmcnt<0>();
  }
  __syncthreads();

  // fragments double-buffered over the k steps of 16: the LDS reads of the
  // next step are issued among the MFMAs of the current one
  uint4 af[2][TM], bf[2][TN];
  auto read = [&](auto set, auto kk, uint32_t sa) {
    static_for<TM>([&](auto i) { af[set][i] = fa.template read<i, kk>(sa); });
    static_for<TN>([&](auto j) { bf[set][j] = fb.template read<j, kk>(sa + A_BYTES); });
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
  // one k tile; par = kt & 1 and last, which loads nothing, for STG only
  auto k_tile = [&](int kt, auto par, auto last) {
    const uint32_t sa = lds0 + (uint32_t)((kt & 1) * STAGE);
    const uint32_t sn = lds0 + (uint32_t)(((kt + 1) & 1) * STAGE);
    const bool db_now = dbw && kt == db_next;
    if (db_now) db_next += db_cols;
    if constexpr (STG != 0) {
      // the other stage was read before the last barrier
      constexpr std::integral_constant<int, 1 - par> other{};
      if (kt + 1 < nk) put(other);
      if constexpr (!last) issue(kt + 3, other);
    }
    read(I1, I1, sa);
    multiply(I0, db_now);
    read(I0, I2, sa);
    multiply(I1, db_now);
    read(I1, I3, sa);
    multiply(I0, db_now);
    if (kt + 1 < nk) {
      if constexpr (STG == 0) wait_vmcnt<0>();  // k tile kt + 1 has landed
      __syncthreads();
      if constexpr (STG == 0) {
        if (kt + 2 < nk) issue(kt + 2, I0);
      }
      read(I0, I0, sn);
    }
    multiply(I1, db_now);
  };
  if constexpr (STG != 0) {
    int kt = 0;
    for (; kt + 1 < nk; kt += 2) {
      k_tile(kt, I0, I0);
      k_tile(kt + 1, I1, I0);
    }
    if (kt < nk) k_tile(kt, I0, I1);
  } else {
    for (int kt = 0; kt < nk; ++kt) k_tile(kt, I0, I0);
  }

  if constexpr (DBS) {
    if (dbw) {
      int bad = 0;
      static_for<TM>([&](auto i) {
        const float other = __shfl_xor(dbs[i], 32);  // the row's other 8 k of every step
        const int64_t row = mw + 32 * i + lane;
        if (lane < 32 && row < g.M) {
          const float v = dbs[i] + other;
          if (db_parts) {
            g.dbp[row * ((int64_t)g.splits * db_cols) + (int64_t)split * db_cols + db_col] = v;
          } else {
            uint16_t h;
            if constexpr (kOwn) h = f2h<DT>(g.db_end(v, row));
            else h = f2h<DT>(v);
            g.db[row] = h;
            bad += h_nonfinite<DT>(h) ? 1 : 0;
          }
        }
      });
      if (g.nonfinite) add_nonfinite(g.nonfinite, bad);
    }
  }
  // the accumulators hold C^T blocks (the MFMA operands are swapped above)
  if constexpr (kOwn) {
    g.template epilogue<DT, BM, BN, WM, WN>(acc, early, m0, n0, mw, nw, lane, wave, split, smem);
    return;
  }
  if (g.splits > 1) {
    gemm_partials<TM, TN>(g, acc, mw, nw, lane, split);
    return;
  }
  __syncthreads();  // every wave is done reading the stage buffers
  uint16_t* lds = reinterpret_cast<uint16_t*>(smem) + wave * (WM * (EC + 4));
  static_for<(TN + 1) / 2>([&](auto c) {
    constexpr int J0 = 2 * c, TC = TN - J0 < 2 ? TN - J0 : 2;
    if (whole)
      gemm_epilogue_lds<DT, TM, TC, E, false, J0>(g, acc, mw, nw + 32 * J0, lane, offC, lds,
                                                  kPF ? pf : nullptr);
    else
      gemm_epilogue_lds<DT, TM, TC, E, true, J0>(g, acc, mw, nw + 32 * J0, lane, offC, lds, nullptr,
                                                 (int)min<int64_t>(WM, g.M - mw),
                                                 (int)min<int64_t>(32 * TC, g.N - nw - 32 * J0));
  });
