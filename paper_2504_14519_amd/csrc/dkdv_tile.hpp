// The two kinds of phase of the key-stationary dk/dv kernels (dense: attn_bwd.hip, which says how they alternate; gathered rows of key
// blocks: block_bwd.hip).
#pragma once
#include "tile_common.hpp"

namespace slimpipe {

template <int D, int BMQ>
struct DkdvState {
  static constexpr int KS = D / 16, DB = D / 32, QB = BMQ / 32;
  bf16x8 kreg[KS];
  f32x16 dk[DB], dv[DB];
  f32x16 s[QB], dp[QB];
  bf16x8 pb[QB][2], dsb[QB][2];      // 16 query rows each
  f32x4 lse2v[QB][4];                // lse2 of this lane's rows of the tile in `s`: fetched by the matrix phase (the LDS
                                     // latency passes while the score MFMAs run), used first thing by the vector phase
};

// LDS layout (bytes): Q ring, dO ring, V rows of the workgroup, statistics ring
template <int D, int NW, int ROWS>
struct DkdvLds {
  static constexpr int BMQ = ROWS, SLOTS = 4;
  static constexpr int TILE_BYTES = BMQ * D * 2;
  static constexpr int Q_BASE = 0, DO_BASE = SLOTS * TILE_BYTES, V_BASE = 2 * SLOTS * TILE_BYTES;
  static constexpr int V_BYTES = NW * 32 * D * 2;
  static constexpr int STAT_BASE = V_BASE + V_BYTES;          // [SLOTS][lse2[BMQ], delta[BMQ]] floats
  static constexpr int STAT_BYTES = 2 * BMQ * 4;
  // ... and, in place of all that, the dk or dv rows of the workgroup on their way out
  static constexpr int RINGS = STAT_BASE + SLOTS * STAT_BYTES, OUT_BYTES = NW * 32 * kOutRow<D> * 4;
  static constexpr int TOTAL = RINGS > OUT_BYTES ? RINGS : OUT_BYTES;
};

template <int D, int NW, int BMQ, bool WITH_ACC, bool WITH_SCORES, int LOOK, class L = DkdvLds<D, NW, BMQ>>
struct DkdvMatrixPhase {
  static constexpr int KS = D / 16, DB = D / 32, QB = BMQ / 32;
  static constexpr int N_AC = WITH_ACC ? 4 * DB * QB : 0, N_SC = WITH_SCORES ? 2 * KS * QB : 0, N = N_AC + N_SC;
  static constexpr int NBUF = LOOK + 1, HALF = 16 * D * 2;
  const TrBase<D>& lo_qt;      // Q(u-1), transposed; dO(u-1) sits DO_BASE further
  const RpBase<D>& lo_q;       // Q(u), row-packed; dO(u) sits DO_BASE further
  const RpBase<D>& lo_v;       // this wave's 32 rows of V
  DkdvState<D, BMQ>& st;
  const float* stat;           // LDS: lse2 of the rows of tile u, this lane's half (rows 8 i4 + 4 g .. + 3 at [8 i4 .. + 3]);
                               // -delta of the same rows BMQ floats further
  bf16x8 abuf[NBUF];
  bf16x8 vb[2];

  // matrix instruction j of the scores: head_dim block ks, query block qb, S or dP
  static constexpr int ks_of(int j) { return j / (2 * QB); }
  static constexpr int qb_of(int j) { return j % (2 * QB) / 2; }

  template <int M>
  SP_DEV void reads() {
    if constexpr (WITH_SCORES && M == N_AC + LOOK + 2) {
#pragma unroll
      for (int qb = 0; qb < QB; ++qb)
#pragma unroll
        for (int i4 = 0; i4 < 4; ++i4) st.lse2v[qb][i4] = *reinterpret_cast<const f32x4*>(stat + 32 * qb + 8 * i4);
    }
    // the accumulator of dP(u) starts from -delta of its rows (dP of the tile before was packed into dsb by the
    // vector phase and is dead): the matrix pipe delivers dP - delta
    if constexpr (WITH_SCORES && M == (N_AC > 0 ? 2 : 0)) {
#pragma unroll
      for (int qb = 0; qb < QB; ++qb)
#pragma unroll
        for (int i4 = 0; i4 < 4; ++i4) {
          const f32x4 nd = *reinterpret_cast<const f32x4*>(stat + L::BMQ + 32 * qb + 8 * i4);
#pragma unroll
          for (int e = 0; e < 4; ++e) st.dp[qb][4 * i4 + e] = nd[e];
        }
    }
    if constexpr (M < N_AC) {
      constexpr int h = M / (2 * DB), db = (M % (2 * DB)) / 2;      // h: 16 query rows
      abuf[M % NBUF] = lds_tr<D>(lo_qt, db, ((M & 1) ? 0 : L::DO_BASE) + h * HALF);
    } else if constexpr (M < N) {
      constexpr int j = M - N_AC, ks = ks_of(j), qb = qb_of(j);
      if constexpr ((j & 1) == 0) {
        abuf[M % NBUF] = lds_rp<D>(lo_q, ks, qb * 32 * D * 2);
      } else {
        abuf[M % NBUF] = lds_rp<D>(lo_q, ks, L::DO_BASE + qb * 32 * D * 2);
        if constexpr (qb == 0) vb[ks & 1] = lds_rp<D>(lo_v, ks, 0);
      }
    }
  }
  template <int M>
  SP_DEV void mfma() {
    if constexpr (M < N_AC) {
      constexpr int h = M / (2 * DB), db = (M % (2 * DB)) / 2;
      if constexpr ((M & 1) == 0) st.dv[db] = mfma32(abuf[M % NBUF], st.pb[h / 2][h % 2], st.dv[db]);
      else st.dk[db] = mfma32(abuf[M % NBUF], st.dsb[h / 2][h % 2], st.dk[db]);
    } else {
      constexpr int j = M - N_AC, ks = ks_of(j), qb = qb_of(j);
      const f32x16 zero = {0};
      if constexpr ((j & 1) == 0) st.s[qb] = mfma32(abuf[M % NBUF], st.kreg[ks], ks == 0 ? zero : st.s[qb]);
      else st.dp[qb] = mfma32(abuf[M % NBUF], vb[ks & 1], st.dp[qb]);
    }
  }
  template <int M>
  SP_DEV void step() {
    if constexpr (M < N) {
      reads<M + LOOK>();
      SP_FENCE();
      mfma<M>();
      SP_FENCE();
      step<M + 1>();
    }
  }
  template <int M>
  SP_DEV void prologue() {
    if constexpr (M < LOOK) { reads<M>(); prologue<M + 1>(); }
  }
  SP_DEV void run() {
    SP_FENCE();
    matrix_phase_begin();
    prologue<0>();
    SP_FENCE();
    step<0>();
    matrix_phase_end();
    SP_FENCE();
  }
};

// P = exp2(c S - lse2) on visible pairs, dS = P (dP - delta), where `dp` arrives as dP - delta; element i of block qb of a lane is
// query row 32 qb + 8*(i/4) + 4g + i%4 of the tile, the lane's column is its key.  `hook(i)`, i = 0..3, is called at four
// points spread over the phase (asynchronous tile copies ride there).
template <int D, int BMQ, class H>
SP_DEV void dkdv_vector_phase(DkdvState<D, BMQ>& st, float c, bool need_mask, int rmin_rel, int rmax_rel, int g, H&& hook) {
  constexpr int QB = BMQ / 32;
  if (need_mask) {
    // row (32 qb + 8*(i/4) + 4g + i%4) in [rmin_rel, rmax_rel), with the lane's part moved to the bounds: the row
    // numbers are immediates then (a register per element otherwise, hoisted out of the tile loop)
    const int lo = rmin_rel - 4 * g, hi = rmax_rel - 4 * g;
#pragma unroll
    for (int qb = 0; qb < QB; ++qb)
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const int r = 32 * qb + 8 * (i >> 2) + (i & 3);
        st.s[qb][i] = ((r >= lo) & (r < hi)) ? st.s[qb][i] : -INFINITY;      // exp2(-inf) = 0
      }
  }
  // Stage by stage over the 16 elements of a block, so that neighbouring instructions do not depend on each other.
  // No LDS read here: lse2 is in registers (the matrix phase fetched it) and delta is in dP already.  This
  // phase is the longer of the two, and an LDS read in it waits for about 280 cycles behind the reads of the
  // group that is in its matrix phase.
#pragma unroll
  for (int qb = 0; qb < QB; ++qb) {
    if (qb == 0) hook(0);
#pragma unroll
    for (int i = 0; i < 16; ++i) st.s[qb][i] = __builtin_fmaf(st.s[qb][i], c, -st.lse2v[qb][i >> 2][i & 3]);
    if (qb == 0) hook(1);
#pragma unroll
    for (int i = 0; i < 16; ++i) st.s[qb][i] = exp2_fast(st.s[qb][i]);
    if (qb == QB - 1) hook(2);
#pragma unroll
    for (int i = 0; i < 16; ++i) st.dp[qb][i] *= st.s[qb][i];       // dp holds dP - delta
    if (qb == QB - 1) hook(3);
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      st.pb[qb][h] = pack8(st.s[qb], 8 * h);
      st.dsb[qb][h] = pack8(st.dp[qb], 8 * h);
      // pin: without a use here the optimiser sinks this arithmetic past the phase barrier
      asm volatile("" : "+v"(st.pb[qb][h]), "+v"(st.dsb[qb][h]));
    }
  }
}

}  // namespace slimpipe
