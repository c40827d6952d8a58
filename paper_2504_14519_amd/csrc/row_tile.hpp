// Attention of 32 query rows a wave on tiles of keys in LDS: the inner loop that the forward kernels of four waves share (gathered
// rows on key blocks, rows on a cache in 4 bits).
//   S^T = K Q^T        A = K rows from LDS (row-packed), B = Q in registers
//   online softmax     one query column a lane: in-lane maxima and sums, one exchange between the half-waves
//   O^T += V^T P^T     A = V through the transposed LDS read, B = P straight from the C registers
// Two workgroups of four waves share a compute unit, so that one's softmax runs beside the other's matrix instructions: no phases.
#pragma once
#include "tile_common.hpp"

namespace slimpipe {

template <int D>
struct RowState {
  bf16x8 q[D / 16];
  f32x16 o[D / 32];
  float m, l;                // running maximum of the scaled scores (log2 units), sum of exp2(score - m), of this half-wave's keys
  SP_DEV void clear() {
#pragma unroll
    for (int db = 0; db < D / 32; ++db)
#pragma unroll
      for (int i = 0; i < 16; ++i) o[db][i] = 0.f;
  }
  SP_DEV void init() {
    clear();
    m = -INFINITY;
    l = 0.f;
  }
  // 1 / sum and lse of the lane's row; (0, -inf) when it saw no key (a sum that is NaN is not that)
  SP_DEV float finish(float* lse) const {
    const float total = xhalf_sum(l);
    const bool none = total == 0.f;
    *lse = none ? -INFINITY : (m + __builtin_log2f(total)) * kLn2;
    return none ? 0.f : 1.0f / total;
  }
};

// One tile of KEYS keys; masked: keys [kmin, kmax] of the tile are the lane's row's (kmin > kmax: none).
template <int D, int KEYS, class LoK, class LoV>
SP_DEV void attend_tile(RowState<D>& st, const LoK& lo_k, const LoV& lo_v, float c, bool masked, int kmin, int kmax, int g) {
  constexpr int KB = KEYS / 32, KS = D / 16, DB = D / 32;
  f32x16 s[KB];
  const f32x16 zero = {0};
  constexpr int LOOK = 3;
  bf16x8 buf[LOOK + 1];
  matrix_run<KS * KB, LOOK>(
      [&](auto m) { buf[m % (LOOK + 1)] = lds_rp<D>(lo_k, m / KB, m % KB * 32 * D * 2); },
      [&](auto m) { s[m % KB] = mfma32(buf[m % (LOOK + 1)], st.q[m / KB], m < KB ? zero : s[m % KB]); });
  if (masked) {
    const int lo = kmin - 4 * g, hi = kmax - 4 * g;
#pragma unroll
    for (int kb = 0; kb < KB; ++kb)
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const int key = kb * 32 + 8 * (i >> 2) + (i & 3);
        s[kb][i] = ((key >= lo) & (key <= hi)) ? s[kb][i] : -INFINITY;
      }
  }
  float mx = -INFINITY;
#pragma unroll
  for (int kb = 0; kb < KB; ++kb)
#pragma unroll
    for (int i = 0; i < 16; i += 2) mx = fmaxf(fmaxf(s[kb][i], s[kb][i + 1]), mx);
  mx = xhalf_max(mx);
  const float m_new = fmaxf(st.m, mx * c);
  const float m_eff = (m_new == -INFINITY) ? 0.f : m_new;
  if (__builtin_amdgcn_ballot_w64(m_new != st.m) != 0) {      // some row's maximum moved
    const float alpha = exp2_fast(st.m - m_eff);              // (m = -inf: 0)
    st.l *= alpha;
#pragma unroll
    for (int db = 0; db < DB; ++db)
#pragma unroll
      for (int i = 0; i < 16; ++i) st.o[db][i] *= alpha;
  }
  st.m = m_new;
  // (probabilities are rounded to bf16 for the matrix unit, relative to the exact running maximum; their sum is not rounded)
  bf16x8 p[KB][2];
  float sum = 0.f;
#pragma unroll
  for (int kb = 0; kb < KB; ++kb) {
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      s[kb][i] = exp2_fast(__builtin_fmaf(s[kb][i], c, -m_eff));
      sum += s[kb][i];
    }
    p[kb][0] = pack8(s[kb], 0);
    p[kb][1] = pack8(s[kb], 8);
  }
  st.l += sum;
  matrix_run<2 * KB * DB, LOOK>(
      [&](auto m) { buf[m % (LOOK + 1)] = lds_tr<D>(lo_v, m % DB, m / DB * 16 * D * 2); },
      [&](auto m) { st.o[m % DB] = mfma32(buf[m % (LOOK + 1)], p[m / DB / 2][m / DB % 2], st.o[m % DB]); });
}

}  // namespace slimpipe
