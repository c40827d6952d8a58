// Choosing the key blocks of sparse attention: block means, scores with their top-k, and the lists that turn "the blocks of a row"
// into "the rows of a block".
#include "blocks.hpp"
#include "tile_common.hpp"

namespace slimpipe {

// ------------------------------------------------------------------------------------ block means
// mean[j] = (1 / n_j) sum of the n_j keys that block j holds before kv_end.  One workgroup a block and kv head, D / 8 lanes a row
// (16 bytes each); sums in 64 bits, in which sums of bf16 numbers of like size are exact, so that the mean is rounded once (to 32
// bits) and does not depend on the order.  Bound by reading the keys once (32 blocks of 512
// keys of 128: 6 us, a third of it the launch).
template <int D>
__global__ __launch_bounds__(1024) void block_means_kernel(const BlockMeansArgs a) {
  constexpr int NC = D / 8, ROWS = 1024 / NC, WROWS = 64 / NC;
  __shared__ double sums[16][D];
  const int j = a.first_block + blockIdx.x, hk = blockIdx.y, b = blockIdx.z;
  const int tid = threadIdx.x, c = tid % NC;
  const int64_t key0 = (int64_t)j * a.block_len;
  const int64_t left = a.kv_end - key0;
  const int n = left < a.block_len ? (int)left : a.block_len;
  const int chunk = kv_chunk_of(a.kv, key0);
  const bf16_t* base = a.kv.k[chunk] + (int64_t)b * a.kv_stride_b + (int64_t)hk * a.kv_stride_h + (key0 - (int64_t)chunk * a.kv.len) * a.kv_stride_s + c * 8;
  double acc[8] = {0, 0, 0, 0, 0, 0, 0, 0};
  for (int r0 = tid / NC; r0 < n; r0 += 4 * ROWS) {
    bf16x8 x[4];
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const int r = r0 + u * ROWS;
      x[u] = *reinterpret_cast<const bf16x8*>(base + (int64_t)(r < n ? r : r0) * a.kv_stride_s);
    }
#pragma unroll
    for (int u = 0; u < 4; ++u)
      if (r0 + u * ROWS < n)
#pragma unroll
        for (int e = 0; e < 8; ++e) acc[e] += (double)(float)x[u][e];
  }
#pragma unroll
  for (int e = 0; e < 8; ++e) {
#pragma unroll
    for (int w = NC; w < 64; w <<= 1) acc[e] += __shfl_xor(acc[e], w, 64);
    if ((tid & 63) < NC) sums[tid >> 6][c * 8 + e] = acc[e];
  }
  static_assert(WROWS * NC == 64, "a wave holds whole rows");
  __syncthreads();
  if (tid < D) {
    double s = 0;
    for (int w = 0; w < 16; ++w) s += sums[w][tid];
    a.means[(((int64_t)b * a.n_kv_heads + hk) * a.blocks_total + j) * D + tid] = (float)(s / (double)n);
  }
}

hipError_t launch_block_means(const BlockMeansArgs& a, int head_dim, hipStream_t st) {
  dim3 grid((unsigned)a.n_blocks, (unsigned)a.n_kv_heads, (unsigned)a.batch), block(1024);
  if (head_dim == 128) hipLaunchKernelGGL(block_means_kernel<128>, grid, block, 0, st, a);
  else hipLaunchKernelGGL(block_means_kernel<64>, grid, block, 0, st, a);
  return hipGetLastError();
}

// ------------------------------------------------------------------------------------ selection
// score[r][j] = q_r . mean_j, compared in 64 bits, without computing most of it in 64 bits.  A float32 mean is the sum of two bf16 numbers to 2^-16
// of itself (each rounded to 2^-8), so bf16 matrix instructions give every score with that and float32 additions as its error.  The
// smaller parts go first: only the D products of the larger ones are added at the size of the score, so that it is off by at most
//   delta_r = ((9/8) D 2^-23 + 2^-16) |q_r| max_j |mean_j|.
// If T is the n-th largest of the approximate scores of a row, the exact n-th largest lies within delta of T: what is above T + 2 delta is
// taken for certain, what is below T - 2 delta is not, and only where more lies between than there are places are scores computed in
// 64 bits (one row in fifty).  Where products might run into the smallest float32 numbers (|q| or max |mean| below 2^-40: the bound has
// 2^-103 to spare then) nothing is certain.  A row of zeros, as padding has them, or means that are all zero have equal scores
// throughout, which needs no computing.
//
// T comes from a first walk over the blocks: a lane keeps the K largest scores of its row that it has seen in order in registers; a score x
// goes into the list t_0 >= t_1 .. by t_i = median(t_(i-1), t_i, x), one instruction a place and no branch.  A second walk computes the scores
// again (cheaper than keeping them: 16 matrix instructions for 32 rows and 32 blocks) and writes down what is not below T - 2 delta.
// The bound goes by the largest mean, so what all means have in common widens it without changing any order, and more rows are settled in 64 bits: the
// case below with a common part of 3, 10 and 30 times the spread of the means takes 72, 98 and 151 us.
// 16384 rows of 8 heads on 256 blocks of means of head_dim 128, top_k 8: 70 us, 18 a walk (7 for Q, 4 at the end, most of it rows settled in 64 bits); with three parts of a mean 77, with sorted pieces of scores kept in LDS 204,
// with every score in 64 bits on the matrix unit 550.

// Places that a row's list of candidates has (what is certain and what is not): with more, which only many equal scores can bring, the row
// is done in 64 bits throughout.
// (few enough of them that the LDS of two workgroups fits a compute unit)
constexpr int select_places(int k) { return k <= 8 ? 16 : k <= 16 ? 28 : kMaxTopK + 32; }
constexpr uint32_t kUnsure = 0x80000000u;      // flag of a candidate within 2 delta of T

// Eight elements of a mean as two bf16 parts (larger first), and their squares.
SP_DEV void split_means(const f32x4& x0, const f32x4& x1, bf16x8 (&part)[2], float& sq) {
  const bf16x4 a0 = __builtin_convertvector(x0, bf16x4), a1 = __builtin_convertvector(x1, bf16x4);
  const f32x4 r0 = x0 - __builtin_convertvector(a0, f32x4), r1 = x1 - __builtin_convertvector(a1, f32x4);      // (exact)
  const bf16x4 b0 = __builtin_convertvector(r0, bf16x4), b1 = __builtin_convertvector(r1, bf16x4);
  part[0] = __builtin_shufflevector(a0, a1, 0, 1, 2, 3, 4, 5, 6, 7);
  part[1] = __builtin_shufflevector(b0, b1, 0, 1, 2, 3, 4, 5, 6, 7);
#pragma unroll
  for (int e = 0; e < 4; ++e) sq += x0[e] * x0[e] + x1[e] * x1[e];
}
template <int K>
SP_DEV void keep_largest(float (&t)[K], float x) {
#pragma unroll
  for (int i = K - 1; i > 0; --i) t[i] = __builtin_amdgcn_fmed3f(t[i - 1], t[i], x);
  t[0] = fmaxf(t[0], x);
}
// Two lists in order -> the K largest of both, in order: the larger ones of one and the other reversed, sorted by halves.
template <int K>
SP_DEV void merge_largest(float (&t)[K], const float (&o)[K]) {
#pragma unroll
  for (int i = 0; i < K; ++i) t[i] = fmaxf(t[i], o[K - 1 - i]);
#pragma unroll
  for (int d = K / 2; d > 0; d >>= 1)
#pragma unroll
    for (int i = 0; i < K; ++i)
      if (!(i & d)) {
        const float big = fmaxf(t[i], t[i + d]);
        t[i + d] = fminf(t[i], t[i + d]);
        t[i] = big;
      }
}
// The K largest of both halves' lists of a row.
template <int K>
SP_DEV void merge_halves(float (&t)[K], int g) {
  float other[K];
#pragma unroll
  for (int i = 0; i < K; ++i) {
    auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(t[i]), __float_as_uint(t[i]), false, false);
    other[i] = __uint_as_float(g ? r[0] : r[1]);
  }
  merge_largest<K>(t, other);
}
template <int K>
SP_DEV float place_of(const float (&t)[K], int n) {      // t[n - 1]
  float v = -INFINITY;
#pragma unroll
  for (int i = 0; i < K; ++i) v = i == n - 1 ? t[i] : v;
  return v;
}

// What a row wants: `need` of the blocks [first_block, own), and block `forced` (or -1) before all others.
struct SelRow { int own, need, forced; };
SP_DEV SelRow select_row_of(const BlockSelectArgs& a, int rh) {
  const int end = a.first_block + a.n_blocks;
  SelRow r = {end, a.top_k, -1};
  if (a.causal) {
    const int own = a.own0 + (int)((unsigned)(a.own_rest + rh % a.s_q) / (unsigned)a.block_len);
    if (own < end) r.own = own;
    if (own >= a.first_block && own < end) { r.forced = own; --r.need; }
  }
  if (r.need <= 0 || r.own < a.first_block) r.own = a.first_block;
  return r;
}
SP_DEV const bf16_t* select_q(const BlockSelectArgs& a, int b, int hk, int rh) {
  const int hl = rh / a.s_q, r = rh - hl * a.s_q;
  return a.q + (int64_t)b * a.q_stride_b + (int64_t)r * a.q_stride_s + (int64_t)(hk * a.group + hl) * a.q_stride_h;
}
SP_DEV uint32_t both_halves(uint32_t m) {
  auto r = __builtin_amdgcn_permlane32_swap(m, m, false, false);
  return r[0] | r[1];
}
// |q| of the lane's row (both halves of a wave have it); -1: all zeros.
template <int KS>
SP_DEV float row_norm(const bf16x8 (&q)[KS]) {
  float norm = 0.f;
  uint32_t any = 0;
#pragma unroll
  for (int ks = 0; ks < KS; ++ks) {
    const u32x4 w = __builtin_bit_cast(u32x4, q[ks]);
#pragma unroll
    for (int i = 0; i < 4; ++i) any |= w[i] & 0x7fff7fffu;
#pragma unroll
    for (int e = 0; e < 8; ++e) norm += (float)q[ks][e] * (float)q[ks][e];
  }
  norm = __builtin_sqrtf(xhalf_sum(norm));
  return both_halves(any) == 0u ? -1.f : norm;
}
// Whether all scores of a row are equal: a row of zeros on finite means (`most`: largest |mean|^2, infinite where one is not), means of zeros.
SP_DEV bool all_equal(float norm, uint32_t most, bool no_mean) { return (norm < 0.f && __uint_as_float(most) < INFINITY) || no_mean; }
// Whether n floats (a multiple of 4) are zeros; for all threads of a workgroup at once, and only where their squares vanish: not kept up in the walk,
// which has no registers to spare.
SP_DEV bool means_are_zero(const float* means, int64_t n, int tid, int threads) {
  uint32_t any = 0;
  for (int64_t i = 4 * tid; i < n; i += 4 * threads) {
    const u32x4 w = *reinterpret_cast<const u32x4*>(means + i);
    any |= (w[0] | w[1] | w[2] | w[3]) << 1;
  }
  return __syncthreads_or((int)(any != 0u)) == 0;
}
// What lies between and above: bounds that are not finite (a mean or a query that is not) or too small leave everything open.
template <int D>
SP_DEV void select_bounds(float t, float norm, uint32_t most, float* lo, float* hi) {
  const float mean = __builtin_sqrtf(__uint_as_float(most)), delta = (1.125f * D * 0x1p-23f + 0x1p-16f) * norm * mean;
  const bool clear = norm >= 0x1p-40f && mean >= 0x1p-40f && delta < INFINITY && fabsf(t) < INFINITY;
  *lo = clear ? t - 2.f * delta : -INFINITY;
  *hi = clear ? t + 2.f * delta : INFINITY;
}
// Bit n of a lane's mask: block n of a tile whose 16 scores of the lane's half are s (NaN counts as open).
SP_DEV uint32_t at_least(const f32x16& s, float lo, int g) {
  uint32_t m = 0;
#pragma unroll
  for (int i = 0; i < 16; ++i) m |= !(s[i] < lo) ? 1u << (8 * (i >> 2) + (i & 3)) : 0u;
  return m << (4 * g);
}
SP_DEV uint32_t above(const f32x16& s, float hi, int g) {
  uint32_t m = 0;
#pragma unroll
  for (int i = 0; i < 16; ++i) m |= s[i] > hi ? 1u << (8 * (i >> 2) + (i & 3)) : 0u;
  return m << (4 * g);
}
SP_DEV uint32_t blocks_below(int n) { return n <= 0 ? 0u : n >= 32 ? 0xffffffffu : (1u << n) - 1u; }      // bits of the tile's blocks before the n-th

template <int D>
SP_DEV double exact_score(const float* mean, const bf16_t* q) {
  double sum = 0;
#pragma unroll 8
  for (int e = 0; e < D / 4; ++e) {
    const f32x4 x = reinterpret_cast<const f32x4*>(mean)[e];
    const bf16x4 y = reinterpret_cast<const bf16x4*>(q)[e];
#pragma unroll
    for (int u = 0; u < 4; ++u) sum += (double)(float)y[u] * (double)x[u];
  }
  // NaN comes last: it counts as -infinity, and that as the lowest finite number (no finite score comes near it: at most D 2^128 2^128)
  return sum == sum ? __builtin_fmax(sum, -__DBL_MAX__) : -INFINITY;
}
SP_DEV double wave_max(double v) {
#pragma unroll
  for (int w = 1; w < 64; w <<= 1) {
    const double o = __shfl_xor(v, w, 64);
    v = o > v ? o : v;
  }
  return v;
}
// A row with more candidates than places, by one wave: scores in 64 bits of those that are not certain, the largest first, of equal ones the
// lower index.  The list (ascending) ends up with `need` entries.
template <int D>
SP_DEV void settle_row(uint32_t* list, int count, int places, int need, const bf16_t* q, const float* means, int first_block, int own, int lane) {
  if (count <= places) {
    constexpr int REGS = (kMaxTopK + 32 + 63) / 64;
    uint32_t c[REGS];
    double d[REGS];
    uint32_t open = 0, taken = 0;
    int room = need;
#pragma unroll
    for (int i = 0; i < REGS; ++i) {
      const int at = 64 * i + lane;
      c[i] = at < count ? list[at] : 0u;
      const bool unsure = at < count && (c[i] & kUnsure), sure = at < count && !(c[i] & kUnsure);
      open |= unsure ? 1u << i : 0u;
      taken |= sure ? 1u << i : 0u;
      room -= __popcll(__builtin_amdgcn_ballot_w64(sure));
      c[i] &= ~kUnsure;
      d[i] = unsure ? exact_score<D>(means + (int64_t)c[i] * D, q) : -INFINITY;
    }
    for (; room > 0; --room) {
      double best = -INFINITY;
#pragma unroll
      for (int i = 0; i < REGS; ++i)
        if (((open >> i) & 1u) && d[i] > best) best = d[i];
      best = wave_max(best);
      bool found = false;                            // (lanes ascend within a register, registers ascend)
#pragma unroll
      for (int i = 0; i < REGS; ++i) {
        const uint64_t eq = __builtin_amdgcn_ballot_w64(((open >> i) & 1u) && d[i] == best);
        if (!found && eq) {
          found = true;
          if (lane == __ffsll((unsigned long long)eq) - 1) { open &= ~(1u << i); taken |= 1u << i; }
        }
      }
    }
    __builtin_amdgcn_wave_barrier();
    int at = 0;
#pragma unroll
    for (int i = 0; i < REGS; ++i) {
      const bool in = (taken >> i) & 1u;
      const uint64_t mask = __builtin_amdgcn_ballot_w64(in);
      if (in) list[at + __popcll(mask & ((1ull << lane) - 1ull))] = c[i];
      at += __popcll(mask);
    }
  } else {
    // Every score once, 64 blocks at a time; lane n keeps the n-th of the `need` best so far (of equal ones the first stays ahead, so that equal
    // scores throughout cost no more than the first ones of them).
    double kept = -INFINITY, border = -INFINITY;     // border: of the last one
    int mine = 0x7fffffff, have = 0;
    for (int j0 = first_block; j0 < own; j0 += 64) {
      const int j = j0 + lane;
      const double s = j < own ? exact_score<D>(means + (int64_t)j * D, q) : -INFINITY;
      for (uint64_t m = __builtin_amdgcn_ballot_w64(j < own && (have < need || s > border)); m; m &= m - 1) {
        const int from = __ffsll((unsigned long long)m) - 1;
        const double x = __shfl(s, from, 64);
        if (have == need && !(x > border)) continue;
        const int pos = __popcll(__builtin_amdgcn_ballot_w64(lane < have && kept >= x));
        const double up = __shfl_up(kept, 1, 64);
        const int up_j = __shfl_up(mine, 1, 64);
        kept = lane > pos ? up : lane == pos ? x : kept;
        mine = lane > pos ? up_j : lane == pos ? j0 + from : mine;
        have = have < need ? have + 1 : need;
        border = __shfl(kept, need - 1, 64);
      }
    }
    int at = 0;                                      // ascending: each goes behind the smaller ones
    for (int n = 0; n < need; ++n) at += __shfl(mine, n, 64) < mine ? 1 : 0;
    __builtin_amdgcn_wave_barrier();
    if (lane < need) list[at] = (uint32_t)mine;
  }
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
}

// Many rows: 32 R rows a wave, four waves; means are split once for all of them, into two LDS slots, and a matrix operand that is read
// from there serves R rows sets (R = 2 where the lists are short: the LDS reads of R = 1 are half of a tile's time).
constexpr int select_sets(int k) { return k <= 16 ? 2 : 1; }
template <int D, int K>
constexpr size_t select_lds_bytes() { return (size_t)2 * 2 * 32 * D * 2 + (size_t)128 * select_sets(K) * select_places(K) * 4; }
template <int D, int K>
__global__ __launch_bounds__(256, 2) void block_select_kernel(const BlockSelectArgs a) {
  constexpr int KS = D / 16, PART = 32 * D * 2, SLOT = 2 * PART, PLACES = select_places(K), PER = D / 8 / 8;      // 16-byte chunks of a part a thread writes
  constexpr int R = select_sets(K), WROWS = 32 * R;
  extern __shared__ __attribute__((aligned(1024))) char smem[];
  __shared__ uint32_t most_s;                        // largest |mean|^2 (bits of a float; all are >= 0)
  __shared__ int last_s;
  const int tid = threadIdx.x, lane = tid & 63, g = lane >> 5, ql = lane & 31, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int hk = blockIdx.y, b = blockIdx.z, rows = a.group * a.s_q, row0 = blockIdx.x * 4 * WROWS + wave * WROWS;
  const float* const means = a.means + ((int64_t)b * a.n_kv_heads + hk) * a.blocks_total * D;
  if (tid == 0) { most_s = 0u; last_s = a.first_block; }
  SelRow want[R];
  bf16x8 q[R][KS];
  float norm[R];
#pragma unroll
  for (int r = 0; r < R; ++r) {
    const int rh = row0 + 32 * r + ql < rows ? row0 + 32 * r + ql : rows - 1;
    want[r] = select_row_of(a, rh);
    const bf16_t* p = select_q(a, b, hk, rh) + 8 * g;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) q[r][ks] = *reinterpret_cast<const bf16x8*>(p + 16 * ks);
  }
  __syncthreads();
#pragma unroll
  for (int r = 0; r < R; ++r) {
    norm[r] = row_norm<KS>(q[r]);
    atomicMax(&last_s, want[r].own);
  }
  __syncthreads();
  const int stop = __builtin_amdgcn_readfirstlane(last_s), nt = (stop - a.first_block + 31) / 32;
  uint32_t* const wave_lists = reinterpret_cast<uint32_t*>(smem + 2 * SLOT) + wave * WROWS * PLACES;

  f32x4 x[2 * PER];
  float most = 0.f;
  auto fetch = [&](int t) {
    const int j = a.first_block + t * 32 + tid / 8;
    const f32x4* mp = reinterpret_cast<const f32x4*>(means + (int64_t)(j < stop ? j : stop - 1) * D + tid % 8 * (D / 8));
#pragma unroll
    for (int i = 0; i < 2 * PER; ++i) x[i] = mp[i];
  };
  auto store = [&](int t) {
    float sq = 0.f;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      bf16x8 part[2];
      split_means(x[2 * i], x[2 * i + 1], part, sq);
#pragma unroll
      for (int p = 0; p < 2; ++p) *reinterpret_cast<bf16x8*>(smem + (t & 1) * SLOT + p * PART + tile_off<D>(tid / 8, tid % 8 * PER + i)) = part[p];
    }
#pragma unroll
    for (int w = 1; w < 8; w <<= 1) sq += __shfl_xor(sq, w, 64);
    most = sq == sq ? fmaxf(most, sq) : INFINITY;    // (a NaN anywhere: nothing is certain)
  };
  RpOffsets<D> lo_m;
  lo_m.init(lane, (int)lds_addr(smem));
  // walks the tiles; use(t, s): scores of tile t
  auto walk = [&](auto&& use) {
    fetch(0);
    store(0);
    __syncthreads();
    for (int t = 0; t < nt; ++t) {
      if (t + 1 < nt) fetch(t + 1);
      f32x16 s[R] = {};
#pragma unroll
      for (int p = 1; p >= 0; --p)
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) {
          const bf16x8 m = lds_rp<D>(lo_m, ks, p * PART);
#pragma unroll
          for (int r = 0; r < R; ++r) s[r] = mfma32(m, q[r][ks], s[r]);
        }
      use(t, s);
      lo_m.add((t & 1) ? -SLOT : SLOT);
      if (t + 1 < nt) store(t + 1);
      __syncthreads();
    }
    if (nt & 1) lo_m.add(-SLOT);
  };
  int count[R];
#pragma unroll
  for (int r = 0; r < R; ++r) count[r] = 0;
  if (nt > 0) {
    float top[R][K];
#pragma unroll
    for (int r = 0; r < R; ++r)
#pragma unroll
      for (int i = 0; i < K; ++i) top[r][i] = -INFINITY;
    walk([&](int t, f32x16 (&s)[R]) {
#pragma unroll
      for (int r = 0; r < R; ++r) {
        const int left = want[r].own - a.first_block - t * 32;      // blocks of the tile that compete for the row
        if (__builtin_amdgcn_ballot_w64(left < 32) != 0)
#pragma unroll
          for (int i = 0; i < 16; ++i) s[r][i] = 8 * (i >> 2) + (i & 3) < left - 4 * g ? s[r][i] : -INFINITY;
#pragma unroll
        for (int i = 0; i < 16; ++i) keep_largest<K>(top[r], s[r][i]);
      }
    });
    atomicMax(&most_s, __float_as_uint(most));
    __syncthreads();
    const bool no_mean = most_s == 0u && means_are_zero(means + (int64_t)a.first_block * D, (int64_t)(stop - a.first_block) * D, tid, 256);
    float lo[R], hi[R];
#pragma unroll
    for (int r = 0; r < R; ++r) {
      merge_halves<K>(top[r], g);
      select_bounds<D>(place_of<K>(top[r], want[r].need), norm[r], most_s, &lo[r], &hi[r]);
      if (want[r].own - a.first_block <= want[r].need) { lo[r] = -INFINITY; hi[r] = INFINITY; }      // no more than are wanted: all
    }
    walk([&](int t, f32x16 (&s)[R]) {
#pragma unroll
      for (int r = 0; r < R; ++r) {
        const uint32_t open = both_halves(at_least(s[r], lo[r], g)) & blocks_below(want[r].own - a.first_block - t * 32);
        const uint32_t certain = both_halves(above(s[r], hi[r], g));
        if (g == 0)
          for (uint32_t m = open; m; m &= m - 1) {
            const int n = __ffs(m) - 1;
            if (count[r] < PLACES) wave_lists[(32 * r + ql) * PLACES + count[r]] = (uint32_t)(a.first_block + t * 32 + n) | ((certain >> n) & 1u ? 0u : kUnsure);
            ++count[r];
          }
      }
    });
#pragma unroll
    for (int r = 0; r < R; ++r)
      if (all_equal(norm[r], most_s, no_mean) && count[r] > want[r].need) count[r] = want[r].need;      // the first ones
  }
#pragma unroll
  for (int r = 0; r < R; ++r) {
    const int first = row0 + 32 * r;
    uint32_t* const lists = wave_lists + 32 * r * PLACES;
    // rows with more candidates than places
    for (uint64_t m = __builtin_amdgcn_ballot_w64(g == 0 && count[r] > want[r].need && first + ql < rows); m; m &= m - 1) {
      const int from = __ffsll((unsigned long long)m) - 1;
      const int n = __builtin_amdgcn_readlane(count[r], from), need = __builtin_amdgcn_readlane(want[r].need, from), own = __builtin_amdgcn_readlane(want[r].own, from);
      settle_row<D>(lists + from * PLACES, n, PLACES, need, select_q(a, b, hk, first + from), means, a.first_block, own, lane);
    }
    const int have = count[r] < want[r].need ? count[r] : want[r].need;
    // the rows of the index, whole lines at a time
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
    const int n_rows = rows - first < 32 ? rows - first : 32;
    int32_t* const to = a.index + (((int64_t)b * a.n_kv_heads + hk) * rows + first) * a.top_k;
    for (int i0 = 0; i0 < n_rows * a.top_k; i0 += 64) {
      const int i = i0 + lane, row = i / a.top_k, slot = i - row * a.top_k, rr = row < 32 ? row : 31;
      const int n = __shfl(have, rr, 64), f = __shfl(want[r].forced, rr, 64);
      const uint32_t v = lists[rr * PLACES + (slot < PLACES ? slot : 0)];
      if (i < n_rows * a.top_k) to[i] = slot < n ? (int)(v & ~kUnsure) : slot == n && f >= 0 ? f : -1;
    }
  }
}

// Few rows (tokens): 32 a workgroup, whose eight waves share out the tiles; means go from memory through registers to the matrix unit.  The waves'
// lists meet in LDS, and so do the second walk's masks, a bit a block.  8 heads of each of 4 sequences on 511 blocks of means of 128, top_k 16: 21 us, of
// which the two tiles of scores of a wave take 8 (vector work of one compute unit), the joins 6.
constexpr int kFewWaves = 8, kFewTiles = 512;
// Tiles of a wave whose scores stay in registers for the second walk: two, or six where there are more and lists leave the registers (8 rows on 2048
// blocks, top_k 16: two 67 us, six 52; 2048 rows of 8 heads on 256 blocks, two tiles a wave: two 34 us, six 39).
constexpr int few_kept(int k, bool many) { return many && k <= 32 ? 6 : 2; }
template <int K>
constexpr int few_list_stride() { return K * 32 + 8; }              // floats of a wave's lists (eight banks on, so that a row's lists are spread)
template <int D, int K>
constexpr size_t select_few_lds_bytes(int tiles) {
  const size_t lists = (size_t)kFewWaves * few_list_stride<K>() * 4, masks = (size_t)tiles * 32 * 2 * 4 + 32 * select_places(K) * 4;
  return lists > masks ? lists : masks;
}
template <int D, int K, int KEPT>
__global__ __launch_bounds__(kFewWaves * 64, 2) void block_select_few_kernel(const BlockSelectArgs a) {
  constexpr int KS = D / 16, PLACES = select_places(K);
  extern __shared__ __attribute__((aligned(1024))) char smem[];
  __shared__ uint32_t most_s;
  __shared__ int last_s;
  __shared__ float border_s[32], norm_s[32];
  __shared__ int count_s[32];
  const int tid = threadIdx.x, lane = tid & 63, g = lane >> 5, ql = lane & 31, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int hk = blockIdx.y, b = blockIdx.z, rows = a.group * a.s_q, row0 = blockIdx.x * 32;
  const float* const means = a.means + ((int64_t)b * a.n_kv_heads + hk) * a.blocks_total * D;
  const int rh = row0 + ql < rows ? row0 + ql : rows - 1;
  if (tid == 0) { most_s = 0u; last_s = a.first_block; }
  bf16x8 q[KS];
  {
    const bf16_t* p = select_q(a, b, hk, rh) + 8 * g;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) q[ks] = *reinterpret_cast<const bf16x8*>(p + 16 * ks);
  }
  const SelRow want = select_row_of(a, rh);
  __syncthreads();
  if (tid < 32) atomicMax(&last_s, want.own);
  __syncthreads();
  const int stop = __builtin_amdgcn_readfirstlane(last_s), nt = (stop - a.first_block + 31) / 32;
  float most = 0.f;
  auto scores = [&](int t) {
    const int j = a.first_block + t * 32 + ql;
    const float* mp = means + (int64_t)(j < stop ? j : stop - 1) * D + 8 * g;
    float sq = 0.f;
    // (a sum for each of the parts: the parts of a step are used at once and need few registers)
    f32x16 x[2] = {};
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) {
      bf16x8 part[2];
      split_means(*reinterpret_cast<const f32x4*>(mp + 16 * ks), *reinterpret_cast<const f32x4*>(mp + 16 * ks + 4), part, sq);
#pragma unroll
      for (int p = 0; p < 2; ++p) x[p] = mfma32(part[p], q[ks], x[p]);
    }
    const f32x16 s = x[1] + x[0];
    sq = xhalf_sum(sq);
    most = sq == sq ? fmaxf(most, sq) : INFINITY;
    return s;
  };
  float top[K];
#pragma unroll
  for (int i = 0; i < K; ++i) top[i] = -INFINITY;
  auto offer = [&](const f32x16& s, int t) {
    const int left = want.own - a.first_block - t * 32 - 4 * g;
#pragma unroll
    for (int i = 0; i < 16; ++i) keep_largest<K>(top, 8 * (i >> 2) + (i & 3) < left ? s[i] : -INFINITY);
  };
  f32x16 kept[KEPT] = {};
#pragma unroll
  for (int i = 0; i < KEPT; ++i) {
    const int t = wave + i * kFewWaves;
    if (t < nt) { kept[i] = scores(t); offer(kept[i], t); }
  }
  for (int t = wave + KEPT * kFewWaves; t < nt; t += kFewWaves) offer(scores(t), t);
  {
    const float norm = row_norm<KS>(q);
    if (tid < 32) norm_s[tid] = norm;
  }
  atomicMax(&most_s, __float_as_uint(most));
  merge_halves<K>(top, g);
  float* const lists = reinterpret_cast<float*>(smem);      // [wave][place][row]
  if (g == 0)
#pragma unroll
    for (int i = 0; i < K; ++i) lists[wave * few_list_stride<K>() + i * 32 + ql] = top[i];
  __syncthreads();
  {
    // eight lists a row, a lane each, four rows a wave (lanes 32 .. 63 do the same)
    static_assert(kFewWaves == 8 && kFewWaves * 4 == 32, "four rows a wave");
    const int r = wave * 4 + ql / 8;
#pragma unroll
    for (int i = 0; i < K; ++i) top[i] = lists[ql % 8 * few_list_stride<K>() + i * 32 + r];
#pragma unroll
    for (int w = 1; w < 8; w <<= 1) {
      float other[K];
#pragma unroll
      for (int i = 0; i < K; ++i) other[i] = __shfl_xor(top[i], w, 64);
      merge_largest<K>(top, other);
    }
    const float v = place_of<K>(top, __shfl(want.need, r, 64));
    if (lane < 32 && lane % 8 == 0) border_s[r] = v;
  }
  __syncthreads();
  const bool no_mean = most_s == 0u && stop > a.first_block && means_are_zero(means + (int64_t)a.first_block * D, (int64_t)(stop - a.first_block) * D, tid, kFewWaves * 64);
  float lo, hi;
  select_bounds<D>(border_s[ql], norm_s[ql], most_s, &lo, &hi);
  if (want.own - a.first_block <= want.need) { lo = -INFINITY; hi = INFINITY; }
  uint32_t* const open_s = reinterpret_cast<uint32_t*>(smem);      // [tile][row]; certain ones behind them, then the rows' lists
  uint32_t* const certain_s = open_s + nt * 32;
  auto mark = [&](const f32x16& s, int t) {
    const uint32_t in = blocks_below(want.own - a.first_block - t * 32), open = both_halves(at_least(s, lo, g)) & in, certain = both_halves(above(s, hi, g)) & in;
    if (g == 0) { open_s[t * 32 + ql] = open; certain_s[t * 32 + ql] = certain; }
  };
#pragma unroll
  for (int i = 0; i < KEPT; ++i)
    if (wave + i * kFewWaves < nt) mark(kept[i], wave + i * kFewWaves);
  for (int t = wave + KEPT * kFewWaves; t < nt; t += kFewWaves) mark(scores(t), t);
  __syncthreads();
  uint32_t* const cand = certain_s + nt * 32;
  {
    // sixteen tiles of a row at a time, a lane each
    const int r = wave * 4 + lane / 16;
    int count = 0;
    for (int t0 = 0; t0 < nt; t0 += 16) {
      const int t = t0 + lane % 16;
      const uint32_t open = t < nt ? open_s[t * 32 + r] : 0u, certain = t < nt ? certain_s[t * 32 + r] : 0u;
      int at = __popc(open);
#pragma unroll
      for (int w = 1; w < 16; w <<= 1) {
        const int o = __shfl_up(at, w, 16);
        if (lane % 16 >= w) at += o;
      }
      const int all = __shfl(at, 15, 16);
      at += count - __popc(open);
      for (uint32_t m = open; m; m &= m - 1, ++at) {
        const int n = __ffs(m) - 1;
        if (at < PLACES) cand[r * PLACES + at] = (uint32_t)(a.first_block + t * 32 + n) | ((certain >> n) & 1u ? 0u : kUnsure);
      }
      count += all;
    }
    if (lane % 16 == 0) count_s[r] = count;
  }
  __syncthreads();
  for (int r = wave; r < 32 && row0 + r < rows; r += kFewWaves) {
    const int n = __builtin_amdgcn_readfirstlane(count_s[r]), need = __builtin_amdgcn_readlane(want.need, r), own = __builtin_amdgcn_readlane(want.own, r);
    if (n > need && !all_equal(norm_s[r], most_s, no_mean)) settle_row<D>(cand + r * PLACES, n, PLACES, need, select_q(a, b, hk, row0 + r), means, a.first_block, own, lane);
    const int forced = __builtin_amdgcn_readlane(want.forced, r), have = n < need ? n : need;
    if (lane < a.top_k)
      a.index[(((int64_t)b * a.n_kv_heads + hk) * rows + row0 + r) * a.top_k + lane] =
          lane < have ? (int)(cand[r * PLACES + lane] & ~kUnsure) : lane == have && forced >= 0 ? forced : -1;
  }
}

template <int D, int K>
static hipError_t launch_select_t(const BlockSelectArgs& a, bool few, hipStream_t st) {
  const int64_t rows = a.group * (int64_t)a.s_q;
  const unsigned heads = (unsigned)a.n_kv_heads, batch = (unsigned)a.batch;
  const int tiles = (a.n_blocks + 31) / 32;
  auto go_few = [&](auto kernel) {
    hipLaunchKernelGGL(kernel, dim3((unsigned)((rows + 31) / 32), heads, batch), dim3(kFewWaves * 64), (select_few_lds_bytes<D, K>(tiles)), st, a);
  };
  if (few) tiles > 2 * kFewWaves ? go_few(block_select_few_kernel<D, K, few_kept(K, true)>) : go_few(block_select_few_kernel<D, K, few_kept(K, false)>);
  else hipLaunchKernelGGL((block_select_kernel<D, K>), dim3((unsigned)((rows + 128 * select_sets(K) - 1) / (128 * select_sets(K))), heads, batch),
                          dim3(256), (select_lds_bytes<D, K>()), st, a);
  return hipGetLastError();
}
template <int D>
static hipError_t launch_select_d(const BlockSelectArgs& a, bool few, hipStream_t st) {
  if (a.top_k <= 8) return launch_select_t<D, 8>(a, few, st);
  if (a.top_k <= 16) return launch_select_t<D, 16>(a, few, st);
  if (a.top_k <= 32) return launch_select_t<D, 32>(a, few, st);
  return launch_select_t<D, 64>(a, few, st);
}
// The few-row kernel has four times the workgroups, and a walk an eighth as long, for calls whose 128-row workgroups would not fill the
// chip; its masks of a call's blocks have to fit LDS.  Means and selection, us with it and without, by 128-row workgroups: 8 of blocks of 512 at
// head_dim 128, 64 workgroups 23 and 57, 128 36 and 58, 255 60 and 59; where lists are long its joins cost more, 24 of blocks of 64 at head_dim 64:
// 64 26 and 50, 128 44 and 50, 255 80 and 54.
hipError_t launch_block_select(const BlockSelectArgs& a, int head_dim, int compute_units, hipStream_t st) {
  const int64_t wgs = (a.group * (int64_t)a.s_q + 127) / 128 * a.n_kv_heads * a.batch;
  const bool few = wgs < (a.top_k <= 16 ? compute_units : compute_units / 2) && a.n_blocks <= kFewTiles * 32;
  return head_dim == 128 ? launch_select_d<128>(a, few, st) : launch_select_d<64>(a, few, st);
}

template <int D, int K>
static hipError_t opt_in_select() {
  const hipFuncAttribute attr = hipFuncAttributeMaxDynamicSharedMemorySize;
  hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(&block_select_kernel<D, K>), attr, (int)select_lds_bytes<D, K>());
  if (e == hipSuccess)
    e = hipFuncSetAttribute(reinterpret_cast<const void*>(&block_select_few_kernel<D, K, few_kept(K, false)>), attr, (int)select_few_lds_bytes<D, K>(kFewTiles));
  if (e == hipSuccess)
    e = hipFuncSetAttribute(reinterpret_cast<const void*>(&block_select_few_kernel<D, K, few_kept(K, true)>), attr, (int)select_few_lds_bytes<D, K>(kFewTiles));
  return e;
}
template <int D>
static hipError_t opt_in_select_d() {
  hipError_t e = opt_in_select<D, 8>();
  if (e == hipSuccess) e = opt_in_select<D, 16>();
  if (e == hipSuccess) e = opt_in_select<D, 32>();
  return e == hipSuccess ? opt_in_select<D, 64>() : e;
}

// ------------------------------------------------------------------------------------ lists
// The rows of every block, in ascending order of (head of the group, row).  Three launches (one where rows are few): places of the rows of a chunk
// within the chunk, starts, entries.  Bound by a few trips to memory each: 8192 rows of 8 heads, 8 slots, 128 blocks: 7, 6 and 7 us
// (15 with delta).
//
// Chunks of kListRows rows have a bit per (block, row) in LDS: setting bits commutes, and a row's place among the chunk's rows of a block
// is a count of the bits below its own, so the lists are the same on every run.  (The index rows of a plane follow each other, and so do the
// slots of part_lse: entry i of the chunk is row i / top_k, slot i % top_k of both.)
constexpr int kListThreads = 512, kListWords = kListRows / 32, kListStride = kListWords + 1;      // (odd: a column of words is spread over the banks)
SP_HOST_DEV int list_lds_words(int n_blocks) { return (n_blocks < kListBlocks ? n_blocks : kListBlocks) * kListStride * 3 / 2 + 1; }
__global__ __launch_bounds__(kListThreads) void block_rank_kernel(const BlockArgs a) {
  extern __shared__ uint32_t bits[];                 // [blocks of the window][kListStride]; bits below each word behind them; the chunk's index
  const int tid = threadIdx.x, chunk = blockIdx.x, plane = blockIdx.y;
  const int rows = a.group * a.s_q, row0 = chunk * kListRows, n_rows = rows - row0 < kListRows ? rows - row0 : kListRows;
  const int64_t first = ((int64_t)plane * rows + row0) * a.top_k;      // (plane = batch index * kv heads + kv head)
  int32_t* index = reinterpret_cast<int32_t*>(bits + list_lds_words(a.n_blocks));
  float* valid = a.part_lse + first;                 // -inf: the slot has no block (and no result)
  uint16_t* rank = a.ranks + first;
  const int n_slots = n_rows * a.top_k;
  uint32_t* counts = a.counts + (int64_t)plane * a.n_blocks * count_stride(a.n_list_chunks) + chunk;
  const float per_row = 1.0f / (float)a.top_k;
  auto row_of = [&](int i) { return (int)(((float)i + 0.5f) * per_row); };      // i / top_k (i < 2^14: the half keeps it off the border)
  static_assert(kListRows * kMaxTopK <= 1 << 14 && kListRows * kMaxTopK <= 32 * kListThreads, "slots of a chunk: exact quotients, a bit each");
  // A row whose entries ascend up to its fill-up names no block twice; where all of the chunk's do (the selection's do) no slot has to look at the ones
  // before it.
  __shared__ uint32_t disorder[kListThreads / 64];
  bool unordered = false;
  for (int i = tid; i < n_slots; i += kListThreads) {
    const int j = a.index[first + i], before = a.index[first + (i > 0 ? i - 1 : 0)];
    index[i] = j;
    unordered |= j >= a.first_block && i != row_of(i) * a.top_k && (before < a.first_block || before >= j);
  }
  const uint64_t some = __builtin_amdgcn_ballot_w64(unordered);
  if ((tid & 63) == 0) disorder[tid >> 6] = some != 0;
  lds_barrier();
  uint32_t repeats = 0;                              // may there be any?
#pragma unroll
  for (int w = 0; w < kListThreads / 64; ++w) repeats |= disorder[w];
  uint32_t ok = 0;                                   // bit: this thread's slots
  for (int i = tid, u = 0; i < n_slots; i += kListThreads, ++u) {
    const int row = row_of(i);
    const bool v = block_slot_valid(a, index + row * a.top_k, i - row * a.top_k, a.q_offset + (row0 + row) % a.s_q, repeats != 0);
    valid[i] = v ? 0.f : -INFINITY;
    ok |= v ? 1u << u : 0u;
  }
  for (int w0 = 0; w0 < a.n_blocks; w0 += kListBlocks) {
    const int n = a.n_blocks - w0 < kListBlocks ? a.n_blocks - w0 : kListBlocks;
    uint16_t* below = reinterpret_cast<uint16_t*>(bits + n * kListStride);
    for (int i = tid; i < n * kListStride; i += kListThreads) bits[i] = 0u;
    lds_barrier();
    for (int i = tid, u = 0; i < n_slots; i += kListThreads, ++u) {
      const int j = index[i] - a.first_block - w0, row = row_of(i);
      if (((ok >> u) & 1u) && j >= 0 && j < n) atomicOr(&bits[j * kListStride + (row >> 5)], 1u << (row & 31));
    }
    lds_barrier();
    for (int j = tid; j < n; j += kListThreads) {
      uint32_t c = 0;
#pragma unroll
      for (int w = 0; w < kListWords; ++w) {
        below[j * kListStride + w] = (uint16_t)c;
        c += __popc(bits[j * kListStride + w]);
      }
      counts[(int64_t)(w0 + j) * count_stride(a.n_list_chunks)] = c;
    }
    lds_barrier();
    for (int i = tid, u = 0; i < n_slots; i += kListThreads, ++u) {
      const int j = index[i] - a.first_block - w0, row = row_of(i);
      if (((ok >> u) & 1u) && j >= 0 && j < n)
        rank[i] = (uint16_t)(below[j * kListStride + (row >> 5)] + __popc(bits[j * kListStride + (row >> 5)] & ((1u << (row & 31)) - 1u)));
    }
    lds_barrier();
  }
}

// delta = -sum_d dO O and lse2 = lse log2(e) (+inf: no key) of the rows of a plane, as the dense backward has them; D / 8 lanes a row.
template <int D>
SP_DEV void block_delta(const BlockArgs& a, int plane, int64_t gid) {
  constexpr int NC = D / 8;
  const int64_t rows = (int64_t)a.group * a.s_q, rh = gid / NC;
  const int c = (int)(gid - rh * NC), b = plane / a.n_kv_heads, hk = plane - b * a.n_kv_heads;
  if (rh >= rows) return;                            // (whole rows: the lanes of one leave together)
  const int hl = (int)(rh / a.s_q), h = hk * a.group + hl, r = (int)(rh - (int64_t)hl * a.s_q);
  const bf16x8 o = *reinterpret_cast<const bf16x8*>(static_cast<const bf16_t*>(a.out) + (int64_t)b * a.o_stride_b + (int64_t)r * a.o_stride_s + (int64_t)h * a.o_stride_h + c * 8);
  const bf16x8 g = *reinterpret_cast<const bf16x8*>(a.d_out + (int64_t)b * a.do_stride_b + (int64_t)r * a.do_stride_s + (int64_t)h * a.do_stride_h + c * 8);
  float acc = 0.f;
#pragma unroll
  for (int e = 0; e < 8; ++e) acc += (float)o[e] * (float)g[e];
#pragma unroll
  for (int w = NC / 2; w >= 1; w >>= 1) acc += __shfl_xor(acc, w, 64);
  if (c != 0) return;
  const int64_t at = plane * rows + rh;
  const float l = a.lse[at];
  a.delta[at] = -acc;
  a.lse2[at] = l == -INFINITY ? INFINITY : l * kLog2e;
}
// Row rh of a plane at place `pos` of block j's list: its entry, and with the first row of a tile or of a dk/dv part that too.  n_full: dk/dv items of
// full length of the plane.
template <bool DKDV>
SP_DEV void put_entry(const BlockArgs& a, int plane, int j, int rh, int slot, const BlockList& list, uint32_t pos, uint32_t n_full) {
  const int hl = rh / a.s_q;
  const uint32_t to = list.tile0 * kBlockTileRows + pos, r = (uint32_t)(rh - hl * a.s_q);
  a.entries[(int64_t)plane * a.item_cap * kBlockTileRows + to] = {r, (uint32_t)(hl << 6 | slot), r * (uint32_t)(a.q_stride_s / 8) + (uint32_t)hl * (uint32_t)(a.q_stride_h / 8),
                                                                   r * (uint32_t)(a.do_stride_s / 8) + (uint32_t)hl * (uint32_t)(a.do_stride_h / 8)};
  const uint32_t left = list.len - pos, block = (uint32_t)(a.first_block + j);
  if (pos % kBlockTileRows == 0)
    a.items[(int64_t)plane * a.item_cap + list.tile0 + pos / kBlockTileRows] = {(int)block, (int)to, (int)(left < kBlockTileRows ? left : kBlockTileRows), 0};
  if (DKDV && pos % (uint32_t)a.chunk_rows == 0) {
    const uint32_t c = pos / (uint32_t)a.chunk_rows;
    const uint32_t first = left >= (uint32_t)a.chunk_rows ? list.item0 + c * (uint32_t)a.n_sub : n_full + list.rest0;
    BlockItem* it = a.dkdv_items + (int64_t)plane * a.dkdv_cap + first;
    for (int s = 0; s < a.n_sub; ++s)
      it[s] = {(int)block * a.n_sub + s, (int)to, (int)(left < (uint32_t)a.chunk_rows ? left : (uint32_t)a.chunk_rows), list.parts ? (int)(list.part0 + c) : -1};
  }
}
// A slot a thread.  D > 0: behind fill_wgs workgroups those that make delta and lse2, which wait for nothing (a launch of their own was 5 to 10 us).
template <int D>
__global__ __launch_bounds__(256) void block_fill_kernel(const BlockArgs a, int fill_wgs) {
  constexpr bool dkdv = D > 0;
  const int plane = blockIdx.y, rows = a.group * a.s_q;
  if constexpr (D > 0) {
    if ((int)blockIdx.x >= fill_wgs) return block_delta<D>(a, plane, (int64_t)((int)blockIdx.x - fill_wgs) * 256 + threadIdx.x);
  }
  const int64_t n_slots = (int64_t)rows * a.top_k, i = (int64_t)blockIdx.x * 256 + threadIdx.x, at = plane * n_slots + i;
  if (i >= n_slots) return;
  const int j = a.index[at] - a.first_block;
  const uint32_t rank = a.ranks[at];                 // (read beside what says whether the slot counts, not behind it)
  if (a.part_lse[at] != 0.f) return;
  const int rh = (int)(i / a.top_k);
  const uint32_t pos = a.counts[((int64_t)plane * a.n_blocks + j) * count_stride(a.n_list_chunks) + rh / kListRows] + rank;
  put_entry<dkdv>(a, plane, j, rh, (int)(i - (int64_t)rh * a.top_k), a.lists[(int64_t)plane * a.n_blocks + j], pos, dkdv ? (uint32_t)a.n_dkdv_items[2 * plane + 1] : 0u);
}

// One workgroup a plane: counts of the chunks -> where each chunk's rows start in the block's list, list starts, tiles.
constexpr int kScanThreads = 1024;
SP_DEV uint32_t wave_scan(uint32_t v) {      // inclusive sum over the lanes up to this one
  v += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x111, 0xf, 0xf, false);
  v += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x112, 0xf, 0xf, false);
  v += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x114, 0xf, 0xf, false);
  v += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x118, 0xf, 0xf, false);
  v += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x142, 0xa, 0xf, false);
  v += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x143, 0xc, 0xf, false);
  return v;
}
// Exclusive sums of four numbers a thread over the workgroup, and the totals.
SP_DEV void scan_add(uint32_t (*tmp)[4], int tid, uint32_t (&v)[4], uint32_t (&total)[4]) {
  const int lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  uint32_t x[4];
  lds_barrier();
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    x[i] = wave_scan(v[i]);
    if (lane == 63) tmp[wave][i] = x[i];
  }
  lds_barrier();
  static_assert(kScanThreads / 64 == 16, "the waves' sums along the lanes");
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint32_t upto = wave_scan(lane < 16 ? tmp[lane][i] : 0u);
    total[i] = (uint32_t)__builtin_amdgcn_readlane((int)upto, 15);
    v[i] = x[i] - v[i] + (wave > 0 ? (uint32_t)__builtin_amdgcn_readlane((int)upto, wave - 1) : 0u);
  }
}
// Bin of a short dk/dv item of 0 < rest < chunk_rows rows, the longest first.
SP_DEV uint32_t bin_of(const BlockArgs& a, uint32_t rest) { return 63u - (uint32_t)(((uint64_t)rest * 64 - 1) / (uint32_t)a.chunk_rows); }
// The list of length `len` of every thread's block, behind those of the threads before it and `before` (short dk/dv items, tiles, dk/dv items of full
// length, partial sums); total: what all threads have of these.  bin_s: where the next short item of a bin goes.
SP_DEV BlockList place_list(const BlockArgs& a, bool dkdv, int tid, uint32_t len, const uint32_t (&before)[4], uint32_t (&total)[4], uint32_t (*tmp)[4], uint32_t* bin_s) {
  const uint32_t full = dkdv ? len / (uint32_t)a.chunk_rows : 0u, rest = dkdv && len > full * (uint32_t)a.chunk_rows ? 1u : 0u, parts = full + rest > 1 ? full + rest : 0u;
  uint32_t v[4] = {rest * (uint32_t)a.n_sub, (len + kBlockTileRows - 1) / kBlockTileRows, full * (uint32_t)a.n_sub, parts};
  scan_add(tmp, tid, v, total);
  const uint32_t rest0 = rest ? atomicAdd(&bin_s[bin_of(a, len - full * (uint32_t)a.chunk_rows)], 1u) * (uint32_t)a.n_sub : 0u;
  return {len, before[1] + v[1], before[2] + v[2], rest0, parts, before[3] + v[3]};
}
// Counts of the chunks of eight blocks -> where each chunk's rows start in its block's list, four chunks a lane, by one wave: blocks j0,
// j0 + step, .., whose lengths go to put_len.
template <class Len>
SP_DEV void chunk_starts(const BlockArgs& a, int plane, int j0, int step, int lane, Len&& put_len) {
  constexpr int PER = 8;
  const int nb = a.n_blocks, nc = a.n_list_chunks;
  uint32_t before[PER] = {};
  for (int c0 = 4 * lane; c0 - 4 * lane < nc; c0 += 256) {
    u32x4 v[PER];
#pragma unroll
    for (int p = 0; p < PER; ++p) {
      v[p] = u32x4{0, 0, 0, 0};
      if (j0 + p * step < nb && c0 < nc) v[p] = *reinterpret_cast<const u32x4*>(a.counts + ((int64_t)plane * nb + j0 + p * step) * count_stride(nc) + c0);
    }
#pragma unroll
    for (int p = 0; p < PER; ++p) {
#pragma unroll
      for (int u = 0; u < 4; ++u) v[p][u] = c0 + u < nc ? v[p][u] : 0u;
      const uint32_t sum = v[p][0] + v[p][1] + v[p][2] + v[p][3], upto = wave_scan(sum);
      uint32_t at = before[p] + upto - sum;
      u32x4 starts;
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        starts[u] = at;
        at += v[p][u];
      }
      if (j0 + p * step < nb && c0 < nc) *reinterpret_cast<u32x4*>(a.counts + ((int64_t)plane * nb + j0 + p * step) * count_stride(nc) + c0) = starts;
      before[p] += (uint32_t)__builtin_amdgcn_readlane((int)upto, 63);
    }
  }
#pragma unroll
  for (int p = 0; p < PER; ++p)
    if (lane == 0 && j0 + p * step < nb) put_len(j0 + p * step, before[p]);
}
// A launch of its own for them, 128 blocks a workgroup, where they are many: 4096 rows of 8 heads, this and the next kernel and the next alone, 2048
// blocks (2^18 counts) 10 and 40 us, 16384 blocks 39 and 333; the launch costs 4 to 6, and with 2^15 counts the next alone takes 6.
__global__ __launch_bounds__(kScanThreads) void block_starts_kernel(const BlockArgs a) {
  constexpr int WAVES = kScanThreads / 64;
  BlockList* const lists = a.lists + (int64_t)blockIdx.y * a.n_blocks;
  chunk_starts(a, blockIdx.y, (int)blockIdx.x * 8 * WAVES + __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), WAVES, threadIdx.x & 63,
               [&](int j, uint32_t n) { lists[j].len = n; });
}
constexpr int64_t kScanCounts = 1 << 16;         // counts that the one workgroup of the next kernel goes through by itself
// started: block_starts_kernel has run.
__global__ __launch_bounds__(kScanThreads) void block_scan_kernel(const BlockArgs a, int dkdv, int started) {
  constexpr int kLens = 8192;                                    // lengths that pass through LDS (more: through memory)
  __shared__ uint32_t tmp[kScanThreads / 64][4], len_s[kLens], bin_s[64];
  const int tid = threadIdx.x, lane = tid & 63, plane = blockIdx.x, nb = a.n_blocks;
  const bool in_lds = nb <= kLens && !started;
  BlockList* lists = a.lists + (int64_t)plane * nb;
  constexpr int WAVES = kScanThreads / 64;
  if (!started)
    for (int j0 = __builtin_amdgcn_readfirstlane(tid >> 6); j0 < nb; j0 += 8 * WAVES)
      chunk_starts(a, plane, j0, WAVES, lane, [&](int j, uint32_t n) {
        if (in_lds) len_s[j] = n;
        else lists[j].len = n;
      });
  if (in_lds) {
    lds_barrier();
  } else {
    __threadfence_block();
    __syncthreads();
  }
  // The short dk/dv items in descending order of length, to a 64th of the full one: the last ones to start are the shortest, and runs dealt out to
  // the XCDs in turn give all of them as much.  (Which of two of one bin goes first is left open: it changes no sum.)
  auto length_of = [&](int j) { return in_lds ? len_s[j] : lists[j].len; };
  if (dkdv) {
    if (tid < 64) bin_s[tid] = 0u;
    lds_barrier();
    for (int j = tid; j < nb; j += kScanThreads) {
      const uint32_t rest = length_of(j) % (uint32_t)a.chunk_rows;
      if (rest) atomicAdd(&bin_s[bin_of(a, rest)], 1u);
    }
    lds_barrier();
    if (tid < 64) {
      const uint32_t n = bin_s[tid];
      bin_s[tid] = wave_scan(n) - n;
    }
    lds_barrier();
  }
  uint32_t before[4] = {0, 0, 0, 0};                             // short dk/dv items, tiles, dk/dv items of full length, partial sums of the blocks before
  for (int j0 = 0; j0 < nb; j0 += kScanThreads) {
    const int j = j0 + tid;
    uint32_t total[4];
    const BlockList list = place_list(a, dkdv != 0, tid, j < nb ? length_of(j) : 0u, before, total, tmp, bin_s);
    if (j < nb) lists[j] = list;
#pragma unroll
    for (int i = 0; i < 4; ++i) before[i] += total[i];
  }
  if (tid == 0) {
    a.n_items[plane] = (int)before[1];
    if (dkdv && plane == 0) *a.inf = INFINITY;
    if (dkdv) { a.n_dkdv_items[2 * plane] = (int)(before[2] + before[0]); a.n_dkdv_items[2 * plane + 1] = (int)before[2]; }
  }
}

// The three in one workgroup a plane, with what passes between them in LDS: for planes of so few rows that launches cost more than it does.  Calls of
// 8 heads on one, us with it and with three launches, forward and backward: 64 rows, 8 of 63 blocks of 64 24 and 30, 51 and 56; 64 rows, 16 of 234 blocks
// of 256 34 and 40, 93 and 97; 200 rows, 2 of 128 blocks of 64 20 and 26, 43 and 48; 128 rows, 8 of 64 blocks of 64 32 and 34, 57 both; 256 rows, 4 of 59 blocks of 512 35 both, 88 and 84; 250 rows, 8 of 126
// blocks of 128 39 and 33, 78 and 66.
// D > 0 as in block_fill_kernel, behind the first workgroup of a plane.
constexpr int kOneListSlots = 8, kOneListRows = 2048;      // slots a thread; rows of a plane
constexpr int64_t kOneListWork = 1 << 23;                   // rows times slots: a thread's slots, and the words of a block's bits behind each other
SP_HOST_DEV int one_list_stride(int rows) { return ((rows + 31) / 32) | 1; }
SP_HOST_DEV size_t one_list_lds_bytes(int rows, int n_blocks) { return (size_t)n_blocks * ((size_t)one_list_stride(rows) * 6 + sizeof(BlockList)) + 16; }
constexpr size_t kOneListLds = 128 * 1024;
template <int D>
__global__ __launch_bounds__(kScanThreads) void block_lists_kernel(const BlockArgs a) {
  constexpr bool dkdv = D > 0;
  const int tid = threadIdx.x, lane = tid & 63, plane = blockIdx.y, rows = a.group * a.s_q, nb = a.n_blocks;
  if constexpr (D > 0) {
    if (blockIdx.x > 0) return block_delta<D>(a, plane, (int64_t)((int)blockIdx.x - 1) * kScanThreads + tid);
  }
  extern __shared__ __attribute__((aligned(16))) char smem[];
  __shared__ uint32_t tmp[kScanThreads / 64][4], bin_s[64], disorder[kScanThreads / 64];
  const int stride = one_list_stride(rows), words = (rows + 31) / 32, n_slots = rows * a.top_k;
  BlockList* const list_s = reinterpret_cast<BlockList*>(smem);
  uint32_t* const bits = reinterpret_cast<uint32_t*>(list_s + nb);
  uint16_t* const below = reinterpret_cast<uint16_t*>(bits + nb * stride);
  const int32_t* const index = a.index + (int64_t)plane * n_slots;
  float* const valid = a.part_lse + (int64_t)plane * n_slots;
  const float per_row = 1.0f / (float)a.top_k;
  auto row_of = [&](int i) { return (int)(((float)i + 0.5f) * per_row); };      // (as in block_rank_kernel)
  static_assert(kOneListSlots * kScanThreads <= 1 << 14, "exact quotients");
  int j[kOneListSlots];                              // blocks of this thread's slots, from the range's first on; -1: none
  bool unordered = false;
#pragma unroll
  for (int u = 0; u < kOneListSlots; ++u) {
    const int i = tid + u * kScanThreads;
    j[u] = -1;
    if (i >= n_slots) continue;
    const int x = index[i], before = index[i > 0 ? i - 1 : 0];
    unordered |= x >= a.first_block && i != row_of(i) * a.top_k && (before < a.first_block || before >= x);
    j[u] = x < a.first_block || x - a.first_block >= nb ? -1 : x - a.first_block;
  }
  for (int i = tid; i < nb * stride; i += kScanThreads) bits[i] = 0u;
  if (tid < 64) bin_s[tid] = 0u;
  const uint64_t some = __builtin_amdgcn_ballot_w64(unordered);
  if (lane == 0) disorder[tid >> 6] = some != 0;
  lds_barrier();
  uint32_t repeats = 0;
#pragma unroll
  for (int w = 0; w < kScanThreads / 64; ++w) repeats |= disorder[w];
#pragma unroll
  for (int u = 0; u < kOneListSlots; ++u) {
    const int i = tid + u * kScanThreads, row = row_of(i);
    if (i >= n_slots) continue;
    if (j[u] >= 0 && !block_slot_valid(a, index + row * a.top_k, i - row * a.top_k, a.q_offset + row % a.s_q, repeats != 0)) j[u] = -1;
    valid[i] = j[u] >= 0 ? 0.f : -INFINITY;
    if (j[u] >= 0) atomicOr(&bits[j[u] * stride + (row >> 5)], 1u << (row & 31));
  }
  lds_barrier();
  uint32_t len = 0;                                  // of block tid
  if (tid < nb)
    for (int w = 0; w < words; ++w) {
      below[tid * stride + w] = (uint16_t)len;
      len += __popc(bits[tid * stride + w]);
    }
  if (dkdv) {
    const uint32_t rest = len % (uint32_t)a.chunk_rows;
    if (rest) atomicAdd(&bin_s[bin_of(a, rest)], 1u);
    lds_barrier();
    if (tid < 64) {
      const uint32_t n = bin_s[tid];
      bin_s[tid] = wave_scan(n) - n;
    }
    lds_barrier();
  }
  uint32_t total[4];
  const uint32_t before[4] = {0, 0, 0, 0};
  const BlockList list = place_list(a, dkdv, tid, len, before, total, tmp, bin_s);
  if (tid < nb) {
    list_s[tid] = list;
    a.lists[(int64_t)plane * nb + tid] = list;
  }
  if (tid == 0) {
    a.n_items[plane] = (int)total[1];
    if (dkdv && plane == 0) *a.inf = INFINITY;
    if (dkdv) { a.n_dkdv_items[2 * plane] = (int)(total[2] + total[0]); a.n_dkdv_items[2 * plane + 1] = (int)total[2]; }
  }
  lds_barrier();
#pragma unroll
  for (int u = 0; u < kOneListSlots; ++u) {
    const int i = tid + u * kScanThreads, row = row_of(i);
    if (j[u] < 0) continue;
    const int at = j[u] * stride + (row >> 5);
    put_entry<dkdv>(a, plane, j[u], row, i - row * a.top_k, list_s[j[u]], below[at] + __popc(bits[at] & ((1u << (row & 31)) - 1u)), total[2]);
  }
}

static size_t list_lds_bytes(const BlockArgs& a) { return ((size_t)list_lds_words(a.n_blocks) + (size_t)kListRows * a.top_k) * 4; }
hipError_t launch_block_lists(const BlockArgs& a, int head_dim, bool is_bwd, hipStream_t st) {
  const unsigned planes = (unsigned)(a.batch * a.n_kv_heads);
  const int64_t rows = (int64_t)a.group * a.s_q, fill = (rows * a.top_k + 255) / 256, delta = is_bwd ? (rows * (head_dim / 8) + 255) / 256 : 0;
  if (rows <= kOneListRows && rows * a.top_k <= kOneListSlots * kScanThreads && rows * rows * a.top_k <= kOneListWork && a.n_blocks <= kScanThreads && one_list_lds_bytes((int)rows, a.n_blocks) <= kOneListLds) {
    const size_t lds = one_list_lds_bytes((int)rows, a.n_blocks);
    const dim3 grid((unsigned)(1 + (delta * 256 + kScanThreads - 1) / kScanThreads), planes), block(kScanThreads);
    if (!is_bwd) hipLaunchKernelGGL(block_lists_kernel<0>, grid, block, lds, st, a);
    else if (head_dim == 128) hipLaunchKernelGGL(block_lists_kernel<128>, grid, block, lds, st, a);
    else hipLaunchKernelGGL(block_lists_kernel<64>, grid, block, lds, st, a);
    return hipGetLastError();
  }
  hipLaunchKernelGGL(block_rank_kernel, dim3((unsigned)a.n_list_chunks, planes), dim3(kListThreads), list_lds_bytes(a), st, a);
  const bool starts = (int64_t)a.n_blocks * a.n_list_chunks > kScanCounts;
  if (starts) hipLaunchKernelGGL(block_starts_kernel, dim3((unsigned)((a.n_blocks + kScanThreads / 8 - 1) / (kScanThreads / 8)), planes), dim3(kScanThreads), 0, st, a);
  hipLaunchKernelGGL(block_scan_kernel, dim3(planes), dim3(kScanThreads), 0, st, a, is_bwd ? 1 : 0, starts ? 1 : 0);
  auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, dim3((unsigned)(fill + delta), planes), dim3(256), 0, st, a, (int)fill); };
  if (!is_bwd) go(block_fill_kernel<0>);
  else if (head_dim == 128) go(block_fill_kernel<128>);
  else go(block_fill_kernel<64>);
  return hipGetLastError();
}

hipError_t opt_in_block_select_kernels() {
  hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(&block_rank_kernel), hipFuncAttributeMaxDynamicSharedMemorySize,
                                     (list_lds_words(kListBlocks) + kListRows * kMaxTopK) * 4);
  const auto lists = [](const void* kernel) { return hipFuncSetAttribute(kernel, hipFuncAttributeMaxDynamicSharedMemorySize, (int)kOneListLds); };
  if (e == hipSuccess) e = lists(reinterpret_cast<const void*>(&block_lists_kernel<0>));
  if (e == hipSuccess) e = lists(reinterpret_cast<const void*>(&block_lists_kernel<64>));
  if (e == hipSuccess) e = lists(reinterpret_cast<const void*>(&block_lists_kernel<128>));
  if (e == hipSuccess) e = opt_in_select_d<128>();
  return e == hipSuccess ? opt_in_select_d<64>() : e;
}

}  // namespace slimpipe
