// Eviction from a key/value cache in 8 bits: the attention weight that every key gathers, the choice of the rows to keep, and the move of these rows to another
// cache.
#include "kv8_values.hpp"
#include "row_tile.hpp"

namespace slimpipe {

// ------------------------------------------------------------------------------------ weights
// weight_j = decay * previous_j + sum over the rows r of the kv head's query heads that see j of exp(scale q_r . k_j - lse_r): the scores once more, an exponential
// and a sum, no second product.
SP_DEV void put_weight(const Kv8WeightArgs& a, int64_t plane, int64_t key, float sum) {
  const int64_t at = plane * a.capacity + key;
  a.weights[at] = a.previous ? __builtin_fmaf(a.decay, a.previous[at], sum) : sum;
}
// lse of a row in log2 units, where exp2(score - that) is 0 for rows that saw nothing, if the score is finite.  Queries of such a row (a padded one, perhaps), or
// keys that it alone sees, may not be: it is masked for every key as well.
SP_DEV float row_norm(float lse) { return lse == -INFINITY ? INFINITY : lse * kLog2e; }

// Tokens: at most 16 SETS rows of a plane.  S^T = K Q^T as in the attention of tokens (kv8.hip): codes go from memory to the matrix unit, a lane holds one row's
// scores with four keys of 16, and the sum over the rows is one over 16 lanes.  A wave takes every fourth (second) step of 32 keys of its head, codes of the next DEPTH
// steps under way.
template <int D, int SETS>
__global__ __launch_bounds__(256, 2) void kv8_weights_few_kernel(const Kv8WeightArgs a) {
  constexpr int NP = D / 64, W = 2 * NP, DEPTH = 2;
  const Kv8Cache& kv = a.cache;
  const int lane = threadIdx.x & 63, h4 = lane >> 4, ql = lane & 15, wave_u = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int hw = kv8_heads_wg(kv.n_kv_heads), subs = 4 / hw, sub = wave_u / hw;
  const int rows = a.group * a.s_q, head_sets = kv.n_kv_heads / hw, planes = a.batch * head_sets;
  const int per = 8 * planes, first = (int)blockIdx.x / per * 8, i0 = (int)blockIdx.x % per, n = a.n_parts - first < 8 ? a.n_parts - first : 8;
  const int part_i = first + i0 % n, plane = i0 / n;
  if (plane >= planes) return;
  const int b = plane / head_sets, hk = (plane - b * head_sets) * hw + wave_u % hw;
  const int64_t plane_out = (int64_t)b * kv.n_kv_heads + hk;
  const int64_t lo = a.kv_begin + (int64_t)part_i * a.part_keys;
  const int64_t hi = lo + a.part_keys < a.kv_end ? lo + a.part_keys : a.kv_end;
  const int n_keys = hi > lo ? (int)(hi - lo) : 0, nt = (n_keys + 31) / 32;

  bf16x8 q[SETS][W];
  float norm[SETS];
  int see_rel[SETS];
#pragma unroll
  for (int r = 0; r < SETS; ++r) {
    const int rh = 16 * r + ql;
    const PlaneRow my = plane_row(a.s_q, a.group, hk, rh < rows ? rh : rows - 1);
    const bf16_t* qp = a.q + (int64_t)b * a.q_stride_b + (int64_t)my.r * a.q_stride_s + (int64_t)my.h * a.q_stride_h + 16 * h4;
#pragma unroll
    for (int j = 0; j < W; ++j) q[r][j] = *reinterpret_cast<const bf16x8*>(qp + 64 * (j / 2) + 8 * (j % 2));
    const float lse = a.lse[((int64_t)b * a.n_q_heads + my.h) * a.s_q + my.r];      // (behind the last row: that row once more, taken away by its norm)
    norm[r] = rh < rows ? row_norm(lse) : INFINITY;
    const int64_t see = (a.causal && a.q_offset + my.r < hi - 1 ? a.q_offset + my.r : hi - 1) - lo;
    see_rel[r] = see < -1 || lse == -INFINITY ? -1 : (int)see;
  }
  int min_see = see_rel[0];
#pragma unroll
  for (int r = 1; r < SETS; ++r) min_see = min_see < see_rel[r] ? min_see : see_rel[r];

  const int64_t base = (int64_t)b * kv.stride_b + (int64_t)hk * kv.stride_h + lo * kv.stride_s + 16 * h4;
  // (the sums of earlier calls come along with the codes: a load of its own at the end of a step would wait for all that is under way)
  const int64_t out0 = plane_out * a.capacity + lo + 4 * h4 + ql;      // entry of the key whose sum the lane writes, ql < 4
  struct Step { u32x4 k[2][NP]; uint32_t ks[2]; float before[2]; };
  auto fetch = [&](Step& s, int t) {
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      s.before[u] = 0.f;
      if (a.previous && ql < 4 && t * 32 + 16 * u + 4 * h4 + ql < n_keys) s.before[u] = a.previous[out0 + t * 32 + 16 * u];
      int key = t * 32 + 16 * u + ql;
      key = key < n_keys ? key : n_keys - 1;                     // (keys behind the last are not read)
      const int64_t at = base + (int64_t)key * kv.stride_s;
#pragma unroll
      for (int p = 0; p < NP; ++p) s.k[u][p] = *reinterpret_cast<const u32x4*>(kv.k.codes + at + 64 * p);
      s.ks[u] = kv.k.scales[kv8_scale_at(kv, b, lo + key, hk)];
    }
  };
  auto work = [&](Step& st, int t, int next) {
    f32x4 s[SETS][2];
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      const float ks = kv8_scale(st.ks[u]);
#pragma unroll
      for (int r = 0; r < SETS; ++r) s[r][u] = f32x4{0, 0, 0, 0};
#pragma unroll
      for (int j = 0; j < W; ++j) {
        const bf16x8 k8 = kv8_values(st.k[u][j / 2][j % 2 * 2], st.k[u][j / 2][j % 2 * 2 + 1], ks);
#pragma unroll
        for (int r = 0; r < SETS; ++r) s[r][u] = mfma16(k8, q[r][j], s[r][u]);
      }
    }
    const float before[2] = {st.before[0], st.before[1]};
    if (next < nt) fetch(st, next);
    const bool masked = __builtin_amdgcn_ballot_w64(min_see < t * 32 + 31) != 0;
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      float sum[4] = {0, 0, 0, 0};
#pragma unroll
      for (int r = 0; r < SETS; ++r)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float p = exp2_fast(__builtin_fmaf(s[r][u][i], a.scale_log2e, -norm[r]));
          sum[i] += masked && t * 32 + 16 * u + 4 * h4 + i > see_rel[r] ? 0.f : p;
        }
#pragma unroll
      for (int i = 0; i < 4; ++i) sum[i] = sixteen_sum(sum[i]);
      const float mine = ql == 0 ? sum[0] : ql == 1 ? sum[1] : ql == 2 ? sum[2] : sum[3];
      const int key = t * 32 + 16 * u + 4 * h4 + ql;
      if (ql < 4 && key < n_keys) a.weights[out0 + t * 32 + 16 * u] = __builtin_fmaf(a.decay, before[u], mine);
    }
  };
  if (sub >= nt) return;
  Step s[DEPTH];
#pragma unroll
  for (int i = 0; i < DEPTH; ++i)
    if (sub + i * subs < nt) fetch(s[i], sub + i * subs);
  for (int t = sub; t < nt; t += DEPTH * subs)
#pragma unroll
    for (int i = 0; i < DEPTH; ++i)
      if (t + i * subs < nt) work(s[i], t + i * subs, t + (i + DEPTH) * subs);
}

// Slices: a workgroup has 256 keys, 64 a wave, converted once and kept in registers, and walks the rows that see any of them (head by head, without the
// rows before its first key), or one part of them, in tiles of 128 through a ring of two in LDS.
//   S^T = K Q^T        A = K in registers, B = rows of Q from LDS: a lane has one row and 32 keys of a block of 32 rows
//   sums               p = exp2(c s - norm) added in place: the lane's sums over its rows, over the lanes at the end
// A pair costs the vector unit three instructions, one of them an exponential, beside 2 D flop: both units have about the same to do at D = 128, twice
// as much the vector unit at 64.  So the scores of a block of 32 rows are computed while the exponentials of the block before are taken, instruction by instruction.
// 4096 rows of 8 heads on 32768 keys of 128: 247 to 259 us, 1.0 PFLOP/s, on machines whose 8192^3 bf16 product runs at 1405 TFLOP/s, 283 on one of 1245.  (On the former:
// with the exponentials behind the matrix instructions of the same block 274; tiles of 64 rows in a ring of three 244, but 368 and 318 us for 16384 rows of 4 heads of 64 on
// 32768 keys; one pipeline over the four blocks of a tile 262: spills.  All but the matrix instructions 175 us, all but the exponentials 215: the two do not overlap
// enough.  At head_dim 64 all but the matrix instructions 300 of 328.)
constexpr int kWeightKeys = kv8_weight_keys(), kWeightRows = 128, kWeightRing = 2;
template <int D>
constexpr size_t kv8_weights_lds_bytes() { return (size_t)kWeightRing * kWeightRows * (D * 2 + 4); }

template <int D>
__global__ __launch_bounds__(256, 2) void kv8_weights_kernel(const Kv8WeightArgs a) {
  constexpr int KS = D / 16, TILE = kWeightRows * D * 2, BLOCKS = kWeightRows / 32, NC = D / 8, PASSES = kWeightRows / (4 * (64 / NC));      // copies of a wave a tile
  extern __shared__ __attribute__((aligned(1024))) char smem[];
  const Kv8Cache& kv = a.cache;
  const int tid = threadIdx.x, lane = tid & 63, g = lane >> 5, wave_u = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int key_blocks = (int)((a.kv_end - a.kv_begin + kWeightKeys - 1) / kWeightKeys);
  const int planes = a.batch * kv.n_kv_heads;
  const int item = xcd_run(blockIdx.x, key_blocks * planes * a.n_parts);      // (plane, part, key block): an XCD's workgroups read the same rows
  if (item < 0) return;
  const int pp = item / key_blocks, kb_i = item - pp * key_blocks, plane = pp / a.n_parts, part_i = pp - plane * a.n_parts;
  const int b = plane / kv.n_kv_heads, hk = plane - b * kv.n_kv_heads;
  const int64_t key0 = a.kv_begin + (int64_t)kb_i * kWeightKeys, wave_key0 = key0 + 64 * wave_u;

  // rows r_min .. s_q - 1 of every head of the group see a key of the workgroup; this part's tiles of them
  int64_t r_first = a.causal ? key0 - a.q_offset : 0;
  r_first = r_first < 0 ? 0 : r_first;
  const int r_min = r_first < a.s_q ? (int)r_first : a.s_q, vis = a.s_q - r_min;
  const int rows = vis * a.group, tiles = (rows + kWeightRows - 1) / kWeightRows;
  const int t0 = (int)((int64_t)tiles * part_i / a.n_parts), t1 = (int)((int64_t)tiles * (part_i + 1) / a.n_parts);

  f32x16 acc[2];
#pragma unroll
  for (int kb = 0; kb < 2; ++kb)
#pragma unroll
    for (int i = 0; i < 16; ++i) acc[kb][i] = 0.f;

  if (t0 < t1) {
    const unsigned lds = lds_addr(smem);
    const bf16_t* const q_base = a.q + (int64_t)b * a.q_stride_b + (int64_t)hk * a.group * a.q_stride_h;
    const float* const lse = a.lse + ((int64_t)b * a.n_q_heads + (int64_t)hk * a.group) * a.s_q;
    const uint32_t row_bytes = (uint32_t)a.q_stride_s * 2;
    // Row rh of those that the workgroup walks is row r_min + rh % vis of head rh / vis.  A tile of one head, most of them, is copied from a uniform base.
    // The rows' lse come along, behind the ring, and into registers, where they are asked for rows that the tile's fast path would not leave out.
    float ahead[kWeightRows / 64];
    constexpr int RPP = 64 / NC;                                      // rows of a copy instruction
    auto copy_tile = [&](int t) {
      const unsigned to = lds + (t % kWeightRing) * TILE, to_lse = lds + kWeightRing * TILE + (t % kWeightRing) * kWeightRows * 4;
      const int rh0 = t * kWeightRows, h0 = __builtin_amdgcn_readfirstlane((int)((unsigned)rh0 / (unsigned)vis)), r0 = rh0 - h0 * vis;
      if (r0 + kWeightRows <= vis) {
        const bf16_t* src = q_base + (int64_t)h0 * a.q_stride_h + (int64_t)(r_min + r0) * a.q_stride_s;
#pragma unroll
        for (int n = 0; n < kWeightRows; n += 64) {
          const float* from = uniform_ptr(lse + (int64_t)h0 * a.s_q + r_min + r0 + n);
          dma4(from, (uint32_t)lane * 4, __builtin_amdgcn_readfirstlane(to_lse + n * 4));
          ahead[n / 64] = from[lane];
        }
#pragma unroll
        for (int n = 0; n < PASSES; ++n) WaveDma<D, kWeightRows>::copy_pass(to, uniform_ptr(src), row_bytes, kWeightRows, lane, wave_u * PASSES + n);
        return;
      }
      auto at = [&](int rh, int& hl) {
        rh = rh < rows ? rh : rows - 1;
        hl = (int)((unsigned)rh / (unsigned)vis);
        return rh - hl * vis + r_min;
      };
      int hl;
#pragma unroll
      for (int n = 0; n < kWeightRows; n += 64) {
        const int rl = at(rh0 + n + lane, hl);
        dma4_at(lse + (int64_t)hl * a.s_q + rl, to_lse + n * 4);
        ahead[n / 64] = lse[(int64_t)hl * a.s_q + rl];
      }
#pragma unroll
      for (int n = 0; n < PASSES; ++n) {
        const int pass = wave_u * PASSES + n, r = at(rh0 + pass * RPP + lane / NC, hl);
        dma16_at(q_base + (int64_t)hl * a.q_stride_h + (int64_t)r * a.q_stride_s + WaveDma<D, kWeightRows>::chunk_off(lane, pass) / 2, to + pass * 1024);
      }
    };
    copy_tile(t0);
    // K in registers.  The contraction may take head_dim in any order: lane group g has elements 32 j + 16 g .. + 15 in steps 2 j and 2 j + 1, one load.
    bf16x8 k[2][KS];
#pragma unroll
    for (int kb = 0; kb < 2; ++kb) {
      int64_t key = wave_key0 + 32 * kb + (lane & 31);
      key = key < a.kv_end ? key : a.kv_end - 1;                  // (keys behind the last are not read)
      const float unit = kv8_scale(kv.k.scales[kv8_scale_at(kv, b, key, hk)]);
      const uint8_t* p = kv.k.codes + (int64_t)b * kv.stride_b + key * kv.stride_s + (int64_t)hk * kv.stride_h + 16 * g;
      u32x4 c[KS / 2];
#pragma unroll
      for (int j = 0; j < KS / 2; ++j) c[j] = *reinterpret_cast<const u32x4*>(p + 32 * j);
#pragma unroll
      for (int j = 0; j < KS / 2; ++j) {
        k[kb][2 * j] = kv8_values(c[j][0], c[j][1], unit);
        k[kb][2 * j + 1] = kv8_values(c[j][2], c[j][3], unit);
      }
    }
    // the rows of Q to go with it: step 2 j + e reads chunk 4 j + 2 g + e, which the swizzle puts at that of chunk 2 g with 4 j + e in bits 4 ..
    int lo_q = (int)lds + tile_off<D>(lane & 31, 2 * g);
    auto q_rows = [&](int ks) { return *lds_ptr<bf16x8>(lo_q ^ ((ks / 2 * 4 + ks % 2) << 4), 0); };
    // norm of the lane's row in a block of 32 (rows behind the last: one that takes all weight away)
    auto norm_of = [&](int block) {
      const float x = *lds_ptr<float>((int)lds + kWeightRing * TILE + (block / BLOCKS % kWeightRing) * kWeightRows * 4 + (block % BLOCKS) * 128 + (lane & 31) * 4, 0);
      return block * 32 + (lane & 31) < rows ? row_norm(x) : INFINITY;
    };
    // Does every row of tile t see every key of the wave?  (Its first row decides, or, where it holds the end of a head, the first of the next.)
    const int64_t rel = a.q_offset - wave_key0 + r_min;
    auto unmasked = [&](int t) {
      const int rh0 = t * kWeightRows, r0 = rh0 - __builtin_amdgcn_readfirstlane((int)((unsigned)rh0 / (unsigned)vis)) * vis;
      return !a.causal || rel + (r0 + kWeightRows <= vis ? r0 : 0) >= 63;
    };
    // Scores of a block into s[x]; with `take_other` the exponentials of the scores s[1 - x], of rows with norm `other`, between the matrix instructions.
    f32x16 s[2][2];
    auto scores = [&](auto x_, bool take_other, float other) {
      constexpr int x = decltype(x_)::value, LOOK = 4, NBUF = LOOK / 2 + 1, E = 32 / (2 * KS);      // two instructions a read
      const f32x16 zero = {0};
      bf16x8 buf[NBUF];
      auto read = [&](auto m) { if constexpr (m % 2 == 0) buf[m / 2 % NBUF] = q_rows(m / 2); };
      if (!take_other) {
        matrix_run<2 * KS, LOOK>(read, [&](auto m) { s[x][m % 2] = mfma32(k[m % 2][m / 2], buf[m / 2 % NBUF], m < 2 ? zero : s[x][m % 2]); });
        return;
      }
      float p[E];
      asm volatile("" : "+v"(other));              // (or the arithmetic below would be done ahead of the branch)
      matrix_run<2 * KS, LOOK>(read, [&](auto m) {
        s[x][m % 2] = mfma32(k[m % 2][m / 2], buf[m / 2 % NBUF], m < 2 ? zero : s[x][m % 2]);
        // an exponential is added one instruction later, when it is there
#pragma unroll
        for (int e = 0; e < E; ++e) {
          constexpr int at = m * E;
          if constexpr (m > 0) acc[(at - E) / 16][(at - E) % 16 + e] += p[e];
          p[e] = exp2_fast(__builtin_fmaf(s[1 - x][at / 16][at % 16 + e], a.scale_log2e, -other));
        }
      });
#pragma unroll
      for (int e = 0; e < E; ++e) acc[1][16 - E + e] += p[e];
    };
    constexpr std::integral_constant<int, 0> even{};
    constexpr std::integral_constant<int, 1> odd{};
    bool left = false;                             // scores in s[1] whose exponentials have not been taken, and their rows' norm
    float left_norm = 0.f;
    auto take_left = [&] {
      asm volatile("" : "+v"(left_norm));
#pragma unroll
      for (int e = 0; e < 32; ++e) acc[e / 16][e % 16] += exp2_fast(__builtin_fmaf(s[1][e / 16][e % 16], a.scale_log2e, -left_norm));
    };
    for (int t = t0; t < t1; ++t) {
      // this wave's copies of tile t have landed, behind the barrier those of all waves; and all have read tile t - 1, whose place tile t + 1 takes
      wait_async();
      __syncthreads();
      // Rows with lse -inf?  (256 us without the question, 259 with it; asked of the LDS copies, which the wave would wait for here, 254 where it was 245, and 361 instead of
      // 326 at head_dim 64.  With a quarter of the rows left out 5 and 13 % more.)
      bool none = false;
#pragma unroll
      for (int n = 0; n < kWeightRows / 64; ++n) none |= ahead[n] == -INFINITY;
      const bool whole = unmasked(t) && __builtin_amdgcn_ballot_w64(none) == 0;
      if (t + 1 < t1) copy_tile(t + 1);
      lo_q += (t % kWeightRing) * TILE;
      if (whole) {
        float norm[BLOCKS];
#pragma unroll
        for (int j = 0; j < BLOCKS; ++j) norm[j] = norm_of(t * BLOCKS + j);
        scores(even, left, left_norm);
#pragma unroll
        for (int j = 1; j < BLOCKS; ++j) {
          lo_q += 32 * D * 2;
          if (j & 1) scores(odd, true, norm[j - 1]);
          else scores(even, true, norm[j - 1]);
        }
        left = true;
        left_norm = norm[BLOCKS - 1];
      } else {
        if (left) take_left();
        left = false;
        for (int j = 0; j < BLOCKS; ++j) {
          if (j > 0) lo_q += 32 * D * 2;
          scores(even, false, 0.f);
          const int rh = (t * BLOCKS + j) * 32 + (lane & 31), rc = rh < rows ? rh : rows - 1;
          const float norm = norm_of(t * BLOCKS + j);
          // last key of the wave that the lane's row sees
          const int64_t far = norm == INFINITY ? -1 : a.causal ? rel + (int)((unsigned)rc % (unsigned)vis) : 63;
          const int see = (far > 63 ? 63 : far < -1 ? -1 : (int)far) - 4 * g;
#pragma unroll
          for (int e = 0; e < 32; ++e) {
            const float p = exp2_fast(__builtin_fmaf(s[0][e / 16][e % 16], a.scale_log2e, -norm));
            acc[e / 16][e % 16] += 32 * (e / 16) + 8 * (e % 16 >> 2) + (e & 3) <= see ? p : 0.f;
          }
        }
      }
      lo_q -= (BLOCKS - 1) * 32 * D * 2 + (t % kWeightRing) * TILE;
    }
    if (left) take_left();
  }
  // over the 32 rows of a half-wave; lane n of it keeps element n
  float mine = 0.f;
  const int n = lane & 31;
#pragma unroll
  for (int e = 0; e < 32; ++e) {
    const float v = half_sum(acc[e / 16][e % 16]);
    mine = n == e ? v : mine;
  }
  __syncthreads();
  float* const out = reinterpret_cast<float*>(smem) + 64 * wave_u;
  out[32 * (n / 16) + 8 * (n % 16 >> 2) + 4 * g + (n & 3)] = mine;
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
  const int64_t key = wave_key0 + lane;
  if (key >= a.kv_end) return;
  if (a.n_parts > 1) a.part[((int64_t)part_i * planes + plane) * (a.kv_end - a.kv_begin) + key - a.kv_begin] = out[lane];
  else put_weight(a, plane, key, out[lane]);
}

// Parts in their order.
__global__ __launch_bounds__(256) void kv8_weights_sum_kernel(const Kv8WeightArgs a) {
  const int64_t keys = a.kv_end - a.kv_begin, planes = (int64_t)a.batch * a.cache.n_kv_heads, i = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (i >= keys * planes) return;
  float sum = 0.f;
  for (int p0 = 0; p0 < a.n_parts; p0 += 8) {      // (eight loads under way at once, zeros behind the last)
    float x[8];
#pragma unroll
    for (int p = 0; p < 8; ++p) x[p] = p0 + p < a.n_parts ? a.part[(p0 + p) * planes * keys + i] : 0.f;
#pragma unroll
    for (int p = 0; p < 8; ++p) sum += x[p];
  }
  put_weight(a, i / keys, a.kv_begin + i % keys, sum);
}

template <int D>
static hipError_t launch_weights_t(const Kv8WeightArgs& a, bool few, hipStream_t st) {
  const int64_t keys = a.kv_end - a.kv_begin, planes = (int64_t)a.batch * a.cache.n_kv_heads;
  if (few) {
    const dim3 grid((unsigned)(a.n_parts * (planes / kv8_heads_wg(a.cache.n_kv_heads)))), block(256);
    if (a.group * a.s_q <= 16) hipLaunchKernelGGL((kv8_weights_few_kernel<D, 1>), grid, block, 0, st, a);
    else hipLaunchKernelGGL((kv8_weights_few_kernel<D, 2>), grid, block, 0, st, a);
    return hipGetLastError();
  }
  const int64_t items = (keys + kWeightKeys - 1) / kWeightKeys * planes * a.n_parts;
  hipLaunchKernelGGL(kv8_weights_kernel<D>, dim3((unsigned)((items + 7) / 8 * 8)), dim3(256), kv8_weights_lds_bytes<D>(), st, a);
  if (a.n_parts > 1) hipLaunchKernelGGL(kv8_weights_sum_kernel, dim3((unsigned)((keys * planes + 255) / 256)), dim3(256), 0, st, a);
  return hipGetLastError();
}
hipError_t opt_in_kv8_evict_kernels() {
  const hipFuncAttribute attr = hipFuncAttributeMaxDynamicSharedMemorySize;
  hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(&kv8_weights_kernel<128>), attr, (int)kv8_weights_lds_bytes<128>());
  if (e == hipSuccess) e = hipFuncSetAttribute(reinterpret_cast<const void*>(&kv8_weights_kernel<64>), attr, (int)kv8_weights_lds_bytes<64>());
  return e;
}
hipError_t launch_kv8_weights(const Kv8WeightArgs& a, int head_dim, bool few, hipStream_t st) {
  return head_dim == 128 ? launch_weights_t<128>(a, few, st) : launch_weights_t<64>(a, few, st);
}

// ------------------------------------------------------------------------------------ keep
// The rows of a plane that are kept: the `recent` last ones and those of the others with the largest weights.  A radix selection (11, 11 and 10 bits) finds the
// smallest weight that is taken and how many rows of exactly that weight are; a last walk writes the indices in order.  Counts alone cross threads, so
// that the order in which they run shows nowhere.  4238 rows of 12 planes 7.2 us; 131072 rows of 8 planes 21.5 us in four launches, 32000 18 (all bins of all chunks added
// up by every workgroup 29 and 24.5; 8192 rows a chunk 22 and 21), and 230 with one workgroup a plane.
constexpr int kKeepThreads = 1024, kKeepWaves = kKeepThreads / 64;
constexpr int kKeepShift[3] = {21, 10, 0}, kKeepBins[3] = {2048, 2048, 1024};

// A number that orders as the weight does: NaN behind everything, both zeros alike
SP_DEV uint32_t weight_order(float w) {
  uint32_t u = __float_as_uint(w);
  if ((u & 0x7fffffffu) > 0x7f800000u) return 0u;
  if (u == 0x80000000u) u = 0u;
  return u & 0x80000000u ? ~u : u | 0x80000000u;
}
// Inclusive sum over the lanes of a half-wave, or of a wave (row_shr by 1, 2, 4 and 8 inside each sixteen, then the last lane of a sixteen to the next one, and of the
// first half to the second).
template <int LANES>
SP_DEV uint32_t lane_scan(uint32_t v) {
  v += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x111, 0xf, 0xf, true);
  v += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x112, 0xf, 0xf, true);
  v += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x114, 0xf, 0xf, true);
  v += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x118, 0xf, 0xf, true);
  v += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x142, 0xa, 0xf, false);
  if constexpr (LANES == 64) v += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x143, 0xc, 0xf, false);
  return v;
}
// Inclusive sum over the workgroup's threads, and the sum of all.  Two barriers.
struct KeepScan { uint32_t upto, total; };
SP_DEV KeepScan keep_scan(uint32_t v, uint32_t (&wave_sums)[kKeepWaves]) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  v = lane_scan<64>(v);
  __syncthreads();
  if (lane == 63) wave_sums[wave] = v;
  __syncthreads();
  KeepScan s{v, 0};
#pragma unroll
  for (int w = 0; w < kKeepWaves; ++w) {
    s.upto += w < wave ? wave_sums[w] : 0u;
    s.total += wave_sums[w];
  }
  return s;
}
struct KeepShared { uint32_t hist[2048], wave_sums[kKeepWaves], found[4], entry[kKeepOneRows / 64]; };

// What is known of the smallest weight that is taken: its leading bits, and how many rows that begin with them are wanted.
struct KeepFound { uint32_t prefix, need; };
// The bin of pass `pass` in which the need-th largest lies; thread t brings the counts of the bins from the top on: `mine` (one bin in the last pass).
SP_DEV KeepFound keep_find(KeepShared& sh, int pass, uint32_t first, uint32_t second, KeepFound so_far) {
  const int per = kKeepBins[pass] / kKeepThreads, top = kKeepBins[pass] - 1 - (int)threadIdx.x * per;
  const uint32_t upto = keep_scan(first + second, sh.wave_sums).upto, ahead = upto - first - second;
  if (ahead < so_far.need && so_far.need <= upto) {
    const bool lower = ahead + first < so_far.need;
    sh.found[0] = (uint32_t)(top - lower);
    sh.found[1] = so_far.need - ahead - (lower ? first : 0u);
  }
  __syncthreads();
  const KeepFound f{so_far.prefix | sh.found[0] << kKeepShift[pass], sh.found[1]};
  __syncthreads();
  return f;
}
// Rows of a wave in the bin of its first one are counted there in one step: many weights may be equal (0 above all), or lie within one bin of a pass, and adds to one
// counter wait for each other (131072 equal weights of 8 planes 22 us, one by one 16 more; uniform ones a microsecond less; 4238 of 12 planes 7.3 and 15.6, 7.2 and 6.8).
SP_DEV void keep_count(KeepShared& sh, int pass, uint32_t u, uint32_t prefix) {
  const int above = kKeepShift[pass] + (pass == 2 ? 10 : 11);
  if (pass > 0 && (u >> above) != (prefix >> above)) return;
  const int bin = (int)(u >> kKeepShift[pass]) & (kKeepBins[pass] - 1);
  const uint64_t same = __builtin_amdgcn_ballot_w64(bin == __builtin_amdgcn_readfirstlane(bin));
  const int lane = threadIdx.x & 63;
  if (!(same >> lane & 1)) atomicAdd(&sh.hist[bin], 1u);
  else if ((same & (((uint64_t)1 << lane) - 1)) == 0) atomicAdd(&sh.hist[bin], (uint32_t)__popcll(same));
}
SP_DEV void keep_clear(KeepShared& sh, int pass) {
  for (int i = threadIdx.x; i < kKeepBins[pass]; i += kKeepThreads) sh.hist[i] = 0;
  __syncthreads();
}
// Writes those of the rows first + v * 1024 + thread (v < V, only rows below `others`) that are taken: weights above f.prefix, and of those equal to it the
// first f.need of the plane.  `above`, `same`: how many rows before `first` are above and equal; both move on.
template <int V>
SP_DEV void keep_write(KeepShared& sh, const uint32_t (&u)[V], int64_t first, int64_t others, KeepFound f, uint32_t& above, uint32_t& same, int32_t* out) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  uint64_t more[V], equal[V];
  __syncthreads();
#pragma unroll
  for (int v = 0; v < V; ++v) {
    const bool there = first + v * kKeepThreads + threadIdx.x < others;
    more[v] = __builtin_amdgcn_ballot_w64(there && u[v] > f.prefix);
    equal[v] = __builtin_amdgcn_ballot_w64(there && u[v] == f.prefix);
    if (lane == 0) sh.entry[v * kKeepWaves + wave] = (uint32_t)__popcll(more[v]) | (uint32_t)__popcll(equal[v]) << 16;
  }
  __syncthreads();
  const uint32_t mine = threadIdx.x < V * kKeepWaves ? sh.entry[threadIdx.x] : 0u;
  const KeepScan s = keep_scan(mine, sh.wave_sums);
  if (threadIdx.x < V * kKeepWaves) sh.entry[threadIdx.x] = s.upto - mine;
  __syncthreads();
  const uint64_t before = ((uint64_t)1 << lane) - 1;
#pragma unroll
  for (int v = 0; v < V; ++v) {
    const uint32_t e = sh.entry[v * kKeepWaves + wave];
    const uint32_t a = above + (e & 0xffffu) + (uint32_t)__popcll(more[v] & before), q = same + (e >> 16) + (uint32_t)__popcll(equal[v] & before);
    const bool is_equal = equal[v] >> lane & 1;
    if ((more[v] >> lane & 1) || (is_equal && q < f.need)) out[a + (q < f.need ? q : f.need)] = (int32_t)(first + v * kKeepThreads + threadIdx.x);
  }
  above += s.total & 0xffffu;
  same += s.total >> 16;
}

// Up to 1024 V rows of a plane: a workgroup, which keeps them in registers.
template <int V>
__global__ __launch_bounds__(kKeepThreads) void kv8_keep_kernel(const Kv8KeepArgs a) {
  __shared__ KeepShared sh;
  const int tid = threadIdx.x, others = a.rows - a.recent;
  const float* const w = a.weights + (int64_t)blockIdx.x * a.capacity;
  int32_t* const out = a.index + (int64_t)blockIdx.x * a.keep;
  uint32_t u[V];
#pragma unroll
  for (int v = 0; v < V; ++v) u[v] = v * kKeepThreads + tid < others ? weight_order(w[v * kKeepThreads + tid]) : 0u;
  KeepFound f{0u, (uint32_t)(a.keep - a.recent)};
  if (f.need >= (uint32_t)others) {            // all of them
    for (int i = tid; i < others; i += kKeepThreads) out[i] = i;
  } else if (f.need > 0) {
#pragma unroll
    for (int pass = 0; pass < 3; ++pass) {
      keep_clear(sh, pass);
#pragma unroll
      for (int v = 0; v < V; ++v)
        if (v * kKeepThreads + tid < others) keep_count(sh, pass, u[v], f.prefix);
      __syncthreads();
      const int per = kKeepBins[pass] / kKeepThreads, top = kKeepBins[pass] - 1 - tid * per;
      const uint32_t first = sh.hist[top], second = per > 1 ? sh.hist[top - 1] : 0u;
      f = keep_find(sh, pass, first, second, f);
    }
    uint32_t above = 0, same = 0;
    keep_write<V>(sh, u, 0, others, f, above, same, out);
  }
  for (int i = tid; i < a.recent; i += kKeepThreads) out[a.keep - a.recent + i] = others + i;
}

// More rows: a workgroup for every a.chunk of them (a multiple of kKeepSpan), a launch a pass.  The counts of a pass stay in the workspace, [plane][chunk], by bin and
// by groups of 32 bins; the first wave of every workgroup of the next pass adds up its plane's counts of the groups, then those of the bins of one group.  Behind
// them, for each chunk, how many of its rows are known to be above; and for each plane what the passes found.
constexpr int kKeepGroup = 32;
struct KeepWork {
  uint32_t *hist[3], *groups[3], *above, *found;
  SP_DEV KeepWork(const Kv8KeepArgs& a, int plane) {
    uint32_t* p = a.work + (int64_t)plane * (a.chunks * (int64_t)kKeepChunkWords + kKeepPlaneWords);
    for (int i = 0; i < 3; ++i) {
      hist[i] = p;
      p += (int64_t)a.chunks * kKeepBins[i];
      groups[i] = p;
      p += a.chunks * (kKeepBins[i] / kKeepGroup);
    }
    above = p;
    found = p + a.chunks;
  }
};
static_assert(kKeepChunkWords == (2048 + 2048 + 1024) * 33 / 32 + 1, "words of a chunk");

// What pass P found, by the counts of all chunks, in one wave; with it the rows of this chunk that the pass puts above (LAST: those of the chunks before, and in
// `same` how many of them are in the bin).
struct KeepStep { KeepFound found; uint32_t above, same; };
template <int P, bool LAST>
SP_DEV KeepStep keep_step(const KeepWork& work, int chunks, int chunk, KeepFound so_far) {
  constexpr int BINS = kKeepBins[P], GROUPS = BINS / kKeepGroup;
  static_assert(GROUPS <= 64 && kKeepGroup == 32, "a lane a group, half a wave the bins of one");
  const int lane = threadIdx.x & 63;
  auto at = [](uint32_t v, int l) { return (uint32_t)__builtin_amdgcn_readlane((int)v, l); };
  // (loads of 16 or 8 chunks under way at once, those behind the last read once more)
  auto add = [&](auto read, int first, int step, auto n_, uint32_t& total, uint32_t& part) {
    constexpr int N = decltype(n_)::value;
    for (int c0 = first; c0 < chunks; c0 += N * step) {
      uint32_t n[N];
#pragma unroll
      for (int i = 0; i < N; ++i) n[i] = read(c0 + i * step < chunks ? c0 + i * step : chunks - 1);
#pragma unroll
      for (int i = 0; i < N; ++i) {
        const int c = c0 + i * step;
        total += c < chunks ? n[i] : 0u;
        part += (LAST ? c < chunk : c == chunk) ? n[i] : 0u;      // (chunk < chunks)
      }
    }
  };
  // groups from the top on, a lane each
  uint32_t total = 0, part = 0;
  if (lane < GROUPS) add([&](int c) { return work.groups[P][c * GROUPS + GROUPS - 1 - lane]; }, 0, 1, std::integral_constant<int, 16>{}, total, part);
  uint32_t upto = lane_scan<64>(total);
  int l = __builtin_ctzll(__builtin_amdgcn_ballot_w64(upto - total < so_far.need && so_far.need <= upto));
  uint32_t need = so_far.need - at(upto - total, l), above = at(lane_scan<64>(part) - part, l);
  // its bins from the top on; the chunks shared out between the half-waves
  const int group = GROUPS - 1 - l, bin = group * kKeepGroup + kKeepGroup - 1 - lane % 32;
  total = part = 0;
  add([&](int c) { return work.hist[P][(int64_t)c * BINS + bin]; }, lane / 32, 2, std::integral_constant<int, 8>{}, total, part);
  total += (uint32_t)__shfl_xor((int)total, 32, 64);
  part += (uint32_t)__shfl_xor((int)part, 32, 64);
  upto = lane_scan<32>(total);
  l = __builtin_ctzll(__builtin_amdgcn_ballot_w64(upto - total < need && need <= upto));
  need -= at(upto - total, l);
  above += at(lane_scan<32>(part) - part, l);
  return {{so_far.prefix | at((uint32_t)bin, l) << kKeepShift[P], need}, above, at(part, l)};
}

// PASS 0 .. 2: counts of a chunk; PASS 3: the indices.
template <int PASS>
__global__ __launch_bounds__(kKeepThreads) void kv8_keep_pass_kernel(const Kv8KeepArgs a) {
  constexpr int V = kKeepSpan / kKeepThreads;      // rows of a thread at a time
  __shared__ KeepShared sh;
  const int tid = threadIdx.x, lane = tid & 63, chunk = blockIdx.x, plane = blockIdx.y;
  const int64_t others = a.rows - a.recent, first = (int64_t)chunk * a.chunk, last = first + a.chunk < others ? first + a.chunk : others;
  const float* const w = a.weights + plane * a.capacity;
  const KeepWork work(a, plane);
  // (the first rows are on their way while the last pass is added up)
  float x[V];
  auto load = [&](int64_t at) {
#pragma unroll
    for (int v = 0; v < V; ++v) x[v] = at + v * kKeepThreads + tid < last ? w[at + v * kKeepThreads + tid] : 0.f;
  };
  load(first);
  KeepFound f{0u, (uint32_t)(a.keep - a.recent)};
  uint32_t above = 0, same = 0;                // PASS 3: rows before the chunk
  const bool all = f.need >= (uint32_t)others, search = f.need > 0 && !all;
  if constexpr (PASS > 0) {
    if (search && tid < 64) {
      if (PASS > 1) f = KeepFound{work.found[2 * PASS - 4], work.found[2 * PASS - 3]};
      KeepStep step = keep_step<PASS - 1, PASS == 3>(work, a.chunks, chunk, f);
      if (PASS == 3) step.above += (uint32_t)__builtin_amdgcn_readlane((int)lane_scan<64>(lane < chunk ? work.above[lane] : 0u), 63);
      if (tid == 0) {
        sh.found[0] = step.found.prefix;
        sh.found[1] = step.found.need;
        sh.found[2] = step.above;
        sh.found[3] = step.same;
        // rows of the chunk that the passes so far have put above; and the first workgroup of a plane writes down what all of them have found
        if (PASS < 3) work.above[chunk] = step.above + (PASS > 1 ? work.above[chunk] : 0u);
        if (PASS < 3 && chunk == 0) { work.found[2 * PASS - 2] = step.found.prefix; work.found[2 * PASS - 1] = step.found.need; }
      }
    }
  }
  if constexpr (PASS < 3) {
    keep_clear(sh, PASS);                      // (and a barrier)
    if (PASS > 0) f = KeepFound{sh.found[0], sh.found[1]};
    for (int64_t at = first; at < last; at += kKeepSpan) {
      if (at > first) load(at);
#pragma unroll
      for (int v = 0; v < V; ++v)
        if (at + v * kKeepThreads + tid < last) keep_count(sh, PASS, weight_order(x[v]), f.prefix);
    }
    __syncthreads();
#pragma unroll
    for (int i = tid; i < kKeepBins[PASS]; i += kKeepThreads) {
      const uint32_t n = sh.hist[i], sum = lane_scan<32>(n);
      work.hist[PASS][(int64_t)chunk * kKeepBins[PASS] + i] = n;
      if (lane % kKeepGroup == kKeepGroup - 1) work.groups[PASS][(chunk * kKeepBins[PASS] + i) / kKeepGroup] = sum;
    }
  } else {
    int32_t* const out = a.index + (int64_t)plane * a.keep;
    __syncthreads();
    if (search) {
      f = KeepFound{sh.found[0], sh.found[1]};
      above = sh.found[2];
      same = sh.found[3];
    }
    for (int64_t at = first; search && at < last; at += kKeepSpan) {
      if (at > first) load(at);
      uint32_t u[V];
#pragma unroll
      for (int v = 0; v < V; ++v) u[v] = weight_order(x[v]);
      keep_write<V>(sh, u, at, last, f, above, same, out);
    }
    if (all)
      for (int64_t i = first + tid; i < last; i += kKeepThreads) out[i] = (int32_t)i;
    for (int64_t i = (int64_t)chunk * kKeepThreads + tid; i < a.recent; i += (int64_t)a.chunks * kKeepThreads) out[a.keep - a.recent + i] = (int32_t)(others + i);
  }
}

hipError_t launch_kv8_keep(const Kv8KeepArgs& a, hipStream_t st) {
  const dim3 block(kKeepThreads);
  if (a.chunks == 0) {
    const dim3 grid((unsigned)a.planes);
    const int others = a.rows - a.recent;
    if (others <= 4 * kKeepThreads) hipLaunchKernelGGL(kv8_keep_kernel<4>, grid, block, 0, st, a);
    else hipLaunchKernelGGL(kv8_keep_kernel<16>, grid, block, 0, st, a);
    return hipGetLastError();
  }
  const dim3 grid((unsigned)a.chunks, (unsigned)a.planes);
  if (a.keep > a.recent && a.keep < a.rows) {
    hipLaunchKernelGGL(kv8_keep_pass_kernel<0>, grid, block, 0, st, a);
    hipLaunchKernelGGL(kv8_keep_pass_kernel<1>, grid, block, 0, st, a);
    hipLaunchKernelGGL(kv8_keep_pass_kernel<2>, grid, block, 0, st, a);
  }
  hipLaunchKernelGGL(kv8_keep_pass_kernel<3>, grid, block, 0, st, a);
  return hipGetLastError();
}

// ------------------------------------------------------------------------------------ gather
// A block of kept rows of a head, keys (blockIdx.y = 0) or values: its scale is the largest that its rows had, rows of smaller scales are rounded to it.  Bound
// by the bytes, in rows of head_dim from anywhere: 32768 of 131072 rows of 8 heads of 128 in 27 us, 134 MB at 5.0 TB/s (behind a kernel that leaves the caches full of
// what it wrote 37; then codes under way while the scales are compared 38, neighbouring heads in neighbouring workgroups 39).
template <int D>
__global__ __launch_bounds__(256) void kv8_gather_kernel(const Kv8GatherArgs a) {
  constexpr int NP = D / 16;
  __shared__ int32_t row[256];
  __shared__ uint8_t was[256];
  __shared__ uint32_t most[4];
  const Kv8Cache &from = a.from, &to = a.to;
  const int L = 1 << to.shift, tid = threadIdx.x;
  const int64_t blocks = (a.keep + L - 1) / L, plane = blockIdx.x / blocks, blk = blockIdx.x - plane * blocks;
  const int64_t b = plane / from.n_kv_heads;
  const int h = (int)(plane - b * from.n_kv_heads), first = (int)blk * L, n = a.keep - first < L ? a.keep - first : L;
  const bool keys = blockIdx.y == 0;
  const Kv8Operand src = keys ? from.k : from.v, dst = keys ? to.k : to.v;
  uint32_t byte = 0;
  if (tid < n) {
    const int32_t r = a.index[plane * a.keep + first + tid];
    const bool there = r >= 0 && r < a.from_rows;      // (another entry is no row: zeros)
    row[tid] = there ? r : -1;
    byte = there ? src.scales[kv8_scale_at(from, b, r, h)] : 0u;
    was[tid] = (uint8_t)byte;
    if (keys && a.kept_weights) a.kept_weights[plane * a.kept_weights_stride + first + tid] = there ? a.weights[plane * a.weights_stride + r] : 0.f;
  }
#pragma unroll
  for (int w = 1; w < 64; w <<= 1) {
    const uint32_t o = (uint32_t)__shfl_xor((int)byte, w, 64);
    byte = byte > o ? byte : o;
  }
  if ((tid & 63) == 0) most[tid >> 6] = byte;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < 4; ++w) byte = byte > most[w] ? byte : most[w];
  byte = byte < kKv8LeastScale ? kKv8LeastScale : byte;      // (a block without a row)
  const float unit = kv8_scale(byte);
  for (int i = tid; i < n * NP; i += 256) {
    const int r = i / NP, c = i % NP;
    u32x4 x = {0, 0, 0, 0};
    if (row[r] >= 0) {
      x = *reinterpret_cast<const u32x4*>(src.codes + b * from.stride_b + (int64_t)row[r] * from.stride_s + h * from.stride_h + 16 * c);
      if (was[r] != byte) {
        const float s = kv8_scale(was[r]);
        const u32x2 lo = kv8_codes(kv8_values(x[0], x[1], s), unit), hi = kv8_codes(kv8_values(x[2], x[3], s), unit);
        x = u32x4{lo[0], lo[1], hi[0], hi[1]};
      }
    }
    *reinterpret_cast<u32x4*>(dst.codes + b * to.stride_b + (int64_t)(first + r) * to.stride_s + h * to.stride_h + 16 * c) = x;
  }
  if (tid == 0) dst.scales[(b * to.blocks + blk) * to.n_kv_heads + h] = (uint8_t)byte;
}
hipError_t launch_kv8_gather(const Kv8GatherArgs& a, int head_dim, hipStream_t st) {
  const int64_t blocks = (a.keep + (1 << a.to.shift) - 1) >> a.to.shift;
  const dim3 grid((unsigned)(blocks * a.batch * a.to.n_kv_heads), 2), block(256);
  if (head_dim == 128) hipLaunchKernelGGL(kv8_gather_kernel<128>, grid, block, 0, st, a);
  else hipLaunchKernelGGL(kv8_gather_kernel<64>, grid, block, 0, st, a);
  return hipGetLastError();
}

}  // namespace slimpipe
