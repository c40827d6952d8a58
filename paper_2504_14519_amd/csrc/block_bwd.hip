// Backward of sparse attention over selected key blocks.
//
// With p_ij = exp(scale q_i.k_j - lse_i) on the visible pairs of the chosen blocks and delta_i = dO_i . O_i:
//   dV_j = sum_i p_ij dO_i            dS_ij = p_ij (dO_i . v_j - delta_i)
//   dQ_i = scale sum_j dS_ij k_j      dK_j  = scale sum_i dS_ij q_i
// As in the dense backward dq and dk/dv have kernels of their own, both over the lists of block_select.hip:
//   dq     tiles of 128 rows of one block, as in the forward; each (row, slot) leaves a partial dq that a last kernel adds in slot order
//   dk/dv  a workgroup owns 256 keys (128 or 64 at head_dim 64 and in small blocks) and walks the rows that chose their block, 32 at a time; long
//          lists are cut into parts whose sums the last kernel adds in list order.
// No sum depends on the order in which workgroups run.
#include "block_tile.hpp"
#include "dkdv_tile.hpp"
#include "row_tile.hpp"

namespace slimpipe {

constexpr int kDqKeys = 64;

// 8192 rows of 8 heads of 128 on 128 blocks of 512 keys, 8 a row: 212 us (910 TFLOP/s); as in the forward a workgroup's start and way out are hidden in part.
template <int D>
constexpr size_t block_dq_lds_bytes() {
  constexpr size_t rings = (size_t)4 * kDqKeys * D * 2, rows = (size_t)4 * 32 * kOutRow<D> * 4;
  return rings > rows ? rings : rows;
}

template <int D>
__global__ __launch_bounds__(256, 2) void block_dq_kernel(const BlockArgs a) {
  constexpr int BN = kDqKeys, TILE = BN * D * 2, KS = D / 16, DB = D / 32;
  extern __shared__ __attribute__((aligned(1024))) char smem[];
  const int tid = threadIdx.x, lane = tid & 63, g = lane >> 5, wave_u = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int plane = blockIdx.y, b = plane / a.n_kv_heads, hk = plane - b * a.n_kv_heads;
  const TileRows rows(a, plane, wave_u, lane);
  if (rows.none) return;
  const BlockItem it = rows.item;
  const BlockEntry e = rows.e;
  const int n_rows = it.count, mine = rows.mine;
  const int h = hk * a.group + (int)(e.head_slot >> 6);
  const int64_t row = ((int64_t)b * a.n_q_heads + h) * a.s_q + e.row;

  const BlockKeys keys(a, it.block, b, hk);
  const TileSight sight(a, keys, e.row, reinterpret_cast<int*>(smem), wave_u, lane);
  const int see_rel = sight.see_rel, n_keys = sight.n_keys;
  const int nt = n_keys > 0 ? (n_keys + BN - 1) / BN : 0;
  const unsigned lds = lds_addr(smem);
  const uint32_t row_bytes = (uint32_t)a.kv_stride_s * 2;
  const bf16_t* const kp = a.kv.k[keys.chunk] + keys.off;
  const bf16_t* const vp = a.kv.v[keys.chunk] + keys.off;
  TileDma<D, BN, 256> dma;
  dma.init(tid);
  auto copy = [&](int t) {
    const int64_t off = (int64_t)t * BN * a.kv_stride_s;
    const int left = n_keys - t * BN, avail = left < BN ? left : BN;
    const unsigned slot = lds + (t & 1) * 2 * TILE;
#pragma unroll
    for (int n = 0; n < TileDma<D, BN, 256>::PASSES; ++n) dma.issue(slot, kp + off, row_bytes, avail, wave_u, n);
#pragma unroll
    for (int n = 0; n < TileDma<D, BN, 256>::PASSES; ++n) dma.issue(slot + TILE, vp + off, row_bytes, avail, wave_u, n);
  };

  f32x16 dq[DB];
#pragma unroll
  for (int db = 0; db < DB; ++db)
#pragma unroll
    for (int i = 0; i < 16; ++i) dq[db][i] = 0.f;
  if (nt > 0) {
    copy(0);
    bf16x8 q[KS], d_o[KS];
    {
      const bf16_t* qp = a.q + (int64_t)b * a.q_stride_b + (int64_t)hk * a.group * a.q_stride_h + (int64_t)e.q_off * 8 + 8 * g;
      const bf16_t* op = a.d_out + (int64_t)b * a.do_stride_b + (int64_t)hk * a.group * a.do_stride_h + (int64_t)e.do_off * 8 + 8 * g;
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) q[ks] = *reinterpret_cast<const bf16x8*>(qp + 16 * ks);
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) d_o[ks] = *reinterpret_cast<const bf16x8*>(op + 16 * ks);
    }
    const float lse2 = a.lse2[row], ndelta = a.delta[row], c = a.scale_log2e;      // (lse2 +inf for a row without keys: p = 0)
    RpOffsets<D> lo_k;
    TrOffsets<D> lo_kt;
    lo_k.init(lane, (int)lds);
    lo_kt.init(lane, (int)lds);
    wait_async();
    __syncthreads();
    for (int t = 0; t < nt; ++t) {
      if (t + 1 < nt) copy(t + 1);
      const int kmax = see_rel - t * BN;
      const bool masked = __builtin_amdgcn_ballot_w64(kmax < BN - 1) != 0;
#pragma unroll
      for (int kb = 0; kb < BN / 32; ++kb) {
        f32x16 s, dp;
#pragma unroll
        for (int i = 0; i < 16; ++i) { s[i] = 0.f; dp[i] = ndelta; }
        constexpr int LOOK = 3;
        bf16x8 buf[LOOK + 1];
        matrix_run<2 * KS, LOOK>(
            [&](auto m) { buf[m % (LOOK + 1)] = lds_rp<D>(lo_k, m / 2, m % 2 * TILE + kb * 32 * D * 2); },
            [&](auto m) {
              if constexpr (m % 2 == 0) s = mfma32(buf[m % (LOOK + 1)], q[m / 2], s);
              else dp = mfma32(buf[m % (LOOK + 1)], d_o[m / 2], dp);
            });
        if (masked) {
          const int hi = kmax - kb * 32 - 4 * g;
#pragma unroll
          for (int i = 0; i < 16; ++i) s[i] = 8 * (i >> 2) + (i & 3) <= hi ? s[i] : -INFINITY;
        }
#pragma unroll
        for (int i = 0; i < 16; ++i) s[i] = exp2_fast(__builtin_fmaf(s[i], c, -lse2)) * dp[i];
        const bf16x8 ds[2] = {pack8(s, 0), pack8(s, 8)};      // (rounded to bf16 for the matrix unit, as in the dense backward)
        matrix_run<2 * DB, LOOK>(
            [&](auto m) { buf[m % (LOOK + 1)] = lds_tr<D>(lo_kt, m % DB, (2 * kb + m / DB) * 16 * D * 2); },
            [&](auto m) { dq[m % DB] = mfma32(buf[m % (LOOK + 1)], ds[m / DB], dq[m % DB]); });
      }
      const int step = (t & 1) ? -2 * TILE : 2 * TILE;
      lo_k.add(step);
      lo_kt.add(step);
      wait_async();
      __syncthreads();
    }
  }
  if (see_rel < 0) {                             // sees no key of the block (weights of 0 times what other rows see, which may not be finite)
#pragma unroll
    for (int db = 0; db < DB; ++db)
#pragma unroll
      for (int i = 0; i < 16; ++i) dq[db][i] = 0.f;
  }
  store_parts<D>(a, reinterpret_cast<float*>(smem) + wave_u * 32 * kOutRow<D>, dq, a.scale, row * a.top_k + (e.head_slot & 63u), n_rows, wave_u, lane);
}

// ------------------------------------------------------------------------------------ dk / dv
// Items that follow each other on one XCD: the parts of a block's keys share the rows of the list, and the parts of its list its keys.  (Runs of 1
// and 4 come within 1 % on blocks of 256, 512 and 1024 keys; with long ones the XCDs have unequal work.)
constexpr int kDkdvRun = 2;
// What a dk/dv item has: keys [kmin, kmax) of the workgroup's KEYS exist, the first of them all lies at element `off` of chunk `chunk`.
template <int D, int KEYS>
struct DkdvItem {
  BlockItem it;
  const BlockEntry* list;
  int sub, kmin, kmax, chunk;
  int64_t key0, off;
  bool none;
  SP_DEV DkdvItem(const BlockArgs& a, int plane, int b, int hk) {
    const int item = __builtin_amdgcn_readfirstlane(xcd_item(blockIdx.x, kDkdvRun, plane));
    none = item >= a.n_dkdv_items[2 * plane];
    if (none) return;
    it = a.dkdv_items[(int64_t)plane * a.dkdv_cap + item];
    const int block = it.block / a.n_sub;
    sub = it.block - block * a.n_sub;
    list = a.entries + (int64_t)plane * a.item_cap * kBlockTileRows + it.first;
    key0 = (int64_t)block * a.block_len + sub * KEYS;
    const int64_t end = (int64_t)(block + 1) * a.block_len < a.kv_end ? (int64_t)(block + 1) * a.block_len : a.kv_end;
    kmin = a.kv_begin > key0 ? (a.kv_begin - key0 < KEYS ? (int)(a.kv_begin - key0) : KEYS) : 0;
    kmax = end - key0 < KEYS ? (int)(end - key0) : KEYS;
    none = kmax <= kmin;
    chunk = kv_chunk_of(a.kv, key0);
    off = (int64_t)b * a.kv_stride_b + (int64_t)hk * a.kv_stride_h + (key0 - (int64_t)chunk * a.kv.len) * a.kv_stride_s;
  }
  // K rows of the lane's key (clamped to those that exist) as B operand: k-slots = head_dim 16 ks + 8 g ..
  SP_DEV void load_k(const BlockArgs& a, int key, int g, bf16x8 (&kreg)[D / 16]) const {
    const int kc = key < kmin ? kmin : (key < kmax ? key : kmax - 1);
    const bf16_t* kp = a.kv.k[chunk] + off + (int64_t)kc * a.kv_stride_s + 8 * g;
#pragma unroll
    for (int ks = 0; ks < D / 16; ++ks) kreg[ks] = *reinterpret_cast<const bf16x8*>(kp + 16 * ks);
  }
  // the wave's 32 V rows to LDS (a wave without keys copies nothing; what its columns come to is not stored)
  SP_DEV void copy_v(const BlockArgs& a, unsigned lds, int w0, int lane) const {
    WaveDma<D, 32> dma;
    dma.init(lane, (uint32_t)a.kv_stride_s * 2);
    if (kmax > w0 && kmin - w0 < 32)
      dma.copy(lds, a.kv.v[chunk] + off + (int64_t)w0 * a.kv_stride_s, (uint32_t)a.kv_stride_s * 2, kmin > w0 ? kmin - w0 : 0, kmax - w0, lane);
  }
  // rows [kmin, kmax) of dk and dv of the wave: to the accumulators, or to the partial sums of this part of the list; `part`: kOutRow<D> * 32
  // floats of LDS of the wave's own
  SP_DEV void flush(const BlockArgs& a, int plane, float* part, const f32x16 (&dk)[D / 32], const f32x16 (&dv)[D / 32], int w0, int lane) const {
    const int keys_pad = a.n_sub * KEYS;
    float *kdst, *vdst;
    int64_t stride;
    bool accumulate = false;
    if (it.part >= 0) {
      kdst = a.dkdv_part + (((int64_t)plane * a.part_cap + it.part) * 2 * keys_pad + sub * KEYS) * D;
      vdst = kdst + (int64_t)keys_pad * D;
      stride = D;
    } else {
      kdst = a.dk_acc[chunk] + off;
      vdst = a.dv_acc[chunk] + off;
      stride = a.kv_stride_s;
      accumulate = a.dkv_accumulate != 0;
    }
    constexpr int PER = D / 4, RPP = 64 / PER;
    const int d4 = lane % PER * 4;
    auto put = [&](const f32x16 (&acc)[D / 32], float factor, float* dst) {
      put_rows<D>(part, acc, factor, lane);
#pragma unroll
      for (int j = 0; j < 32 / RPP; ++j) {
        const int r = j * RPP + lane / PER, kr = w0 + r;
        if (kr < kmin || kr >= kmax) continue;
        f32x4 v = *reinterpret_cast<const f32x4*>(part + r * kOutRow<D> + d4);
        f32x4* to = reinterpret_cast<f32x4*>(dst + (int64_t)kr * stride + d4);
        if (accumulate) v += *to;
        *to = v;
      }
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
      __builtin_amdgcn_wave_barrier();
    };
    put(dk, a.scale, kdst);
    put(dv, 1.0f, vdst);
  }
};

template <int D, int NW>
struct BlockDkdvLds {
  static constexpr int TILE = 32 * D * 2;                  // 32 rows of Q or dO
  static constexpr int V = 4 * TILE, STAT = V + NW * 32 * D * 2, STAT_BYTES = 3 * 32 * 4;      // {Q, dO} x 2, V, {lse2, -delta, position} x 2
  static constexpr int RINGS = STAT + 2 * STAT_BYTES, OUT = NW * 32 * kOutRow<D> * 4;
  static constexpr int TOTAL = RINGS > OUT ? RINGS : OUT;
};

// The other ones: a wave owns 32 keys, rows in tiles of 32 through two LDS slots, two barriers a tile; two workgroups or more share a compute unit, so that
// one's vector work and waits are behind another's matrix work.  3 x 1337 rows of 12 heads of 64 on 64 blocks of 64 keys, 12 a row: 57 us; 8192 rows of 8
// heads of 128 on blocks of 512, in 128 keys each: 332.
template <int D, int NW>
__global__ __launch_bounds__(NW * 64, 2) void block_dkdv_kernel(const BlockArgs a) {
  using L = BlockDkdvLds<D, NW>;
  constexpr int KS = D / 16, DB = D / 32, NC = D / 8, T = NW * 64, RPP = T / NC, PASSES = 32 / RPP, KEYS = NW * 32;
  extern __shared__ __attribute__((aligned(1024))) char smem[];
  const int tid = threadIdx.x, lane = tid & 63, g = lane >> 5, ql = lane & 31, wave_u = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int plane = blockIdx.y, b = plane / a.n_kv_heads, hk = plane - b * a.n_kv_heads;
  const DkdvItem<D, KEYS> item(a, plane, b, hk);
  if (item.none) return;
  const int n_rows = item.it.count;
  const BlockEntry* const list = item.list;
  const int64_t key0 = item.key0;
  const unsigned lds = lds_addr(smem);
  const int key = wave_u * 32 + ql;
  bf16x8 kreg[KS];
  item.load_k(a, key, g, kreg);
  item.copy_v(a, lds + L::V + wave_u * 32 * D * 2, wave_u * 32, lane);
  // This thread's part of a tile copy: rows tid / NC + n * RPP, the chunk that the swizzle puts at its place.
  const int crow = tid / NC, cpos = tid % NC;
  auto chunk_of = [&](int r) {
    return D == 128 ? ((((cpos >> 2) ^ r) & 3) << 2) | (((cpos & 3) ^ (r >> 2)) & 3) : (cpos ^ r) & (NC - 1);
  };
  const bf16_t* const qb = a.q + (int64_t)b * a.q_stride_b + (int64_t)hk * a.group * a.q_stride_h;
  const bf16_t* const ob = a.d_out + (int64_t)b * a.do_stride_b + (int64_t)hk * a.group * a.do_stride_h;
  const int64_t stat0 = ((int64_t)b * a.n_q_heads + hk * a.group) * a.s_q;
  auto entry = [&](int i) { return list + (i < n_rows ? i : n_rows - 1); };
  struct { uint32_t q_off, do_off; } ec[PASSES];
  struct { uint32_t row, head_slot; } es;        // entries of the next tile to copy: the rows this thread copies, the row whose statistics it brings
  auto fetch = [&](int u) {
#pragma unroll
    for (int n = 0; n < PASSES; ++n) {
      const BlockEntry* x = entry(u * 32 + crow + n * RPP);
      ec[n] = {x->q_off, x->do_off};
    }
    const BlockEntry* x = entry(u * 32 + (tid & 31));
    es = {x->row, x->head_slot};
  };
  auto copy = [&](int u) {
    const unsigned slot = lds + (u & 1) * 2 * L::TILE + wave_u * 1024;
#pragma unroll
    for (int n = 0; n < PASSES; ++n) {
      const int c8 = chunk_of(crow + n * RPP) * 8;
      dma16_at(qb + (int64_t)ec[n].q_off * 8 + c8, slot + n * T * 16);
      dma16_at(ob + (int64_t)ec[n].do_off * 8 + c8, slot + L::TILE + n * T * 16);
    }
  };
  float s_lse2, s_ndelta;
  int s_pos;
  auto load_stats = [&](int u) {
    const int64_t i = stat0 + (int64_t)(es.head_slot >> 6) * a.s_q + es.row;
    s_lse2 = u * 32 + (tid & 31) < n_rows ? a.lse2[i] : INFINITY;      // (rows past the list's end: p = 0)
    s_ndelta = a.delta[i];
    const int64_t rel = a.q_offset + es.row - key0;                    // last key of the workgroup that the row sees
    s_pos = !a.causal || rel > KEYS ? KEYS : (rel < -1 ? -1 : (int)rel);
  };
  auto put_stats = [&](int u) {
    float* st = reinterpret_cast<float*>(smem + L::STAT + (u & 1) * L::STAT_BYTES);
    if (tid < 32) { st[tid] = s_lse2; st[32 + tid] = s_ndelta; reinterpret_cast<int*>(st)[64 + tid] = s_pos; }
  };

  f32x16 dk[DB], dv[DB];
#pragma unroll
  for (int db = 0; db < DB; ++db)
#pragma unroll
    for (int i = 0; i < 16; ++i) { dk[db][i] = 0.f; dv[db][i] = 0.f; }
  const int nt = (n_rows + 31) / 32;
  fetch(0);
  load_stats(0);
  copy(0);
  fetch(1);
  put_stats(0);
  RpBase<D> lo_q, lo_v;          // (one register each: they are short here)
  TrBase<D> lo_t;
  lo_q.init(lane, (int)lds);
  lo_t.init(lane, (int)lds);
  lo_v.init(lane, (int)lds + L::V + wave_u * 32 * D * 2);
  wait_async();
  __syncthreads();
  const float c = a.scale_log2e;
  for (int u = 0; u < nt; ++u) {
    if (u + 1 < nt) {
      load_stats(u + 1);
      copy(u + 1);
      fetch(u + 2);
    }
    const float* st = reinterpret_cast<const float*>(smem + L::STAT + (u & 1) * L::STAT_BYTES);
    f32x16 s, dp;
#pragma unroll
    for (int i4 = 0; i4 < 4; ++i4) {
      const f32x4 nd = *reinterpret_cast<const f32x4*>(st + 32 + 8 * i4 + 4 * g);
#pragma unroll
      for (int e = 0; e < 4; ++e) { s[4 * i4 + e] = 0.f; dp[4 * i4 + e] = nd[e]; }
    }
    constexpr int LOOK = 3;
    bf16x8 buf[LOOK + 1], vbuf[2];
    matrix_run<2 * KS, LOOK>(
        [&](auto m) {
          buf[m % (LOOK + 1)] = lds_rp<D>(lo_q, m / 2, m % 2 * L::TILE);
          if constexpr (m % 2 == 1) vbuf[m / 2 % 2] = lds_rp<D>(lo_v, m / 2, 0);
        },
        [&](auto m) {
          if constexpr (m % 2 == 0) s = mfma32(buf[m % (LOOK + 1)], kreg[m / 2], s);
          else dp = mfma32(buf[m % (LOOK + 1)], vbuf[m / 2 % 2], dp);
        });
    const int pos_lane = reinterpret_cast<const int*>(st)[64 + ql];
    if (__builtin_amdgcn_ballot_w64(pos_lane < wave_u * 32 + 31) != 0) {      // some row does not see all keys of the wave
#pragma unroll
      for (int i4 = 0; i4 < 4; ++i4) {
        typedef int i32x4 __attribute__((ext_vector_type(4)));
        const i32x4 ps = *reinterpret_cast<const i32x4*>(st + 64 + 8 * i4 + 4 * g);
#pragma unroll
        for (int e = 0; e < 4; ++e)
          if (key > ps[e]) { s[4 * i4 + e] = -INFINITY; dp[4 * i4 + e] = 0.f; }      // (what no row sees may be NaN)
      }
    }
#pragma unroll
    for (int i4 = 0; i4 < 4; ++i4) {
      const f32x4 l2 = *reinterpret_cast<const f32x4*>(st + 8 * i4 + 4 * g);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        s[4 * i4 + e] = exp2_fast(__builtin_fmaf(s[4 * i4 + e], c, -l2[e]));
        dp[4 * i4 + e] *= s[4 * i4 + e];
      }
    }
    const bf16x8 p[2] = {pack8(s, 0), pack8(s, 8)}, ds[2] = {pack8(dp, 0), pack8(dp, 8)};      // (bf16 for the matrix unit)
    matrix_run<4 * DB, LOOK>(
        [&](auto m) { buf[m % (LOOK + 1)] = lds_tr<D>(lo_t, m % (2 * DB) / 2, (m % 2 == 0 ? L::TILE : 0) + m / (2 * DB) * 16 * D * 2); },
        [&](auto m) {
          constexpr int half = m / (2 * DB), db = m % (2 * DB) / 2;
          if constexpr (m % 2 == 0) dv[db] = mfma32(buf[m % (LOOK + 1)], p[half], dv[db]);
          else dk[db] = mfma32(buf[m % (LOOK + 1)], ds[half], dk[db]);
        });
    const int step = (u & 1) ? -2 * L::TILE : 2 * L::TILE;
    lo_q.add(step);
    lo_t.add(step);
    wait_async();
    if (u + 1 < nt) put_stats(u + 1);
    __syncthreads();
  }

  item.flush(a, plane, reinterpret_cast<float*>(smem) + wave_u * 32 * kOutRow<D>, dk, dv, wave_u * 32, lane);
}

// 256 keys a workgroup (which block lengths take it: dkdv_keys() in block_api.hip): the phases of the dense dk/dv kernel (dkdv_tile.hpp, attn_bwd.hip) on gathered rows.  Eight waves of 32 keys; waves
// 0-3 and 4-7 alternate matrix and vector phases one phase apart.  The group that is in a vector phase VV(u) copies tile u + 3 (group A
// rows of Q, their statistics and row numbers, group B rows of dO, each lane from the address that its row's entry gives) and the entries of
// tile u + 6.  Gathered rows come from beyond the L2, 1700 cycles and more away, longer than a phase: a group waits at the end of
// MM(u) for what it copied in VV(u - 2) and before, and leaves the copies of VV(u - 1) under way.  Tile t is so in LDS at the end of MM(t - 1),
// where it is needed, entries at the end of MM(t - 4), and they are read in MM(t - 3) for VV(t - 3).
// 8192 rows of 8 heads on 128 blocks of 512 keys, 8 a row: 280 us (920 TFLOP/s; matrix units busy 56 % of it.  By clock reads in a copy of the kernel a tile of
// 32 rows takes 1.9 us, 1140 TFLOP/s while the loop runs, a workgroup's start 7.5 us, its way out 4.3).  In parts of 1536 rows, before short parts went in order of length, it was 314, with copies of tile u + 2
// that are waited for in the next phase 335, with four waves of 32 keys, two workgroups a compute unit and no phases 332.
struct WideLds {
  static constexpr int D = 128, BMQ = 32, SLOTS = 5, TILE = BMQ * D * 2, DO_BASE = SLOTS * TILE;      // rings of Q, dO
  static constexpr int V = 2 * SLOTS * TILE, V_BYTES = 8 * 32 * D * 2;
  static constexpr int STAT = V + V_BYTES, STAT_BYTES = 512;                   // lse2, -delta, row of the slice of a tile's 32 rows; 32 unused
  static constexpr int ENTRY = STAT + SLOTS * STAT_BYTES, ENTRY_SLOTS = 8, ENTRY_BYTES = 32 * (int)sizeof(BlockEntry);      // of either group
  static constexpr int ENTRY_RING = (ENTRY_SLOTS + 1) * ENTRY_BYTES;           // (a copy brings 64 entries: the last slot's second half is nobody's)
  static constexpr int RINGS = ENTRY + 2 * ENTRY_RING, OUT = 8 * 32 * kOutRow<D> * 4, TOTAL = RINGS > OUT ? RINGS : OUT;
};
__global__ __launch_bounds__(512) void block_dkdv_wide_kernel(const BlockArgs a) {
  using L = WideLds;
  constexpr int D = L::D, DB = D / 32, NC = D / 8, GT = 256, RPP = GT / NC, PASSES = 32 / RPP, SLOTS = L::SLOTS, TILE = L::TILE;
  extern __shared__ __attribute__((aligned(1024))) char smem[];
  const int tid = threadIdx.x, lane = tid & 63, g = lane >> 5, ql = lane & 31, wave_u = __builtin_amdgcn_readfirstlane(tid >> 6);
  const bool group_b = wave_u >= 4;
  const int plane = blockIdx.y, b = plane / a.n_kv_heads, hk = plane - b * a.n_kv_heads;
  const DkdvItem<D, 256> item(a, plane, b, hk);
  if (item.none) return;
  const int n_rows = item.it.count, cnt = (n_rows + 31) / 32;
  const BlockEntry* const list = item.list;
  const unsigned lds = lds_addr(smem);

  DkdvState<D, 32> st;
#pragma unroll
  for (int db = 0; db < DB; ++db)
#pragma unroll
    for (int i = 0; i < 16; ++i) { st.dk[db][i] = 0.f; st.dv[db][i] = 0.f; }
  // this group's operand, and its thread's part of a tile copy: rows crow + n * RPP, the chunk that the swizzle puts at its place
  const int gtid = tid & (GT - 1), crow = gtid / NC, cpos = gtid % NC;
  const int c8 = (((((cpos >> 2) ^ crow) & 3) << 2) | (((cpos & 3) ^ (crow >> 2)) & 3)) * 8;
  static_assert(RPP % 16 == 0, "the rows of a thread have one swizzle phase");
  const bf16_t* const src = (group_b ? a.d_out + (int64_t)b * a.do_stride_b + (int64_t)hk * a.group * a.do_stride_h
                                     : a.q + (int64_t)b * a.q_stride_b + (int64_t)hk * a.group * a.q_stride_h) + c8;
  const int64_t stat0 = ((int64_t)b * a.n_q_heads + hk * a.group) * a.s_q;
  const unsigned ring = lds + L::ENTRY + (group_b ? L::ENTRY_RING : 0);
  struct Next { uint32_t off[PASSES], row, head_slot; } nx;      // of the next tile to copy
  auto last_row = [&](int i) { return i < n_rows ? i : n_rows - 1; };
  auto copy_entries = [&](int u) { dma16_at(list + last_row(u * 32 + lane), ring + (u & (L::ENTRY_SLOTS - 1)) * L::ENTRY_BYTES); };
  auto read_entries = [&](int u) {
    const char* p = smem + L::ENTRY + (group_b ? L::ENTRY_RING : 0) + (u & (L::ENTRY_SLOTS - 1)) * L::ENTRY_BYTES;
    const int field = group_b ? (int)offsetof(BlockEntry, do_off) : (int)offsetof(BlockEntry, q_off);
#pragma unroll
    for (int n = 0; n < PASSES; ++n) nx.off[n] = *reinterpret_cast<const uint32_t*>(p + (crow + n * RPP) * sizeof(BlockEntry) + field);
    const BlockEntry* e = reinterpret_cast<const BlockEntry*>(p) + (lane & 31);
    nx.row = e->row;
    nx.head_slot = e->head_slot;
  };
  // Copy instructions of a vector phase, the same number in every one: group B two of them less.
  constexpr int COPIES_B = PASSES + 1, COPIES_A = COPIES_B + 2;
  auto copy_part = [&](int u, unsigned slot, int part) {
    if (part < PASSES)
      dma16_at(src + (int64_t)nx.off[part] * 8, lds + (group_b ? L::DO_BASE : 0) + slot * TILE + part * GT * 16 + (wave_u & 3) * 1024);
    if (part == 2 && !group_b) {                           // (all four waves: the same data, no branch)
      const int i = u * 32 + (lane & 31);
      const int64_t at = stat0 + (int64_t)(nx.head_slot >> 6) * a.s_q + nx.row;
      const float* from = lane < 32 ? (i < n_rows ? a.lse2 + at : a.inf) : a.delta + at;      // (rows past the list's end: p = 0)
      dma4_at(from, lds + L::STAT + slot * L::STAT_BYTES);
      dma4_at(&list[last_row(i)].row, lds + L::STAT + slot * L::STAT_BYTES + 256);
    }
  };
  // prologue: entries of tiles 0 .. 5, then K, V and tiles 0, 1, 2
  for (int u = 0; u < 6; u += 2) copy_entries(u);
  item.load_k(a, wave_u * 32 + ql, g, st.kreg);
  item.copy_v(a, lds + L::V + wave_u * 32 * D * 2, wave_u * 32, lane);
  wait_async();
  __syncthreads();
  for (int u = 0; u < 3; ++u) {
    read_entries(u);
#pragma unroll
    for (int part = 0; part < 3; ++part) copy_part(u, u, part);
  }
  wait_async();
  TrBase<D> lo_qt;         // Q(u-1), transposed; dO(u-1) sits DO_BASE further
  RpBase<D> lo_q, lo_v;    // Q(u) and this wave's V rows, row-packed
  lo_qt.init(lane, (int)lds + (SLOTS - 1) * TILE);     // "Q(-1)": never read
  lo_q.init(lane, (int)lds);
  lo_v.init(lane, (int)lds + L::V + wave_u * 32 * D * 2);
  __syncthreads();

  int slot = 0;            // ring slot of tile u
  auto advance = [&]() {
    lo_q.add(slot == SLOTS - 1 ? -(SLOTS - 1) * TILE : TILE);
    lo_qt.add(slot == 0 ? -(SLOTS - 1) * TILE : TILE);      // Q(u-1) sits in slot - 1
    slot = (slot == SLOTS - 1) ? 0 : slot + 1;
  };
  auto stat_of = [&](int at) { return reinterpret_cast<const float*>(smem + L::STAT + at * L::STAT_BYTES) + 4 * ((fresh(tid) >> 5) & 1); };
  // Rows of the slice from here on see the lane's key (at most s_q; without a mask: all), and whether some row of the call sees only a part
  // of the workgroup's keys
  const int64_t see = a.causal ? item.key0 + wave_u * 32 + ql - a.q_offset : 0;
  const int first_row = see < 0 ? 0 : see < a.s_q ? (int)see : a.s_q;
  const bool diagonal = a.causal && item.key0 + item.kmax - 1 > a.q_offset;
  const float c = a.scale_log2e;
  auto vector_phase = [&](int u, int at) {                 // at: ring slot of tile u
    if (diagonal) {
      const int* rows = reinterpret_cast<const int*>(stat_of(at)) + 64;
#pragma unroll
      for (int i4 = 0; i4 < 4; ++i4) {
        typedef int i32x4 __attribute__((ext_vector_type(4)));
        const i32x4 r = *reinterpret_cast<const i32x4*>(rows + 8 * i4);
#pragma unroll
        for (int e = 0; e < 4; ++e)
          if (r[e] < first_row) { st.s[0][4 * i4 + e] = -INFINITY; st.dp[0][4 * i4 + e] = 0.f; }      // (what no row sees may be NaN)
      }
    }
    const int to = at + 3 < SLOTS ? at + 3 : at + 3 - SLOTS;
    dkdv_vector_phase<D, 32>(st, c, false, 0, 32, 0, [&](int part) {
      if (part < 3) copy_part(u + 3, to, part);
      else copy_entries(u + 6);
    });
  };
  auto wait_old = [&]() {      // the copies of the vector phase before the last
    if (group_b) wait_copies<COPIES_B>();
    else wait_copies<COPIES_A>();
  };
  // Both groups run the same code; group B starts one phase (one barrier) later and group A idles one phase at the end.
  if (group_b) phase_end();
  read_entries(3);
  { DkdvMatrixPhase<D, 8, 32, false, true, 2, L> ph{lo_qt, lo_q, lo_v, st, stat_of(0)}; ph.run(); }     // scores of tile 0
  advance();
  phase_end();
  for (int u = 0; u + 1 < cnt; ++u) {
    const int at = slot == 0 ? SLOTS - 1 : slot - 1;
    vector_phase(u, at);
    phase_end();
    asm volatile("" : "+v"(lo_v.off0));      // (V never moves: without this the offsets of its blocks are kept in registers across the loop)
    read_entries(u + 4);
    { DkdvMatrixPhase<D, 8, 32, true, true, 2, L> ph{lo_qt, lo_q, lo_v, st, stat_of(slot)}; ph.run(); }    // sums of tile u, scores of tile u+1
    advance();
    wait_old();
    phase_end();
  }
  vector_phase(cnt - 1, slot == 0 ? SLOTS - 1 : slot - 1);
  phase_end();
  { DkdvMatrixPhase<D, 8, 32, true, false, 2, L> ph{lo_qt, lo_q, lo_v, st, nullptr}; ph.run(); }     // sums of the last tile
  wait_async();
  phase_end();
  if (!group_b) phase_end();
  item.flush(a, plane, reinterpret_cast<float*>(smem) + wave_u * 32 * kOutRow<D>, st.dk, st.dv, wave_u * 32, fresh(tid) & 63);
}

// ------------------------------------------------------------------------------------ reduce
// dq (+)= the partial dq of the slots that have one, in slot order; D / 4 lanes a row.
template <int D, bool F32>
SP_DEV void reduce_dq(const BlockArgs& a, int plane, int64_t gid) {
  constexpr int NC = D / 4;
  const int64_t rows = (int64_t)a.group * a.s_q, rh = gid / NC, row = plane * rows + rh;      // (plane = batch index * kv heads + kv head)
  const int c = (int)(gid - rh * NC) * 4;
  if (rh >= rows) return;
  const float* lp = a.part_lse + row * a.top_k;
  f32x4 x = {0, 0, 0, 0};
#pragma unroll 4
  for (int s = 0; s < a.top_k; ++s)
    if (lp[s] != -INFINITY) {
      const int64_t at = (row * a.top_k + s) * D + c;
      if constexpr (F32) {
        x += *reinterpret_cast<const f32x4*>(static_cast<const float*>(a.part_out) + at);
      } else {
        const f16x4 y = *reinterpret_cast<const f16x4*>(static_cast<const _Float16*>(a.part_out) + at);
        const float w = a.part_scale[row * a.top_k + s];
#pragma unroll
        for (int e = 0; e < 4; ++e) x[e] += w * (float)y[e];
      }
    }
  const int64_t bh = row / a.s_q, b = bh / a.n_q_heads;
  const int64_t to = b * a.q_stride_b + (row - bh * a.s_q) * a.q_stride_s + (bh - b * a.n_q_heads) * a.q_stride_h + c;
  if (a.dq_f32) {
    f32x4* dst = reinterpret_cast<f32x4*>(static_cast<float*>(a.dq) + to);
    if (a.dq_accumulate) x += *dst;
    *dst = x;
  } else {
    *reinterpret_cast<bf16x4*>(static_cast<bf16_t*>(a.dq) + to) = __builtin_convertvector(x, bf16x4);
  }
}

// dk, dv of the keys whose workgroups left partial sums (in list order) and of those that nobody chose; D / 4 lanes a key.
// (From a multiple of four keys on: the keys of a wave then lie in one chunk, whose length is a multiple of 256, as kv_chunk_of has it.)
SP_HOST_DEV int64_t dkdv_reduce_first(const BlockArgs& a) { return a.kv_begin & ~(int64_t)3; }
template <int D>
SP_DEV void reduce_dkdv(const BlockArgs& a, int plane, int64_t gid) {
  constexpr int NC = D / 4;
  const int keys_pad = a.n_sub * a.dkdv_keys;
  const int64_t kk = gid / NC;
  const int c = (int)(gid - kk * NC) * 4, b = plane / a.n_kv_heads, hk = plane - b * a.n_kv_heads;
  const int64_t key = dkdv_reduce_first(a) + kk;
  if (key < a.kv_begin || key >= a.kv_end_range) return;
  const int64_t block = key / a.block_len, j = block - a.first_block;
  uint32_t len = 0, part0 = 0;
  int parts = 0;
  if (key < a.kv_end) {
    const BlockList& l = a.lists[(int64_t)plane * a.n_blocks + j];
    len = l.len; parts = (int)l.parts; part0 = l.part0;
  }
  if (len > 0 ? parts == 0 : a.dkv_accumulate != 0) return;
  const int chunk = kv_chunk_of(a.kv, key);
  const int64_t to = (int64_t)b * a.kv_stride_b + (int64_t)hk * a.kv_stride_h + (key - (int64_t)chunk * a.kv.len) * a.kv_stride_s + c;
  f32x4* kd = reinterpret_cast<f32x4*>(a.dk_acc[chunk] + to);
  f32x4* vd = reinterpret_cast<f32x4*>(a.dv_acc[chunk] + to);
  f32x4 k4 = {0, 0, 0, 0}, v4 = {0, 0, 0, 0};
  const float* src = a.dkdv_part + (((int64_t)plane * a.part_cap + part0) * 2 * keys_pad + (key - block * a.block_len)) * D + c;
#pragma unroll 4
  for (int i = 0; i < parts; ++i) {
    k4 += *reinterpret_cast<const f32x4*>(src + (int64_t)i * 2 * keys_pad * D);
    v4 += *reinterpret_cast<const f32x4*>(src + (int64_t)(2 * i + 1) * keys_pad * D);
  }
  if (a.dkv_accumulate) { k4 += *kd; v4 += *vd; }
  *kd = k4;
  *vd = v4;
}

// Both in one launch: dq_wgs workgroups for the rows of the plane (blockIdx.y), the others for its keys.  Bound by the bytes: 65536 rows of 8 slots of
// 128, 65536 keys with 2 to 3 parts each 70 us (two launches took 67, and 5 us more where there is little to add up).
template <int D, bool F32>
__global__ __launch_bounds__(256) void block_reduce_kernel(const BlockArgs a, int dq_wgs) {
  if ((int)blockIdx.x < dq_wgs) reduce_dq<D, F32>(a, blockIdx.y, (int64_t)blockIdx.x * 256 + threadIdx.x);
  else reduce_dkdv<D>(a, blockIdx.y, (int64_t)((int)blockIdx.x - dq_wgs) * 256 + threadIdx.x);
}

hipError_t launch_block_bwd_dq(const BlockArgs& a, int head_dim, hipStream_t st) {
  dim3 grid((unsigned)a.item_cap, (unsigned)(a.batch * a.n_kv_heads)), block(256);
  if (head_dim == 128) hipLaunchKernelGGL(block_dq_kernel<128>, grid, block, block_dq_lds_bytes<128>(), st, a);
  else hipLaunchKernelGGL(block_dq_kernel<64>, grid, block, block_dq_lds_bytes<64>(), st, a);
  return hipGetLastError();
}
template <int D, int NW>
static void launch_dkdv_t(const BlockArgs& a, hipStream_t st) {
  dim3 grid((unsigned)a.dkdv_cap, (unsigned)(a.batch * a.n_kv_heads)), block(NW * 64);
  hipLaunchKernelGGL((block_dkdv_kernel<D, NW>), grid, block, (BlockDkdvLds<D, NW>::TOTAL), st, a);
}
hipError_t launch_block_bwd_dkdv(const BlockArgs& a, int head_dim, hipStream_t st) {
  if (a.dkdv_keys == 256) hipLaunchKernelGGL(block_dkdv_wide_kernel, dim3((unsigned)a.dkdv_cap, (unsigned)(a.batch * a.n_kv_heads)), dim3(512), WideLds::TOTAL, st, a);
  else if (head_dim == 128) a.dkdv_keys == 128 ? launch_dkdv_t<128, 4>(a, st) : launch_dkdv_t<128, 2>(a, st);
  else a.dkdv_keys == 128 ? launch_dkdv_t<64, 4>(a, st) : launch_dkdv_t<64, 2>(a, st);
  return hipGetLastError();
}
hipError_t launch_block_reduce(const BlockArgs& a, int head_dim, hipStream_t st) {
  const int64_t per = head_dim / 4, keys = a.kv_end_range - dkdv_reduce_first(a);
  const int64_t dq_wgs = ((int64_t)a.group * a.s_q * per + 255) / 256, dkdv_wgs = (keys * per + 255) / 256;
  auto go = [&](auto kernel) {
    hipLaunchKernelGGL(kernel, dim3((unsigned)(dq_wgs + dkdv_wgs), (unsigned)(a.batch * a.n_kv_heads)), dim3(256), 0, st, a, (int)dq_wgs);
  };
  if (head_dim == 128) a.part_f32 ? go(block_reduce_kernel<128, true>) : go(block_reduce_kernel<128, false>);
  else a.part_f32 ? go(block_reduce_kernel<64, true>) : go(block_reduce_kernel<64, false>);
  return hipGetLastError();
}

hipError_t opt_in_block_bwd_kernels() {
  const hipFuncAttribute attr = hipFuncAttributeMaxDynamicSharedMemorySize;
  hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(&block_dq_kernel<128>), attr, (int)block_dq_lds_bytes<128>());
  if (e == hipSuccess) e = hipFuncSetAttribute(reinterpret_cast<const void*>(&block_dq_kernel<64>), attr, (int)block_dq_lds_bytes<64>());
  if (e == hipSuccess) e = hipFuncSetAttribute(reinterpret_cast<const void*>(&block_dkdv_wide_kernel), attr, WideLds::TOTAL);
  if (e == hipSuccess) e = hipFuncSetAttribute(reinterpret_cast<const void*>(&block_dkdv_kernel<128, 4>), attr, (int)BlockDkdvLds<128, 4>::TOTAL);
  if (e == hipSuccess) e = hipFuncSetAttribute(reinterpret_cast<const void*>(&block_dkdv_kernel<128, 2>), attr, (int)BlockDkdvLds<128, 2>::TOTAL);
  if (e == hipSuccess) e = hipFuncSetAttribute(reinterpret_cast<const void*>(&block_dkdv_kernel<64, 4>), attr, (int)BlockDkdvLds<64, 4>::TOTAL);
  if (e == hipSuccess) e = hipFuncSetAttribute(reinterpret_cast<const void*>(&block_dkdv_kernel<64, 2>), attr, (int)BlockDkdvLds<64, 2>::TOTAL);
  return e;
}

}  // namespace slimpipe
