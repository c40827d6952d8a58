// Choosing the key blocks of sparse attention: block means, scores with their top-k, and the lists that turn "the blocks of a row"
// into "the rows of a block".
#include "blocks.hpp"
#include "tile_common.hpp"

namespace slimpipe {

// ------------------------------------------------------------------------------------ block means
// mean[j] = (1 / n_j) sum of the n_j keys that block j holds before kv_end.  One workgroup a block and kv head, D / 8 lanes a row
// (16 bytes each); sums in 64 bits, in which sums of bf16 numbers of like size are exact, so that the mean is rounded once (to 32
// bits) and does not depend on the order.  Bound by reading the keys once.
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
// score[r][j] = q_r . mean_j in 64 bits.  A workgroup takes 16 rows of a plane (they share the means); its four waves share out the
// blocks, 16 at a time on the matrix unit (v_mfma_f64_16x16x4: a lane holds row or block lane & 15, contraction index lane >> 4;
// result register i of a lane is row 4 i + (lane >> 4), column lane & 15), and leave the scores rounded to 32 bits in LDS.
// Rounding keeps order, so only equal 32-bit scores at the border are looked at again, in 64 bits.  Then every wave picks the blocks of
// four rows, the largest score first: scores in registers as unsigned numbers of the same order, a maximum over the wave,
// and all that equal it are taken at once while there is room for them.  Blocks come in chunks of kSelBlocks; what is taken of one
// competes with the next one's.
constexpr int kSelRows = 16, kSelBlocks = 512, kSelRegs = kSelBlocks / 64;

// The order of floats as unsigned numbers: 0 stays free for "no candidate", NaN comes before all others.
SP_DEV uint32_t score_key(float x) {
  uint32_t u = __float_as_uint(x);
  if ((u & 0x7fffffffu) > 0x7f800000u) return 1u;
  if (u == 0x80000000u) u = 0u;                      // -0 = 0
  return (u & 0x80000000u) ? ~u : u | 0x80000000u;   // (-inf: 0x007fffff)
}
SP_DEV uint32_t wave_max(uint32_t v) {
#pragma unroll
  for (int w = 1; w < 64; w <<= 1) {
    const uint32_t o = (uint32_t)__shfl_xor((int)v, w, 64);
    v = v > o ? v : o;
  }
  return v;
}

template <int D>
__global__ __launch_bounds__(256) void block_select_kernel(const BlockSelectArgs a) {
  typedef double f64x4 __attribute__((ext_vector_type(4)));
  constexpr int ROW = kSelBlocks + 1;                // (padded: a column of the tile is 4 banks apart)
  __shared__ uint32_t keys[kSelRows * ROW];
  __shared__ uint32_t carry_key[kSelRows][kMaxTopK];
  __shared__ int32_t carry_idx[kSelRows][kMaxTopK];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int hk = blockIdx.y, b = blockIdx.z;
  const int rows = a.group * a.s_q, row0 = blockIdx.x * kSelRows;
  const float* const means = a.means + ((int64_t)b * a.n_kv_heads + hk) * a.blocks_total * D;
  const int end_block = a.first_block + a.n_blocks;

  auto row_ptr = [&](int rh) {
    const int hl = rh / a.s_q, r = rh - hl * a.s_q;
    return a.q + (int64_t)b * a.q_stride_b + (int64_t)r * a.q_stride_s + (int64_t)(hk * a.group + hl) * a.q_stride_h;
  };
  // one past the last block that competes for a row, and whether the row's own block is taken before all others
  auto own_block = [&](int rh) { return a.causal ? (a.q_offset + rh % a.s_q) / a.block_len : (int64_t)end_block; };

  // this lane's row as A operand: contraction step (v, e) of group g is head_dim 16 v + 4 g + e
  double q[D / 4];
  {
    const int rh = row0 + (lane & 15);
    const bf16_t* p = row_ptr(rh < rows ? rh : rows - 1) + 4 * (lane >> 4);
#pragma unroll
    for (int v = 0; v < D / 16; ++v) {
      const bf16x4 x = *reinterpret_cast<const bf16x4*>(p + 16 * v);
#pragma unroll
      for (int e = 0; e < 4; ++e) q[4 * v + e] = (double)(float)x[e];
    }
  }
  // blocks behind the last own block of the rows are nobody's candidates
  int64_t last = 0;
  for (int i = 0; i < kSelRows && row0 + i < rows; ++i) {
    const int64_t o = own_block(row0 + i);
    last = o > last ? o : last;
  }
  const int stop = last < end_block ? (int)last : end_block;
  int carried[4] = {0, 0, 0, 0};                     // of the wave's four rows

  for (int c0 = a.first_block; c0 < stop; c0 += kSelBlocks) {
    const int n = stop - c0 < kSelBlocks ? stop - c0 : kSelBlocks;
    for (int t = wave; t * 16 < n; t += 4) {
      const int j = c0 + t * 16 + (lane & 15);
      const float* mp = means + (int64_t)(j < stop ? j : stop - 1) * D + 4 * (lane >> 4);
      f32x4 m[D / 16];
#pragma unroll
      for (int v = 0; v < D / 16; ++v) m[v] = *reinterpret_cast<const f32x4*>(mp + 16 * v);
      f64x4 s = {0, 0, 0, 0};
#pragma unroll
      for (int v = 0; v < D / 16; ++v)
#pragma unroll
        for (int e = 0; e < 4; ++e) s = __builtin_amdgcn_mfma_f64_16x16x4f64(q[4 * v + e], (double)m[v][e], s, 0, 0, 0);
#pragma unroll
      for (int i = 0; i < 4; ++i) keys[(4 * i + (lane >> 4)) * ROW + t * 16 + (lane & 15)] = score_key((float)s[i]);
    }
    __syncthreads();
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      const int rl = wave * 4 + w, rh = row0 + rl;
      if (rh >= rows) continue;
      const int64_t own = own_block(rh);
      const bool forced = a.causal && own >= a.first_block && own < end_block;
      int need = a.top_k - (forced ? 1 : 0);
      // register 0: what the chunks before left (their blocks come first); then the chunk's, 64 blocks a register
      uint32_t k[kSelRegs + 1];
      k[0] = lane < carried[w] ? carry_key[rl][lane] : 0u;
#pragma unroll
      for (int i = 0; i < kSelRegs; ++i) {
        const int at = 64 * i + lane;
        k[i + 1] = at < n && c0 + at < own ? keys[rl * ROW + at] : 0u;
      }
      uint32_t taken = 0;                            // bit i: this lane's candidate of register i
      while (need > 0) {
        uint32_t m = 0;
#pragma unroll
        for (int i = 0; i <= kSelRegs; ++i) m = m > k[i] ? m : k[i];
        m = wave_max(m);
        if (m == 0) break;
        int cnt = 0;
#pragma unroll
        for (int i = 0; i <= kSelRegs; ++i) cnt += __popcll(__builtin_amdgcn_ballot_w64(k[i] == m));
        if (cnt <= need) {
#pragma unroll
          for (int i = 0; i <= kSelRegs; ++i)
            if (k[i] == m) { k[i] = 0; taken |= 1u << i; }
          need -= cnt;
          continue;
        }
        // More equal 32-bit scores than room: their scores in 64 bits, each lane its own candidates; then the largest of them, the
        // lowest index first (lanes ascend within a register, registers ascend).
        const bf16_t* qp = row_ptr(rh);
        double d[kSelRegs + 1];
#pragma unroll
        for (int i = 0; i <= kSelRegs; ++i) {
          d[i] = -INFINITY;
          if (k[i] == m) {
            const int j = i == 0 ? carry_idx[rl][lane] : c0 + 64 * (i - 1) + lane;
            const float* mp = means + (int64_t)j * D;
            double s = 0;
            for (int e = 0; e < D; ++e) s += (double)(float)qp[e] * (double)mp[e];
            d[i] = s == s ? s : -INFINITY;           // (NaN: all alike, the lowest index first)
          }
        }
        while (need > 0) {
          double best = -INFINITY;
#pragma unroll
          for (int i = 0; i <= kSelRegs; ++i)
            if (k[i] == m && d[i] > best) best = d[i];
#pragma unroll
          for (int w2 = 1; w2 < 64; w2 <<= 1) {
            const double o = __shfl_xor(best, w2, 64);
            best = o > best ? o : best;
          }
          bool found = false;
#pragma unroll
          for (int i = 0; i <= kSelRegs; ++i) {
            const uint64_t eq = __builtin_amdgcn_ballot_w64(k[i] == m && d[i] == best);
            if (!found && eq) {
              found = true;
              if (lane == __ffsll((unsigned long long)eq) - 1) { k[i] = 0; taken |= 1u << i; }
            }
          }
          --need;
        }
      }
      // what was taken, in ascending order
      int at = 0;
      uint32_t out_key[kSelRegs + 1];
      int out_idx[kSelRegs + 1], out_at[kSelRegs + 1];
#pragma unroll
      for (int i = 0; i <= kSelRegs; ++i) {
        const uint64_t mask = __builtin_amdgcn_ballot_w64((taken >> i) & 1u);
        out_at[i] = (taken >> i) & 1u ? at + __popcll(mask & ((1ull << lane) - 1ull)) : -1;
        at += __popcll(mask);
        out_idx[i] = out_key[i] = 0;
        if (out_at[i] >= 0) {
          out_key[i] = i == 0 ? carry_key[rl][lane] : keys[rl * ROW + 64 * (i - 1) + lane];
          out_idx[i] = i == 0 ? carry_idx[rl][lane] : c0 + 64 * (i - 1) + lane;
        }
      }
      __builtin_amdgcn_wave_barrier();
#pragma unroll
      for (int i = 0; i <= kSelRegs; ++i)
        if (out_at[i] >= 0) { carry_key[rl][out_at[i]] = out_key[i]; carry_idx[rl][out_at[i]] = out_idx[i]; }
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
      __builtin_amdgcn_wave_barrier();
      carried[w] = at;
    }
    __syncthreads();
  }
#pragma unroll
  for (int w = 0; w < 4; ++w) {
    const int rl = wave * 4 + w, rh = row0 + rl;
    if (rh >= rows || lane >= a.top_k) continue;
    const int64_t own = own_block(rh);
    const bool forced = a.causal && own >= a.first_block && own < end_block;
    const int hl = rh / a.s_q, r = rh - hl * a.s_q;
    const int v = lane < carried[w] ? carry_idx[rl][lane] : (lane == carried[w] && forced ? (int)own : -1);
    a.index[(((int64_t)b * a.n_q_heads + hk * a.group + hl) * a.s_q + r) * a.top_k + lane] = v;
  }
}

hipError_t launch_block_select(const BlockSelectArgs& a, int head_dim, hipStream_t st) {
  dim3 grid((unsigned)((a.group * (int64_t)a.s_q + kSelRows - 1) / kSelRows), (unsigned)a.n_kv_heads, (unsigned)a.batch), block(256);
  if (head_dim == 128) hipLaunchKernelGGL(block_select_kernel<128>, grid, block, 0, st, a);
  else hipLaunchKernelGGL(block_select_kernel<64>, grid, block, 0, st, a);
  return hipGetLastError();
}

// ------------------------------------------------------------------------------------ lists
// The rows of every block, in ascending order of (head of the group, row).  Count and fill go over chunks of kListRows rows with a bit
// per (block, row) in LDS: setting bits commutes, and a row's place in the block's list is a count of the bits below its own, so the
// lists are the same on every run.
SP_DEV int64_t list_row_base(const BlockArgs& a, int b, int hk, int rh, int* hl, int* r) {
  *hl = rh / a.s_q;
  *r = rh - *hl * a.s_q;
  return ((int64_t)b * a.n_q_heads + hk * a.group + *hl) * a.s_q + *r;
}
template <bool FILL>
__global__ __launch_bounds__(kListRows) void block_list_kernel(const BlockArgs a) {
  extern __shared__ uint32_t bits[];                 // [blocks of the window][kListRows / 32]
  constexpr int W = kListRows / 32;
  const int tid = threadIdx.x, chunk = blockIdx.x, plane = blockIdx.y;
  const int b = plane / a.n_kv_heads, hk = plane - b * a.n_kv_heads;
  const int rows = a.group * a.s_q, rh = chunk * kListRows + tid;
  int hl = 0, r = 0;
  const int64_t row = rh < rows ? list_row_base(a, b, hk, rh, &hl, &r) : 0;
  const int32_t* idx = a.index + row * a.top_k;
  uint64_t valid = 0;
  if (rh < rows)
    for (int s = 0; s < a.top_k; ++s)
      if (block_slot_valid(a, idx, s, a.q_offset + r)) valid |= 1ull << s;
  uint32_t* counts = a.counts + ((int64_t)plane * a.n_list_chunks + chunk) * a.n_blocks;
  for (int w0 = 0; w0 < a.n_blocks; w0 += kListBlocks) {
    const int n = a.n_blocks - w0 < kListBlocks ? a.n_blocks - w0 : kListBlocks;
    __syncthreads();
    for (int i = tid; i < n * W; i += kListRows) bits[i] = 0u;
    __syncthreads();
    for (uint64_t v = valid; v; v &= v - 1) {
      const int j = idx[__ffsll((unsigned long long)v) - 1] - a.first_block - w0;
      if (j >= 0 && j < n) atomicOr(&bits[j * W + (tid >> 5)], 1u << (tid & 31));
    }
    __syncthreads();
    if constexpr (!FILL) {
      for (int j = tid; j < n; j += kListRows) {
        uint32_t c = 0;
        for (int w = 0; w < W; ++w) c += __popc(bits[j * W + ((w + j) & (W - 1))]);
        counts[w0 + j] = c;
      }
    } else {
      BlockEntry* entries = a.entries + (int64_t)plane * rows * a.top_k;
      const uint32_t* start = a.start + (int64_t)plane * a.n_blocks;
      for (uint64_t v = valid; v; v &= v - 1) {
        const int s = __ffsll((unsigned long long)v) - 1, j = idx[s] - a.first_block - w0;
        if (j < 0 || j >= n) continue;
        uint32_t at = start[w0 + j] + counts[w0 + j];
        for (int w = 0; w < (tid >> 5); ++w) at += __popc(bits[j * W + w]);
        at += __popc(bits[j * W + (tid >> 5)] & ((1u << (tid & 31)) - 1u));
        entries[at] = {(uint32_t)r, (uint32_t)(hl << 6 | s)};
      }
    }
  }
  if (FILL && rh < rows)                             // slots without a result: nothing else writes them
    for (int s = 0; s < a.top_k; ++s) a.part_lse[row * a.top_k + s] = (valid >> s) & 1u ? 0.f : -INFINITY;
}

// One workgroup a plane: counts of the chunks -> where each chunk's rows start in the block's list, list starts, tiles.
constexpr int kScanThreads = 1024, kScanCols = 128, kScanSegs = kScanThreads / kScanCols;
SP_DEV uint32_t scan_add(uint32_t* tmp, int tid, uint32_t v, uint32_t* total) {      // exclusive scan over the workgroup
  const int lane = tid & 63, wave = tid >> 6;
  uint32_t x = v;
#pragma unroll
  for (int w = 1; w < 64; w <<= 1) {
    const uint32_t o = (uint32_t)__shfl_up((int)x, w, 64);
    if (lane >= w) x += o;
  }
  __syncthreads();
  if (lane == 63) tmp[wave] = x;
  __syncthreads();
  uint32_t before = 0, all = 0;
  for (int w = 0; w < kScanThreads / 64; ++w) {
    if (w < wave) before += tmp[w];
    all += tmp[w];
  }
  *total = all;
  return before + x - v;
}
__global__ __launch_bounds__(kScanThreads) void block_scan_kernel(const BlockArgs a, int dkdv) {
  __shared__ uint32_t seg[kScanSegs][kScanCols], tmp[kScanThreads / 64];
  const int tid = threadIdx.x, plane = blockIdx.x, nb = a.n_blocks, nc = a.n_list_chunks;
  uint32_t* counts = a.counts + (int64_t)plane * nc * nb;
  uint32_t* totals = a.start + (int64_t)plane * nb;              // (lengths first, starts in their place afterwards)
  const int per = (nc + kScanSegs - 1) / kScanSegs;
  for (int j0 = 0; j0 < nb; j0 += kScanCols) {
    const int col = tid % kScanCols, s = tid / kScanCols, j = j0 + col;
    const int c0 = s * per, c1 = c0 + per < nc ? c0 + per : nc;
    uint32_t sum = 0;
    if (j < nb)
      for (int c = c0; c < c1; ++c) sum += counts[(int64_t)c * nb + j];
    __syncthreads();
    seg[s][col] = sum;
    __syncthreads();
    if (j < nb) {
      uint32_t at = 0;
      for (int i = 0; i < s; ++i) at += seg[i][col];
      for (int c = c0; c < c1; ++c) {
        const uint32_t x = counts[(int64_t)c * nb + j];
        counts[(int64_t)c * nb + j] = at;
        at += x;
      }
      if (s == kScanSegs - 1) totals[j] = at;
    }
  }
  __threadfence_block();
  __syncthreads();
  uint32_t first = 0, tile = 0, item = 0, part = 0;              // running totals of the blocks before
  for (int j0 = 0; j0 < nb; j0 += kScanThreads) {
    const int j = j0 + tid;
    const uint32_t len = j < nb ? totals[j] : 0u;
    const uint32_t tiles = (len + kBlockTileRows - 1) / kBlockTileRows;
    uint32_t sum_len, sum_tiles;
    const uint32_t f = first + scan_add(tmp, tid, len, &sum_len);
    const uint32_t t = tile + scan_add(tmp, tid, tiles, &sum_tiles);
    first += sum_len;
    tile += sum_tiles;
    if (j < nb) {
      totals[j] = f;
      BlockItem* it = a.items + (int64_t)plane * a.item_cap + t;
      for (uint32_t i = 0; i < tiles; ++i) {
        const uint32_t left = len - i * kBlockTileRows;
        it[i] = {a.first_block + j, (int)(f + i * kBlockTileRows), (int)(left < kBlockTileRows ? left : kBlockTileRows), 0};
      }
    }
    if (dkdv) {
      const uint32_t rows = (uint32_t)a.chunk_rows, chunks = (len + rows - 1) / rows, parts = chunks > 1 ? chunks : 0u;
      uint32_t sum_items, sum_parts;
      const uint32_t i0 = item + scan_add(tmp, tid, chunks * (uint32_t)a.n_sub, &sum_items);
      const uint32_t p0 = part + scan_add(tmp, tid, parts, &sum_parts);
      item += sum_items;
      part += sum_parts;
      if (j < nb) {
        a.sums[(int64_t)plane * nb + j] = {(int)len, (int)parts, (int)p0, 0};
        BlockItem* it = a.dkdv_items + (int64_t)plane * a.dkdv_cap + i0;
        for (uint32_t c = 0; c < chunks; ++c)
          for (int s = 0; s < a.n_sub; ++s) {
            const uint32_t left = len - c * rows;
            *it++ = {(a.first_block + j) * a.n_sub + s, (int)(f + c * rows), (int)(left < rows ? left : rows), parts ? (int)(p0 + c) : -1};
          }
      }
    }
  }
  if (tid == 0) {
    a.n_items[plane] = (int)tile;
    if (dkdv) a.n_dkdv_items[plane] = (int)item;
  }
}

static size_t list_lds_bytes(const BlockArgs& a) {
  return (size_t)(a.n_blocks < kListBlocks ? a.n_blocks : kListBlocks) * (kListRows / 32) * 4;
}
hipError_t launch_block_lists(const BlockArgs& a, bool dkdv, hipStream_t st) {
  const int planes = a.batch * a.n_kv_heads;
  dim3 grid((unsigned)a.n_list_chunks, (unsigned)planes);
  hipLaunchKernelGGL(block_list_kernel<false>, grid, dim3(kListRows), list_lds_bytes(a), st, a);
  hipLaunchKernelGGL(block_scan_kernel, dim3((unsigned)planes), dim3(kScanThreads), 0, st, a, dkdv ? 1 : 0);
  hipLaunchKernelGGL(block_list_kernel<true>, grid, dim3(kListRows), list_lds_bytes(a), st, a);
  return hipGetLastError();
}

hipError_t opt_in_block_select_kernels() {
  const hipFuncAttribute attr = hipFuncAttributeMaxDynamicSharedMemorySize;
  const int most = kListBlocks * (kListRows / 32) * 4;
  hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(&block_list_kernel<false>), attr, most);
  if (e == hipSuccess) e = hipFuncSetAttribute(reinterpret_cast<const void*>(&block_list_kernel<true>), attr, most);
  return e;
}

}  // namespace slimpipe
