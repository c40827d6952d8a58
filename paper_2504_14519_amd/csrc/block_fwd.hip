// Forward of sparse attention over selected key blocks.
//
// A tile is up to 128 rows that chose one block (block_select.hip): four waves of 32 rows each, the block's keys in tiles of 64 through
// two LDS slots.  Every (row, slot) leaves out and lse of its block's keys; part_merge.hip folds a row's slots in 32 bits.  Where the result is
// bf16 the partial outs have 16 bits (float16 with a float32 scale a row; lse is float32 always): rounded to 2^-11 of themselves they add an
// eighth of what one rounding to bf16 does, and the bytes of the partial outs, which every one of them costs twice, are what the fold and a
// third of the tiles' epilogue take.
// 8192 rows of 8 heads of 128 on 128 blocks of 512 keys, 8 a row: 179 us (720 TFLOP/s; matrix units busy 41 % of it).  By clock reads in a copy of the
// kernel a workgroup starts for 3.2 us, is 14 in its 8 tiles of keys (1210 TFLOP/s over the chip) and 2.2 on its way out, behind the other one of its
// compute unit in part.  3 x 1337 rows of 12 heads of 64 on 64 blocks of
// 64 keys, 12 a row: 37 us.
#include "block_tile.hpp"
#include "row_tile.hpp"
#include "tile_common.hpp"

namespace slimpipe {

constexpr int kBlockTileKeys = 64;

template <int D>
constexpr size_t block_fwd_lds_bytes() {       // two slots of K and V; the output rows on their way out take their place
  constexpr size_t rings = (size_t)4 * kBlockTileKeys * D * 2, rows = (size_t)4 * 32 * kOutRow<D> * 4;
  return rings > rows ? rings : rows;
}

template <int D>
__global__ __launch_bounds__(256, 2) void block_fwd_kernel(const BlockArgs a) {
  constexpr int BN = kBlockTileKeys, TILE = BN * D * 2;
  extern __shared__ __attribute__((aligned(1024))) char smem[];
  const int tid = threadIdx.x, lane = tid & 63, g = lane >> 5, wave_u = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int plane = blockIdx.y, b = plane / a.n_kv_heads, hk = plane - b * a.n_kv_heads;
  const TileRows rows(a, plane, wave_u, lane);
  if (rows.none) return;
  const BlockItem it = rows.item;
  const BlockEntry e = rows.e;
  const int n_rows = it.count, mine = rows.mine;
  const int h = hk * a.group + (int)(e.head_slot >> 6);

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

  RowState<D> st;
  st.init();
  if (nt > 0) {
    copy(0);
    {
      const bf16_t* qp = a.q + (int64_t)b * a.q_stride_b + (int64_t)hk * a.group * a.q_stride_h + (int64_t)e.q_off * 8 + 8 * g;
#pragma unroll
      for (int ks = 0; ks < D / 16; ++ks) st.q[ks] = *reinterpret_cast<const bf16x8*>(qp + 16 * ks);
    }
    RpOffsets<D> lo_k;
    TrOffsets<D> lo_v;
    lo_k.init(lane, (int)lds);
    lo_v.init(lane, (int)lds + TILE);
    wait_async();
    __syncthreads();
    for (int t = 0; t < nt; ++t) {
      if (t + 1 < nt) copy(t + 1);
      const int kmax = see_rel - t * BN;
      const bool masked = __builtin_amdgcn_ballot_w64(kmax < BN - 1) != 0;
      attend_tile<D, BN>(st, lo_k, lo_v, a.scale_log2e, masked, 0, kmax, g);
      const int step = (t & 1) ? -2 * TILE : 2 * TILE;
      lo_k.add(step);
      lo_v.add(step);
      wait_async();
      __syncthreads();
    }
  }
  float lse;
  const float norm = st.finish(&lse);
  const int64_t slot = (((int64_t)b * a.n_q_heads + h) * a.s_q + e.row) * a.top_k + (e.head_slot & 63u);
  if (lane < 32 && mine < n_rows) a.part_lse[slot] = lse;
  store_parts<D>(a, reinterpret_cast<float*>(smem) + wave_u * 32 * kOutRow<D>, st.o, norm, slot, n_rows, wave_u, lane);
}

// Calls of few rows (tokens): lists and tiles of 128 rows would be mostly empty, so each (row, slot) has a workgroup of its own, whose four
// waves share out the block's keys.  D / 8 lanes a key row: products summed over these lanes, then every lane weighs its 8 elements of V.
// Bound by memory: 4 tokens of 8 heads of 128, 16 blocks of 256 keys each, 14 us (4.7 TB/s).
template <int D>
__global__ __launch_bounds__(256) void block_fwd_few_kernel(const BlockArgs a) {
  constexpr int NC = D / 8, PER = 64 / NC, STEP = 8;           // lanes a key, keys a wave's load, loads in flight
  __shared__ float acc_s[4][D], m_s[4], l_s[4];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, sub = lane / NC, c = lane % NC;
  const int64_t item = blockIdx.x;
  const int slot = (int)(item % a.top_k);
  const int64_t row = item / a.top_k;
  const int64_t bh = row / a.s_q;
  const int r = (int)(row - bh * a.s_q), b = (int)(bh / a.n_q_heads), h = (int)(bh - (int64_t)b * a.n_q_heads), hk = h / a.group;
  const int32_t* idx = a.index + row * a.top_k;
  const int64_t pos = a.q_offset + r;
  if (!block_slot_valid(a, idx, slot, pos)) {
    if (tid == 0) a.part_lse[item] = -INFINITY;
    return;
  }
  const BlockKeys keys(a, idx[slot], b, hk);
  const int64_t hi = a.causal && pos + 1 < keys.hi ? pos + 1 : keys.hi;
  const int n = hi > keys.lo ? (int)(hi - keys.lo) : 0;
  const bf16_t* const kp = a.kv.k[keys.chunk] + keys.off + c * 8;
  const bf16_t* const vp = a.kv.v[keys.chunk] + keys.off + c * 8;
  float q[8];
  {
    const bf16x8 x = *reinterpret_cast<const bf16x8*>(a.q + (int64_t)b * a.q_stride_b + (int64_t)r * a.q_stride_s + (int64_t)h * a.q_stride_h + c * 8);
#pragma unroll
    for (int e = 0; e < 8; ++e) q[e] = (float)x[e] * a.scale_log2e;
  }
  float m = -INFINITY, l = 0.f, acc[8] = {0, 0, 0, 0, 0, 0, 0, 0};
  for (int k0 = wave * PER * STEP; k0 < n; k0 += 4 * PER * STEP) {
    bf16x8 kx[STEP], vx[STEP];
#pragma unroll
    for (int u = 0; u < STEP; ++u) {
      const int key = k0 + u * PER + sub, kc = key < n ? key : n - 1;
      kx[u] = *reinterpret_cast<const bf16x8*>(kp + (int64_t)kc * a.kv_stride_s);
      vx[u] = *reinterpret_cast<const bf16x8*>(vp + (int64_t)kc * a.kv_stride_s);
    }
    float s[STEP], mx = m;
#pragma unroll
    for (int u = 0; u < STEP; ++u) {
      float d = 0.f;
#pragma unroll
      for (int e = 0; e < 8; ++e) d += q[e] * (float)kx[u][e];
#pragma unroll
      for (int w = 1; w < NC; w <<= 1) d += __shfl_xor(d, w, 64);
      s[u] = k0 + u * PER + sub < n ? d : -INFINITY;
      mx = fmaxf(mx, s[u]);
    }
    const float m_eff = mx == -INFINITY ? 0.f : mx, alpha = exp2_fast(m - m_eff);
    m = mx;
    l *= alpha;
#pragma unroll
    for (int e = 0; e < 8; ++e) acc[e] *= alpha;
#pragma unroll
    for (int u = 0; u < STEP; ++u) {
      const float p = exp2_fast(s[u] - m_eff);
      l += p;
#pragma unroll
      for (int e = 0; e < 8; ++e) acc[e] += p * (float)vx[u][e];
    }
  }
  // the lane groups of a wave, then the waves
#pragma unroll
  for (int w = NC; w < 64; w <<= 1) {
    const float mo = __shfl_xor(m, w, 64), mn = fmaxf(m, mo), me = mn == -INFINITY ? 0.f : mn;
    const float f = exp2_fast(m - me), fo = exp2_fast(mo - me);
    l = l * f + __shfl_xor(l, w, 64) * fo;
#pragma unroll
    for (int e = 0; e < 8; ++e) acc[e] = acc[e] * f + __shfl_xor(acc[e], w, 64) * fo;
    m = mn;
  }
  if (lane < NC) {
#pragma unroll
    for (int e = 0; e < 8; ++e) acc_s[wave][c * 8 + e] = acc[e];
    if (c == 0) { m_s[wave] = m; l_s[wave] = l; }
  }
  __syncthreads();
  if (tid < D) {
    const float mx = fmaxf(fmaxf(m_s[0], m_s[1]), fmaxf(m_s[2], m_s[3])), me = mx == -INFINITY ? 0.f : mx;
    float sum = 0.f, o = 0.f;
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      const float f = exp2_fast(m_s[w] - me);
      sum += l_s[w] * f;
      o += acc_s[w][tid] * f;
    }
    const bool none = sum == 0.f;                    // (a NaN is not that)
    const float r = none ? 0.f : o / sum;
    static_cast<float*>(a.part_out)[item * D + tid] = r;
    if (tid == 0) a.part_lse[item] = none ? -INFINITY : (mx + __builtin_log2f(sum)) * kLn2;
  }
}

hipError_t launch_block_fwd(const BlockArgs& a, int head_dim, hipStream_t st) {
  dim3 grid((unsigned)a.item_cap, (unsigned)(a.batch * a.n_kv_heads)), block(256);
  if (head_dim == 128) hipLaunchKernelGGL(block_fwd_kernel<128>, grid, block, block_fwd_lds_bytes<128>(), st, a);
  else hipLaunchKernelGGL(block_fwd_kernel<64>, grid, block, block_fwd_lds_bytes<64>(), st, a);
  return hipGetLastError();
}
hipError_t launch_block_fwd_few(const BlockArgs& a, int head_dim, hipStream_t st) {
  dim3 grid((unsigned)((int64_t)a.batch * a.n_q_heads * a.s_q * a.top_k)), block(256);
  if (head_dim == 128) hipLaunchKernelGGL(block_fwd_few_kernel<128>, grid, block, 0, st, a);
  else hipLaunchKernelGGL(block_fwd_few_kernel<64>, grid, block, 0, st, a);
  return hipGetLastError();
}
hipError_t opt_in_block_fwd_kernels() {
  const hipFuncAttribute attr = hipFuncAttributeMaxDynamicSharedMemorySize;
  hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(&block_fwd_kernel<128>), attr, (int)block_fwd_lds_bytes<128>());
  if (e == hipSuccess) e = hipFuncSetAttribute(reinterpret_cast<const void*>(&block_fwd_kernel<64>), attr, (int)block_fwd_lds_bytes<64>());
  return e;
}

}  // namespace slimpipe
