// What the kernels on gathered rows share (device side).
#pragma once
#include "blocks.hpp"
#include "tile_common.hpp"

namespace slimpipe {

// The keys of a block that exist, and where the first of them lies.
struct BlockKeys {
  int64_t lo, hi;
  int64_t off;               // element offset of key `lo` of the plane in its chunk
  int chunk;
  SP_DEV BlockKeys(const BlockArgs& a, int block, int b, int hk) {
    const int64_t k0 = (int64_t)block * a.block_len, k1 = k0 + a.block_len;
    lo = k0 > a.kv_begin ? k0 : a.kv_begin;
    hi = k1 < a.kv_end ? k1 : a.kv_end;
    chunk = kv_chunk_of(a.kv, k0);
    off = (int64_t)b * a.kv_stride_b + (int64_t)hk * a.kv_stride_h + (lo - (int64_t)chunk * a.kv.len) * a.kv_stride_s;
  }
};

// This workgroup's tile of a plane and its lane's row of it.  What is read does not wait for each other: the number of tiles, the tile
// and its rows.
struct TileRows {
  BlockItem item;
  BlockEntry e;              // of the lane's row (lanes l and l + 32 have the same; rows past the tile's last: some row of the plane)
  int mine;                  // its place in the tile; item.count or more: none
  bool none;                 // no such tile
  SP_DEV TileRows(const BlockArgs& a, int plane, int wave, int lane) {
    const int tile = __builtin_amdgcn_readfirstlane(xcd_item(blockIdx.x, kXcdRun, plane));
    mine = wave * 32 + (lane & 31);
    const int n = a.n_items[plane];
    item = a.items[(int64_t)plane * a.item_cap + tile];
    e = a.entries[((int64_t)plane * a.item_cap + tile) * kBlockTileRows + mine];
    none = tile >= n;
    if (mine >= item.count) e = {0, 0, 0, 0};
  }
};
// A wave's 32 rows in C layout, times `factor`, to the partial results at `slot` (of the lane's row), through `part` (kOutRow<D> * 32 floats of
// LDS of the wave's own).  In 16 bits they are float16 numbers with a power of two of the row's own in front, which brings the largest
// finite one to 2^14 .. 2^15 (2^-97 and less are taken for that), and `factor` stays outside (part_scale).
template <int D>
SP_DEV void store_parts(const BlockArgs& a, float* part, const f32x16 (&acc)[D / 32], float factor, int64_t slot, int n_rows, int wave, int lane) {
  if (a.part_f32) {
    put_rows<D>(part, acc, factor, lane);
    constexpr int PER = D / 4, RPP = 64 / PER;
#pragma unroll
    for (int j = 0; j < 32 / RPP; ++j) {
      const int r = j * RPP + lane / PER;
      const int64_t to = __shfl(slot, r, 64);
      if (wave * 32 + r < n_rows)
        *reinterpret_cast<f32x4*>(static_cast<float*>(a.part_out) + to * D + lane % PER * 4) = *reinterpret_cast<const f32x4*>(part + r * kOutRow<D> + lane % PER * 4);
    }
    return;
  }
  auto largest = [&](auto&& of) {
    float mx = 0.f;
#pragma unroll
    for (int db = 0; db < D / 32; ++db)
#pragma unroll
      for (int i = 0; i < 16; ++i) mx = fmaxf(mx, of(fabsf(acc[db][i])));
    return xhalf_max(mx);
  };
  float mx = largest([](float x) { return x; });
  if (__builtin_amdgcn_ballot_w64(mx == INFINITY) != 0) mx = largest([](float x) { return x < INFINITY ? x : 0.f; });
  const uint32_t bits = __float_as_uint(mx) >> 23, e = bits < 30u ? 30u : bits;
  if (lane < 32 && wave * 32 + lane < n_rows) a.part_scale[slot] = factor * __uint_as_float((e - 14u) << 23);
  const float up = __uint_as_float((268u - e) << 23);
  constexpr int ROW = D + 4, PER = D / 8, RPP = 64 / PER;      // (rows of two banks more than all: 32 rows' 8 bytes meet no bank twice)
  _Float16* const h = reinterpret_cast<_Float16*>(part);
#pragma unroll
  for (int db = 0; db < D / 32; ++db)
#pragma unroll
    for (int i4 = 0; i4 < 4; ++i4) {
      const f32x4 v = {acc[db][4 * i4] * up, acc[db][4 * i4 + 1] * up, acc[db][4 * i4 + 2] * up, acc[db][4 * i4 + 3] * up};
      *reinterpret_cast<f16x4*>(h + (lane & 31) * ROW + 32 * db + 8 * i4 + 4 * (lane >> 5)) = __builtin_convertvector(v, f16x4);
    }
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
#pragma unroll
  for (int j = 0; j < 32 / RPP; ++j) {
    const int r = j * RPP + lane / PER, d = lane % PER * 8;
    const int64_t to = __shfl(slot, r, 64);
    const f16x4 lo = *reinterpret_cast<const f16x4*>(h + r * ROW + d), hi = *reinterpret_cast<const f16x4*>(h + r * ROW + d + 4);
    if (wave * 32 + r < n_rows) *reinterpret_cast<f16x8*>(static_cast<_Float16*>(a.part_out) + to * D + d) = __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
  }
}

// What the rows of a tile see of its block: the last key that the lane's row does, relative to the first (negative: none), and how many some row
// does: keys behind these are not read (they may hold anything, and a weight of 0 times a NaN is a NaN).  `tmp`: LDS for four numbers, free
// again afterwards.
struct TileSight {
  int see_rel, n_keys;
  SP_DEV TileSight(const BlockArgs& a, const BlockKeys& keys, uint32_t row, int* tmp, int wave, int lane) {
    see_rel = (int)(keys.hi - 1 - keys.lo);
    n_keys = see_rel + 1;
    if (!a.causal || a.q_offset >= keys.hi - 1) return;      // every row of the call sees the whole block
    const int64_t see = a.q_offset + row - keys.lo;
    see_rel = see < see_rel ? (int)see : see_rel;
    int v = see_rel;
#pragma unroll
    for (int w = 1; w < 32; w <<= 1) {                       // (lanes 32 .. 63 hold what 0 .. 31 do)
      const int o = __shfl_xor(v, w, 64);
      v = v > o ? v : o;
    }
    if (lane == 0) tmp[wave] = v;
    __syncthreads();
    int m = tmp[0];
#pragma unroll
    for (int w = 1; w < 4; ++w) m = m > tmp[w] ? m : tmp[w];
    __syncthreads();
    n_keys = __builtin_amdgcn_readfirstlane(m) + 1;
  }
};

}  // namespace slimpipe
