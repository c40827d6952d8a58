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

// Maximum of v over four waves (its lanes 32 .. 63 hold what 0 .. 31 do), through `tmp` in LDS, which is free again afterwards.
SP_DEV int rows_max(int v, int* tmp, int wave, int lane) {
#pragma unroll
  for (int w = 1; w < 32; w <<= 1) {
    const int o = __shfl_xor(v, w, 64);
    v = v > o ? v : o;
  }
  if (lane == 0) tmp[wave] = v;
  __syncthreads();
  int m = tmp[0];
#pragma unroll
  for (int w = 1; w < 4; ++w) m = m > tmp[w] ? m : tmp[w];
  __syncthreads();
  return __builtin_amdgcn_readfirstlane(m);
}

}  // namespace slimpipe
