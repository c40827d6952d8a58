// Argument blocks and launchers of the kernels of a key/value cache held in 4 bits, and of the fold of many partial results (internal
// to the library).
#pragma once
#include "kernels.hpp"

namespace slimpipe {

// A cache operand: codes (two elements a byte) and scales (one byte for 32 elements), both at the same element strides
struct Kv4Operand { uint8_t* codes; uint8_t* scales; };

struct Kv4CopyArgs {
  Kv4Operand k, v;
  const __bf16 *k_src, *v_src;   // store: [batch, rows, n_kv_heads, head_dim]
  __bf16 *k_dst, *v_dst;         // load: the same
  int32_t n_kv_heads;
  int64_t batch, rows, position; // rows of the slice, position of its first one in the cache
  int64_t kv_stride_b, kv_stride_s, kv_stride_h;       // of the cache, in elements
  int64_t x_stride_b, x_stride_s, x_stride_h;          // of the bf16 rows
};

struct Kv4Args {
  const __bf16* q;
  Kv4Operand k, v;
  void* out;
  float* lse;
  int32_t batch, s_q, n_q_heads, n_kv_heads, group, causal, out_f32;
  int64_t q_offset, kv_begin, kv_end;      // kv_end: one past the last key that any row sees
  float scale_log2e;
  int64_t q_stride_b, q_stride_s, q_stride_h;
  int64_t kv_stride_b, kv_stride_s, kv_stride_h;
  int64_t o_stride_b, o_stride_s, o_stride_h;
  int32_t n_parts;               // key ranges of part_keys keys (the last one shorter), a workgroup each; 1: straight to out, lse
  int64_t part_keys;
  int32_t wave_heads, heads_wg;  // few rows: kv heads of a wave (1 or 2), sets of them of a workgroup (1, 2 or 4); their product divides n_kv_heads
  float* part_out;               // [batch, n_q_heads, s_q][n_parts][head_dim], as in PartMergeArgs
  float* part_lse;
};

// Folds the partial results of every row: lse = ln sum_i exp(lse_i), out = sum_i exp(lse_i - lse) out_i, in the order of the parts.
struct PartMergeArgs {
  const void* part_out;          // [row][parts][head_dim], rows in the order (batch index, query head, row of the slice); float32, or float16
  const float* part_scale;       // [row][parts]: what float16 ones are to be multiplied by
  const float* part_lse;         // [row][parts]; -inf: no result, its part_out is not read
  int32_t part_f32, parts, s_q, n_q_heads, out_f32;
  int64_t rows;
  void* out;
  float* lse;
  int64_t o_stride_b, o_stride_s, o_stride_h;
};

hipError_t launch_part_merge(const PartMergeArgs& a, int head_dim, hipStream_t st);
hipError_t launch_kv4_store(const Kv4CopyArgs& a, int head_dim, hipStream_t st);
hipError_t launch_kv4_load(const Kv4CopyArgs& a, int head_dim, hipStream_t st);
hipError_t launch_kv4_fwd(const Kv4Args& a, int head_dim, bool few, hipStream_t st);      // few: group * s_q <= kKv4FewRows
constexpr int kKv4FewRows = 32;      // (8 heads on 100000 keys, us with the kernel of few rows and the other: 2 tokens 17 and 31, 4 tokens 22 and 33)
hipError_t opt_in_kv4_kernels();

}  // namespace slimpipe
