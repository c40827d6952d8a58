// Argument blocks and launchers of the kernels of a key/value cache held in 8 bits (internal to the library).
#pragma once
#include "kv4.hpp"

namespace slimpipe {

// A cache operand: codes (a byte an element, at the element strides), scales ([batch, blocks, heads] bytes, contiguous)
struct Kv8Operand { uint8_t* codes; uint8_t* scales; };

struct Kv8Cache {
  Kv8Operand k, v;
  int32_t n_kv_heads, shift;     // a block has 1 << shift rows
  int64_t stride_b, stride_s, stride_h, blocks;      // blocks of a sequence: ceil(capacity / block_len)
};

struct Kv8CopyArgs {
  Kv8Cache cache;
  const __bf16 *k_src, *v_src;   // store: [batch, rows, n_kv_heads, head_dim]
  __bf16 *k_dst, *v_dst;         // load: the same
  int64_t batch, rows, position; // rows of the slice, position of its first one in the cache
  int64_t x_stride_b, x_stride_s, x_stride_h;          // of the bf16 rows
};

struct Kv8Args {
  const __bf16* q;
  Kv8Cache cache;
  void* out;
  float* lse;
  int32_t batch, s_q, n_q_heads, group, causal, out_f32;
  int64_t q_offset, kv_begin, kv_end;      // kv_end: one past the last key that any row sees
  float scale_log2e;
  int64_t q_stride_b, q_stride_s, q_stride_h;
  int64_t o_stride_b, o_stride_s, o_stride_h;
  int32_t n_parts;               // key ranges of part_keys keys (the last one shorter), a workgroup each; 1: straight to out, lse
  int64_t part_keys;
  float* part_out;               // [batch, n_q_heads, s_q][n_parts][head_dim], as in PartMergeArgs
  float* part_lse;
};

struct Kv8WeightArgs {
  const __bf16* q;
  Kv8Cache cache;                // (of its values nothing is read)
  const float* lse;              // [batch, n_q_heads, s_q]
  const float* previous;         // [batch, n_kv_heads, capacity], or nullptr
  float* weights;                // the same
  float decay;
  int32_t batch, s_q, n_q_heads, group, causal;
  int64_t capacity, q_offset, kv_begin, kv_end;
  float scale_log2e;
  int64_t q_stride_b, q_stride_s, q_stride_h;
  int32_t n_parts;               // few rows: key ranges of part_keys keys; else: parts of a plane's rows, a workgroup each for every 256 keys
  int64_t part_keys;
  float* part;                   // [n_parts][batch, n_kv_heads][keys], slices with n_parts > 1
};

struct Kv8KeepArgs {
  const float* weights;          // [planes][capacity]
  int32_t* index;                // [planes][keep]
  int64_t capacity;
  int32_t planes, rows, keep, recent;
  int32_t chunks;                // 0: a workgroup a plane; else one for every `chunk` rows, which leave their counts in `work`
  int64_t chunk;
  uint32_t* work;                // [planes][chunks * kKeepChunkWords + kKeepPlaneWords]
};

constexpr int kKeepChunkWords = (2048 + 2048 + 1024) * 33 / 32 + 1, kKeepPlaneWords = 4;
// most rows of a plane for one workgroup (8 planes of 16384 rows 16.7 us, of 18000 17.5 in four launches), and rows that a workgroup of several takes at a time
constexpr int kKeepOneRows = 16 * 1024, kKeepSpan = 4 * 1024;

struct Kv8GatherArgs {
  Kv8Cache from, to;
  const int32_t* index;          // [batch, n_kv_heads, keep]
  const float* weights;          // [batch, n_kv_heads, capacity of from], or nullptr
  float* kept_weights;           // [batch, n_kv_heads, capacity of to]
  int64_t weights_stride, kept_weights_stride, from_rows;
  int32_t batch, keep;
};

hipError_t launch_kv8_store(const Kv8CopyArgs& a, int head_dim, hipStream_t st);
hipError_t launch_kv8_load(const Kv8CopyArgs& a, int head_dim, hipStream_t st);
enum class Kv8Kernel { few, four_waves, eight_waves };      // few: group * s_q <= kKv8FewRows; else 128 or 256 rows a workgroup
hipError_t launch_kv8_fwd(const Kv8Args& a, int head_dim, Kv8Kernel kernel, hipStream_t st);
constexpr int kKv8FewRows = 32;
// Rows of a plane from which a bf16 copy of the keys and slimpipe_attn_fwd are faster than tiles converted in the kernel (us with the copy and without: 8 heads on one and
// 32K keys, 512 rows 39 and 31, 1024 44 and 43, 2048 66 and 62, 4096 80 and 88, 32768 455 and 513; 40 heads on 17K keys, 512 rows 254 and 192, 1500 558 and 524,
// 2048 762 and 842; 12 heads of 64 on four, 1800 rows 67 and 65, 4011 87 and 92)
constexpr int kKv8CopyRows = 2048;
hipError_t launch_kv8_weights(const Kv8WeightArgs& a, int head_dim, bool few, hipStream_t st);
hipError_t launch_kv8_keep(const Kv8KeepArgs& a, hipStream_t st);
hipError_t launch_kv8_gather(const Kv8GatherArgs& a, int head_dim, hipStream_t st);
// kv heads of a workgroup of the kernels of few rows, a wave (or two, or all four) each
inline __host__ __device__ constexpr int kv8_heads_wg(int n_kv_heads) { return n_kv_heads % 4 == 0 ? 4 : n_kv_heads % 2 == 0 ? 2 : 1; }
constexpr int kv8_weight_keys() { return 256; }      // keys of a workgroup of the sums over a slice's rows
hipError_t opt_in_kv8_kernels();
hipError_t opt_in_kv8_evict_kernels();

}  // namespace slimpipe
