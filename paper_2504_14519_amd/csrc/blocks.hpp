// Argument blocks and launchers of the kernels of sparse attention over selected key blocks (internal to the library).
//
// A call has, per (batch index, kv head) "plane", R = group * s_q rows (query head within the group, row of the slice) with top_k
// slots each; a valid slot names a key block.  The large kernels are block-stationary: for every block the rows that chose it are
// gathered into a list (as tokens are for an expert), and a tile of such rows walks the block's keys.  Each (row, slot) gives a partial
// result that a last kernel folds per row in slot order, so that no sum depends on the order in which workgroups run.
#pragma once
#include "kernels.hpp"

namespace slimpipe {

constexpr int kMaxTopK = 64;
inline __host__ __device__ int count_stride(int n_list_chunks) { return (n_list_chunks + 3) & ~3; }      // of BlockArgs::counts: 16 bytes a lane
// rows of a plane that one workgroup of the list kernels handles, and blocks it handles at a time (a bit per row and block in LDS)
constexpr int kListRows = 256;
constexpr int kListBlocks = 1024;
constexpr int kBlockTileRows = 128;      // rows of a tile of the forward and dq kernels
// Tiles that follow each other on one XCD (xcd_item); the tables of items are whole rounds of eight runs.  (8192 rows of 8 heads on 128 blocks of
// 512 keys, 8 a row, forward: runs of 16 213 us, 1 221, 4 224, 64 220.)
constexpr int kXcdRun = 16;

// One row of a list: row of the slice, (head within the group << 6 | slot), and where its q and d_out lie behind those of the plane's first
// row, in units of 8 elements.  A block's list starts on a multiple of kBlockTileRows entries, so that tile t's are known without its item.
struct BlockEntry { uint32_t row, head_slot, q_off, do_off; };
// A tile of a list: block (absolute index), first entry within the plane's, entries; the dk/dv items also have the part of the
// block's keys (in units of its workgroup's keys) and the plane's partial-sum slot, or -1 when the sums go straight to the accumulators
struct BlockItem { int32_t block, first, count, part; };

// The list of a block: length, first tile; first dk/dv item of its parts of full length, and of its last part where that is shorter (these come
// behind all of full length, so that no long item starts late); how many partial dk/dv sums it leaves (0: one workgroup has all of it, or
// nobody) and the first of them
struct BlockList { uint32_t len, tile0, item0, rest0, parts, part0, unused[2]; };

struct BlockArgs {
  const __bf16* q;
  KvChunks kv;
  const int32_t* index;          // [batch, n_q_heads, s_q, top_k]
  int32_t batch, s_q, n_q_heads, n_kv_heads, group, causal, top_k;
  int32_t block_len;
  int32_t first_block, n_blocks; // blocks that hold a key of [kv_begin, kv_end): first_block .. first_block + n_blocks - 1
  int64_t q_offset, kv_begin, kv_end;      // kv_end: one past the last key that any row sees
  float scale, scale_log2e;
  int64_t q_stride_b, q_stride_s, q_stride_h;
  int64_t kv_stride_b, kv_stride_s, kv_stride_h;
  int64_t o_stride_b, o_stride_s, o_stride_h;
  int64_t do_stride_b, do_stride_s, do_stride_h;
  // lists (workspace), plane by plane
  int32_t n_list_chunks;         // ceil(group * s_q / kListRows)
  uint16_t* ranks;               // [plane][group * s_q * top_k]: place of a slot's row among the rows of its chunk that chose the block
  uint32_t* counts;              // [plane][n_blocks][count_stride]: rows of the chunk that chose the block, then where they start in its list
  BlockList* lists;              // [plane][n_blocks]
  BlockEntry* entries;           // [plane][item_cap * kBlockTileRows]
  BlockItem* items;              // [plane][item_cap]
  int32_t* n_items;              // [plane]
  int32_t item_cap;
  // partial results (workspace), rows in the order (batch index, query head, row of the slice)
  void* part_out;                // [row][top_k][head_dim], float32, or float16 to be multiplied by part_scale
  int32_t part_f32;
  float* part_scale;             // [row][top_k]
  float* part_lse;               // [row][top_k]; -inf: the slot has no result
  void* out;
  float* lse;                    // forward: written.  backward: the saved one
  int32_t out_f32;
  // backward
  const __bf16* d_out;
  float* delta;                  // negated, and lse in log2 units, as the dense backward's
  float* lse2;
  float* inf;                    // a cell that holds +infinity: the lse2 of rows past a list's end
  void* dq;
  int32_t dq_f32, dq_accumulate, dkv_accumulate;
  float* dk_acc[kMaxChunks];
  float* dv_acc[kMaxChunks];
  int32_t chunk_rows;            // rows of a list that one dk/dv workgroup sums (a multiple of 32)
  int32_t dkdv_keys;             // keys of a dk/dv workgroup: 256, 128 or 64
  int32_t n_sub;                 // parts of a block's keys that have a dk/dv workgroup each
  BlockItem* dkdv_items;         // [plane][dkdv_cap]
  int32_t* n_dkdv_items;         // [plane][2]: all of them, those of full length
  int32_t dkdv_cap;
  float* dkdv_part;              // [plane][part_cap][2][n_sub * dkdv_keys][head_dim]
  int32_t part_cap;
  int64_t kv_end_range;          // end of the call's key range (rows behind the last seen key get gradients of 0)
};

// Whether a slot of a row holds a block that the call computes: a block of the range that the row does not lie before,
// and not one that an earlier slot of the row has named already (not looked for without `repeats`).
inline __host__ __device__ bool block_slot_valid(const BlockArgs& a, const int32_t* row_index, int slot, int64_t pos, bool repeats = true) {
  const int32_t j = row_index[slot];
  if (j < a.first_block || j - a.first_block >= a.n_blocks) return false;
  if (a.causal && (int64_t)j * a.block_len > pos) return false;
  for (int i = 0; repeats && i < slot; ++i)
    if (row_index[i] == j) return false;
  return true;
}

struct BlockMeansArgs {
  KvChunks kv;
  float* means;                  // [batch, n_kv_heads, blocks_total, head_dim]
  int32_t batch, n_kv_heads, block_len, first_block, n_blocks;
  int64_t blocks_total, kv_end;
  int64_t kv_stride_b, kv_stride_s, kv_stride_h;
};
struct BlockSelectArgs {
  const __bf16* q;
  const float* means;
  int32_t* index;
  int32_t batch, s_q, n_q_heads, n_kv_heads, group, causal, top_k, block_len, first_block, n_blocks;
  int64_t blocks_total;
  int32_t own0, own_rest;        // causal: block of position q_offset (clamped to 2^30), and where in it that lies
  int64_t q_stride_b, q_stride_s, q_stride_h;
};

hipError_t launch_block_means(const BlockMeansArgs& a, int head_dim, hipStream_t st);
hipError_t launch_block_select(const BlockSelectArgs& a, int head_dim, int compute_units, hipStream_t st);
// lists and tiles of the call's index; for a backward (is_bwd) the dk/dv items too, and delta and lse2 of out, d_out and lse
hipError_t launch_block_lists(const BlockArgs& a, int head_dim, bool is_bwd, hipStream_t st);
hipError_t launch_block_fwd(const BlockArgs& a, int head_dim, hipStream_t st);
hipError_t launch_block_fwd_few(const BlockArgs& a, int head_dim, hipStream_t st);
hipError_t launch_block_bwd_dq(const BlockArgs& a, int head_dim, hipStream_t st);
hipError_t launch_block_bwd_dkdv(const BlockArgs& a, int head_dim, hipStream_t st);
hipError_t launch_block_reduce(const BlockArgs& a, int head_dim, hipStream_t st);      // dq, dk, dv from what the two above left
hipError_t opt_in_block_select_kernels();
hipError_t opt_in_block_fwd_kernels();
hipError_t opt_in_block_bwd_kernels();

}  // namespace slimpipe
