// C ABI of sparse attention over selected key blocks: argument checks, workspace layout, launches.
#include <math.h>
#include <string.h>

#include "blocks.hpp"
#include "host_common.hpp"
#include "kv4.hpp"

using namespace slimpipe;

namespace {

constexpr int kMinBlockLen = 64, kMaxBlockLen = 1 << 16;

// What every block call checks beyond slimpipe_attn_validate: the block length, and that a block lies in one chunk.
int check_blocks(const slimpipe_attn_params* p, int32_t n_chunks, int64_t chunk_len, int32_t block_len) {
  if (block_len < kMinBlockLen || block_len > kMaxBlockLen || block_len % 64 != 0) return SLIMPIPE_EINVAL_SHAPE;
  if (p->kv_capacity > (int64_t)1 << 36) return SLIMPIPE_EINVAL_SHAPE;                         // block indices, in parts of 64 keys, are 32 bits
  // a launch has less than 2^32 threads: 1024 a block where the means are made
  if (p->kv_end / block_len - p->kv_begin / block_len >= (1 << 22) - 1) return SLIMPIPE_EINVAL_SHAPE;
  const int rc = check_chunks(p, n_chunks, chunk_len);
  if (rc != SLIMPIPE_OK) return rc;
  if (n_chunks > 1 && chunk_len % block_len != 0) return SLIMPIPE_EINVAL_SHAPE;
  if ((int64_t)p->batch * p->n_kv_heads > 65535) return SLIMPIPE_EINVAL_SHAPE;                 // planes are a grid dimension
  return SLIMPIPE_OK;
}
int check_top_k(const slimpipe_attn_params* p, int32_t top_k, int is_bwd) {
  if (top_k < 1 || top_k > kMaxTopK) return SLIMPIPE_EINVAL_SHAPE;
  const int64_t rows = (int64_t)p->n_q_heads / p->n_kv_heads * p->s_q;
  // slots of a plane, and offsets of its rows in units of 8 elements, in 32 bits; less than 2^32 threads, 32 a row and in the backward 32 a key, too
  if (rows * top_k > (int64_t)1 << 30 || rows * p->n_kv_heads * p->batch >= 1 << 27) return SLIMPIPE_EINVAL_SHAPE;
  if (is_bwd && rows + p->kv_end - p->kv_begin >= (1 << 27) - 64) return SLIMPIPE_EINVAL_SHAPE;
  const int64_t heads = p->n_q_heads / p->n_kv_heads - 1, last = p->s_q - 1, most = (int64_t)1 << 35;
  if (p->q_stride_h > most / (heads + 1) || p->q_stride_h * heads + p->q_stride_s * last >= most) return SLIMPIPE_EINVAL_STRIDE;
  if (is_bwd && (p->do_stride_h > most / (heads + 1) || p->do_stride_h * heads + p->do_stride_s * last >= most)) return SLIMPIPE_EINVAL_STRIDE;
  return SLIMPIPE_OK;
}
int set_chunks(KvChunks* kv, const slimpipe_attn_params* p, const void* const* k, const void* const* v, int32_t n_chunks, int64_t chunk_len) {
  memset(kv, 0, sizeof(*kv));
  for (int i = 0; i < n_chunks; ++i) {
    if (p->kv_end > 0 && (!k[i] || (v && !v[i]))) return SLIMPIPE_EINVAL_NULL;
    if (!aligned16(k[i]) || (v && !aligned16(v[i]))) return SLIMPIPE_EINVAL_ALIGN;
    kv->k[i] = static_cast<const __bf16*>(k[i]);
    if (v) kv->v[i] = static_cast<const __bf16*>(v[i]);
  }
  kv->len = chunk_len;
  kv->n = n_chunks;
  return SLIMPIPE_OK;
}

// Blocks that hold a key of [begin, end).
int64_t blocks_of(int64_t begin, int64_t end, int64_t block_len) { return end > begin ? (end + block_len - 1) / block_len - begin / block_len : 0; }

int64_t rows_of(const slimpipe_attn_params* p) { return (int64_t)p->batch * p->n_q_heads * p->s_q; }

// Rows so few that lists and 128-row tiles cost more than a workgroup for each (row, slot), which reads its block for itself: up to 8 of these a
// compute unit, and 2^25 elements of keys in all.  8 heads on one, us with a workgroup each and with lists: 16 slots of blocks of 64 at head_dim 128,
// 16 rows (2048 of them) 18 and 20; 8 slots of 128, 32 rows (2048, 2^25 elements) 20 and 21; 16 slots of 256, 16 rows (2048, 2^26) 27 and 21; 4 slots of 512, 32
// rows (1024, 2^26) 25 both.
bool few_rows(const slimpipe_attn_params* p, int32_t block_len, int32_t top_k) {
  const int64_t slots = rows_of(p) * top_k;
  return slots <= 8 * (int64_t)compute_units() && slots * block_len * p->head_dim <= 1 << 25;
}

// Items of a table, and workgroups of its launch: whole rounds of runs (xcd_item), one at least.
int32_t whole_rounds(size_t n) { return (int32_t)((n + 8 * kXcdRun - 1) / (8 * kXcdRun) * (8 * kXcdRun)) + (n == 0 ? 8 * kXcdRun : 0); }

size_t up(size_t n) { return (n + 255) & ~(size_t)255; }

// Where the parts of the workspace lie, and its size.  Partial results have room for float32 whatever the result's dtype: a workspace serves calls of either,
// and the query of a backward does not know dq's.
struct BlockWorkspace {
  size_t part_out, part_lse, part_scale, ranks, counts, lists, entries, items, n_items, delta, lse2, inf, dkdv_items, n_dkdv_items, dkdv_part, bytes;
  int32_t n_list_chunks, item_cap, chunk_rows, n_sub, dkdv_keys, dkdv_cap, part_cap;
};
// Keys of a dk/dv workgroup: 256 at head_dim 128 where the parts of a block are whole but for a quarter of the last, or there are many; else 128,
// or 64 in the smallest blocks.  Whole backwards, 8192 rows of 8 heads, 8 blocks a row, us with 256 and with 128 keys: blocks of 256 406 and
// 427, 384 560 and 526, 512 609 and 642, 1024 1065 and 1143; 4096 rows, 4 blocks a row: 192 146 and 152, 320 187 and 180, 448 197 and 204, 576 240 and
// 232, 704 247 and 254.  At head_dim 64 256 keys were never faster (blocks of 256 251 and 238, 1024 646 and 643) and have no kernel.
int32_t dkdv_keys(int32_t block_len, int32_t head_dim) {
  if (head_dim == 128 && (block_len % 256 == 0 || block_len % 256 > 128 || block_len >= 1024)) return 256;
  return block_len >= 128 ? 128 : 64;
}
// Rows of a list that one of them walks: few enough that there are three full parts for four compute units (256 keys, one workgroup a unit),
// two for each (128) or four (64), within what keeps a workgroup's start and its sums, which go to memory and back, a small part of it, and
// workspaces small (no more than a dozen a unit).  Whole backwards of 8 heads at head_dim 128, us: 8192 rows, 8 blocks of 512 a row (2048 by
// the rule): 1024 660, 1536 608, 2048 589, 2560 596; 1500 rows, 4 of 512 (512): 384 121, 512 109, 1024 123, 2048 164; 4096 rows, 4 of 256, 128 keys
// (512): 256 190, 512 163, 768 155, 1024 162, 2048 200; 500 rows, 4 of 64 at head_dim 64 (256): 256 56, 512 63, 1024 78.
int32_t dkdv_chunk_rows(int64_t slots, int32_t n_sub, int32_t keys) {
  const int64_t cus = compute_units(), work = slots * n_sub, least = keys == 256 ? 512 : 256, most = keys == 256 ? 2048 : 1536;
  int64_t rows = work / (keys == 256 ? 3 * cus / 4 : keys == 128 ? 2 * cus : 4 * cus);
  rows = rows < least ? least : rows > most ? most : rows;
  if (rows < work / (12 * cus)) rows = work / (12 * cus);
  return (int32_t)(rows > 1 << 20 ? 1 << 20 : (rows + 31) / 32 * 32);
}
BlockWorkspace layout(const slimpipe_attn_params* p, int32_t block_len, int32_t top_k, bool lists, bool is_bwd) {
  BlockWorkspace w;
  memset(&w, 0, sizeof(w));
  const size_t rows = (size_t)rows_of(p), planes = (size_t)p->batch * p->n_kv_heads, plane_rows = rows / planes;
  const size_t blocks = (size_t)blocks_of(p->kv_begin, p->kv_end, block_len);
  size_t at = 0;
  auto take = [&](size_t bytes) { const size_t o = at; at += up(bytes); return o; };
  w.part_out = take(rows * top_k * p->head_dim * 4);
  w.part_lse = take(rows * top_k * 4);
  w.part_scale = take(rows * top_k * 4);
  if (lists) {
    w.n_list_chunks = (int32_t)((plane_rows + kListRows - 1) / kListRows);
    // every tile but a block's last is full
    const size_t tiles = plane_rows * top_k / kBlockTileRows + blocks, slots = plane_rows * top_k;
    w.item_cap = whole_rounds(tiles < slots ? tiles : slots);
    w.ranks = take(planes * slots * 2);
    w.counts = take(planes * count_stride(w.n_list_chunks) * blocks * 4);
    w.lists = take(planes * blocks * sizeof(BlockList));
    w.entries = take(planes * w.item_cap * kBlockTileRows * sizeof(BlockEntry));
    w.items = take(planes * w.item_cap * sizeof(BlockItem));
    w.n_items = take(planes * 4);
  }
  if (is_bwd) {
    w.delta = take(rows * 4);
    w.lse2 = take(rows * 4);
    w.inf = take(4);
    const size_t slots = plane_rows * top_k;
    const int32_t keys = w.dkdv_keys = dkdv_keys(block_len, p->head_dim);
    w.n_sub = (block_len + keys - 1) / keys;
    w.chunk_rows = dkdv_chunk_rows((int64_t)(rows * top_k), w.n_sub, keys);
    // a list of n rows has at most n / chunk_rows + 1 parts, and partial sums only when n > chunk_rows: then at most twice n / chunk_rows
    w.dkdv_cap = whole_rounds((slots / w.chunk_rows + blocks) * w.n_sub);
    w.part_cap = (int32_t)(2 * slots / w.chunk_rows);
    w.dkdv_items = take(planes * w.dkdv_cap * sizeof(BlockItem));
    w.n_dkdv_items = take(planes * 8);
    w.dkdv_part = take(planes * w.part_cap * 2 * (size_t)(w.n_sub * keys) * p->head_dim * 4);
  }
  w.bytes = at;
  return w;
}

// The argument block of a call, without outputs.
void fill(BlockArgs* a, const slimpipe_attn_params* p, const void* q, const int32_t* index, int32_t block_len, int32_t top_k, const BlockWorkspace& w, char* ws) {
  a->q = static_cast<const __bf16*>(q);
  a->index = index;
  a->batch = p->batch; a->s_q = p->s_q; a->n_q_heads = p->n_q_heads; a->n_kv_heads = p->n_kv_heads;
  a->group = p->n_q_heads / p->n_kv_heads; a->causal = p->causal; a->top_k = top_k; a->block_len = block_len;
  a->q_offset = p->q_offset; a->kv_begin = p->kv_begin; a->kv_end = seen_end(p, p->kv_begin, p->kv_end); a->kv_end_range = p->kv_end;
  a->first_block = (int32_t)(p->kv_begin / block_len);
  a->n_blocks = (int32_t)blocks_of(a->kv_begin, a->kv_end, block_len);
  a->scale = p->scale; a->scale_log2e = p->scale * 1.4426950408889634f;
  a->q_stride_b = p->q_stride_b; a->q_stride_s = p->q_stride_s; a->q_stride_h = p->q_stride_h;
  a->kv_stride_b = p->kv_stride_b; a->kv_stride_s = p->kv_stride_s; a->kv_stride_h = p->kv_stride_h;
  a->o_stride_b = p->o_stride_b; a->o_stride_s = p->o_stride_s; a->o_stride_h = p->o_stride_h;
  a->do_stride_b = p->do_stride_b; a->do_stride_s = p->do_stride_s; a->do_stride_h = p->do_stride_h;
  a->part_out = ws + w.part_out;
  a->part_lse = reinterpret_cast<float*>(ws + w.part_lse);
  a->part_scale = reinterpret_cast<float*>(ws + w.part_scale);
  a->n_list_chunks = w.n_list_chunks;
  a->ranks = reinterpret_cast<uint16_t*>(ws + w.ranks);
  a->counts = reinterpret_cast<uint32_t*>(ws + w.counts);
  a->lists = reinterpret_cast<BlockList*>(ws + w.lists);
  a->entries = reinterpret_cast<BlockEntry*>(ws + w.entries);
  a->items = reinterpret_cast<BlockItem*>(ws + w.items);
  a->n_items = reinterpret_cast<int32_t*>(ws + w.n_items);
  a->item_cap = w.item_cap;
  a->delta = reinterpret_cast<float*>(ws + w.delta);
  a->lse2 = reinterpret_cast<float*>(ws + w.lse2);
  a->inf = reinterpret_cast<float*>(ws + w.inf);
  a->chunk_rows = w.chunk_rows; a->n_sub = w.n_sub; a->dkdv_keys = w.dkdv_keys; a->dkdv_cap = w.dkdv_cap; a->part_cap = w.part_cap;
  a->dkdv_items = reinterpret_cast<BlockItem*>(ws + w.dkdv_items);
  a->n_dkdv_items = reinterpret_cast<int32_t*>(ws + w.n_dkdv_items);
  a->dkdv_part = reinterpret_cast<float*>(ws + w.dkdv_part);
}

int status(hipError_t e) { return e == hipSuccess ? SLIMPIPE_OK : SLIMPIPE_ELAUNCH; }

}  // namespace

extern "C" {

int slimpipe_attn_block_means(const slimpipe_attn_params* p, const void* const* k_chunks, int32_t n_chunks, int64_t chunk_len, int32_t block_len,
                              float* means, void* hip_stream) {
  int rc = slimpipe_attn_validate(p, 0);
  if (rc != SLIMPIPE_OK) return rc;
  if (!k_chunks || !means) return SLIMPIPE_EINVAL_NULL;
  rc = check_blocks(p, n_chunks, chunk_len, block_len);
  if (rc != SLIMPIPE_OK) return rc;
  if (p->kv_begin % block_len != 0) return SLIMPIPE_EINVAL_RANGE;
  if (!aligned16(means)) return SLIMPIPE_EINVAL_ALIGN;
  BlockMeansArgs a;
  rc = set_chunks(&a.kv, p, k_chunks, nullptr, n_chunks, chunk_len);
  if (rc != SLIMPIPE_OK) return rc;
  a.means = means;
  a.batch = p->batch; a.n_kv_heads = p->n_kv_heads; a.block_len = block_len;
  a.first_block = (int32_t)(p->kv_begin / block_len);
  a.n_blocks = (int32_t)blocks_of(p->kv_begin, p->kv_end, block_len);
  a.blocks_total = blocks_of(0, p->kv_capacity, block_len);
  a.kv_end = p->kv_end;
  a.kv_stride_b = p->kv_stride_b; a.kv_stride_s = p->kv_stride_s; a.kv_stride_h = p->kv_stride_h;
  if (a.n_blocks == 0) return SLIMPIPE_OK;
  return status(launch_block_means(a, p->head_dim, static_cast<hipStream_t>(hip_stream)));
}

int slimpipe_attn_block_select(const slimpipe_attn_params* p, const void* q_slice, const float* means, int32_t block_len, int32_t top_k, int32_t* index,
                               void* hip_stream) {
  int rc = slimpipe_attn_validate(p, 0);
  if (rc != SLIMPIPE_OK) return rc;
  if (!q_slice || !means || !index) return SLIMPIPE_EINVAL_NULL;
  rc = check_blocks(p, 1, p->kv_capacity > 0 ? p->kv_capacity : 1, block_len);
  if (rc != SLIMPIPE_OK) return rc;
  rc = check_top_k(p, top_k, 0);
  if (rc != SLIMPIPE_OK) return rc;
  if (!aligned16(q_slice) || !aligned16(means) || !aligned4(index)) return SLIMPIPE_EINVAL_ALIGN;
  BlockSelectArgs a;
  a.q = static_cast<const __bf16*>(q_slice);
  a.means = means;
  a.index = index;
  a.batch = p->batch; a.s_q = p->s_q; a.n_q_heads = p->n_q_heads; a.n_kv_heads = p->n_kv_heads; a.group = p->n_q_heads / p->n_kv_heads;
  a.causal = p->causal; a.top_k = top_k; a.block_len = block_len;
  a.first_block = (int32_t)(p->kv_begin / block_len);
  a.n_blocks = (int32_t)blocks_of(p->kv_begin, p->kv_end, block_len);
  a.blocks_total = blocks_of(0, p->kv_capacity, block_len);
  const int64_t own0 = p->q_offset / block_len;
  a.own0 = (int32_t)(own0 < (int64_t)1 << 30 ? own0 : (int64_t)1 << 30);      // (behind every block of a cache, see check_blocks)
  a.own_rest = (int32_t)(p->q_offset % block_len);
  a.q_stride_b = p->q_stride_b; a.q_stride_s = p->q_stride_s; a.q_stride_h = p->q_stride_h;
  if (ensure_device_ready() != SLIMPIPE_OK) return SLIMPIPE_ELAUNCH;
  return status(launch_block_select(a, p->head_dim, compute_units(), static_cast<hipStream_t>(hip_stream)));
}

int slimpipe_attn_block_workspace_bytes(const slimpipe_attn_params* p, int32_t block_len, int32_t top_k, int is_bwd, size_t* bytes) {
  if (!bytes) return SLIMPIPE_EINVAL_NULL;
  int rc = slimpipe_attn_validate(p, is_bwd);
  if (rc != SLIMPIPE_OK) return rc;
  rc = check_blocks(p, 1, p->kv_capacity > 0 ? p->kv_capacity : 1, block_len);
  if (rc == SLIMPIPE_OK) rc = check_top_k(p, top_k, is_bwd);
  if (rc != SLIMPIPE_OK) return rc;
  *bytes = layout(p, block_len, top_k, is_bwd || !few_rows(p, block_len, top_k), is_bwd != 0).bytes;
  return SLIMPIPE_OK;
}

int slimpipe_attn_block_fwd(const slimpipe_attn_params* p, const void* q_slice, const void* const* k_chunks, const void* const* v_chunks, int32_t n_chunks,
                            int64_t chunk_len, int32_t block_len, int32_t top_k, const int32_t* index, void* out, float* lse, void* workspace,
                            size_t workspace_bytes, void* hip_stream) {
  int rc = slimpipe_attn_validate(p, 0);
  if (rc != SLIMPIPE_OK) return rc;
  if (!q_slice || !k_chunks || !v_chunks || !index || !out || !lse) return SLIMPIPE_EINVAL_NULL;
  rc = check_blocks(p, n_chunks, chunk_len, block_len);
  if (rc == SLIMPIPE_OK) rc = check_top_k(p, top_k, 0);
  if (rc != SLIMPIPE_OK) return rc;
  if (!aligned16(q_slice) || !aligned16(out) || !aligned4(lse) || !aligned4(index)) return SLIMPIPE_EINVAL_ALIGN;
  const bool few = few_rows(p, block_len, top_k);
  const BlockWorkspace w = layout(p, block_len, top_k, !few, false);
  if (!workspace || workspace_bytes < w.bytes) return SLIMPIPE_EWORKSPACE;
  if (!aligned16(workspace)) return SLIMPIPE_EINVAL_ALIGN;
  BlockArgs a;
  memset(&a, 0, sizeof(a));
  rc = set_chunks(&a.kv, p, k_chunks, v_chunks, n_chunks, chunk_len);
  if (rc != SLIMPIPE_OK) return rc;
  fill(&a, p, q_slice, index, block_len, top_k, w, static_cast<char*>(workspace));
  a.out = out;
  a.lse = lse;
  a.out_f32 = p->out_dtype == SLIMPIPE_F32;
  a.part_f32 = a.out_f32 || few;
  if (ensure_device_ready() != SLIMPIPE_OK) return SLIMPIPE_ELAUNCH;
  hipStream_t st = static_cast<hipStream_t>(hip_stream);
  if (few) {
    if (launch_block_fwd_few(a, p->head_dim, st) != hipSuccess) return SLIMPIPE_ELAUNCH;
  } else if (launch_block_lists(a, p->head_dim, false, st) != hipSuccess || launch_block_fwd(a, p->head_dim, st) != hipSuccess) {
    return SLIMPIPE_ELAUNCH;
  }
  PartMergeArgs m;
  m.part_out = a.part_out; m.part_f32 = a.part_f32; m.part_scale = a.part_scale; m.part_lse = a.part_lse; m.parts = top_k; m.s_q = p->s_q; m.n_q_heads = p->n_q_heads; m.out_f32 = a.out_f32;
  m.rows = rows_of(p);
  m.out = out; m.lse = lse;
  m.o_stride_b = p->o_stride_b; m.o_stride_s = p->o_stride_s; m.o_stride_h = p->o_stride_h;
  return status(launch_part_merge(m, p->head_dim, st));
}

int slimpipe_attn_block_bwd(const slimpipe_attn_params* p, const void* q_slice, const void* const* k_chunks, const void* const* v_chunks, int32_t n_chunks,
                            int64_t chunk_len, int32_t block_len, int32_t top_k, const int32_t* index, const void* out, const void* d_out, const float* lse,
                            void* dq, int32_t dq_dtype, int32_t dq_accumulate, float* const* dk_chunks, float* const* dv_chunks, int32_t dkv_accumulate,
                            void* workspace, size_t workspace_bytes, void* hip_stream) {
  int rc = slimpipe_attn_validate(p, 1);
  if (rc != SLIMPIPE_OK) return rc;
  if (!q_slice || !k_chunks || !v_chunks || !index || !out || !d_out || !lse || !dq || !dk_chunks || !dv_chunks) return SLIMPIPE_EINVAL_NULL;
  rc = check_blocks(p, n_chunks, chunk_len, block_len);
  if (rc == SLIMPIPE_OK) rc = check_top_k(p, top_k, 1);
  if (rc != SLIMPIPE_OK) return rc;
  if (dq_dtype != SLIMPIPE_BF16 && dq_dtype != SLIMPIPE_F32) return SLIMPIPE_EINVAL_SHAPE;
  if (dq_accumulate && dq_dtype != SLIMPIPE_F32) return SLIMPIPE_EINVAL_SHAPE;
  if (!aligned16(q_slice) || !aligned16(out) || !aligned16(d_out) || !aligned16(dq) || !aligned4(lse) || !aligned4(index)) return SLIMPIPE_EINVAL_ALIGN;
  const BlockWorkspace w = layout(p, block_len, top_k, true, true);
  if (!workspace || workspace_bytes < w.bytes) return SLIMPIPE_EWORKSPACE;
  if (!aligned16(workspace)) return SLIMPIPE_EINVAL_ALIGN;
  BlockArgs a;
  memset(&a, 0, sizeof(a));
  rc = set_chunks(&a.kv, p, k_chunks, v_chunks, n_chunks, chunk_len);
  if (rc != SLIMPIPE_OK) return rc;
  for (int i = 0; i < n_chunks; ++i) {
    if (!dk_chunks[i] || !dv_chunks[i]) return SLIMPIPE_EINVAL_NULL;
    if (!aligned16(dk_chunks[i]) || !aligned16(dv_chunks[i])) return SLIMPIPE_EINVAL_ALIGN;
    a.dk_acc[i] = dk_chunks[i];
    a.dv_acc[i] = dv_chunks[i];
  }
  fill(&a, p, q_slice, index, block_len, top_k, w, static_cast<char*>(workspace));
  a.out = const_cast<void*>(out);
  a.lse = const_cast<float*>(lse);
  a.d_out = static_cast<const __bf16*>(d_out);
  a.dq = dq;
  a.dq_f32 = a.part_f32 = dq_dtype == SLIMPIPE_F32; a.dq_accumulate = dq_accumulate ? 1 : 0; a.dkv_accumulate = dkv_accumulate ? 1 : 0;
  if (ensure_device_ready() != SLIMPIPE_OK) return SLIMPIPE_ELAUNCH;
  hipStream_t st = static_cast<hipStream_t>(hip_stream);
  hipError_t e = launch_block_lists(a, p->head_dim, true, st);
  if (e == hipSuccess) e = launch_block_bwd_dkdv(a, p->head_dim, st);
  if (e == hipSuccess) e = launch_block_bwd_dq(a, p->head_dim, st);
  if (e == hipSuccess) e = launch_block_reduce(a, p->head_dim, st);
  return status(e);
}

}  // extern "C"
