/*
 * slimpipe_attn.h - C ABI of the slice-wise causal attention hot path for AMD MI355X (gfx950).
 *
 * The operation is the attention step of SlimPipe's slice-wise pipeline schedule
 * (paper Sec. 4.1.2): the queries of slice i of a sequence attend causally to the cached
 * keys/values of slices 0..i, forward and backward, the backward passes of the slices running
 * in reverse order.  Any call may be restricted to a key range [kv_begin, kv_end); it then
 * returns the partial output together with the softmax normaliser of that range, which is what
 * the paper's attention context exchange (Sec. 4.2.2) and commutated context parallelism
 * (Sec. 5) ship between devices and fold together with the online-softmax merge rule.
 *
 * Conventions
 *   - All data pointers are DEVICE pointers owned by the caller.  The library allocates nothing on
 *     the device, enqueues its kernels on the caller's HIP stream (a hipStream_t passed as void*,
 *     NULL = default stream) and returns without synchronising.
 *   - State.  Per device the library remembers two facts that depend on the device alone: that its
 *     kernels have been allowed their dynamic LDS (done once, see slimpipe_attn_init) and the number of
 *     compute units.  Both are set under a once-flag / atomically, so the entry points may be called from
 *     several host threads at once (each with its own stream and buffers).  Nothing else persists
 *     between calls; the measurement aids of slimpipe_attn_bench.h keep their own records.
 *   - q, out, d_out, dq:  [batch, s_q, n_q_heads, head_dim], element strides given, head_dim contiguous.
 *   - k, v, dk_acc, dv_acc: [batch, kv_capacity, n_kv_heads, head_dim]; row j of the prefix IS global
 *     key position j (the base pointer is position 0).
 *   - lse: [batch, n_q_heads, s_q] float32, contiguous; lse = ln sum_j exp(scale * q.k_j) over the
 *     visible keys of the call (natural log, scale inside).
 *   - Key j is visible to query row r iff kv_begin <= j < kv_end and (causal == 0 or
 *     j <= q_offset + r).  A row that sees no key gets out = 0, lse = -inf and contributes no
 *     gradient.  A key that no row sees may hold anything, NaN and infinities too; its dk, dv are 0.  (What
 *     is not finite in a key that some row sees may turn results of other rows of the call into NaN; rows
 *     that see no key are kept from it by the sparse, 4-bit and 8-bit calls, not by the dense ones.)  An
 *     empty range is legal.
 *   - Query head h reads KV head h / (n_q_heads / n_kv_heads).
 *   - q, k, v, d_out are bf16.  All strides are in elements, must be multiples of 8 and the base
 *     pointers 16-byte aligned.
 *   - Every function returns SLIMPIPE_OK (0) or a negative slimpipe_status; nothing is printed,
 *     nothing aborts.  Argument validation is pure host code.
 */
#ifndef SLIMPIPE_ATTN_H
#define SLIMPIPE_ATTN_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum slimpipe_status {
  SLIMPIPE_OK = 0,
  SLIMPIPE_EINVAL_NULL = -1,      /* a required pointer is NULL                                   */
  SLIMPIPE_EINVAL_SHAPE = -2,     /* batch/s_q/heads <= 0, Hq % Hkv != 0, head_dim not 64 or 128,  */
                                  /* scale not finite or <= 0, bad dtype code, n_parts out of range,*/
                                  /* batch or n_q_heads > 65535, more than 2^30 work items a launch */
                                  /* (ceil(s_q / 256) * n_q_heads * batch * key ranges)             */
  SLIMPIPE_EINVAL_RANGE = -3,     /* kv_begin > kv_end, kv_end > kv_capacity, negative offsets     */
  SLIMPIPE_EINVAL_STRIDE = -4,    /* a stride is not a positive multiple of 8 elements             */
  SLIMPIPE_EINVAL_ALIGN = -5,     /* a pointer is not 16-byte aligned                              */
  SLIMPIPE_EWORKSPACE = -6,       /* workspace missing or smaller than slimpipe_attn_workspace_bytes */
  SLIMPIPE_ELAUNCH = -7,          /* the HIP runtime refused a launch                              */
  SLIMPIPE_ETOOLARGE = -8         /* slimpipe_attn_bwd_noalloc: the call needs more than its fixed scratch */
} slimpipe_status;

enum { SLIMPIPE_BF16 = 0, SLIMPIPE_F32 = 1 };

typedef struct slimpipe_attn_params {
  int32_t batch;
  int32_t s_q;          /* rows of the query slice                                        */
  int32_t n_q_heads;
  int32_t n_kv_heads;
  int32_t head_dim;     /* 64 or 128                                                      */
  int32_t causal;       /* 0 or 1                                                         */
  int64_t kv_capacity;  /* rows addressable behind k/v (and dk_acc/dv_acc)                */
  int64_t q_offset;     /* global position of query row 0                                 */
  int64_t kv_begin;     /* half-open range of global key positions this call attends to   */
  int64_t kv_end;
  float   scale;        /* softmax scale, > 0 (1/sqrt(head_dim) in every workload)        */
  int32_t out_dtype;    /* forward: dtype of `out` (SLIMPIPE_BF16, or SLIMPIPE_F32 for    */
                        /* partials that will be merged).  Ignored by backward.           */
  int64_t q_stride_b, q_stride_s, q_stride_h;     /* q and dq                              */
  int64_t kv_stride_b, kv_stride_s, kv_stride_h;  /* k, v, dk_acc, dv_acc                  */
  int64_t o_stride_b, o_stride_s, o_stride_h;     /* out                                   */
  int64_t do_stride_b, do_stride_s, do_stride_h;  /* d_out (backward only)                 */
} slimpipe_attn_params;

/* Prepares the CURRENT device (hipSetDevice) for launches: allows every kernel of the library the dynamic LDS
 * it uses (more than the 64 KB a kernel gets by default).  Thread-safe, idempotent, a few microseconds after
 * the first call.  Every launching entry point does the same on its first call on a device, so calling this is
 * optional - except before HIP graph capture: the attribute call is not a stream operation and must have happened
 * before a capture begins, so call slimpipe_attn_init() once per device first; after it a capture needs no
 * eager warm-up launch.  Returns SLIMPIPE_OK or SLIMPIPE_ELAUNCH. */
int slimpipe_attn_init(void);

/* Host-only argument check shared by every entry point (is_bwd != 0 also checks what only the
 * backward needs).  No device access. */
int slimpipe_attn_validate(const slimpipe_attn_params* p, int is_bwd);

/* Bytes of device workspace the call would like.  Forward: 256 bytes for the counters through which the workgroups take
 * their work items (see the backward below), plus, when the call is a short slice over a long cache whose query
 * blocks leave compute units idle, room for the float32 partial (out, lse) of the 2 to 16
 * key ranges of equal work the call is cut into (see slimpipe_attn_fwd).  Backward needs two floats per
 * (batch, q head, row): delta = rowsum(d_out * out) (kept negated) and lse in log2 units, each array rounded up to
 * 256 bytes; slimpipe_attn_bwd refuses less.  On top of that it can use, in this order: 256 bytes for the counters
 * through which the workgroups of the dq and dk/dv kernels take their work items (the hardware hands workgroups to the
 * chip's eight XCDs in turn whatever their speed; with counters a faster XCD takes more items; the results do
 * not depend on who computes what), and room for partial dk/dv sums: when the key tiles of a call do not fill the
 * GPU's compute units evenly, or when the counters are there and more items make for a more even finish, the query
 * rows of each key tile are cut into 2 to 8 chunks that run as work items of their own, each writing float32
 * partial sums [chunk][dk, dv][batch][kv head][keys rounded up to 256][head_dim] that a second kernel adds up
 * in chunk order.  The figure returned here includes that room for the split this call would pick;
 * given less, slimpipe_attn_bwd uses cuts whose sums fit (down to none).  In the same way the dq
 * kernel of a short slice over a long cache is cut into 2 to 16 key ranges of equal work, as the forward is,
 * with float32 partial dq [range][batch, s_q, n_q_heads, head_dim] behind the partial dk/dv that a reduce kernel
 * adds up in range order; that room is included too and used as far as it is there.  A backward call with fewer than
 * two work items per compute unit computes dq and dk/dv in one launch (and adds up their partial sums in one), but for calls
 * of long items that a workspace without room for partial sums leaves undivided.  The smallest of these, given the room
 * returned here, go through workgroups of 32 rows, or of 32 or 64 keys, that keep their partial sums to themselves and leave the room unused. */
int slimpipe_attn_workspace_bytes(const slimpipe_attn_params* p, int is_bwd, size_t* bytes);

/* Forward of one query slice against keys [kv_begin, kv_end) of the cached prefix
 * (Sec. 4.1.2; partial ranges: Sec. 4.2.2).  Writes out (dtype p->out_dtype, strides o_*) and
 * lse [batch, n_q_heads, s_q].  Scores are never stored.
 *   workspace : may be NULL (16-byte aligned otherwise).  Its first 256 bytes, when it has them, hold the counters
 *               through which the workgroups take their work items (set to zero by a one-workgroup kernel ahead of
 *               the forward kernel; the results do not depend on them).  Given slimpipe_attn_workspace_bytes(p, 0)
 *               bytes, a call whose query blocks would not fill the GPU cuts [kv_begin, kv_end) into ranges of
 *               equal work (cut points on multiples of 256 keys), computes them in one launch into float32
 *               partials behind the counters and merges them (the rule of slimpipe_attn_merge) into (out, lse)
 *               in the same call; given less room it uses as many ranges as fit, down to the undivided
 *               computation.  A call of few query blocks that is given what slimpipe_attn_workspace_bytes(p, 0)
 *               asks for may be computed by workgroups of 32 rows whose waves share out the keys (another order of
 *               the float32 sums, and probabilities rounded to bf16 relative to each wave's own maximum); with less it is cut as above, and where not even two ranges fit, or
 *               with NULL, it returns what slimpipe_attn_fwd_ranges returns for its range, bit for bit. */
int slimpipe_attn_fwd(const slimpipe_attn_params* p,
                      const void* q_slice, const void* k_prefix, const void* v_prefix,
                      void* out, float* lse,
                      void* workspace, size_t workspace_bytes, void* hip_stream);

/* Backward of the same call (Sec. 4.1.2: backward per slice in reverse order, K/V kept for it).
 *   out, lse : the rows' FINAL values (for a split computation: the merged ones), out is bf16.
 *   dq       : dq_dtype SLIMPIPE_BF16 (overwritten) or SLIMPIPE_F32 (overwritten, or += when
 *              dq_accumulate != 0, which is how the partial dq of several ranges are summed).
 *              Uses the q strides.
 *   dk_acc, dv_acc : float32 with the kv strides; rows [kv_begin, kv_end) are overwritten
 *              (dkv_accumulate == 0) or incremented (!= 0); other rows are untouched.  Each row is
 *              owned by one workgroup (or a fixed number of them whose partial sums are added in a
 *              fixed order) that sums queries and the heads of a GQA group in a fixed order, so
 *              results are bit-reproducible from run to run for the same workspace size.
 *   shared memory : out and lse are read before any gradient is written, so dq, dk_acc and dv_acc may lie over them (a bf16 dq
 *              in place of out, for one).  No gradient may share memory with q, k, v, d_out, the workspace or another gradient.
 * Enqueues the delta pre-pass, then the dq kernel and the dk/dv kernel, each with a reduce kernel when it was cut, or
 * for small calls one kernel for both and one reduce kernel when either was cut (slimpipe_attn_workspace_bytes).  The smallest calls
 * of head_dim 64 whose gradients do not lie over out or lse enqueue no delta pre-pass: their one kernel does its work. */
int slimpipe_attn_bwd(const slimpipe_attn_params* p,
                      const void* q_slice, const void* k_prefix, const void* v_prefix,
                      const void* out, const void* d_out, const float* lse,
                      void* dq, int32_t dq_dtype, int32_t dq_accumulate,
                      float* dk_acc, float* dv_acc, int32_t dkv_accumulate,
                      void* workspace, size_t workspace_bytes, void* hip_stream);

/* slimpipe_attn_bwd for callers that cannot allocate device memory or hand over a workspace: code under HIP graph
 * capture, tight serving loops, harnesses that forbid hipMalloc.  Same arguments and kernels as slimpipe_attn_bwd,
 * and bit for bit the results it gives with a workspace of the minimum size (the dk/dv query stream is not split,
 * dq is not cut into key ranges), but what the kernels exchange - the two row-statistic arrays (delta and lse in
 * log2 units, one float each per (batch, q head, row)) and the 256 bytes of counters through which workgroups take their
 * work items - lives in a fixed array of 4 MiB + 256 bytes in device memory that belongs to the library, one copy per
 * GPU, held until the process ends.  The call allocates nothing (no hipMalloc / hipFree, no events) and does not
 * synchronise.
 *   limit : batch * n_q_heads * s_q <= slimpipe_attn_noalloc_max_rows() = 524288, each array rounded up to 256
 *           bytes; beyond that SLIMPIPE_ETOOLARGE is returned and nothing is launched.
 *   The array keeps the last call's contents; every call overwrites the entries it reads and sets the counters to
 *   zero itself (nothing has to start at zero).  All calls on one GPU share it: two calls whose kernels may overlap
 *   on one GPU (different streams, or host threads) race - serialise them, or use slimpipe_attn_bwd with a
 *   workspace each.  Graph capture: call slimpipe_attn_init() before the capture begins. */
int slimpipe_attn_bwd_noalloc(const slimpipe_attn_params* p,
                              const void* q_slice, const void* k_prefix, const void* v_prefix,
                              const void* out, const void* d_out, const float* lse,
                              void* dq, int32_t dq_dtype, int32_t dq_accumulate,
                              float* dk_acc, float* dv_acc, int32_t dkv_accumulate, void* hip_stream);
int slimpipe_attn_noalloc_max_rows(void);

/* Online-softmax merge of n_parts (1..16) partial results over disjoint key sets (Sec. 4.2.2):
 *   lse = ln sum_r exp(lse_r),  out = sum_r exp(lse_r - lse) * out_r   (weight 0 when lse_r = -inf).
 * outs / lses are HOST arrays of n_parts DEVICE pointers.  Every partial out is contiguous
 * [rows, n_q_heads, head_dim] of part_dtype, every partial lse [batch, n_q_heads, s_q] with
 * rows = batch * s_q; the merged out has dtype out_dtype and the same contiguous layout. */
int slimpipe_attn_merge(int32_t n_parts, const void* const* outs, const float* const* lses,
                        int32_t part_dtype, int32_t batch, int32_t s_q, int32_t n_q_heads,
                        int32_t head_dim, void* out, int32_t out_dtype, float* lse,
                        void* hip_stream);

/* Round float32 accumulators (dk_acc/dv_acc after the last slice's backward) to bf16, RNE.
 * Contiguous, n_elems elements.  The paper trains in bf16 and says nothing of the precision in which the
 * key/value gradients of the slices of a sequence are added up (Sec. 4.1.2 only fixes that the backward passes
 * run slice by slice); the reading taken here: float32 accumulators across the calls, in call order, and ONE
 * rounding to bf16 at the end, which is this call. */
int slimpipe_attn_finalize_bf16(const float* acc, void* dst_bf16, int64_t n_elems, void* hip_stream);

/* The same two calls with the cached keys / values given the way the paper stores them (Sec. 5): a list
 * of slice-sized chunks instead of one buffer, so that the cache grows in the forward passes and shrinks
 * in the backward passes without copies.
 *   k_chunks, v_chunks (and dk_chunks, dv_chunks) : HOST arrays of n_chunks device pointers; row j of the
 *              prefix is row j % chunk_len of chunk j / chunk_len, laid out inside the chunk with the kv
 *              strides of `p` (kv_stride_s between rows).  The arrays are read during the call only.
 *   n_chunks : 1 .. 64;  n_chunks * chunk_len >= p->kv_capacity;  with more than one chunk, chunk_len is a
 *              multiple of 256 (SLIMPIPE_EINVAL_SHAPE otherwise).  Chunks of slices the range does not
 *              touch are never dereferenced but must be non-NULL.
 * Everything else (ranges, masks, outputs, workspace, accumulation, error codes) is as in the calls above;
 * with one chunk the result is bit-identical to them. */
int slimpipe_attn_fwd_chunked(const slimpipe_attn_params* p, const void* q_slice,
                              const void* const* k_chunks, const void* const* v_chunks,
                              int32_t n_chunks, int64_t chunk_len, void* out, float* lse,
                              void* workspace, size_t workspace_bytes, void* hip_stream);
int slimpipe_attn_bwd_chunked(const slimpipe_attn_params* p, const void* q_slice,
                              const void* const* k_chunks, const void* const* v_chunks,
                              int32_t n_chunks, int64_t chunk_len,
                              const void* out, const void* d_out, const float* lse,
                              void* dq, int32_t dq_dtype, int32_t dq_accumulate,
                              float* const* dk_chunks, float* const* dv_chunks, int32_t dkv_accumulate,
                              void* workspace, size_t workspace_bytes, void* hip_stream);

/* Forward of one query slice over SEVERAL key ranges in one launch (Sec. 4.2.2: the pieces a context exchange
 * cuts a slice's keys into; also how a short slice over a long cache fills the GPU).  Keys / values as a chunk
 * list as above (n_chunks = 1: one buffer).
 *   n_ranges         : 1 .. 16;  kv_begin[r] <= kv_end[r] <= p->kv_capacity (HOST arrays; p->kv_begin / kv_end
 *                      are not used).  Ranges may be empty, overlap or leave gaps: each is computed on its own.
 *   part_out, part_lse : device, float32, [n_ranges][batch, s_q, n_q_heads, head_dim] and
 *                      [n_ranges][batch, n_q_heads, s_q], contiguous: what slimpipe_attn_fwd would return for
 *                      each range with out_dtype SLIMPIPE_F32.
 *   out, lse         : both NULL (parts only), or the merged result of all ranges (out: p->out_dtype, strides
 *                      o_*), written by the merge kernel in the same call. */
int slimpipe_attn_fwd_ranges(const slimpipe_attn_params* p, const void* q_slice,
                             const void* const* k_chunks, const void* const* v_chunks,
                             int32_t n_chunks, int64_t chunk_len,
                             int32_t n_ranges, const int64_t* kv_begin, const int64_t* kv_end,
                             float* part_out, float* part_lse, void* out, float* lse, void* hip_stream);

/* Sparse attention over key blocks that a cheap score selects for each query row.
 * Keys come in blocks: block j holds positions [j * block_len, (j + 1) * block_len).  The three calls below make the blocks' means,
 * pick the blocks of every query row and head, and attend to the keys of these blocks; slimpipe_attn_block_bwd is the gradient of the
 * last with the picks held fixed (they are a choice and have none).  They pay where a row's blocks are a small share of the keys it sees: beyond
 * a quarter of them (blocks of 64 at head_dim 64) to a half (512 at 128) slimpipe_attn_fwd and slimpipe_attn_bwd are as fast.
 * As with every call here the key range [kv_begin, kv_end) may be a part of the prefix, so that the (out, lse) of several ranges can be folded by slimpipe_attn_merge.
 *   block_len : a multiple of 64, 64 .. 65536 (SLIMPIPE_EINVAL_SHAPE otherwise); with several chunks chunk_len is a multiple of it.
 *   top_k     : 1 .. 64 slots per row (SLIMPIPE_EINVAL_SHAPE otherwise).
 *   limits    : batch * n_kv_heads <= 65535, less than 2^27 rows of all heads, 2^30 slots of one kv head, less than 2^22 - 1 blocks in the key range, in the
 *               backward less than 2^27 - 64 keys there and rows of one kv head together, kv_capacity <= 2^36 (SLIMPIPE_EINVAL_SHAPE otherwise); the rows of the query heads of
 *               one kv head, of q and in the backward of d_out, lie within 2^35 elements (SLIMPIPE_EINVAL_STRIDE otherwise).
 *   index     : int32 [batch, n_q_heads, s_q, top_k], contiguous.
 *   means     : float32 [batch, n_kv_heads, ceil(kv_capacity / block_len), head_dim], contiguous. */

/* Means of the blocks that hold a key of [kv_begin, kv_end): mean j = the average of the keys of block j before kv_end (summed in 64
 * bits, rounded once).  kv_begin is a multiple of block_len (SLIMPIPE_EINVAL_RANGE otherwise); other blocks' means are untouched, so a
 * cache that grows by slices has every slice's first and new blocks made as it comes.  Of p the query side (s_q, n_q_heads, strides,
 * q_offset) is only validated; v is not needed. */
int slimpipe_attn_block_means(const slimpipe_attn_params* p, const void* const* k_chunks, int32_t n_chunks, int64_t chunk_len, int32_t block_len,
                              float* means, void* hip_stream);

/* The blocks of every query row and head, as ascending indices, filled up with -1.  Blocks of the range compete by q . mean (in 64 bits,
 * scale left out); the top_k largest are taken, of equal ones the lower index, NaN last.  causal: a row's own block, the one that
 * holds position q_offset + row, is always taken (where the range has it) and counts as one of the top_k, only blocks before it
 * compete, and its mean is not used. */
int slimpipe_attn_block_select(const slimpipe_attn_params* p, const void* q_slice, const float* means, int32_t block_len, int32_t top_k, int32_t* index,
                               void* hip_stream);

/* Device workspace of slimpipe_attn_block_fwd (is_bwd = 0) or _bwd; both refuse less (SLIMPIPE_EWORKSPACE).  Mostly one float32 result row of
 * head_dim per (row, head, slot): what the blocks of a row give before they are folded. */
int slimpipe_attn_block_workspace_bytes(const slimpipe_attn_params* p, int32_t block_len, int32_t top_k, int is_bwd, size_t* bytes);

/* Forward: row r of head h attends to the keys that slimpipe_attn_fwd would let it see and that lie in one of its blocks.  Any index will
 * do: entries outside the range's blocks are no block, a block named twice counts once, order is free.  out, lse, rows without a key and
 * keys that no row sees: as in slimpipe_attn_fwd.  A bf16 out is folded from results of a row's blocks in float16 with a float32
 * scale (weights and sums in float32), a float32 one from float32 results; likewise dq in the backward.  Under results of either dtype, as in
 * slimpipe_attn_fwd and _bwd, the probabilities, and in the backward dS too, are rounded to bf16 once for the matrix units (the forward
 * of a few tokens keeps them in float32); scores, softmax statistics and sums are float32.  Against 64 bits out is off by 0.0020 to 0.0023
 * of its size and the gradients by 0.0024 (root mean square), of which one rounding to bf16 is 0.0017.  Results do not depend on the order in which workgroups run. */
int slimpipe_attn_block_fwd(const slimpipe_attn_params* p, const void* q_slice, const void* const* k_chunks, const void* const* v_chunks, int32_t n_chunks,
                            int64_t chunk_len, int32_t block_len, int32_t top_k, const int32_t* index, void* out, float* lse, void* workspace,
                            size_t workspace_bytes, void* hip_stream);

/* Backward of slimpipe_attn_block_fwd with the same index: gradients through the attention to the chosen keys.  out, lse, dq, dk / dv
 * (a chunk list as k / v), accumulation, row and key order independence and shared memory are as in slimpipe_attn_bwd(_chunked); keys of the range that no
 * row chose or sees get 0 (or nothing is added). */
int slimpipe_attn_block_bwd(const slimpipe_attn_params* p, const void* q_slice, const void* const* k_chunks, const void* const* v_chunks, int32_t n_chunks,
                            int64_t chunk_len, int32_t block_len, int32_t top_k, const int32_t* index, const void* out, const void* d_out, const float* lse,
                            void* dq, int32_t dq_dtype, int32_t dq_accumulate, float* const* dk_chunks, float* const* dv_chunks, int32_t dkv_accumulate,
                            void* workspace, size_t workspace_bytes, void* hip_stream);

/* A key/value cache held in 4 bits, for long prefixes that are only read (answering from a prompt, evaluation): 4.25 bits an element
 * instead of 16.  32 consecutive elements of a head share a scale 2^e, stored as the byte e + 127; e is the smallest integer, at least
 * -125, with max |x| < 7 * 2^e.  An element is the nearest of 0, 0.5, 1, 1.5, 2, 3, 4, 6 (codes 0 .. 7, ties to the even code) times 2^e, a sign
 * bit above the code; two to a byte, the first in the low half.  A group with an infinity or a NaN has scale byte 255 and reads as NaN.
 *   codes, scales : [batch, kv_capacity, n_kv_heads, head_dim / 2] and [.., head_dim / 32] bytes, for keys and for values, at the kv
 *              strides of p, which count ELEMENTS: byte strides are half and a 32nd of them.  They are multiples of 32
 *              (SLIMPIPE_EINVAL_STRIDE otherwise), codes 16-byte aligned.
 *              Magnitudes from 1.75 * 2^127 on read as infinities.
 *   limits   : kv_capacity <= 2^36, batch * n_kv_heads <= 65535, 2^30 keys in a range, less than 2^27 rows of all heads in a slice, a store or a
 *              load (SLIMPIPE_EINVAL_SHAPE otherwise). */

/* Stores the rows of a slice at positions q_offset .. q_offset + s_q - 1.  k_slice, v_slice: bf16 [batch, s_q, n_kv_heads, head_dim] with the q
 * strides.  Other rows of the cache are untouched.  (n_q_heads, causal, scale and the key range are only validated.) */
int slimpipe_attn_kv4_store(const slimpipe_attn_params* p, const void* k_slice, const void* v_slice, void* k_codes, void* k_scales, void* v_codes,
                            void* v_scales, void* hip_stream);
/* Rows [kv_begin, kv_end) as the bf16 numbers they stand for (exactly): k_rows, v_rows [batch, kv_end - kv_begin, n_kv_heads, head_dim] with the
 * o strides. */
int slimpipe_attn_kv4_load(const slimpipe_attn_params* p, const void* k_codes, const void* k_scales, const void* v_codes, const void* v_scales, void* k_rows,
                           void* v_rows, void* hip_stream);
/* slimpipe_attn_fwd over such a cache, from one token to a slice: the same visibility, out, lse and rows without a key, and (out, lse) of key
 * ranges fold with those of bf16 calls (an old prefix in 4 bits, the newest slices in bf16).  workspace: slimpipe_attn_kv4_workspace_bytes
 * (0 for calls that fill the GPU by themselves: may be NULL then), for the float32 partial results of the key ranges that a call of few rows is
 * cut into.  Results do not depend on the order in which workgroups run.  Codes are converted
 * to bf16 exactly; roundings are otherwise those of slimpipe_attn_block_fwd with float32 results of the key ranges. */
int slimpipe_attn_kv4_workspace_bytes(const slimpipe_attn_params* p, size_t* bytes);
int slimpipe_attn_fwd_kv4(const slimpipe_attn_params* p, const void* q_slice, const void* k_codes, const void* k_scales, const void* v_codes,
                          const void* v_scales, void* out, float* lse, void* workspace, size_t workspace_bytes, void* hip_stream);

/* A key/value cache held in 8 bits with a scale for each block of rows and head, for prefixes that are kept for reading (answering from a prompt, token
 * after token).  Rows [j * block_len, (j + 1) * block_len) of a kv head share a scale 2^e, stored as the byte e + 127; e is the smallest integer, at
 * least -110, with max |x| <= 448 * 2^e over the finite elements of the block.  An element is x / 2^e rounded to an 8-bit float: sign, 4 exponent bits (bias 7), 3 mantissa
 * bits, subnormal below 2^-6, ties to the even code, largest 448, 0x7f and 0xff NaN.  Infinities and NaN are stored as NaN; magnitudes
 * that round to 2^128 (from 1.9375 * 2^127 on) read as infinities.
 *   block_len     : a power of two, 16 .. 256 (SLIMPIPE_EINVAL_SHAPE otherwise).
 *   codes         : bytes [batch, kv_capacity, n_kv_heads, head_dim] for keys and for values, at the kv strides of p, multiples of 16
 *              (SLIMPIPE_EINVAL_STRIDE otherwise), 16-byte aligned.
 *   scales        : bytes [batch, ceil(kv_capacity / block_len), n_kv_heads], contiguous.
 *   limits   : kv_capacity <= 2^36, batch * n_kv_heads <= 65535, 2^30 keys in a range, less than 2^27 rows of all heads in a slice, a store or a
 *              load (SLIMPIPE_EINVAL_SHAPE otherwise). */

/* Appends the rows of a slice at positions q_offset .. q_offset + s_q - 1, behind the q_offset rows that the cache holds.  k_slice, v_slice: bf16
 * [batch, s_q, n_kv_heads, head_dim] with the q strides.  A block that holds rows already keeps its scale, or takes the larger one that the new rows need; its rows are
 * then rounded once more (without an error but for elements that fall below 2^-6 of the new scale).  What rows behind the last one of the slice stood for is lost in
 * blocks that the slice touches (their codes stay, the scale may change).  (n_q_heads, causal, scale and the key range are only validated.) */
int slimpipe_attn_kv8_store(const slimpipe_attn_params* p, int32_t block_len, const void* k_slice, const void* v_slice, void* k_codes, void* k_scales,
                            void* v_codes, void* v_scales, void* hip_stream);
/* Rows [kv_begin, kv_end) as the bf16 numbers they stand for (exactly): k_rows, v_rows [batch, kv_end - kv_begin, n_kv_heads, head_dim] with the
 * o strides. */
int slimpipe_attn_kv8_load(const slimpipe_attn_params* p, int32_t block_len, const void* k_codes, const void* k_scales, const void* v_codes,
                           const void* v_scales, void* k_rows, void* v_rows, void* hip_stream);
/* slimpipe_attn_fwd over such a cache, from one token to a slice: the same visibility, out, lse and rows without a key, and (out, lse) of key
 * ranges fold with those of bf16 and 4-bit calls.  workspace: slimpipe_attn_kv8_workspace_bytes (may be 0: NULL then; less is refused with
 * SLIMPIPE_EWORKSPACE).  For slices of 2048 and more rows of a kv head that includes room for a bf16 copy of the keys and values they see (4 * head_dim bytes a key and
 * kv head); such a call may be given less: it then converts tile by tile, in as many key ranges as there is room for, or copies all the same where that is
 * faster.  A call whose blocks of 256 rows fill the chip is up to a third slower then; one of fewer blocks fills it with key ranges, and needs their room (256 rows
 * of 8 heads on one behind 32512 keys, us with 29 MiB, what the query says, 73, with 16 74, 8 106, 2 372, none 722).  Results do not depend on the order in which workgroups
 * run, only on the room.  Codes are converted to bf16 exactly; roundings are otherwise those of slimpipe_attn_fwd. */
int slimpipe_attn_kv8_workspace_bytes(const slimpipe_attn_params* p, int32_t block_len, size_t* bytes);
int slimpipe_attn_fwd_kv8(const slimpipe_attn_params* p, int32_t block_len, const void* q_slice, const void* k_codes, const void* k_scales,
                          const void* v_codes, const void* v_scales, void* out, float* lse, void* workspace, size_t workspace_bytes, void* hip_stream);

/* Eviction: a cache in 8 bits made smaller by the attention weight that its rows have gathered.  The three calls below sum the weights up, choose the rows
 * that stay, and move them, kv head by kv head, to another cache, where they lie one after the other in their old order: attention over it goes by rows
 * (q_offset = rows of the cache), while the positions of queries and keys in slimpipe_attn_norm_rotate go on. */

/* weights[b, h, j] = decay * previous[b, h, j] + sum of exp(scale * q.k_j - lse) over the rows of the slice that see key j and the query heads of kv head h, for
 * the keys of [kv_begin, kv_end); others are untouched.  weights, previous: float32 [batch, n_kv_heads, kv_capacity], contiguous; previous may be NULL (for 0) or
 * weights itself.  previous is read for all of these keys, those of the slice's own rows too: it has to hold 0 for rows that are new.  lse: what the attention
 * of these rows over all their keys returned; a row whose lse is -inf adds nothing, whatever its queries hold (rows of a padded batch, for instance).  Values are
 * not read.
 * workspace: slimpipe_attn_kv8_weights_workspace_bytes (may be 0: NULL then).  Sums run in a fixed order, in 32 bits.
 *   limits : as for the cache's other calls; decay finite; ceil(keys / 256) * batch * n_kv_heads <= 2^24 - 8 (SLIMPIPE_EINVAL_SHAPE otherwise). */
int slimpipe_attn_kv8_weights_workspace_bytes(const slimpipe_attn_params* p, int32_t block_len, size_t* bytes);
int slimpipe_attn_kv8_weights(const slimpipe_attn_params* p, int32_t block_len, const void* q_slice, const void* k_codes, const void* k_scales,
                              const float* lse, const float* previous, float decay, float* weights, void* workspace, size_t workspace_bytes, void* hip_stream);
/* Of the first `rows` entries of each plane (batch index, kv head) of weights [planes, capacity] the `recent` last ones and the keep - recent largest of the
 * others (equal ones, both zeros alike, the lower index first; NaN behind everything): their indices, ascending, in index, int32 [planes, keep], contiguous.
 *   workspace : slimpipe_attn_kv8_keep_workspace_bytes (may be 0: NULL then).
 *   limits    : planes 1 .. 65535, rows 1 .. 2^30 (SLIMPIPE_EINVAL_SHAPE), 0 <= recent <= keep, 1 <= keep <= rows <= capacity (SLIMPIPE_EINVAL_RANGE). */
int slimpipe_attn_kv8_keep_workspace_bytes(int32_t planes, int64_t rows, int64_t keep, size_t* bytes);
int slimpipe_attn_kv8_keep(const float* weights, int32_t planes, int64_t capacity, int64_t rows, int64_t keep, int64_t recent, int32_t* index,
                           void* workspace, size_t workspace_bytes, void* hip_stream);
/* Rows index[b, h, 0 .. keep - 1] of every kv head of a cache (p) as rows 0 .. keep - 1 of another one (to: its kv_capacity and kv strides, the same batch, kv
 * heads and head_dim; the same block_len).  A block's scale is the largest that its rows had (2^-110 where none is a row); rows of smaller scales are rounded to it (without an error
 * but for elements that fall below 2^-6 of it).  Rows of `to` behind them keep their codes.  index: int32 [batch, n_kv_heads, keep]; any will do: a row may come
 * twice, an entry outside [0, kv_capacity) gives a row of zeros.  weights, kept_weights: the sums move along, [batch, n_kv_heads, kv_capacity] of either
 * cache; both or neither NULL.  kept_weights of the rows behind (from `keep` on) are left as they are: before slimpipe_attn_kv8_weights adds to them, rows that are
 * appended there have to get 0, wherever the memory may hold anything else.  The two caches, and the two sums, may not share memory (SLIMPIPE_EINVAL_RANGE). */
int slimpipe_attn_kv8_gather(const slimpipe_attn_params* p, int32_t block_len, const int32_t* index, int64_t keep, const void* k_codes,
                             const void* k_scales, const void* v_codes, const void* v_scales, const float* weights, const slimpipe_attn_params* to,
                             void* to_k_codes, void* to_k_scales, void* to_v_codes, void* to_v_scales, float* kept_weights, void* hip_stream);

/* Norm of every head of queries and keys, and the rotation of pairs of its elements by the row's position, in one pass: what a slice's projections
 * go through before the attention calls.  For a head x of a row at position t
 *     y = x / sqrt(mean(x^2) + eps) * weight;  of the first rotate_dim elements the pairs (i, i + rotate_dim / 2), or (2 i, 2 i + 1) when
 *     interleaved, become (y_a cos - y_b sin, y_b cos + y_a sin) at the angle t * frequencies[i]; the others stay.
 * Angles are computed in 64 bits, norms and products in 32, results rounded to bf16 once.  (A head whose sum of squares passes 2^128, with elements of 2^60
 * and more, has results of 0, and a gradient that may be NaN.)
 *   q, k            : bf16 [batch, rows, heads, head_dim] with the q and k strides (parts of one projected row, for instance); a side with 0 heads is not part
 *                     of the call, its pointers may be NULL.
 *   q_weight, k_weight : float32 [head_dim], NULL for ones.
 *   frequencies     : float64 [rotate_dim / 2], radians a position (NULL when rotate_dim is 0).
 *   positions       : int64 [batch, rows] contiguous, 0 .. 2^52, or NULL: row r is at p->position + r.
 *   q_out, k_out    : bf16 with the qo and ko strides (k_out may be the slice's rows of a prefix).  A result may take the place of its operand (same pointer, same
 *                     strides); tensors that overlap in other ways must not be passed.
 * The backward takes the gradients of q_out and k_out (qo and ko strides, bf16 or float32 each: dk as the accumulators hold it) and gives those of q
 * and k (bf16, the q and k strides; dq may take the place of q or, with equal strides and bf16, of dq_out) and of the weights (float32 [head_dim],
 * overwritten, or added to when weight_accumulate; NULL: not wanted; only for weights that are given).  Sums run in a fixed order.
 *   workspace : slimpipe_attn_norm_rotate_workspace_bytes, needed when a weight's gradient is wanted (SLIMPIPE_EWORKSPACE).
 *   limits    : rotate_dim a multiple of 16, 0 .. head_dim; eps finite and at least 2^-126; heads 0 .. 65535, less than 2^28 rows of all heads
 *               (SLIMPIPE_EINVAL_SHAPE); position + rows <= 2^52 (SLIMPIPE_EINVAL_RANGE). */
typedef struct slimpipe_rotate_params {
  int32_t batch;
  int32_t rows;
  int32_t n_q_heads;    /* any two numbers, not both 0                                    */
  int32_t n_kv_heads;
  int32_t head_dim;     /* 64 or 128                                                      */
  int32_t rotate_dim;
  int32_t interleaved;  /* 0 or 1                                                         */
  float   eps;
  int64_t position;
  int64_t q_stride_b, q_stride_s, q_stride_h;     /* q and dq                              */
  int64_t k_stride_b, k_stride_s, k_stride_h;     /* k and dk                              */
  int64_t qo_stride_b, qo_stride_s, qo_stride_h;  /* q_out and dq_out                      */
  int64_t ko_stride_b, ko_stride_s, ko_stride_h;  /* k_out and dk_out                      */
} slimpipe_rotate_params;

int slimpipe_attn_norm_rotate(const slimpipe_rotate_params* p, const void* q, const void* k, const float* q_weight, const float* k_weight,
                              const double* frequencies, const int64_t* positions, void* q_out, void* k_out, void* hip_stream);
int slimpipe_attn_norm_rotate_workspace_bytes(const slimpipe_rotate_params* p, size_t* bytes);
int slimpipe_attn_norm_rotate_bwd(const slimpipe_rotate_params* p, const void* q, const void* k, const float* q_weight, const float* k_weight,
                                  const double* frequencies, const int64_t* positions, const void* dq_out, int32_t dq_out_dtype, const void* dk_out,
                                  int32_t dk_out_dtype, void* dq, void* dk, float* dq_weight, float* dk_weight, int32_t weight_accumulate,
                                  void* workspace, size_t workspace_bytes, void* hip_stream);

const char* slimpipe_attn_strerror(int code);

#ifdef __cplusplus
}
#endif
#endif /* SLIMPIPE_ATTN_H */
