// C ABI of the norm and rotation of queries and keys: argument checks, launches.
#include <float.h>
#include <math.h>
#include <string.h>

#include "host_common.hpp"
#include "rotate.hpp"

using namespace slimpipe;

namespace {

int check(const slimpipe_rotate_params* p) {
  if (!p) return SLIMPIPE_EINVAL_NULL;
  if (p->batch < 1 || p->rows < 1 || p->n_q_heads < 0 || p->n_kv_heads < 0 || p->n_q_heads > 65535 || p->n_kv_heads > 65535) return SLIMPIPE_EINVAL_SHAPE;
  if (p->n_q_heads + p->n_kv_heads < 1 || (p->head_dim != 64 && p->head_dim != 128)) return SLIMPIPE_EINVAL_SHAPE;
  if (p->rotate_dim < 0 || p->rotate_dim > p->head_dim || p->rotate_dim % 16 != 0) return SLIMPIPE_EINVAL_SHAPE;
  if (!(p->eps >= FLT_MIN) || !isfinite(p->eps)) return SLIMPIPE_EINVAL_SHAPE;      // (1 / sqrt(eps) stays finite: rows of zeros stay zeros)
  const int64_t rows = (int64_t)p->batch * p->rows;
  if (rows >= (int64_t)1 << 28 || rows * (p->n_q_heads + p->n_kv_heads) >= (int64_t)1 << 28) return SLIMPIPE_EINVAL_SHAPE;      // (less than 2^32 threads)
  const int64_t far = (int64_t)1 << 52;      // (a position is a double on its way to an angle)
  if (p->position < 0 || p->position > far - p->rows) return SLIMPIPE_EINVAL_RANGE;
  if (p->n_q_heads > 0 && !(stride_ok(p->q_stride_b) && stride_ok(p->q_stride_s) && stride_ok(p->q_stride_h) && stride_ok(p->qo_stride_b) &&
                            stride_ok(p->qo_stride_s) && stride_ok(p->qo_stride_h) && p->q_stride_h >= p->head_dim && p->qo_stride_h >= p->head_dim))
    return SLIMPIPE_EINVAL_STRIDE;
  if (p->n_kv_heads > 0 && !(stride_ok(p->k_stride_b) && stride_ok(p->k_stride_s) && stride_ok(p->k_stride_h) && stride_ok(p->ko_stride_b) &&
                             stride_ok(p->ko_stride_s) && stride_ok(p->ko_stride_h) && p->k_stride_h >= p->head_dim && p->ko_stride_h >= p->head_dim))
    return SLIMPIPE_EINVAL_STRIDE;
  return SLIMPIPE_OK;
}
bool aligned8(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 7u) == 0; }

// Everything but the pointers of a direction.
int common_args(RotateArgs* a, const slimpipe_rotate_params* p, const void* q, const void* k, const float* q_weight, const float* k_weight,
                const double* frequencies, const int64_t* positions) {
  if ((p->n_q_heads > 0 && !q) || (p->n_kv_heads > 0 && !k) || (p->rotate_dim > 0 && !frequencies)) return SLIMPIPE_EINVAL_NULL;
  if (!aligned16(q) || !aligned16(k) || !aligned4(q_weight) || !aligned4(k_weight) || !aligned8(frequencies) || !aligned8(positions)) return SLIMPIPE_EINVAL_ALIGN;
  memset(a, 0, sizeof(*a));
  RotateSide &sq = a->side[0], &sk = a->side[1];
  sq.x = static_cast<const __bf16*>(q); sq.weight = q_weight; sq.heads = p->n_q_heads;
  sq.stride_b = p->q_stride_b; sq.stride_s = p->q_stride_s; sq.stride_h = p->q_stride_h;
  sq.out_stride_b = p->qo_stride_b; sq.out_stride_s = p->qo_stride_s; sq.out_stride_h = p->qo_stride_h;
  sk.x = static_cast<const __bf16*>(k); sk.weight = k_weight; sk.heads = p->n_kv_heads;
  sk.stride_b = p->k_stride_b; sk.stride_s = p->k_stride_s; sk.stride_h = p->k_stride_h;
  sk.out_stride_b = p->ko_stride_b; sk.out_stride_s = p->ko_stride_s; sk.out_stride_h = p->ko_stride_h;
  a->frequency = frequencies; a->positions = positions; a->position = p->position;
  a->rows = p->rows; a->interleaved = p->interleaved != 0; a->rotate_dim = p->rotate_dim; a->eps = p->eps;
  a->total_rows = (int64_t)p->batch * p->rows;
  const int per = rotate_rows_per_wave(p->head_dim);
  a->row_blocks = (a->total_rows + per - 1) / per;
  return SLIMPIPE_OK;
}
// Cuts the heads of either side into sets of at most `most` and the rows into blocks; `waves` of them at least, where there are heads enough, so that small calls
// fill the chip.
void plan(RotateArgs* a, int most, int64_t waves) {
  a->heads_wave = most;
  auto sets = [&](int i) { return (a->side[i].heads + a->heads_wave - 1) / a->heads_wave; };
  while (a->heads_wave > 1 && a->row_blocks * (sets(0) + sets(1)) < waves) --a->heads_wave;
  a->sets[0] = sets(0);
  a->sets[1] = sets(1);
}
void plan_fwd(RotateArgs* a) {
  plan(a, kRotateFwdHeads, (int64_t)compute_units() * 4);
  a->workgroups = (int32_t)((a->row_blocks + 3) / 4 * (a->sets[0] + a->sets[1]));
}
// Backward: beyond 2 workgroups a compute unit, what it holds at once, the waves take several blocks of rows (16384 rows of 9 heads: 28.2 us,
// with up to 4 a unit 30.8), which leaves few sums of the weights' gradients to add up.
void plan_bwd(RotateArgs* a) {
  plan(a, kRotateBwdHeads, (int64_t)compute_units() * 4);
  const int64_t sets = a->sets[0] + a->sets[1], groups = (a->row_blocks + 3) / 4, fit = (int64_t)compute_units() * 2 / sets;
  const int64_t taken = groups < fit ? groups : fit > 1 ? fit : 1;
  a->wave_blocks = 4 * taken;
  a->workgroups = (int32_t)(taken * sets);
}
size_t bytes_of(const RotateArgs& a, int head_dim) { return (size_t)a.workgroups * head_dim * 4; }

int status(hipError_t e) { return e == hipSuccess ? SLIMPIPE_OK : SLIMPIPE_ELAUNCH; }

}  // namespace

extern "C" {

int slimpipe_attn_norm_rotate(const slimpipe_rotate_params* p, const void* q, const void* k, const float* q_weight, const float* k_weight,
                              const double* frequencies, const int64_t* positions, void* q_out, void* k_out, void* hip_stream) {
  int rc = check(p);
  if (rc != SLIMPIPE_OK) return rc;
  if ((p->n_q_heads > 0 && !q_out) || (p->n_kv_heads > 0 && !k_out)) return SLIMPIPE_EINVAL_NULL;
  RotateArgs a;
  rc = common_args(&a, p, q, k, q_weight, k_weight, frequencies, positions);
  if (rc != SLIMPIPE_OK) return rc;
  if (!aligned16(q_out) || !aligned16(k_out)) return SLIMPIPE_EINVAL_ALIGN;
  a.side[0].out = static_cast<__bf16*>(q_out);
  a.side[1].out = static_cast<__bf16*>(k_out);
  plan_fwd(&a);
  return status(launch_rotate_fwd(a, p->head_dim, static_cast<hipStream_t>(hip_stream)));
}

int slimpipe_attn_norm_rotate_workspace_bytes(const slimpipe_rotate_params* p, size_t* bytes) {
  if (!bytes) return SLIMPIPE_EINVAL_NULL;
  const int rc = check(p);
  if (rc != SLIMPIPE_OK) return rc;
  RotateArgs a;
  memset(&a, 0, sizeof(a));
  a.side[0].heads = p->n_q_heads; a.side[1].heads = p->n_kv_heads;
  const int per = rotate_rows_per_wave(p->head_dim);
  a.row_blocks = ((int64_t)p->batch * p->rows + per - 1) / per;
  plan_bwd(&a);
  *bytes = bytes_of(a, p->head_dim);
  return SLIMPIPE_OK;
}

int slimpipe_attn_norm_rotate_bwd(const slimpipe_rotate_params* p, const void* q, const void* k, const float* q_weight, const float* k_weight,
                                  const double* frequencies, const int64_t* positions, const void* dq_out, int32_t dq_out_dtype, const void* dk_out,
                                  int32_t dk_out_dtype, void* dq, void* dk, float* dq_weight, float* dk_weight, int32_t weight_accumulate, void* workspace,
                                  size_t workspace_bytes, void* hip_stream) {
  int rc = check(p);
  if (rc != SLIMPIPE_OK) return rc;
  if ((p->n_q_heads > 0 && (!dq_out || !dq)) || (p->n_kv_heads > 0 && (!dk_out || !dk)) || (dq_weight && (!q_weight || p->n_q_heads < 1)) ||
      (dk_weight && (!k_weight || p->n_kv_heads < 1)))
    return SLIMPIPE_EINVAL_NULL;
  if ((dq_out_dtype != SLIMPIPE_BF16 && dq_out_dtype != SLIMPIPE_F32) || (dk_out_dtype != SLIMPIPE_BF16 && dk_out_dtype != SLIMPIPE_F32)) return SLIMPIPE_EINVAL_SHAPE;
  RotateArgs a;
  rc = common_args(&a, p, q, k, q_weight, k_weight, frequencies, positions);
  if (rc != SLIMPIPE_OK) return rc;
  if (!aligned16(dq_out) || !aligned16(dk_out) || !aligned16(dq) || !aligned16(dk) || !aligned4(dq_weight) || !aligned4(dk_weight)) return SLIMPIPE_EINVAL_ALIGN;
  plan_bwd(&a);
  if (dq_weight || dk_weight) {
    if (!workspace || workspace_bytes < bytes_of(a, p->head_dim)) return SLIMPIPE_EWORKSPACE;
    if (!aligned16(workspace)) return SLIMPIPE_EINVAL_ALIGN;
    a.part = static_cast<float*>(workspace);
  }
  a.side[0].d_out = dq_out; a.side[0].d_out_f32 = dq_out_dtype == SLIMPIPE_F32; a.side[0].out = static_cast<__bf16*>(dq);
  a.side[1].d_out = dk_out; a.side[1].d_out_f32 = dk_out_dtype == SLIMPIPE_F32; a.side[1].out = static_cast<__bf16*>(dk);
  a.d_weight[0] = dq_weight; a.d_weight[1] = dk_weight;
  a.weight_accumulate = weight_accumulate != 0;
  return status(launch_rotate_bwd(a, p->head_dim, static_cast<hipStream_t>(hip_stream)));
}

}  // extern "C"
