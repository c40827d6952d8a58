// C ABI of the key/value cache held in 4 bits: argument checks, workspace layout, launches.
#include <string.h>

#include "host_common.hpp"
#include "kv4.hpp"

using namespace slimpipe;

namespace {

// What every call on the cache checks beyond slimpipe_attn_validate: whole groups of 32 elements, counts that fit a launch (less than 2^32
// threads) and 32 bits.
int check_cache(const slimpipe_attn_params* p) {
  if (p->kv_stride_b % 32 != 0 || p->kv_stride_s % 32 != 0 || p->kv_stride_h % 32 != 0) return SLIMPIPE_EINVAL_STRIDE;
  if (p->kv_capacity > (int64_t)1 << 36 || (int64_t)p->batch * p->n_kv_heads > 65535) return SLIMPIPE_EINVAL_SHAPE;
  if ((int64_t)p->batch * p->n_q_heads * p->s_q >= 1 << 27 || p->kv_end - p->kv_begin > 1 << 30) return SLIMPIPE_EINVAL_SHAPE;
  return SLIMPIPE_OK;
}
int check_operands(const void* k_codes, const void* k_scales, const void* v_codes, const void* v_scales) {
  if (!k_codes || !k_scales || !v_codes || !v_scales) return SLIMPIPE_EINVAL_NULL;
  return aligned16(k_codes) && aligned16(v_codes) ? SLIMPIPE_OK : SLIMPIPE_EINVAL_ALIGN;
}
int copy_args(Kv4CopyArgs* a, const slimpipe_attn_params* p, int64_t rows) {
  if (rows > 1 << 30 || (int64_t)p->batch * p->n_kv_heads * rows >= 1 << 27) return SLIMPIPE_EINVAL_SHAPE;
  memset(a, 0, sizeof(*a));
  a->n_kv_heads = p->n_kv_heads; a->batch = p->batch; a->rows = rows;
  a->kv_stride_b = p->kv_stride_b; a->kv_stride_s = p->kv_stride_s; a->kv_stride_h = p->kv_stride_h;
  return SLIMPIPE_OK;
}

int64_t rows_of(const slimpipe_attn_params* p) { return (int64_t)p->n_q_heads / p->n_kv_heads * p->s_q; }      // of a plane

// Key ranges that a call is cut into, a workgroup for each and each block of rows, so that the chip is full.
struct Kv4Plan {
  bool few;
  int32_t wave_heads, heads_wg, parts;
  int64_t part_keys;
};
Kv4Plan plan_of(const slimpipe_attn_params* p) {
  const int64_t keys = seen_end(p, p->kv_begin, p->kv_end) - p->kv_begin, rows = rows_of(p), planes = (int64_t)p->batch * p->n_kv_heads;
  Kv4Plan plan{rows <= kKv4FewRows, 1, 1, 1, keys};
  if (plan.few) {
    // two heads a wave: in a cache with heads next to each other their codes share lines (tokens of 4 sequences of 32K keys, us with two and with one:
    // 40 heads 204 and 328, 8 heads 41 and 40)
    plan.wave_heads = rows <= 16 && p->n_kv_heads % 2 == 0 ? 2 : 1;
    const int32_t sets = p->n_kv_heads / plan.wave_heads;
    plan.heads_wg = sets % 4 == 0 ? 4 : sets % 2 == 0 ? 2 : 1;
  }
  const int64_t wgs = plan.few ? planes / (plan.wave_heads * plan.heads_wg) : planes * ((rows + 127) / 128), want = 2 * (int64_t)compute_units();
  // keys of a part (a token of 8 heads on 8000 keys: 256 11.9 us, 512 12.3, 1024 15.7; 256 rows on 8000 keys: 512 34.5 us, 1024 37.3, 2048 53.9)
  const int64_t least = plan.few ? 256 : 512;
  // tokens: whole rounds of the workgroups that the chip holds, two a unit (a token behind 1M keys: one a unit 43 us, two 35, four 42), eight ranges
  // at a time (ranges of the same keys share an XCD)
  int64_t parts = plan.few ? want / wgs : (want + wgs - 1) / wgs;
  if (plan.few && parts >= 8) parts = parts / 8 * 8;
  if (parts > keys / least) parts = keys / least;
  if (parts > 1) {
    const int64_t unit = plan.few ? 32 : 64;      // keys of a step
    plan.part_keys = ((keys + parts - 1) / parts + unit - 1) / unit * unit;
    plan.parts = (int32_t)((keys + plan.part_keys - 1) / plan.part_keys);
  }
  return plan;
}
size_t up(size_t n) { return (n + 255) & ~(size_t)255; }
size_t out_bytes(const slimpipe_attn_params* p, const Kv4Plan& plan) { return up((size_t)p->batch * p->n_q_heads * p->s_q * plan.parts * p->head_dim * 4); }
size_t bytes_of(const slimpipe_attn_params* p, const Kv4Plan& plan) {
  return plan.parts <= 1 ? 0 : out_bytes(p, plan) + up((size_t)p->batch * p->n_q_heads * p->s_q * plan.parts * 4);
}

int status(hipError_t e) { return e == hipSuccess ? SLIMPIPE_OK : SLIMPIPE_ELAUNCH; }

}  // namespace

extern "C" {

int slimpipe_attn_kv4_store(const slimpipe_attn_params* p, const void* k_slice, const void* v_slice, void* k_codes, void* k_scales, void* v_codes,
                            void* v_scales, void* hip_stream) {
  int rc = slimpipe_attn_validate(p, 0);
  if (rc != SLIMPIPE_OK) return rc;
  if (!k_slice || !v_slice) return SLIMPIPE_EINVAL_NULL;
  rc = check_operands(k_codes, k_scales, v_codes, v_scales);
  if (rc == SLIMPIPE_OK) rc = check_cache(p);
  if (rc != SLIMPIPE_OK) return rc;
  if (p->q_offset + p->s_q > p->kv_capacity) return SLIMPIPE_EINVAL_RANGE;
  if (!aligned16(k_slice) || !aligned16(v_slice)) return SLIMPIPE_EINVAL_ALIGN;
  Kv4CopyArgs a;
  rc = copy_args(&a, p, p->s_q);
  if (rc != SLIMPIPE_OK) return rc;
  a.k = {static_cast<uint8_t*>(k_codes), static_cast<uint8_t*>(k_scales)};
  a.v = {static_cast<uint8_t*>(v_codes), static_cast<uint8_t*>(v_scales)};
  a.k_src = static_cast<const __bf16*>(k_slice);
  a.v_src = static_cast<const __bf16*>(v_slice);
  a.position = p->q_offset;
  a.x_stride_b = p->q_stride_b; a.x_stride_s = p->q_stride_s; a.x_stride_h = p->q_stride_h;
  return status(launch_kv4_store(a, p->head_dim, static_cast<hipStream_t>(hip_stream)));
}

int slimpipe_attn_kv4_load(const slimpipe_attn_params* p, const void* k_codes, const void* k_scales, const void* v_codes, const void* v_scales, void* k_rows,
                           void* v_rows, void* hip_stream) {
  int rc = slimpipe_attn_validate(p, 0);
  if (rc != SLIMPIPE_OK) return rc;
  if (!k_rows || !v_rows) return SLIMPIPE_EINVAL_NULL;
  rc = check_operands(k_codes, k_scales, v_codes, v_scales);
  if (rc == SLIMPIPE_OK) rc = check_cache(p);
  if (rc != SLIMPIPE_OK) return rc;
  if (!aligned16(k_rows) || !aligned16(v_rows)) return SLIMPIPE_EINVAL_ALIGN;
  if (p->kv_begin == p->kv_end) return SLIMPIPE_OK;
  Kv4CopyArgs a;
  rc = copy_args(&a, p, p->kv_end - p->kv_begin);
  if (rc != SLIMPIPE_OK) return rc;
  a.k = {static_cast<uint8_t*>(const_cast<void*>(k_codes)), static_cast<uint8_t*>(const_cast<void*>(k_scales))};
  a.v = {static_cast<uint8_t*>(const_cast<void*>(v_codes)), static_cast<uint8_t*>(const_cast<void*>(v_scales))};
  a.k_dst = static_cast<__bf16*>(k_rows);
  a.v_dst = static_cast<__bf16*>(v_rows);
  a.position = p->kv_begin;
  a.x_stride_b = p->o_stride_b; a.x_stride_s = p->o_stride_s; a.x_stride_h = p->o_stride_h;
  return status(launch_kv4_load(a, p->head_dim, static_cast<hipStream_t>(hip_stream)));
}

int slimpipe_attn_kv4_workspace_bytes(const slimpipe_attn_params* p, size_t* bytes) {
  if (!bytes) return SLIMPIPE_EINVAL_NULL;
  int rc = slimpipe_attn_validate(p, 0);
  if (rc == SLIMPIPE_OK) rc = check_cache(p);
  if (rc != SLIMPIPE_OK) return rc;
  *bytes = bytes_of(p, plan_of(p));
  return SLIMPIPE_OK;
}

int slimpipe_attn_fwd_kv4(const slimpipe_attn_params* p, const void* q_slice, const void* k_codes, const void* k_scales, const void* v_codes,
                          const void* v_scales, void* out, float* lse, void* workspace, size_t workspace_bytes, void* hip_stream) {
  int rc = slimpipe_attn_validate(p, 0);
  if (rc != SLIMPIPE_OK) return rc;
  if (!q_slice || !out || !lse) return SLIMPIPE_EINVAL_NULL;
  rc = check_operands(k_codes, k_scales, v_codes, v_scales);
  if (rc == SLIMPIPE_OK) rc = check_cache(p);
  if (rc != SLIMPIPE_OK) return rc;
  if (!aligned16(q_slice) || !aligned16(out) || !aligned4(lse)) return SLIMPIPE_EINVAL_ALIGN;
  const Kv4Plan plan = plan_of(p);
  if (workspace_bytes < bytes_of(p, plan) || (plan.parts > 1 && !workspace)) return SLIMPIPE_EWORKSPACE;
  if (!aligned16(workspace)) return SLIMPIPE_EINVAL_ALIGN;
  Kv4Args a;
  memset(&a, 0, sizeof(a));
  a.q = static_cast<const __bf16*>(q_slice);
  a.k = {static_cast<uint8_t*>(const_cast<void*>(k_codes)), static_cast<uint8_t*>(const_cast<void*>(k_scales))};
  a.v = {static_cast<uint8_t*>(const_cast<void*>(v_codes)), static_cast<uint8_t*>(const_cast<void*>(v_scales))};
  a.out = out;
  a.lse = lse;
  a.batch = p->batch; a.s_q = p->s_q; a.n_q_heads = p->n_q_heads; a.n_kv_heads = p->n_kv_heads; a.group = p->n_q_heads / p->n_kv_heads;
  a.causal = p->causal; a.out_f32 = p->out_dtype == SLIMPIPE_F32;
  a.q_offset = p->q_offset; a.kv_begin = p->kv_begin; a.kv_end = seen_end(p, p->kv_begin, p->kv_end);
  a.scale_log2e = p->scale * 1.4426950408889634f;
  a.q_stride_b = p->q_stride_b; a.q_stride_s = p->q_stride_s; a.q_stride_h = p->q_stride_h;
  a.kv_stride_b = p->kv_stride_b; a.kv_stride_s = p->kv_stride_s; a.kv_stride_h = p->kv_stride_h;
  a.o_stride_b = p->o_stride_b; a.o_stride_s = p->o_stride_s; a.o_stride_h = p->o_stride_h;
  a.n_parts = plan.parts;
  a.part_keys = plan.part_keys;
  a.wave_heads = plan.wave_heads; a.heads_wg = plan.heads_wg;
  if (plan.parts > 1) {
    a.part_out = static_cast<float*>(workspace);
    a.part_lse = reinterpret_cast<float*>(static_cast<char*>(workspace) + out_bytes(p, plan));
  }
  if (ensure_device_ready() != SLIMPIPE_OK) return SLIMPIPE_ELAUNCH;
  hipStream_t st = static_cast<hipStream_t>(hip_stream);
  if (launch_kv4_fwd(a, p->head_dim, plan.few, st) != hipSuccess) return SLIMPIPE_ELAUNCH;
  if (plan.parts <= 1) return SLIMPIPE_OK;
  PartMergeArgs m;
  m.part_out = a.part_out; m.part_f32 = 1; m.part_scale = nullptr; m.part_lse = a.part_lse; m.parts = plan.parts; m.s_q = p->s_q; m.n_q_heads = p->n_q_heads; m.out_f32 = a.out_f32;
  m.rows = (int64_t)p->batch * p->n_q_heads * p->s_q;
  m.out = out; m.lse = lse;
  m.o_stride_b = p->o_stride_b; m.o_stride_s = p->o_stride_s; m.o_stride_h = p->o_stride_h;
  return status(launch_part_merge(m, p->head_dim, st));
}

}  // extern "C"
