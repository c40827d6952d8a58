// C ABI of the key/value cache held in 8 bits: argument checks, workspace layout, launches.
#include <math.h>
#include <string.h>

#include "host_common.hpp"
#include "../../include/slimpipe_attn_bench.h"
#include "kv8.hpp"

using namespace slimpipe;

namespace {

// What every call on the cache checks beyond slimpipe_attn_validate: block lengths, whole pieces of 16 elements, counts that fit a launch (less than
// 2^32 threads) and 32 bits.
int check_cache(const slimpipe_attn_params* p, int32_t block_len) {
  if (block_len < 16 || block_len > 256 || (block_len & (block_len - 1)) != 0) return SLIMPIPE_EINVAL_SHAPE;
  if (p->kv_stride_b % 16 != 0 || p->kv_stride_s % 16 != 0 || p->kv_stride_h % 16 != 0) return SLIMPIPE_EINVAL_STRIDE;
  if (p->kv_capacity > (int64_t)1 << 36 || (int64_t)p->batch * p->n_kv_heads > 65535) return SLIMPIPE_EINVAL_SHAPE;
  if ((int64_t)p->batch * p->n_q_heads * p->s_q >= 1 << 27 || p->kv_end - p->kv_begin > 1 << 30) return SLIMPIPE_EINVAL_SHAPE;
  return SLIMPIPE_OK;
}
int check_operands(const void* k_codes, const void* k_scales, const void* v_codes, const void* v_scales) {
  if (!k_codes || !k_scales || !v_codes || !v_scales) return SLIMPIPE_EINVAL_NULL;
  return aligned16(k_codes) && aligned16(v_codes) ? SLIMPIPE_OK : SLIMPIPE_EINVAL_ALIGN;
}
Kv8Cache cache_of(const slimpipe_attn_params* p, int32_t block_len, const void* k_codes, const void* k_scales, const void* v_codes, const void* v_scales) {
  Kv8Cache c;
  auto bytes = [](const void* x) { return static_cast<uint8_t*>(const_cast<void*>(x)); };
  c.k = {bytes(k_codes), bytes(k_scales)};
  c.v = {bytes(v_codes), bytes(v_scales)};
  c.n_kv_heads = p->n_kv_heads;
  c.shift = __builtin_ctz((unsigned)block_len);
  c.stride_b = p->kv_stride_b; c.stride_s = p->kv_stride_s; c.stride_h = p->kv_stride_h;
  c.blocks = (p->kv_capacity + block_len - 1) / block_len;
  return c;
}
bool rows_fit(const slimpipe_attn_params* p, int64_t rows) { return rows <= 1 << 30 && (int64_t)p->batch * p->n_kv_heads * rows < 1 << 27; }

int64_t rows_of(const slimpipe_attn_params* p) { return (int64_t)p->n_q_heads / p->n_kv_heads * p->s_q; }      // of a plane

// Key ranges of a call of few rows: `least_rounds` workgroups for every compute unit, then as many more (up to `most_rounds`) as the last round needs to be nearly
// full, from 8 on in eights (ranges of the same keys share an XCD).  Attention, 2 to 6: tokens of 4 sequences of 32K keys, 40 heads, us: 8 ranges, 320
// workgroups, 337; 24, 960, 255; 32, 1280, 246; beyond what evens the rounds out the fold of the results costs more than it gives (a token of 8 heads on one behind 1M
// keys: 512 ranges 67, 1024 73, 1536 78).  Sums of weights have no fold, 8 to 12: the same token 42.6 with 2 to 6, 34.9 with 8 to 12; 8 heads of 64 in 8
// sequences of 32K 67 and 42.
int64_t few_parts(int64_t wgs, int64_t most, int64_t least_rounds, int64_t most_rounds) {
  const int64_t units = compute_units();
  if (most * wgs <= least_rounds * units) return most;
  int64_t best = 1;
  double best_full = 0.;
  for (int64_t parts = 1; parts <= most && (parts == 1 || parts * wgs <= most_rounds * units); parts += parts < 8 ? 1 : 8) {
    const int64_t n = parts * wgs;
    const double full = n < least_rounds * units ? 0.5 * (double)n / (double)(least_rounds * units) : (double)n / (double)((n + units - 1) / units * units);
    if (full > best_full) { best = parts; best_full = full; }
    if (full >= 0.95) break;
  }
  return best;
}
// Key ranges of a slice, or parts of its rows: the fewest whose workgroups, `a_unit` a compute unit at once, fill one to three rounds nearly, or those that fill them best (256
// rows of 40 heads on 16640 keys, 80 workgroups of four waves a range: 6 ranges 137 us, 7 167).
int64_t slice_parts(int64_t wgs, int64_t most, int64_t a_unit) {
  const int64_t places = a_unit * compute_units();
  int64_t best = 1;
  double best_full = 0.;
  for (int64_t parts = 1; parts <= most && (parts == 1 || parts * wgs <= 3 * places); ++parts) {
    const int64_t n = parts * wgs;
    const double full = (double)n / (double)((n + places - 1) / places * places);
    if (full > best_full) { best = parts; best_full = full; }
    if (full >= 0.9) break;
  }
  return best;
}
// Which kernel, and key ranges that a call is cut into, a workgroup for each and each block of rows, so that the chip is full.  Eight waves share a converted tile
// where four would convert it twice, but fill the chip later (us with eight and with four, 256 rows of 40 heads on 16640 keys 119 and 140, 800 rows of a kv head on
// 32100 keys 38 and 39; 512 rows of one 33 and 29, 100 rows of 16 heads 51 and 47).
struct Kv8Plan {
  Kv8Kernel kernel;
  int32_t parts;
  int64_t part_keys;
};
void cut_keys(Kv8Plan* plan, int64_t keys, int64_t parts) {
  plan->parts = 1;
  plan->part_keys = keys;
  if (parts <= 1) return;
  const int64_t unit = plan->kernel == Kv8Kernel::few ? 32 : 64;      // keys of a step
  plan->part_keys = ((keys + parts - 1) / parts + unit - 1) / unit * unit;
  plan->parts = (int32_t)((keys + plan->part_keys - 1) / plan->part_keys);
}
Kv8Plan plan_of(const slimpipe_attn_params* p) {
  const int64_t keys = seen_end(p, p->kv_begin, p->kv_end) - p->kv_begin, rows = rows_of(p), planes = (int64_t)p->batch * p->n_kv_heads;
  Kv8Plan plan{Kv8Kernel::few, 1, keys};
  int64_t parts;
  if (rows <= kKv8FewRows) {
    parts = few_parts(planes / kv8_heads_wg(p->n_kv_heads), keys / 256, 2, 6);
  } else {
    const int64_t long_parts = keys / 512, eight = planes * ((rows + 255) / 256);
    plan.kernel = rows > 128 && eight * long_parts >= compute_units() ? Kv8Kernel::eight_waves : Kv8Kernel::four_waves;
    if (plan.kernel == Kv8Kernel::eight_waves) {
      parts = slice_parts(eight, long_parts, 1);
    } else {
      // Ranges of 512 keys or more, or of 128 up to a workgroup a unit where that leaves units idle (us of 512 and of 128: 48 rows of 8 heads on 2 behind 1306 keys
      // 24.8 and 15.8, 500 rows on 1000 keys 29.2 and 20.0).
      const int64_t wgs = planes * ((rows + 127) / 128), units = compute_units();
      int64_t most = long_parts;
      if (most * wgs < units) most = keys / 128 < units / wgs ? keys / 128 : units / wgs;
      parts = slice_parts(wgs, most, 2);
    }
  }
  cut_keys(&plan, keys, parts);
  return plan;
}
// Sums of weights: key ranges of the kernel of few rows, or parts of a plane's rows, whose sums a second launch adds up.
struct Kv8WeightPlan {
  bool few;
  int32_t parts;
  int64_t part_keys;
};
Kv8WeightPlan weight_plan_of(const slimpipe_attn_params* p) {
  const int64_t keys = p->kv_end - p->kv_begin, rows = rows_of(p), planes = (int64_t)p->batch * p->n_kv_heads;
  Kv8WeightPlan plan{rows <= kKv8FewRows, 1, keys};
  if (plan.few) {
    const int64_t parts = few_parts(planes / kv8_heads_wg(p->n_kv_heads), keys / 256, 8, 12);
    if (parts > 1) {
      plan.part_keys = ((keys + parts - 1) / parts + 31) / 32 * 32;
      plan.parts = (int32_t)((keys + plan.part_keys - 1) / plan.part_keys);
    }
    return plan;
  }
  // Parts of 256 rows or more that fill the chip, or one a unit of 128 (a tile) where that leaves units idle (us of parts of 128 and of 256 rows: 652 rows of a kv
  // head on 1547 keys 15.2 and 19.3, 948 on 3156 14.7 and 19.9; 3936 rows of two on 4660 27.9 and 25.6).
  const int64_t wgs = planes * ((keys + kv8_weight_keys() - 1) / kv8_weight_keys()), units = compute_units();
  int64_t parts = wgs > 0 ? slice_parts(wgs, rows / 256, 2) : 1;
  if (parts * wgs < units && wgs > 0) {
    parts = (units + wgs - 1) / wgs;
    if (parts > (rows + 127) / 128) parts = (rows + 127) / 128;
  }
  if (parts > 64) parts = 64;
  plan.parts = parts > 1 ? (int32_t)parts : 1;
  return plan;
}
size_t up(size_t n) { return (n + 255) & ~(size_t)255; }
size_t out_bytes(const slimpipe_attn_params* p, const Kv8Plan& plan) { return up((size_t)p->batch * p->n_q_heads * p->s_q * plan.parts * p->head_dim * 4); }
size_t bytes_of(const slimpipe_attn_params* p, const Kv8Plan& plan) {
  return plan.parts <= 1 ? 0 : out_bytes(p, plan) + up((size_t)p->batch * p->n_q_heads * p->s_q * plan.parts * 4);
}
// Long slices go to slimpipe_attn_fwd over a bf16 copy of the keys that they see, in the workspace.  (Not where early rows see no key: that call does not
// keep them from keys that are not finite.)
bool copies(const slimpipe_attn_params* p) {
  return rows_of(p) >= kKv8CopyRows && seen_end(p, p->kv_begin, p->kv_end) > p->kv_begin && !(p->causal && p->kv_begin > p->q_offset) &&
         rows_fit(p, p->kv_end - p->kv_begin) && (int64_t)p->n_kv_heads * p->head_dim < 1 << 22;      // (a row that slimpipe_attn_fwd takes)
}
size_t copy_bytes(const slimpipe_attn_params* p) {      // keys or values
  return up((size_t)p->batch * (size_t)(seen_end(p, p->kv_begin, p->kv_end) - p->kv_begin) * p->n_kv_heads * p->head_dim * 2);
}
slimpipe_attn_params copy_params(const slimpipe_attn_params* p) {
  slimpipe_attn_params c = *p;
  c.kv_end = seen_end(p, p->kv_begin, p->kv_end);
  c.kv_stride_h = p->head_dim;
  c.kv_stride_s = (int64_t)p->n_kv_heads * p->head_dim;
  c.kv_stride_b = (c.kv_end - c.kv_begin) * c.kv_stride_s;
  return c;
}
// How a call goes with this much room: by a copy of the keys, or by this plan.  (plan.parts 0: it needs more.)
struct Kv8Path {
  bool copy;
  Kv8Plan plan;
};
Kv8Path path_within(const slimpipe_attn_params* p, size_t room) {
  Kv8Path path{false, plan_of(p)};
  Kv8Plan& plan = path.plan;
  const bool may_copy = copies(p);
  const int64_t blocks = (int64_t)p->batch * p->n_kv_heads * ((rows_of(p) + 255) / 256), units = compute_units();
  if (room < bytes_of(p, plan)) {
    if (!may_copy) { plan.parts = 0; return path; }
    // A long slice: as many key ranges as there is room for, and workgroups of four waves where the chip would be half empty with eight (256 rows of 8 heads on one and 32768
    // keys, us with eight and with four, 1 range 834 and 723, 3 302 and 254, 12 90 and 79; 4096 rows of 4 heads on 16096 keys, 2 ranges, 128 workgroups of eight, 231 and
    // 197, 3 163 and 189).
    const int64_t keys = seen_end(p, p->kv_begin, p->kv_end) - p->kv_begin;
    for (int64_t parts = plan.parts - 1; room < bytes_of(p, plan); --parts) cut_keys(&plan, keys, parts);
    if (plan.kernel == Kv8Kernel::eight_waves && 2 * blocks * plan.parts <= units) plan.kernel = Kv8Kernel::four_waves;
  }
  if (!may_copy || room < 2 * copy_bytes(p)) return path;
  const slimpipe_attn_params c = copy_params(p);
  const size_t rest = room - 2 * copy_bytes(p);
  size_t wanted = 0;
  slimpipe_call_path dense;
  if (slimpipe_attn_workspace_bytes(&c, 0, &wanted) != SLIMPIPE_OK) return path;
  path.copy = rest >= wanted;
  if (path.copy || slimpipe_attn_call_path(&c, 0, 1, rest, &dense) != SLIMPIPE_OK) return path;
  // With less beside the copy than the dense call asks for: what a compute unit has to do, in blocks of rows and all keys, tiles 1.22 times as long (us by the copy and by
  // tiles in the same room: 2048 rows of 8 heads on 32768 keys, no range fits, 585 and 704; 4096 of 40 on 18688, as many blocks as fill the chip, 1288 and 1568; 4096 of 4
  // on 16096 307 and 163).
  auto load = [&](int64_t ranges) { return fmax(1.0 / (double)ranges, (double)blocks / (double)units); };
  path.copy = load(dense.ranges) <= 1.22 * load(plan.parts);
  return path;
}
int fwd_by_copy(const slimpipe_attn_params* p, const Kv8Cache& cache, const void* q, void* out, float* lse, char* ws, size_t bytes, void* stream) {
  const slimpipe_attn_params c = copy_params(p);
  const size_t each = copy_bytes(p);
  Kv8CopyArgs a;
  memset(&a, 0, sizeof(a));
  a.cache = cache;
  a.k_dst = reinterpret_cast<__bf16*>(ws);
  a.v_dst = reinterpret_cast<__bf16*>(ws + each);
  a.batch = p->batch; a.rows = c.kv_end - c.kv_begin; a.position = c.kv_begin;
  a.x_stride_b = c.kv_stride_b; a.x_stride_s = c.kv_stride_s; a.x_stride_h = c.kv_stride_h;
  if (launch_kv8_load(a, p->head_dim, static_cast<hipStream_t>(stream)) != hipSuccess) return SLIMPIPE_ELAUNCH;
  // (where row 0 of the copies would be; rows before kv_begin are not read)
  const uintptr_t back = (uintptr_t)(c.kv_begin * c.kv_stride_s * 2);
  return slimpipe_attn_fwd(&c, q, reinterpret_cast<const void*>(reinterpret_cast<uintptr_t>(ws) - back), reinterpret_cast<const void*>(reinterpret_cast<uintptr_t>(ws + each) - back),
                           out, lse, ws + 2 * each, bytes - 2 * each, stream);
}
size_t weight_bytes_of(const slimpipe_attn_params* p, const Kv8WeightPlan& plan) {
  return plan.few || plan.parts <= 1 ? 0 : up((size_t)plan.parts * p->batch * p->n_kv_heads * (size_t)(p->kv_end - p->kv_begin) * 4);
}
// What the sums check beyond check_cache: less than 2^32 threads, 256 for each of the workgroups, which are launched in eights.  (Parts of the rows are cut only where
// there are few.)
int check_weights(const slimpipe_attn_params* p) {
  const int64_t blocks = (p->kv_end - p->kv_begin + kv8_weight_keys() - 1) / kv8_weight_keys();
  return blocks * p->batch * p->n_kv_heads <= ((int64_t)1 << 24) - 8 ? SLIMPIPE_OK : SLIMPIPE_EINVAL_SHAPE;
}
int check_keep(int32_t planes, int64_t capacity, int64_t rows, int64_t keep, int64_t recent) {
  if (planes < 1 || planes > 65535 || rows < 1 || rows > (int64_t)1 << 30 || capacity > (int64_t)1 << 36) return SLIMPIPE_EINVAL_SHAPE;
  return rows <= capacity && keep >= 1 && keep <= rows && recent >= 0 && recent <= keep ? SLIMPIPE_OK : SLIMPIPE_EINVAL_RANGE;
}
// Workgroups of kKeepSpan rows, of more where there would be more than 64 of them (each adds up the counts of all of its plane).
struct KeepPlan {
  int32_t chunks;
  int64_t chunk;
};
KeepPlan keep_plan_of(int64_t rows) {
  if (rows <= kKeepOneRows) return {0, 0};
  const int64_t chunk = (rows + 64 * kKeepSpan - 1) / (64 * kKeepSpan) * kKeepSpan;
  return {(int32_t)((rows + chunk - 1) / chunk), chunk};
}
size_t keep_bytes_of(int32_t planes, const KeepPlan& plan) { return plan.chunks ? (size_t)planes * ((size_t)plan.chunks * kKeepChunkWords + kKeepPlaneWords) * 4 : 0; }
// A move writes its rows while others are still to be read: the two caches, and the two sums, may not share memory.
bool overlap(const Kv8GatherArgs& a, int head_dim) {
  const int64_t heads = a.to.n_kv_heads;
  auto codes = [&](const uint8_t* x, const Kv8Cache& c, int64_t rows) { return span_of(x, 1, a.batch, rows, heads, head_dim, c.stride_b, c.stride_s, c.stride_h); };
  auto bytes = [](const void* x, int64_t n) { return span_of(x, 1, 1, 1, 1, n, 1, 1, 1); };
  const Span from[] = {codes(a.from.k.codes, a.from, a.from_rows), codes(a.from.v.codes, a.from, a.from_rows), bytes(a.from.k.scales, a.batch * a.from.blocks * heads),
                       bytes(a.from.v.scales, a.batch * a.from.blocks * heads), bytes(a.weights, a.weights ? 4 * a.batch * heads * a.weights_stride : 0)};
  const Span to[] = {codes(a.to.k.codes, a.to, a.keep), codes(a.to.v.codes, a.to, a.keep), bytes(a.to.k.scales, a.batch * a.to.blocks * heads),
                     bytes(a.to.v.scales, a.batch * a.to.blocks * heads), bytes(a.kept_weights, a.kept_weights ? 4 * a.batch * heads * a.kept_weights_stride : 0)};
  for (const Span& x : from)
    for (const Span& y : to)
      if (share_memory(x, y)) return true;
  return false;
}

int status(hipError_t e) { return e == hipSuccess ? SLIMPIPE_OK : SLIMPIPE_ELAUNCH; }

}  // namespace

extern "C" {

int slimpipe_attn_kv8_store(const slimpipe_attn_params* p, int32_t block_len, const void* k_slice, const void* v_slice, void* k_codes, void* k_scales,
                            void* v_codes, void* v_scales, void* hip_stream) {
  int rc = slimpipe_attn_validate(p, 0);
  if (rc != SLIMPIPE_OK) return rc;
  if (!k_slice || !v_slice) return SLIMPIPE_EINVAL_NULL;
  rc = check_operands(k_codes, k_scales, v_codes, v_scales);
  if (rc == SLIMPIPE_OK) rc = check_cache(p, block_len);
  if (rc != SLIMPIPE_OK) return rc;
  if (p->q_offset + p->s_q > p->kv_capacity) return SLIMPIPE_EINVAL_RANGE;
  if (!aligned16(k_slice) || !aligned16(v_slice)) return SLIMPIPE_EINVAL_ALIGN;
  if (!rows_fit(p, p->s_q)) return SLIMPIPE_EINVAL_SHAPE;
  Kv8CopyArgs a;
  memset(&a, 0, sizeof(a));
  a.cache = cache_of(p, block_len, k_codes, k_scales, v_codes, v_scales);
  a.k_src = static_cast<const __bf16*>(k_slice);
  a.v_src = static_cast<const __bf16*>(v_slice);
  a.batch = p->batch; a.rows = p->s_q; a.position = p->q_offset;
  a.x_stride_b = p->q_stride_b; a.x_stride_s = p->q_stride_s; a.x_stride_h = p->q_stride_h;
  return status(launch_kv8_store(a, p->head_dim, static_cast<hipStream_t>(hip_stream)));
}

int slimpipe_attn_kv8_load(const slimpipe_attn_params* p, int32_t block_len, const void* k_codes, const void* k_scales, const void* v_codes,
                           const void* v_scales, void* k_rows, void* v_rows, void* hip_stream) {
  int rc = slimpipe_attn_validate(p, 0);
  if (rc != SLIMPIPE_OK) return rc;
  if (!k_rows || !v_rows) return SLIMPIPE_EINVAL_NULL;
  rc = check_operands(k_codes, k_scales, v_codes, v_scales);
  if (rc == SLIMPIPE_OK) rc = check_cache(p, block_len);
  if (rc != SLIMPIPE_OK) return rc;
  if (!aligned16(k_rows) || !aligned16(v_rows)) return SLIMPIPE_EINVAL_ALIGN;
  if (p->kv_begin == p->kv_end) return SLIMPIPE_OK;
  if (!rows_fit(p, p->kv_end - p->kv_begin)) return SLIMPIPE_EINVAL_SHAPE;
  Kv8CopyArgs a;
  memset(&a, 0, sizeof(a));
  a.cache = cache_of(p, block_len, k_codes, k_scales, v_codes, v_scales);
  a.k_dst = static_cast<__bf16*>(k_rows);
  a.v_dst = static_cast<__bf16*>(v_rows);
  a.batch = p->batch; a.rows = p->kv_end - p->kv_begin; a.position = p->kv_begin;
  a.x_stride_b = p->o_stride_b; a.x_stride_s = p->o_stride_s; a.x_stride_h = p->o_stride_h;
  return status(launch_kv8_load(a, p->head_dim, static_cast<hipStream_t>(hip_stream)));
}

int slimpipe_attn_kv8_workspace_bytes(const slimpipe_attn_params* p, int32_t block_len, size_t* bytes) {
  if (!bytes) return SLIMPIPE_EINVAL_NULL;
  int rc = slimpipe_attn_validate(p, 0);
  if (rc == SLIMPIPE_OK) rc = check_cache(p, block_len);
  if (rc != SLIMPIPE_OK) return rc;
  *bytes = bytes_of(p, plan_of(p));
  if (copies(p)) {
    const slimpipe_attn_params c = copy_params(p);
    size_t attention = 0;
    rc = slimpipe_attn_workspace_bytes(&c, 0, &attention);
    if (rc == SLIMPIPE_OK && *bytes < 2 * copy_bytes(p) + attention) *bytes = 2 * copy_bytes(p) + attention;
  }
  return rc;
}

int slimpipe_attn_kv8_call_path(const slimpipe_attn_params* p, int32_t block_len, size_t workspace_bytes, slimpipe_kv8_call_path* out) {
  if (!p || !out) return SLIMPIPE_EINVAL_NULL;
  int rc = slimpipe_attn_validate(p, 0);
  if (rc == SLIMPIPE_OK) rc = check_cache(p, block_len);
  if (rc != SLIMPIPE_OK) return rc;
  const Kv8Path path = path_within(p, workspace_bytes);
  if (path.plan.parts < 1) return SLIMPIPE_EWORKSPACE;
  if (path.copy) {
    const slimpipe_attn_params c = copy_params(p);
    slimpipe_call_path dense;
    rc = slimpipe_attn_call_path(&c, 0, 1, workspace_bytes - 2 * copy_bytes(p), &dense);
    if (rc == SLIMPIPE_OK) *out = {1, dense.ranges, 0};
    return rc;
  }
  *out = {0, path.plan.parts, path.plan.kernel == Kv8Kernel::few ? kKv8FewRows : path.plan.kernel == Kv8Kernel::four_waves ? 128 : 256};
  return SLIMPIPE_OK;
}

int slimpipe_attn_fwd_kv8(const slimpipe_attn_params* p, int32_t block_len, const void* q_slice, const void* k_codes, const void* k_scales,
                          const void* v_codes, const void* v_scales, void* out, float* lse, void* workspace, size_t workspace_bytes, void* hip_stream) {
  int rc = slimpipe_attn_validate(p, 0);
  if (rc != SLIMPIPE_OK) return rc;
  if (!q_slice || !out || !lse) return SLIMPIPE_EINVAL_NULL;
  rc = check_operands(k_codes, k_scales, v_codes, v_scales);
  if (rc == SLIMPIPE_OK) rc = check_cache(p, block_len);
  if (rc != SLIMPIPE_OK) return rc;
  if (!aligned16(q_slice) || !aligned16(out) || !aligned4(lse)) return SLIMPIPE_EINVAL_ALIGN;
  if (!aligned16(workspace)) return SLIMPIPE_EINVAL_ALIGN;
  if (!workspace) workspace_bytes = 0;
  const Kv8Path path = path_within(p, workspace_bytes);
  const Kv8Plan& plan = path.plan;
  if (plan.parts < 1) return SLIMPIPE_EWORKSPACE;
  const Kv8Cache cache = cache_of(p, block_len, k_codes, k_scales, v_codes, v_scales);
  if (path.copy) {
    if (ensure_device_ready() != SLIMPIPE_OK) return SLIMPIPE_ELAUNCH;
    return fwd_by_copy(p, cache, q_slice, out, lse, static_cast<char*>(workspace), workspace_bytes, hip_stream);
  }
  Kv8Args a;
  memset(&a, 0, sizeof(a));
  a.q = static_cast<const __bf16*>(q_slice);
  a.cache = cache;
  a.out = out;
  a.lse = lse;
  a.batch = p->batch; a.s_q = p->s_q; a.n_q_heads = p->n_q_heads; a.group = p->n_q_heads / p->n_kv_heads;
  a.causal = p->causal; a.out_f32 = p->out_dtype == SLIMPIPE_F32;
  a.q_offset = p->q_offset; a.kv_begin = p->kv_begin; a.kv_end = seen_end(p, p->kv_begin, p->kv_end);
  a.scale_log2e = p->scale * 1.4426950408889634f;
  a.q_stride_b = p->q_stride_b; a.q_stride_s = p->q_stride_s; a.q_stride_h = p->q_stride_h;
  a.o_stride_b = p->o_stride_b; a.o_stride_s = p->o_stride_s; a.o_stride_h = p->o_stride_h;
  a.n_parts = plan.parts;
  a.part_keys = plan.part_keys;
  if (plan.parts > 1) {
    a.part_out = static_cast<float*>(workspace);
    a.part_lse = reinterpret_cast<float*>(static_cast<char*>(workspace) + out_bytes(p, plan));
  }
  if (ensure_device_ready() != SLIMPIPE_OK) return SLIMPIPE_ELAUNCH;
  hipStream_t st = static_cast<hipStream_t>(hip_stream);
  if (launch_kv8_fwd(a, p->head_dim, plan.kernel, st) != hipSuccess) return SLIMPIPE_ELAUNCH;
  if (plan.parts <= 1) return SLIMPIPE_OK;
  PartMergeArgs m;
  m.part_out = a.part_out; m.part_f32 = 1; m.part_scale = nullptr; m.part_lse = a.part_lse; m.parts = plan.parts; m.s_q = p->s_q; m.n_q_heads = p->n_q_heads; m.out_f32 = a.out_f32;
  m.rows = (int64_t)p->batch * p->n_q_heads * p->s_q;
  m.out = out; m.lse = lse;
  m.o_stride_b = p->o_stride_b; m.o_stride_s = p->o_stride_s; m.o_stride_h = p->o_stride_h;
  return status(launch_part_merge(m, p->head_dim, st));
}

int slimpipe_attn_kv8_weights_workspace_bytes(const slimpipe_attn_params* p, int32_t block_len, size_t* bytes) {
  if (!bytes) return SLIMPIPE_EINVAL_NULL;
  int rc = slimpipe_attn_validate(p, 0);
  if (rc == SLIMPIPE_OK) rc = check_cache(p, block_len);
  if (rc == SLIMPIPE_OK) rc = check_weights(p);
  if (rc != SLIMPIPE_OK) return rc;
  *bytes = weight_bytes_of(p, weight_plan_of(p));
  return SLIMPIPE_OK;
}

int slimpipe_attn_kv8_weights(const slimpipe_attn_params* p, int32_t block_len, const void* q_slice, const void* k_codes, const void* k_scales, const float* lse,
                              const float* previous, float decay, float* weights, void* workspace, size_t workspace_bytes, void* hip_stream) {
  int rc = slimpipe_attn_validate(p, 0);
  if (rc != SLIMPIPE_OK) return rc;
  if (!q_slice || !lse || !weights) return SLIMPIPE_EINVAL_NULL;
  rc = check_operands(k_codes, k_scales, k_codes, k_scales);
  if (rc == SLIMPIPE_OK) rc = check_cache(p, block_len);
  if (rc == SLIMPIPE_OK) rc = check_weights(p);
  if (rc != SLIMPIPE_OK) return rc;
  if (!isfinite(decay)) return SLIMPIPE_EINVAL_SHAPE;
  if (!aligned16(q_slice) || !aligned4(lse) || !aligned4(previous) || !aligned4(weights)) return SLIMPIPE_EINVAL_ALIGN;
  const Kv8WeightPlan plan = weight_plan_of(p);
  const size_t need = weight_bytes_of(p, plan);
  if (workspace_bytes < need || (need > 0 && !workspace)) return SLIMPIPE_EWORKSPACE;
  if (!aligned16(workspace)) return SLIMPIPE_EINVAL_ALIGN;
  if (p->kv_begin == p->kv_end) return SLIMPIPE_OK;
  Kv8WeightArgs a;
  memset(&a, 0, sizeof(a));
  a.q = static_cast<const __bf16*>(q_slice);
  a.cache = cache_of(p, block_len, k_codes, k_scales, nullptr, nullptr);
  a.lse = lse; a.previous = previous; a.weights = weights; a.decay = decay;
  a.batch = p->batch; a.s_q = p->s_q; a.n_q_heads = p->n_q_heads; a.group = p->n_q_heads / p->n_kv_heads; a.causal = p->causal;
  a.capacity = p->kv_capacity; a.q_offset = p->q_offset; a.kv_begin = p->kv_begin; a.kv_end = p->kv_end;
  a.scale_log2e = p->scale * 1.4426950408889634f;
  a.q_stride_b = p->q_stride_b; a.q_stride_s = p->q_stride_s; a.q_stride_h = p->q_stride_h;
  a.n_parts = plan.parts; a.part_keys = plan.part_keys;
  a.part = static_cast<float*>(workspace);
  if (ensure_device_ready() != SLIMPIPE_OK) return SLIMPIPE_ELAUNCH;
  return status(launch_kv8_weights(a, p->head_dim, plan.few, static_cast<hipStream_t>(hip_stream)));
}

int slimpipe_attn_kv8_keep_workspace_bytes(int32_t planes, int64_t rows, int64_t keep, size_t* bytes) {
  if (!bytes) return SLIMPIPE_EINVAL_NULL;
  const int rc = check_keep(planes, rows, rows, keep, 0);
  if (rc == SLIMPIPE_OK) *bytes = keep_bytes_of(planes, keep_plan_of(rows));
  return rc;
}

int slimpipe_attn_kv8_keep(const float* weights, int32_t planes, int64_t capacity, int64_t rows, int64_t keep, int64_t recent, int32_t* index,
                           void* workspace, size_t workspace_bytes, void* hip_stream) {
  if (!weights || !index) return SLIMPIPE_EINVAL_NULL;
  const int rc = check_keep(planes, capacity, rows, keep, recent);
  if (rc != SLIMPIPE_OK) return rc;
  if (!aligned4(weights) || !aligned4(index)) return SLIMPIPE_EINVAL_ALIGN;
  const KeepPlan plan = keep_plan_of(rows);
  const size_t need = keep_bytes_of(planes, plan);
  if (workspace_bytes < need || (need > 0 && !workspace)) return SLIMPIPE_EWORKSPACE;
  if (!aligned16(workspace)) return SLIMPIPE_EINVAL_ALIGN;
  Kv8KeepArgs a;
  a.chunks = plan.chunks; a.chunk = plan.chunk; a.work = static_cast<uint32_t*>(workspace);
  a.weights = weights; a.index = index; a.capacity = capacity;
  a.planes = planes; a.rows = (int32_t)rows; a.keep = (int32_t)keep; a.recent = (int32_t)recent;
  return status(launch_kv8_keep(a, static_cast<hipStream_t>(hip_stream)));
}

int slimpipe_attn_kv8_gather(const slimpipe_attn_params* p, int32_t block_len, const int32_t* index, int64_t keep, const void* k_codes, const void* k_scales,
                             const void* v_codes, const void* v_scales, const float* weights, const slimpipe_attn_params* to, void* to_k_codes,
                             void* to_k_scales, void* to_v_codes, void* to_v_scales, float* kept_weights, void* hip_stream) {
  int rc = slimpipe_attn_validate(p, 0);
  if (rc == SLIMPIPE_OK) rc = slimpipe_attn_validate(to, 0);
  if (rc != SLIMPIPE_OK) return rc;
  if (!index || (weights == nullptr) != (kept_weights == nullptr)) return SLIMPIPE_EINVAL_NULL;
  rc = check_operands(k_codes, k_scales, v_codes, v_scales);
  if (rc == SLIMPIPE_OK) rc = check_operands(to_k_codes, to_k_scales, to_v_codes, to_v_scales);
  if (rc == SLIMPIPE_OK) rc = check_cache(p, block_len);
  if (rc == SLIMPIPE_OK) rc = check_cache(to, block_len);
  if (rc != SLIMPIPE_OK) return rc;
  if (p->batch != to->batch || p->n_kv_heads != to->n_kv_heads || p->head_dim != to->head_dim) return SLIMPIPE_EINVAL_SHAPE;
  if (keep < 0 || keep > to->kv_capacity) return SLIMPIPE_EINVAL_RANGE;
  if (!rows_fit(p, keep)) return SLIMPIPE_EINVAL_SHAPE;
  if (!aligned4(index) || !aligned4(weights) || !aligned4(kept_weights)) return SLIMPIPE_EINVAL_ALIGN;
  if (keep == 0) return SLIMPIPE_OK;
  Kv8GatherArgs a;
  memset(&a, 0, sizeof(a));
  a.from = cache_of(p, block_len, k_codes, k_scales, v_codes, v_scales);
  a.to = cache_of(to, block_len, to_k_codes, to_k_scales, to_v_codes, to_v_scales);
  a.index = index; a.weights = weights; a.kept_weights = kept_weights;
  a.weights_stride = p->kv_capacity; a.kept_weights_stride = to->kv_capacity;
  a.from_rows = p->kv_capacity;
  a.batch = p->batch; a.keep = (int32_t)keep;
  if (overlap(a, p->head_dim)) return SLIMPIPE_EINVAL_RANGE;
  return status(launch_kv8_gather(a, p->head_dim, static_cast<hipStream_t>(hip_stream)));
}

}  // extern "C"
