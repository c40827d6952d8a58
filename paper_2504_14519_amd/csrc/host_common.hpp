// Host helpers shared by the files that implement the C entry points (internal to the library).
#pragma once
#include <stddef.h>
#include <stdint.h>

#include "../../include/slimpipe_attn.h"
#include "kernels.hpp"

namespace slimpipe {

inline bool stride_ok(int64_t s) { return s > 0 && (s % 8) == 0; }
inline bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }
inline bool aligned4(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 3u) == 0; }

// One past the last key before `end` that any row sees (`begin` when none does).
inline int64_t seen_end(const slimpipe_attn_params* p, int64_t begin, int64_t end) {
  if (p->causal && p->q_offset + p->s_q < end) end = p->q_offset + p->s_q;
  return end > begin ? end : begin;
}

// A chunk list is legal when it covers kv_capacity rows; with more than one chunk the chunk length is a
// multiple of the dk/dv key tile (256), so that no key tile of any kernel straddles two chunks.
inline int check_chunks(const slimpipe_attn_params* p, int32_t n_chunks, int64_t chunk_len) {
  if (n_chunks < 1 || n_chunks > kMaxChunks || chunk_len < 1) return SLIMPIPE_EINVAL_SHAPE;
  if (n_chunks * chunk_len < p->kv_capacity) return SLIMPIPE_EINVAL_RANGE;
  if (n_chunks > 1 && chunk_len % dkdv_keys_per_workgroup() != 0) return SLIMPIPE_EINVAL_SHAPE;
  return SLIMPIPE_OK;
}

// Makes the current device ready for launches: SLIMPIPE_OK, or SLIMPIPE_ELAUNCH when the runtime refuses (api.hip).
int ensure_device_ready(void** scratch_ptr = nullptr);
// Compute units of the current device (256 on MI355X, also assumed when no device can be asked, so that the
// workspace queries stay pure host functions) (api.hip).
int compute_units();

}  // namespace slimpipe
