// Conversions of the cache in 8 bits, shared by its kernels.
#pragma once
#include "kv8.hpp"
#include "tile_common.hpp"

namespace slimpipe {

typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));

constexpr uint32_t kKv8LeastScale = 17;      // 2^-110
SP_DEV float kv8_scale(uint32_t byte) { return __uint_as_float(byte << 23); }
SP_DEV int64_t kv8_scale_at(const Kv8Cache& c, int64_t b, int64_t row, int h) { return (b * c.blocks + (row >> c.shift)) * c.n_kv_heads + h; }

// 8 elements (8 bytes of codes) -> bf16, and back
SP_DEV bf16x8 kv8_values(uint32_t lo, uint32_t hi, float scale) {
  const bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, scale, false), b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, scale, true);
  const bf16x2 c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, scale, false), d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, scale, true);
  bf16x8 r;
  r[0] = a[0]; r[1] = a[1]; r[2] = b[0]; r[3] = b[1]; r[4] = c[0]; r[5] = c[1]; r[6] = d[0]; r[7] = d[1];
  return r;
}
SP_DEV u32x2 kv8_codes(bf16x8 x, float scale) {
  typedef short s16x2 __attribute__((ext_vector_type(2)));
  s16x2 lo = {0, 0}, hi = {0, 0};
  lo = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(lo, __builtin_shufflevector(x, x, 0, 1), scale, false);
  lo = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(lo, __builtin_shufflevector(x, x, 2, 3), scale, true);
  hi = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(hi, __builtin_shufflevector(x, x, 4, 5), scale, false);
  hi = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(hi, __builtin_shufflevector(x, x, 6, 7), scale, true);
  return u32x2{__builtin_bit_cast(uint32_t, lo), __builtin_bit_cast(uint32_t, hi)};
}

}  // namespace slimpipe
