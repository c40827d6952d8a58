// The fold of the partial results of a row that several workgroups computed over disjoint keys.
#include "kv4.hpp"
#include "tile_common.hpp"

namespace slimpipe {

// Writes 8 elements of a row's result, and its lse.
SP_DEV void put_result(const PartMergeArgs& a, int64_t row, int d, f32x4 x0, f32x4 x1, float m, float l) {
  const float inv = l == 0.f ? 0.f : 1.0f / l;      // (NaN, from a NaN among what the row saw: stays)
  const int64_t bh = row / a.s_q, b = bh / a.n_q_heads;
  const int64_t to = b * a.o_stride_b + (row - bh * a.s_q) * a.o_stride_s + (bh - b * a.n_q_heads) * a.o_stride_h + d;
  x0 *= inv;
  x1 *= inv;
  if (a.out_f32) {
    f32x4* dst = reinterpret_cast<f32x4*>(static_cast<float*>(a.out) + to);
    dst[0] = x0;
    dst[1] = x1;
  } else {
    const bf16x4 lo = __builtin_convertvector(x0, bf16x4), hi = __builtin_convertvector(x1, bf16x4);
    *reinterpret_cast<bf16x8*>(static_cast<bf16_t*>(a.out) + to) = __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
  }
  if (d == 0) a.lse[row] = l == 0.f ? -INFINITY : m + __builtin_log2f(l) * kLn2;
}
// Adds N parts (s, s + step, ..) of 8 elements of a row, relative to the maximum m of all lse.  Their loads are under way at once (calls of 1200 rows of 45 parts 43.5 us, one by
// one 57.7; of 1500 of 39 50 and 61.6; of 4000 of 15 51.5 and 54.3); of those that add nothing there are none (sparse attention of 8192 rows of 8 heads with one of 16
// slots filled 60 us, with their loads 101; of a whole first slice of 16 blocks 223 and 250).
template <int D, bool F32, int N>
SP_DEV void add_parts(const PartMergeArgs& a, int64_t row, int d, int s, int step, f32x4& x0, f32x4& x1, float m, float& l) {
  typedef std::conditional_t<F32, float, _Float16> part_t;
  typedef part_t part8 __attribute__((ext_vector_type(8)));
  float lse[N], scale[N];
  part8 y[N];
#pragma unroll
  for (int i = 0; i < N; ++i) lse[i] = a.part_lse[row * a.parts + s + i * step];
#pragma unroll
  for (int i = 0; i < N; ++i) {
    if (lse[i] == -INFINITY) continue;
    const int64_t part = row * a.parts + s + i * step;
    y[i] = *reinterpret_cast<const part8*>(static_cast<const part_t*>(a.part_out) + part * D + d);
    if constexpr (!F32) scale[i] = a.part_scale[part];
  }
#pragma unroll
  for (int i = 0; i < N; ++i) {
    if (lse[i] == -INFINITY) continue;
    float w = exp2_fast((lse[i] - m) * kLog2e);      // (m is -inf only where all are that or NaN, which gives NaN)
    l += w;
    if constexpr (!F32) w *= scale[i];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      x0[e] += w * (float)y[i][e];
      x1[e] += w * (float)y[i][4 + e];
    }
  }
}
// Parts first, first + step, .. of 8 elements of a row: maximum of their lse, sum of weights, weighted sum.
template <int D, bool F32>
SP_DEV void fold_parts(const PartMergeArgs& a, int64_t row, int d, int first, int step, f32x4& x0, f32x4& x1, float& m, float& l) {
  const float* lp = a.part_lse + row * a.parts;
  m = -INFINITY;
  l = 0.f;
  x0 = x1 = f32x4{0, 0, 0, 0};
#pragma unroll 4
  for (int s = first; s < a.parts; s += step) m = fmaxf(m, lp[s]);
  int s = first;
  for (; s + 7 * step < a.parts; s += 8 * step) add_parts<D, F32, 8>(a, row, d, s, step, x0, x1, m, l);
  if (s + 3 * step < a.parts) { add_parts<D, F32, 4>(a, row, d, s, step, x0, x1, m, l); s += 4 * step; }
  if (s + step < a.parts) { add_parts<D, F32, 2>(a, row, d, s, step, x0, x1, m, l); s += 2 * step; }
  if (s < a.parts) add_parts<D, F32, 1>(a, row, d, s, step, x0, x1, m, l);
}

// Many rows: D / 8 lanes a row.  Bound by the bytes: 65536 rows of 8 parts of 128 in 24 us (6.3 TB/s: they have just been written).
template <int D, bool F32>
__global__ __launch_bounds__(256) void part_merge_kernel(const PartMergeArgs a) {
  constexpr int NC = D / 8;
  const int64_t gid = (int64_t)blockIdx.x * 256 + threadIdx.x, row = gid / NC;
  const int d = (int)(gid - row * NC) * 8;
  if (row >= a.rows) return;
  f32x4 x0, x1;
  float m, l;
  fold_parts<D, F32>(a, row, d, 0, 1, x0, x1, m, l);
  put_result(a, row, d, x0, x1, m, l);
}

// Few rows: a workgroup has 32 elements of one row, and its 64 sets of four lanes share out the parts, where the chain of dependent loads of
// one set would be the time.  Sets of a wave are folded by exchanges, the waves through LDS, always in the same order.
template <int D, bool F32>
__global__ __launch_bounds__(256) void part_merge_few_kernel(const PartMergeArgs a) {
  __shared__ float acc_s[4][32], m_s[4], l_s[4];
  const int64_t row = blockIdx.x;
  const int set = threadIdx.x / 4, c = threadIdx.x % 4, d = blockIdx.y * 32 + c * 8, wave = threadIdx.x >> 6;
  f32x4 x0, x1;
  float m, l;
  fold_parts<D, F32>(a, row, d, set, 64, x0, x1, m, l);
#pragma unroll
  for (int w = 4; w < 64; w <<= 1) {
    const float mo = __shfl_xor(m, w, 64), lo = __shfl_xor(l, w, 64), mx = fmaxf(m, mo), me = mx == -INFINITY ? 0.f : mx;
    const float f = exp2_fast((m - me) * kLog2e), fo = exp2_fast((mo - me) * kLog2e);
    l = l * f + lo * fo;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      x0[e] = x0[e] * f + __shfl_xor(x0[e], w, 64) * fo;
      x1[e] = x1[e] * f + __shfl_xor(x1[e], w, 64) * fo;
    }
    m = mx;
  }
  if ((threadIdx.x & 63) < 4) {
    *reinterpret_cast<f32x4*>(&acc_s[wave][c * 8]) = x0;
    *reinterpret_cast<f32x4*>(&acc_s[wave][c * 8 + 4]) = x1;
    if (c == 0) { m_s[wave] = m; l_s[wave] = l; }
  }
  __syncthreads();
  if (threadIdx.x >= 4) return;
  m = fmaxf(fmaxf(m_s[0], m_s[1]), fmaxf(m_s[2], m_s[3]));
  l = 0.f;
  x0 = x1 = f32x4{0, 0, 0, 0};
  const float me = m == -INFINITY ? 0.f : m;
#pragma unroll
  for (int w = 0; w < 4; ++w) {
    const float f = exp2_fast((m_s[w] - me) * kLog2e);
    l += f * l_s[w];
    x0 += f * *reinterpret_cast<const f32x4*>(&acc_s[w][c * 8]);
    x1 += f * *reinterpret_cast<const f32x4*>(&acc_s[w][c * 8 + 4]);
  }
  put_result(a, row, d, x0, x1, m, l);
}

// Few rows: us of a call with the few-row kernel and without, 8 rows of 512 parts 36 and 228; 256 rows of 128 29 and 84, 1024 of 64 40 and 59; of 16 parts
// 256 rows 37 and 43, 1024 44 and 44, 2048 57 and 50; of four parts no gain at 256 rows (13.4 both), 38 and 32 at 1024.
template <int D, bool F32>
static void launch_merge_t(const PartMergeArgs& a, hipStream_t st) {
  if (a.rows <= 1024 && a.parts > 4) hipLaunchKernelGGL((part_merge_few_kernel<D, F32>), dim3((unsigned)a.rows, D / 32), dim3(256), 0, st, a);
  else hipLaunchKernelGGL((part_merge_kernel<D, F32>), dim3((unsigned)((a.rows * (D / 8) + 255) / 256)), dim3(256), 0, st, a);
}
hipError_t launch_part_merge(const PartMergeArgs& a, int head_dim, hipStream_t st) {
  if (head_dim == 128) a.part_f32 ? launch_merge_t<128, true>(a, st) : launch_merge_t<128, false>(a, st);
  else a.part_f32 ? launch_merge_t<64, true>(a, st) : launch_merge_t<64, false>(a, st);
  return hipGetLastError();
}

}  // namespace slimpipe
