// The fold of the partial results of a row that several workgroups computed over disjoint keys.
#include "kv4.hpp"
#include "tile_common.hpp"

namespace slimpipe {

// D / 8 lanes hold a row; GROUPS such sets share out its parts (1: sixteen rows a workgroup for D = 128, many rows; 16: few rows of many
// parts, where the chain of dependent loads of one set would be the time).  Sums in float32, parts in order, sets in order.
template <int D, int GROUPS>
__global__ __launch_bounds__(256) void part_merge_kernel(const PartMergeArgs a) {
  constexpr int NC = D / 8, SETS = 256 / NC, ROWS = SETS / GROUPS, STRIDE = GROUPS;
  __shared__ float acc_s[GROUPS > 1 ? SETS : 1][D + 4], m_s[SETS], l_s[SETS];
  const int set = threadIdx.x / NC, c = threadIdx.x % NC, g = set / ROWS;
  const int64_t row = (int64_t)blockIdx.x * ROWS + set % ROWS;
  const bool mine = row < a.rows;
  const int64_t first = (mine ? row : 0) * a.parts;
  const float* lp = a.part_lse + first;
  const float* op = a.part_out + first * D + c * 8;
  float m = -INFINITY, l = 0.f;
  f32x4 x0 = {0, 0, 0, 0}, x1 = {0, 0, 0, 0};
  if (mine) {
    for (int s = g; s < a.parts; s += STRIDE) m = fmaxf(m, lp[s]);
    if (m != -INFINITY)
#pragma unroll 4
      for (int s = g; s < a.parts; s += STRIDE) {
        const float ls = lp[s];
        if (ls == -INFINITY) continue;
        const float w = exp2_fast((ls - m) * kLog2e);
        l += w;
        x0 += w * *reinterpret_cast<const f32x4*>(op + (int64_t)s * D);
        x1 += w * *reinterpret_cast<const f32x4*>(op + (int64_t)s * D + 4);
      }
  }
  if constexpr (GROUPS > 1) {
    if (c == 0) { m_s[set] = m; l_s[set] = l; }
    *reinterpret_cast<f32x4*>(&acc_s[set][c * 8]) = x0;
    *reinterpret_cast<f32x4*>(&acc_s[set][c * 8 + 4]) = x1;
    __syncthreads();
    if (g != 0) return;
    const int r = set;                               // (sets 0 .. ROWS - 1 are the rows)
    float mx = -INFINITY;
    for (int i = 0; i < GROUPS; ++i) mx = fmaxf(mx, m_s[r + i * ROWS]);
    x0 = x1 = f32x4{0, 0, 0, 0};
    l = 0.f;
    m = mx;
    if (mx != -INFINITY)
      for (int i = 0; i < GROUPS; ++i) {
        const int o = r + i * ROWS;
        const float w = exp2_fast((m_s[o] - mx) * kLog2e);
        l += w * l_s[o];
        x0 += w * *reinterpret_cast<const f32x4*>(&acc_s[o][c * 8]);
        x1 += w * *reinterpret_cast<const f32x4*>(&acc_s[o][c * 8 + 4]);
      }
  }
  if (!mine) return;
  const float inv = l > 0.f ? 1.0f / l : 0.f;
  const int64_t bh = row / a.s_q, b = bh / a.n_q_heads;
  const int64_t to = b * a.o_stride_b + (row - bh * a.s_q) * a.o_stride_s + (bh - b * a.n_q_heads) * a.o_stride_h + c * 8;
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
  if (c == 0) a.lse[row] = m == -INFINITY ? -INFINITY : m + __builtin_log2f(l) * kLn2;
}

template <int D, int GROUPS>
static void launch_t(const PartMergeArgs& a, hipStream_t st) {
  constexpr int ROWS = 256 / (D / 8) / GROUPS;
  hipLaunchKernelGGL((part_merge_kernel<D, GROUPS>), dim3((unsigned)((a.rows + ROWS - 1) / ROWS)), dim3(256), 0, st, a);
}
hipError_t launch_part_merge(const PartMergeArgs& a, int head_dim, hipStream_t st) {
  const bool spread = a.rows <= 4096 && a.parts > 2;
  if (head_dim == 128) spread ? launch_t<128, 16>(a, st) : launch_t<128, 1>(a, st);
  else spread ? launch_t<64, 16>(a, st) : launch_t<64, 1>(a, st);
  return hipGetLastError();
}

}  // namespace slimpipe
