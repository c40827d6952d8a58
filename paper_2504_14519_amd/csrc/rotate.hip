// Norm of every head of queries and keys, and the rotation of pairs of its elements by the row's position, in one pass; and the gradient.
//
//   n = x r, r = (mean x^2 + eps)^(-1/2);   y = n w;   (y_a, y_b) -> (y_a cos - y_b sin, y_b cos + y_a sin), angle = position * frequency
//   backward: dy = the result's gradient turned back;  dw = sum over rows and heads of dy n;  g = dy w;  dx = r (g - n mean(g n))
//
// Bound by the bytes: x in, result out.  A lane has two chunks of 8 elements that hold whole pairs, so that nothing but the two sums over a head
// crosses lanes, head_dim / 16 lanes have a head of a row, and they walk heads of that row: the angles are made once a row.  An angle is made in 64 bits as a
// fraction of a turn (position * frequency passes 2^20, where 32 bits leave an error of a sixteenth), its sine and cosine in 32.
#include "rotate.hpp"
#include "tile_common.hpp"

namespace slimpipe {

// Sum over the lanes of a head, in all of them: 4 or 8 consecutive lanes.
template <int LANES>
SP_DEV float head_sum(float v) {
  auto add = [&](auto ctrl) { v += __uint_as_float(__builtin_amdgcn_update_dpp(0, __float_as_uint(v), decltype(ctrl)::value, 0xf, 0xf, true)); };
  add(std::integral_constant<int, 0xb1>{});                            // lane ^ 1
  add(std::integral_constant<int, 0x4e>{});                            // lane ^ 2
  if constexpr (LANES == 8) add(std::integral_constant<int, 0x141>{});  // 7 - lane of eight: the other four, whose sums are equal by now
  return v;
}

// position * frequency / 2 pi less the whole turns, in [-1/2, 1/2].  Products keep what their rounding leaves behind: one 64-bit product alone
// is off by position * frequency * 2^-53, which shows in a bf16 result from positions of 2^38 on.
SP_DEV float turn_of(int64_t position, double frequency) {
  constexpr double kHigh = 0.15915494309189533577, kLow = -9.839338337591243e-18;      // 1 / 2 pi
  const double t = (double)position;
  double per = frequency * kHigh;
  asm("" : "+v"(per));                                       // (or the remainder below might be taken to be 0)
  const double per_low = __builtin_fma(frequency, kHigh, -per) + frequency * kLow;
  double turns = t * per;
  asm("" : "+v"(turns));
  const double low = __builtin_fma(t, per, -turns) + t * per_low;
  return (float)((turns - __builtin_rint(turns)) + low);
}

// What a lane does for its row: which chunks it has, and the cosines and sines of its 8 pairs.
template <int D, bool INTERLEAVED>
struct Turn {
  static constexpr int LANES = D / 16;
  int ca, cb;                  // elements 8 ca .. 8 ca + 7 and 8 cb ..
  bool turns;                  // of the rotated part (all or nothing: rotate_dim is a multiple of 16)
  float c[8], s[8];
  SP_DEV void init(const RotateArgs& a, int lane) {
    const int l = lane % LANES, n = a.rotate_dim / 16;
    turns = l < n;
    ca = INTERLEAVED ? 2 * l : turns ? l : 2 * l;
    cb = INTERLEAVED ? 2 * l + 1 : turns ? l + n : 2 * l + 1;
  }
  SP_DEV void angles(const RotateArgs& a, int lane, int64_t position) {
    if (!turns) return;
    const double* f = a.frequency + 8 * (lane % LANES);
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const float part = turn_of(position, f[j]);
      c[j] = __builtin_amdgcn_cosf(part);      // (of 2 pi times its operand)
      s[j] = __builtin_amdgcn_sinf(part);
    }
  }
  // x: the elements of both chunks; BACK: by the negative angle
  template <bool BACK>
  SP_DEV void apply(float (&x)[16]) const {
    if (!turns) return;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      float& p = x[INTERLEAVED ? 2 * j : j];
      float& q = x[INTERLEAVED ? 2 * j + 1 : 8 + j];
      const float p0 = p, sj = BACK ? -s[j] : s[j];
      p = p0 * c[j] - q * sj;
      q = q * c[j] + p0 * sj;
    }
  }
};

SP_DEV void widen(const bf16x8& lo, const bf16x8& hi, float (&x)[16]) {
#pragma unroll
  for (int j = 0; j < 8; ++j) { x[j] = (float)lo[j]; x[8 + j] = (float)hi[j]; }
}
SP_DEV bf16x8 narrow(const float* x) {
  const f32x4 a = {x[0], x[1], x[2], x[3]}, b = {x[4], x[5], x[6], x[7]};
  return __builtin_shufflevector(__builtin_convertvector(a, bf16x4), __builtin_convertvector(b, bf16x4), 0, 1, 2, 3, 4, 5, 6, 7);
}
template <int D, bool I>
SP_DEV void load_weight(const RotateSide& s, const Turn<D, I>& t, float (&w)[16]) {
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    w[j] = s.weight ? s.weight[8 * t.ca + j] : 1.0f;
    w[8 + j] = s.weight ? s.weight[8 * t.cb + j] : 1.0f;
  }
}

constexpr int kRotateAhead = 4;      // heads whose loads are under way together

template <int D, bool INTERLEAVED>
__global__ __launch_bounds__(256) void rotate_fwd_kernel(const RotateArgs a) {
  constexpr int LANES = D / 16, ROWS = 64 / LANES;
  const int lane = threadIdx.x & 63;
  const int64_t w = (int64_t)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int set = __builtin_amdgcn_readfirstlane((int)(w / a.row_blocks));
  if (set >= a.head_sets) return;
  const int64_t row = (w - (int64_t)set * a.row_blocks) * ROWS + lane / LANES;
  if (row >= a.total_rows) return;                                    // (whole heads' lanes leave together)
  const int64_t b = row / a.rows, r = row - b * a.rows;
  Turn<D, INTERLEAVED> t;
  t.init(a, lane);
  t.angles(a, lane, a.positions ? a.positions[row] : a.position + r);
  const int first = set * a.heads_wave, last = first + a.heads_wave;
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const RotateSide& s = a.side[i];
    const int base = i == 0 ? 0 : a.side[0].heads;
    int h = first > base ? first - base : 0;
    const int end = last - base < s.heads ? last - base : s.heads;
    if (h >= end) continue;
    float wt[16];
    load_weight(s, t, wt);
    const bf16_t* x = s.x + b * s.stride_b + r * s.stride_s;
    bf16_t* out = s.out + b * s.out_stride_b + r * s.out_stride_s;
    for (; h < end; h += kRotateAhead) {
      bf16x8 lo[kRotateAhead], hi[kRotateAhead];
#pragma unroll
      for (int u = 0; u < kRotateAhead; ++u) {
        const bf16_t* p = x + (int64_t)(h + u < end ? h + u : end - 1) * s.stride_h;
        lo[u] = *reinterpret_cast<const bf16x8*>(p + 8 * t.ca);
        hi[u] = *reinterpret_cast<const bf16x8*>(p + 8 * t.cb);
      }
#pragma unroll
      for (int u = 0; u < kRotateAhead; ++u) {
        float v[16], sum = 0.f;
        widen(lo[u], hi[u], v);
#pragma unroll
        for (int j = 0; j < 16; ++j) sum = __builtin_fmaf(v[j], v[j], sum);
        const float inv = __builtin_amdgcn_rsqf(head_sum<LANES>(sum) * (1.0f / D) + a.eps);
#pragma unroll
        for (int j = 0; j < 16; ++j) v[j] *= inv * wt[j];
        t.template apply<false>(v);
        if (h + u < end) {
          bf16_t* p = out + (int64_t)(h + u) * s.out_stride_h;
          *reinterpret_cast<bf16x8*>(p + 8 * t.ca) = narrow(v);
          *reinterpret_cast<bf16x8*>(p + 8 * t.cb) = narrow(v + 8);
        }
      }
    }
  }
}

// The gradient.  The weights' gradients are summed in the lanes over the rows and heads of a wave, over the waves of a workgroup in LDS, and over the
// workgroups by rotate_weights_kernel, all in a fixed order.
template <int D, bool INTERLEAVED, bool DOUT_F32>
SP_DEV void rotate_back_heads(const RotateArgs& a, const RotateSide& s, const Turn<D, INTERLEAVED>& t, int64_t b, int64_t r, int h, int end, float (&dw)[16]) {
  constexpr int LANES = D / 16, AHEAD = DOUT_F32 ? 2 : kRotateAhead;
  typedef std::conditional_t<DOUT_F32, float, bf16_t> dout_t;
  typedef dout_t dout8 __attribute__((ext_vector_type(8)));
  float wt[16];
  load_weight(s, t, wt);
  const bf16_t* x = s.x + b * s.stride_b + r * s.stride_s;
  bf16_t* dx = s.out + b * s.stride_b + r * s.stride_s;
  const dout_t* d = static_cast<const dout_t*>(s.d_out) + b * s.out_stride_b + r * s.out_stride_s;
  for (; h < end; h += AHEAD) {
    bf16x8 lo[AHEAD], hi[AHEAD];
    dout8 dlo[AHEAD], dhi[AHEAD];
#pragma unroll
    for (int u = 0; u < AHEAD; ++u) {
      const int64_t hh = h + u < end ? h + u : end - 1;
      const bf16_t* p = x + hh * s.stride_h;
      const dout_t* e = d + hh * s.out_stride_h;
      lo[u] = *reinterpret_cast<const bf16x8*>(p + 8 * t.ca);
      hi[u] = *reinterpret_cast<const bf16x8*>(p + 8 * t.cb);
      dlo[u] = *reinterpret_cast<const dout8*>(e + 8 * t.ca);
      dhi[u] = *reinterpret_cast<const dout8*>(e + 8 * t.cb);
    }
#pragma unroll
    for (int u = 0; u < AHEAD; ++u) {
      if (h + u >= end) break;
      float y[16];
#pragma unroll
      for (int j = 0; j < 8; ++j) { y[j] = (float)dlo[u][j]; y[8 + j] = (float)dhi[u][j]; }
      float v[16], sum = 0.f, dot = 0.f;
      widen(lo[u], hi[u], v);
      t.template apply<true>(y);
#pragma unroll
      for (int j = 0; j < 16; ++j) {
        sum = __builtin_fmaf(v[j], v[j], sum);
        dot = __builtin_fmaf(v[j], y[j] * wt[j], dot);
      }
      const float inv = __builtin_amdgcn_rsqf(head_sum<LANES>(sum) * (1.0f / D) + a.eps);
      const float back = head_sum<LANES>(dot) * (1.0f / D) * inv * inv;       // mean(g n) r: what n = x r is taken away with, less one r
#pragma unroll
      for (int j = 0; j < 16; ++j) {
        dw[j] = __builtin_fmaf(y[j], v[j] * inv, dw[j]);
        v[j] = (y[j] * wt[j] - v[j] * back) * inv;
      }
      bf16_t* p = dx + (int64_t)(h + u) * s.stride_h;
      *reinterpret_cast<bf16x8*>(p + 8 * t.ca) = narrow(v);
      *reinterpret_cast<bf16x8*>(p + 8 * t.cb) = narrow(v + 8);
    }
  }
}

template <int D, bool INTERLEAVED>
__global__ __launch_bounds__(256) void rotate_bwd_kernel(const RotateArgs a) {
  constexpr int LANES = D / 16, ROWS = 64 / LANES;
  __shared__ float sums[2][4][D];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int64_t w = (int64_t)blockIdx.x * 4 + wave;
  const int set = __builtin_amdgcn_readfirstlane((int)(w / a.wave_blocks));
  Turn<D, INTERLEAVED> t;
  t.init(a, lane);
  float dw[2][16];
#pragma unroll
  for (int i = 0; i < 2; ++i)
#pragma unroll
    for (int j = 0; j < 16; ++j) dw[i][j] = 0.f;
  if (set < a.head_sets) {
    const int first = set * a.heads_wave, last = first + a.heads_wave;
    for (int64_t blk = w - (int64_t)set * a.wave_blocks; blk < a.row_blocks; blk += a.wave_blocks) {
      const int64_t row = blk * ROWS + lane / LANES;
      if (row >= a.total_rows) continue;
      const int64_t b = row / a.rows, r = row - b * a.rows;
      t.angles(a, lane, a.positions ? a.positions[row] : a.position + r);
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const RotateSide& s = a.side[i];
        const int base = i == 0 ? 0 : a.side[0].heads;
        const int h = first > base ? first - base : 0, end = last - base < s.heads ? last - base : s.heads;
        if (h >= end) continue;
        if (s.d_out_f32) rotate_back_heads<D, INTERLEAVED, true>(a, s, t, b, r, h, end, dw[i]);
        else rotate_back_heads<D, INTERLEAVED, false>(a, s, t, b, r, h, end, dw[i]);
      }
    }
  }
  if (!a.part) return;
#pragma unroll
  for (int i = 0; i < 2; ++i)
#pragma unroll
    for (int j = 0; j < 16; ++j) {
      float v = dw[i][j];
#pragma unroll
      for (int k = LANES; k < 64; k <<= 1) v += __shfl_xor(v, k, 64);
      if (lane < LANES) sums[i][wave][8 * (j < 8 ? t.ca : t.cb) + j % 8] = v;
    }
  __syncthreads();
  for (int i = threadIdx.x; i < 2 * D; i += 256) {
    const int e = i % D, side = i / D;
    a.part[((int64_t)side * a.workgroups + blockIdx.x) * D + e] = (sums[side][0][e] + sums[side][1][e]) + (sums[side][2][e] + sums[side][3][e]);
  }
}

// Sums of the workgroups: 16 elements of one side a workgroup, 16 threads an element.
template <int D>
__global__ __launch_bounds__(256) void rotate_weights_kernel(const RotateArgs a) {
  __shared__ float sums[16][16];
  const int side = blockIdx.y, e = blockIdx.x * 16 + threadIdx.x % 16, k = threadIdx.x / 16;
  if (!a.d_weight[side]) return;
  const float* p = a.part + (int64_t)side * a.workgroups * D + e;
  float v = 0.f;
#pragma unroll 8
  for (int i = k; i < a.workgroups; i += 16) v += p[(int64_t)i * D];
  sums[k][threadIdx.x % 16] = v;
  __syncthreads();
  if (k) return;
  v = a.weight_accumulate ? a.d_weight[side][e] : 0.f;
#pragma unroll
  for (int i = 0; i < 16; ++i) v += sums[i][threadIdx.x];
  a.d_weight[side][e] = v;
}

template <int D>
static hipError_t launch_fwd_t(const RotateArgs& a, hipStream_t st) {
  const dim3 grid((unsigned)((a.row_blocks * a.head_sets + 3) / 4)), block(256);
  if (a.interleaved) hipLaunchKernelGGL((rotate_fwd_kernel<D, true>), grid, block, 0, st, a);
  else hipLaunchKernelGGL((rotate_fwd_kernel<D, false>), grid, block, 0, st, a);
  return hipGetLastError();
}
hipError_t launch_rotate_fwd(const RotateArgs& a, int head_dim, hipStream_t st) { return head_dim == 128 ? launch_fwd_t<128>(a, st) : launch_fwd_t<64>(a, st); }

template <int D>
static hipError_t launch_bwd_t(const RotateArgs& a, hipStream_t st) {
  const dim3 grid((unsigned)a.workgroups), block(256);
  if (a.interleaved) hipLaunchKernelGGL((rotate_bwd_kernel<D, true>), grid, block, 0, st, a);
  else hipLaunchKernelGGL((rotate_bwd_kernel<D, false>), grid, block, 0, st, a);
  if (a.part) hipLaunchKernelGGL((rotate_weights_kernel<D>), dim3(D / 16, 2), block, 0, st, a);
  return hipGetLastError();
}
hipError_t launch_rotate_bwd(const RotateArgs& a, int head_dim, hipStream_t st) { return head_dim == 128 ? launch_bwd_t<128>(a, st) : launch_bwd_t<64>(a, st); }

}  // namespace slimpipe
