// Norm of every head of queries and keys, and the rotation of pairs of its elements by the row's position, in one pass; and the gradient.
//
//   n = x r, r = (mean x^2 + eps)^(-1/2);   y = n w;   (y_a, y_b) -> (y_a cos - y_b sin, y_b cos + y_a sin), angle = position * frequency
//   backward: dy = the result's gradient turned back;  dw = sum over rows and heads of dy n;  g = dy w;  dx = r (g - n mean(g n))
//
// Bound by the bytes: x in, result out (past the caches: a slice's results do not fit them).  A lane has two chunks of 8 elements that hold whole pairs, so that
// nothing but the two sums over a head crosses lanes, head_dim / 16 lanes have a head of a row, and a wave has a few heads of its 8 (head_dim 64: 16) rows: all of
// its loads are under way before the angles are made, which serve all of its heads.  An angle is made in 64 bits as a fraction of a turn (position * frequency
// passes 2^20, where 32 bits leave an error of a sixteenth), its sine and cosine in 32.
#include "rotate.hpp"
#include "row_tile.hpp"

namespace slimpipe {

// Sum over the lanes of a head, in all of them: 4 or 8 consecutive lanes.
template <int LANES>
SP_DEV float head_sum(float v) {
  v = add_lane<0xb1>(v);                                 // lane ^ 1
  v = add_lane<0x4e>(v);                                 // lane ^ 2
  return LANES == 8 ? add_lane<0x141>(v) : v;            // 7 - lane of eight: the other four, whose sums are equal by now
}
// Sum over the heads of a wave: the lanes with the same place in a head.
template <int LANES>
SP_DEV float rows_sum(float v) {
  if constexpr (LANES == 4) v = add_lane<0x124>(v);      // lane + 4 of sixteen
  return quarters_sum(add_lane<0x128>(v));               // lane + 8, then over the sixteens
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

// Which side, heads and rows a wave has.  Sets of heads are numbered through, those of the queries first, fastest over the workgroups: neighbours read
// the same rows.
struct RotateWave { int side, first, heads; int64_t block; };
SP_DEV RotateWave rotate_wave(const RotateArgs& a, int wave_u) {
  const int sets = a.sets[0] + a.sets[1], set = __builtin_amdgcn_readfirstlane((int)(blockIdx.x % (unsigned)sets));
  const int side = set >= a.sets[0], first = (side ? set - a.sets[0] : set) * a.heads_wave, left = a.side[side].heads - first;
  return {side, first, left < a.heads_wave ? left : a.heads_wave, (int64_t)(blockIdx.x / (unsigned)sets) * 4 + wave_u};
}

// 4096 rows of 80 heads of 128: 28 us, 168 MB at 6.1 TB/s; with results that stay in the caches 37, and the attention that reads them next
// is as fast either way.  2 heads a wave 35, 8 27, but 16384 rows of 8 query heads and a key head 18.2 and 17.4 us (4 heads: 17.0).
template <int D, bool INTERLEAVED>
__global__ __launch_bounds__(256) void rotate_fwd_kernel(const RotateArgs a) {
  constexpr int LANES = D / 16, ROWS = 64 / LANES, N = kRotateFwdHeads;
  const int lane = threadIdx.x & 63;
  const RotateWave w = rotate_wave(a, __builtin_amdgcn_readfirstlane(threadIdx.x >> 6));
  const int64_t row = w.block * ROWS + lane / LANES;
  if (row >= a.total_rows) return;                                    // (whole heads' lanes leave together)
  const RotateSide& s = a.side[w.side];
  const int64_t b = (uint32_t)row / (uint32_t)a.rows, r = row - b * a.rows;      // (less than 2^28 rows)
  Turn<D, INTERLEAVED> t;
  t.init(a, lane);
  const bf16_t* x = s.x + b * s.stride_b + r * s.stride_s + w.first * s.stride_h;
  bf16x8 lo[N], hi[N];
#pragma unroll
  for (int u = 0; u < N; ++u) {
    const bf16_t* p = x + (int64_t)(u < w.heads ? u : 0) * s.stride_h;
    lo[u] = *reinterpret_cast<const bf16x8*>(p + 8 * t.ca);
    hi[u] = *reinterpret_cast<const bf16x8*>(p + 8 * t.cb);
  }
  float wt[16];
  load_weight(s, t, wt);
  t.angles(a, lane, a.positions ? a.positions[row] : a.position + r);
  bf16_t* out = s.out + b * s.out_stride_b + r * s.out_stride_s + w.first * s.out_stride_h;
#pragma unroll
  for (int u = 0; u < N; ++u) {
    if (u >= w.heads) break;
    float v[16], sum = 0.f;
    widen(lo[u], hi[u], v);
#pragma unroll
    for (int j = 0; j < 16; ++j) sum = __builtin_fmaf(v[j], v[j], sum);
    const float inv = __builtin_amdgcn_rsqf(head_sum<LANES>(sum) * (1.0f / D) + a.eps);
#pragma unroll
    for (int j = 0; j < 16; ++j) v[j] *= inv * wt[j];
    t.template apply<false>(v);
    bf16_t* p = out + (int64_t)u * s.out_stride_h;
    __builtin_nontemporal_store(narrow(v), reinterpret_cast<bf16x8*>(p + 8 * t.ca));
    __builtin_nontemporal_store(narrow(v + 8), reinterpret_cast<bf16x8*>(p + 8 * t.cb));
  }
}

// The gradient.  The weights' gradients are summed in the lanes over the rows and heads of a wave, over the waves of a workgroup in LDS, and over the
// workgroups by rotate_weights_kernel, all in a fixed order.  16384 rows of 8 query heads and a key head of 128 (gradients in bf16 and float32): 24 us, 117 MB at
// 4.9 TB/s, and 3 to 4 for the last sums; what is left is the start of a block of rows, whose loads nothing hides but the other wave of the SIMD (loads of the next
// block ahead do not fit the registers).
template <int D, bool INTERLEAVED, bool DOUT_F32>
SP_DEV void rotate_back_rows(const RotateArgs& a, const RotateWave& w, Turn<D, INTERLEAVED>& t, int lane, float (&dw)[16]) {
  constexpr int LANES = D / 16, ROWS = 64 / LANES, N = kRotateBwdHeads;
  typedef std::conditional_t<DOUT_F32, float, bf16_t> dout_t;
  typedef dout_t dout8 __attribute__((ext_vector_type(8)));
  const RotateSide& s = a.side[w.side];
  float wt[16];
  load_weight(s, t, wt);
  for (int64_t block = w.block; block < a.row_blocks; block += a.wave_blocks) {
    const int64_t row = block * ROWS + lane / LANES;
    if (row >= a.total_rows) break;
    const int64_t b = (uint32_t)row / (uint32_t)a.rows, r = row - b * a.rows;
    const bf16_t* x = s.x + b * s.stride_b + r * s.stride_s + w.first * s.stride_h;
    const dout_t* d = static_cast<const dout_t*>(s.d_out) + b * s.out_stride_b + r * s.out_stride_s + w.first * s.out_stride_h;
    bf16x8 lo[N], hi[N];
    dout8 dlo[N], dhi[N];
#pragma unroll
    for (int u = 0; u < N; ++u) {
      const bf16_t* p = x + (int64_t)(u < w.heads ? u : 0) * s.stride_h;
      const dout_t* e = d + (int64_t)(u < w.heads ? u : 0) * s.out_stride_h;
      lo[u] = *reinterpret_cast<const bf16x8*>(p + 8 * t.ca);
      hi[u] = *reinterpret_cast<const bf16x8*>(p + 8 * t.cb);
      dlo[u] = *reinterpret_cast<const dout8*>(e + 8 * t.ca);
      dhi[u] = *reinterpret_cast<const dout8*>(e + 8 * t.cb);
    }
    t.angles(a, lane, a.positions ? a.positions[row] : a.position + r);
    bf16_t* dx = s.out + b * s.stride_b + r * s.stride_s + w.first * s.stride_h;
#pragma unroll
    for (int u = 0; u < N; ++u) {
      if (u >= w.heads) break;
      float y[16], v[16], sum = 0.f, dot = 0.f;
#pragma unroll
      for (int j = 0; j < 8; ++j) { y[j] = (float)dlo[u][j]; y[8 + j] = (float)dhi[u][j]; }
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
      bf16_t* p = dx + (int64_t)u * s.stride_h;
      __builtin_nontemporal_store(narrow(v), reinterpret_cast<bf16x8*>(p + 8 * t.ca));
      __builtin_nontemporal_store(narrow(v + 8), reinterpret_cast<bf16x8*>(p + 8 * t.cb));
    }
  }
}

template <int D, bool INTERLEAVED>
__global__ __launch_bounds__(256) void rotate_bwd_kernel(const RotateArgs a) {
  constexpr int LANES = D / 16;
  __shared__ float sums[4][D];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const RotateWave w = rotate_wave(a, wave);
  Turn<D, INTERLEAVED> t;
  t.init(a, lane);
  float dw[16];
#pragma unroll
  for (int j = 0; j < 16; ++j) dw[j] = 0.f;
  if (a.side[w.side].d_out_f32) rotate_back_rows<D, INTERLEAVED, true>(a, w, t, lane, dw);
  else rotate_back_rows<D, INTERLEAVED, false>(a, w, t, lane, dw);
  if (!a.part) return;
#pragma unroll
  for (int j = 0; j < 16; ++j) {
    const float v = rows_sum<LANES>(dw[j]);
    if (lane < LANES) sums[wave][8 * (j < 8 ? t.ca : t.cb) + j % 8] = v;
  }
  __syncthreads();
  // (sums of the queries' workgroups, then those of the keys')
  const int sets = a.sets[0] + a.sets[1], set = blockIdx.x % sets, group = blockIdx.x / sets, groups = gridDim.x / sets;
  const int64_t at = w.side ? (int64_t)groups * a.sets[0] + (int64_t)group * a.sets[1] + set - a.sets[0] : (int64_t)group * a.sets[0] + set;
  if (threadIdx.x < D) a.part[at * D + threadIdx.x] = (sums[0][threadIdx.x] + sums[1][threadIdx.x]) + (sums[2][threadIdx.x] + sums[3][threadIdx.x]);
}

// Sums of the workgroups: 16 elements of one side a workgroup, 64 threads an element.
template <int D>
__global__ __launch_bounds__(1024) void rotate_weights_kernel(const RotateArgs a) {
  __shared__ float sums[64][17];
  const int side = blockIdx.y, c = threadIdx.x % 16, e = blockIdx.x * 16 + c, k = threadIdx.x / 16;
  if (!a.d_weight[side]) return;
  const int groups = a.workgroups / (a.sets[0] + a.sets[1]), n = groups * a.sets[side];
  const float* p = a.part + (side ? (int64_t)groups * a.sets[0] * D : 0) + e;
  float v = 0.f;
  // (eight loads under way at once, zeros behind the last)
  for (int i0 = k; i0 < n; i0 += 8 * 64) {
    float x[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = i0 + 64 * i < n ? p[(int64_t)(i0 + 64 * i) * D] : 0.f;
#pragma unroll
    for (int i = 0; i < 8; ++i) v += x[i];
  }
  sums[k][c] = v;
  __syncthreads();
  if (k >= 4) return;                                     // (the first wave: 4 threads an element)
  v = 0.f;
#pragma unroll
  for (int i = 0; i < 16; ++i) v += sums[k * 16 + i][c];
  v += __shfl_xor(v, 16, 64);
  v += __shfl_xor(v, 32, 64);
  if (k == 0) a.d_weight[side][e] = a.weight_accumulate ? a.d_weight[side][e] + v : v;
}

template <int D>
static hipError_t launch_fwd_t(const RotateArgs& a, hipStream_t st) {
  const dim3 grid((unsigned)a.workgroups), block(256);
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
  if (a.part) hipLaunchKernelGGL((rotate_weights_kernel<D>), dim3(D / 16, 2), dim3(1024), 0, st, a);
  return hipGetLastError();
}
hipError_t launch_rotate_bwd(const RotateArgs& a, int head_dim, hipStream_t st) { return head_dim == 128 ? launch_bwd_t<128>(a, st) : launch_bwd_t<64>(a, st); }

}  // namespace slimpipe
