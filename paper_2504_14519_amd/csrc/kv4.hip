// A key/value cache held in 4 bits: rows stored and read back, and attention of a query slice or of single tokens over it.
//
// 32 consecutive elements of a head share a scale 2^e; an element is a 4-bit float (sign, 2 exponent bits, 1 mantissa bit: 0, 0.5, 1, 1.5,
// 2, 3, 4, 6).  gfx950 converts such numbers with their scale in one instruction, two at a time, exactly, to bf16, so that the attention
// below is the bf16 one on converted tiles: 4.25 bits an element are read instead of 16.
#include "kv4.hpp"
#include "row_tile.hpp"

namespace slimpipe {

// Scale byte as the float whose exponent the conversions use (255, a group with an infinity or a NaN: NaN).
SP_DEV float kv4_scale(uint32_t byte) { return __uint_as_float(byte == 255u ? 0x7fc00000u : byte << 23); }

// 8 elements (4 bytes of codes) -> bf16
SP_DEV bf16x8 kv4_values(uint32_t codes, float scale) {
  const bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 0), b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 1);
  const bf16x2 c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 2), d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 3);
  bf16x8 r;
  r[0] = a[0]; r[1] = a[1]; r[2] = b[0]; r[3] = b[1]; r[4] = c[0]; r[5] = c[1]; r[6] = d[0]; r[7] = d[1];
  return r;
}

// ------------------------------------------------------------------------------------ store, load
// Four lanes a group, 16 bytes of bf16 and 4 bytes of codes each: bound by the bytes (4096 rows of 40
// heads of 128: stored in 22.5 us, 4.7 TB/s, read back in 20).  blockIdx.y: keys or values.
template <int D, bool LOAD>
__global__ __launch_bounds__(256) void kv4_copy_kernel(const Kv4CopyArgs a) {
  constexpr int NC = D / 8;
  const int64_t gid = (int64_t)blockIdx.x * 256 + threadIdx.x, rh = gid / NC;      // (batch index, row, head) flattened
  const int c = (int)(gid - rh * NC);
  const bool keys = blockIdx.y == 0;
  if (rh >= a.batch * a.rows * a.n_kv_heads) return;             // (whole rows: the lanes of a group leave together)
  const int64_t br = rh / a.n_kv_heads, h = rh - br * a.n_kv_heads, b = br / a.rows, r = br - b * a.rows;
  const int64_t x = b * a.x_stride_b + r * a.x_stride_s + h * a.x_stride_h + c * 8;
  const int64_t y = b * a.kv_stride_b + (a.position + r) * a.kv_stride_s + h * a.kv_stride_h + c * 8;
  const Kv4Operand to = keys ? a.k : a.v;
  uint32_t* const codes = reinterpret_cast<uint32_t*>(to.codes + y / 2);
  uint8_t* const scale = to.scales + y / 32;
  if constexpr (LOAD) {
    const uint32_t s = *scale;
    bf16x8 v = kv4_values(*codes, kv4_scale(s));
    if (s == 255u) {
      typedef uint16_t u16x8 __attribute__((ext_vector_type(8)));
      v = __builtin_bit_cast(bf16x8, (u16x8)(0x7fc0));
    }
    *reinterpret_cast<bf16x8*>((keys ? a.k_dst : a.v_dst) + x) = v;
  } else {
    const u32x4 w = *reinterpret_cast<const u32x4*>((keys ? a.k_src : a.v_src) + x);
    uint32_t most = 0;                                            // largest magnitude, as bf16 bits
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const uint32_t lo = w[i] & 0x7fffu, hi = (w[i] >> 16) & 0x7fffu;
      most = most > lo ? most : lo;
      most = most > hi ? most : hi;
    }
#pragma unroll
    for (int k = 1; k < 4; k <<= 1) {
      const uint32_t o = (uint32_t)__shfl_xor((int)most, k, 64);
      most = most > o ? most : o;
    }
    // largest = 1.m 2^(E - 127): 2^e with e = E - 127 - 2, one more where 1.m >= 1.75, and at least -125
    const bool finite = most < 0x7f80u;
    int byte = (int)(most >> 7) - 2 + ((most & 0x7fu) >= 0x60u ? 1 : 0);
    byte = byte < 2 ? 2 : byte;
    const float s = __uint_as_float((uint32_t)byte << 23);
    const bf16x8 x8 = __builtin_bit_cast(bf16x8, w);
    uint32_t packed = 0;
    packed = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(packed, __builtin_shufflevector(x8, x8, 0, 1), s, 0);
    packed = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(packed, __builtin_shufflevector(x8, x8, 2, 3), s, 1);
    packed = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(packed, __builtin_shufflevector(x8, x8, 4, 5), s, 2);
    packed = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(packed, __builtin_shufflevector(x8, x8, 6, 7), s, 3);
    *codes = finite ? packed : 0u;
    if (c % 4 == 0) *scale = (uint8_t)(finite ? byte : 255);
  }
}

template <bool LOAD>
static hipError_t launch_copy(const Kv4CopyArgs& a, int head_dim, hipStream_t st) {
  const int64_t lanes = a.batch * a.rows * a.n_kv_heads * (head_dim / 8);
  dim3 grid((unsigned)((lanes + 255) / 256), 2), block(256);
  if (head_dim == 128) hipLaunchKernelGGL((kv4_copy_kernel<128, LOAD>), grid, block, 0, st, a);
  else hipLaunchKernelGGL((kv4_copy_kernel<64, LOAD>), grid, block, 0, st, a);
  return hipGetLastError();
}
hipError_t launch_kv4_store(const Kv4CopyArgs& a, int head_dim, hipStream_t st) { return launch_copy<false>(a, head_dim, st); }
hipError_t launch_kv4_load(const Kv4CopyArgs& a, int head_dim, hipStream_t st) { return launch_copy<true>(a, head_dim, st); }

// ------------------------------------------------------------------------------------ attention
// Rows of a plane (batch index, kv head) are numbered head of the group major: row rh is row rh % s_q of head rh / s_q.
struct Kv4Row { int r, h; };
SP_DEV Kv4Row kv4_row(const Kv4Args& a, int hk, int rh) {
  const int hl = rh / a.s_q;
  return {rh - hl * a.s_q, hk * a.group + hl};
}

template <int D>
constexpr size_t kv4_fwd_lds_bytes() {         // two slots of converted K and V tiles; then the output rows
  constexpr size_t rings = (size_t)4 * 64 * D * 2, rows = (size_t)4 * 32 * kOutRow<D> * 4;
  return rings > rows ? rings : rows;
}

// Slices: 128 rows a workgroup, 32 a wave (row_tile.hpp).  Codes of a tile of 64 keys are fetched one tile ahead into registers and
// converted into LDS, a group of 32 elements a thread, for all four waves at once.  4096 rows of 8 heads on 32768 keys of one: 530 us (970
// TFLOP/s, the fold of two ranges included), and the bf16 call 455: this form saves memory, not time.  Matrix units are busy 47 % of it, vector units 15 %,
// and 42 MB come from memory: none of them is full.
template <int D>
__global__ __launch_bounds__(256, 2) void kv4_fwd_kernel(const Kv4Args a) {
  constexpr int BN = 64, TILE = BN * D * 2, NG = D / 32, GROUPS = 2 * BN * NG, PER = GROUPS / 256;      // groups of K and V; a thread's
  extern __shared__ __attribute__((aligned(1024))) char smem[];
  const int tid = threadIdx.x, lane = tid & 63, g = lane >> 5, wave_u = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int rows = a.group * a.s_q, blocks = (rows + 127) / 128;
  const int part_i = blockIdx.x / blocks, blk = blocks - 1 - (blockIdx.x - part_i * blocks);
  const int plane = blockIdx.y, b = plane / a.n_kv_heads, hk = plane - b * a.n_kv_heads;
  const int rh = blk * 128 + wave_u * 32 + (lane & 31);
  const Kv4Row my = kv4_row(a, hk, rh < rows ? rh : rows - 1);
  const int64_t lo = a.kv_begin + (int64_t)part_i * a.part_keys;
  int64_t hi = lo + a.part_keys < a.kv_end ? lo + a.part_keys : a.kv_end;
  // last row of the block: of its head, or of the head before where the block holds the end of one
  if (a.causal) {
    const int r0 = blk * 128, r1 = r0 + 127 < rows ? r0 + 127 : rows - 1;
    const int64_t last = r0 / a.s_q == r1 / a.s_q ? r1 % a.s_q : a.s_q - 1;
    if (a.q_offset + last + 1 < hi) hi = a.q_offset + last + 1;
  }
  const int n_keys = hi > lo ? (int)(hi - lo) : 0, nt = (n_keys + BN - 1) / BN;
  const int64_t see = a.causal && a.q_offset + my.r < hi - 1 ? a.q_offset + my.r : hi - 1;
  const int64_t see_far = see - lo;
  const int see_rel = see_far < -1 ? -1 : (int)see_far;
  const unsigned lds = lds_addr(smem);

  // This thread's groups: a wave takes 64 / NG keys of K or V at a time, 16 keys along its lanes (sixteen rows in a column of chunks: no bank
  // twice in the LDS writes)
  constexpr int KEYS = 64 / NG, RUNS = BN / KEYS;
  const int grp = (lane >> 4) % NG;
  auto group_kv = [&](int n) { return (n * 4 + wave_u) / RUNS; };
  auto group_key = [&](int n) { return (n * 4 + wave_u) % RUNS * KEYS + (lane >> 4) / NG * 16 + (lane & 15); };
  const int64_t base = (int64_t)b * a.kv_stride_b + (int64_t)hk * a.kv_stride_h + lo * a.kv_stride_s;
  u32x4 codes[PER];
  uint32_t scales[PER];
  auto fetch = [&](int t) {
#pragma unroll
    for (int n = 0; n < PER; ++n) {
      const int kv = group_kv(n), key = group_key(n);
      const int k = t * BN + key < n_keys ? t * BN + key : n_keys - 1;      // (keys behind the last are not read)
      const int64_t at = base + (int64_t)k * a.kv_stride_s + grp * 32;
      const Kv4Operand& op = kv ? a.v : a.k;
      codes[n] = *reinterpret_cast<const u32x4*>(op.codes + at / 2);
      scales[n] = op.scales[at / 32];
    }
  };
  auto convert = [&](int t) {
#pragma unroll
    for (int n = 0; n < PER; ++n) {
      const int kv = group_kv(n), key = group_key(n);
      const float s = kv4_scale(scales[n]);
      char* tile = smem + (t & 1) * 2 * TILE + kv * TILE;
#pragma unroll
      for (int j = 0; j < 4; ++j) *reinterpret_cast<bf16x8*>(tile + tile_off<D>(key, 4 * grp + j)) = kv4_values(codes[n][j], s);
    }
  };

  RowState<D> st;
  st.init();
  if (nt > 0) {
    fetch(0);
    {
      const bf16_t* qp = a.q + (int64_t)b * a.q_stride_b + (int64_t)my.r * a.q_stride_s + (int64_t)my.h * a.q_stride_h + 8 * g;
#pragma unroll
      for (int ks = 0; ks < D / 16; ++ks) st.q[ks] = *reinterpret_cast<const bf16x8*>(qp + 16 * ks);
    }
    RpOffsets<D> lo_k;
    TrOffsets<D> lo_v;
    lo_k.init(lane, (int)lds);
    lo_v.init(lane, (int)lds + TILE);
    convert(0);
    if (nt > 1) fetch(1);
    __syncthreads();
    for (int t = 0; t < nt; ++t) {
      const int kmax = see_rel - t * BN;
      const bool masked = __builtin_amdgcn_ballot_w64(kmax < BN - 1) != 0;
      attend_tile<D, BN>(st, lo_k, lo_v, a.scale_log2e, masked, 0, kmax, g);
      const int step = (t & 1) ? -2 * TILE : 2 * TILE;
      lo_k.add(step);
      lo_v.add(step);
      if (t + 1 < nt) convert(t + 1);
      if (t + 2 < nt) fetch(t + 2);
      __syncthreads();
    }
  }
  float lse;
  const float norm = st.finish(&lse);
  if (norm == 0.f) st.clear();                   // (weights of 0 times what other rows see, which may not be finite)
  float* const part = reinterpret_cast<float*>(smem) + wave_u * 32 * kOutRow<D>;
  put_rows<D>(part, st.o, norm, lane);
  const int64_t row = ((int64_t)b * a.n_q_heads + my.h) * a.s_q + my.r;
  const int n_mine = rows - (blk * 128 + wave_u * 32);
  if (a.n_parts > 1) {
    const int64_t slot = row * a.n_parts + part_i;
    if (lane < 32 && lane < n_mine) a.part_lse[slot] = lse;
    constexpr int PERR = D / 4, RPP = 64 / PERR;
#pragma unroll
    for (int j = 0; j < 32 / RPP; ++j) {
      const int r = j * RPP + lane / PERR;
      const int64_t to = __shfl(slot, r, 64);
      if (r < n_mine) *reinterpret_cast<f32x4*>(a.part_out + to * D + lane % PERR * 4) = *reinterpret_cast<const f32x4*>(part + r * kOutRow<D> + lane % PERR * 4);
    }
    return;
  }
  if (lane < 32 && lane < n_mine) a.lse[row] = lse;
  const int64_t at = (int64_t)b * a.o_stride_b + (int64_t)my.r * a.o_stride_s + (int64_t)my.h * a.o_stride_h;
  constexpr int PERR = D / 8, RPP = 64 / PERR;
#pragma unroll
  for (int j = 0; j < 32 / RPP; ++j) {
    const int r = j * RPP + lane / PERR, d = lane % PERR * 8;
    const int64_t to = __shfl(at, r, 64) + d;
    const f32x4 x0 = *reinterpret_cast<const f32x4*>(part + r * kOutRow<D> + d), x1 = *reinterpret_cast<const f32x4*>(part + r * kOutRow<D> + d + 4);
    if (r >= n_mine) continue;
    if (a.out_f32) {
      f32x4* dst = reinterpret_cast<f32x4*>(static_cast<float*>(a.out) + to);
      dst[0] = x0;
      dst[1] = x1;
    } else {
      const bf16x4 y0 = __builtin_convertvector(x0, bf16x4), y1 = __builtin_convertvector(x1, bf16x4);
      *reinterpret_cast<bf16x8*>(static_cast<bf16_t*>(a.out) + to) = __builtin_shufflevector(y0, y1, 0, 1, 2, 3, 4, 5, 6, 7);
    }
  }
}

// Tokens: at most 16 SETS rows of a plane (its query heads and a few tokens), all in every wave; the four waves of a workgroup have a head
// each (or two, or all of them one) and share out the 32-key steps of its keys.  v_mfma_f32_16x16x32_bf16: with lane = 16 h + r an operand's lane holds row or column r, contraction slots
// 8 h .. 8 h + 7, a result's column r, register i row 4 h + i.
//   S^T = K Q^T      K goes from memory to the matrix unit without LDS: since the contraction may take head_dim in any order, lane group h
//                    takes the h-th quarter of a row, 8 elements a step, and a lane's codes of 16 keys are one load
//   O^T += V^T P^T   V passes through 32 rows of LDS of the wave's own for the transposed read (lane group h: keys 4 h .. 4 h + 3 of either 16)
// Codes of the next two steps are under way in registers (one with two heads a wave, whose loads start in the middle of the step before).
// A row's codes are 64 bytes and its scales 4, of lines of 128 that hold the next heads' too: hence neighbouring heads in a workgroup, and the
// workgroups that cover the same keys of a sequence one after the other on one XCD.  4 tokens of 40 heads on 32768 keys of 128: 200 us (720 MB,
// 3.6 TB/s; the bf16 call 455).  Neither the memory, which gives a copy 4.8, nor the matrix units (busy 10 %), nor the vector units (8 %) are full: what is
// left is the wait for codes.
template <int D, int SETS, int HEADS>
constexpr size_t kv4_few_lds_bytes() {
  constexpr size_t tiles = (size_t)4 * 32 * D * 2, out = (size_t)4 * 16 * SETS * HEADS * (kOutRow<D> + 2) * 4;
  return tiles > out ? tiles : out;
}
SP_DEV f32x4 mfma16(bf16x8 a, bf16x8 b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }
SP_DEV float quarters_max(float v) {      // over the four lane groups
  auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return xhalf_max(fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1])));
}
SP_DEV float quarters_sum(float v) {
  auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return xhalf_sum(__uint_as_float(r[0]) + __uint_as_float(r[1]));
}
template <int D, int SETS, int HEADS>
__global__ __launch_bounds__(256, 2) void kv4_few_kernel(const Kv4Args a) {
  constexpr int W = D / 32, N = SETS * HEADS, DEPTH = HEADS == 1 ? 2 : 1, DB = D / 16, QUARTER = D / 4;      // dwords of codes of a quarter row (= matrix steps), output blocks
  typedef uint32_t codes_t __attribute__((ext_vector_type(W)));
  extern __shared__ __attribute__((aligned(1024))) char smem[];
  const int tid = threadIdx.x, lane = tid & 63, h4 = lane >> 4, ql = lane & 15, wave_u = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int hw = a.heads_wg, subs = 4 / hw, sub = wave_u / hw;      // sets of HEADS heads of the workgroup, waves of a set, which of them this is
  const int rows = a.group * a.s_q, head_sets = a.n_kv_heads / (hw * HEADS), planes = a.batch * head_sets;
  int part_i = 0, plane = blockIdx.x;
  if (a.n_parts > 1) {
    const int per = 8 * planes, first = (int)blockIdx.x / per * 8, i = (int)blockIdx.x % per, n = a.n_parts - first < 8 ? a.n_parts - first : 8;
    part_i = first + i % n;
    plane = i / n;
  } else {
    plane = xcd_run(blockIdx.x, planes);
  }
  if (plane < 0 || plane >= planes) return;
  const int b = plane / head_sets, hk0 = (plane - b * head_sets) * hw * HEADS, hk = hk0 + wave_u % hw * HEADS;
  const int64_t lo = a.kv_begin + (int64_t)part_i * a.part_keys;
  const int64_t hi = lo + a.part_keys < a.kv_end ? lo + a.part_keys : a.kv_end;
  const int n_keys = hi > lo ? (int)(hi - lo) : 0, nt = (n_keys + 31) / 32;
  char* const tile_p = smem + wave_u * 32 * D * 2;

  // element n: row set n % SETS of head n / SETS
  bf16x8 q[N][W];
  f32x4 o[N][DB];
  float m[N], l[N];
  int see_rel[SETS];
#pragma unroll
  for (int r = 0; r < N; ++r) {
    const int rh = 16 * (r % SETS) + ql;
    const Kv4Row my = kv4_row(a, hk + r / SETS, rh < rows ? rh : rows - 1);
    const bf16_t* qp = a.q + (int64_t)b * a.q_stride_b + (int64_t)my.r * a.q_stride_s + (int64_t)my.h * a.q_stride_h + QUARTER * h4;
#pragma unroll
    for (int j = 0; j < W; ++j) q[r][j] = *reinterpret_cast<const bf16x8*>(qp + 8 * j);
#pragma unroll
    for (int db = 0; db < DB; ++db) o[r][db] = f32x4{0, 0, 0, 0};
    m[r] = -INFINITY;
    l[r] = 0.f;
    const int64_t see = (a.causal && a.q_offset + my.r < hi - 1 ? a.q_offset + my.r : hi - 1) - lo;
    see_rel[r % SETS] = see < -1 ? -1 : (int)see;
  }
  int min_see = see_rel[0];                      // keys up to here: every row of the lane sees them
#pragma unroll
  for (int r = 1; r < SETS; ++r) min_see = min_see < see_rel[r] ? min_see : see_rel[r];

  // LDS addresses: where this lane writes its quarter of a key's row (of 16 keys), and where it reads
  int to[W];
#pragma unroll
  for (int j = 0; j < W; ++j) to[j] = tile_off<D>(ql, h4 * W + j);
  const int from = (int)lds_addr(smem) + wave_u * 32 * D * 2 + tile_off<D>(4 * h4 + ql / 4, (ql & 3) >> 1) + ((ql & 1) << 3);

  const int64_t base = (int64_t)b * a.kv_stride_b + (int64_t)hk * a.kv_stride_h + lo * a.kv_stride_s + QUARTER * h4;
  const int64_t lane_off = (int64_t)ql * a.kv_stride_s, step_off = 16 * a.kv_stride_s;
  struct Step { codes_t k[HEADS][2], v[HEADS][2]; uint32_t ks[HEADS][2], vs[HEADS][2]; };
  auto fetch = [&](Step& s, int t) {
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      int64_t at = base + (2 * t + u) * step_off + lane_off;
      const int over = t * 32 + 16 * u + ql - (n_keys - 1);      // (keys behind the last are not read)
      if (t * 32 + 32 > n_keys) at -= (over > 0 ? over : 0) * a.kv_stride_s;
#pragma unroll
      for (int hd = 0; hd < HEADS; ++hd, at += a.kv_stride_h) {
        s.k[hd][u] = *reinterpret_cast<const codes_t*>(a.k.codes + at / 2);
        s.v[hd][u] = *reinterpret_cast<const codes_t*>(a.v.codes + at / 2);
        s.ks[hd][u] = a.k.scales[at / 32];
        s.vs[hd][u] = a.v.scales[at / 32];
      }
    }
  };
  auto work = [&](Step& st, int t, int next) {
#pragma unroll
    for (int hd = 0; hd < HEADS; ++hd) {
      f32x4 s[SETS][2];
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        const float ks = kv4_scale(st.ks[hd][u]), vs = kv4_scale(st.vs[hd][u]);
#pragma unroll
        for (int r = 0; r < SETS; ++r) s[r][u] = f32x4{0, 0, 0, 0};
#pragma unroll
        for (int j = 0; j < W; ++j) {
          const bf16x8 k8 = kv4_values(st.k[hd][u][j], ks);
#pragma unroll
          for (int r = 0; r < SETS; ++r) s[r][u] = mfma16(k8, q[hd * SETS + r][j], s[r][u]);
          *reinterpret_cast<bf16x8*>(tile_p + 16 * u * D * 2 + to[j]) = kv4_values(st.v[hd][u][j], vs);
        }
      }
      if (hd == HEADS - 1 && next < nt) fetch(st, next);
      if (__builtin_amdgcn_ballot_w64(min_see < t * 32 + 31) != 0)
#pragma unroll
        for (int r = 0; r < SETS; ++r)
#pragma unroll
          for (int u = 0; u < 2; ++u)
#pragma unroll
            for (int i = 0; i < 4; ++i) s[r][u][i] = t * 32 + 16 * u + 4 * h4 + i <= see_rel[r] ? s[r][u][i] : -INFINITY;
      bf16x8 p[SETS];
#pragma unroll
      for (int r = 0; r < SETS; ++r) {
        const int n = hd * SETS + r;
        float mx = -INFINITY;
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
          for (int i = 0; i < 4; ++i) mx = fmaxf(mx, s[r][u][i]);
        mx = quarters_max(mx);
        const float m_new = fmaxf(m[n], mx * a.scale_log2e), m_eff = m_new == -INFINITY ? 0.f : m_new;
        if (__builtin_amdgcn_ballot_w64(m_new != m[n]) != 0) {
          const float alpha = exp2_fast(m[n] - m_eff);
          l[n] *= alpha;
#pragma unroll
          for (int db = 0; db < DB; ++db) o[n][db] *= alpha;
        }
        m[n] = m_new;
#pragma unroll
        for (int u = 0; u < 2; ++u) {
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            s[r][u][i] = exp2_fast(__builtin_fmaf(s[r][u][i], a.scale_log2e, -m_eff));
            l[n] += s[r][u][i];
          }
        }
        // (probabilities rounded to bf16 relative to the exact running maximum; their sum is not rounded)
        const bf16x4 p0 = __builtin_convertvector(s[r][0], bf16x4), p1 = __builtin_convertvector(s[r][1], bf16x4);
        p[r] = __builtin_shufflevector(p0, p1, 0, 1, 2, 3, 4, 5, 6, 7);
      }
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
      __builtin_amdgcn_wave_barrier();
#pragma unroll
      for (int db = 0; db < DB; ++db) {
        // (the swizzle makes block db's offset that of block 0 with db in bits 5 ..)
        const bf16x4 v0 = __builtin_amdgcn_ds_read_tr16_b64_v4bf16(lds_ptr<bf16x4>(from ^ (db << 5), 0));
        const bf16x4 v1 = __builtin_amdgcn_ds_read_tr16_b64_v4bf16(lds_ptr<bf16x4>(from ^ (db << 5), 16 * D * 2));
        const bf16x8 v8 = __builtin_shufflevector(v0, v1, 0, 1, 2, 3, 4, 5, 6, 7);
#pragma unroll
        for (int r = 0; r < SETS; ++r) o[hd * SETS + r][db] = mfma16(v8, p[r], o[hd * SETS + r][db]);
      }
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
      __builtin_amdgcn_wave_barrier();
    }
  };
  if (sub < nt) {
    Step s[DEPTH];
#pragma unroll
    for (int i = 0; i < DEPTH; ++i)
      if (sub + i * subs < nt) fetch(s[i], sub + i * subs);
    for (int t = sub; t < nt; t += DEPTH * subs)
#pragma unroll
      for (int i = 0; i < DEPTH; ++i)
        if (t + i * subs < nt) work(s[i], t + i * subs, t + (i + DEPTH) * subs);
  }
  // the results of a head's waves, unnormalised, and their (maximum, sum), folded in wave order
  __syncthreads();
  constexpr int RW = 16 * N;
  float* const acc = reinterpret_cast<float*>(smem);                         // [wave][row][kOutRow]
  float* const stat = acc + 4 * RW * kOutRow<D>;                             // [wave][2][row]
#pragma unroll
  for (int r = 0; r < N; ++r) {
    const float sum = quarters_sum(l[r]);
    if (lane < 16) { stat[wave_u * 2 * RW + 16 * r + ql] = m[r]; stat[wave_u * 2 * RW + RW + 16 * r + ql] = sum; }
    if (16 * (r % SETS) + ql < rows)
#pragma unroll
      for (int db = 0; db < DB; ++db) *reinterpret_cast<f32x4*>(acc + (wave_u * RW + 16 * r + ql) * kOutRow<D> + 16 * db + 4 * h4) = o[r][db];
  }
  __syncthreads();
  constexpr int PER = D / 8;
  for (int i = tid; i < hw * HEADS * rows * PER; i += 256) {
    const int hh = i / (rows * PER), rr = (i - hh * rows * PER) / PER, d = i % PER * 8;
    const int w0 = hh / HEADS, r = hh % HEADS * 16 * SETS + rr;      // first wave of the head, row among its wave's
    float mx = -INFINITY, sum = 0.f;
    for (int w = w0; w < 4; w += hw) mx = fmaxf(mx, stat[w * 2 * RW + r]);
    f32x4 x0 = {0, 0, 0, 0}, x1 = {0, 0, 0, 0};
    const float m_eff = mx == -INFINITY ? 0.f : mx;
    for (int w = w0; w < 4; w += hw) {
      const float f = exp2_fast(stat[w * 2 * RW + r] - m_eff);
      sum += f * stat[w * 2 * RW + RW + r];
      x0 += f * *reinterpret_cast<const f32x4*>(acc + (w * RW + r) * kOutRow<D> + d);
      x1 += f * *reinterpret_cast<const f32x4*>(acc + (w * RW + r) * kOutRow<D> + d + 4);
    }
    const float norm = sum == 0.f ? 0.f : 1.0f / sum, lse = sum == 0.f ? -INFINITY : (mx + __builtin_log2f(sum)) * kLn2;      // (a NaN is not 0)
    x0 = sum == 0.f ? f32x4{0, 0, 0, 0} : x0 * norm;      // (as above)
    x1 = sum == 0.f ? f32x4{0, 0, 0, 0} : x1 * norm;
    const Kv4Row at = kv4_row(a, hk0 + hh, rr);
    const int64_t row = ((int64_t)b * a.n_q_heads + at.h) * a.s_q + at.r;
    if (a.n_parts > 1) {
      f32x4* dst = reinterpret_cast<f32x4*>(a.part_out + (row * a.n_parts + part_i) * D + d);
      dst[0] = x0;
      dst[1] = x1;
      if (d == 0) a.part_lse[row * a.n_parts + part_i] = lse;
      continue;
    }
    const int64_t to_out = (int64_t)b * a.o_stride_b + (int64_t)at.r * a.o_stride_s + (int64_t)at.h * a.o_stride_h + d;
    if (a.out_f32) {
      f32x4* dst = reinterpret_cast<f32x4*>(static_cast<float*>(a.out) + to_out);
      dst[0] = x0;
      dst[1] = x1;
    } else {
      const bf16x4 y0 = __builtin_convertvector(x0, bf16x4), y1 = __builtin_convertvector(x1, bf16x4);
      *reinterpret_cast<bf16x8*>(static_cast<bf16_t*>(a.out) + to_out) = __builtin_shufflevector(y0, y1, 0, 1, 2, 3, 4, 5, 6, 7);
    }
    if (d == 0) a.lse[row] = lse;
  }
}

template <int D, int SETS, int HEADS>
static void launch_few_t(const Kv4Args& a, hipStream_t st) {
  const unsigned planes = (unsigned)(a.batch * (a.n_kv_heads / (a.heads_wg * HEADS)));
  hipLaunchKernelGGL((kv4_few_kernel<D, SETS, HEADS>), dim3(a.n_parts > 1 ? (unsigned)a.n_parts * planes : (planes + 7) / 8 * 8), dim3(256),
                     (kv4_few_lds_bytes<D, SETS, HEADS>()), st, a);
}
template <int D>
static void launch_fwd_t(const Kv4Args& a, bool few, hipStream_t st) {
  const unsigned planes = (unsigned)(a.batch * a.n_kv_heads);
  const int rows = a.group * a.s_q;
  if (few && a.wave_heads == 2) launch_few_t<D, 1, 2>(a, st);
  else if (few) rows <= 16 ? launch_few_t<D, 1, 1>(a, st) : launch_few_t<D, 2, 1>(a, st);
  else hipLaunchKernelGGL(kv4_fwd_kernel<D>, dim3((unsigned)a.n_parts * (unsigned)((rows + 127) / 128), planes), dim3(256), kv4_fwd_lds_bytes<D>(), st, a);
}
hipError_t launch_kv4_fwd(const Kv4Args& a, int head_dim, bool few, hipStream_t st) {
  if (head_dim == 128) launch_fwd_t<128>(a, few, st);
  else launch_fwd_t<64>(a, few, st);
  return hipGetLastError();
}

hipError_t opt_in_kv4_kernels() {
  const hipFuncAttribute attr = hipFuncAttributeMaxDynamicSharedMemorySize;
  hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(&kv4_fwd_kernel<128>), attr, (int)kv4_fwd_lds_bytes<128>());
  if (e == hipSuccess) e = hipFuncSetAttribute(reinterpret_cast<const void*>(&kv4_fwd_kernel<64>), attr, (int)kv4_fwd_lds_bytes<64>());
  if (e == hipSuccess) e = hipFuncSetAttribute(reinterpret_cast<const void*>(&kv4_few_kernel<128, 2, 1>), attr, (int)kv4_few_lds_bytes<128, 2, 1>());
  if (e == hipSuccess) e = hipFuncSetAttribute(reinterpret_cast<const void*>(&kv4_few_kernel<128, 1, 2>), attr, (int)kv4_few_lds_bytes<128, 1, 2>());
  return e;
}

}  // namespace slimpipe
