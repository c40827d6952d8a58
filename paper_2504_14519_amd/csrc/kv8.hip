// A key/value cache held in 8 bits: rows appended and read back, and attention of a query slice or of single tokens over it.
//
// A block of consecutive rows of a head shares a scale 2^e; an element is an 8-bit float (sign, 4 exponent bits, 3 mantissa bits, largest 448).  gfx950
// converts such numbers with their scale in one instruction, two at a time, exactly, to bf16, so that the attention below is the bf16 one on
// converted tiles.  The scale is a power of two because the rows of a block come one after the other: when a larger one comes, those that are there
// move to the larger scale without an error (but for elements below 2^-6 of it), which another factor would not allow.
#include "kv8_values.hpp"
#include "row_tile.hpp"

namespace slimpipe {

// ------------------------------------------------------------------------------------ store, load
// Largest magnitude (bf16 bits) of 8 elements, two at a time; FINITE_ONLY: among those that are neither infinite nor NaN.
template <bool FINITE_ONLY>
SP_DEV u16x2 most_of(u32x4 w, u16x2 most) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    u16x2 m = __builtin_bit_cast(u16x2, w[i] & 0x7fff7fffu);
    if constexpr (FINITE_ONLY) {
      m[0] = m[0] >= 0x7f80 ? 0 : m[0];
      m[1] = m[1] >= 0x7f80 ? 0 : m[1];
    }
    most = __builtin_elementwise_max(most, m);
  }
  return most;
}
// A block of a head by T threads (a wave, or a workgroup): its new rows are read once, into registers, their largest magnitude gives the scale, and the
// codes leave.  Rows that the block has already are looked at only where the scale grows.  Bound by the bytes: 4096 rows of 40 heads of 128 in blocks of 128
// 22 us, 126 MB at 5.7 TB/s.
template <int D, int T>
__global__ __launch_bounds__(256) void kv8_store_kernel(const Kv8CopyArgs a) {
  constexpr int NC = D / 8, RPP = T / NC, PASSES = T == 64 ? 16 : 2 * D / 16;      // rows a pass; passes of the longest block that T threads take
  __shared__ uint32_t shared_most[4];
  const int tid = threadIdx.x % T, c = tid % NC;
  const Kv8Cache& k = a.cache;
  const int64_t first = a.position >> k.shift, n_blocks = ((a.position + a.rows - 1) >> k.shift) - first + 1;
  const int64_t item = T == 64 ? (int64_t)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) : blockIdx.x;      // (batch index, block, head)
  if (item >= a.batch * n_blocks * k.n_kv_heads) return;
  const int64_t bb = item / k.n_kv_heads, b = bb / n_blocks;
  const int h = (int)(item - bb * k.n_kv_heads);
  const int64_t blk = first + (bb - b * n_blocks), row0 = blk << k.shift;      // the block and its first row
  const int64_t lo = row0 > a.position ? row0 : a.position;
  const int64_t hi = a.position + a.rows < row0 + (1 << k.shift) ? a.position + a.rows : row0 + (1 << k.shift);
  const bool keys = blockIdx.y == 0;
  const bf16_t* src = (keys ? a.k_src : a.v_src) + b * a.x_stride_b + (lo - a.position) * a.x_stride_s + h * a.x_stride_h + c * 8;
  const Kv8Operand to = keys ? k.k : k.v;
  uint8_t* codes = to.codes + b * k.stride_b + h * k.stride_h + c * 8;
  uint8_t* const scale = to.scales + (b * k.blocks + blk) * k.n_kv_heads + h;
  const int n = (int)(hi - lo), r0 = tid / NC;
  const uint32_t old = lo > row0 ? *scale : 0u;
  u32x4 w[PASSES];
#pragma unroll
  for (int p = 0; p < PASSES; ++p) {
    w[p] = u32x4{0, 0, 0, 0};
    if (r0 + p * RPP < n) w[p] = *reinterpret_cast<const u32x4*>(src + (int64_t)(r0 + p * RPP) * a.x_stride_s);
  }
  auto reduce = [&](u16x2 m) {
    uint32_t most = m[0] > m[1] ? m[0] : m[1];
#pragma unroll
    for (int i = 1; i < 64; i <<= 1) {
      const uint32_t o = (uint32_t)__shfl_xor((int)most, i, 64);
      most = most > o ? most : o;
    }
    if constexpr (T > 64) {
      __syncthreads();
      if ((threadIdx.x & 63) == 0) shared_most[threadIdx.x >> 6] = most;
      __syncthreads();
#pragma unroll
      for (int i = 0; i < 4; ++i) most = most > shared_most[i] ? most : shared_most[i];
    }
    return most;
  };
  u16x2 m = {0, 0};
#pragma unroll
  for (int p = 0; p < PASSES; ++p) m = most_of<false>(w[p], m);
  uint32_t most = reduce(m);
  if (most >= 0x7f80u) {                       // an infinity or a NaN: stored as NaN, and no part of the scale
    m = u16x2{0, 0};
#pragma unroll
    for (int p = 0; p < PASSES; ++p) {
      m = most_of<true>(w[p], m);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        if ((w[p][i] & 0x7fffu) >= 0x7f80u) w[p][i] |= 0x7fffu;
        if ((w[p][i] & 0x7fff0000u) >= 0x7f800000u) w[p][i] |= 0x7fff0000u;
      }
    }
    most = reduce(m);
  }
  // largest = 1.m 2^(E - 127): 448 = 1.75 * 2^8, so e = E - 127 - 8, one more where 1.m > 1.75, and at least -110
  int byte = (int)(most >> 7) - 8 + ((most & 0x7fu) > 0x60u ? 1 : 0);
  byte = byte < (int)kKv8LeastScale ? (int)kKv8LeastScale : byte;
  byte = byte < (int)old ? (int)old : byte;
  const float unit = kv8_scale((uint32_t)byte);
#pragma unroll
  for (int p = 0; p < PASSES; ++p)
    if (r0 + p * RPP < n)
      *reinterpret_cast<u32x2*>(codes + (lo + r0 + p * RPP) * k.stride_s) = kv8_codes(__builtin_bit_cast(bf16x8, w[p]), unit);
  if (lo > row0 && byte > (int)old) {          // the rows before move to the larger scale
    const float was = kv8_scale(old);
    for (int64_t r = row0 + r0; r < lo; r += RPP) {
      u32x2* at = reinterpret_cast<u32x2*>(codes + r * k.stride_s);
      const u32x2 x = *at;
      *at = kv8_codes(kv8_values(x[0], x[1], was), unit);
    }
  }
  if (tid == 0) *scale = (uint8_t)byte;
}

// Bound by the bytes: 8 elements a thread, read and written past the caches.  The same rows back in 20 us (6.1 TB/s); rows left in the caches take as long, but
// delay the kernels around the call, which have to write them out (the store 25 us instead of 22, a move of 32768 rows of 8 heads 37 instead of 27).
template <int D>
__global__ __launch_bounds__(256) void kv8_load_kernel(const Kv8CopyArgs a) {
  constexpr int NC = D / 8;
  const Kv8Cache& k = a.cache;
  // (less than 2^27 rows of all heads: 32 bits, in which a division is a fifth of the instructions)
  const uint32_t gid = blockIdx.x * 256u + threadIdx.x, rh = gid / NC, rows = (uint32_t)a.rows;      // (batch index, row, head) flattened
  const int c = (int)(gid % NC);
  if (rh >= (uint32_t)a.batch * rows * (uint32_t)k.n_kv_heads) return;
  const uint32_t br = rh / (uint32_t)k.n_kv_heads, bu = br / rows;
  const int64_t b = bu, r = br - bu * rows;
  const int h = (int)(rh - br * (uint32_t)k.n_kv_heads);
  const Kv8Operand from = blockIdx.y == 0 ? k.k : k.v;
  const u32x2 x = __builtin_nontemporal_load(reinterpret_cast<const u32x2*>(from.codes + b * k.stride_b + (a.position + r) * k.stride_s + h * k.stride_h + c * 8));
  const float unit = kv8_scale(from.scales[kv8_scale_at(k, b, a.position + r, h)]);
  bf16_t* to = (blockIdx.y == 0 ? a.k_dst : a.v_dst) + b * a.x_stride_b + r * a.x_stride_s + h * a.x_stride_h + c * 8;
  __builtin_nontemporal_store(kv8_values(x[0], x[1], unit), reinterpret_cast<bf16x8*>(to));
}

hipError_t launch_kv8_store(const Kv8CopyArgs& a, int head_dim, hipStream_t st) {
  const int64_t first = a.position >> a.cache.shift, blocks = ((a.position + a.rows - 1) >> a.cache.shift) - first + 1;
  const int64_t items = a.batch * blocks * a.cache.n_kv_heads;
  const bool wave = ((int64_t)head_dim << a.cache.shift) <= 8192;
  const dim3 grid((unsigned)(wave ? (items + 3) / 4 : items), 2), block(256);
  if (head_dim == 128) {
    if (wave) hipLaunchKernelGGL((kv8_store_kernel<128, 64>), grid, block, 0, st, a);
    else hipLaunchKernelGGL((kv8_store_kernel<128, 256>), grid, block, 0, st, a);
  } else {
    if (wave) hipLaunchKernelGGL((kv8_store_kernel<64, 64>), grid, block, 0, st, a);
    else hipLaunchKernelGGL((kv8_store_kernel<64, 256>), grid, block, 0, st, a);
  }
  return hipGetLastError();
}
hipError_t launch_kv8_load(const Kv8CopyArgs& a, int head_dim, hipStream_t st) {
  const int64_t lanes = a.batch * a.rows * a.cache.n_kv_heads * (head_dim / 8);
  const dim3 grid((unsigned)((lanes + 255) / 256), 2), block(256);
  if (head_dim == 128) hipLaunchKernelGGL((kv8_load_kernel<128>), grid, block, 0, st, a);
  else hipLaunchKernelGGL((kv8_load_kernel<64>), grid, block, 0, st, a);
  return hipGetLastError();
}

// ------------------------------------------------------------------------------------ attention
template <int D, int NW>
constexpr size_t kv8_fwd_lds_bytes() {         // two slots of converted K and V tiles; then the output rows
  constexpr size_t rings = (size_t)4 * 64 * D * 2, rows = (size_t)NW * 32 * kOutRow<D> * 4;
  return rings > rows ? rings : rows;
}

// Slices of less than 2048 rows of a kv head (or where there is no room for a bf16 copy of the keys): 256 or 128 rows a workgroup of NW waves, 32 a wave
// (row_tile.hpp).  Codes of a tile of 64 keys are fetched one tile ahead into registers and converted into LDS for all waves at once.  256 rows of 40 heads on
// 16640 keys: 104 us (830 TFLOP/s, the fold of the ranges included), and 102 on a bf16 cache; 4096 rows of 8 heads on 32768 keys 513 us, by the copy 455:
// the waves' matrix and vector phases are not kept apart as in the dense kernel.  (On a machine whose 8192^3 bf16 product runs at 1405 TFLOP/s; on one of 1245 119
// and, by the copy, 516.)
template <int D, int NW>
__global__ __launch_bounds__(NW * 64, 2) void kv8_fwd_kernel(const Kv8Args a) {
  constexpr int BN = 64, TILE = BN * D * 2, NP = D / 16, PER = 2 * BN * NP / (NW * 64), ROWS = NW * 32;      // pieces of 16 elements of a row; of a thread, K and V
  extern __shared__ __attribute__((aligned(1024))) char smem[];
  const Kv8Cache& kv = a.cache;
  const int tid = threadIdx.x, lane = tid & 63, g = lane >> 5, wave_u = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int rows = a.group * a.s_q, blocks = (rows + ROWS - 1) / ROWS;
  const int part_i = blockIdx.x / blocks, blk = blocks - 1 - (blockIdx.x - part_i * blocks);
  const int plane = blockIdx.y, b = plane / kv.n_kv_heads, hk = plane - b * kv.n_kv_heads;
  const int rh = blk * ROWS + wave_u * 32 + (lane & 31);
  const PlaneRow my = plane_row(a.s_q, a.group, hk, rh < rows ? rh : rows - 1);
  const int64_t lo = a.kv_begin + (int64_t)part_i * a.part_keys;
  int64_t hi = lo + a.part_keys < a.kv_end ? lo + a.part_keys : a.kv_end;
  // last row of the block: of its head, or of the head before where the block holds the end of one
  if (a.causal) {
    const int r0 = blk * ROWS, r1 = r0 + ROWS - 1 < rows ? r0 + ROWS - 1 : rows - 1;
    const int64_t last = r0 / a.s_q == r1 / a.s_q ? r1 % a.s_q : a.s_q - 1;
    if (a.q_offset + last + 1 < hi) hi = a.q_offset + last + 1;
  }
  const int n_keys = hi > lo ? (int)(hi - lo) : 0, nt = (n_keys + BN - 1) / BN;
  const int64_t see = a.causal && a.q_offset + my.r < hi - 1 ? a.q_offset + my.r : hi - 1;
  const int64_t see_far = see - lo;
  const int see_rel = see_far < -1 ? -1 : (int)see_far;
  const unsigned lds = lds_addr(smem);

  // This thread's pieces: a wave takes 16 keys of K or V and four pieces of each at a time (sixteen rows in a column of chunks: no bank twice in the LDS
  // writes)
  constexpr int RUNS = BN / 16 * (NP / 4);
  auto piece_kv = [&](int n) { return (n * NW + wave_u) / RUNS; };
  auto piece_key = [&](int n) { return (n * NW + wave_u) % RUNS / (NP / 4) * 16 + (lane & 15); };
  auto piece_at = [&](int n) { return (n * NW + wave_u) % (NP / 4) * 4 + (lane >> 4); };
  const int64_t base = (int64_t)b * kv.stride_b + (int64_t)hk * kv.stride_h + lo * kv.stride_s;
  u32x4 codes[PER];
  uint32_t scales[PER];
  auto fetch = [&](int t) {
#pragma unroll
    for (int n = 0; n < PER; ++n) {
      const int key = piece_key(n);
      const int k = t * BN + key < n_keys ? t * BN + key : n_keys - 1;      // (keys behind the last are not read)
      const Kv8Operand& op = piece_kv(n) ? kv.v : kv.k;
      codes[n] = *reinterpret_cast<const u32x4*>(op.codes + base + (int64_t)k * kv.stride_s + piece_at(n) * 16);
      scales[n] = op.scales[kv8_scale_at(kv, b, lo + k, hk)];
    }
  };
  auto convert = [&](int t) {
#pragma unroll
    for (int n = 0; n < PER; ++n) {
      const float s = kv8_scale(scales[n]);
      char* tile = smem + (t & 1) * 2 * TILE + piece_kv(n) * TILE;
      *reinterpret_cast<bf16x8*>(tile + tile_off<D>(piece_key(n), 2 * piece_at(n))) = kv8_values(codes[n][0], codes[n][1], s);
      *reinterpret_cast<bf16x8*>(tile + tile_off<D>(piece_key(n), 2 * piece_at(n) + 1)) = kv8_values(codes[n][2], codes[n][3], s);
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
  const int n_mine = rows - (blk * ROWS + wave_u * 32);
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
// each (or two, or all of them one) and share out the 32-key steps of its keys.
//   S^T = K Q^T      K goes from memory to the matrix unit without LDS: since the contraction may take head_dim in any order, lane group h
//                    takes bytes 16 h .. 16 h + 15 of every 64 of a row, two steps, and 16 rows' codes are a load of whole lines
//   O^T += V^T P^T   V passes through 32 rows of LDS of the wave's own for the transposed read (lane group h: keys 4 h .. 4 h + 3 of either 16)
// Codes of the next DEPTH steps are under way in registers.  Neighbouring heads lie in a workgroup, and the workgroups that cover the same keys of a sequence
// follow one another on one XCD.  Tokens of 4 sequences of 32768 keys, 40 heads of 128: 241 us (with a profiler 250), 1.34 GB at 5.6 TB/s; matrix units busy 8 %, vector units 23 %
// (one step under way 250 us, three or four 246; 128 registers for four workgroups a unit with two steps: spilled, 500).
template <int D, int SETS>
constexpr size_t kv8_few_lds_bytes() {
  constexpr size_t tiles = (size_t)4 * 32 * D * 2, out = (size_t)4 * 16 * SETS * (kOutRow<D> + 2) * 4;
  return tiles > out ? tiles : out;
}
template <int D, int SETS>
__global__ __launch_bounds__(256, 2) void kv8_few_kernel(const Kv8Args a) {
  constexpr int NP = D / 64, W = 2 * NP, DEPTH = 2, DB = D / 16;      // pieces of 16 bytes of a lane's row (two matrix steps each), output blocks
  extern __shared__ __attribute__((aligned(1024))) char smem[];
  const Kv8Cache& kv = a.cache;
  const int tid = threadIdx.x, lane = tid & 63, h4 = lane >> 4, ql = lane & 15, wave_u = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int hw = kv8_heads_wg(kv.n_kv_heads), subs = 4 / hw, sub = wave_u / hw;      // heads of the workgroup, waves of a head, which of them this is
  const int rows = a.group * a.s_q, head_sets = kv.n_kv_heads / hw, planes = a.batch * head_sets;
  int part_i = 0, plane = blockIdx.x;
  if (a.n_parts > 1) {
    const int per = 8 * planes, first = (int)blockIdx.x / per * 8, i = (int)blockIdx.x % per, n = a.n_parts - first < 8 ? a.n_parts - first : 8;
    part_i = first + i % n;
    plane = i / n;
  } else {
    plane = xcd_run(blockIdx.x, planes);
  }
  if (plane < 0 || plane >= planes) return;
  const int b = plane / head_sets, hk0 = (plane - b * head_sets) * hw, hk = hk0 + wave_u % hw;
  const int64_t lo = a.kv_begin + (int64_t)part_i * a.part_keys;
  const int64_t hi = lo + a.part_keys < a.kv_end ? lo + a.part_keys : a.kv_end;
  const int n_keys = hi > lo ? (int)(hi - lo) : 0, nt = (n_keys + 31) / 32;
  char* const tile_p = smem + wave_u * 32 * D * 2;

  bf16x8 q[SETS][W];
  f32x4 o[SETS][DB];
  float m[SETS], l[SETS];
  int see_rel[SETS];
#pragma unroll
  for (int r = 0; r < SETS; ++r) {
    const int rh = 16 * r + ql;
    const PlaneRow my = plane_row(a.s_q, a.group, hk, rh < rows ? rh : rows - 1);
    const bf16_t* qp = a.q + (int64_t)b * a.q_stride_b + (int64_t)my.r * a.q_stride_s + (int64_t)my.h * a.q_stride_h + 16 * h4;
#pragma unroll
    for (int j = 0; j < W; ++j) q[r][j] = *reinterpret_cast<const bf16x8*>(qp + 64 * (j / 2) + 8 * (j % 2));
#pragma unroll
    for (int db = 0; db < DB; ++db) o[r][db] = f32x4{0, 0, 0, 0};
    m[r] = -INFINITY;
    l[r] = 0.f;
    const int64_t see = (a.causal && a.q_offset + my.r < hi - 1 ? a.q_offset + my.r : hi - 1) - lo;
    see_rel[r] = see < -1 ? -1 : (int)see;
  }
  int min_see = see_rel[0];                      // keys up to here: every row of the lane sees them
#pragma unroll
  for (int r = 1; r < SETS; ++r) min_see = min_see < see_rel[r] ? min_see : see_rel[r];

  // LDS addresses: where this lane writes its pieces of a key's row (of 16 keys), and where it reads
  int to[W];
#pragma unroll
  for (int j = 0; j < W; ++j) to[j] = tile_off<D>(ql, 8 * (j / 2) + 2 * h4 + j % 2);
  const int from = (int)lds_addr(smem) + wave_u * 32 * D * 2 + tile_off<D>(4 * h4 + ql / 4, (ql & 3) >> 1) + ((ql & 1) << 3);

  const int64_t base = (int64_t)b * kv.stride_b + (int64_t)hk * kv.stride_h + lo * kv.stride_s + 16 * h4;
  struct Step { u32x4 k[2][NP], v[2][NP]; uint32_t ks[2], vs[2]; };
  auto fetch = [&](Step& s, int t) {
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      int key = t * 32 + 16 * u + ql;
      key = key < n_keys ? key : n_keys - 1;                     // (keys behind the last are not read)
      const int64_t at = base + (int64_t)key * kv.stride_s, sc = kv8_scale_at(kv, b, lo + key, hk);
#pragma unroll
      for (int p = 0; p < NP; ++p) {
        s.k[u][p] = *reinterpret_cast<const u32x4*>(kv.k.codes + at + 64 * p);
        s.v[u][p] = *reinterpret_cast<const u32x4*>(kv.v.codes + at + 64 * p);
      }
      s.ks[u] = kv.k.scales[sc];
      s.vs[u] = kv.v.scales[sc];
    }
  };
  auto work = [&](Step& st, int t, int next) {
    f32x4 s[SETS][2];
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      const float ks = kv8_scale(st.ks[u]), vs = kv8_scale(st.vs[u]);
#pragma unroll
      for (int r = 0; r < SETS; ++r) s[r][u] = f32x4{0, 0, 0, 0};
#pragma unroll
      for (int j = 0; j < W; ++j) {
        const bf16x8 k8 = kv8_values(st.k[u][j / 2][j % 2 * 2], st.k[u][j / 2][j % 2 * 2 + 1], ks);
#pragma unroll
        for (int r = 0; r < SETS; ++r) s[r][u] = mfma16(k8, q[r][j], s[r][u]);
        *reinterpret_cast<bf16x8*>(tile_p + 16 * u * D * 2 + to[j]) = kv8_values(st.v[u][j / 2][j % 2 * 2], st.v[u][j / 2][j % 2 * 2 + 1], vs);
      }
    }
    if (next < nt) fetch(st, next);
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
      float mx = -INFINITY;
#pragma unroll
      for (int u = 0; u < 2; ++u)
#pragma unroll
        for (int i = 0; i < 4; ++i) mx = fmaxf(mx, s[r][u][i]);
      mx = quarters_max(mx);
      const float m_new = fmaxf(m[r], mx * a.scale_log2e), m_eff = m_new == -INFINITY ? 0.f : m_new;
      if (__builtin_amdgcn_ballot_w64(m_new != m[r]) != 0) {
        const float alpha = exp2_fast(m[r] - m_eff);
        l[r] *= alpha;
#pragma unroll
        for (int db = 0; db < DB; ++db) o[r][db] *= alpha;
      }
      m[r] = m_new;
#pragma unroll
      for (int u = 0; u < 2; ++u) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          s[r][u][i] = exp2_fast(__builtin_fmaf(s[r][u][i], a.scale_log2e, -m_eff));
          l[r] += s[r][u][i];
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
      for (int r = 0; r < SETS; ++r) o[r][db] = mfma16(v8, p[r], o[r][db]);
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
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
  constexpr int RW = 16 * SETS;
  float* const acc = reinterpret_cast<float*>(smem);                         // [wave][row][kOutRow]
  float* const stat = acc + 4 * RW * kOutRow<D>;                             // [wave][2][row]
#pragma unroll
  for (int r = 0; r < SETS; ++r) {
    const float sum = quarters_sum(l[r]);
    if (lane < 16) { stat[wave_u * 2 * RW + 16 * r + ql] = m[r]; stat[wave_u * 2 * RW + RW + 16 * r + ql] = sum; }
    if (16 * r + ql < rows)
#pragma unroll
      for (int db = 0; db < DB; ++db) *reinterpret_cast<f32x4*>(acc + (wave_u * RW + 16 * r + ql) * kOutRow<D> + 16 * db + 4 * h4) = o[r][db];
  }
  __syncthreads();
  constexpr int PER = D / 8;
  for (int i = tid; i < hw * rows * PER; i += 256) {
    const int hh = i / (rows * PER), rr = (i - hh * rows * PER) / PER, d = i % PER * 8;      // (first wave of head hh: hh)
    float mx = -INFINITY, sum = 0.f;
    for (int w = hh; w < 4; w += hw) mx = fmaxf(mx, stat[w * 2 * RW + rr]);
    f32x4 x0 = {0, 0, 0, 0}, x1 = {0, 0, 0, 0};
    const float m_eff = mx == -INFINITY ? 0.f : mx;
    for (int w = hh; w < 4; w += hw) {
      const float f = exp2_fast(stat[w * 2 * RW + rr] - m_eff);
      sum += f * stat[w * 2 * RW + RW + rr];
      x0 += f * *reinterpret_cast<const f32x4*>(acc + (w * RW + rr) * kOutRow<D> + d);
      x1 += f * *reinterpret_cast<const f32x4*>(acc + (w * RW + rr) * kOutRow<D> + d + 4);
    }
    const float norm = sum == 0.f ? 0.f : 1.0f / sum, lse = sum == 0.f ? -INFINITY : (mx + __builtin_log2f(sum)) * kLn2;      // (a NaN is not 0)
    x0 = sum == 0.f ? f32x4{0, 0, 0, 0} : x0 * norm;      // (as above)
    x1 = sum == 0.f ? f32x4{0, 0, 0, 0} : x1 * norm;
    const PlaneRow at = plane_row(a.s_q, a.group, hk0 + hh, rr);
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

template <int D, int SETS>
static void launch_few_t(const Kv8Args& a, hipStream_t st) {
  const unsigned planes = (unsigned)(a.batch * (a.cache.n_kv_heads / kv8_heads_wg(a.cache.n_kv_heads)));
  hipLaunchKernelGGL((kv8_few_kernel<D, SETS>), dim3(a.n_parts > 1 ? (unsigned)a.n_parts * planes : (planes + 7) / 8 * 8), dim3(256),
                     (kv8_few_lds_bytes<D, SETS>()), st, a);
}
template <int D, int NW>
static void launch_slice_t(const Kv8Args& a, hipStream_t st) {
  const unsigned blocks = (unsigned)((a.group * a.s_q + NW * 32 - 1) / (NW * 32));
  hipLaunchKernelGGL((kv8_fwd_kernel<D, NW>), dim3((unsigned)a.n_parts * blocks, (unsigned)(a.batch * a.cache.n_kv_heads)), dim3(NW * 64),
                     (kv8_fwd_lds_bytes<D, NW>()), st, a);
}
template <int D>
static void launch_fwd_t(const Kv8Args& a, Kv8Kernel kernel, hipStream_t st) {
  switch (kernel) {
    case Kv8Kernel::few: a.group * a.s_q <= 16 ? launch_few_t<D, 1>(a, st) : launch_few_t<D, 2>(a, st); break;
    case Kv8Kernel::four_waves: launch_slice_t<D, 4>(a, st); break;
    case Kv8Kernel::eight_waves: launch_slice_t<D, 8>(a, st);
  }
}
hipError_t launch_kv8_fwd(const Kv8Args& a, int head_dim, Kv8Kernel kernel, hipStream_t st) {
  if (head_dim == 128) launch_fwd_t<128>(a, kernel, st);
  else launch_fwd_t<64>(a, kernel, st);
  return hipGetLastError();
}

template <int D, int NW>
static hipError_t opt_in_slice() {
  return hipFuncSetAttribute(reinterpret_cast<const void*>(&kv8_fwd_kernel<D, NW>), hipFuncAttributeMaxDynamicSharedMemorySize, (int)kv8_fwd_lds_bytes<D, NW>());
}
hipError_t opt_in_kv8_kernels() {
  hipError_t e = opt_in_slice<128, 4>();
  if (e == hipSuccess) e = opt_in_slice<64, 4>();
  if (e == hipSuccess) e = opt_in_slice<128, 8>();
  if (e == hipSuccess) e = opt_in_slice<64, 8>();
  if (e == hipSuccess)
    e = hipFuncSetAttribute(reinterpret_cast<const void*>(&kv8_few_kernel<128, 2>), hipFuncAttributeMaxDynamicSharedMemorySize, (int)kv8_few_lds_bytes<128, 2>());
  return e;
}

}  // namespace slimpipe
