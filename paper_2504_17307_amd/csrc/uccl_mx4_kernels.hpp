// Rows to microscaled 4 bits, and products grouped by expert of weights in them (device code).  Internal to the library.
#pragma once

#include "uccl_product_kernels.hpp"

namespace {

constexpr uint32_t kMx4Block = 32;

// Four bytes, two elements each, times 2^(byte - 127) as eight bf16: exact below 2^128, for bf16 has all these powers; an infinity from there on.
__device__ __forceinline__ u32x4 widen_e2m1(uint32_t eight, float scale) {
  return u32x4{__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(eight, scale, 0)), __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(eight, scale, 1)),
               __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(eight, scale, 2)), __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(eight, scale, 3))};
}

// The same as eight f16, which is exact for scales of 2^-23 to 2^13 (a half of 2^-23 is f16's least number, 6 x 2^13 below its greatest) and NaN.
__device__ __forceinline__ u32x4 widen_e2m1_f16(uint32_t eight, float scale) {
  return u32x4{__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(eight, scale, 0)), __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(eight, scale, 1)),
               __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(eight, scale, 2)), __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(eight, scale, 3))};
}
struct QuantiseArgs {
  Rows q, values, x;      // values.data: nullptr if there is none
  uint32_t cols, pieces;  // pieces of a row of x
  uint32_t padded, down, along;   // pieces of a row with those that would complete its last block; how many rows and pieces further 256 pieces are
  uint64_t all;           // rows padded
};

// The greatest magnitude of a piece, as a binary32's bits.
__device__ __forceinline__ uint32_t greatest(const Piece<float>& p) {
  const u32x4 v = __builtin_bit_cast(u32x4, p) & 0x7FFFFFFFu;
  return max(max(v.x, v.y), max(v.z, v.w));
}
template <class T>
__device__ __forceinline__ uint32_t greatest(const Piece<T>& p) {
  typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));
  const u32x4 v = __builtin_bit_cast(u32x4, p) & 0x7FFF7FFFu;
  auto pairs = [](uint32_t x, uint32_t y) { return __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(u16x2, x), __builtin_bit_cast(u16x2, y))); };
  const uint32_t both = pairs(pairs(v.x, v.y), pairs(v.z, v.w));
  return __builtin_bit_cast(uint32_t, widen(__builtin_bit_cast(T, static_cast<uint16_t>(max(both >> 16, both & 0xFFFFu)))));
}

// Elements divided by s, as the instructions for it round them: to nearest even, 6 at most.  s as a binary32's bits: an exponent of 0 is 2^-127 to them.
__device__ __forceinline__ uint32_t to_e2m1(const Piece<float>& p, float s) {
  uint32_t c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(0u, p.v[0], p.v[1], s, 0);
  return __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, p.v[2], p.v[3], s, 1);
}
__device__ __forceinline__ uint32_t to_e2m1(const Piece<__bf16>& p, float s) {
  uint32_t c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(0u, bf16x2{p.v[0], p.v[1]}, s, 0);
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, bf16x2{p.v[2], p.v[3]}, s, 1);
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, bf16x2{p.v[4], p.v[5]}, s, 2);
  return __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, bf16x2{p.v[6], p.v[7]}, s, 3);
}
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
__device__ __forceinline__ uint32_t to_e2m1(const Piece<_Float16>& p, float s) {
  uint32_t c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f16(0u, f16x2{p.v[0], p.v[1]}, s, 0);
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f16(c, f16x2{p.v[2], p.v[3]}, s, 1);
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f16(c, f16x2{p.v[4], p.v[5]}, s, 2);
  return __builtin_amdgcn_cvt_scalef32_pk_fp4_f16(c, f16x2{p.v[6], p.v[7]}, s, 3);
}

// What codes stand for: exact in f32 and bf16, which have all these powers of two, and in f16, whose elements are multiples of 2^-24 below 2^16.
__device__ __forceinline__ void from_e2m1(uint32_t codes, float s, Piece<float>& p) {
  typedef float f32x2 __attribute__((ext_vector_type(2)));
  const f32x2 a = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, s, 0), b = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, s, 1);
  p.v[0] = a.x;
  p.v[1] = a.y;
  p.v[2] = b.x;
  p.v[3] = b.y;
}
__device__ __forceinline__ void from_e2m1(uint32_t codes, float s, Piece<__bf16>& p) { p = __builtin_bit_cast(Piece<__bf16>, widen_e2m1(codes, s)); }
__device__ __forceinline__ void from_e2m1(uint32_t codes, float s, Piece<_Float16>& p) { p = __builtin_bit_cast(Piece<_Float16>, widen_e2m1_f16(codes, s)); }

// A block's scale is 2^(floor(log2 of its greatest element) - 2), so that the greatest lies in [4, 8) and becomes 4 or 6; an element is its quotient, rounded to nearest even.
// A lane has 16 bytes of a row, and the neighbours that share a block (4 of 16-bit elements, 8 of 32-bit) its greatest element; NV of them a lane, every load
// issued before the first is waited for.  Bound by memory: 4096 x 7168 bf16 13.7 us, 5.4 TB/s, with the values that the codes stand for 23.1, 5.8 TB/s; 128 rows of it 4.7 and
// 999 x 2043 f32 with them 5.2, one load's latency and a launch.
template <class T, uint32_t NV, bool ONCE>
__global__ __launch_bounds__(256) void quantise_kernel(QuantiseArgs a) {
  constexpr uint32_t N = Piece<T>::N, SHARE = kMx4Block / N;
  const uint64_t first = blockIdx.x * static_cast<uint64_t>(256u * NV) + threadIdx.x;
  uint64_t row = first >> 32 == 0u ? static_cast<uint32_t>(first) / a.padded : first / a.padded;
  uint32_t at = static_cast<uint32_t>(first - row * a.padded);
  Piece<T> x[NV];
  uint64_t rows[NV];
  uint32_t pieces[NV];
#pragma unroll
  for (uint32_t k = 0; k < NV; ++k) {
    rows[k] = row;
    pieces[k] = first + k * 256u < a.all ? at : 0xFFFFFFFFu;   // behind the last row: nothing
    if (pieces[k] < a.pieces) x[k] = load_piece_once<T>(a.x.data + row * a.x.stride, at);
    else x[k] = Piece<T>{};
    row += a.down;
    at += a.along;
    if (at >= a.padded) {
      at -= a.padded;
      ++row;
    }
  }
#pragma unroll
  for (uint32_t k = 0; k < NV; ++k) {
    const uint32_t valid = valid_of<T>(pieces[k], a.pieces, a.cols);
    blank(x[k], valid);
    uint32_t most = greatest(x[k]);
    most = max(most, static_cast<uint32_t>(__builtin_amdgcn_mov_dpp(static_cast<int>(most), 0xB1, 0xF, 0xF, true)));   // a neighbour's
    most = max(most, static_cast<uint32_t>(__builtin_amdgcn_mov_dpp(static_cast<int>(most), 0x4E, 0xF, 0xF, true)));   // the other pair's
    if constexpr (SHARE == 8u) most = max(most, static_cast<uint32_t>(__builtin_amdgcn_mov_dpp(static_cast<int>(most), 0x141, 0xF, 0xF, true)));   // of 8 lanes, the other end's
    const bool finite = most < 0x7F800000u;
    const uint32_t exponent = most >> 23, byte = !finite ? 255u : exponent < 2u ? 0u : exponent - 2u;
    const float s = __builtin_bit_cast(float, byte << 23);
    const uint32_t codes = finite ? to_e2m1(x[k], s) : 0u;
    if (valid == 0u) continue;
    char* q = a.q.data + rows[k] * a.q.stride + pieces[k] * static_cast<uint64_t>(N / 2u);
    if (valid >= N) {
      if constexpr (N == 8u) *reinterpret_cast<uint32_t*>(q) = codes;
      else *reinterpret_cast<uint16_t*>(q) = static_cast<uint16_t>(codes);
    } else {
#pragma unroll
      for (uint32_t i = 0; i < N; i += 2u)
        if (i < valid) q[i / 2u] = static_cast<char>(codes >> (4u * i));
    }
    if (threadIdx.x % SHARE == 0u) reinterpret_cast<uint8_t*>(a.q.scales + rows[k] * a.q.scale_stride)[pieces[k] / SHARE] = static_cast<uint8_t>(byte);
    if (a.values.data != nullptr) {
      Piece<T> out;
      from_e2m1(codes, s, out);
      store_piece<ONCE>(a.values.data + rows[k] * a.values.stride, pieces[k], out, valid);
    }
  }
}

// ---- products ---------------------------------------------------------------------------------------
//
// out[i, n] = sum_k a[index[i], k] b[g, n, k] with b in microscaled 4 bits.  A lane has of a row 32 elements at a time, a block with a scale of its own.

typedef int i32x8 __attribute__((ext_vector_type(8)));

// Rows in 4 bits too: the matrix instruction for them takes the blocks' scales.  It has the products of a block exactly and adds the four
// blocks one after the other in binary32.
enum Mx4Rows : uint32_t { kRows4, kRowsBf16, kRowsF16 };

// f16 has 11 bits, which are two bf16 exactly: the first 8 of them and what is left, with the same sign.  (The nearest bf16 of the greatest f16 is above them all, and its product may
// be past binary32 where theirs is not.)  What an infinity leaves is any number, for the difference, NaN, would make every sum of the row NaN.
// Twice the products, and 5 operations for an element: rows in their own order, 8192^3 2390 us, 1100 where no scale asks for it, 16 rows in 8 groups, 7168 -> 2048, 20.3 and 14.9.
__device__ __forceinline__ void split_f16(u32x4 v, u32x4& high, u32x4& low) {
  const f16x8 f = __builtin_bit_cast(f16x8, v);
  auto upper_halves = [](float x, float y) { return __builtin_amdgcn_perm(__builtin_bit_cast(uint32_t, y), __builtin_bit_cast(uint32_t, x), 0x07060302u); };   // two bf16
  auto left = [](float x) { return fminf(x - __builtin_bit_cast(float, __builtin_bit_cast(uint32_t, x) & 0xFFFF0000u), 1024.0f); };   // (the lesser of NaN and a number is the number; 224 is the greatest other)
#pragma unroll
  for (uint32_t i = 0; i < 4u; ++i) {
    const float x = static_cast<float>(f[2u * i]), y = static_cast<float>(f[2u * i + 1u]);
    high[i] = upper_halves(x, y);
    low[i] = upper_halves(left(x), left(y));
  }
}

// Scales are the lowest bytes.
__device__ __forceinline__ f32x4 multiply_4(u32x4 w, uint32_t sw, u32x4 x, uint32_t sx, f32x4 acc) {
  const i32x8 vw{static_cast<int>(w.x), static_cast<int>(w.y), static_cast<int>(w.z), static_cast<int>(w.w), 0, 0, 0, 0};
  const i32x8 vx{static_cast<int>(x.x), static_cast<int>(x.y), static_cast<int>(x.z), static_cast<int>(x.w), 0, 0, 0, 0};
  return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(vw, vx, acc, 4, 4, 0, static_cast<int>(sw), 0, static_cast<int>(sx));
}

// 64 lanes' 4 bytes from memory into the LDS at `to`, as load_to_lds().
__device__ __forceinline__ void load_word_to_lds(const char* from, uint32_t to) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dword %1, off" ::"s"(to), "v"(from) : "m0");
}

// Scales by which weights are exact as f16.  (That of NaN is left to the other way.)
__device__ __forceinline__ bool exact_in_f16(uint32_t scale) { return scale - (127u - 23u) <= 36u; }

// ---- tiles, rows in 4 bits --------------------------------------------------------------------------

// As product_tile_kernel: a stage is 128 bytes along the sum, 256 elements, and is multiplied in two halves; a half is one matrix instruction for
// 16 x 16 of the output.  The LDS holds two stages of each operand, or RING: three where a compute unit has one small tile (64 x 64 or 64 x 128; of 64 x 128, 2551 rows, 5208 -> 523, 20.9 us with two and
// 18.5 with three; five take as long: what is left is a stage's chain of reads, products and addresses).  When every wavefront has read its last fragments of a stage, a little into its
// second half, the stage RING further is asked for in its place, by loads that SPREAD rows of blocks have between them; the barrier there, which the
// next stage's arrival is waited for at too, is the only one in a stage.
// Scales come 32 bytes of a row at a time, for four stages, into one of two places: a load of 64 words touches as few rows as one of 64 pieces does.  (4 bytes of
// 64 rows at every stage: 8192^3 388 us, 306 without them.)
// Bound by the loads into the LDS where the sum is long: 8192^3 by 256 x 256 313 to 338 us, 3.5 to 3.3 PFLOP/s, half of what the instruction does out of registers; by the one round
// of tiles where groups are ragged: 4096 rows in 16 groups, 7168 -> 2048, 69 us by 192 x 256, about 240 tiles, half of them the last rows of a group.
template <uint32_t BM, uint32_t BN, uint32_t WR, uint32_t WC, uint32_t SPREAD, uint32_t RING>
__global__ __launch_bounds__(WR * WC * 64) void mx4_tile_kernel(ProductArgs a) {
  constexpr uint32_t THREADS = WR * WC * 64u, SIDE = 16u, NA = BM / WR / SIDE, NB = BN / WC / SIDE, EACH = THREADS / 8u;   // rows of a load
  constexpr uint32_t A_LOADS = BM / EACH, B_LOADS = BN / EACH, LOADS = A_LOADS + B_LOADS, S_LOADS = (LOADS + 1u) / 2u;   // of scales, in the first two of four stages
  static_assert(RING == 2u || RING == 3u);   // scales of the first two of four stages have come when all but the newest stage's loads have
  constexpr uint32_t A_STAGE = BM * kStageBytes, B_STAGE = BN * kStageBytes, S_STAGE = (BM + BN) * 32u;
  static_assert(BM % EACH == 0u && BN % EACH == 0u);
  __shared__ __align__(1024) char lds_a[RING * A_STAGE], lds_b[RING * B_STAGE], lds_s[2u * S_STAGE];
  const char* zeros = reinterpret_cast<const char*>(page_of_zeros);
  asm volatile("" : "+s"(zeros));   // an address in registers: not looked up again at every load
  const uint32_t across = (a.wide + BN - 1u) / BN;
  Group g;
  uint32_t r0, c0;
  if (!find_tile(a, BM, across, g, r0, c0)) return;
  c0 *= BN;
  const char *const x_data = a.a.data, *const x_scales = a.a.scales, *const w_scales = a.b.scales;
  const uint64_t x_stride = a.a.stride, x_scale_stride = a.a.scale_stride, w_scale_stride = a.b.scale_stride, w_stride = a.b.stride;
  const uint32_t x_rows = a.indexed_rows, wide = a.wide;
  const uint64_t w0 = static_cast<uint64_t>(g.index) * a.wide;
  const uint32_t bytes = (a.cols + 1u) / 2u, words = (a.cols + 127u) / 128u, steps = (bytes + kStageBytes - 1u) / kStageBytes;

  // Load i of an operand is of rows i EACH + thread / 8, a piece or, of scales, a word each.  Rows and columns past the tile's end stand for its last ones: what
  // they make is not stored.  Pieces lie in the LDS as Operand<true> has them, words at word ^ (row / 8 % 2).
  const uint32_t own_row = threadIdx.x / 8u, own_piece = (threadIdx.x % 8u ^ (own_row >> 1 & 7u)) * 16u, own_word = threadIdx.x % 8u ^ (own_row >> 3 & 1u);
  uint32_t row[A_LOADS];   // of x; one that it has not stands for zeros
  const char* lb = a.b.data + (w0 + min(c0 + own_row, a.wide - 1u)) * a.b.stride + own_piece;   // w's rows lie at a constant distance
  uint32_t columns = 0u;   // bit i: w has the row of load i
#pragma unroll
  for (uint32_t i = 0; i < A_LOADS; ++i) {
    row[i] = min(r0 + i * EACH + own_row, g.end - 1u);
    if (a.index != nullptr) row[i] = static_cast<uint32_t>(a.index[row[i]]);
  }
#pragma unroll
  for (uint32_t i = 0; i < B_LOADS; ++i) columns |= c0 + i * EACH + own_row < a.wide ? 1u << i : 0u;
  const uint32_t mine = __builtin_amdgcn_readfirstlane(threadIdx.x & ~63u);
  const uint32_t here_a = lds_address(lds_a) + mine * 16u, here_b = lds_address(lds_b) + mine * 16u, here_s = lds_address(lds_s) + mine * 4u;
  // Load i of stage k: rows, then columns.  What lies behind the end of the sum, in its last stage, comes from a page of zeros.
  auto load = [&](uint32_t k, uint32_t i, bool last) {
    const bool behind = last && k * kStageBytes + own_piece >= bytes;
    if (i < A_LOADS) {
      // (a row's number is all that is kept of it from one load to the next)
      uint32_t r = row[i];
      asm volatile("" : "+v"(r));
      const char* from = x_data + k * static_cast<uint64_t>(kStageBytes) + r * x_stride + own_piece;
      if (behind || r >= x_rows) from = zeros;
      load_to_lds(from, __builtin_amdgcn_readfirstlane(here_a + k % RING * A_STAGE + i * THREADS * 16u));
    } else {
      const uint32_t n = i - A_LOADS;
      const char* from = columns >> n & 1u ? lb + n * EACH * w_stride : lb;
      if (behind) from = zeros;
      load_to_lds(from, __builtin_amdgcn_readfirstlane(here_b + k % RING * B_STAGE + n * THREADS * 16u));
      if (n + 1u == B_LOADS) lb += kStageBytes;
    }
  };
  // Load i of the scales of stages 4 j to 4 j + 3.
  auto load_scales = [&](uint32_t j, uint32_t i) {
    const uint32_t word = j * 8u + own_word;
    const char* from;
    uint32_t r = i < A_LOADS ? row[i < A_LOADS ? i : 0u] : own_row;
    asm volatile("" : "+v"(r));
    if (i < A_LOADS) {
      from = x_scales + r * x_scale_stride + word * 4u;
      if (r >= x_rows) from = zeros;
    } else {
      from = w_scales + (w0 + min(c0 + (i - A_LOADS) * EACH + r, wide - 1u)) * w_scale_stride + word * 4u;
    }
    if (word >= words) from = zeros;
    load_word_to_lds(from, __builtin_amdgcn_readfirstlane(here_s + j % 2u * S_STAGE + i * THREADS * 4u));
  };
  // The piece and the word of scales that the sum ends in have what is behind the row's end: that is blanked, for a scale may be NaN.
  const uint32_t tail = a.cols % 256u;   // elements in the last stage
  const bool ragged = tail % 128u != 0u;
  auto trim = [&] {
    const uint32_t k = steps - 1u, p = tail / 32u, in = tail % 32u, scales = (tail + 31u) / 32u % 4u;
    for (uint32_t r = threadIdx.x; r < BM + BN; r += THREADS) {
      const uint32_t in_operand = r < BM ? r : r - BM;
      if (in != 0u) {
        uint32_t* piece = reinterpret_cast<uint32_t*>((r < BM ? lds_a + k % RING * A_STAGE : lds_b + k % RING * B_STAGE) + in_operand * kStageBytes + ((p ^ (in_operand >> 1 & 7u)) << 4));
#pragma unroll
        for (uint32_t i = 0; i < 4u; ++i)
          if (in < (i + 1u) * 8u) piece[i] &= in <= i * 8u ? 0u : (1u << (in - i * 8u) * 4u) - 1u;
      }
      if (scales != 0u) reinterpret_cast<uint32_t*>(lds_s + k / 4u % 2u * S_STAGE + r * 32u)[(words - 1u) % 8u ^ (r >> 3 & 1u)] &= (1u << scales * 8u) - 1u;
    }
    wait_for_reads<0>();   // and the writes
  };

  const uint32_t wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64u), lane = threadIdx.x & 63u, quarter = lane / 16u;
  const uint32_t ra = wave / WC * (BM / WR), cb = wave % WC * (BN / WC);
  // Blocks of rows that the wavefront has in this tile, at most NA: the others are not multiplied
  const uint32_t high = __builtin_amdgcn_readfirstlane(r0 + ra < g.end ? min((g.end - r0 - ra + SIDE - 1u) / SIDE, NA) : 0u);
  f32x4 acc[NB][NA] = {};
  u32x4 fa[NA], fb[2][NB];
  uint32_t sa[NA], sb[2][NB];
  // Where the lane reads: of row lane % 16 of 16, the piece of its quarter, and the byte of its scale: stage k's half has word 2 (k % 4) + half.
  const uint32_t r16 = lane % 16u, in_piece = (quarter ^ (r16 >> 1 & 7u)) << 4, in_word = (lane >> 3 & 1u) * 4u;
  const uint32_t at_a = lds_address(lds_a) + (ra + r16) * kStageBytes, at_b = lds_address(lds_b) + (cb + r16) * kStageBytes, at_s = lds_address(lds_s) + r16 * 32u + quarter;   // (of scales, for the first rows of x)
  struct Places {
    uint32_t a, b, sa, sb;
  };
  auto places = [&](uint32_t k, uint32_t half) {
    const uint32_t piece = in_piece ^ half * 64u;
    Places p{at_a + k % RING * A_STAGE + piece, at_b + k % RING * B_STAGE + piece, at_s + k / 4u % 2u * S_STAGE + ra * 32u + ((k % 4u * 8u + half * 4u) ^ in_word), 0u};
    p.sb = p.sa + (BM + cb - ra) * 32u;
    asm volatile("" : "+v"(p.a), "+v"(p.b), "+v"(p.sa), "+v"(p.sb));   // four registers, and not one for every stage and half
    return p;
  };
  auto read_a = [&](const Places& p, uint32_t m) {
    fa[m] = *reinterpret_cast<const __attribute__((address_space(3))) u32x4*>(static_cast<uintptr_t>(p.a + m * SIDE * kStageBytes));
    sa[m] = *reinterpret_cast<const __attribute__((address_space(3))) uint8_t*>(static_cast<uintptr_t>(p.sa + m * SIDE * 32u));
  };
  auto read_b = [&](const Places& p, uint32_t half, uint32_t n) {
    sb[half][n] = *reinterpret_cast<const __attribute__((address_space(3))) uint8_t*>(static_cast<uintptr_t>(p.sb + n * SIDE * 32u));
    fb[half][n] = *reinterpret_cast<const __attribute__((address_space(3))) u32x4*>(static_cast<uintptr_t>(p.b + n * SIDE * kStageBytes));
  };
  // STEADY: stage k + RING is there to be asked for, and is not the last
  auto work = [&](uint32_t k, auto steady) {
    constexpr bool STEADY = decltype(steady)::value;
    constexpr uint32_t FROM = NA / 4u == 0u ? 1u : NA / 4u, ALL = LOADS + S_LOADS, OVER = SPREAD;
    const bool more = STEADY || k + RING < steps, last = !STEADY && k + RING + 1u == steps, scales = k % 4u < 2u && (k / 4u + 1u) * 4u < steps;
    // the first half's fragments are fa and fb[0]: multiply, and read the second half's
    Places p = places(k, 1);
#pragma unroll
    for (uint32_t n = 0; n < NB; ++n) read_b(p, 1, n);
#pragma unroll
    for (uint32_t m = 0; m < NA; ++m) {
      if (m < high)
#pragma unroll
        for (uint32_t n = 0; n < NB; ++n) acc[n][m] = multiply_4(fb[0][n], sb[0][n], fa[m], sa[m], acc[n][m]);
      __builtin_amdgcn_sched_barrier(0);   // the next fragment takes the registers of this one
      read_a(p, m);
      __builtin_amdgcn_sched_barrier(0);
    }
    p = places(k + 1u, 0);
#pragma unroll
    for (uint32_t m = 0; m < NA; ++m) {
      if (m < high)
#pragma unroll
        for (uint32_t n = 0; n < NB; ++n) acc[n][m] = multiply_4(fb[1][n], sb[1][n], fa[m], sa[m], acc[n][m]);
      __builtin_amdgcn_sched_barrier(0);
      if (m + 1u == FROM) {
        // every wavefront has its last fragments of the stage, and the next stage is there
        if (STEADY || k + RING - 1u < steps) asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"((RING - 2u) * LOADS) : "memory");
        else asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
        if (!STEADY && ragged && k + 2u == steps) trim();
#pragma unroll
        for (uint32_t n = 0; n < NB; ++n) read_b(p, 0, n);   // behind the last stage: read, and not used
#pragma unroll
        for (uint32_t i = 0; i < FROM; ++i) read_a(p, i);
      }
      if (m >= FROM) read_a(p, m);
#pragma unroll
      for (uint32_t i = 0; i < ALL; ++i)
        if (m + 1u >= FROM && i * OVER / ALL == m + 1u - FROM) {
          if (i < LOADS) {
            if (more) load(k + RING, i, last);
          } else if (scales) {
            if (k % 4u == 0u) load_scales(k / 4u + 1u, i - LOADS);
            else if (i - LOADS + S_LOADS < LOADS) load_scales(k / 4u + 1u, i - LOADS + S_LOADS);
          }
        }
      __builtin_amdgcn_sched_barrier(0);
    }
  };
  if (steps != 0u) {
#pragma unroll
    for (uint32_t i = 0; i < LOADS; ++i) load_scales(0, i);
#pragma unroll
    for (uint32_t k = 0; k < RING; ++k)
      if (k < steps) {
#pragma unroll
        for (uint32_t i = 0; i < LOADS; ++i) load(k, i, k + 1u == steps);
      }
    if (steps >= RING) wait_for_loads<(RING - 1u) * LOADS>();
    else wait_for_loads<0>();
    if (ragged && steps == 1u) trim();
    const Places p = places(0, 0);
#pragma unroll
    for (uint32_t n = 0; n < NB; ++n) read_b(p, 0, n);
#pragma unroll
    for (uint32_t m = 0; m < NA; ++m) read_a(p, m);
    uint32_t k = 0;
    for (; k + RING + 1u < steps; ++k) work(k, std::true_type{});
    for (; k < steps; ++k) work(k, std::false_type{});
  }
#pragma unroll
  for (uint32_t m = 0; m < NA; ++m) {
    constexpr uint32_t BLOCKS = NB % 4u == 0u ? 4u : 2u;
    const uint32_t top = r0 + ra + m * SIDE, rows = top < g.end ? g.end - top : 0u;   // of the 16 rows that the wavefront has
#pragma unroll
    for (uint32_t n = 0; n < NB; n += BLOCKS) {
      f32x4 v[BLOCKS];
#pragma unroll
      for (uint32_t b = 0; b < BLOCKS; ++b) v[b] = acc[n + b][m];
      store_blocks<(BM > 128u)>(a, top, rows, c0 + cb + n * SIDE, a.wide, v);
    }
  }
}

// ---- tiles, rows in 16 bits -------------------------------------------------------------------------

// A workgroup computes BM x BN of the output, 8 / WC x WC wavefronts a part each, 64 elements of the sum at a time, a step: 128 bytes of x's rows and 32 of w's, which come
// 128 at a time, for four steps.  The LDS holds AHEAD steps of x, and two times four of w with their scales.  A lane has 16 neighbouring elements of a step, half a block: they
// go into two matrix instructions, whose order of the elements is the same for both operands.  While a step is multiplied, the next one's fragments are read; when every
// wavefront has had its last fragment of the step, a quarter into its products, the step AHEAD further takes its place.
// Bound by what prepares the products: a fragment of w is widened in registers, 8 elements an instruction or four, under the matrix instructions of 16 bits: 8192^3 in bf16 952 to 1020 us,
// 1.15 to 1.08 PFLOP/s of 1.45, in f16 1140 to 1195; 4000 rows in 4 groups, 7168 -> 2048, 119 and 138; 2999 rows in 24 groups, 2043 -> 1003, in f16 28 by 64 x 128: one
// round of tiles, two on a compute unit, whose 32 steps take twice the products' time, most of them in the barrier and the waits that a step of so few products has too.
template <bool F16, uint32_t BM, uint32_t BN, uint32_t WC, uint32_t AHEAD>
__global__ __launch_bounds__(512) void mx4_wide_kernel(ProductArgs a) {
  constexpr uint32_t SIDE = 16u, WR = 8u / WC, NA = BM / WR / SIDE, NB = BN / WC / SIDE, A_LOADS = BM / 64u, B_LOADS = BN / 64u, FROM = NA / 4u == 0u ? 1u : NA / 4u;
  constexpr uint32_t A_STEP = BM * 128u, B_STAGE = BN * 128u, S_STAGE = 2048u;   // scales: 8 bytes of 256 rows
  static_assert(AHEAD >= 3u && AHEAD <= 5u);
  __shared__ __align__(1024) char lds_a[AHEAD * A_STEP], lds_b[2u * B_STAGE], lds_s[2u * S_STAGE];
  const char* zeros = reinterpret_cast<const char*>(page_of_zeros);
  asm volatile("" : "+s"(zeros));
  const uint32_t across = (a.wide + BN - 1u) / BN;
  Group g;
  uint32_t r0, c0;
  if (!find_tile(a, BM, across, g, r0, c0)) return;
  c0 *= BN;
  const uint64_t w0 = static_cast<uint64_t>(g.index) * a.wide;
  const uint64_t w_stride = a.b.stride;
  const uint32_t cols = a.cols, w_bytes = (cols + 1u) / 2u, words = (cols + 127u) / 128u, steps = (cols + 63u) / 64u, stages = (cols + 255u) / 256u;

  // Load i of an operand is of rows 64 i + thread / 8, a piece of 16 bytes each.  Rows and columns past the tile's end stand for its last ones.
  const uint32_t own_row = threadIdx.x / 8u, own_piece = (threadIdx.x % 8u ^ (own_row >> 1 & 7u)) * 16u;
  const char* la[A_LOADS];
  uint32_t still = 0u;   // bit i: the piece of load i is of a row of zeros and stays where it is
#pragma unroll
  for (uint32_t i = 0; i < A_LOADS; ++i) {
    uint32_t r = min(r0 + i * 64u + own_row, g.end - 1u);
    if (a.index != nullptr) r = static_cast<uint32_t>(a.index[r]);
    la[i] = r < a.indexed_rows ? a.a.data + r * a.a.stride + own_piece : zeros;
    still |= r < a.indexed_rows ? 0u : 1u << i;
  }
  const char* lb = a.b.data + (w0 + min(c0 + own_row, a.wide - 1u)) * w_stride + own_piece;
  const char* ls = a.b.scales + (w0 + min(c0 + min(threadIdx.x / 2u, BN - 1u), a.wide - 1u)) * a.b.scale_stride + threadIdx.x % 2u * 4u;
  uint32_t columns = 0u;   // bit i: w has the row of load i
#pragma unroll
  for (uint32_t i = 0; i < B_LOADS; ++i) columns |= c0 + i * 64u + own_row < a.wide ? 1u << i : 0u;
  const uint32_t mine = __builtin_amdgcn_readfirstlane(threadIdx.x & ~63u);
  const uint32_t here_a = lds_address(lds_a) + mine * 16u, here_b = lds_address(lds_b) + mine * 16u, here_s = lds_address(lds_s) + mine * 4u;
  auto load_a = [&](uint32_t t, uint32_t slot, uint32_t i, bool inside) {   // inside: not the last step, whose end may lie in it
    const char* from = la[i];
    if (!inside && t * 64u + own_piece / 2u >= cols) from = zeros;
    load_to_lds(from, __builtin_amdgcn_readfirstlane(here_a + slot * A_STEP + i * 8192u));
    la[i] += still >> i & 1u ? 0u : 128u;
  };
  auto load_b = [&](uint32_t k, uint32_t i, bool inside) {   // the last one of a stage is of its scales
    if (i < B_LOADS) {
      const char* from = columns >> i & 1u ? lb + i * 64u * w_stride : lb;
      if (!inside && k * 128u + own_piece >= w_bytes) from = zeros;
      load_to_lds(from, __builtin_amdgcn_readfirstlane(here_b + k % 2u * B_STAGE + i * 8192u));
      if (i + 1u == B_LOADS) lb += 128u;
    } else {
      load_word_to_lds(inside || k * 2u + threadIdx.x % 2u < words ? ls : zeros, __builtin_amdgcn_readfirstlane(here_s + k % 2u * S_STAGE));
      ls += 8u;
    }
  };
  // What is behind the row's end in the piece that it ends in, and in the word of scales, is blanked: a scale may be NaN.
  auto trim_a = [&](uint32_t slot) {
    if (threadIdx.x < BM) {
      const uint32_t r = threadIdx.x, in = cols % 8u;
      uint16_t* piece = reinterpret_cast<uint16_t*>(lds_a + slot * A_STEP + r * 128u + ((cols % 64u / 8u ^ (r >> 1 & 7u)) << 4));
#pragma unroll
      for (uint32_t i = 0; i < 8u; ++i)
        if (i >= in) piece[i] = 0;
    }
    wait_for_reads<0>();
  };
  auto trim_b = [&] {
    if (threadIdx.x < BN) {
      const uint32_t r = threadIdx.x, odd = (stages - 1u) % 2u, tail = cols % 256u, in = tail % 32u, scales = (tail + 31u) / 32u;
      if (in != 0u) {
        uint32_t* piece = reinterpret_cast<uint32_t*>(lds_b + odd * B_STAGE + r * 128u + ((tail / 32u ^ (r >> 1 & 7u)) << 4));
#pragma unroll
        for (uint32_t i = 0; i < 4u; ++i)
          if (in < (i + 1u) * 8u) piece[i] &= in <= i * 8u ? 0u : (1u << (in - i * 8u) * 4u) - 1u;
      }
      if (scales % 4u != 0u) reinterpret_cast<uint32_t*>(lds_s + odd * S_STAGE + r * 8u)[scales / 4u] &= (1u << scales % 4u * 8u) - 1u;
    }
    wait_for_reads<0>();
  };

  const uint32_t wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64u), lane = threadIdx.x & 63u, quarter = lane / 16u, r16 = lane % 16u;
  const uint32_t ra = wave / WC * (BM / WR), cb = wave % WC * (BN / WC);
  const uint32_t high = __builtin_amdgcn_readfirstlane(r0 + ra < g.end ? min((g.end - r0 - ra + SIDE - 1u) / SIDE, NA) : 0u);
  f32x4 acc[NB][NA] = {};
  u32x4 fa[NA][2];
  u32x2 fb[NB];
  uint32_t sb[NB];
  const uint32_t turned = r16 >> 1 & 7u, in_a = (quarter * 2u ^ turned) << 4;   // the lane's first piece; the second is at ^ 16
  auto read_a = [&](uint32_t slot, uint32_t m) {
    const char* at = lds_a + slot * A_STEP + (ra + m * SIDE + r16) * 128u;
    fa[m][0] = *reinterpret_cast<const u32x4*>(at + in_a);
    fa[m][1] = *reinterpret_cast<const u32x4*>(at + (in_a ^ 16u));
  };
  auto read_b = [&](uint32_t t, uint32_t n) {
    const uint32_t odd = t / 4u % 2u, block = t % 4u * 2u + quarter / 2u, r = cb + n * SIDE + r16;
    fb[n] = *reinterpret_cast<const u32x2*>(lds_b + odd * B_STAGE + r * 128u + ((block ^ turned) << 4) + quarter % 2u * 8u);
    sb[n] = *reinterpret_cast<const uint8_t*>(lds_s + odd * S_STAGE + r * 8u + block);
  };
  uint32_t slot = 0;
  // Step t, the STEP-th of its stage.  STEADY: all that is asked for is there.
  auto work = [&](uint32_t t, auto step, auto steady) {
    constexpr uint32_t STEP = decltype(step)::value;
    constexpr bool STEADY = decltype(steady)::value;
    const uint32_t next = slot + 1u == AHEAD ? 0u : slot + 1u;
    const bool more = STEADY || t + AHEAD < steps, more_b = STEP == 3u && (STEADY || t / 4u + 2u < stages);
    u32x4 w[NB][2];
    bool in_f16 = F16;
    if constexpr (F16) {
#pragma unroll
      for (uint32_t n = 0; n < NB; ++n) in_f16 &= exact_in_f16(sb[n]);
      in_f16 = __all(in_f16);
    }
    if (F16 && in_f16) {
#pragma unroll
      for (uint32_t n = 0; n < NB; ++n)
#pragma unroll
        for (uint32_t j = 0; j < 2u; ++j) w[n][j] = widen_e2m1_f16(fb[n][j], __builtin_bit_cast(float, sb[n] << 23));
    } else {
#pragma unroll
      for (uint32_t n = 0; n < NB; ++n)
#pragma unroll
        for (uint32_t j = 0; j < 2u; ++j) w[n][j] = widen_e2m1(fb[n][j], __builtin_bit_cast(float, sb[n] << 23));
    }
#pragma unroll
    for (uint32_t m = 0; m < NA; ++m) {
      if (m < high) {
        if (F16 && in_f16) {
#pragma unroll
          for (uint32_t j = 0; j < 2u; ++j)
#pragma unroll
            for (uint32_t n = 0; n < NB; ++n) acc[n][m] = multiply<kF16>(w[n][j], fa[m][j], acc[n][m]);
        } else {
#pragma unroll
          for (uint32_t j = 0; j < 2u; ++j) {
            u32x4 upper = fa[m][j], lower{};
            if constexpr (F16) split_f16(fa[m][j], upper, lower);
#pragma unroll
            for (uint32_t n = 0; n < NB; ++n) {
              acc[n][m] = multiply<kBf16>(w[n][j], upper, acc[n][m]);
              if constexpr (F16) acc[n][m] = multiply<kBf16>(w[n][j], lower, acc[n][m]);
            }
          }
        }
      }
      __builtin_amdgcn_sched_barrier(0);   // the next fragments take the registers of these
      if (m + 1u == FROM) {
        // every wavefront has the step's fragments, and the next step is there: of later ones, all that was asked for may be under way
        // (that is of x the steps from t + 2 on, and of w a stage, if it was asked for since)
        constexpr uint32_t LATER = (AHEAD - 2u) * A_LOADS + (STEP + 3u <= AHEAD ? B_LOADS + 1u : 0u);
        if (STEADY) asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(LATER) : "memory");
        else asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
        if (!STEADY && cols % 8u != 0u && t + 2u == steps) trim_a(next);
        if (!STEADY && STEP == 3u && cols % 128u != 0u && t / 4u + 2u == stages) trim_b();
#pragma unroll
        for (uint32_t n = 0; n < NB; ++n) read_b(t + 1u, n);   // behind the last step: read, and not used
#pragma unroll
        for (uint32_t i = 0; i < FROM; ++i) read_a(next, i);
      }
      if (m >= FROM) read_a(next, m);
      if (m + 1u == FROM || NA == 1u) {
        if (more) {
#pragma unroll
          for (uint32_t i = 0; i < A_LOADS; ++i) load_a(t + AHEAD, slot, i, STEADY);
        }
      }
      if (m + 1u == NA && more_b) {
#pragma unroll
        for (uint32_t i = 0; i <= B_LOADS; ++i) load_b(t / 4u + 2u, i, STEADY);
      }
      __builtin_amdgcn_sched_barrier(0);
    }
    slot = next;
  };
  if (steps != 0u) {
    // in the order in which steps before the first would have asked for them, by which the waits count
#pragma unroll
    for (uint32_t i = 0; i <= B_LOADS; ++i) load_b(0, i, false);
#pragma unroll
    for (uint32_t t = 0; t < AHEAD; ++t)
      if (t < steps) {
#pragma unroll
        for (uint32_t i = 0; i < A_LOADS; ++i) load_a(t, t, i, false);
      }
    if (stages > 1u) {
#pragma unroll
      for (uint32_t i = 0; i <= B_LOADS; ++i) load_b(1, i, false);
    }
    if (steps > 4u && steps >= AHEAD) wait_for_loads<(AHEAD - 1u) * A_LOADS + B_LOADS + 1u>();
    else wait_for_loads<0>();
    if (cols % 8u != 0u && steps == 1u) trim_a(0);
    if (cols % 128u != 0u && stages == 1u) trim_b();
#pragma unroll
    for (uint32_t n = 0; n < NB; ++n) read_b(0, n);
#pragma unroll
    for (uint32_t m = 0; m < NA; ++m) read_a(0, m);
    using S0 = std::integral_constant<uint32_t, 0>;
    using S1 = std::integral_constant<uint32_t, 1>;
    using S2 = std::integral_constant<uint32_t, 2>;
    using S3 = std::integral_constant<uint32_t, 3>;
    uint32_t t = 0;
    for (; t + AHEAD + 8u < steps; t += 4u) {
      work(t, S0{}, std::true_type{});
      work(t + 1u, S1{}, std::true_type{});
      work(t + 2u, S2{}, std::true_type{});
      work(t + 3u, S3{}, std::true_type{});
    }
    for (; t < steps; t += 4u) {
      work(t, S0{}, std::false_type{});
      if (t + 1u < steps) work(t + 1u, S1{}, std::false_type{});
      if (t + 2u < steps) work(t + 2u, S2{}, std::false_type{});
      if (t + 3u < steps) work(t + 3u, S3{}, std::false_type{});
    }
  }
#pragma unroll
  for (uint32_t m = 0; m < NA; ++m) {
    constexpr uint32_t BLOCKS = NB % 4u == 0u ? 4u : 2u;
    const uint32_t top = r0 + ra + m * SIDE, rows = top < g.end ? g.end - top : 0u;   // of the 16 rows that the wavefront has
#pragma unroll
    for (uint32_t n = 0; n < NB; n += BLOCKS) {
      f32x4 v[BLOCKS];
#pragma unroll
      for (uint32_t b = 0; b < BLOCKS; ++b) v[b] = acc[n + b][m];
      store_blocks<false>(a, top, rows, c0 + cb + n * SIDE, a.wide, v);
    }
  }
}

// ---- few rows a group -------------------------------------------------------------------------------

// As product_few_kernel: 16 rows x WIDE columns, every wavefront a part of the sum, 256 elements of it at a time in turn with the others, through a ring of its own in
// the LDS.  Rows of x that the tile does not have are not asked for: what makes of theirs whatever lies there is not stored.
// Bound by memory: 128 rows of 4 bits in 32 groups, 7168 -> 2048, 49 us, 5.1 TB/s; 16 bf16 rows in 8 of them 14.4, 66 MB at 4.6 TB/s.
template <Mx4Rows X, uint32_t WIDE, uint32_t WAVES, uint32_t RING>
__global__ __launch_bounds__(WAVES * 64) void mx4_few_kernel(ProductArgs a) {
  constexpr uint32_t THREADS = WAVES * 64u, HIGH = 16u, NB = WIDE / 16u;
  constexpr uint32_t X_PITCH = X == kRows4 ? 128u : 512u, X_AT_ONCE = 1024u / X_PITCH, X_LOADS = HIGH / X_AT_ONCE;   // bytes of a row in a stage, rows of a load
  constexpr uint32_t W_LOADS = WIDE / 8u, SCALED = (X == kRows4 ? HIGH : 0u) + WIDE, S_LOADS = (SCALED * 2u + 63u) / 64u;   // rows that have scales: x's, then w's
  constexpr uint32_t W_AT = HIGH * X_PITCH, S_AT = W_AT + WIDE * 128u, STAGE = S_AT + S_LOADS * 256u;
  __shared__ __align__(1024) char lds[WAVES][RING][STAGE];
  const uint32_t across = (a.wide + WIDE - 1u) / WIDE, lane = threadIdx.x & 63u, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64u);
  Group g;
  uint32_t r0, c0;
  if (!find_tile(a, HIGH, across, g, r0, c0)) return;
  c0 *= WIDE;
  const uint64_t w0 = static_cast<uint64_t>(g.index) * a.wide;
  const char* zeros = reinterpret_cast<const char*>(page_of_zeros);
  asm volatile("" : "+s"(zeros));
  const uint32_t cols = a.cols, stages = (cols + 255u) / 256u, words = (cols + 127u) / 128u, w_bytes = (cols + 1u) / 2u, x_bytes = X == kRows4 ? w_bytes : cols * 2u;
  // how many loads bring x's rows, of 1, 2, 4 and 8
  const uint32_t have = __builtin_amdgcn_readfirstlane(min(g.end - r0, HIGH));
  uint32_t x_loads = 1u;
  while (x_loads < X_LOADS && x_loads * X_AT_ONCE < have) x_loads *= 2u;
  x_loads = __builtin_amdgcn_readfirstlane(x_loads);

  // Pieces of 16 bytes lie within a row so that 16 lanes that read the same of 16 rows meet different banks: of 8 at piece ^ (row / 2 % 8), of 32 at piece ^ row.
  auto row_of = [&](uint32_t r) {   // of x, or one that it has not
    r += r0;
    if (r >= g.end) return 0xFFFFFFFFu;
    return a.index != nullptr ? static_cast<uint32_t>(a.index[r]) : r;
  };
  const char* at_x[X_LOADS];
  uint32_t in_x[X_LOADS];   // where the lane's piece is in the stage, or past everything for a row of zeros
#pragma unroll
  for (uint32_t i = 0; i < X_LOADS; ++i) {
    const uint32_t r = i * X_AT_ONCE + lane / (X_PITCH / 16u), from = row_of(r), slot = lane % (X_PITCH / 16u);
    in_x[i] = (X == kRows4 ? slot ^ (r >> 1 & 7u) : slot ^ r) * 16u;
    at_x[i] = a.a.data + from * a.a.stride + in_x[i] + wave * X_PITCH;
    if (from >= a.indexed_rows) in_x[i] = 0x80000000u;
  }
  const uint32_t w_row = lane / 8u, w_piece = (lane % 8u ^ (lane / 16u & 3u)) * 16u;   // of rows 16 i + lane / 8; rows 8 further have it ^ 64
  const char* at_w = a.b.data + (w0 + min(c0 + w_row, a.wide - 1u)) * a.b.stride + wave * 128u;
  const uint64_t apart = 8u * a.b.stride;
  uint32_t columns = 0u;   // bit i: w has the row of load i
#pragma unroll
  for (uint32_t i = 0; i < W_LOADS; ++i) columns |= c0 + i * 8u + w_row < a.wide ? 1u << i : 0u;
  const char* at_s[S_LOADS];
  uint32_t no_s = 0u;   // bit i: zeros
#pragma unroll
  for (uint32_t i = 0; i < S_LOADS; ++i) {
    uint32_t r = (i * 64u + lane) / 2u;
    if (X == kRows4 && r < HIGH) {
      r = row_of(r);
      at_s[i] = a.a.scales + r * a.a.scale_stride;
      if (r >= a.indexed_rows) no_s |= 1u << i;
    } else {
      r = min(r - (X == kRows4 ? HIGH : 0u), WIDE - 1u);
      at_s[i] = a.b.scales + (w0 + min(c0 + r, a.wide - 1u)) * a.b.scale_stride;
    }
    at_s[i] += wave * 8u + lane % 2u * 4u;
  }
  const uint32_t base = lds_address(lds[wave]);
  auto load = [&](uint32_t k, uint32_t slot) {   // the wavefront's stages come in turn: wave, wave + WAVES, ...
    const uint32_t to = __builtin_amdgcn_readfirstlane(base + slot * STAGE);
#pragma unroll
    for (uint32_t i = 0; i < X_LOADS; ++i)
      if (i < x_loads) {
        const char* from = at_x[i];
        if (in_x[i] >= 0x80000000u || k * X_PITCH + in_x[i] >= x_bytes) from = zeros;
        load_to_lds(from, to + i * 1024u);
        at_x[i] += WAVES * X_PITCH;
      }
#pragma unroll
    for (uint32_t i = 0; i < W_LOADS; ++i) {
      const uint32_t piece = w_piece ^ i % 2u * 64u;
      const char* from = (columns >> i & 1u ? at_w + i * apart : at_w) + piece;
      if (k * 128u + piece >= w_bytes) from = zeros;
      load_to_lds(from, to + W_AT + i * 1024u);
    }
    at_w += WAVES * 128u;
#pragma unroll
    for (uint32_t i = 0; i < S_LOADS; ++i) {
      const char* from = at_s[i];
      if ((no_s >> i & 1u) || k * 2u + lane % 2u >= words) from = zeros;
      load_word_to_lds(from, to + S_AT + i * 256u);
      at_s[i] += WAVES * 8u;
    }
  };
  // All but the newest `newer` stages have come.
  constexpr uint32_t OTHER = W_LOADS + S_LOADS;
  auto wait = [&](uint32_t newer) {
    if (newer == 0u) wait_for_own_loads<0>();
    else if (newer == 1u || RING == 2u) {
      if (x_loads == 1u) wait_for_own_loads<OTHER + 1u>();
      else if (x_loads == 2u) wait_for_own_loads<OTHER + 2u>();
      else if (x_loads == 4u) wait_for_own_loads<OTHER + 4u>();
      else wait_for_own_loads<OTHER + 8u>();
    } else {
      if (x_loads == 1u) wait_for_own_loads<2u * OTHER + 2u>();
      else if (x_loads == 2u) wait_for_own_loads<2u * OTHER + 4u>();
      else if (x_loads == 4u) wait_for_own_loads<2u * OTHER + 8u>();
      else wait_for_own_loads<2u * OTHER + 16u>();
    }
  };
  const uint32_t r16 = lane % 16u, quarter = lane / 16u;
  f32x4 acc[NB] = {};
#pragma unroll
  for (uint32_t i = 0; i < RING; ++i)
    if (wave + i * WAVES < stages) load(wave + i * WAVES, i);
  uint32_t slot = 0;
  for (uint32_t k = wave; k < stages; k += WAVES) {
    if (k + (RING - 1u) * WAVES < stages) wait(RING - 1u);
    else if (RING == 3u && k + WAVES < stages) wait(1u);
    else wait(0u);
    char* stage = lds[wave][slot];
    if (k + 1u == stages && cols % 128u != 0u) {   // the piece and the word of scales that the rows end in
      const uint32_t tail = cols % 256u, p = tail / 32u, in = tail % 32u, scales = (tail + 31u) / 32u;
      for (uint32_t r = lane; r < SCALED; r += 64u) {
        const bool of_x = X == kRows4 && r < HIGH;
        const uint32_t row = of_x ? r : r - (X == kRows4 ? HIGH : 0u);
        if (in != 0u) {
          uint32_t* piece = reinterpret_cast<uint32_t*>(stage + (of_x ? 0u : W_AT) + row * 128u + ((p ^ (row >> 1 & 7u)) << 4));
#pragma unroll
          for (uint32_t i = 0; i < 4u; ++i)
            if (in < (i + 1u) * 8u) piece[i] &= in <= i * 8u ? 0u : (1u << (in - i * 8u) * 4u) - 1u;
        }
        if (scales % 4u != 0u) reinterpret_cast<uint32_t*>(stage + S_AT + r * 8u)[scales / 4u] &= (1u << scales % 4u * 8u) - 1u;
      }
      if (X != kRows4 && tail % 8u != 0u && lane < HIGH) {
        uint16_t* piece = reinterpret_cast<uint16_t*>(stage + lane * X_PITCH + ((tail / 8u ^ lane) << 4));
#pragma unroll
        for (uint32_t i = 0; i < 8u; ++i)
          if (i >= tail % 8u) piece[i] = 0;
      }
    }
    u32x4 fx[X == kRows4 ? 2u : 8u], fw[NB][2];
    uint32_t sx[2], sw[NB][2];
#pragma unroll
    for (uint32_t h = 0; h < 2u; ++h) {
      const uint32_t block = h * 4u + quarter, place = (block ^ (r16 >> 1 & 7u)) << 4;
      if constexpr (X == kRows4) {
        fx[h] = *reinterpret_cast<const u32x4*>(stage + r16 * 128u + place);
        sx[h] = *reinterpret_cast<const uint8_t*>(stage + S_AT + r16 * 8u + block);
      } else {
#pragma unroll
        for (uint32_t j = 0; j < 4u; ++j) fx[h * 4u + j] = *reinterpret_cast<const u32x4*>(stage + r16 * X_PITCH + ((block * 4u + j ^ r16) << 4));
      }
#pragma unroll
      for (uint32_t n = 0; n < NB; ++n) {
        fw[n][h] = *reinterpret_cast<const u32x4*>(stage + W_AT + (n * 16u + r16) * 128u + place);
        sw[n][h] = *reinterpret_cast<const uint8_t*>(stage + S_AT + ((X == kRows4 ? HIGH : 0u) + n * 16u + r16) * 8u + block);
      }
    }
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");   // the ring's place is free
    if (k + RING * WAVES < stages) load(k + RING * WAVES, slot);
    slot = slot + 1u == RING ? 0u : slot + 1u;
#pragma unroll
    for (uint32_t h = 0; h < 2u; ++h) {
      if constexpr (X == kRows4) {
#pragma unroll
        for (uint32_t n = 0; n < NB; ++n) acc[n] = multiply_4(fw[n][h], sw[n][h], fx[h], sx[h], acc[n]);
      } else {
        bool in_f16 = X == kRowsF16;
        if constexpr (X == kRowsF16) {
#pragma unroll
          for (uint32_t n = 0; n < NB; ++n) in_f16 &= exact_in_f16(sw[n][h]);
          in_f16 = __all(in_f16);
        }
        if (in_f16) {   // the weights as f16
#pragma unroll
          for (uint32_t j = 0; j < 4u; ++j)
#pragma unroll
            for (uint32_t n = 0; n < NB; ++n) acc[n] = multiply<kF16>(widen_e2m1_f16(fw[n][h][j], __builtin_bit_cast(float, sw[n][h] << 23)), fx[h * 4u + j], acc[n]);
        } else {
#pragma unroll
          for (uint32_t j = 0; j < 4u; ++j) {
            u32x4 high = fx[h * 4u + j], low{};
            if constexpr (X == kRowsF16) split_f16(fx[h * 4u + j], high, low);
#pragma unroll
            for (uint32_t n = 0; n < NB; ++n) {
              const u32x4 b = widen_e2m1(fw[n][h][j], __builtin_bit_cast(float, sw[n][h] << 23));
              acc[n] = multiply<kBf16>(b, high, acc[n]);
              if constexpr (X == kRowsF16) acc[n] = multiply<kBf16>(b, low, acc[n]);
            }
          }
        }
      }
    }
  }
  // the parts of the sum, wavefront by wavefront: [row][column], each in the wavefront's own ring, which has been read
  constexpr uint32_t PITCH = WIDE + 4u;
  static_assert(HIGH * PITCH * 4u <= RING * STAGE);
  float* mine = reinterpret_cast<float*>(lds[wave]);
#pragma unroll
  for (uint32_t n = 0; n < NB; ++n) *reinterpret_cast<f32x4*>(mine + r16 * PITCH + n * 16u + quarter * 4u) = acc[n];
  __syncthreads();
  for (uint32_t i = threadIdx.x; i < HIGH * WIDE; i += THREADS) {
    const uint32_t r = r0 + i / WIDE, c = c0 + i % WIDE;
    if (r >= g.end || c >= a.wide) continue;
    float v = 0.0f;
#pragma unroll
    for (uint32_t w = 0; w < WAVES; ++w) v += reinterpret_cast<const float*>(lds[w])[i / WIDE * PITCH + i % WIDE];
    char* out = a.out.data + r * a.out.stride;
    if (a.out_type == kOutF32) reinterpret_cast<float*>(out)[c] = v;
    else if (a.out_type == kOutBf16) reinterpret_cast<__bf16*>(out)[c] = static_cast<__bf16>(v);
    else reinterpret_cast<_Float16*>(out)[c] = static_cast<_Float16>(v);
  }
}

}  // namespace
