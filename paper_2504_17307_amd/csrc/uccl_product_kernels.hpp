// Matrix products grouped by expert, and their gradients (device code).  Internal to the library.
#pragma once

#include <type_traits>

#include "uccl_row_elements.hpp"

// Loads that must bring zeros go here.
static __device__ __align__(256) uint32_t page_of_zeros[64];

namespace {

struct E4m3 { uint8_t bits; };

// Four e4m3 values are four bf16 values exactly.
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
__device__ __forceinline__ u32x2 widen_e4m3(uint32_t four) {
  return u32x2{__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(four, 1.0f, false)),
               __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(four, 1.0f, true))};
}

enum Product : uint32_t { kForward, kGradX, kGradW };
enum OutType : uint32_t { kOutF32 = 0, kOutBf16 = 1, kOutF16 = 2 };

// kForward: out[i, n] = sum_k a[index[i], k] b[g, n, k]        a = x, b = w (e4m3: times their rows' scales)
// kGradX:   out[i, k] = sum_n a[i, n] b[g, n, k]               a = dy, b = w
// kGradW:   out[g, n, k] = sum_i a[i, n] b[index[i], k]        a = dy, b = x
// over the rows i of group g.  `wide`: rows of w a group, n; `cols`: k.
struct ProductArgs {
  Rows out, a, b;
  const int32_t* index;     // or nullptr: row i itself
  const int32_t* offsets;   // groups + 1
  uint32_t groups, rows, indexed_rows, wide, cols, out_type;
  uint32_t together;        // by rows: the order of the tiles, find_tile()
};

struct Group {
  uint32_t index, begin, end;   // rows begin .. end - 1
};

// Offsets are taken as they can be used, whatever they hold: each is at least the one before it, at least 0 and at most
// `rows`.  Groups never overlap then and no row outside the matrix is touched.
//
// 64 groups' ranges, a lane each.  `before`: the greatest offset of earlier groups.
struct Ranges {
  uint32_t begin, end;
  int32_t most;   // up to and with the lane's
};
__device__ __forceinline__ Ranges group_ranges(const ProductArgs& a, uint32_t at, int32_t before) {
  const uint32_t lane = threadIdx.x & 63u, mine = at + lane;
  const int32_t begin = mine <= a.groups ? a.offsets[mine] : 0, end = mine < a.groups ? a.offsets[mine + 1u] : 0;
  const int32_t limit = static_cast<int32_t>(a.rows);
  Ranges r;
  r.most = lane == 0u ? max(max(end, begin), before) : end;
#pragma unroll
  for (uint32_t d = 1; d < 64u; d <<= 1) {
    const int32_t other = __shfl_up(r.most, d);
    if (lane >= d) r.most = max(r.most, other);
  }
  const int32_t previous = __shfl_up(r.most, 1);
  r.begin = static_cast<uint32_t>(min(max(lane == 0u ? max(begin, before) : previous, 0), limit));
  r.end = mine < a.groups ? static_cast<uint32_t>(min(max(r.most, 0), limit)) : r.begin;
  return r;
}
// A sum up to and with the lane's.
__device__ __forceinline__ uint32_t sum_to_lane(uint32_t v) {
#pragma unroll
  for (uint32_t d = 1; d < 64u; d <<= 1) {
    const uint32_t other = __shfl_up(v, d);
    if ((threadIdx.x & 63u) >= d) v += other;
  }
  return v;
}

// How many tiles of `height` rows the lanes' groups are cut into (every group into tiles of its own): full ones, and those that a group ends
// in above them in the same word.
constexpr uint32_t kFullBits = 25;   // a launch has at most 2^24 tiles, and 64 groups end in at most 64
__device__ __forceinline__ uint32_t full_and_ends(const Ranges& r, uint32_t height) {
  const uint32_t n = r.end - r.begin;
  return n / height | (n % height != 0u ? 1u << kFullBits : 0u);
}

// Workgroups of a launch go round the eight XCDs in turn, and start in order.  Each XCD gets a contiguous eighth of the n tiles, so
// that tiles with the same rows or the same weights, which are neighbours, share an L2.  `place`: the workgroup's turn on its XCD;
// false: there is no tile for it.
__device__ __forceinline__ bool tile_of_xcd(uint32_t place, uint32_t n, uint32_t& tile) {
  const uint32_t each = (n + 7u) / 8u;
  tile = blockIdx.x % 8u * each + place;
  return place < each && tile < n;
}

// The tiles of an XCD are taken in bands of 4 rows of tiles, column by column: the 32 that its compute units work on at a time
// are 4 x 8 and read 12 panels of rows and weights, where a row of 32 would read 33.
constexpr uint32_t kBand = 4;
__device__ __forceinline__ void place_in_band(uint32_t& tile, uint32_t down, uint32_t across, uint32_t& place) {
  const uint32_t band = tile / (kBand * across), high = min(kBand, down - band * kBand), at = tile - band * kBand * across;
  place = at / high;
  tile = band * kBand + at % high;
}

// Full tiles first, and tiles that groups end in, which take less, after them: they fill up what the last round leaves.
__device__ __forceinline__ bool find_tile_by_size(const ProductArgs& a, uint32_t height, uint32_t across, Group& g, uint32_t& first_row, uint32_t& place) {
  constexpr uint32_t kFull = (1u << kFullBits) - 1u;
  Ranges r = group_ranges(a, 0, 0);
  uint32_t own = full_and_ends(r, height), to = sum_to_lane(own);
  uint32_t sum = __builtin_amdgcn_readlane(to, 63), full = sum & kFull, ends = sum >> kFullBits;
  if (a.groups > 64u) {
    int32_t before = __builtin_amdgcn_readlane(r.most, 63);
    for (uint32_t at = 64; at < a.groups; at += 64u) {
      const Ranges next = group_ranges(a, at, before);
      before = __builtin_amdgcn_readlane(next.most, 63);
      sum = __builtin_amdgcn_readlane(sum_to_lane(full_and_ends(next, height)), 63);
      full += sum & kFull;
      ends += sum >> kFullBits;
    }
  }
  const uint32_t turn = blockIdx.x / 8u, each = (full * across + 7u) / 8u;
  const bool whole = turn < each;
  uint32_t tile;
  if (!tile_of_xcd(whole ? turn : turn - each, (whole ? full : ends) * across, tile)) return false;
  place_in_band(tile, whole ? full : ends, across, place);
  uint32_t passed = 0;
  for (uint32_t at = 0;; at += 64u) {
    const uint32_t count = whole ? to & kFull : to >> kFullBits, mine = whole ? own & kFull : own >> kFullBits;
    const uint64_t holds = __ballot(passed + count > tile);
    if (holds != 0u) {
      const int l = __ffsll(static_cast<unsigned long long>(holds)) - 1;
      g = Group{at + static_cast<uint32_t>(l), static_cast<uint32_t>(__builtin_amdgcn_readlane(r.begin, l)), static_cast<uint32_t>(__builtin_amdgcn_readlane(r.end, l))};
      const uint32_t nth = whole ? tile - passed - (__builtin_amdgcn_readlane(count, l) - __builtin_amdgcn_readlane(mine, l)) : (g.end - g.begin) / height;
      first_row = g.begin + nth * height;
      return true;
    }
    passed += __builtin_amdgcn_readlane(count, 63);
    r = group_ranges(a, at + 64u, __builtin_amdgcn_readlane(r.most, 63));
    own = full_and_ends(r, height);
    to = sum_to_lane(own);
  }
}

// Each XCD takes an eighth of every group's tiles, column by column: those that read the same weights are on one XCD at the same time.
__device__ __forceinline__ bool find_tile_by_group(const ProductArgs& a, uint32_t height, uint32_t across, Group& g, uint32_t& first_row, uint32_t& place) {
  uint32_t turn = blockIdx.x / 8u;
  int32_t before = 0;
  for (uint32_t at = 0; at < a.groups; at += 64u) {
    const Ranges r = group_ranges(a, at, before);
    // the remainders of the eighths go round with the groups
    const uint32_t eighth = (blockIdx.x + at + (threadIdx.x & 63u)) % 8u, down = (r.end - r.begin + height - 1u) / height, tiles = down * across;
    const uint32_t first = tiles * eighth / 8u, own = tiles * (eighth + 1u) / 8u - first, to = sum_to_lane(own);
    const uint64_t holds = __ballot(to > turn);
    if (holds != 0u) {
      const int l = __ffsll(static_cast<unsigned long long>(holds)) - 1;
      g = Group{at + static_cast<uint32_t>(l), static_cast<uint32_t>(__builtin_amdgcn_readlane(r.begin, l)), static_cast<uint32_t>(__builtin_amdgcn_readlane(r.end, l))};
      const uint32_t tile = __builtin_amdgcn_readlane(first, l) + turn - (__builtin_amdgcn_readlane(to, l) - __builtin_amdgcn_readlane(own, l)), high = __builtin_amdgcn_readlane(down, l);
      first_row = g.begin + tile % high * height;
      place = tile / high;
      return true;
    }
    turn -= __builtin_amdgcn_readlane(to, 63);
    before = __builtin_amdgcn_readlane(r.most, 63);
  }
  return false;
}

// The workgroup's tile of the products by rows: its group, its first row and its place across.  All lanes of a wavefront call
// it.  The launch has a workgroup for every tile that there could be; which there are is known here only.
__device__ __forceinline__ bool find_tile(const ProductArgs& a, uint32_t height, uint32_t across, Group& g, uint32_t& first_row, uint32_t& place) {
  return a.together != 0u ? find_tile_by_group(a, height, across, g, first_row, place) : find_tile_by_size(a, height, across, g, first_row, place);
}

// The rows of group g, by the same rule.
__device__ __forceinline__ Group group_rows(const ProductArgs& a, uint32_t g) {
  const uint32_t lane = threadIdx.x & 63u;
  int32_t most = 0, next = 0;
  for (uint32_t at = lane; at <= g; at += 64u) most = max(most, a.offsets[at]);
#pragma unroll
  for (int d = 32; d > 0; d >>= 1) most = max(most, __shfl_xor(most, d));
  next = max(most, a.offsets[g + 1u]);
  const int32_t limit = static_cast<int32_t>(a.rows);
  return Group{g, static_cast<uint32_t>(__builtin_amdgcn_readfirstlane(min(most, limit))), static_cast<uint32_t>(__builtin_amdgcn_readfirstlane(min(next, limit)))};
}

// The gradient of the weights has as many tiles in every group, but they take as long as the group has rows: each group's tiles are cut
// into eighths of at least 16 tiles, column by column, which go round the XCDs.  (An eighth of all tiles would be two of 16 groups: 4096 rows in
// 16 ragged groups, 7168 x 2048, 295 us against 341; 3000 rows in 8 groups, 3360 x 1120, 74 against 87, and 76 with eighths of 9.  2000 rows in 32 groups,
// 1003 x 600, lose: 43 against 40.)
struct Slices {
  uint32_t each, n;   // tiles of a slice, slices of a group
};
__device__ __host__ __forceinline__ Slices slices_of(uint32_t tiles) {
  const uint32_t eighth = (tiles + 7u) / 8u, each = eighth >= 16u ? eighth : tiles < 16u ? tiles : 16u;
  return Slices{each, (tiles + each - 1u) / each};
}

// The same for either kind of product: tiles of `height` output rows, `across` to a row of tiles.
template <Product P>
__device__ __forceinline__ bool find_output(const ProductArgs& a, uint32_t height, uint32_t across, Group& g, uint32_t& first_row, uint32_t& place) {
  if constexpr (P != kGradW) return find_tile(a, height, across, g, first_row, place);
  const uint32_t down = (a.wide + height - 1u) / height, turn = blockIdx.x / 8u;
  const Slices s = slices_of(down * across);
  const uint32_t slice = turn / s.each * 8u + blockIdx.x % 8u, tile = slice % s.n * s.each + turn % s.each;
  if (slice / s.n >= a.groups || tile >= down * across) return false;
  g = group_rows(a, slice / s.n);
  first_row = tile % down * height;
  place = tile / down;
  return true;
}

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));

template <class T>
__device__ __forceinline__ uint32_t narrow_pair(float a, float b) {
  typedef T pair __attribute__((ext_vector_type(2)));
  return __builtin_bit_cast(uint32_t, pair{static_cast<T>(a), static_cast<T>(b)});
}

// Blocks of 16 x 16 of the output as the matrix instruction leaves them: a lane has of row lane % 16 four neighbouring columns,
// lane / 16 * 4 on.  They are stored 16 bytes a lane, with as much of a 128-byte line at a time as there is.
//
// Eight neighbouring columns in 16 bits from two blocks side by side: odd quarters of x against even quarters of y.  The lane's are then
// quarter % 2 * 16 + quarter / 2 * 8 on.
__device__ __forceinline__ u32x4 narrow_blocks(uint32_t out_type, f32x4 x, f32x4 y) {
  uint32_t wx[2], wy[2];
#pragma unroll
  for (uint32_t i = 0; i < 2u; ++i) {
    wx[i] = out_type == kOutBf16 ? narrow_pair<__bf16>(x[2 * i], x[2 * i + 1]) : narrow_pair<_Float16>(x[2 * i], x[2 * i + 1]);
    wy[i] = out_type == kOutBf16 ? narrow_pair<__bf16>(y[2 * i], y[2 * i + 1]) : narrow_pair<_Float16>(y[2 * i], y[2 * i + 1]);
  }
  const u32x2 s0 = __builtin_bit_cast(u32x2, __builtin_amdgcn_permlane16_swap(wx[0], wy[0], false, false));
  const u32x2 s1 = __builtin_bit_cast(u32x2, __builtin_amdgcn_permlane16_swap(wx[1], wy[1], false, false));
  return u32x4{s0.x, s1.x, s0.y, s1.y};
}

// Two pieces a lane that are APART columns from each other make lines of 128 bytes of 8 rows at a time: lanes 8 apart exchange the first
// row's second piece for the second row's first one.  The lane's pieces start at column `c` of rows `row` + lane % 16 of 16, of which
// those below `rows` are stored.
template <class T, uint32_t APART, bool ONCE>
__device__ __forceinline__ void store_lines(const ProductArgs& a, uint64_t row, uint32_t rows, uint32_t c, uint32_t cols, u32x4 p, u32x4 q) {
  const bool upper = (threadIdx.x & 8u) != 0u;
  u32x4 x, y;
#pragma unroll
  for (uint32_t i = 0; i < 4u; ++i) {
    const uint32_t other = static_cast<uint32_t>(__builtin_amdgcn_mov_dpp(static_cast<int>(upper ? p[i] : q[i]), 0x128, 0xF, 0xF, true));   // a row of lanes by 8
    x[i] = upper ? other : p[i];
    y[i] = upper ? q[i] : other;
  }
  if (upper) c += APART;
  const uint32_t r = threadIdx.x & 7u;
  char* at = a.out.data + (row + r) * a.out.stride;
  if (r < rows && c < cols) store_piece<ONCE>(at, c / Piece<T>::N, __builtin_bit_cast(Piece<T>, x), cols - c);
  if (r + 8u < rows && c < cols) store_piece<ONCE>(at + 8u * a.out.stride, c / Piece<T>::N, __builtin_bit_cast(Piece<T>, y), cols - c);
}

// Four blocks side by side (two, if there are no more) from column `first` on.
template <bool ONCE, uint32_t BLOCKS>
__device__ __forceinline__ void store_blocks(const ProductArgs& a, uint64_t row, uint32_t rows, uint32_t first, uint32_t cols, const f32x4 (&v)[BLOCKS]) {
  static_assert(BLOCKS == 2u || BLOCKS == 4u);
  const uint32_t quarter = threadIdx.x % 64u / 16u;
  if (a.out_type == kOutF32) {
#pragma unroll
    for (uint32_t n = 0; n < BLOCKS; n += 2u)
      store_lines<float, 16, ONCE>(a, row, rows, first + n * 16u + quarter * 4u, cols, __builtin_bit_cast(u32x4, v[n]), __builtin_bit_cast(u32x4, v[n + 1u]));
    return;
  }
  const uint32_t c = first + quarter % 2u * 16u + quarter / 2u * 8u;
  const u32x4 p = narrow_blocks(a.out_type, v[0], v[1]);
  if constexpr (BLOCKS == 4u) {
    store_lines<uint16_t, 32, ONCE>(a, row, rows, c, cols, p, narrow_blocks(a.out_type, v[2], v[3]));
  } else {
    const uint32_t r = threadIdx.x & 15u;
    if (r < rows && c < cols) store_piece<false>(a.out.data + (row + r) * a.out.stride, c / 8u, __builtin_bit_cast(Piece<uint16_t>, p), cols - c);
  }
}

// ---- tiles through the LDS --------------------------------------------------------------------------

typedef short s16x4 __attribute__((ext_vector_type(4)));

// kWidened: 8-bit operands as bf16, whose products are exact and are added as those of 16 bits are; kWidenedLarge: the same in tiles of 256 columns.
// (The instructions for 8-bit operands add 8 products at a time and drop of each what is below 2^-13 of the greatest of the 8, those for 16 bits what is
// below 2^-24, a binary32's last place: beside 448 x 448 and its opposite, all that 8-bit instructions keep of 6 products below 24 is 0.)
enum Arithmetic : uint32_t { kBf16, kF16, kWidened, kWidenedLarge };

// A stage is 128 bytes along the sum: 64 steps of 16 bits or 128 of 8.  It is multiplied in two halves.  Rows are loaded 128 bytes at
// a time: the L2 takes a request for 64 bytes as long as one for 128.
constexpr uint32_t kStageBytes = 128;

__device__ __forceinline__ uint32_t lds_address(const void* p) {
  return static_cast<uint32_t>(reinterpret_cast<uintptr_t>((const __attribute__((address_space(3))) char*)(p)));
}

// 64 lanes' 16 bytes from memory into the LDS at `to` (the same in every lane), lane by lane.  The compiler does not see the
// write: wait_for_loads() orders it before the reads.
__device__ __forceinline__ void load_to_lds(const char* from, uint32_t to) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off" ::"s"(to), "v"(from) : "m0");
}
// Every wavefront has at most its newest `N` loads under way.  (Other loads of the wavefront that are counted too only make this
// stricter: they return in order.)
template <uint32_t N>
__device__ __forceinline__ void wait_for_loads() { asm volatile("s_waitcnt vmcnt(%0)\n\ts_barrier" ::"n"(N) : "memory"); }
// Every wavefront has what it asked of the LDS but for its newest `N` reads.
template <uint32_t N>
__device__ __forceinline__ void wait_for_reads() { asm volatile("s_waitcnt lgkmcnt(%0)\n\ts_barrier" ::"n"(N) : "memory"); }

// Operands lie in the LDS in 16-byte pieces as they come from memory, in another order within a row so that the lanes of a
// read meet different banks (64 of 4 bytes; 16 lanes at a time with 16 bytes, 32 with 8): along the sum, piece p of row r is at
// p ^ (r / 2 % 8); across it (rows of a tile's width), pairs of pieces are at pair ^ turn(r).
__device__ __forceinline__ uint32_t turn(uint32_t r) { return ((r & 1u) * 2u) ^ ((r >> 1 & 1u) * 5u) ^ (r >> 3 & 1u); }

template <Arithmetic M>
__device__ __forceinline__ f32x4 multiply(u32x4 x, u32x4 y, f32x4 acc) {
  if constexpr (M == kF16) return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, x), __builtin_bit_cast(f16x8, y), acc, 0, 0, 0);
  else return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, x), __builtin_bit_cast(bf16x8, y), acc, 0, 0, 0);
}
struct Widened { u32x4 low, high; };
__device__ __forceinline__ Widened widen_e4m3(u32x4 v) {
  const u32x2 a = widen_e4m3(v.x), b = widen_e4m3(v.y), c = widen_e4m3(v.z), d = widen_e4m3(v.w);
  return Widened{u32x4{a.x, a.y, b.x, b.y}, u32x4{c.x, c.y, d.x, d.y}};
}

// One operand of a tile: SIDE rows (ALONG: rows of the matrix lie along the sum) or SIDE columns (rows of the matrix are steps
// of the sum), loaded a stage at a time by THREADS threads.
template <bool ALONG, uint32_t SIDE, uint32_t THREADS>
struct Operand {
  static constexpr uint32_t LOADS = SIDE * kStageBytes / 16u / THREADS, PITCH = ALONG ? kStageBytes / 16u : SIDE / 8u;   // pieces
  static_assert(SIDE * kStageBytes / 16u % THREADS == 0);
  const char* at[LOADS];     // the thread's next pieces; of an operand across the sum through an index: the piece in row 0
  uint32_t next[LOADS];      // through an index across the sum: the next row
  uint32_t still;            // along the sum: bit i, the piece of load i is of a row of zeros and stays where it is

  static __device__ __forceinline__ uint32_t row(uint32_t i) { return (i * THREADS + threadIdx.x) / PITCH; }
  static __device__ __forceinline__ uint32_t piece(uint32_t i) {
    const uint32_t slot = threadIdx.x % PITCH, r = row(i);
    return ALONG ? slot ^ (r >> 1 & 7u) : slot ^ (turn(r) << 1);
  }
  // The lane's part of half a stage for the 16 rows / columns from `first`, a multiple of 16, on: 16 bytes of one row, a quarter of the
  // wavefront the first 16 bytes, and so on
  static __device__ __forceinline__ u32x4 fragment(const char* stage, uint32_t first, uint32_t half) {
    const uint32_t lane = threadIdx.x & 63u;
    if constexpr (ALONG) {
      const uint32_t r = lane % 16u, p = half * 4u + lane / 16u;
      return *reinterpret_cast<const u32x4*>(stage + first * kStageBytes + (r * kStageBytes + ((p ^ (r >> 1 & 7u)) << 4)));
    } else {
      // 16 lanes bring a block of 4 steps x 16 columns and get it transposed: a lane its column's 4 steps
      const uint32_t step = lane / 16u * 8u + lane % 16u / 4u;
      stage += half * 32u * PITCH * 16u + lane % 4u * 8u;
      typedef __attribute__((address_space(3))) s16x4 lds_s16x4;
      const char* p = stage + step * PITCH * 16u + ((first / 16u ^ turn(step)) << 5);
      const u32x2 lo = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(p)));
      const char* q = stage + (step + 4u) * PITCH * 16u + ((first / 16u ^ turn(step + 4u)) << 5);
      const u32x2 hi = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(q)));
      return u32x4{lo.x, lo.y, hi.x, hi.y};
    }
  }
};

// A workgroup computes BM x BN of the output, WR x WC wavefronts a part each.  While the matrix cores work on half a stage, the
// next half's fragments are read from the LDS and loads straight into the LDS bring later stages, one between every few of a
// wavefront's multiplications: loads that are issued together hold up what comes after them.  The LDS holds AHEAD + 1 stages of one
// operand and AHEAD of the other: in the first half of stage k the former's stage k + AHEAD is asked for, and in its second half, when
// every wavefront has read its last fragments of stage k, the latter's takes the place of stage k.  The matrix instruction has the
// output's columns as its rows, so that a lane holds 4 neighbouring columns of one row.  It is the one for blocks of 16 x 16: what
// bounds long products is power, and from registers alone it reaches 1.98 PFLOP/s in bf16 where the one for 32 x 32 reaches 1.70.
// 8192^3 in bf16 864 us, 1.27 PFLOP/s (the library's product on that box 766); 8190 rows in 16 groups, 2048 -> 7168, 267 us.
template <Arithmetic M, Product P, uint32_t BM, uint32_t BN, uint32_t WR, uint32_t WC, uint32_t AHEAD>
__global__ __launch_bounds__(WR * WC * 64) void product_tile_kernel(ProductArgs a) {
  constexpr uint32_t THREADS = WR * WC * 64u, E = M == kWidened || M == kWidenedLarge ? 1u : 2u, DEEP = kStageBytes / E;
  constexpr uint32_t SIDE = 16u, NA = BM / WR / SIDE, NB = BN / WC / SIDE;
  constexpr bool A_ALONG = P != kGradW, B_ALONG = P == kForward;
  using A = Operand<A_ALONG, BM, THREADS>;
  using B = Operand<B_ALONG, BN, THREADS>;
  constexpr uint32_t A_STAGE = BM * kStageBytes, B_STAGE = BN * kStageBytes;
  __shared__ __align__(1024) char lds_a[(AHEAD + 1u) * A_STAGE], lds_b[AHEAD * B_STAGE];
  const char* zeros = reinterpret_cast<const char*>(page_of_zeros);
  asm volatile("" : "+s"(zeros));   // an address in registers: not looked up again at every load
  const uint32_t out_cols = P == kForward ? a.wide : a.cols, across = (out_cols + BN - 1u) / BN;
  Group g;
  uint32_t r0, c0;
  if (!find_output<P>(a, BM, across, g, r0, c0)) return;
  c0 *= BN;
  const uint64_t w0 = static_cast<uint64_t>(g.index) * a.wide;
  const uint32_t out_rows = P == kGradW ? a.wide : g.end;   // its rows end here
  const uint32_t depth = P == kForward ? a.cols : P == kGradX ? a.wide : g.end - g.begin;
  const uint32_t steps = (depth + DEEP - 1u) / DEEP;

  // Where the thread's pieces are.  Rows and columns past the tile's end stand for its last ones: what they make is not stored.
  A la;
  B lb;
  la.still = 0u;
#pragma unroll
  for (uint32_t i = 0; i < A::LOADS; ++i) {
    if constexpr (A_ALONG) {
      uint32_t r = min(r0 + A::row(i), out_rows - 1u);
      if (P == kForward && a.index != nullptr) r = static_cast<uint32_t>(a.index[r]);
      la.at[i] = a.a.data + r * a.a.stride + A::piece(i) * 16u;
      if (P == kForward && r >= a.indexed_rows) {           // zeros from the first stage to the last
        la.at[i] = zeros;
        la.still |= 1u << i;
      }
    } else {
      la.at[i] = a.a.data + min(r0 / 8u + A::piece(i), (a.wide - 1u) / 8u) * 16ull + (static_cast<uint64_t>(g.begin) + A::row(i)) * a.a.stride;
    }
  }
  // Row d of the group, read through the index by scalar loads: the rows of a wavefront's load are few.  (Vector loads would
  // be waited for together with the loads into the LDS.)
  auto indexed = [&](uint32_t d) -> uint32_t {
    constexpr uint32_t ROWS = 64u / B::PITCH;
    const uint32_t first = __builtin_amdgcn_readfirstlane(d);
    uint32_t r = 0xFFFFFFFFu;
#pragma unroll
    for (uint32_t i = 0; i < ROWS; ++i) {
      const uint32_t at = first + i;
      if (at < depth) {
        const uint32_t v = a.index == nullptr ? g.begin + at : static_cast<uint32_t>(((const __attribute__((address_space(4))) int32_t*)(uintptr_t)(a.index))[g.begin + at]);
        r = d == at ? v : r;
      }
    }
    return r;
  };
#pragma unroll
  for (uint32_t i = 0; i < B::LOADS; ++i) {
    if constexpr (B_ALONG) {
      lb.at[i] = a.b.data + (w0 + min(c0 + B::row(i), out_cols - 1u)) * a.b.stride + B::piece(i) * 16u;
    } else {
      lb.at[i] = a.b.data + min(c0 / 8u + B::piece(i), (a.cols - 1u) / 8u) * 16ull;
      if constexpr (P == kGradX) lb.at[i] += (w0 + B::row(i)) * a.b.stride;
      else lb.next[i] = indexed(B::row(i));
    }
  }

  // Ask for a thread's load i of stage k, into the LDS at `slot`.  What lies behind the end of the sum, in its last stage, comes from
  // a page of zeros.
  const uint32_t mine = __builtin_amdgcn_readfirstlane(threadIdx.x & ~63u) * 16u;
  const uint32_t here_a = lds_address(lds_a) + mine, here_b = lds_address(lds_b) + mine;
  auto load_a = [&](uint32_t k, uint32_t slot, uint32_t i, bool last) {
    const char* from = la.at[i];
    if constexpr (A_ALONG) {
      if (last && k * kStageBytes + A::piece(i) * 16u >= depth * E) from = zeros;
      la.at[i] += P == kForward && (la.still >> i & 1u) ? 0u : kStageBytes;
    } else {
      if (last && k * DEEP + A::row(i) >= depth) from = zeros;
      la.at[i] += DEEP * a.a.stride;
    }
    load_to_lds(from, here_a + slot + i * THREADS * 16u);
  };
  auto load_b = [&](uint32_t k, uint32_t slot, uint32_t i, bool last) {
    const char* from = lb.at[i];
    if constexpr (B_ALONG) {
      if (last && k * kStageBytes + B::piece(i) * 16u >= depth * E) from = zeros;
      lb.at[i] += kStageBytes;
    } else if constexpr (P == kGradX) {
      if (last && k * DEEP + B::row(i) >= depth) from = zeros;
      lb.at[i] += DEEP * a.b.stride;
    } else {
      from = lb.next[i] < a.indexed_rows ? from + lb.next[i] * a.b.stride : zeros;
      lb.next[i] = indexed((k + 1u) * DEEP + B::row(i));
    }
    load_to_lds(from, here_b + slot + i * THREADS * 16u);
  };
  // The piece that the sum ends in has what is behind the row's end: that is blanked.
  const bool ragged = (A_ALONG || B_ALONG) && depth * E % 16u != 0u;
  auto trim = [&](char* stage_a, char* stage_b) {
    const uint32_t tail = depth * E % kStageBytes, p = tail / 16u;
    auto blank_rows = [&](char* stage, uint32_t rows) {
      for (uint32_t r = threadIdx.x; r < rows; r += THREADS) {
        char* piece = stage + r * kStageBytes + ((p ^ (r >> 1 & 7u)) << 4);
#pragma unroll
        for (uint32_t b = 0; b < 16u; b += E)
          if (b >= tail % 16u) {
            if constexpr (E == 1) piece[b] = 0;
            else *reinterpret_cast<uint16_t*>(piece + b) = 0;
          }
      }
    };
    if (A_ALONG) blank_rows(stage_a, BM);
    if (B_ALONG) blank_rows(stage_b, BN);
    wait_for_reads<0>();   // and the writes
  };

  const uint32_t wave = threadIdx.x / 64u, lane = threadIdx.x & 63u;
  const uint32_t ra = wave / WC * (BM / WR), cb = wave % WC * (BN / WC);
  // Blocks of rows that the wavefront has in this tile, at most NA: the others are not multiplied
  const uint32_t high = __builtin_amdgcn_readfirstlane(r0 + ra < out_rows ? min((out_rows - r0 - ra + SIDE - 1u) / SIDE, NA) : 0u);
  f32x4 acc[NB][NA] = {};
  u32x4 fa[NA], fb[2][NB];
  uint32_t a_slot = 0, b_slot = 0;   // stage k's, bytes
  auto after = [](uint32_t slot, uint32_t by, uint32_t end) { return slot + by >= end ? slot + by - end : slot + by; };
  // Half a stage, whose fragments are fa and fb[HALF]: multiply, and read the next half's.  `load(i)` asks for a load of a later stage,
  // FROM: not before that many rows of blocks are done.
  auto multiply_half = [&](auto half, const char* next_a, const char* next_b, auto count, auto from, auto&& load) {
    constexpr uint32_t HALF = decltype(half)::value, COUNT = decltype(count)::value, FROM = decltype(from)::value;
#pragma unroll
    for (uint32_t n = 0; n < NB; ++n) fb[HALF ^ 1u][n] = B::fragment(next_b, cb + n * SIDE, HALF ^ 1u);
#pragma unroll
    for (uint32_t m = 0; m < NA; ++m) {
      if (m >= high) {
      } else if constexpr (E == 1u) {
        const Widened x = widen_e4m3(fa[m]);
#pragma unroll
        for (uint32_t n = 0; n < NB; ++n) {
          const Widened w = widen_e4m3(fb[HALF][n]);
          acc[n][m] = multiply<M>(w.low, x.low, acc[n][m]);
          acc[n][m] = multiply<M>(w.high, x.high, acc[n][m]);
        }
      } else {
#pragma unroll
        for (uint32_t n = 0; n < NB; ++n) acc[n][m] = multiply<M>(fb[HALF][n], fa[m], acc[n][m]);
      }
      __builtin_amdgcn_sched_barrier(0);   // the next fragment takes the registers of this one
      fa[m] = A::fragment(next_a, ra + m * SIDE, HALF ^ 1u);
      if constexpr (FROM != 0u)
        if (m + 1u == FROM) load(COUNT);   // the wait that lets the loads begin
      if (m >= FROM)
#pragma unroll
        for (uint32_t i = (m - FROM) * COUNT / (NA - FROM); i < (m + 1u - FROM) * COUNT / (NA - FROM); ++i) load(i);
      __builtin_amdgcn_sched_barrier(0);
    }
  };
  using First = std::integral_constant<uint32_t, 0>;
  using Second = std::integral_constant<uint32_t, 1>;
  // A quarter into the second half a wavefront has had all it asked of the stage before: what is newer are the other half's reads
  using Quarter = std::integral_constant<uint32_t, NA / 4u == 0u ? 1u : NA / 4u>;
  // STEADY: stage k + AHEAD is there to be asked for, and is not the last
  auto work = [&](uint32_t k, auto steady) {
    constexpr bool STEADY = decltype(steady)::value;
    const bool more = STEADY || k + AHEAD < steps, last = !STEADY && k + AHEAD + 1u == steps;
    const uint32_t a_next = after(a_slot, A_STAGE, (AHEAD + 1u) * A_STAGE), b_next = after(b_slot, B_STAGE, AHEAD * B_STAGE);
    const uint32_t a_load = after(a_slot, AHEAD * A_STAGE, (AHEAD + 1u) * A_STAGE);
    multiply_half(First{}, lds_a + a_slot, lds_b + b_slot, std::integral_constant<uint32_t, A::LOADS>{}, First{}, [&](uint32_t i) {
      if (more) load_a(k + AHEAD, a_load, i, last);
    });
    if (more) wait_for_loads<(AHEAD - 2u) * (A::LOADS + B::LOADS) + A::LOADS>();
    else if (k + 1u < steps) wait_for_loads<0>();
    if (!STEADY && ragged && k + 2u == steps) trim(lds_a + a_next, lds_b + b_next);
    // behind the last stage: read, and not used
    multiply_half(Second{}, lds_a + a_next, lds_b + b_next, std::integral_constant<uint32_t, B::LOADS>{}, Quarter{}, [&](uint32_t i) {
      if (!more) return;
      if (i == B::LOADS) wait_for_reads<NB + Quarter::value - 1u>();
      else load_b(k + AHEAD, b_slot, i, last);
    });
    a_slot = a_next;
    b_slot = b_next;
  };
  if (steps != 0u) {
#pragma unroll
    for (uint32_t k = 0; k < AHEAD; ++k)
      if (k < steps) {
#pragma unroll
        for (uint32_t i = 0; i < A::LOADS; ++i) load_a(k, k * A_STAGE, i, k + 1u == steps);
#pragma unroll
        for (uint32_t i = 0; i < B::LOADS; ++i) load_b(k, k * B_STAGE, i, k + 1u == steps);
      }
    if (steps >= AHEAD) wait_for_loads<(AHEAD - 1u) * (A::LOADS + B::LOADS)>();
    else wait_for_loads<0>();
    if (ragged && steps == 1u) trim(lds_a, lds_b);
#pragma unroll
    for (uint32_t n = 0; n < NB; ++n) fb[0][n] = B::fragment(lds_b, cb + n * SIDE, 0);
#pragma unroll
    for (uint32_t m = 0; m < NA; ++m) fa[m] = A::fragment(lds_a, ra + m * SIDE, 0);
    uint32_t k = 0;
    for (; k + AHEAD + 1u < steps; ++k) work(k, std::true_type{});
    for (; k < steps; ++k) work(k, std::false_type{});
  }

#pragma unroll
  for (uint32_t m = 0; m < NA; ++m) {
    const uint32_t r = r0 + ra + m * SIDE + lane % SIDE;   // this lane's row of the output
    float sx = 1.0f;
    if (E == 1u && r < out_rows) {
      const uint32_t from = a.index == nullptr ? r : static_cast<uint32_t>(a.index[r]);
      if (from < a.indexed_rows) sx = *reinterpret_cast<const float*>(a.a.scales + from * a.a.scale_stride);
    }
    auto scaled = [&](float v, uint32_t c) {
      if constexpr (E == 1u) return v * sx * *reinterpret_cast<const float*>(a.b.scales + (w0 + min(c, out_cols - 1u)) * a.b.scale_stride);
      else return v;
    };
    constexpr uint32_t BLOCKS = NB % 4u == 0u ? 4u : 2u;
    const uint32_t top = r0 + ra + m * SIDE;   // of the 16 rows that the wavefront has
    const uint32_t rows = top < out_rows ? out_rows - top : 0u;
#pragma unroll
    for (uint32_t n = 0; n < NB; n += BLOCKS) {
      const uint32_t first = c0 + cb + n * SIDE;
      f32x4 v[BLOCKS];
#pragma unroll
      for (uint32_t b = 0; b < BLOCKS; ++b) {
        v[b] = acc[n + b][m];
#pragma unroll
        for (uint32_t i = 0; i < 4u; ++i) v[b][i] = scaled(v[b][i], first + b * SIDE + lane / 16u * 4u + i);
      }
      // a launch of tiles of 256 x 256 writes more than the L2s keep
      store_blocks<BM == 256u>(a, P == kGradW ? w0 + top : top, rows, first, out_cols, v);
    }
  }
}

// ---- few rows a group -------------------------------------------------------------------------------

template <uint32_t N>
__device__ __forceinline__ void wait_for_own_loads() { asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory"); }

// kForward for groups of about 16 rows and less, where the reading of the weights is all there is to do: a workgroup computes
// 16 rows x WIDE columns, and every wavefront a part of the sum for them, 128 bytes along it at a time in turn with the others.
// A wavefront has a ring of its own in the LDS, loads whole 128-byte pieces of rows straight into it, and waits for no other one before
// the parts are added up.  Bound by HBM where a group has 16 rows at most: 16 rows in 8 of 32 groups, 7168 -> 2048, in bf16 38 us, 128 rows in 32
// groups in e4m3 76: 6.2 TB/s of weights.
template <Arithmetic M, uint32_t WIDE, uint32_t WAVES>
__global__ __launch_bounds__(WAVES * 64) void product_few_kernel(ProductArgs a) {
  constexpr uint32_t THREADS = WAVES * 64u, E = M == kWidened ? 1u : 2u, HIGH = 16u, TURN = 128u, RING = 3u, NB = WIDE / 16u;
  constexpr uint32_t ROWS = HIGH + WIDE, LOADS = ROWS / 8u;    // rows of a stage: x's, then w's; 8 of them a load
  __shared__ __align__(1024) char lds[WAVES][RING][ROWS * TURN];
  const uint32_t across = (a.wide + WIDE - 1u) / WIDE, lane = threadIdx.x & 63u, wave = threadIdx.x / 64u;
  Group g;
  uint32_t r0, c0;
  if (!find_tile(a, HIGH, across, g, r0, c0)) return;
  c0 *= WIDE;
  const uint64_t w0 = static_cast<uint64_t>(g.index) * a.wide;
  const char* zeros = reinterpret_cast<const char*>(page_of_zeros);
  asm volatile("" : "+s"(zeros));
  const uint32_t bytes = a.cols * E, stages = (bytes + TURN - 1u) / TURN;
  // piece p of a row lies at p ^ (row / 2 % 8), as 16 lanes read 16 rows at a time
  const uint32_t piece = lane % 8u ^ (lane / 16u & 3u);   // of rows 16 i + lane / 8; rows 8 further have it ^ 4
  const char* at[LOADS];
  bool there[LOADS];
#pragma unroll
  for (uint32_t i = 0; i < LOADS; ++i) {
    const uint32_t r = i * 8u + lane / 8u, p = (piece ^ (i % 2u * 4u)) * 16u + wave * TURN;
    there[i] = true;
    if (i < HIGH / 8u) {
      uint32_t from = r0 + r;
      there[i] = from < g.end;
      if (there[i] && a.index != nullptr) {
        from = static_cast<uint32_t>(a.index[from]);
      }
      there[i] = there[i] && from < a.indexed_rows;
      at[i] = a.a.data + from * a.a.stride + p;
    } else {
      at[i] = a.b.data + (w0 + min(c0 + r - HIGH, a.wide - 1u)) * a.b.stride + p;
    }
  }
  const uint32_t base = lds_address(lds[wave]);
  auto load = [&](uint32_t k, uint32_t slot) {   // the wavefront's stages come in turn: wave, wave + WAVES, ...
#pragma unroll
    for (uint32_t i = 0; i < LOADS; ++i) {
      const bool inside = there[i] && k * TURN + (piece ^ (i % 2u * 4u)) * 16u < bytes;
      load_to_lds(inside ? at[i] : zeros, __builtin_amdgcn_readfirstlane(base + (slot * ROWS + i * 8u) * TURN));
      at[i] += WAVES * TURN;
    }
  };
  auto fragment = [&](const char* stage, uint32_t first, uint32_t j) {
    const uint32_t r = first + lane % 16u;
    return *reinterpret_cast<const u32x4*>(stage + r * TURN + (((j * 4u + lane / 16u) ^ (r >> 1 & 7u)) << 4));
  };
  f32x4 acc[NB] = {};
#pragma unroll
  for (uint32_t i = 0; i < RING; ++i)
    if (wave + i * WAVES < stages) load(wave + i * WAVES, i);
  uint32_t slot = 0;
  for (uint32_t k = wave; k < stages; k += WAVES) {
    if (k + (RING - 1u) * WAVES < stages) wait_for_own_loads<(RING - 1u) * LOADS>();
    else if (k + (RING - 2u) * WAVES < stages) wait_for_own_loads<(RING - 2u) * LOADS>();
    else wait_for_own_loads<0>();
    char* stage = lds[wave][slot];
    if (k + 1u == stages && bytes % 16u != 0u && lane < ROWS) {   // the piece that the rows end in
      char* last = stage + lane * TURN + ((bytes % TURN / 16u ^ (lane >> 1 & 7u)) << 4);
#pragma unroll
      for (uint32_t b = 0; b < 16u; b += E)
        if (b >= bytes % 16u) {
          if constexpr (E == 1) last[b] = 0;
          else *reinterpret_cast<uint16_t*>(last + b) = 0;
        }
    }
    u32x4 fx[2], fw[NB][2];
#pragma unroll
    for (uint32_t j = 0; j < 2u; ++j) {
      fx[j] = fragment(stage, 0, j);
#pragma unroll
      for (uint32_t n = 0; n < NB; ++n) fw[n][j] = fragment(stage, HIGH + n * 16u, j);
    }
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");   // the ring's place is free
    if (k + RING * WAVES < stages) load(k + RING * WAVES, slot);
    slot = slot + 1u == RING ? 0u : slot + 1u;
#pragma unroll
    for (uint32_t j = 0; j < 2u; ++j) {
      if constexpr (E == 1u) {
        const Widened x = widen_e4m3(fx[j]);
#pragma unroll
        for (uint32_t n = 0; n < NB; ++n) {
          const Widened w = widen_e4m3(fw[n][j]);
          acc[n] = multiply<M>(w.low, x.low, acc[n]);
          acc[n] = multiply<M>(w.high, x.high, acc[n]);
        }
      } else {
#pragma unroll
        for (uint32_t n = 0; n < NB; ++n) acc[n] = multiply<M>(fw[n][j], fx[j], acc[n]);
      }
    }
  }
  // the parts of the sum, wavefront by wavefront: [row][column], each in the wavefront's own ring, which has been read
  constexpr uint32_t PITCH = WIDE + 4u;
  static_assert(HIGH * PITCH * 4u <= RING * ROWS * TURN);
  float* mine = reinterpret_cast<float*>(lds[wave]);
#pragma unroll
  for (uint32_t n = 0; n < NB; ++n) *reinterpret_cast<f32x4*>(mine + lane % 16u * PITCH + n * 16u + lane / 16u * 4u) = acc[n];
  __syncthreads();
  for (uint32_t i = threadIdx.x; i < HIGH * WIDE; i += THREADS) {
    const uint32_t r = r0 + i / WIDE, c = c0 + i % WIDE;
    if (r >= g.end || c >= a.wide) continue;
    float v = 0.0f;
#pragma unroll
    for (uint32_t w = 0; w < WAVES; ++w) v += reinterpret_cast<const float*>(lds[w])[i / WIDE * PITCH + i % WIDE];
    if constexpr (E == 1u) {
      const uint32_t from = a.index == nullptr ? r : static_cast<uint32_t>(a.index[r]);
      const float sx = from < a.indexed_rows ? *reinterpret_cast<const float*>(a.a.scales + from * a.a.scale_stride) : 1.0f;
      v = v * sx * *reinterpret_cast<const float*>(a.b.scales + (w0 + c) * a.b.scale_stride);
    }
    char* out = a.out.data + r * a.out.stride;
    if (a.out_type == kOutF32) reinterpret_cast<float*>(out)[c] = v;
    else if (a.out_type == kOutBf16) reinterpret_cast<__bf16*>(out)[c] = static_cast<__bf16>(v);
    else reinterpret_cast<_Float16*>(out)[c] = static_cast<_Float16>(v);
  }
}

}  // namespace
