// Microscaled 4 bits, gfx950 (MI355X): rows to them (an entry point of uccl_experts.h), and the grouped products of weights in them, which
// uccl_group_product makes.  Host side: argument checks and the choice of the kernel.
#include <hip/hip_runtime.h>

#include <math.h>
#include <stdint.h>

#include "uccl_experts.h"

#include "uccl_mx4_kernels.hpp"
#include "uccl_product_launch.hpp"

namespace {

// How long a launch of `tiles` takes that has room for `room` at a time, in rounds.  (The tiles are estimated: a little more than a round may be one.)
double rounds_of(double tiles, double room) {
  const double rounds = tiles / room;
  return rounds <= 1.05 ? 1.0 : rounds <= 2.0 ? 2.0 : rounds + 0.5;
}

// Tiles of 64 x 64 while there is a compute unit for each: the tiles of ragged groups are fewer than estimated, one group's are not.  Measured, one group, 260 to 280 of them / half as many of 64 x 128, us:
// rows in 4 bits, depth 512 5.7 to 6.0 / 5.5 to 5.7, 5000 16.9 to 19.2 / 15.1 to 15.5; bf16, 512 8.2 to 8.6 / 7.2 to 7.5, 5000 33 to 48 / 28 to 30; f16, 5000 42 to 50 / 40; 256 of them, 5000, 12.8, 25 and 31.
bool takes_least(const ProductArgs& a, double least_tiles) { return least_tiles <= (a.groups == 1u ? 256.0 : 280.0); }

// Rows of 4 bits, in us for 256 elements of the sum.  Few rows: 2.0e-5 for 16 rows of a column, 2.6e-5 for a column's weights where they are read once;
// tiles of 128 x 128, two on a compute unit: 1.7 a round, 1 where most of them are idle.  Measured, 16 rows at a time / 128 x 128, 7168 -> 2048, us: one group, 1 / 100 rows, 8.0 / 10.4 against
// 23 / 28; 8 of 32 groups, 16 rows, 13.3 against 28; 32 groups, 128 rows, 49 against 54; 8 groups, 300 rows, 27 against 27; 16 groups, 1000 rows, 81 against 47.
// Tiles: in units of one of 256 x 256 (67 us with a depth of 7168, one a compute unit) 192 x 256 costs 0.91, and 128 x 128 0.62, two on a compute unit.  Measured, 256 x 256 / 192 x 256 / 128 x 128, us:
// 4096 rows in 16 ragged groups, 7168 -> 2048, 83 / 76 / 93; 2048 rows 77 / 73 / 66; 1000 rows 63 / 61 / 44; 4000 rows in 4 groups 67 / 61 / 51; 8192 rows in 8 groups 80 / 135 / 110; 8190 rows in 16 groups,
// 2048 -> 7168, 131 / 139 / 137; 8192^3 313 / 367 / 429.  (128 x 256, of which one fits a compute unit, takes 52 where 128 x 128 takes 51, and more elsewhere.)
int product_4(const ProductArgs& a, hipStream_t s) {
  const double wide = a.wide, small_tiles = tiles_down(a, 128u) * blocks_for(a.wide, 128u);
  const double few_tiles = fmax(tiles_down(a, 16u), used_groups(a));
  double few = fmax(tiles_down(a, 16u) * wide * 2.0e-5, used_groups(a) * wide * 2.6e-5);
  double tiles = fmax(rounds_of(small_tiles, 512.0) * (1.0 + 0.7 * fmin(1.0, small_tiles / 256.0)), used_groups(a) * wide * 3.0e-5);
  // While there is a compute unit for each tile of 64 x 64, or of 64 x 128, in us and with what a call takes at the least.  Measured, 16 rows at a
  // time / 64 x 64 / 64 x 128, us: one group, 130 rows, 7168 -> 2048, 14.6 / 16.1 / 19.8, 227 rows, 5387 -> 1960, 16.0 / 14.0 / 16.6, 614 rows, 3304 -> 1923, 27.5 / 14.2 / 12.9; 300 rows in 8 groups,
  // 7168 -> 2048, 26.4 / 18.0 / 21.0; 691 rows in 12 groups, 2296 -> 1232, 19.6 / 12.1 / 11.2.
  const double deep = blocks_for(a.cols, 256u), least_tiles = tiles_down(a, 64u) * blocks_for(a.wide, 64u), low_tiles = tiles_down(a, 64u) * blocks_for(a.wide, 128u);
  const bool least = takes_least(a, least_tiles), low = low_tiles <= 256.0;
  if (least || low) {
    const double weights = used_groups(a) * wide * a.cols * 1.1e-7;   // from memory
    few = fmax(weights, 3.5 + fmax(0.65, few_tiles * blocks_for(a.wide, 32u) / 512.0) * (2.0 + 0.85 * ceil(deep / 4.0)));
    tiles = fmax(weights, least ? 4.8 + deep * (0.38 + 0.08 * least_tiles / 256.0) : 5.0 + deep * (0.45 + 0.2 * low_tiles / 256.0));
  }
  if (few <= tiles && (static_cast<uint64_t>(a.rows) / 16u + used_groups(a)) * blocks_for(a.wide, 32u) <= 1u << 23)
    return product_tiles<kForward>(mx4_few_kernel<kRows4, 32, 4, 3>, 16, 32, 256, a, s);
  // 64 x 128 while there is a compute unit for each: 725 rows in 2 of 9 groups, 4839 -> 1929, 22 -> 19 us; 500 rows in 8 groups, 7168 -> 2048, 27.3 -> 26.4; 600 rows in one, 2048 -> 2048, 10.9 -> 8.8;
  // 1000 rows in 16 groups, where there is not, 44 -> 56
  if (least) return product_tiles<kForward>(mx4_tile_kernel<64, 64, 4, 2, 1, 3>, 64, 64, 512, a, s);
  if (low) return product_tiles<kForward>(mx4_tile_kernel<64, 128, 2, 4, 2, 3>, 64, 128, 512, a, s);
  const double across = blocks_for(a.wide, 256u), large = rounds_of(tiles_down(a, 256u) * across, 256.0), middle = 0.91 * rounds_of(tiles_down(a, 192u) * across, 256.0);
  const double small = 0.62 * rounds_of(small_tiles, 512.0);
  if (large <= middle && large <= small) return product_tiles<kForward>(mx4_tile_kernel<256, 256, 2, 4, 6, 2>, 256, 256, 512, a, s);
  if (middle <= small) return product_tiles<kForward>(mx4_tile_kernel<192, 256, 2, 4, 5, 2>, 192, 256, 512, a, s);
  return product_tiles<kForward>(mx4_tile_kernel<128, 128, 2, 4, 3, 2>, 128, 128, 512, a, s);
}

// Rows of 16 bits, the same.  Few rows by 64 columns: 2.9e-5 for 16 rows of a column, 3.3e-5 for a column's weights; by 16 columns where that would leave most compute units idle.
// Tiles, in units of a round of 128 x 256 (114 us with a depth of 7168, 4.1 for 256 elements): 128 x 128 costs 0.57, 64 x 128, two on a compute unit, 0.66, and 0.37 while there is one on each.  Measured in bf16, 16 rows at a
// time / 64 x 128 / 128 x 128 / 128 x 256, 7168 -> 2048, us: one group, 100 rows, 15 / - / 61 / 92; 8 of 32 groups, 16 rows, 15 / - / 57 / 73; 32 groups, 128 rows, 65 / - / 122 / 93; 8 groups, 300 rows, 40 / - / 61 / 79, 500 rows
// 56 / 40 / 48 / 70; 16 groups, 1000 rows, 121 / 80 / 65 / 100, 4096 rows 428 / 180 / 187 / 200; 4000 rows in 4 groups 415 / 145 / 130 / 114; 8190 rows in 16 groups, 2048 -> 7168, - / 332 / 338 / 275; 2999 rows in 24
// groups, 2043 -> 1003, 81 / 26 / 42 / 35, in f16 86 / 29 / 52 / 41; 8192^3 in bf16 by 128 x 256 952.  One row by 64 / 16 columns 11.1 / 7.4.
template <Mx4Rows X>
int product_16(const ProductArgs& a, hipStream_t s) {
  constexpr bool F16 = X == kRowsF16;
  const double wide = a.wide, narrow = blocks_for(a.wide, 128u), low_tiles = tiles_down(a, 64u) * narrow, few_tiles = fmax(tiles_down(a, 16u), used_groups(a));
  const double large = rounds_of(tiles_down(a, 128u) * blocks_for(a.wide, 256u), 256.0), square = 0.57 * rounds_of(tiles_down(a, 128u) * narrow, 256.0);
  const double low = low_tiles <= 256.0 ? 0.37 : 0.66 * rounds_of(low_tiles, 512.0);
  double few = fmax(tiles_down(a, 16u) * wide * 2.9e-5, used_groups(a) * wide * 3.3e-5), tiles = 4.1 * fmin(fmin(large, square), low);
  // As in product_4().  Measured, 16 rows at a time / 64 x 64 / 64 x 128, us: bf16, one group, 130 rows, 7168 -> 2048, 23.9 / 30.0 / 36.9, 385 rows, 4816 -> 1851, 34.0 / 24.6 / 29.4, 600 rows, 2048 -> 2048,
  // 33.0 / 18.1 / 16.5; 298 rows in 3 groups, 1545 -> 1757, 19.4 / 12.9 / 15.1; 200 in 8, 7168 -> 2048, 29.2 / - / 35.5; 500 in 8 62.8 / 46.4 / 39.7; f16, 595 rows in one, 5096 -> 623, 26.3 / 31.4 / 40.3,
  // 385 rows, 4816 -> 1851, 37.2 / 30.6 / 39.1.
  const double least_tiles = tiles_down(a, 64u) * blocks_for(a.wide, 64u);
  const bool least = takes_least(a, least_tiles);
  if (least || low_tiles <= 256.0) {
    const double steps = blocks_for(a.cols, 64u);
    few = 3.0 + ceil(few_tiles * blocks_for(a.wide, 64u) / 256.0 - 0.1) * (3.0 + 1.4 * ceil(steps / 16.0)) * (F16 ? 1.08 : 1.0);
    tiles = least ? 5.5 + steps * (F16 ? 0.3 + 0.04 * least_tiles / 256.0 : 0.2 + 0.06 * least_tiles / 256.0)
                  : 7.0 + steps * (F16 ? 0.33 + 0.14 * low_tiles / 256.0 : 0.25 + 0.07 * low_tiles / 256.0);
  }
  if (few < tiles && (static_cast<uint64_t>(a.rows) / 16u + used_groups(a)) * blocks_for(a.wide, 16u) <= 1u << 23) {
    if (few_tiles * blocks_for(a.wide, 64u) <= 64.0) return product_tiles<kForward>(mx4_few_kernel<X, 16, 4, 3>, 16, 16, 256, a, s);
    return product_tiles<kForward>(mx4_few_kernel<X, 64, 4, 2>, 16, 64, 256, a, s);
  }
  if (least) return product_tiles<kForward>(mx4_wide_kernel<F16, 64, 64, 2, 5>, 64, 64, 512, a, s);
  if (low < square && low < large && (static_cast<uint64_t>(a.rows) / 64u + used_groups(a)) * static_cast<uint64_t>(narrow) <= 1u << 23) return product_tiles<kForward>(mx4_wide_kernel<F16, 64, 128, 4, 5>, 64, 128, 512, a, s);
  if (large <= square) return product_tiles<kForward>(mx4_wide_kernel<F16, 128, 256, 4, 5>, 128, 256, 512, a, s);
  return product_tiles<kForward>(mx4_wide_kernel<F16, 128, 128, 4, 5>, 128, 128, 512, a, s);
}

}  // namespace

int uccl_internal_load_mx4() {
  hipStreamCaptureMode mode = hipStreamCaptureModeRelaxed;   // another stream of the program may be under capture
  const bool relaxed = hipThreadExchangeStreamCaptureMode(&mode) == hipSuccess;
  void* at = nullptr;
  const hipError_t e = hipGetSymbolAddress(&at, HIP_SYMBOL(page_of_zeros));
  if (relaxed) (void)hipThreadExchangeStreamCaptureMode(&mode);
  return e == hipSuccess ? UCCL_OK : uccl_internal_failed(e);
}

int uccl_internal_product_mx4(const void* product_args, uint32_t x_dtype, hipStream_t s) {
  const ProductArgs& a = *static_cast<const ProductArgs*>(product_args);
  return x_dtype == UCCL_MX4 ? product_4(a, s) : x_dtype == UCCL_BF16 ? product_16<kRowsBf16>(a, s) : product_16<kRowsF16>(a, s);
}

extern "C" {

int uccl_quantise_rows(const uccl_rows* q, const uccl_rows* values, const uccl_rows* x, void* stream) {
  int e = check(q, x);
  if (e == UCCL_OK && values != nullptr) e = check(values);
  if (e != UCCL_OK) return e;
  if (q->dtype != UCCL_MX4 || !is_float(x->dtype) || !same_shape(q, x) || (values != nullptr && (values->dtype != x->dtype || !same_shape(values, x)))) return UCCL_EINVAL;
  if (x->rows == 0u || x->cols == 0u) return UCCL_OK;
  if (q->rows > 1u && q->scale_stride < blocks_for(q->cols, kMx4Block)) return UCCL_EINVAL;   // every row writes its own scales
  const hipStream_t s = static_cast<hipStream_t>(stream);
  return with_type(x->dtype, [&](auto t) {
    using T = decltype(t);
    constexpr uint32_t share = kMx4Block / Piece<T>::N;
    const uint32_t pieces = blocks_for(x->cols, Piece<T>::N), padded = (pieces + share - 1u) / share * share;
    const QuantiseArgs a{rows_of(q), rows_of(values), rows_of(x), x->cols, pieces, padded, 256u / padded, 256u % padded, static_cast<uint64_t>(x->rows) * padded};
    const uint64_t groups = (a.all + 255u) / 256u;
    // few pieces: one a thread, so that all compute units have some
    if (groups <= 1024u) return launch(quantise_kernel<T, 1, false>, groups, 256, s, a);
    if (values != nullptr && row_bytes(values) * values->rows > 32ull << 20) return launch(quantise_kernel<T, 4, true>, (groups + 3u) / 4u, 256, s, a);
    return launch(quantise_kernel<T, 4, false>, (groups + 3u) / 4u, 256, s, a);
  });
}

}  // extern "C"
