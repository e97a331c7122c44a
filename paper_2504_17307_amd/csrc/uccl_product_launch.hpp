// How a grouped product is launched: tiles and their order (host side).  Internal to the library.
#pragma once

#include "uccl_product_kernels.hpp"
#include "uccl_row_checks.hpp"

// A product whose weights are in microscaled 4 bits, and its rows too or in 16 bits (uccl_mx4.hip); takes a ProductArgs.
__attribute__((visibility("hidden"))) int uccl_internal_product_mx4(const void* product_args, uint32_t x_dtype, hipStream_t s);

namespace {

uint32_t used_groups(const ProductArgs& a) { return a.groups < a.rows ? a.groups : a.rows; }   // that have rows, at most

// How many tiles of so many rows the groups are cut into: the last one of a group is half empty on average.
double tiles_down(const ProductArgs& a, uint32_t high) {
  return a.groups == 1u ? blocks_for(a.rows, high) : static_cast<double>(a.rows) / high + 0.5 * used_groups(a);
}

// A launch over tiles of BM x BN: a workgroup for each that there could be whatever the offsets are, by eights.
//
// The tiles of products by rows come in one of two orders.  Full ones first keep the last round short; all of a group's together read its
// weights once, which pays where a group has many.  Measured, by size / by group, us: 8190 rows in 16 groups, 2048 -> 7168, bf16 (70 tiles a group) 297 / 273
// (1.10 / 0.93 GB read); gradients of 4096 rows in 16 groups, 7168 x 2048 (42) 183 / 167; by 16 rows, 3000 -> 1200, bf16, 100 rows in one group / 3 / 8 (266, 98,
// 49) 10.6 / 8.9, 13.8 / 8.9, 17.2 / 15.2; 200 rows in one group, 7168 -> 2048 (32) 48 / 50; 400 rows in 8 groups (14) 47 / 50; gradients of 2000 rows in
// 32 groups, 1003 x 600 (5) 13 / 17.
constexpr double kTogether = 40.0;

template <Product P, class K>
int product_tiles(K kernel, uint32_t bm, uint32_t bn, uint32_t threads, ProductArgs a, hipStream_t stream) {
  const uint64_t across = blocks_for(P == kForward ? a.wide : a.cols, bn);
  auto by_eights = [](uint64_t n) { return (n + 7u) / 8u * 8u; };
  uint64_t tiles;
  if (P == kGradW) {
    const uint64_t group = blocks_for(a.wide, bm) * across;
    if (group > 1u << 24) return UCCL_ETOOBIG;
    const Slices s = slices_of(static_cast<uint32_t>(group));
    tiles = by_eights(static_cast<uint64_t>(a.groups) * s.n) * s.each;
  } else {
    // by group, an XCD has of every group one tile more than its eighth at most
    const uint64_t by_group = by_eights((a.rows / bm + used_groups(a)) * across) + 8ull * used_groups(a);
    a.together = tiles_down(a, bm) * across >= kTogether * used_groups(a) && by_group <= 1u << 24 && fits(by_group, threads);
    tiles = a.together ? by_group : by_eights(a.rows / bm * across) + by_eights(used_groups(a) * across);
  }
  if (tiles > 1u << 24) return UCCL_ETOOBIG;   // find_tile() counts them in 25 bits
  return launch(kernel, tiles, threads, stream, a);
}

}  // namespace
