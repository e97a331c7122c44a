// Row operators around an all-to-all dispatch, gfx950 (MI355X): norm of rows, products grouped by expert, combination
// of rows, and their gradients.  Host side: argument checks, the choice of the kernel, the entry points of uccl_rows.h.
#include <hip/hip_runtime.h>

#include <math.h>
#include <stdint.h>

#include "uccl_rows.h"

#include "uccl_product_kernels.hpp"
#include "uccl_product_launch.hpp"
#include "uccl_row_checks.hpp"
#include "uccl_row_kernels.hpp"

namespace {

// Outputs of more than this do not stay in the L2s (8 of 4 MiB) until they are read, and are stored past them: norm of 4096 x 7168 in
// bf16 to e4m3 48 -> 39 us (loads past them too), combination of 8 x 4096 rows 104 -> 86.
bool too_large_to_keep(const uccl_rows* m) { return static_cast<uint64_t>(m->rows) * m->cols * element_bytes(m->dtype) > (32ull << 20); }

// A workgroup a row, with its row in registers.  Many rows: two pieces a thread (4096 x 7168, bf16 to e4m3: 36.5 us with 512 threads,
// 39 with 256 and four pieces, 43 with 1024 and one); few rows, where latency counts: one piece (one row of 7168: 3.4 us, 4.9 with 256 threads).
template <class T, bool E8, bool ONCE>
int norm(const NormArgs& a, hipStream_t s) {
  const uint32_t pieces = blocks_for(a.cols, Piece<T>::N);
  if (pieces <= 64u) return launch(norm_kernel<T, E8, 64, 1, ONCE>, a.rows, 64, s, a);
  if (pieces <= 256u) return launch(norm_kernel<T, E8, 256, 1, ONCE>, a.rows, 256, s, a);
  if (pieces <= 512u) return launch(norm_kernel<T, E8, 512, 1, ONCE>, a.rows, 512, s, a);
  if (pieces <= 1024u && a.rows > 512u) return launch(norm_kernel<T, E8, 512, 2, ONCE>, a.rows, 512, s, a);
  if (pieces <= 1024u) return launch(norm_kernel<T, E8, 1024, 1, false>, a.rows, 1024, s, a);   // 8 MiB at most
  if (pieces <= 2048u) return launch(norm_kernel<T, E8, 512, 4, ONCE>, a.rows, 512, s, a);
  return launch(norm_long_kernel<T, E8>, a.rows, 1024, s, a);
}

// Workgroups that share the rows of a norm's gradient, at most: one a compute unit.  (512 of them come in two rounds: 4096 x 7168 in bf16
// 44 against 52 us, and half the sums to add up.)
constexpr uint32_t kGradGroups = 256;

template <class T, bool ONCE>
int norm_grad(const NormGradArgs& a, uint32_t groups, hipStream_t s) {
  const uint32_t pieces = blocks_for(a.cols, Piece<T>::N);
  if (pieces <= 256u) return launch(norm_grad_kernel<T, 256, 1, ONCE>, groups, 256, s, a);
  if (pieces <= 512u) return launch(norm_grad_kernel<T, 512, 1, ONCE>, groups, 512, s, a);
  if (pieces <= 1024u) return launch(norm_grad_kernel<T, 1024, 1, ONCE>, groups, 1024, s, a);
  // (bf16: 2048 x 16384 62 us, 154 by the kernel for any length; 4096 x 12288 82, 235; 100 x 12288 14.5, 13.5)
  if (pieces <= 2048u) return launch(norm_grad_kernel<T, 512, 4, ONCE>, groups, 512, s, a);
  return launch(norm_grad_long_kernel<T>, groups, 1024, s, a);
}

OutType out_type(const uccl_rows* m) { return m->dtype == UCCL_F32 ? kOutF32 : m->dtype == UCCL_BF16 ? kOutBf16 : kOutF16; }

// What a tile costs is about the same whether one compute unit works or all do, and whether all of its rows are there or a few, and
// a launch of few tiles takes as long as the compute units that get one more than others.  256 x 256 does the most work for what
// it reads; smaller tiles leave less of themselves empty in small groups and fill the machine when there are few.  In units of
// a tile of 256 x 256 (180 us with a depth of 7168 in bf16, one a compute unit), 128 x 256 costs 0.69 and 128 x 128 0.45.  Measured in bf16,
// 256 x 256 / 128 x 256 / 128 x 128, us: 4096 rows in 16 ragged groups, 7168 -> 2048, 182 / 223 / 240; 2048 rows 163 / 132 / 164; 1024 rows
// 152 / 119 / 112; 2999 rows in 24 groups, 2043 -> 1003, 50 / 35 / 44; 8190 rows in 16 groups, 2048 -> 7168, 290 / 339 / 398; 512 rows in one group,
// 2048 -> 2048, 45 / 28 / 18; both gradients of 3000 rows in 8 groups, 3360 -> 1120, 123 / 153 / 184.
// Large tiles of 8-bit operands have no 128 x 128 beside them, and 128 x 256 costs 0.59.  Measured, 256 x 256 / 128 x 256 / 128 x 128, us: 4096 rows in 16 groups,
// 7168 -> 2048, 172 / 184 / 194; 2048 rows 161 / 98 / 117; 1000 rows 113 / 92 / 114; 8190 rows 294 / 266 / 295; 8190 rows, 2048 -> 7168, 275 / 281 / 347; 3000 rows in
// 32 groups, 1500 -> 800, 36 / 29 / 38.
enum Tile : uint32_t { kTile256, kTile128x256, kTile128 };

template <Product P>
Tile choose_tile(const ProductArgs& a, bool large_8_bit) {
  auto cost = [&](uint32_t high, uint32_t wide, double unit) {
    const double down = P == kGradW ? static_cast<double>(a.groups) * blocks_for(a.wide, high) : tiles_down(a, high);
    const double rounds = down * blocks_for(P == kForward ? a.wide : a.cols, wide) / 256.0;   // over 256 compute units
    return unit * (rounds <= 2.0 ? ceil(rounds) : rounds + 0.5);
  };
  const double large = cost(256u, 256u, 1.0), middle = cost(128u, 256u, large_8_bit ? 0.59 : 0.69);
  if (large_8_bit) return large <= middle ? kTile256 : kTile128x256;
  const double small = cost(128u, 128u, 0.45);
  return large <= middle && large <= small ? kTile256 : middle <= small ? kTile128x256 : kTile128;
}

// Which 8-bit products go by large tiles if they go by tiles: those with outputs of 16 bits and long sums.  The others go by 128 x 128 (4096 rows in 16 groups, 7168 -> 2048,
// to f32 179 us, 167 by 256 x 256; 2048 rows 117, 97 by 128 x 256).
bool takes_large_8_bit(const ProductArgs& a) { return a.out_type != kOutF32 && a.cols >= 512u; }

// Few rows a group: 16 rows at a time, which read the weights again from the L2 for every 16, against a tile's, which read them once
// and leave most of the machine idle if there are few tiles.  In us for 128 bytes along the sum.  Measured, few rows against tiles, 7168 -> 2048, us:
// one group in bf16, 20 / 100 rows, 8 / 20 against 42 / 46; 8 groups, 50 / 100 / 200 rows, 32 / 52 / 69 against 41 / 43 / 42; 24 groups, 20 / 200 / 400 rows,
// 88 / 119 / 185 against 124 / 134 / 138.  In e4m3 against large tiles: one group, 200 / 333 / 512 rows, 25 / 37 / 51 against 90 / 91 / 91; 8 groups, 300 rows, 39 against 72;
// 16 groups, 600 / 1000 rows, 71 / 106 against 76 / 92; 24 groups, 400 rows, 81 against 69.
// 1003 -> 777, one group in bf16, 200 rows 6.2 against 11.7; 8 groups, 200 / 400 rows 6.2 / 19 against 10.7 / 11.5.
template <Arithmetic M>
bool takes_few_rows(const ProductArgs& a) {
  if ((static_cast<uint64_t>(a.rows) / 16u + used_groups(a)) * blocks_for(a.wide, 32u) > 1u << 23) return false;   // more tiles than a launch can have, where larger ones fit
  const double wide = a.wide, weights = used_groups(a) * wide, rounds = tiles_down(a, 128u) * blocks_for(a.wide, 128u) / 256.0;
  const double few = fmax(tiles_down(a, 16u) * wide * (M == kWidened ? 2.3e-5 : 2.0e-5), weights * 1.9e-5);   // 1.9e-5: 6.7 TB/s
  const double tiles = fmax(fmax(rounds, 1.0) * (M != kWidened ? 0.4 : takes_large_8_bit(a) ? 1.5 : 0.7), weights * 2.4e-5);
  return few < tiles;
}

template <Arithmetic M, Product P>
int product_of(const ProductArgs& a, hipStream_t s) {
  if constexpr (P == kForward)
    if (takes_few_rows<M>(a)) {
      // 32 columns a workgroup of 4 wavefronts, two workgroups on a compute unit; 16 columns and 8 wavefronts where that would leave most
      // compute units idle (7168 -> 2048, bf16: one row 8.7 us so, 16.9 with 32 columns; 16 rows in 8 of 32 groups 50, 41 with 32; 100 rows in one
      // group 30, 20 with 32)
      if (fmax(tiles_down(a, 16u), used_groups(a)) * blocks_for(a.wide, 32u) <= 256.0) return product_tiles<P>(product_few_kernel<M, 16, 8>, 16, 16, 512, a, s);
      return product_tiles<P>(product_few_kernel<M, 32, 4>, 16, 32, 256, a, s);
    }
  if constexpr (M == kWidened) {
    if (takes_large_8_bit(a)) {
      if (choose_tile<P>(a, true) == kTile256) return product_tiles<P>(product_tile_kernel<kWidenedLarge, P, 256, 256, 2, 4, 2>, 256, 256, 512, a, s);
      return product_tiles<P>(product_tile_kernel<kWidenedLarge, P, 128, 256, 2, 4, 3>, 128, 256, 512, a, s);
    }
  } else {
    const Tile tile = choose_tile<P>(a, false);
    if (tile == kTile256) return product_tiles<P>(product_tile_kernel<M, P, 256, 256, 2, 4, 2>, 256, 256, 512, a, s);
    if (tile == kTile128x256) return product_tiles<P>(product_tile_kernel<M, P, 128, 256, 2, 4, 3>, 128, 256, 512, a, s);
  }
  return product_tiles<P>(product_tile_kernel<M, P, 128, 128, 2, 4, 4>, 128, 128, 512, a, s);
}

template <Product P>
int product(const ProductArgs& a, uint32_t dtype, hipStream_t s) {
  if constexpr (P == kForward)
    if (dtype == UCCL_E4M3) return product_of<kWidened, P>(a, s);
  return dtype == UCCL_BF16 ? product_of<kBf16, P>(a, s) : product_of<kF16, P>(a, s);
}

}  // namespace

int uccl_internal_load_rows() {
  hipStreamCaptureMode mode = hipStreamCaptureModeRelaxed;   // another stream of the program may be under capture
  const bool relaxed = hipThreadExchangeStreamCaptureMode(&mode) == hipSuccess;
  void* at = nullptr;
  const hipError_t e = hipGetSymbolAddress(&at, HIP_SYMBOL(page_of_zeros));
  if (relaxed) (void)hipThreadExchangeStreamCaptureMode(&mode);
  return e == hipSuccess ? UCCL_OK : uccl_internal_failed(e);
}

extern "C" {

int uccl_norm_rows(const uccl_rows* y, const uccl_rows* h, float* rstd, const uccl_rows* x, const uccl_rows* r, const void* weight,
                   const uccl_norm_opts* opts, void* stream) {
  if (y == nullptr || x == nullptr || !is_float(x->dtype) || (y->dtype != x->dtype && y->dtype != UCCL_E4M3) || !same_shape(y, x)) return UCCL_EINVAL;
  if ((h != nullptr && (h->dtype != x->dtype || !same_shape(h, x))) || (r != nullptr && (r->dtype != x->dtype || !same_shape(r, x)))) return UCCL_EINVAL;
  if (opts == nullptr || !(opts->eps >= 0.0f) || isinf(opts->eps) || opts->reserved[0] || opts->reserved[1] || opts->reserved[2]) return UCCL_EINVAL;
  int e = check(y, x);
  if (e == UCCL_OK && h != nullptr) e = check(h);
  if (e == UCCL_OK && r != nullptr) e = check(r);
  if (e != UCCL_OK) return e;
  if (x->rows == 0u || x->cols == 0u) return UCCL_OK;
  if (weight == nullptr || (y->dtype == UCCL_E4M3 && y->rows > 1u && y->scale_stride == 0u)) return UCCL_EINVAL;   // every row writes its own scale
  if (misaligned(weight, 16) || misaligned(rstd, 4)) return UCCL_EALIGN;
  const float shrink = ldexpf(1.0f, -ilogbf(static_cast<float>(x->cols)) / 2);
  const NormArgs a{rows_of(y), rows_of(h), rows_of(x), rows_of(r), static_cast<const char*>(weight), rstd, x->rows, x->cols, opts->eps, shrink,
                   1.0f / (static_cast<float>(x->cols) * shrink * shrink)};
  const bool once = too_large_to_keep(y) || (h != nullptr && too_large_to_keep(h));
  const hipStream_t s = static_cast<hipStream_t>(stream);
  return with_type(x->dtype, [&](auto t) {
    using T = decltype(t);
    if (y->dtype == UCCL_E4M3) return once ? norm<T, true, true>(a, s) : norm<T, true, false>(a, s);
    return once ? norm<T, false, true>(a, s) : norm<T, false, false>(a, s);
  });
}

uint64_t uccl_norm_rows_scratch(uint32_t rows, uint32_t cols) {
  const uint64_t bytes = static_cast<uint64_t>(rows < kGradGroups ? rows : kGradGroups) * cols * sizeof(float);
  return (bytes + 15u) / 16u * 16u;
}

int uccl_norm_rows_grad(const uccl_rows* dx, float* dweight, const uccl_rows* dy, const uccl_rows* dh, const uccl_rows* h,
                        const float* rstd, const void* weight, void* scratch, uint64_t scratch_bytes, void* stream) {
  if (dx == nullptr || dy == nullptr || h == nullptr || !is_float(h->dtype)) return UCCL_EINVAL;
  if (dx->dtype != h->dtype || dy->dtype != h->dtype || !same_shape(dx, h) || !same_shape(dy, h)) return UCCL_EINVAL;
  if (dh != nullptr && (dh->dtype != h->dtype || !same_shape(dh, h))) return UCCL_EINVAL;
  int e = check(dx, dy, h);
  if (e == UCCL_OK && dh != nullptr) e = check(dh);
  if (e != UCCL_OK) return e;
  if (h->cols == 0u) return UCCL_OK;
  if (dweight == nullptr) return UCCL_EINVAL;
  if (misaligned(dweight, 4)) return UCCL_EALIGN;
  const uint32_t sums = blocks_for(h->cols, 64u);
  if (!fits(sums, 1024)) return UCCL_ETOOBIG;   // before the first of the two launches
  const hipStream_t s = static_cast<hipStream_t>(stream);
  const uint32_t groups = h->rows < kGradGroups ? h->rows : kGradGroups;
  if (h->rows != 0u) {
    if (rstd == nullptr || weight == nullptr || scratch == nullptr || scratch_bytes < uccl_norm_rows_scratch(h->rows, h->cols)) return UCCL_EINVAL;
    if (misaligned(weight, 16) || misaligned(rstd, 4) || misaligned(scratch, 16)) return UCCL_EALIGN;
    const NormGradArgs a{rows_of(dx), rows_of(dy), rows_of(h), rows_of(dh), static_cast<const char*>(weight), rstd, static_cast<float*>(scratch), h->rows, h->cols};
    void* const stop = uccl_internal_stop_event();   // the first launch has it as well: one that HIP does not take is refused there
    e = with_type(h->dtype, [&](auto t) {
      using T = decltype(t);
      return too_large_to_keep(dx) ? norm_grad<T, true>(a, groups, s) : norm_grad<T, false>(a, groups, s);
    });
    if (e != UCCL_OK) return e;
    (void)uccl_time_next_launch(nullptr, stop);
  }
  return launch(column_sum_kernel, sums, 1024, s, dweight, static_cast<const float*>(scratch), groups, h->cols);
}

// What the three products have in common.  `x` of kForward and kGradW is read through the index.
static int check_product(const uccl_rows* rows, const uccl_rows* w, const int32_t* index, const int32_t* offsets, uint32_t n_groups, uint32_t* wide) {
  if (n_groups > kMost || (n_groups == 0u && w->rows != 0u)) return UCCL_EINVAL;
  if (n_groups != 0u && w->rows % n_groups != 0u) return UCCL_EINVAL;
  *wide = n_groups == 0u ? 0u : w->rows / n_groups;
  if (n_groups != 0u && offsets == nullptr && rows->rows != 0u) return UCCL_EINVAL;
  return misaligned(offsets, 4) || misaligned(index, 4) ? UCCL_EALIGN : UCCL_OK;
}

int uccl_group_product(const uccl_rows* y, const uccl_rows* x, const int32_t* index, const uccl_rows* w, const int32_t* offsets,
                       uint32_t n_groups, void* stream) {
  int e = check(y, x, w);
  if (e != UCCL_OK) return e;
  uint32_t wide = 0;
  const bool mx4 = w->dtype == UCCL_MX4 && (x->dtype == UCCL_MX4 || is_16(x->dtype));
  if (!is_float(y->dtype) || !(mx4 || ((is_16(x->dtype) || x->dtype == UCCL_E4M3) && w->dtype == x->dtype)) || w->cols != x->cols) return UCCL_EINVAL;
  e = check_product(y, w, index, offsets, n_groups, &wide);
  if (e != UCCL_OK) return e;
  if ((n_groups != 0u && y->cols != wide) || (index == nullptr && x->rows < y->rows)) return UCCL_EINVAL;
  if (n_groups == 0u || y->rows == 0u || y->cols == 0u) return UCCL_OK;
  const uint32_t depth = x->rows == 0u ? 0u : x->cols;   // no row of x: nothing to add
  const ProductArgs a{rows_of(y), rows_of(x), rows_of(w), index, offsets, n_groups, y->rows, x->rows, wide, depth, out_type(y), 0};
  return mx4 ? uccl_internal_product_mx4(&a, x->dtype, static_cast<hipStream_t>(stream)) : product<kForward>(a, x->dtype, static_cast<hipStream_t>(stream));
}

int uccl_group_product_grad_x(const uccl_rows* dx, const uccl_rows* dy, const uccl_rows* w, const int32_t* offsets, uint32_t n_groups, void* stream) {
  int e = check(dx, dy, w);
  if (e != UCCL_OK) return e;
  uint32_t wide = 0;
  if (!is_float(dx->dtype) || !is_16(dy->dtype) || w->dtype != dy->dtype || w->cols != dx->cols || dx->rows != dy->rows) return UCCL_EINVAL;
  e = check_product(dx, w, nullptr, offsets, n_groups, &wide);
  if (e != UCCL_OK) return e;
  if (n_groups != 0u && dy->cols != wide) return UCCL_EINVAL;
  if (n_groups == 0u || dx->rows == 0u || dx->cols == 0u) return UCCL_OK;
  const ProductArgs a{rows_of(dx), rows_of(dy), rows_of(w), nullptr, offsets, n_groups, dx->rows, dx->rows, wide, dx->cols, out_type(dx), 0};
  return product<kGradX>(a, dy->dtype, static_cast<hipStream_t>(stream));
}

int uccl_group_product_grad_w(const uccl_rows* dw, const uccl_rows* dy, const uccl_rows* x, const int32_t* index, const int32_t* offsets,
                              uint32_t n_groups, void* stream) {
  int e = check(dw, dy, x);
  if (e != UCCL_OK) return e;
  uint32_t wide = 0;
  if (!is_float(dw->dtype) || !is_16(dy->dtype) || x->dtype != dy->dtype || dw->cols != x->cols) return UCCL_EINVAL;
  e = check_product(dy, dw, index, offsets, n_groups, &wide);
  if (e != UCCL_OK) return e;
  if ((n_groups != 0u && dy->cols != wide) || (index == nullptr && x->rows < dy->rows) || (n_groups != 0u && offsets == nullptr)) return UCCL_EINVAL;
  if (n_groups == 0u || wide == 0u || dw->cols == 0u) return UCCL_OK;
  const ProductArgs a{rows_of(dw), rows_of(dy), rows_of(x), index, offsets, n_groups, dy->rows, x->rows, wide, dw->cols, out_type(dw), 0};
  return product<kGradW>(a, dy->dtype, static_cast<hipStream_t>(stream));
}

// pos, weights and the like of a combination.
static int check_slots(const uccl_rows* tokens, const uccl_rows* y, const int32_t* pos, const float* weights, uint32_t slots) {
  if (y->cols != tokens->cols || y->dtype != tokens->dtype || !is_float(y->dtype) || slots > kMost) return UCCL_EINVAL;
  if (pos == nullptr && tokens->rows != 0u && slots != 0u) return UCCL_EINVAL;
  return misaligned(pos, 4) || misaligned(weights, 4) ? UCCL_EALIGN : UCCL_OK;
}

int uccl_combine_rows(const uccl_rows* out, const uccl_rows* y, const int32_t* pos, const float* weights, uint32_t slots, const uccl_rows* r, void* stream) {
  int e = check(out, y);
  if (e == UCCL_OK && r != nullptr) e = check(r);
  if (e != UCCL_OK) return e;
  if (r != nullptr && (r->dtype != out->dtype || !same_shape(r, out))) return UCCL_EINVAL;
  e = check_slots(out, y, pos, weights, slots);
  if (e != UCCL_OK) return e;
  if (out->rows == 0u || out->cols == 0u) return UCCL_OK;
  return with_type(out->dtype, [&](auto t) {
    using T = decltype(t);
    const uint32_t blocks = blocks_for(blocks_for(out->cols, Piece<T>::N), 128u);
    const uint64_t grid = static_cast<uint64_t>(out->rows) * blocks;
    const CombineArgs a{rows_of(out), rows_of(y), rows_of(r), pos, weights, out->rows, y->rows == 0u ? 0u : slots, y->rows, out->cols, blocks};
    const hipStream_t s = static_cast<hipStream_t>(stream);
    return too_large_to_keep(out) ? launch(combine_kernel<T, 128, true>, grid, 128, s, a) : launch(combine_kernel<T, 128, false>, grid, 128, s, a);
  });
}

int uccl_combine_rows_grad(const uccl_rows* dy, float* dweights, const uccl_rows* dout, const uccl_rows* y, const int32_t* pos, const float* weights,
                           uint32_t slots, void* stream) {
  int e = check(dy, dout, y);
  if (e != UCCL_OK) return e;
  if (dy->dtype != y->dtype || !same_shape(dy, y)) return UCCL_EINVAL;
  e = check_slots(dout, y, pos, weights, slots);
  if (e != UCCL_OK) return e;
  if (misaligned(dweights, 4)) return UCCL_EALIGN;
  if (dout->rows == 0u || slots == 0u) return UCCL_OK;
  return with_type(y->dtype, [&](auto t) {
    using T = decltype(t);
    // (without a row there is nothing to write but the weights' gradient: an empty sum for every slot)
    const CombineGradArgs a{rows_of(dy), rows_of(dout), rows_of(y), pos, weights, dweights, dout->rows, slots, y->rows, y->rows == 0u ? 0u : dout->cols};
    const hipStream_t s = static_cast<hipStream_t>(stream);
    return too_large_to_keep(dy) ? launch(combine_grad_kernel<T, true>, dout->rows, 256, s, a) : launch(combine_grad_kernel<T, false>, dout->rows, 256, s, a);
  });
}

}  // extern "C"
