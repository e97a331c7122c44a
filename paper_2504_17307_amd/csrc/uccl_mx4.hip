// Microscaled 4 bits, gfx950 (MI355X): rows to them (an entry point of uccl_experts.h), and the grouped products of weights in them, which
// uccl_group_product makes.  Host side: argument checks and the choice of the kernel.
#include <hip/hip_runtime.h>

#include <math.h>
#include <stdint.h>

#include "uccl_experts.h"

#include "uccl_mx4_kernels.hpp"
#include "uccl_product_launch.hpp"

namespace {

template <Mx4Rows X>
int product(const ProductArgs& a, hipStream_t s) {
  return product_tiles<kForward>(mx4_simple_kernel<X>, 16, 16, 64, a, s);
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
  return x_dtype == UCCL_MX4 ? product<kRows4>(a, s) : x_dtype == UCCL_BF16 ? product<kRowsBf16>(a, s) : product<kRowsF16>(a, s);
}

extern "C" {

int uccl_quantise_rows(const uccl_rows* q, const uccl_rows* values, const uccl_rows* x, void* stream) {
  int e = check(q, x);
  if (e == UCCL_OK && values != nullptr) e = check(values);
  if (e != UCCL_OK) return e;
  if (q->dtype != UCCL_MX4 || !is_float(x->dtype) || !same_shape(q, x) || (values != nullptr && (values->dtype != x->dtype || !same_shape(values, x)))) return UCCL_EINVAL;
  if (x->rows == 0u || x->cols == 0u) return UCCL_OK;
  if (q->rows > 1u && q->scale_stride < blocks_for(q->cols, kMx4Block)) return UCCL_EINVAL;   // every row writes its own scales
  return with_type(x->dtype, [&](auto t) {
    using T = decltype(t);
    const uint32_t pieces = blocks_for(x->cols, Piece<T>::N), groups = blocks_for(pieces, 256u);
    const QuantiseArgs a{rows_of(q), rows_of(values), rows_of(x), x->rows, x->cols, pieces, groups};
    return launch(quantise_kernel<T, false>, static_cast<uint64_t>(x->rows) * groups, 256, static_cast<hipStream_t>(stream), a);
  });
}

}  // extern "C"
