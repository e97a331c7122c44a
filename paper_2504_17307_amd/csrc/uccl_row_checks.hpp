// What the entry points of the row operators check of a matrix, and how they launch (host side).  Internal to the library.
#pragma once

#include <stdint.h>

#include "uccl_rows.h"

#include "uccl_launch.hpp"
#include "uccl_row_elements.hpp"

namespace {

constexpr uint32_t kMost = 0x7FFFFFFFu, kMostCols = 1u << 30;   // rows, slots, groups; columns

bool misaligned(const void* p, uintptr_t to) { return reinterpret_cast<uintptr_t>(p) % to != 0; }

uint32_t element_bytes(uint32_t dtype) {   // of types whose elements have whole bytes
  switch (dtype) {
    case UCCL_F32: return 4;
    case UCCL_BF16: case UCCL_F16: return 2;
    case UCCL_E4M3: return 1;
    default: return 0;
  }
}
uint64_t row_bytes(const uccl_rows* m) { return m->dtype == UCCL_MX4 ? (m->cols + 1ull) / 2u : static_cast<uint64_t>(m->cols) * element_bytes(m->dtype); }
bool is_16(uint32_t dtype) { return dtype == UCCL_BF16 || dtype == UCCL_F16; }
bool is_float(uint32_t dtype) { return dtype == UCCL_F32 || is_16(dtype); }
bool has_scales(uint32_t dtype) { return dtype == UCCL_E4M3 || dtype == UCCL_MX4; }
bool same_shape(const uccl_rows* a, const uccl_rows* b) { return a->rows == b->rows && a->cols == b->cols; }

// What holds for every matrix by itself.
int check(const uccl_rows* m) {
  if (m == nullptr || m->reserved != 0u || (element_bytes(m->dtype) == 0u && m->dtype != UCCL_MX4) || m->rows > kMost || m->cols > kMostCols) return UCCL_EINVAL;
  if (has_scales(m->dtype) != (m->scales != nullptr) && m->rows != 0u) return UCCL_EINVAL;
  if (m->rows == 0u || m->cols == 0u) return UCCL_OK;
  if (m->data == nullptr) return UCCL_EINVAL;
  if (m->rows > 1u && m->stride < row_bytes(m)) return UCCL_EINVAL;   // rows would overlap
  if (misaligned(m->data, 16) || (m->rows > 1u && m->stride % 16u != 0u)) return UCCL_EALIGN;
  if (m->scales != nullptr && (misaligned(m->scales, 4) || (m->rows > 1u && m->scale_stride % 4u != 0u))) return UCCL_EALIGN;
  return UCCL_OK;
}
template <class... M>
int check(const uccl_rows* first, const M*... others) {
  const int e = check(first);
  return e != UCCL_OK ? e : check(others...);
}

Rows rows_of(const uccl_rows* m) {
  if (m == nullptr) return Rows{nullptr, 0, nullptr, 0};
  return Rows{static_cast<char*>(m->data), m->stride, static_cast<char*>(m->scales), m->scale_stride};
}

uint32_t blocks_for(uint64_t n, uint32_t each) { return static_cast<uint32_t>((n + each - 1) / each); }

// A grid of `groups` workgroups; HIP takes fewer than 2^32 threads a launch.
bool fits(uint64_t groups, uint32_t threads) { return groups <= 0xFFFFFFFFull / threads; }

template <class K, class... A>
int launch(K kernel, uint64_t groups, uint32_t threads, hipStream_t s, A... a) {
  return fits(groups, threads) ? enqueue(kernel, dim3(static_cast<uint32_t>(groups)), threads, s, a...) : static_cast<int>(UCCL_ETOOBIG);
}

// Calls f with a value of the element type of 16- or 32-bit rows.
template <class F>
int with_type(uint32_t dtype, F f) {
  return dtype == UCCL_F32 ? f(float{}) : dtype == UCCL_BF16 ? f(__bf16{}) : f(_Float16{});
}

}  // namespace
