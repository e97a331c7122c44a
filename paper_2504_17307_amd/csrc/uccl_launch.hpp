// What the library's translation units share on the host side.  Internal to the library.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include <tuple>
#include <utility>

// Enqueue a kernel and return UCCL_OK or UCCL_ELAUNCH, whose text uccl_last_error_detail() then has; takes the
// calling thread's one-shot timing events (uccl_chunk.hip).
__attribute__((visibility("hidden"))) int uccl_internal_launch(const void* kernel, dim3 grid, dim3 block, hipStream_t s, void** args);
// The stop event that the calling thread's next launch would take: a call of several launches gives it (uccl_time_next_launch) to the last one too.
__attribute__((visibility("hidden"))) void* uccl_internal_stop_event();
// Load the code object of the row operators on the current device (uccl_rows.hip).
__attribute__((visibility("hidden"))) int uccl_internal_load_rows();
// The same for a HIP error that another call returned.
__attribute__((visibility("hidden"))) int uccl_internal_failed(hipError_t e);

namespace {

template <class... Params, size_t... I>
int enqueue_params(void (*kernel)(Params...), dim3 grid, uint32_t threads, hipStream_t s, std::tuple<Params...>& params, std::index_sequence<I...>) {
  void* ptrs[] = {static_cast<void*>(&std::get<I>(params))...};
  return uccl_internal_launch(reinterpret_cast<const void*>(kernel), grid, dim3(threads), s, ptrs);
}

template <class... Params, class... KernelArgs>
int enqueue(void (*kernel)(Params...), dim3 grid, uint32_t threads, hipStream_t s, KernelArgs... a) {
  static_assert(sizeof...(Params) == sizeof...(KernelArgs), "one argument per kernel parameter");
  std::tuple<Params...> params(static_cast<Params>(a)...);
  return enqueue_params(kernel, grid, threads, s, params, std::index_sequence_for<Params...>{});
}

}  // namespace
