// Rows and their elements, as the row operators' kernels take them (device code).  Internal to the library.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

// A matrix by rows in device memory.  Rows start on 16-byte boundaries, so the 16-byte piece that holds a row's last
// element can always be read whole: an aligned piece with one byte in an allocation has no byte on another page.
// Writes never leave the row.
struct Rows {
  char* data;
  uint64_t stride;         // bytes
  char* scales;            // f32, one a row (8-bit rows), or nullptr
  uint64_t scale_stride;   // bytes
};

template <class T>
__device__ __forceinline__ float widen(T v) { return static_cast<float>(v); }

template <class T>
struct Piece {   // 16 bytes of a row
  static constexpr uint32_t N = 16u / sizeof(T);
  T v[N];
};

template <class T>
__device__ __forceinline__ Piece<T> load_piece(const char* row, uint32_t piece) {
  return __builtin_bit_cast(Piece<T>, *reinterpret_cast<const u32x4*>(row + piece * 16ull));
}

// The same for what is not read again soon: it does not stay in the L2.
template <class T>
__device__ __forceinline__ Piece<T> load_piece_once(const char* row, uint32_t piece) {
  return __builtin_bit_cast(Piece<T>, __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(row + piece * 16ull)));
}

// How many elements of a thread's piece `p` are the row's; threads past the row's end read its last piece and have none.
template <class T>
__device__ __forceinline__ uint32_t valid_of(uint32_t p, uint32_t pieces, uint32_t cols) { return p < pieces ? cols - p * Piece<T>::N : 0u; }

// Elements from `valid` on are not the row's: they read as zero.
template <class T>
__device__ __forceinline__ void blank(Piece<T>& p, uint32_t valid) {
  if (valid >= Piece<T>::N) return;
#pragma unroll
  for (uint32_t i = 0; i < Piece<T>::N; ++i)
    if (i >= valid) p.v[i] = static_cast<T>(0.0f);
}

// Whole pieces with one store, the last piece of a ragged row element by element.  ONCE: outputs that are too large for the caches,
// which then keep what others left there.
template <bool ONCE, class T>
__device__ __forceinline__ void store_piece(char* row, uint32_t piece, const Piece<T>& p, uint32_t valid) {
  if (valid >= Piece<T>::N) {
    u32x4* at = reinterpret_cast<u32x4*>(row + piece * 16ull);
    if constexpr (ONCE) __builtin_nontemporal_store(__builtin_bit_cast(u32x4, p), at);
    else *at = __builtin_bit_cast(u32x4, p);
  } else {
    T* at = reinterpret_cast<T*>(row + piece * 16ull);
#pragma unroll
    for (uint32_t i = 0; i < Piece<T>::N; ++i)
      if (i < valid) at[i] = p.v[i];
  }
}

// Sum / maximum over a wavefront; every lane has the result.
__device__ __forceinline__ float wave_sum(float v) {
#pragma unroll
  for (int d = 32; d > 0; d >>= 1) v += __shfl_xor(v, d);
  return v;
}
__device__ __forceinline__ float wave_max(float v) {
#pragma unroll
  for (int d = 32; d > 0; d >>= 1) v = fmaxf(v, __shfl_xor(v, d));
  return v;
}

}  // namespace
