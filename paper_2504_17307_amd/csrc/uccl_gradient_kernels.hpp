// The norm of many matrices together, and their scaling to it (device code).  Internal to the library.
#pragma once

#include "uccl_row_elements.hpp"

namespace {

// The matrices of a launch, in the kernel's arguments (4 KiB at most): most are one row, of which less has to be said.  A workgroup has `share` pieces of 16 bytes of
// one of them: matrix i has the workgroups from first[i] on.
template <bool FLAT>
struct GradientArgs {
  static constexpr uint32_t MOST = FLAT ? 150u : 60u, STRIDED = FLAT ? 1u : MOST;
  const char* in[MOST];
  char* out[MOST];
  uint64_t in_stride[STRIDED], out_stride[STRIDED];
  uint32_t first[MOST], cols[MOST], rows[STRIDED];
  uint8_t dtype[MOST];           // 0: f32, 1: bf16, 2: f16
  uint32_t n, share;
  double* parts;                 // the norm: a workgroup's sum
  const float* norm;             // the clipping
  float most;
};
static_assert(sizeof(GradientArgs<true>) <= 4096u && sizeof(GradientArgs<false>) <= 4096u);

struct Matrix {
  const char* in;
  char* out;
  uint64_t in_stride, out_stride;
  uint32_t rows, cols, pieces, dtype;   // pieces of a row
};

constexpr uint32_t kGradientThreads = 256, kGradientUnroll = 4;

// The workgroup's: the last one that begins at it or before.  `begin`: its first piece.
template <bool FLAT>
__device__ __forceinline__ Matrix matrix_of(const GradientArgs<FLAT>& a, uint32_t group, uint64_t& begin) {
  const uint32_t lane = threadIdx.x % 64u;
  uint32_t before = 0;
#pragma unroll
  for (uint32_t at = 0; at < GradientArgs<FLAT>::MOST; at += 64u)
    before += __popcll(__ballot(at + lane < a.n && a.first[at + lane < GradientArgs<FLAT>::MOST ? at + lane : 0u] <= group));
  const uint32_t i = __builtin_amdgcn_readfirstlane(before - 1u);
  Matrix m{a.in[i], a.out[i], 0u, 0u, 1u, a.cols[i], 0u, a.dtype[i]};
  if constexpr (!FLAT) {
    m.in_stride = a.in_stride[i];
    m.out_stride = a.out_stride[i];
    m.rows = a.rows[i];
  }
  const uint32_t n = m.dtype == 0u ? 4u : 8u;
  m.pieces = m.cols / n + (m.cols % n != 0u);
  begin = static_cast<uint64_t>(group - a.first[i]) * a.share;
  return m;
}

// Calls f(row, piece, valid elements of it) for every piece of the workgroup's that is the thread's, kGradientUnroll at a time: load() first, then use().
template <class T, bool FLAT, class L, class U>
__device__ __forceinline__ void over_pieces(const Matrix& m, uint64_t begin, uint32_t share, L load, U use) {
  constexpr uint32_t N = Piece<T>::N;
  const uint64_t all = static_cast<uint64_t>(m.rows) * m.pieces, end = min(begin + share, all);
  for (uint64_t at = begin + threadIdx.x; at < end; at += kGradientThreads * kGradientUnroll) {
    Piece<T> p[kGradientUnroll];
    uint64_t row[kGradientUnroll];
    uint32_t piece[kGradientUnroll];
#pragma unroll
    for (uint32_t u = 0; u < kGradientUnroll; ++u) {
      const uint64_t mine = min(at + u * kGradientThreads, end - 1u);
      row[u] = FLAT ? 0u : end >> 32 == 0u ? static_cast<uint32_t>(mine) / m.pieces : mine / m.pieces;
      piece[u] = static_cast<uint32_t>(mine - row[u] * m.pieces);
      p[u] = load(row[u], piece[u]);
    }
#pragma unroll
    for (uint32_t u = 0; u < kGradientUnroll; ++u)
      if (at + u * kGradientThreads < end) use(row[u], piece[u], p[u], m.cols - piece[u] * N);
  }
}

template <class T, bool FLAT>
__device__ __forceinline__ double square_sum(const Matrix& m, uint64_t begin, uint32_t share) {
  double sum = 0.0;
  over_pieces<T, FLAT>(m, begin, share, [&](uint64_t row, uint32_t piece) { return load_piece<T>(m.in + row * m.in_stride, piece); },
    [&](uint64_t, uint32_t, Piece<T>& p, uint32_t valid) {
      blank(p, valid);
#pragma unroll
      for (uint32_t i = 0; i < Piece<T>::N; ++i) sum = __builtin_fma(static_cast<double>(widen(p.v[i])), static_cast<double>(widen(p.v[i])), sum);
    });
  return sum;
}

__device__ __forceinline__ double wave_sum_64(double v) {
#pragma unroll
  for (int d = 32; d > 0; d >>= 1) v += __shfl_xor(v, d);
  return v;
}

// Squares in binary64, which has them exactly and does not overflow; a workgroup's sum has its place, and they are added in a fixed order.  Bound by memory: three matrices of
// together 1.88 GB f32 312 us, 6.0 TB/s; 300 of 9.5 MB bf16 together, two launches by the arguments' size, 6.7 and 5.5, which is latency.
template <bool FLAT>
__global__ __launch_bounds__(kGradientThreads) void square_sum_kernel(GradientArgs<FLAT> a) {
  __shared__ double buffer[kGradientThreads / 64u];
  uint64_t begin;
  const Matrix m = matrix_of(a, blockIdx.x, begin);
  double sum = m.dtype == 0u ? square_sum<float, FLAT>(m, begin, a.share) : m.dtype == 1u ? square_sum<__bf16, FLAT>(m, begin, a.share) : square_sum<_Float16, FLAT>(m, begin, a.share);
  sum = wave_sum_64(sum);
  if (threadIdx.x % 64u == 0u) buffer[threadIdx.x / 64u] = sum;
  __syncthreads();
  if (threadIdx.x != 0u) return;
#pragma unroll
  for (uint32_t w = 1; w < kGradientThreads / 64u; ++w) sum += buffer[w];
  a.parts[blockIdx.x] = sum;
}

__global__ __launch_bounds__(1024) void square_root_kernel(float* norm, const double* parts, uint32_t n) {
  __shared__ double buffer[16];
  double sum = 0.0;
#pragma unroll 4
  for (uint32_t i = threadIdx.x; i < n; i += 1024u) sum += parts[i];
  sum = wave_sum_64(sum);
  if (threadIdx.x % 64u == 0u) buffer[threadIdx.x / 64u] = sum;
  __syncthreads();
  if (threadIdx.x != 0u) return;
#pragma unroll
  for (uint32_t w = 1; w < 16u; ++w) sum += buffer[w];
  *norm = static_cast<float>(sqrt(sum));
}

template <class T, bool FLAT, bool ONCE>
__device__ __forceinline__ void scale_pieces(const Matrix& m, uint64_t begin, uint32_t share, float by) {
  over_pieces<T, FLAT>(m, begin, share,
    [&](uint64_t row, uint32_t piece) { return ONCE ? load_piece_once<T>(m.in + row * m.in_stride, piece) : load_piece<T>(m.in + row * m.in_stride, piece); },
    [&](uint64_t row, uint32_t piece, Piece<T>& p, uint32_t valid) {
#pragma unroll
      for (uint32_t i = 0; i < Piece<T>::N; ++i) {
        float v = widen(p.v[i]) * by;
        asm("" : "+v"(v));   // a product in binary32 for f16 too, not an instruction that rounds the exact one to 16 bits
        p.v[i] = static_cast<T>(v);
      }
      store_piece<ONCE>(m.out + row * m.out_stride, piece, p, valid);
    });
}

// out = grad min(1, most / norm), the product in binary32, rounded once more to the type.  Bound by memory: 1.88 GB f32 709 us, 5.3 TB/s read and written.
// The last workgroups' pieces first: they are what the norm has read last, and the caches have.
template <bool FLAT, bool ONCE>
__global__ __launch_bounds__(kGradientThreads) void gradient_clip_kernel(GradientArgs<FLAT> a) {
  uint64_t begin;
  const Matrix m = matrix_of(a, gridDim.x - 1u - blockIdx.x, begin);
  const float norm = *a.norm, by = norm <= a.most ? 1.0f : a.most / norm;   // NaN of NaN
  if (by == 1.0f && m.in == m.out && m.in_stride == m.out_stride) return;
  if (m.dtype == 0u) scale_pieces<float, FLAT, ONCE>(m, begin, a.share, by);
  else if (m.dtype == 1u) scale_pieces<__bf16, FLAT, ONCE>(m, begin, a.share, by);
  else scale_pieces<_Float16, FLAT, ONCE>(m, begin, a.share, by);
}

}  // namespace
