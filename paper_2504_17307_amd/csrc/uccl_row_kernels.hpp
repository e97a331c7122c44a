// Norm of rows, combination of rows, and their gradients (device code).  Internal to the library.
#pragma once

#include "uccl_row_elements.hpp"

namespace {

constexpr float kE4m3Max = 448.0f;
constexpr float kLeastScale = 1.17549435e-38f;   // 2^-126

// Reduce over the threads of a workgroup that share a row; `buffer`: one float a wavefront, of its own for every use.
template <uint32_t THREADS, bool MAX>
__device__ __forceinline__ float group_reduce(float v, float* buffer) {
  v = MAX ? wave_max(v) : wave_sum(v);
  if constexpr (THREADS > 64u) {
    if ((threadIdx.x & 63u) == 0u) buffer[threadIdx.x / 64u] = v;
    __syncthreads();
    v = buffer[0];
#pragma unroll
    for (uint32_t i = 1; i < THREADS / 64u; ++i) v = MAX ? fmaxf(v, buffer[i]) : v + buffer[i];
  }
  return v;
}

// Quotients by one scale, as a binary32 division rounds them (Markstein's method: the product with the rounded reciprocal is off by less than
// two steps, its remainder is exact, and what that adds rounds once).  A tiny scale is divided by as if it and the quotient's numerator were 2^64 times as large, so that
// no remainder that can move an e4m3 value underflows.  4096 x 7168 in bf16 with a residual to e4m3: 37.5 us so, 38.7 by division, 36.8 by the reciprocal alone, which
// gives the neighbour beside some ties.
struct Divisor {
  float scale, per, up;
};
__device__ __forceinline__ Divisor divisor(float scale) {
  const float up = scale < 0x1p-60f ? 0x1p64f : 1.0f;
  return Divisor{scale * up, 1.0f / (scale * up), up};
}
__device__ __forceinline__ float quotient(float v, const Divisor& d) {
  v *= d.up;
  const float q = v * d.per;
  return d.per == 0.0f ? q : __builtin_fmaf(-__builtin_fmaf(q, d.scale, -v), d.per, q);   // an infinite scale: 0, or NaN for an infinity
}

struct NormArgs {
  Rows y, h, x, r;     // h.data, r.data: nullptr if there is none
  const char* weight;
  float* rstd;         // or nullptr
  uint32_t rows, cols;
  float eps;
  float shrink, mean;  // a power of two near 1 / sqrt(cols), and 1 / (cols shrink^2)
};

// The mean square is summed from (h shrink)^2, which is exact and no greater than the mean itself: a row whose mean
// square binary32 can hold has it, however long the row is.
__device__ __forceinline__ float add_square(float h, float shrink, float sum) { return __builtin_fmaf(h * shrink, h * shrink, sum); }

// One workgroup a row.  h = x + r; s = rsqrt(mean h^2 + eps); y = h s w, from h as it was summed in 32 bits, not as it
// is rounded for storage.  E8: y in e4m3 with a scale a row.  All loads are issued before the first is waited for: threads past
// the row's end load its last piece.  Bound by HBM: 4096 x 7168 in bf16 with a residual to e4m3 37.5 us, 5.5 TB/s.
template <class T, bool E8, uint32_t THREADS, uint32_t NV, bool ONCE>
__global__ __launch_bounds__(THREADS) void norm_kernel(NormArgs a) {
  constexpr uint32_t N = Piece<T>::N;
  __shared__ float buffer[2][THREADS / 64u];
  const uint64_t row = blockIdx.x;
  const uint32_t pieces = (a.cols + N - 1) / N;
  const char* x = a.x.data + row * a.x.stride;
  Piece<T> px[NV], pr[NV], w[NV];
  uint32_t valid[NV];
#pragma unroll
  for (uint32_t k = 0; k < NV; ++k) px[k] = load_piece_once<T>(x, min(threadIdx.x + k * THREADS, pieces - 1u));
  if (a.r.data != nullptr) {
    const char* r = a.r.data + row * a.r.stride;
#pragma unroll
    for (uint32_t k = 0; k < NV; ++k) pr[k] = load_piece_once<T>(r, min(threadIdx.x + k * THREADS, pieces - 1u));
  } else {
#pragma unroll
    for (uint32_t k = 0; k < NV; ++k) pr[k] = Piece<T>{};
  }
#pragma unroll
  for (uint32_t k = 0; k < NV; ++k) w[k] = load_piece<T>(a.weight, min(threadIdx.x + k * THREADS, pieces - 1u));
  float h[NV][N];
  float ss = 0.0f;
#pragma unroll
  for (uint32_t k = 0; k < NV; ++k) {
    valid[k] = valid_of<T>(threadIdx.x + k * THREADS, pieces, a.cols);
    blank(px[k], valid[k]);
    blank(pr[k], valid[k]);
    blank(w[k], valid[k]);
#pragma unroll
    for (uint32_t i = 0; i < N; ++i) {
      h[k][i] = widen(px[k].v[i]) + widen(pr[k].v[i]);
      ss = add_square(h[k][i], a.shrink, ss);
    }
  }
  ss = group_reduce<THREADS, false>(ss, buffer[0]);
  const float s = 1.0f / sqrtf(ss * a.mean + a.eps);
  if (a.rstd != nullptr && threadIdx.x == 0u) a.rstd[row] = s;
  float most = 0.0f;
#pragma unroll
  for (uint32_t k = 0; k < NV; ++k) {
    const uint32_t p = threadIdx.x + k * THREADS;
    Piece<T> out;
    if (a.h.data != nullptr) {
#pragma unroll
      for (uint32_t i = 0; i < N; ++i) out.v[i] = static_cast<T>(h[k][i]);
      store_piece<ONCE>(a.h.data + row * a.h.stride, p, out, valid[k]);
    }
#pragma unroll
    for (uint32_t i = 0; i < N; ++i) {
      h[k][i] = h[k][i] * s * widen(w[k].v[i]);
      if constexpr (E8) most = fmaxf(most, fabsf(h[k][i]));
      else out.v[i] = static_cast<T>(h[k][i]);
    }
    if constexpr (!E8) store_piece<ONCE>(a.y.data + row * a.y.stride, p, out, valid[k]);
  }
  if constexpr (E8) {
    most = group_reduce<THREADS, true>(most, buffer[1]);
    const float scale = fmaxf(most / kE4m3Max, kLeastScale);
    if (threadIdx.x == 0u) *reinterpret_cast<float*>(a.y.scales + row * a.y.scale_stride) = scale;
    const Divisor by = divisor(scale);
    char* y = a.y.data + row * a.y.stride;
#pragma unroll
    for (uint32_t k = 0; k < NV; ++k) {
      const uint32_t p = threadIdx.x + k * THREADS;
      uint32_t q[N / 4];
#pragma unroll
      for (uint32_t i = 0; i < N / 4; ++i) {
        int v = __builtin_amdgcn_cvt_pk_fp8_f32(quotient(h[k][4 * i], by), quotient(h[k][4 * i + 1], by), 0, false);
        q[i] = static_cast<uint32_t>(__builtin_amdgcn_cvt_pk_fp8_f32(quotient(h[k][4 * i + 2], by), quotient(h[k][4 * i + 3], by), v, true));
      }
      char* at = y + p * N;
      if (valid[k] >= N) {
        if constexpr (N == 8 && ONCE) __builtin_nontemporal_store(u32x2{q[0], q[1]}, reinterpret_cast<u32x2*>(at));
        else if constexpr (N == 8) *reinterpret_cast<u32x2*>(at) = u32x2{q[0], q[1]};
        else if constexpr (ONCE) __builtin_nontemporal_store(q[0], reinterpret_cast<uint32_t*>(at));
        else *reinterpret_cast<uint32_t*>(at) = q[0];
      } else {
#pragma unroll
        for (uint32_t i = 0; i < N; ++i)
          if (i < valid[k]) at[i] = static_cast<char>(q[i / 4] >> (8 * (i % 4)));
      }
    }
  }
}

// The same for rows of any length: three passes over the row, which is in the L2 after the first one (2048 x 40000 in bf16 155 us, 4.2 TB/s).
template <class T, bool E8>
__global__ __launch_bounds__(1024) void norm_long_kernel(NormArgs a) {
  constexpr uint32_t N = Piece<T>::N, THREADS = 1024;
  __shared__ float buffer[2][THREADS / 64u];
  const uint64_t row = blockIdx.x;
  const uint32_t pieces = (a.cols + N - 1) / N;
  const char* x = a.x.data + row * a.x.stride;
  const char* r = a.r.data == nullptr ? nullptr : a.r.data + row * a.r.stride;
  char* y = a.y.data + row * a.y.stride;
  float h[N];
  auto load = [&](uint32_t p) {
    const uint32_t valid = a.cols - p * N;
    Piece<T> px = load_piece<T>(x, p), pr{};
    if (r != nullptr) pr = load_piece<T>(r, p);
    blank(px, valid);
    blank(pr, valid);
#pragma unroll
    for (uint32_t i = 0; i < N; ++i) h[i] = widen(px.v[i]) + widen(pr.v[i]);
  };
  float ss = 0.0f;
  for (uint32_t p = threadIdx.x; p < pieces; p += THREADS) {
    load(p);
#pragma unroll
    for (uint32_t i = 0; i < N; ++i) ss = add_square(h[i], a.shrink, ss);
  }
  ss = group_reduce<THREADS, false>(ss, buffer[0]);
  const float s = 1.0f / sqrtf(ss * a.mean + a.eps);
  if (a.rstd != nullptr && threadIdx.x == 0u) a.rstd[row] = s;
  Divisor by{1.0f, 1.0f, 1.0f};
  if constexpr (E8) {
    float most = 0.0f;
    for (uint32_t p = threadIdx.x; p < pieces; p += THREADS) {
      load(p);
      Piece<T> w = load_piece<T>(a.weight, p);
      blank(w, a.cols - p * N);
#pragma unroll
      for (uint32_t i = 0; i < N; ++i) most = fmaxf(most, fabsf(h[i] * s * widen(w.v[i])));
    }
    most = group_reduce<THREADS, true>(most, buffer[1]);
    const float scale = fmaxf(most / kE4m3Max, kLeastScale);
    if (threadIdx.x == 0u) *reinterpret_cast<float*>(a.y.scales + row * a.y.scale_stride) = scale;
    by = divisor(scale);
  }
  // a piece is read and written by the same thread, so h may lie where x or r does
  for (uint32_t p = threadIdx.x; p < pieces; p += THREADS) {
    load(p);
    const uint32_t valid = a.cols - p * N;
    Piece<T> w = load_piece<T>(a.weight, p), out;
    blank(w, valid);
    if (a.h.data != nullptr) {
#pragma unroll
      for (uint32_t i = 0; i < N; ++i) out.v[i] = static_cast<T>(h[i]);
      store_piece<false>(a.h.data + row * a.h.stride, p, out, valid);
    }
#pragma unroll
    for (uint32_t i = 0; i < N; ++i) {
      const float v = h[i] * s * widen(w.v[i]);
      if constexpr (E8) {
        if (i < valid) y[p * static_cast<uint64_t>(N) + i] = static_cast<char>(__builtin_amdgcn_cvt_pk_fp8_f32(quotient(v, by), 0.0f, 0, false));
      } else {
        out.v[i] = static_cast<T>(v);
      }
    }
    if constexpr (!E8) store_piece<false>(y, p, out, valid);
  }
}

struct NormGradArgs {
  Rows dx, dy, h, dh;   // dh.data: nullptr if there is none
  const char* weight;
  const float* rstd;
  float* parts;         // [gridDim.x][cols] sums of the weight's gradient over a workgroup's rows
  uint32_t rows, cols;
};

// n = h s, g = dy w: dx = dh + s (g - n mean(g n)); the weight's gradient is the sum of dy n over the rows, of which a
// workgroup takes every gridDim.x-th and leaves its sum for column_sum_kernel: no atomics, the order is always the same.  A row's
// loads are issued before the row before it is reduced and written.  Bound by HBM: 4096 x 7168 in bf16 46.8 us with the second launch, 5.0 TB/s.
template <class T, uint32_t THREADS, uint32_t NV, bool ONCE>
__global__ __launch_bounds__(THREADS) void norm_grad_kernel(NormGradArgs a) {
  constexpr uint32_t N = Piece<T>::N;
  constexpr bool LATE = NV * N > 16u;   // no registers for the next row's dh as well: a row's is asked for when its sum is formed
  __shared__ float buffer[2][THREADS / 64u];
  const uint32_t pieces = (a.cols + N - 1) / N;
  uint32_t at[NV], valid[NV];
#pragma unroll
  for (uint32_t k = 0; k < NV; ++k) {
    at[k] = min(threadIdx.x + k * THREADS, pieces - 1u);
    valid[k] = valid_of<T>(threadIdx.x + k * THREADS, pieces, a.cols);
  }
  struct Row {
    Piece<T> d[NV], h[NV], c[NV];
    float s;
  };
  auto load_carry = [&](Row& r, uint64_t row) {
    if (a.dh.data != nullptr) {
#pragma unroll
      for (uint32_t k = 0; k < NV; ++k) r.c[k] = load_piece_once<T>(a.dh.data + row * a.dh.stride, at[k]);
    } else {
#pragma unroll
      for (uint32_t k = 0; k < NV; ++k) r.c[k] = Piece<T>{};
    }
  };
  auto load = [&](uint64_t row) {
    Row r;
#pragma unroll
    for (uint32_t k = 0; k < NV; ++k) {
      r.d[k] = load_piece_once<T>(a.dy.data + row * a.dy.stride, at[k]);
      r.h[k] = load_piece_once<T>(a.h.data + row * a.h.stride, at[k]);
    }
    if constexpr (!LATE) load_carry(r, row);
    r.s = a.rstd[row];
    return r;
  };
  float dw[NV][N];
  Piece<T> w[NV];
  Row next = load(blockIdx.x);
#pragma unroll
  for (uint32_t k = 0; k < NV; ++k) {
    w[k] = load_piece<T>(a.weight, at[k]);
    blank(w[k], valid[k]);
#pragma unroll
    for (uint32_t i = 0; i < N; ++i) dw[k][i] = 0.0f;
  }
  uint32_t turn = 0;
  for (uint64_t row = blockIdx.x; row < a.rows; row += gridDim.x, turn ^= 1u) {
    Row r = next;
    if constexpr (LATE) {
      load_carry(r, row);
#pragma unroll
      for (uint32_t k = 0; k < NV; ++k) {   // the weight stays in 16 bits: it is not widened ahead of all rows
        u32x4 bits = __builtin_bit_cast(u32x4, w[k]);
        asm volatile("" : "+v"(bits));
        w[k] = __builtin_bit_cast(Piece<T>, bits);
      }
    }
    // dx may lie where dy or dh does, but a row is only written when it has been read, and by no other workgroup; the last row
    // is loaded once more for nothing, before it is written
    next = load(row + gridDim.x < a.rows ? row + gridDim.x : row);
    float along = 0.0f;
#pragma unroll
    for (uint32_t k = 0; k < NV; ++k) {
      blank(r.d[k], valid[k]);
      blank(r.h[k], valid[k]);
#pragma unroll
      for (uint32_t i = 0; i < N; ++i) {
        const float n = widen(r.h[k].v[i]) * r.s, d = widen(r.d[k].v[i]);
        dw[k][i] = __builtin_fmaf(d, n, dw[k][i]);
        along = __builtin_fmaf(d * widen(w[k].v[i]), n, along);
      }
    }
    // two buffers in turn: a wavefront that is ahead writes the other one, and the barrier of that row keeps it from the next
    along = group_reduce<THREADS, false>(along, buffer[turn]) / static_cast<float>(a.cols);
#pragma unroll
    for (uint32_t k = 0; k < NV; ++k) {
      Piece<T> out;
#pragma unroll
      for (uint32_t i = 0; i < N; ++i) {
        const float n = widen(r.h[k].v[i]) * r.s, g = widen(r.d[k].v[i]) * widen(w[k].v[i]);
        out.v[i] = static_cast<T>(__builtin_fmaf(r.s, g - n * along, widen(r.c[k].v[i])));
      }
      store_piece<ONCE>(a.dx.data + row * a.dx.stride, threadIdx.x + k * THREADS, out, valid[k]);
    }
  }
#pragma unroll
  for (uint32_t k = 0; k < NV; ++k)
#pragma unroll
    for (uint32_t i = 0; i < N; ++i)
      if (i < valid[k]) a.parts[static_cast<uint64_t>(blockIdx.x) * a.cols + (threadIdx.x + k * THREADS) * N + i] = dw[k][i];
}

// The same for rows of any length: the row's sum first, then what needs it; the weight's sums stay in memory (2048 x 40000 in bf16 422 us).
template <class T>
__global__ __launch_bounds__(1024) void norm_grad_long_kernel(NormGradArgs a) {
  constexpr uint32_t N = Piece<T>::N, THREADS = 1024;
  __shared__ float buffer[2][THREADS / 64u];
  const uint32_t pieces = (a.cols + N - 1) / N;
  uint32_t turn = 0;
  bool first = true;
  for (uint64_t row = blockIdx.x; row < a.rows; row += gridDim.x, turn ^= 1u, first = false) {
    const char* dy = a.dy.data + row * a.dy.stride;
    const char* h = a.h.data + row * a.h.stride;
    const char* dh = a.dh.data == nullptr ? nullptr : a.dh.data + row * a.dh.stride;
    const float s = a.rstd[row];
    float along = 0.0f;
    for (uint32_t p = threadIdx.x; p < pieces; p += THREADS) {
      Piece<T> pd = load_piece<T>(dy, p), ph = load_piece<T>(h, p), w = load_piece<T>(a.weight, p);
      const uint32_t valid = a.cols - p * N;
      blank(pd, valid);
      blank(ph, valid);
      blank(w, valid);
      float* part = a.parts + static_cast<uint64_t>(blockIdx.x) * a.cols + p * static_cast<uint64_t>(N);
#pragma unroll
      for (uint32_t i = 0; i < N; ++i) {
        const float n = widen(ph.v[i]) * s, d = widen(pd.v[i]);
        along = __builtin_fmaf(d * widen(w.v[i]), n, along);
        if (i < valid) part[i] = __builtin_fmaf(d, n, first ? 0.0f : part[i]);   // this thread's own at every row
      }
    }
    along = group_reduce<THREADS, false>(along, buffer[turn]) / static_cast<float>(a.cols);
    for (uint32_t p = threadIdx.x; p < pieces; p += THREADS) {
      Piece<T> pd = load_piece<T>(dy, p), ph = load_piece<T>(h, p), w = load_piece<T>(a.weight, p), pc{}, out;
      if (dh != nullptr) pc = load_piece<T>(dh, p);
#pragma unroll
      for (uint32_t i = 0; i < N; ++i) {
        const float n = widen(ph.v[i]) * s, g = widen(pd.v[i]) * widen(w.v[i]);
        out.v[i] = static_cast<T>(__builtin_fmaf(s, g - n * along, widen(pc.v[i])));
      }
      store_piece<false>(a.dx.data + row * a.dx.stride, p, out, a.cols - p * N);
    }
  }
}

// sums[c] = parts[0][c] + parts[1][c] + ...: 64 columns a workgroup, every one of 16 wavefronts a share of the parts, 8 loads at a time.
__global__ __launch_bounds__(1024) void column_sum_kernel(float* sums, const float* parts, uint32_t n, uint32_t cols) {
  __shared__ float buffer[16][64];
  const uint32_t lane = threadIdx.x & 63u, c = blockIdx.x * 64u + lane, wave = threadIdx.x / 64u;
  float v = 0.0f;
  if (c < cols)
    for (uint32_t i = wave; i < n; i += 16u * 8u) {
      float p[8];
#pragma unroll
      for (uint32_t j = 0; j < 8u; ++j) p[j] = i + j * 16u < n ? parts[static_cast<uint64_t>(i + j * 16u) * cols + c] : 0.0f;
#pragma unroll
      for (uint32_t j = 0; j < 8u; ++j) v += p[j];
    }
  buffer[wave][lane] = v;
  __syncthreads();
  if (wave == 0u && c < cols) {
#pragma unroll
    for (uint32_t i = 1; i < 16u; ++i) v += buffer[i][lane];
    sums[c] = v;
  }
}

struct CombineArgs {
  Rows out, y, r;          // r.data: nullptr if there is none
  const int32_t* pos;      // [tokens][slots]
  const float* weights;    // [tokens][slots], or nullptr: 1
  uint32_t tokens, slots, y_rows, cols;
  uint32_t blocks;         // workgroups a token
};

// out = r + sum_j w_j y[pos_j].  A thread has one 16-byte piece of the token's row and loads it from up to 8 of the rows
// before it adds the first: the work is the reading of those rows.  A slot without a row reads row 0 and does not count, so that no load
// waits for another; the host sees to it that there is a row 0, or no slot.  Bound by HBM: 4096 tokens x 8 slots x 7168 in bf16 89 us, 6.0 TB/s.
constexpr uint32_t kSlotsAtOnce = 8;

struct Slots {
  uint32_t row[kSlotsAtOnce];
  bool there[kSlotsAtOnce];
  float weight[kSlotsAtOnce];   // 0 where there is no row
};
__device__ __forceinline__ Slots load_slots(const int32_t* pos, const float* weights, uint32_t first, uint32_t slots, uint32_t y_rows) {
  Slots s;
#pragma unroll
  for (uint32_t j = 0; j < kSlotsAtOnce; ++j) s.row[j] = static_cast<uint32_t>(pos[min(first + j, slots - 1u)]);
  if (weights != nullptr) {
#pragma unroll
    for (uint32_t j = 0; j < kSlotsAtOnce; ++j) s.weight[j] = weights[min(first + j, slots - 1u)];
  } else {
#pragma unroll
    for (uint32_t j = 0; j < kSlotsAtOnce; ++j) s.weight[j] = 1.0f;
  }
#pragma unroll
  for (uint32_t j = 0; j < kSlotsAtOnce; ++j) {
    s.there[j] = first + j < slots && s.row[j] < y_rows;
    s.row[j] = s.there[j] ? s.row[j] : 0u;
    s.weight[j] = s.there[j] ? s.weight[j] : 0.0f;
  }
  return s;
}

template <class T, uint32_t THREADS, bool ONCE>
__global__ __launch_bounds__(THREADS) void combine_kernel(CombineArgs a) {
  constexpr uint32_t N = Piece<T>::N;
  const uint64_t token = blockIdx.x / a.blocks;
  const uint32_t p = (blockIdx.x % a.blocks) * THREADS + threadIdx.x, pieces = (a.cols + N - 1) / N;
  if (p >= pieces) return;
  Piece<T> pr{};
  if (a.r.data != nullptr) pr = load_piece_once<T>(a.r.data + token * a.r.stride, p);
  float sum[N];
  for (uint32_t j0 = 0; j0 < a.slots; j0 += kSlotsAtOnce) {
    const Slots s = load_slots(a.pos + token * a.slots, a.weights == nullptr ? nullptr : a.weights + token * a.slots, j0, a.slots, a.y_rows);
    Piece<T> py[kSlotsAtOnce];
#pragma unroll
    for (uint32_t j = 0; j < kSlotsAtOnce; ++j) py[j] = load_piece_once<T>(a.y.data + s.row[j] * a.y.stride, p);
    if (j0 == 0u) {
#pragma unroll
      for (uint32_t i = 0; i < N; ++i) sum[i] = widen(pr.v[i]);
    }
#pragma unroll
    for (uint32_t j = 0; j < kSlotsAtOnce; ++j)
#pragma unroll
      for (uint32_t i = 0; i < N; ++i) sum[i] = __builtin_fmaf(s.weight[j], s.there[j] ? widen(py[j].v[i]) : 0.0f, sum[i]);
  }
  if (a.slots == 0u) {
#pragma unroll
    for (uint32_t i = 0; i < N; ++i) sum[i] = widen(pr.v[i]);
  }
  Piece<T> out;
#pragma unroll
  for (uint32_t i = 0; i < N; ++i) out.v[i] = static_cast<T>(sum[i]);
  store_piece<ONCE>(a.out.data + token * a.out.stride, p, out, a.cols - p * N);
}

struct CombineGradArgs {
  Rows dy, dout, y;
  const int32_t* pos;
  const float* weights;   // or nullptr: 1
  float* dw;              // [tokens][slots], or nullptr: not wanted
  uint32_t tokens, slots, y_rows, cols;
};

// dy[pos_j] = w_j dout; dw_j = dout . y[pos_j].  One workgroup a token, 8 slots at a time, so that dout is read once for them.  Bound by HBM:
// 1024 tokens x 8 slots x 7168 in bf16 50.6 us, 4.9 TB/s.
template <class T, bool ONCE>
__global__ __launch_bounds__(256) void combine_grad_kernel(CombineGradArgs a) {
  constexpr uint32_t N = Piece<T>::N;
  __shared__ float buffer[4][kSlotsAtOnce];
  const uint64_t token = blockIdx.x;
  const uint32_t pieces = (a.cols + N - 1) / N;
  const char* dout = a.dout.data + token * a.dout.stride;
  for (uint32_t j0 = 0; j0 < a.slots; j0 += kSlotsAtOnce) {
    const Slots s = load_slots(a.pos + token * a.slots, a.weights == nullptr ? nullptr : a.weights + token * a.slots, j0, a.slots, a.y_rows);
    float dot[kSlotsAtOnce];
#pragma unroll
    for (uint32_t j = 0; j < kSlotsAtOnce; ++j) dot[j] = 0.0f;
    for (uint32_t p = threadIdx.x; p < pieces; p += 256u) {
      const uint32_t valid = a.cols - p * N;
      Piece<T> pd = load_piece<T>(dout, p), py[kSlotsAtOnce];
      if (a.dw != nullptr) {
#pragma unroll
        for (uint32_t j = 0; j < kSlotsAtOnce; ++j) py[j] = load_piece_once<T>(a.y.data + s.row[j] * a.y.stride, p);
#pragma unroll
        for (uint32_t j = 0; j < kSlotsAtOnce; ++j) blank(py[j], s.there[j] ? valid : 0u);
        blank(pd, valid);
#pragma unroll
        for (uint32_t j = 0; j < kSlotsAtOnce; ++j)
#pragma unroll
          for (uint32_t i = 0; i < N; ++i) dot[j] = __builtin_fmaf(widen(pd.v[i]), widen(py[j].v[i]), dot[j]);
      }
#pragma unroll
      for (uint32_t j = 0; j < kSlotsAtOnce; ++j)
        if (s.there[j]) {
          Piece<T> out;
#pragma unroll
          for (uint32_t i = 0; i < N; ++i) out.v[i] = static_cast<T>(s.weight[j] * widen(pd.v[i]));
          store_piece<ONCE>(a.dy.data + s.row[j] * a.dy.stride, p, out, valid);
        }
    }
    if (a.dw != nullptr) {
#pragma unroll
      for (uint32_t j = 0; j < kSlotsAtOnce; ++j) {
        const float v = wave_sum(dot[j]);
        if ((threadIdx.x & 63u) == 0u) buffer[threadIdx.x / 64u][j] = v;
      }
      __syncthreads();
      if (threadIdx.x < kSlotsAtOnce && j0 + threadIdx.x < a.slots)
        a.dw[token * a.slots + j0 + threadIdx.x] =
            (buffer[0][threadIdx.x] + buffer[1][threadIdx.x]) + (buffer[2][threadIdx.x] + buffer[3][threadIdx.x]);
      __syncthreads();
    }
  }
}

}  // namespace
