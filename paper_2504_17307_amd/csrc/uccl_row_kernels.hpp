// Norm of rows, combination of rows, and their gradients (device code).  Internal to the library.
#pragma once

#include "uccl_row_elements.hpp"

namespace {

constexpr float kE4m3Max = 448.0f;
constexpr float kLeastScale = 1.17549435e-38f;   // 2^-126: its reciprocal is finite

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
// is rounded for storage.  E8: y in e4m3 with a scale a row.
template <class T, bool E8, uint32_t THREADS, uint32_t NV>
__global__ __launch_bounds__(THREADS) void norm_kernel(NormArgs a) {
  constexpr uint32_t N = Piece<T>::N;
  __shared__ float buffer[2][THREADS / 64u];
  const uint64_t row = blockIdx.x;
  const uint32_t pieces = (a.cols + N - 1) / N;
  const char* x = a.x.data + row * a.x.stride;
  const char* r = a.r.data == nullptr ? nullptr : a.r.data + row * a.r.stride;
  float h[NV][N];
  float ss = 0.0f;
#pragma unroll
  for (uint32_t k = 0; k < NV; ++k) {
    const uint32_t p = threadIdx.x + k * THREADS;
    Piece<T> px{}, pr{};
    if (p < pieces) {
      px = load_piece<T>(x, p);
      if (r != nullptr) pr = load_piece<T>(r, p);
      const uint32_t valid = a.cols - p * N;
      blank(px, valid);
      blank(pr, valid);
    }
#pragma unroll
    for (uint32_t i = 0; i < N; ++i) {
      h[k][i] = widen(px.v[i]) + widen(pr.v[i]);
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
    if (p < pieces) {
      const uint32_t valid = a.cols - p * N;
      Piece<T> w = load_piece<T>(a.weight, p);
      blank(w, valid);
      Piece<T> out;
      if (a.h.data != nullptr) {
#pragma unroll
        for (uint32_t i = 0; i < N; ++i) out.v[i] = static_cast<T>(h[k][i]);
        store_piece(a.h.data + row * a.h.stride, p, out, valid);
      }
#pragma unroll
      for (uint32_t i = 0; i < N; ++i) {
        h[k][i] = h[k][i] * s * widen(w.v[i]);
        if constexpr (E8) most = fmaxf(most, fabsf(h[k][i]));
        else out.v[i] = static_cast<T>(h[k][i]);
      }
      if constexpr (!E8) store_piece(a.y.data + row * a.y.stride, p, out, valid);
    }
  }
  if constexpr (E8) {
    most = group_reduce<THREADS, true>(most, buffer[1]);
    const float scale = fmaxf(most / kE4m3Max, kLeastScale);
    if (threadIdx.x == 0u) *reinterpret_cast<float*>(a.y.scales + row * a.y.scale_stride) = scale;
    const float per = 1.0f / scale;
    char* y = a.y.data + row * a.y.stride;
#pragma unroll
    for (uint32_t k = 0; k < NV; ++k) {
      const uint32_t p = threadIdx.x + k * THREADS;
      if (p < pieces) {
        const uint32_t valid = a.cols - p * N;
        uint32_t q[N / 4];
#pragma unroll
        for (uint32_t i = 0; i < N / 4; ++i) {
          int v = __builtin_amdgcn_cvt_pk_fp8_f32(h[k][4 * i] * per, h[k][4 * i + 1] * per, 0, false);
          q[i] = static_cast<uint32_t>(__builtin_amdgcn_cvt_pk_fp8_f32(h[k][4 * i + 2] * per, h[k][4 * i + 3] * per, v, true));
        }
        char* at = y + p * N;
        if (valid >= N) {
          if constexpr (N == 8) *reinterpret_cast<u32x2*>(at) = u32x2{q[0], q[1]};
          else *reinterpret_cast<uint32_t*>(at) = q[0];
        } else {
#pragma unroll
          for (uint32_t i = 0; i < N; ++i)
            if (i < valid) at[i] = static_cast<char>(q[i / 4] >> (8 * (i % 4)));
        }
      }
    }
  }
}

// The same for rows of any length: three passes over the row, which is in the L2 after the first one.
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
  float per = 1.0f;
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
    per = 1.0f / scale;
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
      store_piece(a.h.data + row * a.h.stride, p, out, valid);
    }
#pragma unroll
    for (uint32_t i = 0; i < N; ++i) {
      const float v = h[i] * s * widen(w.v[i]);
      if constexpr (E8) {
        if (i < valid) y[p * static_cast<uint64_t>(N) + i] = static_cast<char>(__builtin_amdgcn_cvt_pk_fp8_f32(v * per, 0.0f, 0, false));
      } else {
        out.v[i] = static_cast<T>(v);
      }
    }
    if constexpr (!E8) store_piece(y, p, out, valid);
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
// workgroup takes every gridDim.x-th and leaves its sum for column_sum_kernel: no atomics, the order is always the same.
template <class T, uint32_t THREADS, uint32_t NV>
__global__ __launch_bounds__(THREADS) void norm_grad_kernel(NormGradArgs a) {
  constexpr uint32_t N = Piece<T>::N;
  __shared__ float buffer[2][THREADS / 64u];
  const uint32_t pieces = (a.cols + N - 1) / N;
  float dw[NV][N];
  Piece<T> w[NV];
#pragma unroll
  for (uint32_t k = 0; k < NV; ++k) {
    const uint32_t p = threadIdx.x + k * THREADS;
    w[k] = Piece<T>{};
    if (p < pieces) w[k] = load_piece<T>(a.weight, p);
#pragma unroll
    for (uint32_t i = 0; i < N; ++i) dw[k][i] = 0.0f;
  }
  uint32_t turn = 0;
  for (uint64_t row = blockIdx.x; row < a.rows; row += gridDim.x, turn ^= 1u) {
    const char* dy = a.dy.data + row * a.dy.stride;
    const char* h = a.h.data + row * a.h.stride;
    const char* dh = a.dh.data == nullptr ? nullptr : a.dh.data + row * a.dh.stride;
    Piece<T> pd[NV], ph[NV], pc[NV];
#pragma unroll
    for (uint32_t k = 0; k < NV; ++k) {
      const uint32_t p = threadIdx.x + k * THREADS;
      pd[k] = ph[k] = pc[k] = Piece<T>{};
      if (p < pieces) {
        pd[k] = load_piece<T>(dy, p);
        ph[k] = load_piece<T>(h, p);
        if (dh != nullptr) pc[k] = load_piece<T>(dh, p);
        const uint32_t valid = a.cols - p * N;
        blank(pd[k], valid);
        blank(ph[k], valid);
        blank(w[k], valid);
      }
    }
    const float s = a.rstd[row];
    float along = 0.0f;
#pragma unroll
    for (uint32_t k = 0; k < NV; ++k)
#pragma unroll
      for (uint32_t i = 0; i < N; ++i) {
        const float n = widen(ph[k].v[i]) * s, d = widen(pd[k].v[i]);
        dw[k][i] = __builtin_fmaf(d, n, dw[k][i]);
        along = __builtin_fmaf(d * widen(w[k].v[i]), n, along);
      }
    // two buffers in turn: a wavefront that is ahead writes the other one, and the barrier of that row keeps it from the next
    along = group_reduce<THREADS, false>(along, buffer[turn]) / static_cast<float>(a.cols);
#pragma unroll
    for (uint32_t k = 0; k < NV; ++k) {
      const uint32_t p = threadIdx.x + k * THREADS;
      if (p < pieces) {
        Piece<T> out;
#pragma unroll
        for (uint32_t i = 0; i < N; ++i) {
          const float n = widen(ph[k].v[i]) * s, g = widen(pd[k].v[i]) * widen(w[k].v[i]);
          out.v[i] = static_cast<T>(__builtin_fmaf(s, g - n * along, widen(pc[k].v[i])));
        }
        store_piece(a.dx.data + row * a.dx.stride, p, out, a.cols - p * N);
      }
    }
  }
#pragma unroll
  for (uint32_t k = 0; k < NV; ++k) {
    const uint32_t p = threadIdx.x + k * THREADS;
#pragma unroll
    for (uint32_t i = 0; i < N; ++i)
      if (p < pieces && p * N + i < a.cols) a.parts[static_cast<uint64_t>(blockIdx.x) * a.cols + p * N + i] = dw[k][i];
  }
}

// The same for rows of any length, a column block of 4096 / N pieces at a time: the row's sum first, then what needs it.
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
      store_piece(a.dx.data + row * a.dx.stride, p, out, a.cols - p * N);
    }
  }
}

// sums[c] = parts[0][c] + parts[1][c] + ...: 64 columns a workgroup, every wavefront a share of the parts.
__global__ __launch_bounds__(256) void column_sum_kernel(float* sums, const float* parts, uint32_t n, uint32_t cols) {
  __shared__ float buffer[4][64];
  const uint32_t c = blockIdx.x * 64u + (threadIdx.x & 63u), wave = threadIdx.x / 64u;
  float v = 0.0f;
  if (c < cols)
    for (uint32_t i = wave; i < n; i += 4u) v += parts[static_cast<uint64_t>(i) * cols + c];
  buffer[wave][threadIdx.x & 63u] = v;
  __syncthreads();
  if (wave == 0u && c < cols) sums[c] = (buffer[0][threadIdx.x] + buffer[1][threadIdx.x]) + (buffer[2][threadIdx.x] + buffer[3][threadIdx.x]);
}

struct CombineArgs {
  Rows out, y, r;          // r.data: nullptr if there is none
  const int32_t* pos;      // [tokens][slots]
  const float* weights;    // [tokens][slots], or nullptr: 1
  uint32_t tokens, slots, y_rows, cols;
  uint32_t blocks;         // workgroups a token
};

// out = r + sum_j w_j y[pos_j].  A thread has one 16-byte piece of the token's row and loads it from up to 8 of the rows
// before it adds the first: the work is the reading of those rows.
template <class T>
__global__ __launch_bounds__(256) void combine_kernel(CombineArgs a) {
  constexpr uint32_t N = Piece<T>::N, AT_ONCE = 8;
  const uint64_t token = blockIdx.x / a.blocks;
  const uint32_t p = (blockIdx.x % a.blocks) * 256u + threadIdx.x, pieces = (a.cols + N - 1) / N;
  if (p >= pieces) return;
  float sum[N];
  if (a.r.data != nullptr) {
    const Piece<T> pr = load_piece<T>(a.r.data + token * a.r.stride, p);
#pragma unroll
    for (uint32_t i = 0; i < N; ++i) sum[i] = widen(pr.v[i]);
  } else {
#pragma unroll
    for (uint32_t i = 0; i < N; ++i) sum[i] = 0.0f;
  }
  const int32_t* pos = a.pos + token * a.slots;
  for (uint32_t j0 = 0; j0 < a.slots; j0 += AT_ONCE) {
    Piece<T> py[AT_ONCE];
    float w[AT_ONCE];
    bool there[AT_ONCE];
#pragma unroll
    for (uint32_t j = 0; j < AT_ONCE; ++j) {
      const uint32_t at = j0 + j < a.slots ? static_cast<uint32_t>(pos[j0 + j]) : 0xFFFFFFFFu;
      there[j] = at < a.y_rows;
      w[j] = 1.0f;
      if (there[j]) {
        py[j] = load_piece<T>(a.y.data + at * a.y.stride, p);
        if (a.weights != nullptr) w[j] = a.weights[token * a.slots + j0 + j];
      }
    }
#pragma unroll
    for (uint32_t j = 0; j < AT_ONCE; ++j)
      if (there[j]) {
#pragma unroll
        for (uint32_t i = 0; i < N; ++i) sum[i] = __builtin_fmaf(w[j], widen(py[j].v[i]), sum[i]);
      }
  }
  Piece<T> out;
#pragma unroll
  for (uint32_t i = 0; i < N; ++i) out.v[i] = static_cast<T>(sum[i]);
  store_piece(a.out.data + token * a.out.stride, p, out, a.cols - p * N);
}

struct CombineGradArgs {
  Rows dy, dout, y;
  const int32_t* pos;
  const float* weights;   // or nullptr: 1
  float* dw;              // [tokens][slots], or nullptr: not wanted
  uint32_t tokens, slots, y_rows, cols;
};

// dy[pos_j] = w_j dout; dw_j = dout . y[pos_j].  One workgroup a token, 8 slots at a time, so that dout is read once for them.
template <class T>
__global__ __launch_bounds__(256) void combine_grad_kernel(CombineGradArgs a) {
  constexpr uint32_t N = Piece<T>::N, AT_ONCE = 8;
  __shared__ float buffer[4][AT_ONCE];
  const uint64_t token = blockIdx.x;
  const uint32_t pieces = (a.cols + N - 1) / N;
  const char* dout = a.dout.data + token * a.dout.stride;
  for (uint32_t j0 = 0; j0 < a.slots; j0 += AT_ONCE) {
    float dot[AT_ONCE], w[AT_ONCE];
    uint32_t at[AT_ONCE];
#pragma unroll
    for (uint32_t j = 0; j < AT_ONCE; ++j) {
      at[j] = j0 + j < a.slots ? static_cast<uint32_t>(a.pos[token * a.slots + j0 + j]) : 0xFFFFFFFFu;
      w[j] = at[j] < a.y_rows && a.weights != nullptr ? a.weights[token * a.slots + j0 + j] : 1.0f;
      dot[j] = 0.0f;
    }
    for (uint32_t p = threadIdx.x; p < pieces; p += 256u) {
      const uint32_t valid = a.cols - p * N;
      Piece<T> pd = load_piece<T>(dout, p), py[AT_ONCE];
      if (a.dw != nullptr) {
#pragma unroll
        for (uint32_t j = 0; j < AT_ONCE; ++j)
          if (at[j] < a.y_rows) py[j] = load_piece<T>(a.y.data + at[j] * a.y.stride, p);
      }
      blank(pd, valid);
#pragma unroll
      for (uint32_t j = 0; j < AT_ONCE; ++j)
        if (at[j] < a.y_rows) {
          Piece<T> out;
          if (a.dw != nullptr) blank(py[j], valid);
#pragma unroll
          for (uint32_t i = 0; i < N; ++i) {
            if (a.dw != nullptr) dot[j] = __builtin_fmaf(widen(pd.v[i]), widen(py[j].v[i]), dot[j]);
            out.v[i] = static_cast<T>(w[j] * widen(pd.v[i]));
          }
          store_piece(a.dy.data + at[j] * a.dy.stride, p, out, valid);
        }
    }
    if (a.dw != nullptr) {
#pragma unroll
      for (uint32_t j = 0; j < AT_ONCE; ++j) {
        const float v = wave_sum(dot[j]);
        if ((threadIdx.x & 63u) == 0u) buffer[threadIdx.x / 64u][j] = v;
      }
      __syncthreads();
      if (threadIdx.x < AT_ONCE && j0 + threadIdx.x < a.slots)
        a.dw[token * a.slots + j0 + threadIdx.x] =
            (buffer[0][threadIdx.x] + buffer[1][threadIdx.x]) + (buffer[2][threadIdx.x] + buffer[3][threadIdx.x]);
      __syncthreads();
    }
  }
}

}  // namespace
