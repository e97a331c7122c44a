// Rows to microscaled 4 bits, and products grouped by expert of weights in them (device code).  Internal to the library.
#pragma once

#include "uccl_product_kernels.hpp"

namespace {

constexpr uint32_t kMx4Block = 32;

struct QuantiseArgs {
  Rows q, values, x;   // values.data: nullptr if there is none
  uint32_t rows, cols, pieces, groups;   // pieces of a row of x, workgroups of a row
};

// A lane has 16 bytes of a row, and the neighbours that share a block (4 of 16-bit elements, 8 of 32-bit) its greatest element.  x / s is exact:
// s is a power of two.  What is below the smallest normal number then is 0 in 4 bits all the same.
template <class T, bool ONCE>
__global__ __launch_bounds__(256) void quantise_kernel(QuantiseArgs a) {
  constexpr uint32_t N = Piece<T>::N, SHARE = kMx4Block / N;
  const uint64_t row = blockIdx.x / a.groups;
  const uint32_t piece = blockIdx.x % a.groups * 256u + threadIdx.x;
  Piece<T> x = load_piece_once<T>(a.x.data + row * a.x.stride, min(piece, a.pieces - 1u));
  const uint32_t valid = valid_of<T>(piece, a.pieces, a.cols);
  blank(x, valid);
  uint32_t most = 0u;
#pragma unroll
  for (uint32_t i = 0; i < N; ++i) most = max(most, __builtin_bit_cast(uint32_t, widen(x.v[i])) & 0x7FFFFFFFu);
#pragma unroll
  for (uint32_t d = 1; d < SHARE; d <<= 1) most = max(most, static_cast<uint32_t>(__shfl_xor(static_cast<int>(most), static_cast<int>(d))));
  const bool finite = most < 0x7F800000u;
  const uint32_t exponent = most >> 23, byte = !finite ? 255u : exponent < 2u ? 0u : exponent - 2u;
  const float by = finite ? __builtin_bit_cast(float, (254u - byte) << 23) : 0.0f;                                    // 1 / s
  const float s = !finite ? __builtin_nanf("") : byte == 0u ? 0x1p-127f : __builtin_bit_cast(float, byte << 23);
  uint32_t codes = 0u;
  Piece<T> out;
#pragma unroll
  for (uint32_t i = 0; i < N; ++i) {
    const float v = finite ? widen(x.v[i]) * by : 0.0f, m = fminf(fabsf(v), 6.0f);
    // the steps are 0.5 below 2, 1 below 4, 2 above
    const uint32_t number = m < 2.0f ? static_cast<uint32_t>(__builtin_rintf(m * 2.0f)) : m < 4.0f ? static_cast<uint32_t>(__builtin_rintf(m)) + 2u : static_cast<uint32_t>(__builtin_rintf(m * 0.5f)) + 4u;
    const uint32_t sign = __builtin_bit_cast(uint32_t, v) >> 31;
    codes |= (number | sign << 3) << (4u * i);
    const float value = number < 4u ? number * 0.5f : number == 4u ? 2.0f : number == 5u ? 3.0f : number == 6u ? 4.0f : 6.0f;
    out.v[i] = static_cast<T>((sign != 0u ? -value : value) * s);
  }
  if (valid == 0u) return;
  char* q = a.q.data + row * a.q.stride + piece * static_cast<uint64_t>(N / 2u);
  if (valid >= N) {
    if constexpr (N == 8u) *reinterpret_cast<uint32_t*>(q) = codes;
    else *reinterpret_cast<uint16_t*>(q) = static_cast<uint16_t>(codes);
  } else {
#pragma unroll
    for (uint32_t i = 0; i < N; i += 2u)
      if (i < valid) q[i / 2u] = static_cast<char>(codes >> (4u * i));
  }
  if (threadIdx.x % SHARE == 0u) reinterpret_cast<uint8_t*>(a.q.scales + row * a.q.scale_stride)[piece / SHARE] = static_cast<uint8_t>(byte);
  if (a.values.data != nullptr) store_piece<ONCE>(a.values.data + row * a.values.stride, piece, out, valid);
}

// ---- products ---------------------------------------------------------------------------------------
//
// out[i, n] = sum_k a[index[i], k] b[g, n, k] with b in microscaled 4 bits.  A lane has of a row 32 elements at a time, a block with a scale of its own.

typedef int i32x8 __attribute__((ext_vector_type(8)));

// Rows in 4 bits too: the matrix instruction for them takes the blocks' scales.  It has the products of a block exactly and adds the four
// blocks one after the other in binary32.
enum Mx4Rows : uint32_t { kRows4, kRowsBf16, kRowsF16 };

// Four bytes, two elements each, times 2^(byte - 127) as eight bf16: exact, for bf16 has all these powers.
__device__ __forceinline__ u32x4 widen_e2m1(uint32_t eight, float scale) {
  return u32x4{__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(eight, scale, 0)), __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(eight, scale, 1)),
               __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(eight, scale, 2)), __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(eight, scale, 3))};
}

// f16 has 11 bits, which are two bf16 exactly: the nearest one and what is left.
__device__ __forceinline__ void split_f16(u32x4 v, u32x4& high, u32x4& low) {
  const f16x8 f = __builtin_bit_cast(f16x8, v);
  bf16x8 h, l;
#pragma unroll
  for (uint32_t i = 0; i < 8u; ++i) {
    h[i] = static_cast<__bf16>(static_cast<float>(f[i]));
    l[i] = static_cast<__bf16>(static_cast<float>(f[i]) - static_cast<float>(h[i]));
  }
  high = __builtin_bit_cast(u32x4, h);
  low = __builtin_bit_cast(u32x4, l);
}

// One wavefront has 16 rows and 16 columns, straight from memory.
template <Mx4Rows X>
__global__ __launch_bounds__(64) void mx4_simple_kernel(ProductArgs a) {
  const uint32_t across = (a.wide + 15u) / 16u, lane = threadIdx.x, r = lane % 16u, quarter = lane / 16u;
  Group g;
  uint32_t r0, c0;
  if (!find_tile(a, 16u, across, g, r0, c0)) return;
  c0 *= 16u;
  const uint64_t n = static_cast<uint64_t>(g.index) * a.wide + min(c0 + r, a.wide - 1u);
  const char* w = a.b.data + n * a.b.stride;
  const uint8_t* ws = reinterpret_cast<const uint8_t*>(a.b.scales + n * a.b.scale_stride);
  uint32_t from = r0 + r;
  bool there = from < g.end;
  if (there && a.index != nullptr) from = static_cast<uint32_t>(a.index[from]);
  there = there && from < a.indexed_rows;
  const char* x = a.a.data + from * a.a.stride;
  const uint8_t* xs = reinterpret_cast<const uint8_t*>(a.a.scales + from * a.a.scale_stride);
  // a block's 16 bytes, of which those behind the row's end are 0
  auto load_4 = [&](const char* row, uint32_t first, bool some) {
    u32x4 v{};
    if (!some || first >= a.cols) return v;
    v = *reinterpret_cast<const u32x4*>(row + first / 2u);
    const uint32_t valid = a.cols - first;
#pragma unroll
    for (uint32_t i = 0; i < 4u; ++i)
      if (valid < (i + 1u) * 8u) v[i] &= valid <= i * 8u ? 0u : (1u << (valid - i * 8u) * 4u) - 1u;
    return v;
  };
  f32x4 acc{};
  for (uint32_t k = 0; k < a.cols; k += 128u) {
    const uint32_t first = k + quarter * 32u;
    const u32x4 fw = load_4(w, first, true);
    const uint32_t sw = first < a.cols ? ws[first / 32u] : 0u;
    if constexpr (X == kRows4) {
      const u32x4 fx = load_4(x, first, there);
      const uint32_t sx = there && first < a.cols ? xs[first / 32u] : 0u;
      const i32x8 vw{static_cast<int>(fw.x), static_cast<int>(fw.y), static_cast<int>(fw.z), static_cast<int>(fw.w), 0, 0, 0, 0};
      const i32x8 vx{static_cast<int>(fx.x), static_cast<int>(fx.y), static_cast<int>(fx.z), static_cast<int>(fx.w), 0, 0, 0, 0};
      acc = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(vw, vx, acc, 4, 4, 0, static_cast<int>(sw), 0, static_cast<int>(sx));
    } else {
      const float s = __builtin_bit_cast(float, sw << 23);
#pragma unroll
      for (uint32_t j = 0; j < 4u; ++j) {
        u32x4 fx{};
        const uint32_t at = first + j * 8u;
        if (there && at < a.cols) {
          Piece<uint16_t> p = load_piece<uint16_t>(x, at / 8u);
#pragma unroll
          for (uint32_t i = 0; i < 8u; ++i)
            if (at + i >= a.cols) p.v[i] = 0;
          fx = __builtin_bit_cast(u32x4, p);
        }
        const u32x4 b = widen_e2m1(fw[j], s);
        if constexpr (X == kRowsF16) {
          u32x4 high, low;
          split_f16(fx, high, low);
          acc = multiply<kBf16>(b, high, acc);
          acc = multiply<kBf16>(b, low, acc);
        } else {
          acc = multiply<kBf16>(b, fx, acc);
        }
      }
    }
  }
  const uint32_t row = r0 + r;
  if (row >= g.end) return;
  char* out = a.out.data + row * a.out.stride;
#pragma unroll
  for (uint32_t i = 0; i < 4u; ++i) {
    const uint32_t c = c0 + quarter * 4u + i;
    if (c >= a.wide) continue;
    if (a.out_type == kOutF32) reinterpret_cast<float*>(out)[c] = acc[i];
    else if (a.out_type == kOutBf16) reinterpret_cast<__bf16*>(out)[c] = static_cast<__bf16>(acc[i]);
    else reinterpret_cast<_Float16*>(out)[c] = static_cast<_Float16>(acc[i]);
  }
}

}  // namespace
