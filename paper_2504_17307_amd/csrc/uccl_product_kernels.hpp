// Matrix products grouped by expert, and their gradients (device code).  Internal to the library.
#pragma once

#include <type_traits>

#include "uccl_row_elements.hpp"

namespace {

struct E4m3 { uint8_t bits; };

// Four e4m3 values are four bf16 values exactly.
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
__device__ __forceinline__ u32x2 widen_e4m3(uint32_t four) {
  return u32x2{__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(four, 1.0f, false)),
               __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(four, 1.0f, true))};
}

enum Product : uint32_t { kForward, kGradX, kGradW };
enum OutType : uint32_t { kOutF32 = 0, kOutBf16 = 1, kOutF16 = 2 };

// kForward: out[i, n] = sum_k a[index[i], k] b[g, n, k]        a = x, b = w (e4m3: times their rows' scales)
// kGradX:   out[i, k] = sum_n a[i, n] b[g, n, k]               a = dy, b = w
// kGradW:   out[g, n, k] = sum_i a[i, n] b[index[i], k]        a = dy, b = x
// over the rows i of group g.  `wide`: rows of w a group, n; `cols`: k.
struct ProductArgs {
  Rows out, a, b;
  const int32_t* index;     // or nullptr: row i itself
  const int32_t* offsets;   // groups + 1
  uint32_t groups, rows, indexed_rows, wide, cols, out_type;
};

struct Group {
  uint32_t index, begin, end;   // rows begin .. end - 1
};

// Offsets are taken as they can be used, whatever they hold: each is at least the one before it, at least 0 and at most
// `rows`.  Groups never overlap then and no row outside the matrix is touched.
// Finds the group of the `tile`th tile of `height` rows (every group's rows are cut into tiles of its own); false: there are fewer tiles.
// All lanes of a wavefront call it; 64 groups a turn.
__device__ __forceinline__ bool find_tile(const ProductArgs& a, uint32_t height, uint32_t tile, Group& g, uint32_t& first_row) {
  const uint32_t lane = threadIdx.x & 63u;
  int32_t before = 0;       // the greatest offset so far
  uint32_t passed = 0;      // tiles of earlier groups
  for (uint32_t at = 0; at < a.groups; at += 64u) {
    const uint32_t mine = at + lane;
    int32_t begin = mine <= a.groups ? a.offsets[mine] : 0, end = mine < a.groups ? a.offsets[mine + 1u] : 0;
    int32_t most = end;
    if (lane == 0u) most = max(max(most, begin), before);
#pragma unroll
    for (uint32_t d = 1; d < 64u; d <<= 1) {
      const int32_t other = __shfl_up(most, d);
      if (lane >= d) most = max(most, other);
    }
    const int32_t limit = static_cast<int32_t>(a.rows);
    const int32_t previous = __shfl_up(most, 1);
    const uint32_t b = static_cast<uint32_t>(min(max(lane == 0u ? max(begin, before) : previous, 0), limit));
    const uint32_t e = static_cast<uint32_t>(min(max(most, 0), limit));
    const uint32_t tiles = mine < a.groups ? (e - b + height - 1u) / height : 0u;
    uint32_t sum = tiles;
#pragma unroll
    for (uint32_t d = 1; d < 64u; d <<= 1) {
      const uint32_t other = __shfl_up(sum, d);
      if (lane >= d) sum += other;
    }
    const uint64_t holds = __ballot(passed + sum > tile);
    if (holds != 0u) {
      const int l = __ffsll(static_cast<unsigned long long>(holds)) - 1;
      g.index = at + static_cast<uint32_t>(l);
      g.begin = __builtin_amdgcn_readlane(b, l);
      g.end = __builtin_amdgcn_readlane(e, l);
      first_row = g.begin + (tile - passed - (__builtin_amdgcn_readlane(sum, l) - __builtin_amdgcn_readlane(tiles, l))) * height;
      return true;
    }
    passed += __builtin_amdgcn_readlane(sum, 63);
    before = __builtin_amdgcn_readlane(most, 63);
  }
  return false;
}

// The rows of group g, by the same rule.
__device__ __forceinline__ Group group_rows(const ProductArgs& a, uint32_t g) {
  const uint32_t lane = threadIdx.x & 63u;
  int32_t most = 0, next = 0;
  for (uint32_t at = lane; at <= g; at += 64u) most = max(most, a.offsets[at]);
#pragma unroll
  for (int d = 32; d > 0; d >>= 1) most = max(most, __shfl_xor(most, d));
  next = max(most, a.offsets[g + 1u]);
  const int32_t limit = static_cast<int32_t>(a.rows);
  return Group{g, static_cast<uint32_t>(__builtin_amdgcn_readfirstlane(min(most, limit))), static_cast<uint32_t>(__builtin_amdgcn_readfirstlane(min(next, limit)))};
}

__device__ __forceinline__ void store_out(const ProductArgs& a, uint64_t row, uint32_t col, float v) {
  char* at = a.out.data + row * a.out.stride;
  if (a.out_type == kOutF32) reinterpret_cast<float*>(at)[col] = v;
  else if (a.out_type == kOutBf16) reinterpret_cast<__bf16*>(at)[col] = static_cast<__bf16>(v);
  else reinterpret_cast<_Float16*>(at)[col] = static_cast<_Float16>(v);
}

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));

// The plainest form: tiles of 64 x 64, 32 deep, both operands through the LDS element by element.  8-bit operands are
// widened to bf16 and multiplied exactly: the matrix instructions for 8 bits drop what is below about 2^-13 of the largest
// of the products that they add at a time.
template <class T, Product P>
__global__ __launch_bounds__(256) void product_plain_kernel(ProductArgs a) {
  using M = std::conditional_t<sizeof(T) == 1, __bf16, T>;
  constexpr uint32_t DEEP = 32, PITCH = DEEP + 8;
  __shared__ __align__(16) M ta[64][PITCH], tb[64][PITCH];
  const uint32_t out_cols = P == kForward ? a.wide : a.cols, across = (out_cols + 63u) / 64u;
  const uint32_t c0 = blockIdx.x % across * 64u;
  Group g;
  uint32_t r0;
  if constexpr (P == kGradW) {
    const uint32_t down = (a.wide + 63u) / 64u, t = blockIdx.x / across;
    g = group_rows(a, t / down);
    r0 = t % down * 64u;
  } else {
    if (!find_tile(a, 64u, blockIdx.x / across, g, r0)) return;
  }
  const uint64_t w0 = static_cast<uint64_t>(g.index) * a.wide;
  const uint32_t depth = P == kForward ? a.cols : P == kGradX ? a.wide : g.end - g.begin;
  auto element = [&](const Rows& m, uint64_t row, uint32_t col) {
    const T v = reinterpret_cast<const T*>(m.data + row * m.stride)[col];
    if constexpr (sizeof(T) == 1) return __builtin_bit_cast(bf16x2, widen_e4m3(v.bits).x).x;
    else return v;
  };
  auto source = [&](uint32_t i, uint32_t& row) {   // the row that row i reads
    row = a.index == nullptr ? i : static_cast<uint32_t>(a.index[i]);
    return row < a.indexed_rows;
  };
  f32x4 acc[4] = {};
  for (uint32_t d0 = 0; d0 < depth; d0 += DEEP) {
    __syncthreads();
    for (uint32_t i = threadIdx.x; i < 64u * DEEP; i += 256u) {
      const uint32_t r = P == kGradW ? i % 64u : i / DEEP, d = P == kGradW ? i / 64u : i % DEEP;
      const uint32_t rb = P == kForward ? i / DEEP : i % 64u, db = P == kForward ? i % DEEP : i / 64u;
      M va{}, vb{};
      uint32_t from;
      if constexpr (P == kForward) {
        if (r0 + r < g.end && d0 + d < depth && source(r0 + r, from)) va = element(a.a, from, d0 + d);
        if (c0 + rb < a.wide && d0 + db < depth) vb = element(a.b, w0 + c0 + rb, d0 + db);
      } else if constexpr (P == kGradX) {
        if (r0 + r < g.end && d0 + d < depth) va = element(a.a, r0 + r, d0 + d);
        if (c0 + rb < a.cols && d0 + db < depth) vb = element(a.b, w0 + d0 + db, c0 + rb);
      } else {
        if (r0 + r < a.wide && d0 + d < depth) va = element(a.a, g.begin + d0 + d, r0 + r);
        if (c0 + rb < a.cols && d0 + db < depth && source(g.begin + d0 + db, from)) vb = element(a.b, from, c0 + rb);
      }
      ta[r][d] = va;
      tb[rb][db] = vb;
    }
    __syncthreads();
    const uint32_t lane = threadIdx.x & 63u, wave = threadIdx.x / 64u;
    const M* pa = &ta[wave * 16u + lane % 16u][lane / 16u * 8u];
#pragma unroll
    for (uint32_t n = 0; n < 4; ++n) {
      const M* pb = &tb[n * 16u + lane % 16u][lane / 16u * 8u];
      if constexpr (__is_same(M, __bf16)) acc[n] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(*reinterpret_cast<const bf16x8*>(pa), *reinterpret_cast<const bf16x8*>(pb), acc[n], 0, 0, 0);
      else acc[n] = __builtin_amdgcn_mfma_f32_16x16x32_f16(*reinterpret_cast<const f16x8*>(pa), *reinterpret_cast<const f16x8*>(pb), acc[n], 0, 0, 0);
    }
  }
  const uint32_t lane = threadIdx.x & 63u, wave = threadIdx.x / 64u;
#pragma unroll
  for (uint32_t n = 0; n < 4; ++n)
#pragma unroll
    for (uint32_t i = 0; i < 4; ++i) {
      const uint32_t r = r0 + wave * 16u + lane / 16u * 4u + i, c = c0 + n * 16u + lane % 16u;
      if (r >= (P == kGradW ? a.wide : g.end) || c >= out_cols) continue;
      float v = acc[n][i];
      if constexpr (sizeof(T) == 1) {
        uint32_t from;
        const float sx = source(r, from) ? *reinterpret_cast<const float*>(a.a.scales + from * a.a.scale_stride) : 0.0f;
        v = v * sx * *reinterpret_cast<const float*>(a.b.scales + (w0 + c) * a.b.scale_stride);
      }
      store_out(a, P == kGradW ? w0 + r : r, c, v);
    }
}

}  // namespace
