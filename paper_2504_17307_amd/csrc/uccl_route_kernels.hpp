// A router's choice of experts, its gradient, the balance loss, and the order of rows that the choice makes (device code).  Internal to the library.
#pragma once

#include "uccl_row_elements.hpp"

namespace {

// ---- a token's experts ------------------------------------------------------------------------------
//
// LANES neighbouring lanes have a token, and a lane K pieces of 16 bytes of its scores, LANES pieces apart: element i of piece k is expert
// (k LANES + lane) N + i.  As many lanes as there are pieces, if they are at most 64: the choice is a chain of operations, whose length goes by what a lane has.

template <uint32_t BY>
__device__ __forceinline__ uint32_t turned(uint32_t v) { return static_cast<uint32_t>(__builtin_amdgcn_mov_dpp(static_cast<int>(v), 0x120 + BY, 0xF, 0xF, true)); }   // within 16 lanes

// What a wavefront's lanes have left in the LDS is there for its other lanes: its accesses are in order, so that only the compiler has to keep them so.
__device__ __forceinline__ void left_for_other_lanes() {
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
}

// Reduce over a token's lanes; every lane has the result.
template <uint32_t LANES, class F>
__device__ __forceinline__ uint32_t over_lanes(uint32_t v, F f) {
  static_assert(LANES == 16u || LANES == 32u || LANES == 64u);
  v = f(v, turned<8>(v));
  v = f(v, turned<4>(v));
  v = f(v, turned<2>(v));
  v = f(v, turned<1>(v));
  if constexpr (LANES >= 32u) {   // the neighbouring 16 lanes'
    const u32x2 w = __builtin_bit_cast(u32x2, __builtin_amdgcn_permlane16_swap(v, v, false, false));
    v = f(w[0], w[1]);
  }
  if constexpr (LANES == 64u) {
    const u32x2 w = __builtin_bit_cast(u32x2, __builtin_amdgcn_permlane32_swap(v, v, false, false));
    v = f(w[0], w[1]);
  }
  return v;
}
__device__ __forceinline__ uint32_t bits_of(float v) { return __builtin_bit_cast(uint32_t, v); }
__device__ __forceinline__ float float_of(uint32_t v) { return __builtin_bit_cast(float, v); }
template <uint32_t LANES>
__device__ __forceinline__ float lanes_sum(float v) {
  return float_of(over_lanes<LANES>(bits_of(v), [](uint32_t a, uint32_t b) { return bits_of(float_of(a) + float_of(b)); }));
}
template <uint32_t LANES>
__device__ __forceinline__ float lanes_max(float v) {
  return float_of(over_lanes<LANES>(bits_of(v), [](uint32_t a, uint32_t b) { return bits_of(fmaxf(float_of(a), float_of(b))); }));
}

// Keys as numbers in their order: 0 for what is never chosen (-infinity, NaN), the same for both zeros.
__device__ __forceinline__ uint32_t ordered(float key) {
  const uint32_t b = bits_of(key + 0.0f);
  return key > -INFINITY ? b ^ (static_cast<uint32_t>(static_cast<int32_t>(b) >> 31) | 0x80000000u) : 0u;
}
// A key and its expert as one binary64, 2^52 and 42 bits: of equal keys the lower expert's is the greater, and the greatest of two is one instruction.
__device__ __forceinline__ u32x2 ranked(uint32_t key, uint32_t expert) { return u32x2{key << 10 | (1023u - expert), 0x43300000u | key >> 22}; }
// (fmax would quiet NaNs first, which are none here.)
__device__ __forceinline__ double greater(double a, double b) {
  double r;
  asm("v_max_f64 %0, %1, %2" : "=v"(r) : "v"(a), "v"(b));
  return r;
}
template <uint32_t BY>
__device__ __forceinline__ double greater_turned(double v) {
  const u32x2 w = __builtin_bit_cast(u32x2, v);
  return greater(v, __builtin_bit_cast(double, u32x2{turned<BY>(w[0]), turned<BY>(w[1])}));
}
template <uint32_t LANES>
__device__ __forceinline__ double greatest_of_lanes(double v) {
  v = greater_turned<8>(v);
  v = greater_turned<4>(v);
  v = greater_turned<2>(v);
  v = greater_turned<1>(v);
  if constexpr (LANES >= 32u) {
    const u32x2 w = __builtin_bit_cast(u32x2, v), x = __builtin_bit_cast(u32x2, __builtin_amdgcn_permlane16_swap(w[0], w[0], false, false)),
                y = __builtin_bit_cast(u32x2, __builtin_amdgcn_permlane16_swap(w[1], w[1], false, false));
    v = greater(__builtin_bit_cast(double, u32x2{x[0], y[0]}), __builtin_bit_cast(double, u32x2{x[1], y[1]}));
  }
  if constexpr (LANES == 64u) {
    const u32x2 w = __builtin_bit_cast(u32x2, v), x = __builtin_bit_cast(u32x2, __builtin_amdgcn_permlane32_swap(w[0], w[0], false, false)),
                y = __builtin_bit_cast(u32x2, __builtin_amdgcn_permlane32_swap(w[1], w[1], false, false));
    v = greater(__builtin_bit_cast(double, u32x2{x[0], y[0]}), __builtin_bit_cast(double, u32x2{x[1], y[1]}));
  }
  return v;
}
// The greatest of N, two by two.
template <uint32_t N>
__device__ __forceinline__ double greatest_of(const u32x2 (&v)[N]) {
  double w[N];
#pragma unroll
  for (uint32_t i = 0; i < N; ++i) w[i] = __builtin_bit_cast(double, v[i]);
#pragma unroll
  for (uint32_t n = N / 2u; n != 0u; n /= 2u)
#pragma unroll
    for (uint32_t i = 0; i < n; ++i) w[i] = greater(w[i], w[i + n]);
  return w[0];
}

struct RouteArgs {
  int32_t* experts;
  float* weights;
  int32_t* counts;      // or nullptr
  float* sums;          // or nullptr
  uint32_t* parts;      // [gridDim.x][2][cols]: a workgroup's counts and sums; nullptr: there is one workgroup, and what it has is the result
  Rows scores;
  const float* bias;    // or nullptr
  uint32_t tokens, cols, slots, normalise;
  float scale;
};

// What a token's lanes have of its scores: z, -infinity past the row's end, and the greatest of all (0 if that is -infinity: exp(z - most) is 0 then).
template <class T, uint32_t LANES, uint32_t K>
struct Scores {
  static constexpr uint32_t N = Piece<T>::N, V = K * N;
  float z[V], most;
  struct Loaded {
    Piece<T> p[K];
  };
  static __device__ __forceinline__ Loaded load(const Rows& rows, uint64_t row, uint32_t cols) {
    const uint32_t lane = threadIdx.x % LANES, pieces = (cols + N - 1u) / N;
    Loaded l;
#pragma unroll
    for (uint32_t k = 0; k < K; ++k) l.p[k] = load_piece<T>(rows.data + row * rows.stride, min(k * LANES + lane, pieces - 1u));
    return l;
  }
  __device__ __forceinline__ Scores(const Loaded& l, uint32_t cols) {
    const uint32_t lane = threadIdx.x % LANES;
    most = -INFINITY;
#pragma unroll
    for (uint32_t k = 0; k < K; ++k)
#pragma unroll
      for (uint32_t i = 0; i < N; ++i) {
        const float v = (k * LANES + lane) * N + i < cols ? widen(l.p[k].v[i]) : -INFINITY;
        z[k * N + i] = v;
        most = fmaxf(most, v);
      }
    most = lanes_max<LANES>(most);
    if (most == -INFINITY) most = 0.0f;
  }
};

// 1 / (sum of exp(z - most)); 0 for a token whose scores are all -infinity.
__device__ __forceinline__ float per_sum(float sum) { return sum == 0.0f ? 0.0f : 1.0f / sum; }

// p = softmax(z), the `slots` experts of greatest z + bias, and of those p or the softmax over themselves, times scale.  The greatest keys come one after the other: the
// greatest of the lane's own, then of the token's lanes'.  Few tokens are bound by that chain, many by the instructions (for f32, 256 experts and 8 slots with the sums about
// 1200 a wavefront's four tokens, half of them in the choice), in neither case by memory.  Measured without sums, 8 slots, bf16, us: one token of 256 experts 3.6, 4096 of 256 5.3.
// The biases lie in the LDS: in registers they took a wavefront's place, and each its own look at whether there are any (32768 tokens of 256 in bf16 19.2 us, 13.8 now).
// SUMS: workgroups take tokens in turn, and add up counts and probabilities in their order; no atomics between workgroups, so that the sums are the same from call to
// call.  The registers of four wavefronts' quarter, so that two workgroups are on a compute unit: 32768 x 256 f32 21.6 us,
// and 3.8 for the workgroups' sums, of which reading takes 6.5; one workgroup on each 24 and 4.5.
constexpr uint32_t kRouteSumThreads = 512;

template <class T, uint32_t LANES, uint32_t K, bool SUMS>
__global__ __launch_bounds__(SUMS ? kRouteSumThreads : 256, SUMS ? 4 : 1) void route_kernel(RouteArgs a) {
  using S = Scores<T, LANES, K>;
  constexpr uint32_t N = S::N, V = S::V, KEEP = 32u / LANES == 0u ? 1u : 32u / LANES, THREADS = SUMS ? kRouteSumThreads : 256u, EACH = THREADS / LANES;
  constexpr uint32_t WAVES = THREADS / 64u, MOST = LANES * V;
  __shared__ uint32_t counted[SUMS ? MOST : 1u];
  __shared__ float added[SUMS ? WAVES : 1u][SUMS ? MOST : 1u];
  __shared__ float scores[EACH][MOST];
  __shared__ float biases[MOST];
  const uint32_t lane = threadIdx.x % LANES;
  for (uint32_t e = threadIdx.x; e < MOST; e += THREADS) {
    biases[e] = a.bias != nullptr ? a.bias[min(e, a.cols - 1u)] : 0.0f;
    if constexpr (SUMS) counted[e] = 0u;
  }
  __syncthreads();
  float total[V];
#pragma unroll
  for (uint32_t v = 0; v < V; ++v) total[v] = 0.0f;
  for (uint32_t first = blockIdx.x * EACH; first < a.tokens; first += gridDim.x * EACH) {
    const uint32_t at = first + threadIdx.x / LANES;
    const bool here = at < a.tokens;
    const uint64_t token = min(at, a.tokens - 1u);
    const S s(S::load(a.scores, token, a.cols), a.cols);
    u32x2 key[V];
    float sum = 0.0f, p[V];
#pragma unroll
    for (uint32_t v = 0; v < V; ++v) {
      const uint32_t e = (v / N * LANES + lane) * N + v % N;
      scores[threadIdx.x / LANES][e] = s.z[v];
      key[v] = ranked(ordered(s.z[v] + biases[e]), e);
    }
    if (SUMS || a.normalise == 0u) {
#pragma unroll
      for (uint32_t v = 0; v < V; ++v) {
        p[v] = expf(s.z[v] - s.most);
        sum += p[v];
      }
    } else {   // only whether it is a number
      bool number = true;
#pragma unroll
      for (uint32_t v = 0; v < V; ++v) number = number && s.z[v] < INFINITY;
      sum = number ? 1.0f : __builtin_nanf("");
    }
    left_for_other_lanes();
    sum = lanes_sum<LANES>(sum);
    const float per = per_sum(sum);
    if constexpr (SUMS) {
#pragma unroll
      for (uint32_t v = 0; v < V; ++v) total[v] += here ? p[v] * per : 0.0f;
    }
    int32_t mine[KEEP];
#pragma unroll
    for (uint32_t k = 0; k < KEEP; ++k) mine[k] = -1;
    for (uint32_t j = 0; j < a.slots; ++j) {
      const uint64_t found = __builtin_bit_cast(uint64_t, greatest_of_lanes<LANES>(greatest_of(key)));
      const uint32_t low = static_cast<uint32_t>(found);   // the expert's number is in it, so no other key has it
#pragma unroll
      for (uint32_t v = 0; v < V; ++v) key[v][1] = key[v][0] == low ? 0u : key[v][1];   // below all others then
#pragma unroll
      for (uint32_t k = 0; k < KEEP; ++k)
        if (j == k * LANES + lane && found >= 0x4330000000000400ull) mine[k] = static_cast<int32_t>(1023u - (low & 1023u));
    }
    // a lane has the token's slots lane, lane + LANES
    float z[KEEP], most = -INFINITY, some = 0.0f;
#pragma unroll
    for (uint32_t k = 0; k < KEEP; ++k) {
      z[k] = mine[k] < 0 ? -INFINITY : scores[threadIdx.x / LANES][mine[k]];   // its own wavefront's
      most = fmaxf(most, z[k]);
    }
    // normalised, relative to the greatest of the chosen: a bias may choose experts all of whose p are 0 in binary32
    most = a.normalise != 0u ? lanes_max<LANES>(most) : s.most;
#pragma unroll
    for (uint32_t k = 0; k < KEEP; ++k) {
      z[k] = mine[k] < 0 ? 0.0f : expf(z[k] - most);
      some += z[k];
    }
    some = a.normalise != 0u ? per_sum(lanes_sum<LANES>(some)) : per;
    if (sum != sum) some = sum;   // of a NaN that was not chosen
#pragma unroll
    for (uint32_t k = 0; k < KEEP; ++k) {
      const uint32_t j = k * LANES + lane;
      if (here && j < a.slots) {
        a.experts[token * a.slots + j] = mine[k];
        a.weights[token * a.slots + j] = mine[k] < 0 ? 0.0f : a.scale * (z[k] * some);
        if constexpr (SUMS)
          if (mine[k] >= 0) atomicAdd(&counted[mine[k]], 1u);
      }
    }
    left_for_other_lanes();   // and read, before the next token's
  }
  if constexpr (SUMS) {
    const uint32_t wave = threadIdx.x / 64u;
#pragma unroll
    for (uint32_t v = 0; v < V; ++v) {
      // the wavefront's four tokens, or two
      if constexpr (LANES == 16u) total[v] += __shfl_xor(total[v], 16);
      if constexpr (LANES <= 32u) total[v] += __shfl_xor(total[v], 32);
      if (threadIdx.x % 64u < LANES) added[wave][(v / N * LANES + lane) * N + v % N] = total[v];
    }
    __syncthreads();
    for (uint32_t e = threadIdx.x; e < a.cols; e += THREADS) {
      float sum = 0.0f;
#pragma unroll
      for (uint32_t w = 0; w < WAVES; ++w) sum += added[w][e];
      if (a.parts != nullptr) {
        uint32_t* part = a.parts + blockIdx.x * 2ull * a.cols + e;
        part[0] = counted[e];
        part[a.cols] = bits_of(sum);
      } else {
        if (a.counts != nullptr) a.counts[e] = static_cast<int32_t>(counted[e]);
        if (a.sums != nullptr) a.sums[e] = sum;
      }
    }
  }
}

// The workgroups' counts and sums, 64 of them at a time for 16 experts.
__global__ __launch_bounds__(1024) void route_sum_kernel(int32_t* counts, float* sums, const uint32_t* parts, uint32_t n, uint32_t cols) {
  __shared__ uint32_t counted[64][16];
  __shared__ float added[64][16];
  const uint32_t at = threadIdx.x % 16u, e = blockIdx.x * 16u + at, turn = threadIdx.x / 16u;
  uint32_t c = 0u;
  float s = 0.0f;
  if (e < cols)
#pragma unroll 4
    for (uint32_t i = turn; i < n; i += 64u) {
      c += parts[(i * 2ull) * cols + e];
      s += float_of(parts[(i * 2ull + 1u) * cols + e]);
    }
  counted[turn][at] = c;
  added[turn][at] = s;
  __syncthreads();
  if (turn < 8u) {
#pragma unroll
    for (uint32_t i = 8; i < 64u; i += 8u) {
      c += counted[turn + i][at];
      s += added[turn + i][at];
    }
    counted[turn][at] = c;
    added[turn][at] = s;
  }
  __syncthreads();
  if (turn != 0u || e >= cols) return;
#pragma unroll
  for (uint32_t i = 1; i < 8u; ++i) {
    c += counted[i][at];
    s += added[i][at];
  }
  if (counts != nullptr) counts[e] = static_cast<int32_t>(c);
  if (sums != nullptr) sums[e] = s;
}

struct RouteGradArgs {
  Rows dscores, scores;
  const int32_t* experts;   // or nullptr
  const float* dweights;
  const float* dsums;       // or nullptr
  uint32_t tokens, cols, slots, normalise;
  float scale;
};

// With g_j = scale dw_j: weights that are p themselves make dz_e = p_e (g_e - sum of g p), normalised ones dz_e = q_e (g_e - sum of g q), where q is the
// softmax over the chosen; and the sums of probabilities add p_e (d_e - sum of d p).  p is made again from the scores, which are less to read than p kept in binary32 would be.
// Measured: 32768 x 256 f32, 8 slots, 13.8 us, 5.1 TB/s, in bf16 12.0; with the sums' gradient read by each lane, and not from the LDS, 16.4 and 21.4.  1777 x 61 f16 4.5, which is the chain of sums over lanes.
template <class T, uint32_t LANES, uint32_t K>
__global__ __launch_bounds__(256) void route_grad_kernel(RouteGradArgs a) {
  using S = Scores<T, LANES, K>;
  constexpr uint32_t N = S::N, V = S::V, KEEP = 32u / LANES == 0u ? 1u : 32u / LANES, EACH = 256u / LANES;
  __shared__ float part[EACH][LANES * V], of_sums[LANES * V];
  for (uint32_t e = threadIdx.x; e < LANES * V; e += 256u) of_sums[e] = a.dsums != nullptr && e < a.cols ? a.dsums[e] : 0.0f;   // (behind the last expert p is 0, which an infinity would make NaN)
  __syncthreads();
  const uint32_t lane = threadIdx.x % LANES, at = blockIdx.x * EACH + threadIdx.x / LANES;
  const bool here = at < a.tokens;
  const uint64_t token = min(at, a.tokens - 1u);
  int32_t mine[KEEP];
  float g[KEEP], q[KEEP];
#pragma unroll
  for (uint32_t k = 0; k < KEEP; ++k) {
    const uint32_t j = k * LANES + lane;
    mine[k] = -1;
    g[k] = 0.0f;
    if (a.experts != nullptr && j < a.slots) {
      mine[k] = a.experts[token * a.slots + j];
      if (static_cast<uint32_t>(mine[k]) >= a.cols) mine[k] = -1;
      else g[k] = a.scale * a.dweights[token * a.slots + j];
    }
  }
  const S s(S::load(a.scores, token, a.cols), a.cols);
  float p[V], sum = 0.0f;
#pragma unroll
  for (uint32_t v = 0; v < V; ++v) {
    p[v] = expf(s.z[v] - s.most);
    sum += p[v];
  }
  sum = lanes_sum<LANES>(sum);
  const float per = per_sum(sum);
  float along = 0.0f, d[V];
#pragma unroll
  for (uint32_t v = 0; v < V; ++v) {
    d[v] = of_sums[(v / N * LANES + lane) * N + v % N];
    p[v] *= per;
    along = __builtin_fmaf(p[v], d[v], along);
  }
  float most = -INFINITY;
#pragma unroll
  for (uint32_t k = 0; k < KEEP; ++k) {
    q[k] = mine[k] < 0 ? -INFINITY : widen(reinterpret_cast<const T*>(a.scores.data + token * a.scores.stride)[mine[k]]);
    most = fmaxf(most, q[k]);
  }
  most = a.normalise != 0u ? lanes_max<LANES>(most) : s.most;
  float some = 0.0f, chosen = 0.0f;
#pragma unroll
  for (uint32_t k = 0; k < KEEP; ++k) {
    q[k] = mine[k] < 0 ? 0.0f : expf(q[k] - most);
    some += q[k];
  }
  some = a.normalise != 0u ? per_sum(lanes_sum<LANES>(some)) : per;
  if (sum != sum) some = sum;
#pragma unroll
  for (uint32_t k = 0; k < KEEP; ++k) {
    q[k] = mine[k] < 0 ? 0.0f : q[k] * some;
    chosen = __builtin_fmaf(q[k], g[k], chosen);
  }
  chosen = lanes_sum<LANES>(chosen);
  // what all experts have, then the chosen ones', slot by slot
  along = lanes_sum<LANES>(along) + (a.normalise != 0u ? 0.0f : chosen);
#pragma unroll
  for (uint32_t v = 0; v < V; ++v) p[v] *= d[v] - along;
#pragma unroll
  for (uint32_t k = 0; k < KEEP; ++k) q[k] *= a.normalise != 0u ? g[k] - chosen : g[k];
  // the chosen ones' part lies in the LDS by expert; slots follow each other, so one that names an expert again adds to it in a fixed order
  float* const chosen_part = part[threadIdx.x / LANES];
  if (a.experts != nullptr) {
#pragma unroll
    for (uint32_t v = 0; v < V; ++v) chosen_part[(v / N * LANES + lane) * N + v % N] = 0.0f;
#pragma unroll
    for (uint32_t k = 0; k < KEEP; ++k) {
      const uint32_t n = a.slots > k * LANES ? min(a.slots - k * LANES, LANES) : 0u;
      for (uint32_t j = 0; j < n; ++j) {
        left_for_other_lanes();
        if (lane == j && mine[k] >= 0) chosen_part[mine[k]] += q[k];
      }
    }
    left_for_other_lanes();
#pragma unroll
    for (uint32_t v = 0; v < V; ++v) p[v] += chosen_part[(v / N * LANES + lane) * N + v % N];
  }
  if (!here) return;
#pragma unroll
  for (uint32_t k = 0; k < K; ++k) {
    const uint32_t piece = k * LANES + lane, pieces = (a.cols + N - 1u) / N;
    Piece<T> out;
#pragma unroll
    for (uint32_t i = 0; i < N; ++i) out.v[i] = static_cast<T>(p[k * N + i]);
    store_piece<false>(a.dscores.data + token * a.dscores.stride, piece, out, valid_of<T>(piece, pieces, a.cols));
  }
}

// ---- balance loss -----------------------------------------------------------------------------------

__device__ __forceinline__ double wave_sum(double v) {
#pragma unroll
  for (int d = 32; d > 0; d >>= 1) v += __shfl_xor(v, d);
  return v;
}

// loss = coef n / (slots tokens^2) sum of counts_e sums_e, whose gradient along sums_e is what counts_e is multiplied by.  One workgroup and a fixed order: 1.8 us, a launch.
__global__ __launch_bounds__(256) void balance_kernel(float* loss, float* dsums, const int32_t* counts, const float* sums, uint32_t n, double factor) {
  __shared__ double parts[4];
  double v = 0.0;
  for (uint32_t e = threadIdx.x; e < n; e += 256u) {
    const double f = factor * counts[e];
    v += f * static_cast<double>(sums[e]);
    if (dsums != nullptr) dsums[e] = static_cast<float>(f);   // a thread reads an expert's sum before it writes there
  }
  v = wave_sum(v);
  if (threadIdx.x % 64u == 0u) parts[threadIdx.x / 64u] = v;
  __syncthreads();
  if (threadIdx.x == 0u && loss != nullptr) *loss = static_cast<float>(parts[0] + parts[1] + parts[2] + parts[3]);
}

// ---- the order of rows ------------------------------------------------------------------------------
//
// A stable counting sort.  A workgroup has a share of the choices and goes through it by tiles, a wavefront a run of a tile's choices: a choice's place among its
// expert's is the workgroup's first one, what earlier tiles, earlier wavefronts and earlier lanes of the same expert have.  Where there
// are several workgroups, each counts all choices, or each has counted its share before.  Lanes of the same expert are found bit by bit of its number, by a ballot each: a chain, and what bounds this
// (memory does not: 32768 choices are 0.4 MB).  Measured: 8 choices 3.1 us, 32768 of 256 experts 7.3.

constexpr uint32_t kPlanThreads = 512, kPlanWaves = kPlanThreads / 64u, kMostExperts = 1024, kPlanCounts = 2080 + 32;

struct PlanArgs {
  int32_t* index;
  int32_t* offsets;
  int32_t* pos;
  const int32_t* experts;
  const uint32_t* counts;   // [gridDim.x][n_experts], or nullptr: there is one workgroup, or each counts all choices
  uint32_t choices, slots, n_experts, share;   // share: of a workgroup, a multiple of a tile
};

__global__ __launch_bounds__(kPlanThreads) void plan_count_kernel(uint32_t* counts, const int32_t* experts, uint32_t choices, uint32_t n_experts, uint32_t share) {
  __shared__ uint32_t counted[kMostExperts];
  for (uint32_t e = threadIdx.x; e < n_experts; e += kPlanThreads) counted[e] = 0u;
  __syncthreads();
  const uint64_t begin = static_cast<uint64_t>(blockIdx.x) * share, end = min(begin + share, static_cast<uint64_t>(choices));
  for (uint64_t c = begin + threadIdx.x; c < end; c += kPlanThreads) {
    const uint32_t e = static_cast<uint32_t>(experts[c]);
    if (e < n_experts) atomicAdd(&counted[e], 1u);
  }
  __syncthreads();
  for (uint32_t e = threadIdx.x; e < n_experts; e += kPlanThreads) counts[static_cast<uint64_t>(blockIdx.x) * n_experts + e] = counted[e];
}

// ROUNDS: choices of a lane in a tile.
template <uint32_t ROUNDS>
__global__ __launch_bounds__(kPlanThreads) void plan_kernel(PlanArgs a) {
  constexpr uint32_t TILE = kPlanThreads * ROUNDS;
  __shared__ uint32_t seen[kPlanWaves][kMostExperts];   // of the tile, by wavefront; then the first place of each wavefront
  __shared__ uint32_t next[kPlanCounts];               // the place of the workgroup's next choice of an expert
  __shared__ uint32_t totals[kPlanCounts];
  __shared__ uint32_t sums[kPlanWaves];
  const uint32_t lane = threadIdx.x % 64u, wave = threadIdx.x / 64u;
  const uint64_t begin = static_cast<uint64_t>(blockIdx.x) * a.share, end = min(begin + a.share, static_cast<uint64_t>(a.choices));
  uint32_t bits = 0;
  while ((1u << bits) <= a.n_experts) ++bits;   // of the experts' numbers and of n_experts, which stands for none
  uint32_t expert[ROUNDS], rank[ROUNDS];
  auto read_tile = [&](uint64_t tile) {
#pragma unroll
    for (uint32_t r = 0; r < ROUNDS; ++r) {
      const uint64_t c = tile + (wave * ROUNDS + r) * 64u + lane;
      expert[r] = c < end ? min(static_cast<uint32_t>(a.experts[c]), a.n_experts) : a.n_experts;
    }
  };
  auto rank_tile = [&] {
    for (uint32_t e = lane; e < a.n_experts; e += 64u) seen[wave][e] = 0u;
#pragma unroll
    for (uint32_t r = 0; r < ROUNDS; ++r) {
      left_for_other_lanes();
      uint64_t same = ~0ull;
      for (uint32_t b = 0; b < bits; ++b) {
        const bool set = (expert[r] >> b & 1u) != 0u;
        const uint64_t with = __ballot(set);
        same &= set ? with : ~with;
      }
      const uint32_t before = __popcll(same & ((1ull << lane) - 1ull));
      rank[r] = before;
      if (expert[r] < a.n_experts) {
        rank[r] += seen[wave][expert[r]];
        left_for_other_lanes();
        if (before == 0u) seen[wave][expert[r]] = rank[r] + __popcll(same);   // one lane for each expert, when all have read
      }
    }
  };
  read_tile(begin);
  rank_tile();
  __syncthreads();
  // what the experts have in all, and in earlier workgroups
  uint32_t copies = 1u;
  const uint32_t stride = a.n_experts | 1u;   // of copies: a count of an expert and its copies are in different banks
  const bool counts_all = gridDim.x > 1u && a.counts == nullptr;
  if (counts_all)
    while (copies < 32u && copies * 2u * stride <= kPlanCounts - 32u) copies *= 2u;
  if (gridDim.x > 1u) {
    for (uint32_t i = threadIdx.x; i < copies * stride; i += kPlanThreads) totals[i] = next[i] = 0u;
    __syncthreads();
  }
  if (counts_all) {
    // Copies of the counts for neighbouring lanes, as many as there is room for: 65536 choices of one expert 59 us without, 11.6 with 8 of them.  What is no expert lies behind them.
    constexpr uint32_t AT_ONCE = 8, EACH = kPlanThreads * AT_ONCE;
    const uint32_t mine = lane % copies * stride, none = copies * stride + lane % 32u;
    auto count = [&](uint32_t first, bool whole) {
      uint32_t e[AT_ONCE];
#pragma unroll
      for (uint32_t r = 0; r < AT_ONCE; ++r) {
        const uint32_t c = first + r * kPlanThreads + threadIdx.x;
        e[r] = whole || c < a.choices ? static_cast<uint32_t>(a.experts[c]) : a.n_experts;
      }
#pragma unroll
      for (uint32_t r = 0; r < AT_ONCE; ++r) atomicAdd((first + r * kPlanThreads < begin ? next : totals) + (e[r] < a.n_experts ? mine + e[r] : none), 1u);
    };
    uint32_t first = 0;
    for (; first + EACH <= a.choices; first += EACH) count(first, true);
    if (first < a.choices) count(first, false);
    __syncthreads();
  } else if (a.counts != nullptr) {
    const uint32_t slices = a.n_experts < kPlanThreads ? kPlanThreads / a.n_experts : 1u;   // threads that share an expert's groups
    for (uint32_t i = threadIdx.x; i < a.n_experts * slices; i += kPlanThreads) {
      const uint32_t slice = i / a.n_experts, e = i - slice * a.n_experts;
      uint32_t all = 0u, earlier = 0u;
#pragma unroll 8
      for (uint32_t b = slice; b < gridDim.x; b += slices) {
        const uint32_t n = a.counts[b * a.n_experts + e];
        all += n;
        earlier += b < blockIdx.x ? n : 0u;
      }
      atomicAdd(&totals[e], all);
      atomicAdd(&next[e], earlier);
    }
    __syncthreads();
  }
  // the experts' first rows: two neighbouring experts a thread
  uint32_t total[2], before[2];
#pragma unroll
  for (uint32_t i = 0; i < 2u; ++i) {
    const uint32_t e = threadIdx.x * 2u + i;
    total[i] = before[i] = 0u;
    if (e < a.n_experts) {
      if (gridDim.x > 1u) {
        for (uint32_t k = 0; k < copies; ++k) {
          before[i] += next[k * stride + e];
          total[i] += totals[k * stride + e];
        }
        if (counts_all) total[i] += before[i];
      } else {
#pragma unroll
        for (uint32_t w = 0; w < kPlanWaves; ++w) total[i] += seen[w][e];
      }
    }
  }
  uint32_t to = total[0] + total[1];
#pragma unroll
  for (uint32_t d = 1; d < 64u; d <<= 1) {
    const uint32_t other = __shfl_up(to, d);
    if (lane >= d) to += other;
  }
  if (lane == 63u) sums[wave] = to;
  __syncthreads();
  uint32_t rows = 0;
#pragma unroll
  for (uint32_t w = 0; w < kPlanWaves; ++w) {
    if (w == wave) to += rows;
    rows += sums[w];
  }
#pragma unroll
  for (uint32_t i = 0; i < 2u; ++i) {
    const uint32_t e = threadIdx.x * 2u + i, first = to - total[1] - (i == 0u ? total[0] : 0u);
    if (e < a.n_experts) {
      next[e] = first + before[i];
      if (blockIdx.x == 0u) a.offsets[e] = static_cast<int32_t>(first);
    }
  }
  if (blockIdx.x == 0u && threadIdx.x == 0u) a.offsets[a.n_experts] = static_cast<int32_t>(rows);
  for (uint64_t tile = begin;; ) {
    __syncthreads();
    for (uint32_t e = threadIdx.x; e < a.n_experts; e += kPlanThreads) {
      uint32_t place = next[e];
#pragma unroll
      for (uint32_t w = 0; w < kPlanWaves; ++w) {
        const uint32_t n = seen[w][e];
        seen[w][e] = place;
        place += n;
      }
      next[e] = place;
    }
    __syncthreads();
#pragma unroll
    for (uint32_t r = 0; r < ROUNDS; ++r) {
      const uint64_t c = tile + (wave * ROUNDS + r) * 64u + lane;
      if (c >= end) continue;
      const bool there = expert[r] < a.n_experts;
      const uint32_t place = there ? seen[wave][expert[r]] + rank[r] : 0u;
      if (a.pos != nullptr) a.pos[c] = there ? static_cast<int32_t>(place) : -1;
      if (there && a.index != nullptr) a.index[place] = static_cast<int32_t>(static_cast<uint32_t>(c) / a.slots);
      if (c >= rows && a.index != nullptr) a.index[c] = -1;   // behind the last group
    }
    tile += TILE;
    if (tile >= end) break;
    read_tile(tile);
    __syncthreads();
    rank_tile();
  }
}

}  // namespace
