// Routing, the order of rows and clipping, gfx950 (MI355X).  Host side: argument checks, the choice of the kernel, entry points of uccl_experts.h.
#include <hip/hip_runtime.h>

#include <math.h>
#include <stdint.h>

#include "uccl_experts.h"

#include "uccl_gradient_kernels.hpp"
#include "uccl_route_kernels.hpp"
#include "uccl_row_checks.hpp"

static __device__ uint32_t loaded_with_this;   // what uccl_init() looks up

namespace {

// A call of several launches: the calling thread's start event is on the first of them and its stop event on the last (and on the first, so that one
// that HIP does not take is refused there).
class Launches {
 public:
  template <class K, class... A>
  int operator()(bool last, K kernel, uint64_t groups, uint32_t threads, hipStream_t s, A... a) {
    if (first_) {
      if (!last) stop_ = uccl_internal_stop_event();
      first_ = false;
    } else if (last && stop_ != nullptr) {
      (void)uccl_time_next_launch(nullptr, stop_);
    }
    return launch(kernel, groups, threads, s, a...);
  }

 private:
  bool first_ = true;
  void* stop_ = nullptr;
};

// ---- routing ----------------------------------------------------------------------------------------

constexpr uint32_t kRouteGroups = 512;   // that add up counts and probabilities, at most: two a compute unit

// Few tokens: as many lanes for each as it has pieces, up to 64; many, which fill the machine: 16, where what goes over the lanes is done for four tokens at once.  Measured, 16 / as many,
// 256 experts, with 8 slots, us: f32, 1 / 600 / 4096 / 32768 tokens, 4.3 / 5.2 / 4.9 / 14.7 against 3.3 / 3.7 / 5.6 / 25.7; the gradient 4.5 / 4.9 / 5.4 / 16.1 against 3.1 / 3.6 / 5.4 / 19.7; bf16, 4.4 / 4.5 /
// 4.6 / 14.2 against 3.6 / 4.1 / 4.6 / 16.5.
bool takes_16_lanes(uint32_t tokens, uint32_t cols) { return cols <= 256u && tokens > 2048u; }

// Calls f with the lanes of a token and the pieces of a lane, for rows of `cols` elements of T.
template <class T, class F>
auto with_lanes(uint32_t tokens, uint32_t cols, F f) {
  constexpr uint32_t N = Piece<T>::N;
  using std::integral_constant;
  using One = integral_constant<uint32_t, 1>;
  using Two = integral_constant<uint32_t, 2>;
  using L16 = integral_constant<uint32_t, 16>;
  using L64 = integral_constant<uint32_t, 64>;
  if (cols <= 16u * N) return f(L16{}, One{});
  if (takes_16_lanes(tokens, cols)) {
    if (cols <= 32u * N) return f(L16{}, Two{});
    if constexpr (N == 4u) return f(L16{}, integral_constant<uint32_t, 4>{});
  }
  if (cols <= 32u * N) return f(integral_constant<uint32_t, 32>{}, One{});
  if (cols <= 64u * N) return f(L64{}, One{});
  if constexpr (N == 4u)
    if (cols <= 512u) return f(L64{}, Two{});
  return f(L64{}, integral_constant<uint32_t, 16u / N>{});
}

// Workgroups of kernels that add up counts and probabilities.  (As many as any type needs: a call's scratch memory does not go by the type.)
uint32_t route_groups(uint32_t tokens, uint32_t cols) {
  const uint32_t lanes = cols <= 64u || takes_16_lanes(tokens, cols) ? 16u : cols <= 128u ? 32u : 64u, n = blocks_for(tokens, kRouteSumThreads / lanes);
  return n < kRouteGroups ? n : kRouteGroups;
}

int check_route(const uccl_rows* scores, const uccl_route_opts* o) {
  const int e = check(scores);
  if (e != UCCL_OK) return e;
  if (!is_float(scores->dtype) || scores->cols > UCCL_MOST_EXPERTS || o == nullptr || o->reserved != 0u || o->normalise > 1u || !isfinite(o->scale)) return UCCL_EINVAL;
  return o->slots == 0u || o->slots > scores->cols || o->slots > UCCL_MOST_SLOTS ? UCCL_EINVAL : UCCL_OK;
}

// ---- the order of rows ------------------------------------------------------------------------------

// Several workgroups, which have to know what the others' choices are: up to this many, each counts them all, beyond, or where the choices are written over, a launch before
// has counted every workgroup's.  Measured, 256 experts, all counted by each / a launch before, us: 1280 choices 4.7 / 5.4, 8192 5.2 / 8.3, 32768 7.3 / 10.9,
// 65536 10.5 / 13.1, of one expert all 11.6 / 13.6, 131072 17.5 / 17.5.
constexpr uint64_t kPlanCountsAll = 1ull << 16;
constexpr uint32_t kPlanGroups = 128;   // workgroups with a launch before, at most

// How the choices are shared out.  Where each workgroup counts them all, it has 512 at a time, one of a lane; with a launch before 1024 or 2048: more at a time are fewer workgroups, each of
// which reads the others' counts.  Measured, 1024 / 2048 at a time, 256 experts, us: 4096 choices 7.6 / 8.7, 32768 11.6 / 11.2, 131072 26.5 / 18.6.
struct PlanShape {
  uint32_t rounds, groups, share;
};
PlanShape plan_shape(uint64_t choices, uint32_t n_experts, bool counts_all) {
  const uint32_t rounds = counts_all ? 1u : (choices + 1023u) / 1024u * n_experts <= 4096u ? 2u : 4u, tile = rounds * kPlanThreads;
  const uint64_t tiles = (choices + tile - 1u) / tile, each = counts_all ? 1u : (tiles + kPlanGroups - 1u) / kPlanGroups;
  if (tiles == 0u) return PlanShape{rounds, 1u, tile};
  return PlanShape{rounds, static_cast<uint32_t>((tiles + each - 1u) / each), static_cast<uint32_t>(each * tile)};
}

// ---- gradients --------------------------------------------------------------------------------------

constexpr uint32_t kGradientGroups = 4096, kLeastShare = 1024;   // workgroups of a call, about, and pieces of a workgroup at least
constexpr uint64_t kStayInCaches = 32ull << 20;                  // outputs of more than this are stored past them

uint32_t pieces_of(const uccl_rows* m) { return blocks_for(row_bytes(m), 16u); }

// How a call's matrices are shared out: pieces of a workgroup, and how many matrices that have elements are one row, and are not.
struct Shares {
  uint32_t share, flat, strided;
  uint64_t bytes;
};
// Rows that follow each other without a gap are one (whose elements have to be counted in 32 bits).
bool is_flat(const uccl_rows* in, const uccl_rows* out) {
  if (in->rows == 1u) return true;
  return in->stride == row_bytes(in) && (out == nullptr || out->stride == in->stride) && static_cast<uint64_t>(in->rows) * in->cols <= 0xFFFFFFFFull;
}
Shares shares_of(const uccl_rows* in, const uccl_rows* out, uint32_t n) {
  uint64_t pieces = 0;
  Shares s{};
  for (uint32_t i = 0; i < n; ++i) {
    const uint64_t mine = static_cast<uint64_t>(in[i].rows) * pieces_of(in + i);
    pieces += mine;
    if (mine != 0u) ++(is_flat(in + i, out == nullptr ? nullptr : out + i) ? s.flat : s.strided);
  }
  const uint64_t share = (pieces / kGradientGroups + kLeastShare) / kLeastShare * kLeastShare;
  s.share = static_cast<uint32_t>(share < 1u << 30 ? share : 1u << 30);
  s.bytes = pieces * 16u;
  return s;
}

// Goes through those of one kind, as many at a time as a launch takes: f(args, workgroups, whether they are the last of `left`).
template <bool FLAT, class F>
int over_matrices(const uccl_rows* in, const uccl_rows* out, uint32_t n, uint32_t share, uint32_t left, F f) {
  GradientArgs<FLAT> a{};
  a.share = share;
  uint64_t groups = 0;
  for (uint32_t i = 0; i < n && left != 0u; ++i) {
    const uint64_t mine = static_cast<uint64_t>(in[i].rows) * pieces_of(in + i);
    if (mine == 0u || is_flat(in + i, out == nullptr ? nullptr : out + i) != FLAT) continue;
    a.in[a.n] = static_cast<const char*>(in[i].data);
    a.out[a.n] = out == nullptr ? nullptr : static_cast<char*>(out[i].data);
    a.dtype[a.n] = static_cast<uint8_t>(in[i].dtype == UCCL_F32 ? 0u : in[i].dtype == UCCL_BF16 ? 1u : 2u);
    a.cols[a.n] = FLAT ? static_cast<uint32_t>(static_cast<uint64_t>(in[i].rows) * in[i].cols) : in[i].cols;
    if constexpr (!FLAT) {
      a.in_stride[a.n] = in[i].stride;
      a.out_stride[a.n] = out == nullptr ? 0u : out[i].stride;
      a.rows[a.n] = in[i].rows;
    }
    a.first[a.n++] = static_cast<uint32_t>(groups);
    groups += (mine + share - 1u) / share;
    const bool last = --left == 0u;
    if (a.n == GradientArgs<FLAT>::MOST || last) {
      const int e = f(a, groups, last);
      if (e != UCCL_OK) return e;
      a.n = 0u;
      groups = 0u;
    }
  }
  return UCCL_OK;
}

int check_gradients(const uccl_rows* m, uint32_t n) {
  if ((m == nullptr && n != 0u) || n > kMost) return UCCL_EINVAL;
  for (uint32_t i = 0; i < n; ++i) {
    const int e = check(m + i);
    if (e != UCCL_OK) return e;
    if (!is_float(m[i].dtype)) return UCCL_EINVAL;
  }
  return UCCL_OK;
}

}  // namespace

int uccl_internal_load_experts() {
  hipStreamCaptureMode mode = hipStreamCaptureModeRelaxed;   // another stream of the program may be under capture
  const bool relaxed = hipThreadExchangeStreamCaptureMode(&mode) == hipSuccess;
  void* at = nullptr;
  const hipError_t e = hipGetSymbolAddress(&at, HIP_SYMBOL(loaded_with_this));
  if (relaxed) (void)hipThreadExchangeStreamCaptureMode(&mode);
  return e == hipSuccess ? UCCL_OK : uccl_internal_failed(e);
}

extern "C" {

uint64_t uccl_route_rows_scratch(uint32_t tokens, uint32_t n_experts) {
  const uint32_t groups = route_groups(tokens, n_experts);
  return groups <= 1u ? 0u : (groups * 8ull * n_experts + 15u) / 16u * 16u;
}

int uccl_route_rows(int32_t* experts, float* weights, int32_t* counts, float* sums, const uccl_rows* scores, const float* bias,
                    const uccl_route_opts* opts, void* scratch, uint64_t scratch_bytes, void* stream) {
  const int e = check_route(scores, opts);
  if (e != UCCL_OK) return e;
  if (scores->rows != 0u && (experts == nullptr || weights == nullptr)) return UCCL_EINVAL;
  if (misaligned(experts, 4) || misaligned(weights, 4) || misaligned(counts, 4) || misaligned(sums, 4) || misaligned(bias, 4)) return UCCL_EALIGN;
  const bool wanted = counts != nullptr || sums != nullptr;
  if (scores->rows == 0u && !wanted) return UCCL_OK;
  const uint32_t groups = route_groups(scores->rows, scores->cols);
  if (wanted && groups > 1u) {
    if (scratch == nullptr || scratch_bytes < uccl_route_rows_scratch(scores->rows, scores->cols)) return UCCL_EINVAL;
    if (misaligned(scratch, 16)) return UCCL_EALIGN;
  }
  const RouteArgs a{experts, weights, counts, sums, groups > 1u ? static_cast<uint32_t*>(scratch) : nullptr, rows_of(scores), bias, scores->rows, scores->cols, opts->slots, opts->normalise, opts->scale};
  const hipStream_t s = static_cast<hipStream_t>(stream);
  Launches go;
  if (scores->rows == 0u) return go(true, route_sum_kernel, blocks_for(scores->cols, 16u), 1024, s, counts, sums, static_cast<const uint32_t*>(nullptr), 0u, scores->cols);
  return with_type(scores->dtype, [&](auto t) {
    using T = decltype(t);
    return with_lanes<T>(scores->rows, scores->cols, [&](auto lanes, auto pieces) -> int {
      constexpr uint32_t L = decltype(lanes)::value, K = decltype(pieces)::value;
      if (!wanted) return go(true, route_kernel<T, L, K, false>, blocks_for(scores->rows, 256u / L), 256, s, a);
      const int first = go(groups == 1u, route_kernel<T, L, K, true>, groups, kRouteSumThreads, s, a);
      if (first != UCCL_OK || groups == 1u) return first;
      return go(true, route_sum_kernel, blocks_for(scores->cols, 16u), 1024, s, counts, sums, static_cast<const uint32_t*>(a.parts), groups, scores->cols);
    });
  });
}

int uccl_route_rows_grad(const uccl_rows* dscores, const uccl_rows* scores, const int32_t* experts, const float* dweights, const float* dsums,
                         const uccl_route_opts* opts, void* stream) {
  int e = check_route(scores, opts);
  if (e == UCCL_OK) e = check(dscores);
  if (e != UCCL_OK) return e;
  if (dscores->dtype != scores->dtype || !same_shape(dscores, scores)) return UCCL_EINVAL;
  if (scores->rows != 0u && (experts == nullptr) != (dweights == nullptr)) return UCCL_EINVAL;
  if (misaligned(experts, 4) || misaligned(dweights, 4) || misaligned(dsums, 4)) return UCCL_EALIGN;
  if (scores->rows == 0u) return UCCL_OK;
  const RouteGradArgs a{rows_of(dscores), rows_of(scores), experts, dweights, dsums, scores->rows, scores->cols, opts->slots, opts->normalise, opts->scale};
  return with_type(scores->dtype, [&](auto t) {
    using T = decltype(t);
    return with_lanes<T>(scores->rows, scores->cols, [&](auto lanes, auto pieces) {
      constexpr uint32_t L = decltype(lanes)::value, K = decltype(pieces)::value;
      return launch(route_grad_kernel<T, L, K>, blocks_for(scores->rows, 256u / L), 256, static_cast<hipStream_t>(stream), a);
    });
  });
}

int uccl_balance_loss(float* loss, float* dsums, const int32_t* counts, const float* sums, uint32_t n_experts, const uccl_balance_opts* o, void* stream) {
  if (o == nullptr || o->tokens == 0u || o->slots == 0u || !isfinite(o->coef) || n_experts > kMost || (n_experts != 0u && (counts == nullptr || sums == nullptr))) return UCCL_EINVAL;
  if (misaligned(loss, 4) || misaligned(dsums, 4) || misaligned(counts, 4) || misaligned(sums, 4)) return UCCL_EALIGN;
  if (loss == nullptr && (dsums == nullptr || n_experts == 0u)) return UCCL_OK;
  const double tokens = static_cast<double>(o->tokens), factor = static_cast<double>(o->coef) * n_experts / (o->slots * tokens * tokens);
  return launch(balance_kernel, 1, 256, static_cast<hipStream_t>(stream), loss, dsums, counts, sums, n_experts, factor);
}

uint64_t uccl_plan_rows_scratch(uint64_t choices, uint32_t n_experts) {
  const uint32_t groups = plan_shape(choices, n_experts, false).groups;
  return groups == 1u ? 0u : (groups * 4ull * n_experts + 15u) / 16u * 16u;
}

int uccl_plan_rows(int32_t* index, int32_t* offsets, int32_t* pos, const int32_t* experts, uint32_t tokens, uint32_t slots, uint32_t n_experts,
                   void* scratch, uint64_t scratch_bytes, void* stream) {
  const uint64_t choices = static_cast<uint64_t>(tokens) * slots;
  if (choices > kMost || n_experts == 0u || n_experts > UCCL_MOST_EXPERTS || offsets == nullptr || (experts == nullptr && choices != 0u)) return UCCL_EINVAL;
  if (index != nullptr && (index == experts || index == pos)) return UCCL_EINVAL;
  if (misaligned(index, 4) || misaligned(offsets, 4) || misaligned(pos, 4) || misaligned(experts, 4)) return UCCL_EALIGN;
  const uint64_t needed = uccl_plan_rows_scratch(choices, n_experts);
  if (needed != 0u) {
    if (scratch == nullptr || scratch_bytes < needed) return UCCL_EINVAL;
    if (misaligned(scratch, 16)) return UCCL_EALIGN;
  }
  const bool counts_all = choices <= kPlanCountsAll && pos != experts;
  const PlanShape shape = plan_shape(choices, n_experts, counts_all);
  const hipStream_t s = static_cast<hipStream_t>(stream);
  Launches go;
  uint32_t* const counts = counts_all || shape.groups == 1u ? nullptr : static_cast<uint32_t*>(scratch);
  const PlanArgs a{index, offsets, pos, experts, counts, static_cast<uint32_t>(choices), slots, n_experts, shape.share};
  if (counts != nullptr) {
    const int e = go(false, plan_count_kernel, shape.groups, kPlanThreads, s, counts, experts, a.choices, n_experts, shape.share);
    if (e != UCCL_OK) return e;
  }
  if (counts_all) return go(true, plan_kernel<1>, shape.groups, kPlanThreads, s, a);
  return shape.rounds == 2u ? go(true, plan_kernel<2>, shape.groups, kPlanThreads, s, a) : go(true, plan_kernel<4>, shape.groups, kPlanThreads, s, a);
}

// kGradientGroups and one more for every matrix, whose last workgroup may have less than its share.
uint64_t uccl_gradient_norm_scratch(uint32_t n) { return ((kGradientGroups + static_cast<uint64_t>(n)) * 8u + 15u) / 16u * 16u; }

int uccl_gradient_norm(float* norm, const uccl_rows* grads, uint32_t n, void* scratch, uint64_t scratch_bytes, void* stream) {
  const int e = check_gradients(grads, n);
  if (e != UCCL_OK) return e;
  if (norm == nullptr || scratch == nullptr || scratch_bytes < uccl_gradient_norm_scratch(n)) return UCCL_EINVAL;
  if (misaligned(norm, 4) || misaligned(scratch, 16)) return UCCL_EALIGN;
  const hipStream_t s = static_cast<hipStream_t>(stream);
  Launches go;
  double* const parts = static_cast<double*>(scratch);
  uint64_t done = 0;
  const Shares shares = shares_of(grads, nullptr, n);
  auto add = [&](auto& a, uint64_t groups, auto kernel) {
    a.parts = parts + done;
    done += groups;
    return go(false, kernel, groups, kGradientThreads, s, a);
  };
  int code = over_matrices<true>(grads, nullptr, n, shares.share, shares.flat, [&](auto& a, uint64_t groups, bool) { return add(a, groups, square_sum_kernel<true>); });
  if (code == UCCL_OK) code = over_matrices<false>(grads, nullptr, n, shares.share, shares.strided, [&](auto& a, uint64_t groups, bool) { return add(a, groups, square_sum_kernel<false>); });
  return code != UCCL_OK ? code : go(true, square_root_kernel, 1, 1024, s, norm, static_cast<const double*>(parts), static_cast<uint32_t>(done));
}

int uccl_gradient_clip(const uccl_rows* out, const uccl_rows* grads, uint32_t n, const float* norm, const uccl_clip_opts* opts, void* stream) {
  int e = check_gradients(grads, n);
  if (e == UCCL_OK) e = check_gradients(out, n);
  if (e != UCCL_OK) return e;
  if (opts == nullptr || !(opts->most > 0.0f) || isinf(opts->most) || opts->reserved[0] || opts->reserved[1] || opts->reserved[2]) return UCCL_EINVAL;
  for (uint32_t i = 0; i < n; ++i)
    if (out[i].dtype != grads[i].dtype || !same_shape(out + i, grads + i)) return UCCL_EINVAL;
  if (n == 0u) return UCCL_OK;
  if (norm == nullptr) return UCCL_EINVAL;
  if (misaligned(norm, 4)) return UCCL_EALIGN;
  Launches go;
  const hipStream_t s = static_cast<hipStream_t>(stream);
  const Shares shares = shares_of(grads, out, n);
  const bool once = shares.bytes > kStayInCaches;
  auto clip = [&](auto& a, uint64_t groups, bool last, auto kernel) {
    a.norm = norm;
    a.most = opts->most;
    return go(last, kernel, groups, kGradientThreads, s, a);
  };
  e = over_matrices<true>(grads, out, n, shares.share, shares.flat, [&](auto& a, uint64_t groups, bool last) {
    last = last && shares.strided == 0u;
    return once ? clip(a, groups, last, gradient_clip_kernel<true, true>) : clip(a, groups, last, gradient_clip_kernel<true, false>);
  });
  if (e != UCCL_OK) return e;
  return over_matrices<false>(grads, out, n, shares.share, shares.strided, [&](auto& a, uint64_t groups, bool last) {
    return once ? clip(a, groups, last, gradient_clip_kernel<false, true>) : clip(a, groups, last, gradient_clip_kernel<false, false>);
  });
}

}  // extern "C"
