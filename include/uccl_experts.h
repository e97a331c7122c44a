/*
 * uccl_experts.h -- C ABI of what decides where rows go, of experts in 4 bits, and of clipping, on AMD Instinct MI355X (gfx950).
 *
 * Beside the row operators of uccl_rows.h, which take the experts of a dispatch as given:
 *     uccl_route_rows        a router's scores to every token's experts and their weights, counts and probabilities; its gradient
 *     uccl_balance_loss      the loss that keeps experts evenly used, and its gradient
 *     uccl_plan_rows         the tokens' experts to what uccl_group_product and uccl_combine_rows go by
 *     uccl_quantise_rows     rows to microscaled 4 bits (UCCL_MX4), which uccl_group_product takes
 *     uccl_gradient_norm     the norm of many gradients together
 *     uccl_gradient_clip     gradients scaled down to a norm
 *
 * As there: pointers that are not to a HOST struct are DEVICE pointers owned by the caller; `stream` is a hipStream_t passed as void*; a call
 * only enqueues work on `stream` and returns: no allocation, no host synchronisation, no host read of device memory.  Calls may be captured
 * into a graph.  The results of a call on the same inputs are the same bit for bit.  `scratch` is device memory of at least as many bytes
 * as the call's _scratch function says, 16-byte aligned, the call's own until the stream has passed it; what it holds before is of no matter, and no two
 * calls that may run at the same time share it (two captured graphs, say).
 * What a call writes overlaps nothing else that it reads or writes, but where an entry says that it may be the same.
 *
 * Every call returns UCCL_OK, also where there is nothing to compute; UCCL_EINVAL: a null pointer, shapes or types that do not match, a number
 * out of its range; UCCL_EALIGN; UCCL_ETOOBIG: more workgroups than one launch can have (2^32 threads); UCCL_ELAUNCH: HIP's, the text in
 * uccl_last_error_detail().  Nothing has been enqueued then, but where HIP takes the first launches of a call of several and refuses a
 * later one.  uccl_time_next_launch times these calls too, with its start on the first of a call's launches and its stop on the last.
 */
#ifndef UCCL_EXPERTS_H
#define UCCL_EXPERTS_H

#include "uccl_rows.h"

#ifdef __cplusplus
extern "C" {
#endif

#define UCCL_MOST_EXPERTS 1024
#define UCCL_MOST_SLOTS 32

/*
 * uccl_route_rows -- with z a token's scores and p = softmax(z) over its experts:
 *     key_e = z_e + bias_e in binary32;  the token's experts are the `slots` with the greatest keys, in that order, of equal keys the lowest
 *     expert first;  weight = scale p_e, or, normalised, scale p_e / (sum of p over the token's experts).
 * (The bias is the score's, not p's: a router that adds it to a probability, or whose probabilities are sigmoids, is another.)
 *
 *   experts  written: tokens x slots int32, 4-byte aligned.  An expert whose key is -infinity or NaN is never chosen; where too few are left, -1
 *   weights  written: tokens x slots floats, 4-byte aligned; 0 beside a -1
 *   counts   written: how many tokens each expert has, int32; NULL = not wanted
 *   sums     written: the sum of p over the tokens, one float an expert; NULL = not wanted
 *   scores   read: tokens rows of at most UCCL_MOST_EXPERTS columns, UCCL_F32, UCCL_BF16 or UCCL_F16
 *   bias     read: one float an expert, 4-byte aligned; NULL = none.  It moves the choice, not p
 *   opts     slots: 1 to the number of experts, UCCL_MOST_SLOTS at most; normalise: 0 or 1; scale: finite
 *   scratch  if counts or sums are wanted: uccl_route_rows_scratch(tokens, experts) bytes
 * A token whose scores are all -infinity has no expert, and p = 0.  A NaN or +infinity among a token's scores makes its p, and so the weights
 * that are not 0 beside a -1, NaN.
 */
typedef struct uccl_route_opts { /* HOST struct, read during the call */
  uint32_t slots;
  uint32_t normalise;
  float scale;
  uint32_t reserved; /* 0 */
} uccl_route_opts;

int uccl_route_rows(int32_t* experts, float* weights, int32_t* counts, float* sums, const uccl_rows* scores, const float* bias,
                    const uccl_route_opts* opts, void* scratch, uint64_t scratch_bytes, void* stream);
uint64_t uccl_route_rows_scratch(uint32_t tokens, uint32_t n_experts);

/*
 * uccl_route_rows_grad -- the gradient of the scores, for gradients of the weights and of the sums of probabilities; the choice is constant.
 *
 *   dscores   written: scores' type; may be scores itself
 *   scores    read, with opts, as uccl_route_rows had them
 *   experts   read: as uccl_route_rows wrote them; a number that is no expert adds nothing.  NULL = no gradient of the weights
 *   dweights  read: tokens x slots floats, 4-byte aligned; NULL if and only if experts is
 *   dsums     read: one float an expert, 4-byte aligned; NULL = none
 */
int uccl_route_rows_grad(const uccl_rows* dscores, const uccl_rows* scores, const int32_t* experts, const float* dweights,
                         const float* dsums, const uccl_route_opts* opts, void* stream);

/*
 * uccl_balance_loss -- loss = coef E / (slots tokens^2) * (sum over the E experts of counts sums), which is coef where all are used evenly;
 * dsums_e = coef E / (slots tokens^2) counts_e, its gradient (the counts are constant).
 *
 *   loss     written: one float; NULL = not wanted
 *   dsums    written: one float an expert; NULL = not wanted.  May be sums itself
 *   counts, sums   read: as uccl_route_rows wrote them, or added up over ranks
 *   opts     tokens: of all of these ranks; slots; at least 1 each.  coef: finite
 * All 4-byte aligned.  The sum is held in binary64.
 */
typedef struct uccl_balance_opts { /* HOST struct, read during the call */
  uint64_t tokens;
  uint32_t slots;
  float coef;
} uccl_balance_opts;

int uccl_balance_loss(float* loss, float* dsums, const int32_t* counts, const float* sums, uint32_t n_experts, const uccl_balance_opts* opts,
                      void* stream);

/*
 * uccl_plan_rows -- the choices (token t's slot j is choice t slots + j) in order of their experts, of one expert in their own order:
 *
 *   index    written: the token of every row, tokens x slots int32: what uccl_group_product reads its rows through.  -1 behind the last group
 *   offsets  written: n_experts + 1 int32, the experts' first rows; the last is the number of all rows
 *   pos      written: the row of every choice, tokens x slots int32: what uccl_combine_rows takes.  -1 for one without an expert
 *   experts  read: tokens x slots int32; a number below 0 or from n_experts on is no expert
 *   scratch  uccl_plan_rows_scratch(choices, n_experts) bytes, which may be none; choices = tokens x slots
 * All 4-byte aligned; at most 2^31 - 1 choices, 1 to UCCL_MOST_EXPERTS experts.  index and pos may be NULL: not wanted.  pos may be experts itself where
 * index is NULL or another.
 */
int uccl_plan_rows(int32_t* index, int32_t* offsets, int32_t* pos, const int32_t* experts, uint32_t tokens, uint32_t slots,
                   uint32_t n_experts, void* scratch, uint64_t scratch_bytes, void* stream);
uint64_t uccl_plan_rows_scratch(uint64_t choices, uint32_t n_experts);

/*
 * uccl_quantise_rows -- rows to UCCL_MX4: for every block of 32 elements of a row, s = 2^(floor(log2(max |x|)) - 2), at least 2^-127, and of every
 * element the nearest of 0, 0.5, 1, 1.5, 2, 3, 4, 6 to |x| / s, of two the one with an even number, 6 from there on, with its sign.
 *
 *   q        written: UCCL_MX4.  The bits behind a row's last element in its byte are 0; no scale behind the last block is written
 *   values   written: what q stands for, in x's type; NULL = not wanted.  May be x itself
 *   x        read: UCCL_F32, UCCL_BF16 or UCCL_F16
 * A block with a NaN or an infinity has the scale that is NaN, elements 0, and values NaN.
 */
int uccl_quantise_rows(const uccl_rows* q, const uccl_rows* values, const uccl_rows* x, void* stream);

/*
 * uccl_gradient_norm -- the root of the sum of the squares of all elements of n matrices, held in binary64 and rounded once.
 *
 *   norm     written: one float, 4-byte aligned
 *   grads    HOST array of n matrices, read during the call: UCCL_F32, UCCL_BF16 or UCCL_F16, each its own.  What a matrix has contiguous is given
 *            as one row where its rows are not a multiple of 16 bytes
 *   scratch  uccl_gradient_norm_scratch(n) bytes
 * A NaN or an infinity among them makes the norm what the formula makes it.
 *
 * uccl_gradient_clip -- out = grad * min(1, most / norm) for each of n matrices, products in binary32, then rounded to the type.
 *
 *   out      HOST array of n matrices, written: type and shape of the grad beside it, and may be that itself: then nothing is written where the
 *            factor is 1.  A matrix may be twice among the grads of a norm, and counts twice; among out each is once
 *   norm     read: one float, 4-byte aligned, as uccl_gradient_norm wrote it, or of more than one rank
 *   opts     most: above 0, finite
 * A norm of NaN makes every element NaN; one of infinity makes finite elements 0.
 */
int uccl_gradient_norm(float* norm, const uccl_rows* grads, uint32_t n, void* scratch, uint64_t scratch_bytes, void* stream);
uint64_t uccl_gradient_norm_scratch(uint32_t n);

typedef struct uccl_clip_opts { /* HOST struct, read during the call */
  float most;
  uint32_t reserved[3]; /* 0 */
} uccl_clip_opts;

int uccl_gradient_clip(const uccl_rows* out, const uccl_rows* grads, uint32_t n, const float* norm, const uccl_clip_opts* opts, void* stream);

#ifdef __cplusplus
}
#endif
#endif /* UCCL_EXPERTS_H */
