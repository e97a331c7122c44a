/*
 * uccl_rows.h -- C ABI of the row operators around an all-to-all dispatch, on AMD Instinct MI355X (gfx950).
 *
 * A rank of an expert-parallel layer normalises its tokens' rows and dispatches them (uccl_chunk_segment, the network,
 * uccl_chunk_scatter on the other side), multiplies the rows that it received with the weights of its own experts, and
 * adds what comes back to its tokens.  These calls are the work on either side of the dispatch:
 *     uccl_norm_rows       residual's addition, root-mean-square norm, output in 16 / 32 bits or in 8 bits with a scale a row
 *     uccl_group_product   products grouped by expert, ragged groups whose sizes are known to the GPU only
 *     uccl_combine_rows    every token's weighted sum of its experts' rows, and the residual
 * and their gradients.  As in uccl_chunk.h: every pointer inside a uccl_rows, and every pointer that is not one to a
 * HOST struct, is a DEVICE pointer owned by the caller; `stream` is a hipStream_t passed as void*; a call only enqueues
 * work on `stream` and returns: no allocation, no host synchronisation, no host read of device memory.  Calls may be
 * captured into a graph.  The results of a call on the same inputs are the same bit for bit: no atomics.
 *
 * Every call returns UCCL_OK, also where there is nothing to compute; UCCL_EINVAL: a null pointer, shapes or types that do not
 * match; UCCL_EALIGN; UCCL_ETOOBIG: more workgroups than one launch can have (2^32 threads: 2^22 - 1 rows of a norm, and fewer than 2^22 tiles
 * of 128 x 128 elements of a product always fit; split the call); UCCL_ELAUNCH: HIP's, the text in uccl_last_error_detail().  Nothing has
 * been enqueued then, but for uccl_norm_rows_grad: two launches, of which HIP may take the first and refuse the second.
 * uccl_time_next_launch times these calls too; uccl_norm_rows_grad has its start on the first of its launches and its stop on the last.
 *
 * The operators are no passage of the paper, which moves such rows and leaves the work on them to the application
 * (its evaluation has expert-parallel prefill and decode among the applications).
 */
#ifndef UCCL_ROWS_H
#define UCCL_ROWS_H

#include "uccl_chunk.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Element types of rows, besides UCCL_F32, UCCL_BF16 and UCCL_F16: OCP e4m3 (4 exponent bits, bias 7, no infinity, largest
 * value 448), with one binary32 scale a row: an element stands for its value times its row's scale. */
#define UCCL_E4M3 16
/* ... and microscaled 4 bits (OCP MXFP4): e2m1 elements, 0, 0.5, 1, 1.5, 2, 3, 4, 6 with a sign above, two a byte, the earlier one in the lower half; and for
 * every 32 of a row one byte of scale: the power of two with that number less 127 as its exponent, 255 is NaN. */
#define UCCL_MX4 17

/* A matrix by rows (HOST struct, read during the call).  `data` is 16-byte aligned and `stride` (bytes from one row to the
 * next) a multiple of 16; `cols` may be any number of elements.  The 16-byte piece that holds a row's last element may be
 * read whole, past the row's end; nothing past the end is written, and what is there never changes a result.  8-bit rows
 * have their scales at scales + i * scale_stride, 4-byte aligned, scale_stride a multiple of 4: side by side with the values
 * they make a row that is dispatched as one piece; 0 is one scale for all rows, where rows are read.  Rows of 4 bits have ceil(cols / 32) bytes of scales
 * there, by the same rules; the aligned 4 bytes that hold a row's last scale may be read whole.  A matrix of one row, or of
 * none, may have any stride. */
typedef struct uccl_rows {
  void* data;
  uint64_t stride;
  void* scales;          /* UCCL_E4M3 and UCCL_MX4 only, NULL otherwise */
  uint64_t scale_stride; /* bytes */
  uint32_t rows, cols;   /* at most 2^31 - 1 rows of at most 2^30 columns */
  uint32_t dtype;        /* UCCL_F32, UCCL_BF16, UCCL_F16, UCCL_E4M3 or UCCL_MX4 */
  uint32_t reserved;     /* 0 */
} uccl_rows;

/*
 * uccl_norm_rows -- h = x + r;  s = 1 / sqrt(mean of h^2 over the row + eps);  y = h s w.
 *
 *   y        written: x's type, or UCCL_E4M3: the row's scale is max |y| / 448 (at least 2^-126) and its elements are
 *            y / scale, a binary32 quotient, rounded to nearest even
 *   h        written: the sum in x's type, the next residual; NULL = not wanted.  May be x or r itself
 *   rstd     written: s, one float a row, 4-byte aligned; NULL = not wanted
 *   x, r     read: UCCL_F32, UCCL_BF16 or UCCL_F16, the same; r NULL = no residual
 *   weight   read: `cols` elements of x's type, 16-byte aligned
 *   opts     eps: at least 0, finite
 * Sums are held in binary32, and y is computed from h before that is rounded for storage.  y may be x or r itself if it has
 * its type and stride.  A NaN or an infinity in a row makes the row's y what the formula makes it; elements that are not finite do
 * not enter the scale unless they are infinities.
 */
typedef struct uccl_norm_opts { /* HOST struct, read during the call */
  float eps;
  uint32_t reserved[3]; /* 0 */
} uccl_norm_opts;

int uccl_norm_rows(const uccl_rows* y, const uccl_rows* h, float* rstd, const uccl_rows* x, const uccl_rows* r,
                   const void* weight, const uccl_norm_opts* opts, void* stream);

/*
 * uccl_norm_rows_grad -- with n = h s and g = dy w:  dx = dh + s (g - n mean of (g n) over the row), which is the gradient
 * of x and of r alike;  dweight = sum of dy n over the rows.
 *
 *   dx       written: h's type; may be dy or dh itself
 *   dweight  written: `cols` floats, 4-byte aligned (zeros if there are no rows)
 *   dy, h    read, with rstd and weight as uccl_norm_rows has them; all of one type
 *   dh       read: what arrives along the residual, the gradient of h; NULL = nothing
 *   scratch  device memory of at least uccl_norm_rows_scratch(rows, cols) bytes, 16-byte aligned, the call's own until
 *            the stream has passed it
 */
int uccl_norm_rows_grad(const uccl_rows* dx, float* dweight, const uccl_rows* dy, const uccl_rows* dh, const uccl_rows* h,
                        const float* rstd, const void* weight, void* scratch, uint64_t scratch_bytes, void* stream);
uint64_t uccl_norm_rows_scratch(uint32_t rows, uint32_t cols);

/*
 * uccl_group_product -- y[i] = x[index[i]] . w[g]^T for the rows i of every group g: offsets[g] <= i < offsets[g + 1].
 *
 *   y        written: n columns, UCCL_F32, UCCL_BF16 or UCCL_F16.  Rows of no group are left alone
 *   x        read: k columns, UCCL_BF16, UCCL_F16, UCCL_E4M3 or UCCL_MX4
 *   index    read: the row of x for every row of y, int32, 4-byte aligned; NULL = row i itself.  A row may be named any
 *            number of times; a number that is no row of x stands for a row of zeros
 *   w        read: n_groups * n rows of k columns, x's type, or UCCL_MX4 beside rows in 16 bits; the n rows of a group follow each other
 *   offsets  read: n_groups + 1 int32, 4-byte aligned, in ascending order; one that is below its predecessor counts as
 *            that, below 0 as 0, above the rows of y as these
 * Sums are held in binary32 and rounded once; 8-bit operands are multiplied as they are, exactly, and the sum by both scales.  Operands in 4 bits stand
 * for their values with their blocks' scales: of two of them a block's 32 products are added exactly; beside rows in 16 bits they are what
 * bf16 holds exactly, or f16; one of 2^128 and above (4 and 6 by the scale 2^126, 2 and above by 2^127: no uccl_quantise_rows makes them) makes its sums there infinities or NaN.
 * What a call is cut into depends on its sizes alone, never on the offsets' values.
 */
int uccl_group_product(const uccl_rows* y, const uccl_rows* x, const int32_t* index, const uccl_rows* w,
                       const int32_t* offsets, uint32_t n_groups, void* stream);

/* dx[i] = dy[i] . w[g], the gradient of row i as uccl_group_product read it: the gradient of a row of x that `index` names
 * several times is the sum of theirs (uccl_combine_rows).  dy, w: UCCL_BF16 or UCCL_F16; dx: UCCL_F32, UCCL_BF16, UCCL_F16. */
int uccl_group_product_grad_x(const uccl_rows* dx, const uccl_rows* dy, const uccl_rows* w, const int32_t* offsets,
                              uint32_t n_groups, void* stream);

/* dw[g] = sum over the group's rows of dy[i]^T x[index[i]]; zeros for a group without rows.  dy, x: UCCL_BF16 or UCCL_F16;
 * dw: UCCL_F32, UCCL_BF16 or UCCL_F16, n_groups * n rows of k columns. */
int uccl_group_product_grad_w(const uccl_rows* dw, const uccl_rows* dy, const uccl_rows* x, const int32_t* index,
                              const int32_t* offsets, uint32_t n_groups, void* stream);

/*
 * uccl_combine_rows -- out[t] = r[t] + sum over j < slots of weights[t, j] y[pos[t, j]].
 *
 *   out      written: y's type
 *   y, r     read: UCCL_F32, UCCL_BF16 or UCCL_F16, the same; r NULL = nothing added; out may be r itself
 *   pos      read: tokens x slots int32, 4-byte aligned; a number that is no row of y (-1, say) adds nothing
 *   weights  read: tokens x slots floats, 4-byte aligned; NULL = 1
 * Sums are held in binary32 in the order of the slots and rounded once.
 */
int uccl_combine_rows(const uccl_rows* out, const uccl_rows* y, const int32_t* pos, const float* weights, uint32_t slots,
                      const uccl_rows* r, void* stream);

/* dy[pos[t, j]] = weights[t, j] dout[t], and dweights[t, j] = dout[t] . y[pos[t, j]] (0 where pos names no row).  Every row of
 * y is named at most once (the caller's to keep: of two slots that name one row either may leave its gradient); rows that
 * no slot names are left alone.  dweights NULL: not wanted, and y is not read (but its rows and columns count). */
int uccl_combine_rows_grad(const uccl_rows* dy, float* dweights, const uccl_rows* dout, const uccl_rows* y,
                           const int32_t* pos, const float* weights, uint32_t slots, void* stream);

#ifdef __cplusplus
}
#endif
#endif /* UCCL_ROWS_H */
