/*
 * tsenor_layer.h - C ABI of the operators that run and retrain a layer whose weights carry a transposable mask
 * (tsenor.h finds it), on MI355X (gfx950).
 *
 * A transposable mask prunes W and its transpose alike (Sec. 1), so the forward product x W^T, the input gradient dy W and the
 * weight gradient dy^T x are one kernel here, on operands in 8-bit floating point:
 *
 *   tsenor_quantize        masked weights, tokens or gradients into 8 bits, along the rows, along the columns or both
 *   tsenor_norm            residual addition, root-mean-square norm and its 8-bit output; tsenor_norm_backward: its gradients
 *   tsenor_product         a b^T of two matrices in 8 bits
 *   tsenor_clip            the norm of all gradients of a model, and the gradients scaled down to a largest norm
 *
 * Conventions are those of tsenor.h: pointers are DEVICE pointers of the caller, problem structs (and the table of
 * tsenor_clip) live in HOST memory and are read before the call returns, work is enqueued on `stream` and not synchronised,
 * nothing is allocated, all arguments are checked before the first launch, calls that overlap in time do not share a
 * workspace, and every call can be captured in a HIP graph.  Besides:
 *   - rows, columns and counts may be zero (no tokens this time): outputs that have elements are still written, and pointers to
 *     matrices without elements may be NULL.
 *   - Matrices have at most 2^31 - 256 rows, 2^24 columns, 2^23 - 1 tiles of 128 x 128 and a leading dimension of at most 2^40 (times
 *     the rows 2^60), else TSENOR_ERR_SHAPE.  Rows need not be aligned (matrices whose rows all begin at multiples of 16 bytes are
 *     read and written faster); scaled matrices have to be, see below.
 *   - A misaligned pointer or leading dimension is TSENOR_ERR_ALIGN (pointers: to their elements, workspaces to 256 bytes).
 *   - Results do not depend on what else runs, nor on earlier calls: sums have a fixed order, and there are no atomics.
 *   - Infinities and NaN are inputs like others.
 *   - The GPU of the pointers and of the stream is the calling thread's current one (layer.py makes it current).
 */
#ifndef TSENOR_LAYER_H
#define TSENOR_LAYER_H

#include "tsenor.h"

#ifdef __cplusplus
extern "C" {
#endif

/* A scaled matrix: rows x cols values of 8-bit floating point (e4m3: 4 exponent and 3 mantissa bits, largest value 448, NaN
 * 0x7F and 0xFF, no infinities) with a power of two for each row and TSENOR_SCALE_BLOCK columns,
 *   x[i][j] = e4m3(values[i * ld + j]) * 2^(scales[(j / 128) * scale_ld + i] - 127).
 * A power of two costs a floating-point format nothing but range, and the matrix cores apply it on the way.
 *   - values: 16-byte aligned, ld a multiple of 128, at least cols.  The columns from cols to the next multiple of 128 take
 *     part in products: they hold zeros.  tsenor_quantize and tsenor_norm write them.
 *   - scales: 16-byte aligned, scale_ld a multiple of 16, at least rows.  A byte of 255 means NaN.  What lies past the last row
 *     is neither written nor used.
 * A matrix with one scale for 128 x 128 values holds it once for each of the 128 rows, and its transpose the same ones. */
enum { TSENOR_SCALE_BLOCK = 128 };
typedef struct tsenor_scaled {
  uint8_t* values;
  uint8_t* scales;
  int64_t rows, cols, ld, scale_ld;
} tsenor_scaled;

/* Quantisation.  For each block, 1 x 128 along the row (the last one shorter), or 128 x 128 with `square`:
 *   e = the smallest integer in [-126, 127] with max |x| <= 448 * 2^e over the finite entries (0 where all of them are 0),
 *   value = x * 2^-e to the nearest 8-bit value, ties to even; infinities and NaN give NaN.
 * Entries that the mask drops are +0, whatever they were, and take no part in the maximum. */
typedef struct tsenor_quantize_problem {
  const void* x;          /* rows x cols of `dtype`, leading dimension ld */
  int32_t dtype;          /* TSENOR_F32 or TSENOR_BF16 */
  int32_t square;         /* 0: a scale for 1 x 128, 1: for 128 x 128 */
  int64_t rows, cols, ld;
  const uint8_t* mask;    /* optional, rows x cols bytes, leading dimension cols: 0 drops the entry (the mask of tsenor_mask) */
  tsenor_scaled out;      /* rows x cols; values NULL: not wanted */
  tsenor_scaled out_t;    /* cols x rows, the transpose, its blocks along ITS rows; values NULL: not wanted.  One of the two is */
} tsenor_quantize_problem;
int tsenor_quantize(const tsenor_quantize_problem* p, tsenor_stream_t stream);

/* Residual addition and root-mean-square norm:
 *   h = x + residual, rounded to `dtype` (the residual stream as the rest of the network sees it; x itself without residual)
 *   y = h * (mean over the row of h^2 + eps)^-1/2 * gain, in single precision, the sum of squares too
 * `out` is y in 8 bits, 1 x 128 along the row, as tsenor_quantize makes it from the single-precision values; `y_out` is y
 * rounded to `dtype`.  sum_out may be residual or x (leading dimension cols), y_out may not be any of them. */
typedef struct tsenor_norm_problem {
  const void* x;          /* rows x cols of `dtype`, leading dimension ld */
  const void* residual;   /* optional, leading dimension residual_ld */
  const void* gain;       /* cols of `gain_dtype` */
  int32_t dtype, gain_dtype;
  int64_t rows, cols, ld, residual_ld;
  double eps;             /* finite, >= 0 */
  void* sum_out;          /* optional: h, rows x cols of `dtype`, leading dimension cols */
  void* y_out;            /* optional: y, rows x cols of `dtype`, leading dimension cols */
  tsenor_scaled out;      /* rows x cols; values NULL: not wanted.  One of the three outputs is */
} tsenor_norm_problem;
int tsenor_norm(const tsenor_norm_problem* p, tsenor_stream_t stream);

/* Its gradients, from h as tsenor_norm left it (the rounding of y to 8 bits passes gradients through unchanged):
 *   c_i = (mean_j h_ij^2 + eps)^-1/2
 *   dh_ij = c_i gain_j dy_ij - h_ij c_i^3 mean_k(gain_k dy_ik h_ik) + dsum_ij     (dsum: the gradient that reaches h past the norm)
 *   dgain_j = sum_i dy_ij h_ij c_i                                                 (in single precision, a fixed order)
 * dh is the gradient of x and of residual.  dh_out may be dy or dsum (leading dimension cols). */
typedef struct tsenor_norm_backward_problem {
  const void* h;          /* rows x cols of `dtype`, leading dimension ld */
  const void* gain;       /* cols of `gain_dtype` */
  const void* dy;         /* rows x cols of `dtype`, leading dimension dy_ld */
  const void* dsum;       /* optional, leading dimension dsum_ld */
  int32_t dtype, gain_dtype;
  int64_t rows, cols, ld, dy_ld, dsum_ld;
  double eps;
  void* dh_out;           /* rows x cols of `dtype`, leading dimension cols */
  float* dgain_out;       /* cols floats */
} tsenor_norm_backward_problem;
size_t tsenor_norm_backward_workspace_bytes(const tsenor_norm_backward_problem* p); /* 0 on invalid arguments */
int tsenor_norm_backward(const tsenor_norm_backward_problem* p, void* workspace, size_t workspace_bytes, tsenor_stream_t stream);

/* out[i][j] = sum_k a[i][k] b[j][k], rounded to bf16; 0 where the mask drops it.  The forward pass of a layer takes tokens and W
 * (rows: output columns), the input gradient dy and the transposed W, the weight gradient the transposes of dy and of x with
 * the mask of W.  Sums are in single precision.  The matrix cores line 8-bit products up with the largest of a group and keep 16
 * bits below it, so a result of normal operands is 1.6e-5 off before its rounding to bf16 (2e-3), and operands
 * in 8 bits are 3e-2 off each. */
typedef struct tsenor_product_problem {
  tsenor_scaled a, b;     /* a.cols == b.cols; ld at most 2^22, ceil(cols / 128) * scale_ld below 2^31, b.rows at most 2^24 */
  void* out;              /* a.rows x b.rows bf16, leading dimension out_ld */
  int64_t out_ld;
  const uint8_t* mask;    /* optional, a.rows x b.rows bytes, leading dimension b.rows: 0 drops the result */
} tsenor_product_problem;
/* 0 on invalid arguments, and where no scratch is needed */
size_t tsenor_product_workspace_bytes(const tsenor_product_problem* p);
int tsenor_product(const tsenor_product_problem* p, void* workspace, size_t workspace_bytes, tsenor_stream_t stream);

/* Norm and clipping of gradients: norm = sqrt(sum of squares over all tensors), summed in double;
 *   factor = max_norm / norm where norm is finite and larger than max_norm, 1 otherwise;  out = in * factor, rounded to its dtype.
 * A norm that is not finite, in single precision, leaves the gradients as they are: norm_out says so, and the caller drops the step. */
typedef struct tsenor_gradient {
  const void* in;         /* count elements of `dtype`, in any order */
  void* out;              /* the same; in itself, or memory that overlaps no gradient */
  int64_t count;
  int32_t dtype;          /* TSENOR_F32 or TSENOR_BF16 */
} tsenor_gradient;
typedef struct tsenor_clip_problem {
  const tsenor_gradient* gradients; /* HOST array */
  int32_t count;          /* at most 2^20 tensors of at most 2^40 elements */
  double max_norm;        /* >= 0; infinity: the norm alone is wanted where out is in */
  float* norm_out;        /* 2 floats: norm, factor */
} tsenor_clip_problem;
size_t tsenor_clip_workspace_bytes(const tsenor_clip_problem* p); /* 0 on invalid arguments */
int tsenor_clip(const tsenor_clip_problem* p, void* workspace, size_t workspace_bytes, tsenor_stream_t stream);

#ifdef __cplusplus
}
#endif
#endif /* TSENOR_LAYER_H */
