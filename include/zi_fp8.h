/*
 * zi_fp8.h — C ABI of the layer operators in 8-bit floating point that surround the optimizer step.
 *
 * The step of zi.h takes 16-bit gradients and leaves fp32 masters and a 16-bit copy.  These calls make the
 * products between the two with weights, activations and gradients in 8 bits:
 *
 *   zi_fp8_quantize       masters, copy, activations or gradients to 8 bits, as they are, transposed, or both
 *   zi_fp8_matmul         D = A B^T (+ C): a layer's product, and with transposed operands the gradients of its
 *                         input and of its weights; one token's row up to a whole batch
 *   zi_rms_norm           residual addition, root-mean-square norm, output in 8 bits (and 16)
 *   zi_rms_norm_backward  gradients of the norm's input and of gamma, ready for zi_grad_norm and zi_adamw_step
 *
 * A matrix in 8 bits holds e4m3 numbers (sign, 4 bits of exponent, 3 of fraction, largest finite 448, NaN, no
 * infinity) and one scale for each block: 128 consecutive columns of one row (block_rows 1: activations and
 * gradients) or of 128 rows (block_rows 128: weights).  Blocks start at row 0 and column 0; the last of a row or
 * column may be short.  A scale is a power of two in one byte (e8m0: b stands for 2^(b - 127), 255 for NaN), which the
 * matrix cores apply as they multiply.  An element's value is its number times its block's scale.
 *
 * The scale of a block is the smallest power of two, 2^-127 at least, that brings its largest finite magnitude to 448 or
 * less; 1 if there is none above zero.  Numbers are rounded once, to nearest even, ties included.  An infinity or NaN
 * becomes NaN in its own place only and has no part in the scale: it reaches whatever is made of it, and the gradients
 * so made raise found_inf in zi_grad_norm.
 *
 * Conventions are those of zi.h: plain addresses, statuses and zi_last_error(), nothing kept after a call, everything
 * checked before anything is launched, asynchronous on hip_stream, no allocation (calls can be captured into a
 * graph).  Sizes of zero are valid.  An output shares no byte with an input or another output, except where in-place use is
 * said to work; then both have the same address and pitch.  Columns or rows of one buffer may be input and output of a call,
 * if their pitches are the same or one is a multiple of the other; an output in 8 bits has its rows' pitches to itself.  The results of a call do not depend on the order in which
 * the GPU runs its workgroups.
 */
#ifndef ZI_FP8_H
#define ZI_FP8_H

#include "zi.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Beside ZI_BF16 and ZI_FP16, where a call says that it takes it. */
#define ZI_FP32 2

#define ZI_FP8_BLOCK 128

/*
 * A matrix in 8 bits.  data: rows of cols bytes and up to the next multiple of 16, each ld bytes from the one before, 16-byte
 * aligned, ld a multiple of 16 and at least cols; what these bytes hold from column cols on is never used (zi_fp8_quantize
 * writes zeros up to the next multiple of 8, or 16 in `turned`; zi_rms_norm of 8).  scale: ceil(rows / block_rows) rows of
 * ceil(cols / 128) bytes and up to the next multiple of 4, scale_ld bytes apart, 4-byte aligned, scale_ld a multiple of 4 and at
 * least ceil(cols / 128); the bytes behind the last block's are read, and neither used nor written.  block_rows: 1 or 128.
 */
typedef struct {
    void* data;
    void* scale;
    int64_t rows, cols;
    int64_t ld, scale_ld;
    int32_t block_rows;
    int32_t reserved;      /* 0 */
} zi_fp8_matrix;

/*
 * x (rows x cols, pitch ld elements, ZI_BF16, ZI_FP16 or ZI_FP32, aligned to its element) in 8 bits.  out: rows x cols, or NULL.
 * turned: the transposed matrix, cols x rows, quantised along its own rows (block_rows 1: a block is 128 rows of x in
 * one column; 128: the blocks of `out`, transposed), or NULL.  Both are written in one pass over x.
 */
zi_status zi_fp8_quantize(const void* x, int32_t dtype, int64_t rows, int64_t cols, int64_t ld, const zi_fp8_matrix* out,
                          const zi_fp8_matrix* turned, void* hip_stream);

/*
 * D = A B^T + C: a is m x k, b is n x k, d and c are m x n with pitch ldd, ZI_BF16 or ZI_FP16, aligned to their
 * element; c may be NULL (nothing is added) or d (accumulation over micro-batches, rounded in each).  k = 0 gives C,
 * or zeros.  Pitches of operands are below 2^23.
 * The matrix cores add the products of 16 neighbouring k at a time, with fewer bits than fp32 has: what lies more than
 * about 2^-14 below the largest of the 16 is dropped, 1.5e-5 of the result (2-norm) on normal numbers, 5e-5 where one
 * column in 64 is twenty times the others.  Their sums are added in fp32, and so is c; the result is rounded once.
 * The order of k, and with it these roundings, depends on the sizes and on the place in D: the same call gives the same bits, but
 * rows of A that are equal may give rows of D that differ by a rounding, and so may a row in a call with other rows.
 *   a layer y = x W^T:    a = x (block_rows 1), b = W (block_rows 128, n x k)
 *   its input's gradient: a = dy, b = W turned
 *   its weights':         a = dy turned, b = x turned (both block_rows 1)
 * d_workspace: device, 16-byte aligned, of at least zi_fp8_matmul_workspace_bytes(m, n, k) bytes (NULL where that is
 * 0); needs no initialisation, holds garbage afterwards; two calls that share one are ordered on one stream.
 */
size_t zi_fp8_matmul_workspace_bytes(int64_t m, int64_t n, int64_t k);
zi_status zi_fp8_matmul(const zi_fp8_matrix* a, const zi_fp8_matrix* b, void* d, int32_t dtype, int64_t ldd, const void* c,
                        void* d_workspace, size_t workspace_bytes, void* hip_stream);

/*
 * Row by row, with h = x + residual rounded to dtype (h = x without a residual):
 *   rstd = 1 / sqrt(mean(h^2) + eps)      y = h * rstd * gamma
 * The mean and rstd are in fp32: a row whose squares pass 3.4e38 in sum has rstd 0; with eps 0, one of magnitudes below
 * 2^-75 (2.6e-23) throughout has an infinite one, as a row of zeros has.  x, residual, sum, y: rows x cols in dtype (ZI_BF16 or ZI_FP16), aligned to their element, each with its own pitch in elements.  gamma: cols in dtype.  sum (h; needs a residual), y,
 * rstd (rows fp32) and y8 (block_rows 1, of the unrounded y) are outputs, NULL where they are not wanted; at least one is.
 * sum may be x or residual, y may be x, in place.  1 <= cols <= 65536.
 */
#define ZI_RMS_NORM_MAX_COLS 65536
typedef struct {
    const void* x;
    const void* residual;
    const void* gamma;
    void* sum;
    void* y;
    float* rstd;
    int64_t rows, cols;
    int64_t x_ld, residual_ld, sum_ld, y_ld;
    float eps;
    int32_t dtype;
} zi_rms_norm_args;

zi_status zi_rms_norm(const zi_rms_norm_args* args, const zi_fp8_matrix* y8, void* hip_stream);

/*
 * With u = dy * gamma and n = h * rstd, row by row:
 *   dx = rstd * (u - n * mean(u * n)) + dsum       dgamma = sum over rows of dy * n
 * dx is the gradient of x and of the residual alike.  dsum: what reaches h by another way (the residual stream), or
 * NULL.  dy, h, dsum, dx: rows x cols in dtype with their own pitches; h and rstd as zi_rms_norm left them.  dgamma:
 * cols in dgamma_dtype (dtype or ZI_FP32), or NULL; with accumulate != 0 it is added to, rounded once.  dx may be NULL,
 * or dy, or dsum in place.  The sum over rows is made in fp32 in a fixed order.  d_workspace: device, 16-byte aligned, at least
 * zi_rms_norm_workspace_bytes(rows, cols) bytes, as in zi_fp8_matmul; may be NULL if dgamma is and
 * cols is at most 8192.  1 <= cols <= 65536.
 */
typedef struct {
    const void* dy;
    const void* h;
    const void* gamma;
    const float* rstd;
    const void* dsum;
    void* dx;
    void* dgamma;
    int64_t rows, cols;
    int64_t dy_ld, h_ld, dsum_ld, dx_ld;
    int32_t dtype, dgamma_dtype;
    int32_t accumulate;
    int32_t reserved;      /* 0 */
} zi_rms_norm_backward_args;

size_t zi_rms_norm_workspace_bytes(int64_t rows, int64_t cols);
zi_status zi_rms_norm_backward(const zi_rms_norm_backward_args* args, void* d_workspace, size_t workspace_bytes,
                               void* hip_stream);

#ifdef __cplusplus
}
#endif
#endif /* ZI_FP8_H */
