/*
 * tq_mx.h -- microscaled 4-bit matrices on AMD MI355X (gfx950): the OCP microscaling format MXFP4, cast to it and
 *            back, and the matrix products that training and serving make of it.
 *
 * The layers whose gradients tq.h compresses, with the same means: a block of elements shares a scale, an element takes a
 * few bits, and what has to be unbiased is rounded stochastically with draws that are a pure function of
 * (seed, worker, step, element).  Conventions as in tq.h: *_dev are device pointers owned by the caller, `stream` is a
 * hipStream_t as void*, calls enqueue and return, nothing is allocated or kept, nothing is enqueued on error.
 *
 * A matrix [rows, cols] in this form is two arrays.  32 consecutive elements of a row are a block; a row is padded with
 * zeros to groups of 128 elements (4 blocks), G = ceil(cols / 128).
 *   codes   [rows][64 G] bytes: element j of a row in byte j / 2, the even one in the low half.  A code is a sign (8) and
 *           one of the magnitudes 0, 0.5, 1, 1.5, 2, 3, 4, 6.
 *   scales  [G][rows][4] bytes: the four blocks of a group and row.  s stands for 2^(s - 127); 255 for a block that has
 *           no value (NaN).  Blocks past the last element hold 0.
 * The groups are the scales' outer axis because a product takes many rows' scales of one group at a time.
 */
#ifndef TQ_MX_H
#define TQ_MX_H

#include "tq.h"

#ifdef __cplusplus
extern "C" {
#endif

enum { TQ_F16 = 2 };                                   /* beside TQ_F32 and TQ_BF16 */
enum { TQ_MX_NEAREST = 0, TQ_MX_STOCHASTIC = 1 };      /* rounding */

/* Bytes of the two arrays.  Pure host arithmetic; 0 for a matrix without elements. */
uint64_t tq_mx_code_bytes(uint64_t rows, uint64_t cols);
uint64_t tq_mx_scale_bytes(uint64_t rows, uint64_t cols);

/*
 * tq_mx_quantize -- a matrix to its 4-bit form, its transpose to its 4-bit form, or both from one pass over it.
 *   x_dev      [rows][ld] of TQ_F32, TQ_BF16 or TQ_F16, aligned to an element; ld >= cols elements from row to row
 *   rounding   TQ_MX_NEAREST: with A the largest magnitude of the block, scale 2^(floor(log2 A) - 2), elements to the
 *              nearest, ties to the even code, beyond 6 to 6 (the OCP rule).
 *              TQ_MX_STOCHASTIC: the smallest power of two with A <= 6 * scale, so that nothing is clipped; an element
 *              between two neighbours l < h of the grid, t = (|v| / scale - l) / (h - l), goes up if
 *              floor(65536 t) + r >= 65536 with 16 random bits r: the mean over the draws is v up to 2^-16 of the step.
 *              Scales are at least 2^-127.  A block that holds a NaN or an infinity gets scale 255 and codes 0.
 *   seed, worker, step   element (i, j) draws the 16 bits at place j % 8 of Philox4x32-10 with the counter
 *              (j / 8, i, worker, step) and the key `seed`, the same for both forms; not used by TQ_MX_NEAREST.  Two matrices
 *              cast with one (seed, worker, step) draw the same numbers, and so do a matrix's first row and the payload that
 *              tq_compress makes with them: roundings that are to be independent, as the mean of what is made of several of
 *              them wants it, take different ones, a seed for each matrix of a step say
 *   codes_dev, scales_dev       the form of x [rows, cols], blocks along a row; both NULL if not wanted
 *   codes_t_dev, scales_t_dev   the form of x^T [cols, rows], blocks along a column of x; both NULL if not wanted
 * All four 16-byte aligned, written in full, padding included.  rows, cols = 1 .. 2^31 - 1, rows * ld <= 2^40.
 */
int tq_mx_quantize(const void* x_dev, int dtype, uint64_t rows, uint64_t cols, uint64_t ld, int rounding, uint64_t seed,
                   uint32_t worker, uint32_t step, void* codes_dev, void* scales_dev, void* codes_t_dev, void* scales_t_dev,
                   void* stream);

/*
 * tq_mx_dequantize -- out[i][j] = the value that a matrix in 4-bit form stands for, exactly.
 *   out_dev   [rows][ldo] of TQ_F32 or TQ_BF16 (TQ_F16 does not hold the range)
 */
int tq_mx_dequantize(const void* codes_dev, const void* scales_dev, uint64_t rows, uint64_t cols, void* out_dev, int out_dtype,
                     uint64_t ldo, void* stream);

/*
 * tq_mx_matmul -- out = A B^T (+ add): A [m, k] and B [n, k] in 4-bit form, blocks along k in both, which is what a linear
 * layer's three products want: y = x W^T, dx = dy (W^T)^T, dW = dy^T (x^T)^T, the transposes from tq_mx_quantize.
 * Products are exact, sums are binary32, one rounding to out's type at the end.  The same call on the same device gives
 * the same bits every time.
 *   add_dev        NULL, or [m][lda] floats, each added once, to the finished sum in binary32, before the rounding to out's
 *                  type; may be out_dev (gradients that are accumulated over batches), with the same row length then
 *   out_dev        [m][ldo] of TQ_F32, TQ_BF16 or TQ_F16 (infinite beyond its range); ldo >= n elements from row to row
 *   workspace_dev  at least tq_mx_matmul_workspace_bytes(m, n, k) bytes, 16-byte aligned (NULL if that is 0): partial
 *                  sums where k is split; contents undefined afterwards; calls that share it have to be ordered
 * m, n, k = 1 .. 2^31 - 1, m * k, n * k, m * ldo and m * lda <= 2^40.
 */
uint64_t tq_mx_matmul_workspace_bytes(uint64_t m, uint64_t n, uint64_t k);
int tq_mx_matmul(const void* a_codes_dev, const void* a_scales_dev, const void* b_codes_dev, const void* b_scales_dev,
                 uint64_t m, uint64_t n, uint64_t k, const float* add_dev, uint64_t lda, void* out_dev, int out_dtype,
                 uint64_t ldo, void* workspace_dev, uint64_t workspace_bytes, void* stream);

/*
 * tq_mx_linear -- out = Q(x) W^T: a linear layer on tokens as the layer before left them, Q the nearest rounding of
 * tq_mx_quantize.  Equals tq_mx_quantize and tq_mx_matmul up to the order of the sums; few tokens (serving, one token for
 * each of a few requests) are cast inside the product.
 *   x_dev          [m][ldx] of TQ_F32, TQ_BF16 or TQ_F16
 *   out_dev        [m][ldo] of out_dtype
 *   workspace_dev  tq_mx_linear_workspace_bytes(m, n, k) bytes, rules as in tq_mx_matmul
 */
uint64_t tq_mx_linear_workspace_bytes(uint64_t m, uint64_t n, uint64_t k);
int tq_mx_linear(const void* x_dev, int dtype, uint64_t m, uint64_t ldx, const void* w_codes_dev, const void* w_scales_dev,
                 uint64_t n, uint64_t k, void* out_dev, int out_dtype, uint64_t ldo, void* workspace_dev,
                 uint64_t workspace_bytes, void* stream);

#ifdef __cplusplus
}
#endif
#endif /* TQ_MX_H */
