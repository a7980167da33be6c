/*
 * tq_i8.h -- matrices of 8-bit integers with a scale for each row on AMD MI355X (gfx950): cast to them and back, products, and a
 *            linear layer for few or many tokens.
 *
 * Beside the 4-bit matrices of tq_mx.h: twice the bytes, for a student whose forward pass wants more than 4 bits; weights have a
 * scale for each output channel, activations one for each token.  Conventions as in tq.h and tq_mx.h.
 *
 * A matrix [rows, cols] in this form is two arrays:
 *   codes   [rows][128 G] int8, G = ceil(cols / 128), zeros behind the last element
 *   scales  [rows] floats; element (i, j) stands for codes[i][j] * scales[i]
 */
#ifndef TQ_I8_H
#define TQ_I8_H

#include "tq_mx.h"

#ifdef __cplusplus
extern "C" {
#endif

#define TQ_I8_MAX_K 131071      /* 128 * 128 * TQ_I8_MAX_K < 2^31: a sum of products never leaves 32 bits */

/* Bytes of the codes (the scales are 4 a row).  Pure host arithmetic; 0 for a matrix without elements. */
uint64_t tq_i8_code_bytes(uint64_t rows, uint64_t cols);

/*
 * tq_i8_quantize -- with A the largest magnitude of a row: its scale is A / 127, rounded to binary32, and an element's code is
 * the whole number nearest to 127 x / A, ties to even, of the quotient itself and not of a rounded one.  A row of zeros has scale 0; a
 * row that holds a NaN or an infinity has scale NaN and codes 0.  Codes are -127 .. 127.
 *   x_dev      [rows][ldx] of TQ_F32, TQ_BF16 or TQ_F16, aligned to an element; ldx >= cols elements from row to row
 *   codes_dev, scales_dev   16-byte and 4-byte aligned, written in full, padding included
 * rows, cols = 1 .. 2^31 - 1, rows * ldx and rows * 128 G <= 2^40.
 */
int tq_i8_quantize(const void* x_dev, int dtype, uint64_t rows, uint64_t cols, uint64_t ldx, void* codes_dev, float* scales_dev,
                   void* stream);

/* tq_i8_dequantize -- out[i][j] = codes[i][j] * scales[i], rounded once to out's type.  out_dev [rows][ldo] of any of the three types. */
int tq_i8_dequantize(const void* codes_dev, const float* scales_dev, uint64_t rows, uint64_t cols, void* out_dev, int out_dtype,
                     uint64_t ldo, void* stream);

/*
 * tq_i8_matmul -- out = A B^T (+ bias): A [m, k] and B [n, k] in 8-bit form.  The sum of products is exact, then
 * ((float(sum) * scale of A's row) * scale of B's row) + bias in binary32, each rounded once, and one rounding to out's type.
 *   bias_dev       NULL, or [n] floats
 *   out_dev        [m][ldo] of TQ_F32, TQ_BF16 or TQ_F16 (infinite beyond its range); ldo >= n elements from row to row
 *   workspace_dev  at least tq_i8_matmul_workspace_bytes(m, n, k) bytes, 16-byte aligned (NULL if that is 0); contents undefined
 *                  afterwards; calls that share it have to be ordered
 * Any codes in a row's first k bytes may be used (-128 too); those behind them have to be 0 in one of the two matrices.
 * m, n = 1 .. 2^31 - 1, k = 1 .. TQ_I8_MAX_K, m * k, n * k and m * ldo <= 2^40.
 */
uint64_t tq_i8_matmul_workspace_bytes(uint64_t m, uint64_t n, uint64_t k);
int tq_i8_matmul(const void* a_codes_dev, const float* a_scales_dev, const void* b_codes_dev, const float* b_scales_dev, uint64_t m,
                 uint64_t n, uint64_t k, const float* bias_dev, void* out_dev, int out_dtype, uint64_t ldo, void* workspace_dev,
                 uint64_t workspace_bytes, void* stream);

/*
 * tq_i8_linear -- out = Q(x) W^T (+ bias): a linear layer on tokens as the layer before left them, Q the rounding of tq_i8_quantize.
 * Equals tq_i8_quantize and tq_i8_matmul bit for bit; few tokens are cast inside the product.
 *   x_dev          [m][ldx] of TQ_F32, TQ_BF16 or TQ_F16
 *   workspace_dev  tq_i8_linear_workspace_bytes(m, n, k) bytes, rules as in tq_i8_matmul
 */
uint64_t tq_i8_linear_workspace_bytes(uint64_t m, uint64_t n, uint64_t k);
int tq_i8_linear(const void* x_dev, int dtype, uint64_t m, uint64_t ldx, const void* w_codes_dev, const float* w_scales_dev,
                 uint64_t n, uint64_t k, const float* bias_dev, void* out_dev, int out_dtype, uint64_t ldo, void* workspace_dev,
                 uint64_t workspace_bytes, void* stream);

#ifdef __cplusplus
}
#endif
#endif /* TQ_I8_H */
