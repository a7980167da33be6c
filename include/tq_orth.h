/*
 * tq_orth.h -- orthogonalised updates of matrices on AMD MI355X (gfx950): the server's step of tq_decompress_aggregate_update for a
 *              layer whose momentum is replaced by the nearest matrix with orthogonal rows (or columns).
 *
 * Newton-Schulz steps on U [rows, cols]: X = U / (|U|_F + eps), transposed where rows > cols, and `steps` times
 *     A = X X^T,   X <- (a I + b A + c A A) X,
 * transposed back: an odd polynomial of U's singular values, which drives all that are not small to about 1.
 * Conventions as in tq.h, but that matrices need only be aligned to an element.  Matrices whose rows follow each other directly, any
 * size; a layer's part of a flat gradient or parameter vector is one.
 *
 *   rows, cols     1 .. TQ_ORTH_MAX_LENGTH, the smaller of them at most TQ_ORTH_MAX_SIDE
 *   count          1 .. TQ_ORTH_MAX_COUNT matrices of one shape in one call; *_host are host arrays of `count` device pointers.  Results
 *                  are those of `count` calls, up to the order of a product's sums.
 *   steps          1 .. TQ_ORTH_MAX_STEPS
 *   coefficients_host   [steps][3] floats a, b, c of each step, or NULL: 3.4445, -4.7750, 2.0315 for all of them.  The polynomials have
 *                  to keep singular values that begin in [0, 1] within [-3, 3], and |a + b s^2 + c s^4| within 12 on the way;
 *                  others are refused (TQ_EINVAL), for the products' operands have a fixed range.
 *   precision      TQ_ORTH_SPLIT: operands of the products are held as the sum of two binary16 numbers, 22 bits, with 32-bit sums: the
 *                  accuracy of binary32 arithmetic.  TQ_ORTH_HALF: as one binary16 number, at a third of the multiplications: each
 *                  rounding is 2^-12 of the matrix (in its 2-norm, evenly over all directions), which steps that lift small singular
 *                  values lift with them.  For matrices of random numbers the result is 1.1e-3 to 1.4e-3 of its norm off, less than
 *                  a bf16 result's own rounding (1.7e-3) but six times an fp16 result's (2e-4), beside which that of TQ_ORTH_SPLIT does not show;
 *                  where directions that are k times below the largest matter, k times as much relative to those.
 *                  Either way an element of X below 2^-26 has fewer bits, and one below 2^-37 none: a matrix with |U|_F below
 *                  about 2^-20 eps loses what eps left of it.
 *   eps            at least 1e-30, finite
 *   workspace_dev  at least tq_orthogonalize_workspace_bytes(rows, cols, count, precision) bytes, 16-byte aligned, contents undefined
 *                  afterwards; calls that share it have to be ordered
 * A matrix of zeros gives zeros; one that holds a NaN or an infinity gives NaN throughout.  |U|_F is summed in 64 bits.  The same call
 * on the same device gives the same bits every time.
 */
#ifndef TQ_ORTH_H
#define TQ_ORTH_H

#include "tq_mx.h"

#ifdef __cplusplus
extern "C" {
#endif

#define TQ_ORTH_MAX_LENGTH (1 << 21)
#define TQ_ORTH_MAX_SIDE 32768
#define TQ_ORTH_MAX_COUNT 64
#define TQ_ORTH_MAX_STEPS 16
enum { TQ_ORTH_HALF = 0, TQ_ORTH_SPLIT = 1 };          /* precision */

/* 0 for sizes that the calls refuse. */
uint64_t tq_orthogonalize_workspace_bytes(uint64_t rows, uint64_t cols, int count, int precision);

/*
 * tq_orthogonalize -- out = the steps' result for g.
 *   g_dev     [rows][cols] of TQ_F32, TQ_BF16 or TQ_F16
 *   out_dev   [rows][cols] of out_dtype; may be g_dev if the types are the same, otherwise apart from all g
 */
int tq_orthogonalize(const void* g_dev, int dtype, uint64_t rows, uint64_t cols, int steps, const float* coefficients_host,
                     int precision, float eps, void* out_dev, int out_dtype, void* workspace_dev, uint64_t workspace_bytes,
                     void* stream);
int tq_orthogonalize_multi(const void* const* g_host, int count, int dtype, uint64_t rows, uint64_t cols, int steps,
                           const float* coefficients_host, int precision, float eps, void* const* out_host, int out_dtype,
                           void* workspace_dev, uint64_t workspace_bytes, void* stream);

/*
 * tq_orthogonal_update -- momentum, orthogonalisation and the new parameters:
 *     v' = momentum * v + g,   U = nesterov ? g + momentum * v' : v',   O = the steps' result for U,
 *     theta' = theta - eta * (scale * O + weight_decay * theta)
 * in binary32, each product and sum rounded once, O not rounded before it is used.
 *   g_dev          [rows][cols] of TQ_F32, TQ_BF16 or TQ_F16: what tq_decompress_aggregate leaves for this layer, say
 *   velocity_dev, theta_dev           [rows][cols] floats
 *   velocity_out_dev, theta_out_dev   where v' and theta' go: the same buffers (updated in place) or others, apart from all else
 *   eta, momentum, weight_decay, scale   finite
 */
int tq_orthogonal_update(const void* g_dev, int dtype, uint64_t rows, uint64_t cols, float eta, float momentum, int nesterov,
                         float weight_decay, float scale, int steps, const float* coefficients_host, int precision, float eps,
                         const float* velocity_dev, float* velocity_out_dev, const float* theta_dev, float* theta_out_dev,
                         void* workspace_dev, uint64_t workspace_bytes, void* stream);
int tq_orthogonal_update_multi(const void* const* g_host, int count, int dtype, uint64_t rows, uint64_t cols, float eta, float momentum,
                               int nesterov, float weight_decay, float scale, int steps, const float* coefficients_host, int precision,
                               float eps, const float* const* velocity_host, float* const* velocity_out_host,
                               const float* const* theta_host, float* const* theta_out_host, void* workspace_dev,
                               uint64_t workspace_bytes, void* stream);

#ifdef __cplusplus
}
#endif
#endif /* TQ_ORTH_H */
