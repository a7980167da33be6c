/*
 * tq_norm.h -- layer norm on AMD MI355X (gfx950): forward and backward pass, with the gradients of weight and bias.
 *
 * For each row of x [rows, cols], sums over its elements:
 *     m = mean(x),   r = 1 / sqrt(mean((x - m)^2) + eps),   h = (x - m) r,   y = h * weight + bias,
 * and with dy the gradient of y, g = dy * weight:
 *     dx = r (g - mean(g) - h mean(g h)),   dweight = sum over rows of dy h,   dbias = sum over rows of dy.
 * Conventions as in tq.h, but that matrices need only be aligned to an element: *_dev are device pointers owned by the caller,
 * calls enqueue and return, nothing is allocated or kept, nothing is enqueued on error.
 *
 *   x_dev, y_dev, dy_dev, dx_dev   [rows] rows of `cols` elements of `dtype` (TQ_F32, TQ_BF16 or TQ_F16), ld* >= cols elements
 *               from row to row
 *   weight_dev, bias_dev   [cols] of wtype; NULL for ones, or for zeros
 *   stats_dev   [rows][2] floats: m and r of each row, which the backward pass takes
 *   eps         at least 1e-30, finite
 * rows, cols = 1 .. 2^31 - 1, rows * ld* <= 2^40.
 *
 * Sums are binary32, along rows of more than 32768 columns binary64, of x around a first estimate of its mean, so that a mean far
 * larger than the deviations costs no bits of those, in either pass: the h that follows in the backward pass from m, which is one
 * binary32 number, has its own mean taken out.
 * Rows of any finite values have their result, also where squares would leave the range of binary32.  A row that holds a
 * NaN or an infinity has NaN for r and for all of y, dx, and, through them, dweight; no other row does.  A row of equal elements has h = 0.
 * The same call on the same device gives the same bits every time.
 */
#ifndef TQ_NORM_H
#define TQ_NORM_H

#include "tq_mx.h"

#ifdef __cplusplus
extern "C" {
#endif

/*
 * tq_layernorm_forward
 *   y_dev       may be x_dev (with ldy = ldx); otherwise apart from it
 *   stats_dev   NULL if not wanted
 */
int tq_layernorm_forward(const void* x_dev, int dtype, uint64_t rows, uint64_t cols, uint64_t ldx, const void* weight_dev,
                         const void* bias_dev, int wtype, float eps, void* y_dev, uint64_t ldy, float* stats_dev, void* stream);

/*
 * tq_layernorm_backward
 *   dx_dev      NULL if not wanted; may be dy_dev (with lddx = lddy) or x_dev (with lddx = ldx), otherwise apart from them
 *   dweight_dev, dbias_dev   [cols] floats, each NULL if not wanted
 *   accumulate  0: dweight, dbias = result; 1: += result, the finished sums added once
 *   workspace_dev   at least tq_layernorm_workspace_bytes(rows, cols) bytes, 16-byte aligned, contents undefined afterwards; calls that
 *               share it have to be ordered.  NULL where neither dweight nor dbias is wanted.
 */
uint64_t tq_layernorm_workspace_bytes(uint64_t rows, uint64_t cols);
int tq_layernorm_backward(const void* x_dev, int dtype, uint64_t rows, uint64_t cols, uint64_t ldx, const void* dy_dev,
                          uint64_t lddy, const void* weight_dev, int wtype, const float* stats_dev, void* dx_dev, uint64_t lddx,
                          float* dweight_dev, float* dbias_dev, int accumulate, void* workspace_dev, uint64_t workspace_bytes,
                          void* stream);

#ifdef __cplusplus
}
#endif
#endif /* TQ_NORM_H */
