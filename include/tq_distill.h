/*
 * tq_distill.h -- distillation from a teacher's top logits on AMD MI355X (gfx950): loss and gradient.
 *
 * For each row: z [vocab] the student's logits, (ids, t) [top] the teacher's largest logits and their places,
 *     p = softmax of t / tau over the row's present entries,   q = softmax of z / tau over the whole vocabulary,
 *     loss = tau^2 sum_i p_i (ln p_i - ln q_{ids_i}),          dz_j = tau * grad * (q_j - sum_{i: ids_i = j} p_i),
 * tau the temperature and `grad` what the program above hands down for that row's loss (a mask, a weight, 1 / rows).  The
 * factor tau^2 keeps the gradient's size when tau changes.  Conventions as in tq.h.
 *
 *   z_dev     [rows][ldz] of TQ_F32, TQ_BF16 or TQ_F16, aligned to an element; ldz >= vocab
 *   ids_dev   [rows][top] of int32 (ids_bytes = 4) or int64 (8).  An entry is absent if its id is not in [0, vocab) or its
 *             logit is -inf.  An id may occur twice: in the gradient its probabilities add up.  The loss is the sum over the
 *             entries as it stands above, ln p_i of each entry alone: below the divergence of the added probabilities by
 *             tau^2 sum_i p_i ln(P_i / p_i), P_i the sum of what shares entry i's id, so that it can be negative.  That does not
 *             depend on z: the gradient is the loss's.
 *   t_dev     [rows][top] floats
 *   loss_dev, grad_dev   [rows] floats
 *   stats_dev   [rows][2] floats: the row's largest logit M and ln sum_j exp((z_j - M) / tau).  Apart, because their sum
 *             M / tau + ln(...) has no bits left for the second where a mask made every logit the type's lowest value.
 *   dz_dev    [rows][lddz], of z's type; may be z_dev (with lddz = ldz)
 * top = 1 .. TQ_DISTILL_MAX_TOP; rows, vocab = 1 .. 2^31 - 1, rows * ldz and rows * lddz <= 2^40; 0 < temperature <= 1e4,
 * at least 1e-4.
 *
 * A row with no entry present has loss 0 and gradient 0, whatever its logits.  A row with grad 0 has gradient 0.  A student's
 * logit of -inf has q = 0 (its loss is infinite where the teacher has p > 0, its gradient is not).  NaN and +inf among the
 * student's logits, or NaN and +inf among the teacher's present ones, make the row's loss and gradient NaN.
 * Sums and statistics are binary32, results do not depend on anything but the arguments.
 */
#ifndef TQ_DISTILL_H
#define TQ_DISTILL_H

#include "tq_mx.h"

#ifdef __cplusplus
extern "C" {
#endif

#define TQ_DISTILL_MAX_TOP 1024

/* The loss, and the statistics that tq_distill_backward takes.  Reads z once. */
int tq_distill_forward(const void* z_dev, int dtype, uint64_t rows, uint64_t vocab, uint64_t ldz, const void* ids_dev,
                       int ids_bytes, const float* t_dev, uint64_t top, float temperature, float* loss_dev, float* stats_dev,
                       void* stream);

/* The gradient, from the statistics of the forward call.  Reads z once and writes dz once. */
int tq_distill_backward(const void* z_dev, int dtype, uint64_t rows, uint64_t vocab, uint64_t ldz, const void* ids_dev,
                        int ids_bytes, const float* t_dev, uint64_t top, float temperature, const float* stats_dev,
                        const float* grad_dev, void* dz_dev, uint64_t lddz, void* stream);

/* Both at once, for a program that knows grad beforehand: z is read from memory once. */
int tq_distill(const void* z_dev, int dtype, uint64_t rows, uint64_t vocab, uint64_t ldz, const void* ids_dev, int ids_bytes,
               const float* t_dev, uint64_t top, float temperature, const float* grad_dev, float* loss_dev, void* dz_dev,
               uint64_t lddz, void* stream);

#ifdef __cplusplus
}
#endif
#endif /* TQ_DISTILL_H */
