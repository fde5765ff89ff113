/*
 * aed_vocab.h -- C ABI of the operators on rows of logits: sampling the next
 * token, a row's largest logits, and distillation from those of a teacher.
 *
 * Conventions are those of aed_train.h: dtype 0 float32 / 1 bfloat16; the
 * caller owns all memory, the library allocates none on the device; work is
 * enqueued on the stream given at create and calls return after enqueueing;
 * errors are aed_status codes found on the host before any launch, with a
 * message from aed_train_last_error(); the same calls give the same bits.
 * Calls are launches only, so they can be recorded in a graph.  A handle has no
 * memory on the device.  One handle = one stream = one host thread.
 *
 * Logits: DEVICE [rows, vocab] in dtype, aligned to their elements, row_stride
 * elements (>= vocab, at most 2^38) between rows; any vocab from 1 to 2^18,
 * else AED_EUNSUPPORTED; at most 2^22 - 1 rows a call, else AED_EUNSUPPORTED;
 * no rows: nothing is done.  Row r of any other tensor is at r times its
 * columns.  Outputs share no memory with inputs or each other, but where
 * said.
 * The order of a row: larger logits first, equal ones by rising id.  Logits of
 * minus infinity or NaN are not in it (ids that the caller takes out).
 */
#ifndef AED_VOCAB_H
#define AED_VOCAB_H

#include "aed_train.h"

#ifdef __cplusplus
extern "C" {
#endif

/* ---- sampling ----
 * Of row z with its largest logit z_max, temperature t, w_i = exp((z_i - z_max) / t):
 *     A    the first top_k of the order (all, if top_k is 0 or at least vocab)
 *     B    those of A in front of which less than top_p of A's sum of w lies (all, if top_p is 1)
 *     C    those of B with w_i >= min_p
 *     token  the least id for which the sum of w over the ids up to it in C is above u times C's sum
 *     logp   log(w_token / C's sum), float32
 * The first of the order is always in C; t = 0 leaves it alone (logp 0).  Sums
 * are of whole multiples of 2^-44 or finer (2^-50 for a vocab of 4096), in 64
 * bits, so no order of adding changes a token; what is below that is not
 * drawn.  A row without any logit in the order: token -1, logp minus infinity. */
typedef struct aed_sampler aed_sampler; /* opaque */

typedef struct aed_sampler_config {
    uint32_t struct_size;  /* = sizeof(aed_sampler_config) */
    int32_t vocab, dtype;
} aed_sampler_config;

typedef struct aed_sampling {
    uint32_t struct_size;  /* = sizeof(aed_sampling) */
    int32_t top_k;         /* >= 0 */
    float temperature;     /* finite, >= 0 */
    float top_p, min_p;    /* in [0, 1] */
    /* DEVICE [rows], each NULL or in the place of the number above.  What is out of its range counts as: temperature
     * not above 0: 0; top_k below 0: 0; top_p not below 1: 1, below 0: 0; min_p not above 0: 0, above 1: 1. */
    const float *temperatures;
    const int32_t *top_ks;
    const float *top_ps, *min_ps;
} aed_sampling;

/* Errors: AED_EINVAL (NULL, struct_size, vocab < 1, dtype), AED_EUNSUPPORTED. */
aed_status aed_sampler_create(const aed_sampler_config *cfg, void *hip_stream, aed_sampler **out);
/* Waits for the stream.  NULL is allowed. */
aed_status aed_sampler_destroy(aed_sampler *plan);

/* uniforms: DEVICE float32[rows], in [0, 1) (others, and NaN, count as the nearer end, NaN as 0); tokens: DEVICE int32[rows];
 * logp: DEVICE float32[rows].
 * Errors: AED_EINVAL (NULL, alignment, row_stride, rows < 0, a number out of its range), AED_EUNSUPPORTED, AED_EHIP. */
aed_status aed_sample(aed_sampler *plan, const void *logits, int64_t row_stride, int32_t rows, const float *uniforms,
                      const aed_sampling *how, int32_t *tokens, float *logp);

/* ---- a row's largest logits ----
 * values, ids: the first `top` of the order; where the row has fewer: minus
 * infinity and -1.  rest = log of the sum of exp(z_i / temperature) over all
 * others of the order, minus infinity if there are none. */
typedef struct aed_top aed_top; /* opaque */

typedef struct aed_top_config {
    uint32_t struct_size;  /* = sizeof(aed_top_config) */
    int32_t vocab, dtype;
    int32_t top;           /* 1 to 128, at most vocab */
    float temperature;     /* 1e-20 to 1e20 */
} aed_top_config;

/* Errors: AED_EINVAL (NULL, struct_size, vocab, dtype, top, temperature not above 0 or not finite), AED_EUNSUPPORTED (vocab; top above 128; other temperatures). */
aed_status aed_top_create(const aed_top_config *cfg, void *hip_stream, aed_top **out);
aed_status aed_top_destroy(aed_top *plan);
/* values: DEVICE float32[rows, top]; ids: DEVICE int32[rows, top]; rest: DEVICE float32[rows]. */
aed_status aed_top_logits(aed_top *plan, const void *logits, int64_t row_stride, int32_t rows, float *values, int32_t *ids, float *rest);

/* ---- distillation ----
 * A teacher's list of row r: logits v_k of the ids i_k, and, with `rest`, the
 * log of the sum of exp(its logits / T) over all other ids (aed_top_logits
 * gives both); T = temperature.  Entries with an id outside [0, vocab) or a
 * value of minus infinity are left out.  The student's logits z:
 *     q_k = exp(v_k / T) / n,  n = sum_k exp(v_k / T) [+ exp(rest);  q_R = exp(rest) / n]
 *     p = softmax(z / T);  p_R: p's sum over the ids that are not in the list
 *     L_r  = T^2 (sum_k q_k log(q_k / p_(i_k)) [+ q_R log(q_R / p_R)])      0 log 0 = 0
 *     loss = sum_r weight_r L_r
 *     d loss / d z_i = weight_r T (p_i - q's sum over the entries of id i)  for ids in the list
 *                    = weight_r T p_i (1 - q_R / p_R)                       for others (without rest: q_R = 0)
 * An id may stand in a list more than once.  A row of weight 0 has L_r 0 and
 * gradient 0, whatever its logits and list hold, and so has one with neither
 * an entry nor a finite rest.  Student's logits of minus infinity have p = 0 (L_r is
 * infinite where q is not 0 there); NaN and plus infinity, the student's, an
 * entry's or, beside an entry, the rest's, give NaN.  p's sums are float32:
 * L_r is good to some 2^-22 T^2. */
typedef struct aed_distill aed_distill; /* opaque */

typedef struct aed_distill_config {
    uint32_t struct_size;  /* = sizeof(aed_distill_config) */
    int32_t vocab, dtype;
    int32_t top;           /* entries of a list, 1 to 128; may be more than vocab */
    float temperature;     /* 1e-20 to 1e20 */
} aed_distill_config;

aed_status aed_distill_create(const aed_distill_config *cfg, void *hip_stream, aed_distill **out);
aed_status aed_distill_destroy(aed_distill *plan);

/* values: DEVICE float32[rows, top]; ids: DEVICE int32[rows, top]; rest: DEVICE float32[rows] or NULL (the list alone adds up to one); weights: DEVICE
 * float32[rows] or NULL (1 / rows each); loss: DEVICE float32[1] (0 without rows); row_loss: DEVICE float32[rows]; stats: DEVICE float32[rows, top + 2], for
 * aed_distill_backward.
 * Errors: AED_EINVAL (NULL, alignment, row_stride, rows < 0), AED_EUNSUPPORTED, AED_EHIP. */
aed_status aed_distill_forward(aed_distill *plan, const void *logits, int64_t row_stride, int32_t rows, const float *values, const int32_t *ids,
                               const float *rest, const float *weights, float *loss, float *row_loss, float *stats);

/* logits, ids, weights, stats: aed_distill_forward's.  d_logits: [rows, vocab] in dtype, d_row_stride elements between rows; may be the
 * logits themselves.  d_loss: DEVICE float32[1], the gradient by the loss, or NULL = 1. */
aed_status aed_distill_backward(aed_distill *plan, const void *logits, int64_t row_stride, int32_t rows, const int32_t *ids, const float *weights,
                                const float *stats, const float *d_loss, void *d_logits, int64_t d_row_stride);

#ifdef __cplusplus
}
#endif
#endif
