/*
 * aed_train.h -- C ABI of the operators next to the decoder step that scoring
 * and training need: attention of ragged batches with many rows a sequence
 * (forward and backward, cross- and self-attention, learned relative position
 * bias) and the preference loss on pairs of transcripts.
 *
 * Conventions are those of aed.h: row-major, dtype 0 float32 / 1 bfloat16,
 * scores, softmax, statistics and sums in float32; the caller owns all memory,
 * the library allocates none on the device; lengths are HOST arrays that are read
 * by create; work is enqueued on the stream given at create and calls return
 * after enqueueing; errors are aed_status codes found on the host before any
 * launch; the same calls give the same bits.
 *
 * A handle belongs to one batch's lengths and is kept for all layers and for
 * forward and backward: create copies its work lists into the workspace.  Its
 * calls are launches only (no allocation, copy or wait), so they can be
 * recorded in a graph (the handle and its workspace outlive it).  One handle =
 * one stream = one host thread.
 */
#ifndef AED_TRAIN_H
#define AED_TRAIN_H

#include "aed.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Message of the calling thread's most recent failed call of this header. */
const char *aed_train_last_error(void);

/* ---- attention ----
 * Sequence b has q_lens[b] query rows and k_lens[b] keys, both any number
 * from 0 on.  Query rows are packed in batch order.  Keys are packed too, or
 * begin at row k_starts[b] of a longer tensor (a cache of fixed capacity per
 * sequence, frames that several sequences share).
 *     s_ij = scale q_i . k_j + bias[bucket(i + k_len - q_len - j)][head]
 *     p    = softmax over the keys that row i sees;  out_i = sum_j p_ij v_j
 *     lse_i = log sum_j exp s_ij
 * Row i sees key j unless key_mask has a zero for it or (causal) j > i +
 * k_len - q_len: the last query row stands at the last key.  A row that sees
 * nothing has output 0, lse -inf and adds nothing to any gradient.  Keys and
 * values that are masked or beyond a length are never used, whatever they hold.
 * (by key_mask; what a causal row does not see has weight 0 and has to be
 * finite, and so have the queries and gradients of rows that see nothing.)
 * Heads: query head h reads key head h / (n_heads / n_kv_heads).
 * With bfloat16 tensors the weights p are rounded to bfloat16 where they enter
 * the products with v and d_out, and their gradients where they enter those
 * with q (16 bits in those with k, and in small batches of few rows).  Against
 * exact arithmetic, in the 2-norm: outputs 0.002, dk and dv 0.0024; dq and
 * d_bias have the 0.0017 of their own rounding (dq more where more than 128
 * keys and no bias meet very sharp attention). */
typedef struct aed_attn aed_attn; /* opaque */

typedef struct aed_attn_config {
    uint32_t struct_size;          /* = sizeof(aed_attn_config) */
    int32_t n_heads, n_kv_heads;   /* n_kv_heads divides n_heads */
    int32_t head_dim;              /* 64 or 128 */
    int32_t dtype;                 /* 0 float32, 1 bfloat16 */
    int32_t causal;
    int32_t bias_buckets;          /* rows of the bias table; 0: no bias.  At most 256 */
    int32_t bias_max_distance;     /* distances from here on share a bucket; at most 1024 */
    int32_t bias_bidirectional;    /* 0: keys behind the query's place have bucket 0's bias.  1: they have the second
                                      half of the table (bias_buckets even) by their distance */
    int32_t training;              /* 1: aed_attn_backward will be called (packed keys only) */
    float scale;                   /* 0: 1 / sqrt(head_dim) */
} aed_attn_config;
/* Buckets of a side (all of the table, or half of it): with half = side / 2,
 * distances below half have a bucket each; bucket half + i begins at the first
 * distance n with (n / half)^(side - half) >= (bias_max_distance / half)^i.  A
 * side has 2 buckets or more and bias_max_distance > half.
 * An entry of minus infinity takes its pairs out, as the masks do; finite ones
 * beyond 2.35e38 in size count as that.  Weights add up to one whatever the
 * size of a row's bias, forward and backward. */

/* Rows of n_heads (or n_kv_heads) vectors of head_dim elements: element (row,
 * head, c) at data + row * row_stride + head * head_stride + c, strides in
 * elements.  DEVICE pointer, aligned to 16 bytes, strides multiples of 16
 * bytes, not negative and at most 2^38 (0 in an input: the same vector for
 * all; vectors of an output share no element), rows less than 16 MiB apart
 * (else AED_EUNSUPPORTED).  A part of a wider product's result is given by its strides, without a copy. */
typedef struct aed_rows {
    void *data;
    int64_t row_stride, head_stride;
} aed_rows;

/* Bytes of device workspace for a batch of these lengths.
 * Errors: AED_EINVAL (NULL, struct_size, a negative length or start, a start
 * above 2^38, batch < 1, heads, flags, a bias that the rule above does not
 * allow, training with k_starts), AED_EUNSUPPORTED (head_dim, buckets or distance above the limits,
 * more than 2^31 - 1 rows or keys, more than 2^24 - 1 workgroups in a launch:
 * items of 128 rows or keys of a sequence, 64 in small batches, 32 where no
 * sequence has more rows, times heads). */
aed_status aed_attn_workspace_bytes(const aed_attn_config *cfg, const int32_t *q_lens, const int32_t *k_lens,
                                    const int64_t *k_starts /*or NULL*/, int32_t batch, size_t *bytes);

/* workspace: DEVICE, 256-byte aligned; it and the stream outlive the handle.
 * Errors: as above, AED_EINVAL for the workspace, AED_EHIP. */
aed_status aed_attn_create(const aed_attn_config *cfg, const int32_t *q_lens, const int32_t *k_lens, const int64_t *k_starts,
                           int32_t batch, void *workspace, size_t workspace_bytes, void *hip_stream, aed_attn **out);
/* Waits for the stream.  NULL is allowed. */
aed_status aed_attn_destroy(aed_attn *plan);

/* bias: DEVICE [bias_buckets, n_heads] in dtype, contiguous, NULL iff there is
 * none; key_mask: DEVICE uint8 by key row (where the keys' rows are, with
 * k_starts), 0 = not seen, or NULL; out: as q, not overlapping an input; lse:
 * DEVICE float32 [query rows, n_heads].
 * Errors: AED_EINVAL (NULL, alignment, strides), AED_EHIP. */
aed_status aed_attn_forward(aed_attn *plan, const aed_rows *q, const aed_rows *k, const aed_rows *v, const void *bias,
                            const uint8_t *key_mask, const aed_rows *out, float *lse);

/* Gradients of a loss from d_out, that by out.  out and lse are aed_attn_forward's.
 * dq, dk, dv: as q, k, v (heads that share a key head are summed); d_bias:
 * [bias_buckets, n_heads] in dtype, NULL iff there is no bias.  All are
 * written whole, not added to.
 * Errors: AED_ESTATE (the handle is not for training), AED_EINVAL, AED_EHIP. */
aed_status aed_attn_backward(aed_attn *plan, const aed_rows *d_out, const aed_rows *q, const aed_rows *k, const aed_rows *v,
                             const aed_rows *out, const float *lse, const void *bias, const uint8_t *key_mask,
                             const aed_rows *dq, const aed_rows *dk, const aed_rows *dv, void *d_bias);

/* ---- preference loss ----
 * 2 n_pairs sequences of logits rows, packed: the preferred transcript of
 * pair 0, the other one of pair 0, the preferred one of pair 1, ...
 *     ratio_s = sum over the scored rows t of s of (log softmax(z_t)[label_t] - ref_logp_t)
 *     x_p     = beta (ratio_2p - ratio_2p+1)
 *     loss    = mean over pairs of -(1 - label_smoothing) log sigmoid(x_p) - label_smoothing log sigmoid(-x_p)
 * A row is scored if its label is in [0, vocab); others add nothing and have
 * gradient 0.  ref_logp is the frozen model's log-probability of the label. */
typedef struct aed_preference aed_preference; /* opaque */

typedef struct aed_preference_config {
    uint32_t struct_size;   /* = sizeof(aed_preference_config) */
    int32_t vocab;          /* any number from 1 on */
    int32_t dtype;          /* of the logits: 0 float32, 1 bfloat16 */
    float beta;             /* > 0 */
    float label_smoothing;  /* in [0, 0.5) */
} aed_preference_config;

/* seq_lens: HOST int32[2 n_pairs], rows of every sequence, 0 or more.
 * Errors: AED_EINVAL, AED_EUNSUPPORTED (more than 2^26 - 4 rows). */
aed_status aed_preference_workspace_bytes(const aed_preference_config *cfg, const int32_t *seq_lens, int32_t n_pairs, size_t *bytes);
aed_status aed_preference_create(const aed_preference_config *cfg, const int32_t *seq_lens, int32_t n_pairs, void *workspace,
                                 size_t workspace_bytes, void *hip_stream, aed_preference **out);
aed_status aed_preference_destroy(aed_preference *plan);

/* logits: DEVICE [rows, vocab], row_stride elements between rows (>= vocab);
 * labels: DEVICE int32[rows]; ref_logp: DEVICE float32[rows]; loss: DEVICE
 * float32[1]; ratio: DEVICE float32[2 n_pairs]; lse: DEVICE float32[rows][2],
 * of a scored row its largest logit m and log sum exp(z - m), 0 of others.
 * Errors: AED_EINVAL (NULL, a pointer not aligned to its type, row_stride), AED_EHIP. */
aed_status aed_preference_forward(aed_preference *plan, const void *logits, int64_t row_stride, const int32_t *labels,
                                  const float *ref_logp, float *loss, float *ratio, float *lse);

/* d_logits: [rows, vocab] in the logits' type, d_row_stride elements between rows; may be the logits themselves, otherwise apart from them.
 * ratio and lse are aed_preference_forward's; d_loss: DEVICE float32[1], the gradient by the loss, or NULL = 1. */
aed_status aed_preference_backward(aed_preference *plan, const void *logits, int64_t row_stride, const int32_t *labels,
                                   const float *ratio, const float *lse, const float *d_loss, void *d_logits, int64_t d_row_stride);

#ifdef __cplusplus
}
#endif
#endif
