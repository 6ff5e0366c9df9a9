/*
 * hr_scores.h — C ABI of the operators around a matrix of scores [rows, n] on MI355X (gfx950): queries against candidates.
 *
 * What a retrieval service and the models on both sides of it do with such scores besides taking the k best of them
 * (hr_ivf.h): make them from rows kept in 8 bits (hr_i8_*), read a row as a distribution over its candidates
 * (hr_logprobs: how likely were the given ones, how sure is the row, what else was likely), and teach the model that
 * made them from another model's scores of a few candidates each (hr_distill_*; the lists of ids are those that
 * hr_ivf_search returns, empty places -1).  A row's candidates may as well be the entries of a vocabulary.
 *
 * Conventions are those of hr_ivf.h: DEV pointers on the current device, error codes, hr_last_error(); on any error but
 * HR_ERR_HIP nothing was enqueued.  The calls only enqueue kernels on `stream` (no allocation, no host synchronisation, no
 * memset or copy nodes: they can be captured in a HIP graph).  Matrices are row-major; `ld...` is the distance between rows in
 * elements, at least the row's length, so a matrix may be a slice of columns of a wider one.  Types are HR_F32 / HR_F16 /
 * HR_BF16, pointers aligned to their element; 16-byte alignment of pointers and rows is faster, not required.  Outputs must
 * not overlap inputs or each other, except where it says so.  Same inputs give bit-identical outputs.  Zero rows are a
 * no-op.  A workspace is DEV scratch, HR_WORKSPACE_ALIGN-aligned; two calls that overlap in time must not share one.
 */
#ifndef HR_SCORES_H
#define HR_SCORES_H

#include "hr_ivf.h"

#ifdef __cplusplus
extern "C" {
#endif

#define HR_I8_K_MAX 131071        /* longest rows of a product in 8 bits: 2^17 products of -128 x -128 no longer fit 32 bits */
#define HR_LIST_MAX 512           /* most given entries, or entries of a teacher's list, of a row */
#define HR_ROW_MAX (1 << 30)      /* longest row of scores */

/*
 * hr_i8_quantize — rows of x as 8-bit integers with a scale for each row:
 *   scale[i] = max_t |x[i, t]| / 127,   q[i, t] = x[i, t] / scale[i] rounded to the nearest whole number (even on ties),
 * both quotients rounded to float32 first, the whole number limited to -127 .. 127 (a scale below the smallest normal number has few
 * bits: of a row with magnitudes below 2.3e-41 the largest may be cut off, by a third at most).  A row whose scale is 0 becomes zeros; a
 * row with a NaN or an infinity becomes zeros with scale NaN, so that every score of it is NaN.
 *   x  DEV [m, k] in `dtype`;   q  DEV [m, k] int8, ldq >= k: the bytes behind a row, up to the next multiple of 64 or to the next
 *   row, are set to zero (ldq a multiple of 64 makes products fast);   scale  DEV [m] float32.
 */
int hr_i8_quantize(const void* x, int64_t ldx, int32_t dtype, int64_t m, int64_t k, int8_t* q, int64_t ldq, float* scale,
                   void* stream);

/* Bytes of workspace for hr_i8_product and hr_i8_linear of this shape; 0 on invalid arguments.  Enough for fewer rows a as well. */
size_t hr_i8_workspace_bytes(int64_t m, int64_t n, int64_t k);

/*
 * hr_i8_product — out[i, j] = (sum_t a[i, t] * b[j, t]) * a_scale[i] * b_scale[j] + bias[j].
 * The sum is exact (32-bit integers), the rest is float32 in this order, rounded once to out_dtype.
 *   a  DEV [m, k] int8, a_scale DEV [m]: queries or tokens;   b  DEV [n, k] int8, b_scale DEV [n]: candidate rows or channels;
 *   bias DEV [n] float32 or NULL;   out DEV [m, n] in out_dtype;   1 <= k <= HR_I8_K_MAX.
 * Where a pointer and its ld are multiples of 16, a row's bytes between k and the next multiple of 16 are read as well
 * (their values do not matter).
 */
int hr_i8_product(const int8_t* a, int64_t lda, const float* a_scale, const int8_t* b, int64_t ldb, const float* b_scale,
                  const float* bias, int64_t m, int64_t n, int64_t k, void* out, int64_t ldo, int32_t out_dtype,
                  void* workspace, size_t workspace_bytes, void* stream);

/* hr_i8_linear — hr_i8_quantize of x [m, k] (into the workspace), then hr_i8_product: the same bits. */
int hr_i8_linear(const void* x, int64_t ldx, int32_t x_dtype, const int8_t* b, int64_t ldb, const float* b_scale,
                 const float* bias, int64_t m, int64_t n, int64_t k, void* out, int64_t ldo, int32_t out_dtype,
                 void* workspace, size_t workspace_bytes, void* stream);

/*
 * hr_logprobs — rows of scores z read as distributions p = softmax(scale * z), 0 < scale <= 1e30 (the inverse temperature).
 *   logits   DEV [rows, n] in `dtype`, 1 <= n <= HR_ROW_MAX.  A score of -inf is no candidate: probability 0.  (The lowest finite value
 *            of the type is a candidate like any other: a row of nothing else is uniform.)
 *   given    DEV [rows, ngiven] int64 entries of the row, 0 <= ngiven <= HR_LIST_MAX (NULL if 0); outside 0..n-1 (-1): none.
 *   k        0 .. HR_K_MAX alternatives.
 *   out_logprobs      DEV [rows, ngiven] float32 or NULL if ngiven = 0: ln p of the given entries; -inf for none and for no candidate.
 *   out_entropy       DEV [rows] float32 or NULL: -sum p ln p.
 *   out_norm          DEV [rows, 2] float32 or NULL: (largest score, ln sum exp(scale * (z - largest))): what turns a score
 *                     into ln p = scale * (z - norm[0]) - norm[1] without losing either part.  Input of the backward call.
 *   out_top_ids       DEV [rows, k] int64, out_top_logprobs DEV [rows, k] float32 (NULL if k = 0): the k best candidates, best first,
 *                     equal scores by ascending entry; empty places -1 and -inf.
 * A row without candidates has entropy 0, norm (-inf, 0) and empty places.  A row with a NaN or +inf has no distribution: its
 * log probabilities (of candidates), entropy and norm[1] are NaN, its alternatives empty places with NaN.
 * Sums are kept in float32.
 */
size_t hr_logprobs_workspace_bytes(int64_t rows, int64_t n, int32_t k);   /* 0 on invalid arguments; enough for fewer rows and k as well */
int hr_logprobs(const void* logits, int64_t ld, int32_t dtype, int64_t rows, int64_t n, float scale, const int64_t* given,
                int32_t ngiven, int32_t k, float* out_logprobs, float* out_entropy, float* out_norm, int64_t* out_top_ids,
                float* out_top_logprobs, void* workspace, size_t workspace_bytes, void* stream);

/*
 * hr_logprobs_backward — gradient of a loss on the log probabilities of the given entries and on the entropy:
 *   grad[i] = scale * ( sum_g G_g ((i = given_g) - p_i) - H' p_i (ln p_i + H) ),   0 where the score is -inf.
 * Given entries that are none or no candidates take no part.
 *   entropy, norm   what hr_logprobs wrote (entropy may be NULL without grad_entropy);   grad_logprobs DEV [rows, ngiven] float32 or NULL (0) and grad_entropy DEV
 *   [rows] float32 or NULL (0): G and H';   grad_logits DEV [rows, n] in the type of logits, rounded once; may be logits itself (the
 *   same pointer and ld).  An entry given twice counts twice.
 */
int hr_logprobs_backward(const void* logits, int64_t ld, int32_t dtype, int64_t rows, int64_t n, float scale,
                         const int64_t* given, int32_t ngiven, const float* entropy, const float* norm, const float* grad_logprobs,
                         const float* grad_entropy, void* grad_logits, int64_t ldg, void* stream);

/*
 * hr_distill_* — a teacher's scores of k entries of every row teach the student that made the rows (forward Kullback-Leibler
 * divergence from the teacher's distribution over its entries to the student's over the whole row):
 *   q = softmax(scale * teacher) over the entries that count, p = softmax(scale * z),
 *   loss = sum_j q_j (ln q_j - ln p[ids_j]),    grad[i] = weight * scale * (p_i - sum of q_j with ids_j = i).
 * An entry counts if its id lies in 0..n-1 (-1: empty place), its teacher's score is above -inf and so is the student's.  A row
 * without any has loss 0 and gradient 0; so has the gradient of a row of weight 0, and a place whose score is -inf.
 *   ids DEV [rows, k] int64, teacher DEV [rows, k] float32, 1 <= k <= HR_LIST_MAX; an id listed twice counts twice.
 *   out_loss DEV [rows] float32 (not weighted).   out_norm DEV [rows, 2], out_q DEV [rows, k] float32: what the backward call needs.
 *   weights DEV [rows] float32 or NULL (1): the gradient of the caller's loss with respect to every row's.
 *   grad_logits as in hr_logprobs_backward (may be logits itself).
 * hr_distill_step is both calls in one, for a caller who knows the weights beforehand (a mean, masked rows): a row's scores are
 * read again while they are in registers and caches.  out_norm and out_q may be NULL there.
 */
size_t hr_distill_workspace_bytes(int64_t rows, int64_t n, int32_t k);    /* 0 on invalid arguments; enough for fewer rows and k as well */
int hr_distill_forward(const void* logits, int64_t ld, int32_t dtype, int64_t rows, int64_t n, float scale, const int64_t* ids,
                       const float* teacher, int32_t k, float* out_loss, float* out_norm, float* out_q, void* workspace,
                       size_t workspace_bytes, void* stream);
int hr_distill_backward(const void* logits, int64_t ld, int32_t dtype, int64_t rows, int64_t n, float scale, const int64_t* ids,
                        const float* q, int32_t k, const float* norm, const float* weights, void* grad_logits, int64_t ldg,
                        void* stream);
int hr_distill_step(const void* logits, int64_t ld, int32_t dtype, int64_t rows, int64_t n, float scale, const int64_t* ids,
                    const float* teacher, int32_t k, const float* weights, float* out_loss, float* out_norm, float* out_q,
                    void* grad_logits, int64_t ldg, void* workspace, size_t workspace_bytes, void* stream);

#ifdef __cplusplus
}
#endif
#endif /* HR_SCORES_H */
