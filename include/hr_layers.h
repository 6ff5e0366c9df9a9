/*
 * hr_layers.h — C ABI of what an encoder or a reader is made of and taught with, on MI355X (gfx950): layer norm, the gated half of a
 * feed-forward block, both with their gradients, and the step that updates parameters (AdamW).
 *
 * They stand between a search (hr_ivf.h) and the loss that its lists give (hr_scores.h): a batch of questions goes through layers of norms and
 * gated blocks to the vectors that are searched with; hr_distill_step gives the gradient at the scores, the ..._backward
 * calls here take it back through the layers, hr_adamw takes the step.
 *
 * Conventions are those of hr_scores.h: DEV pointers on the current device, row-major matrices with the distance between rows in elements, types
 * HR_F32 / HR_F16 / HR_BF16, error codes and hr_last_error(), nothing enqueued on any error but HR_ERR_HIP, kernels only (no allocation, no
 * host synchronisation, no memset or copy nodes; capture in a HIP graph is fine), bit-identical results for the same inputs.  Outputs must not
 * overlap inputs or each other, except where it says so.  Of 16-bit rows that begin or end inside an aligned word of 4 bytes the whole word may be read; what is
 * not the row's is not used, and may be written meanwhile.  Zero rows are a no-op, but for gradients that sum over rows: those are zeros.
 */
#ifndef HR_LAYERS_H
#define HR_LAYERS_H

#include "hr_scores.h"

#ifdef __cplusplus
extern "C" {
#endif

/*
 * hr_layer_norm — rows of x with their mean and spread taken out, scaled and shifted:
 *   mean = sum x / n,  rstd = 1 / sqrt(sum (x - mean)^2 / n + eps),  out[i, j] = (x[i, j] - mean[i]) * rstd[i] * weight[j] + bias[j].
 *   x        DEV [rows, n] in `dtype`, 1 <= n <= HR_ROW_MAX.   eps  >= 0, finite.
 *   weight, bias  DEV [n] in `weight_dtype`, HR_F32 or `dtype`; NULL: 1 and 0.
 *   out      DEV [rows, n] in `dtype`, rounded once; may be x itself (the same pointer and ld).
 *   out_stats  DEV [rows, 2] float32 or NULL: mean and rstd, what the backward call needs.
 * A row with a NaN or an infinity becomes NaN; a row without spread has no result where eps is 0.  Sums are kept in float32.
 */
int hr_layer_norm(const void* x, int64_t ldx, int32_t dtype, int64_t rows, int64_t n, const void* weight, const void* bias,
                  int32_t weight_dtype, float eps, void* out, int64_t ldo, float* out_stats, void* stream);

/*
 * hr_layer_norm_backward — with u = (x - mean) * rstd and g = grad_out * weight:
 *   grad_x = rstd * (g - sum g / n - u * sum(g u) / n)  (sums over a row),   grad_weight = sum grad_out * u,   grad_bias = sum grad_out  (over the rows).
 *   stats    what hr_layer_norm wrote.   weight  as there (NULL: 1).
 *   grad_x   DEV [rows, n] in `dtype`, or NULL: not wanted; may be grad_out itself (the same pointer and ld).
 *   grad_weight, grad_bias  DEV [n] in `weight_dtype`, each NULL where it is not wanted; overwritten, rounded once.
 *   workspace  DEV scratch of hr_layer_norm_workspace_bytes, HR_WORKSPACE_ALIGN-aligned.
 */
size_t hr_layer_norm_workspace_bytes(int64_t rows, int64_t n);       /* 0 on invalid arguments; enough for fewer rows as well */
int hr_layer_norm_backward(const void* x, int64_t ldx, int32_t dtype, int64_t rows, int64_t n, const void* weight, int32_t weight_dtype,
                           const float* stats, const void* grad_out, int64_t ldg, void* grad_x, int64_t ldgx, void* grad_weight,
                           void* grad_bias, void* workspace, size_t workspace_bytes, void* stream);

#define HR_SILU 0            /* z / (1 + exp(-z)) */
#define HR_GELU 1            /* z * (1 + erf(z / sqrt 2)) / 2 */
#define HR_GELU_TANH 2       /* z * (1 + tanh(sqrt(2 / pi) * (z + 0.044715 z^3))) / 2 */

#define HR_GATED_MAX (1 << 19)       /* largest m, k and f */

/*
 * hr_gated — the gated half of a feed-forward block, one pass over x and over both matrices:
 *   out[i, j] = act(gate[i, j]) * up[i, j],   gate = x w_gate', up = x w_up'.
 *   x       DEV [m, k];   w_gate, w_up  DEV [f, k] (halves of one [2 f, k] matrix, or two);   out  DEV [m, f]; all in `dtype`.
 *   out_pre DEV [m, 2, f] float32 or NULL: gate and up of every row, what the backward call needs.
 * Products are summed in float32, act and its product with up taken in float32, out rounded once.
 *   1 <= k, f <= HR_GATED_MAX, 0 <= m <= HR_GATED_MAX; HR_ERR_UNSUPPORTED where [m, 2 f], [2 f, k] and [m, k] together have about 2^36 elements or more.
 */
size_t hr_gated_workspace_bytes(int64_t m, int64_t k, int64_t f, int32_t dtype);       /* 0 on invalid arguments; enough for fewer rows as well; has room for copies of rows at odd places */
int hr_gated(const void* x, int64_t ldx, const void* w_gate, int64_t ldwg, const void* w_up, int64_t ldwu, int32_t dtype, int64_t m, int64_t k,
             int64_t f, int32_t activation, void* out, int64_t ldo, float* out_pre, void* workspace, size_t workspace_bytes, void* stream);

/*
 * hr_gated_backward — with d_up = grad_out * act(gate) and d_gate = grad_out * up * act'(gate), both rounded to as many bits as `dtype` has once, for the
 * matrix instructions that take them:
 *   grad_x = d_gate w_gate + d_up w_up,   grad_w_gate = d_gate' x,   grad_w_up = d_up' x.
 *   pre   DEV [m, 2, f] float32, as hr_gated wrote it.   grad_out  DEV [m, f] in `dtype`.
 * (The rounding is as large as that of the result: together they are 1.4 times as far off as one of them.)
 * In binary16 each row of d_gate and d_up (for grad_x) and each column (for the matrices) is held times a power of two, so that they may be of any size that
 * float32 has: only the results have to fit the type.  What is less than 2^-28 of the largest of its row (column) has fewer bits, below 2^-40 none.
 *   grad_x  DEV [m, k] or NULL: not wanted.   grad_w_gate, grad_w_up  DEV [f, k], both or neither (NULL); overwritten; all in `dtype`, rounded once.
 */
size_t hr_gated_backward_workspace_bytes(int64_t m, int64_t k, int64_t f, int32_t dtype);        /* as above */
int hr_gated_backward(const void* x, int64_t ldx, const void* w_gate, int64_t ldwg, const void* w_up, int64_t ldwu, int32_t dtype, int64_t m,
                      int64_t k, int64_t f, int32_t activation, const float* pre, const void* grad_out, int64_t ldgo, void* grad_x,
                      int64_t ldgx, void* grad_w_gate, int64_t ldgg, void* grad_w_up, int64_t ldgu, void* workspace, size_t workspace_bytes,
                      void* stream);

#define HR_ADAMW_BLOCK 256           /* numbers of a tensor that share an exponent, moments in 8 bits */

/* One tensor of hr_adamw: contiguous, n numbers, pointers DEV and aligned to their elements. */
typedef struct {
    void* param;             /* in param_dtype; updated */
    const void* grad;        /* in grad_dtype */
    float* master;           /* NULL, or the parameter in 32 bits: updated, and param only written (rounded once) */
    void* m;                 /* first moment: float32, or uint8 codes; updated */
    void* v;                 /* second moment: the same */
    uint8_t* exponents;      /* moments in 8 bits: [ceil(n / HR_ADAMW_BLOCK), 2], updated; NULL: moments in 32 bits */
    int64_t n;               /* 0 .. 2^36 */
    float weight_decay;      /* finite */
    int32_t param_dtype, grad_dtype;
} hr_adamw_tensor;

/*
 * hr_adamw — one step of AdamW over `count` tensors, in one launch for every 48 of them that have numbers:
 *   g = grad * *grad_scale,   m = beta1 m + (1 - beta1) g,   v = beta2 v + (1 - beta2) g^2,
 *   param = param (1 - lr weight_decay) - lr / (1 - beta1^step) * m / (sqrt(v / (1 - beta2^step)) + eps).
 * The arithmetic is float32, (1 - beta...) and what depends on step are taken in 64 bits and rounded.
 *   tensors    HOST array, read before the call returns.  No two may overlap.
 *   step       the number of this step, from 1 on; or device_step DEV int64 [1], read by the kernels (a captured step, whose number the
 *              program raises between replays; a number below 1 counts as 1): step is not looked at then.
 *   grad_scale DEV float32 [1] or NULL (1).
 *   0 <= beta1, beta2 < 1,  eps >= 0, lr finite.
 *
 * Moments in 8 bits, blocks of 256 numbers, exponents (em, ev) of a block:
 *   m is held as s 2^(em - 134), s a number of 4 bits of exponent and 3 of mantissa (OCP e4m3), rounded to even; em is the exponent field (of a
 *   float32) of the block's largest magnitude, 8 at least.
 *   v is held by the upper 12 bits of its float32, rounded to even, less 8 (ev - 31): a number of 5 bits of exponent and 3 of mantissa, code 0 for
 *   0.  ev is the exponent field of the largest after rounding, 31 at least.  A v above 0 never becomes 0 (the least code above 0 stands for
 *   it): what is held of an element's m is then divided by no less than it was made with, and its step grows by no more than the roundings.
 *   Before that every product and sum of m and v above is rounded to float32 by itself: the codes are the same on any machine.
 *   Zeros throughout, exponents too, are moments of 0: how a tensor begins.
 *   A block with a NaN or an infinity in m or v has exponent 255 there: all of its m (v) is NaN from then on.
 */
int hr_adamw(const hr_adamw_tensor* tensors, int32_t count, double lr, double beta1, double beta2, double eps, int64_t step,
             const int64_t* device_step, const float* grad_scale, void* stream);

/* hr_adamw_moments — the numbers that moments in 8 bits stand for: out_m, out_v DEV [n] float32, each NULL where it is not wanted. */
int hr_adamw_moments(const uint8_t* m, const uint8_t* v, const uint8_t* exponents, int64_t n, float* out_m, float* out_v, void* stream);

#ifdef __cplusplus
}
#endif
#endif /* HR_LAYERS_H */
