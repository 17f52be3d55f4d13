/*
 * rafiki_tokens.h -- answers over a vocabulary: the ensemble combine for language models.
 *
 * rafiki_combine_mean (rafiki_ensemble.h) averages the selected models' softmax and takes
 * the best class, for up to 1024 classes.  Where the members are language models the classes
 * are the tokens of a vocabulary, and the same average (Section 1; Section 5.2) is asked other
 * questions: draw a token from it (rafiki_combine_sample), list the likeliest tokens with
 * their log-probabilities (rafiki_combine_topk), and train one small model to answer like the
 * ensemble, from such a list (rafiki_distill_loss).  rafiki_quantize_rows_i8 and rafiki_fc_i8
 * are the final FC layer that makes the logits, in 8-bit integers.
 *
 * Conventions (those of rafiki_ensemble.h, and)
 * - All pointers are device pointers of the current device; every call only enqueues work on
 *   `stream` (hipStream_t as void*; 0 = the null stream), allocates nothing and can be captured
 *   into a graph.  Argument errors return RAFIKI_ERR_INVALID before any device call.
 * - `dtype` is RAFIKI_FP32 or RAFIKI_BF16.  Logits are rows of n_classes contiguous values;
 *   ld_row (and ld_model) are the distances between rows (and between models) in elements,
 *   any value >= 0; no alignment beyond the element's is needed.  1 <= n_classes <= 2^20.
 * - A logit of -inf masks its class.  Offsets are 64-bit.
 * - `workspace` holds at least the stated number of bytes on a 16-byte boundary; its contents
 *   need not be set and mean nothing afterwards.  Calls whose work may overlap on the device
 *   (two streams, two graphs) need a workspace each.  It may be null where 0 bytes are asked.
 * - Outputs must not alias inputs, the workspace or each other.  Results are deterministic.
 */
#ifndef RAFIKI_TOKENS_H
#define RAFIKI_TOKENS_H

#include <stdint.h>

#include "rafiki_ensemble.h"

#ifdef __cplusplus
extern "C" {
#endif

/* The combined distribution of row i at temperature T:
 *     p_c = 1/n_models * sum_m softmax(z_m / T)_c        (z_m = logits[m][i][:])
 * taken in 64 bits from the logits as stored (below 2^-960, of several models, to 2^-15 of
 * itself).  A class below 2^-1000 counts as having no probability.  Classes are ranked by p, ties
 * by the lower index; two whose p agree but for the rounding of 64 bits, as logits permuted
 * between the models make them, rank as those round.  A row has no distribution where a model's
 * logits hold NaN or +inf, or nothing above -inf, or where T is NaN or negative; T = +inf weighs
 * all classes above -inf alike. */

/* Bytes of workspace for rafiki_combine_sample and rafiki_combine_topk. */
int rafiki_combine_workspace(int n_models, int n, int n_classes, long long* bytes);

/* Draw one class per row from the combined distribution.  Per row (arrays of n; a null array
 * leaves its filter off, and a null temperature is 1):
 *   temperature  T as above; T = 0 takes the first-ranked class at T = 1 (the filters and
 *                uniform do not matter);
 *   top_k        keep the first top_k classes (<= 0, or >= n_classes: all);
 *   top_p        of those, keep the shortest leading run whose sum is >= top_p times the sum
 *                of all of those (at least one class; >= 1 or NaN: all);
 *   min_p        of those, keep the classes with p >= min_p * p of the first (<= 0 or NaN:
 *                all; above 1 counts as 1);
 *   uniform      u in [0, 1): the label is the lowest class index c for which the sum of p
 *                over the kept classes with index <= c is > u times the sum of all kept (u >= 1:
 *                the last kept class, u < 0 or NaN: as 0).  Classes below 2^-62 count as 0 in these
 *                sums and are not drawn.  Required.
 * out_labels int32 [n]; out_probs fp32 [n]: the label's p over the sum of all kept (1 for
 * T = 0).  A row without a distribution has label -1, and probability 0 if a mask left it
 * empty, NaN otherwise.  Sums are held in units of 2^-62; that of a row of more than 1024 classes
 * comes from partial sums in 64-bit floating point.
 * 1 <= n_models <= 32, n >= 1. */
int rafiki_combine_sample(const void* logits, int dtype, long long ld_model, long long ld_row, int n_models, int n,
                          int n_classes, const float* temperature, const int32_t* top_k, const float* top_p,
                          const float* min_p, const float* uniform, int32_t* out_labels, float* out_probs,
                          void* workspace, long long workspace_bytes, void* stream);

/* The k first-ranked classes of every row, best first, and their log p at one temperature
 * (> 0, finite): out_labels int32 [n][k], out_logp fp32 [n][k].  Where fewer than k classes
 * have a probability the rest is -1 and -inf; a row without a distribution is all -1, with
 * -inf if a mask left it empty, NaN otherwise.  1 <= k <= 1024 (k may exceed n_classes);
 * other limits as above. */
int rafiki_combine_topk(const void* logits, int dtype, long long ld_model, long long ld_row, int n_models, int n,
                        int n_classes, float temperature, int k, int32_t* out_labels, float* out_logp,
                        void* workspace, long long workspace_bytes, void* stream);

/* Distillation of a teacher's top classes into a student (the student's logits z, one row per
 * position), with its gradient.  Row i has k slots (teacher_labels int32 [n][k], teacher_logp
 * fp32 [n][k], as rafiki_combine_topk writes them at the same temperature T); a slot whose
 * label is outside [0, n_classes) is empty, and slots of one class add up.  With K the classes
 * of row i, p = softmax(z / T) and q_j the sum of exp(teacher_logp) over the slots of class j:
 *   rest = 0: q is divided by its sum (the teacher's values may then be any logits / T);
 *             loss_i = T^2 sum_{j in K} q_j (log q_j - log p_j);
 *             a row with no q above 0 has loss 0 and gradient 0;
 *   rest = 1: all other classes count as one more, with q_r = 1 - sum q and p_r their sum of p:
 *             loss_i = T^2 [ the sum above + q_r (log q_r - log p_r) ]; q_r below 2^-20
 *             (rounding of the fp32 values), or with K all classes, counts as 0.
 * Terms with q = 0 are 0.  With Q = sum q + q_r the gradient is
 *   dz_c = T g_i (Q p_c - q_c) for c in K,  T g_i (Q p_c - q_r p_c / p_r) otherwise; q_r is
 *   0 here, in Q too, without rest and where p_r = 0 (nothing above -inf outside K; the loss is then
 *   +inf if q_r > 0),
 * where g_i = grad_loss[i] (fp32 [n], dL / d loss_i; null: 1); a row with g_i = 0 has gradient
 * 0 whatever it holds.  A class with p = 0 in K and q > 0 gives loss +inf, as does a log p
 * beyond fp32; NaN, +inf or a row of only -inf in the student, or NaN in the teacher, gives NaN.
 * out_loss fp32 [n] or null, grad_logits [n] rows of the logits' dtype ld_grad >= n_classes
 * elements apart, or null; not both null (the backward pass alone: out_loss null).  fp32
 * arithmetic, each gradient rounded once.  T > 0 and finite (below fp32's normal range it may count as
 * 8.5e-39); 1 <= k <= 1024, n >= 1. */
int rafiki_distill_loss(const void* logits, int dtype, long long ld_row, int n, int n_classes,
                        const int32_t* teacher_labels, const float* teacher_logp, int k, float temperature, int rest,
                        const float* grad_loss, float* out_loss, void* grad_logits, long long ld_grad, void* stream);

/* Rows of x [n][c] (dtype, ld_x elements apart, any alignment) in 8 bits: scale[i] =
 * max |x_i| / 127 in fp32 (0 for a row of zeros), q = x / scale rounded to the nearest integer,
 * ties to even, exactly, into int8 rows ld_q bytes apart (ld_q >= c).  A row with a NaN or an
 * infinity has scale NaN and q = 0.  Rows whose scale would be below 2^-126 are quantised as zeros.
 * n >= 1, 1 <= c <= 2^30. */
int rafiki_quantize_rows_i8(const void* x, int dtype, long long ld_x, int n, int c, int8_t* q, long long ld_q,
                            float* scale, void* stream);

/* FC layer in 8 bits: y[i][o] = act(x_scale[i] * w_scale[o] * sum_c x[i][c] w[o][c] + bias[o]), x int8 [n]
 * rows ld_x bytes apart, w int8 [c_out] rows ld_w bytes apart (the FC layout [c_out, c_in]), the scales
 * fp32 [n] and [c_out], bias fp32 [c_out] or null, act ReLU if relu != 0.  Sums are exact int32; the
 * epilogue is fp32, the two scales multiplied first, and y (y_dtype, rows ld_y >= c_out elements
 * apart) is rounded once.  Rows of x and w start on 16-byte boundaries (pointers and ld multiples of 16) and are readable up to the next
 * multiple of 16 of c_in; what lies behind c_in is ignored.  1 <= c_in <= 131071 (128^2 c_in fits an
 * int32), 1 <= n, c_out <= 2^24; ld_x, ld_w <= 2^22. */
int rafiki_fc_i8(const int8_t* x, long long ld_x, const float* x_scale, const int8_t* w, long long ld_w,
                 const float* w_scale, const float* bias, int n, int c_in, int c_out, int relu, void* y, int y_dtype,
                 long long ld_y, void* workspace, long long workspace_bytes, void* stream);

/* Bytes of workspace for rafiki_fc_i8. */
int rafiki_fc_i8_workspace(int n, int c_in, int c_out, long long* bytes);

#ifdef __cplusplus
}
#endif

#endif /* RAFIKI_TOKENS_H */
