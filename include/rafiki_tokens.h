/*
 * rafiki_tokens.h -- answers over a vocabulary: the ensemble combine for language models.
 *
 * rafiki_combine_mean (rafiki_ensemble.h) averages the selected models' softmax and takes
 * the best class, for up to 1024 classes.  Where the members are language models the classes
 * are the tokens of a vocabulary, and the same average (Section 1; Section 5.2) is asked other
 * questions: draw a token from it (rafiki_combine_sample), list the likeliest tokens with
 * their log-probabilities (rafiki_combine_topk), and train one small model to answer like the
 * ensemble, from such a list (rafiki_distill_loss), or from answers that were drawn and then
 * rewarded or compared (rafiki_token_logp, rafiki_policy_loss, rafiki_preference_loss).
 * rafiki_quantize_rows_i8 and rafiki_fc_i8 are the final FC layer that makes the logits, in 8-bit
 * integers; rafiki_quantize_rows_mx4 and rafiki_fc_mx4 in 4-bit floating point with a scale for
 * every 32 values.
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

/* Log-probabilities of given tokens.  Row i of the logits z has the label y = labels[i] (int32 [n]);
 * a label outside [0, n_classes) means that the position has no token (a prompt's, padding): the
 * row is not read, its outputs are 0 and its gradient row is 0.  With x = z / T and p = softmax(x):
 *     out_logp[i]    = log p_y,
 *     out_entropy[i] = H = - sum_c p_c log p_c           (a term with p = 0 is 0),
 *     dz_c = 1/T [ a_i (1[c = y] - p_c) - h_i p_c (log p_c + H) ]
 * with a = grad_logp = dL / d logp and h = grad_entropy = dL / dH (fp32 [n]; null: 0; grad_logits
 * needs one of them); here and below grad_logits shares no element with the logits, which are read again for it (the
 * binding refuses such a call).  A row with a_i = h_i = 0 has gradient 0 whatever it holds.  A masked label
 * (logit -inf) has log p = -inf, as has a log p beyond fp32; NaN, +inf or a row of only -inf gives NaN
 * in all outputs of the row.  Any output may be null, not all.  Powers of classes are fp32, their sums and what is made of
 * them 64 bits, since what follows subtracts and sums log-probabilities; each output and each gradient is rounded once.
 * Before that log p is off by 3e-8 rms, nearly as often up as down (a power is off by at most 2^-23 (4.5 + d), d its distance
 * below the likeliest class in units of log p, and log p by their mean under p), and relatively where p is near 1.  H is not
 * negative and is off by a few times that relatively, however small it is and whatever the label.  2^-20 <= T <= 2^20,
 * 1 <= n <= 2^30. */
int rafiki_token_logp(const void* logits, int dtype, long long ld_row, int n, int n_classes, const int32_t* labels,
                      double temperature, const float* grad_logp, const float* grad_entropy, float* out_logp,
                      float* out_entropy, void* grad_logits, long long ld_grad, void* workspace,
                      long long workspace_bytes, void* stream);

/* Bytes of workspace for rafiki_token_logp and rafiki_policy_loss (0 unless few rows are long). */
int rafiki_token_workspace(int n, int n_classes, long long* bytes);

/* Clipped policy loss of drawn tokens with its gradient.  Rows, labels, T, log p and H as above; per
 * row (fp32 [n]) an advantage A, the log p of the policy that drew the token (old_logp; null: the present one, held
 * constant: r = 1) and that of a reference (ref_logp; null: no KL term).  With r = exp(log p - old),
 * d = ref - log p:
 *     kl     = exp(d) - d - 1,
 *     loss_i = - min(r A, clip(r, 1 - clip_low, 1 + clip_high) A) + kl_coef kl - entropy_coef H,
 *     a_i    = d loss_i / d log p = (r A <= clip(r, ..) A ? - r A : 0) + kl_coef (1 - exp(d)),
 * and the gradient is that of rafiki_token_logp with a_i and h_i = - entropy_coef, times g_i = grad_loss[i]
 * (fp32 [n], dL / d loss_i; null: 1).  A = 0 gives no policy term, kl_coef = 0 no KL term and entropy_coef = 0 no
 * entropy term, whatever they would hold; a row with g_i = 0 has gradient 0.  r or exp(d) beyond fp32 are +inf,
 * and where a_i is not finite the gradient row is NaN, as it is where log p, H or the loss is NaN.  Rows without a
 * token have loss, log p, kl and H 0.  out_loss, out_logp, out_kl (0 without ref_logp), out_entropy fp32 [n] and
 * grad_logits; any may be null, not all.  0 <= clip_low <= 1, clip_high >= 0 (may be +inf); the
 * coefficients are finite. */
int rafiki_policy_loss(const void* logits, int dtype, long long ld_row, int n, int n_classes, const int32_t* labels,
                       const float* advantage, const float* old_logp, const float* ref_logp, double temperature,
                       double clip_low, double clip_high, double kl_coef, double entropy_coef, const float* grad_loss,
                       float* out_loss, float* out_logp, float* out_kl, float* out_entropy, void* grad_logits,
                       long long ld_grad, void* workspace, long long workspace_bytes, void* stream);

/* Preference loss over n_pairs pairs of answers with its gradient.  The rows of pair p's chosen answer are
 * offsets[2 p] .. offsets[2 p + 1] - 1, those of its rejected one offsets[2 p + 1] .. offsets[2 p + 2] - 1
 * (int32 [2 n_pairs + 1], not decreasing, within [0, n]; null: 2 n_pairs answers of n / (2 n_pairs)
 * rows each, which then divides).  Answers in another order are brought into this one first.  Labels, T and log p as above; rows without a token count for nothing.  With
 * ref_logp the reference's log p (fp32 [n]; null: 0) and the sums over an answer's tokens (mean != 0: divided by their
 * number, an answer without tokens has score 0):
 *     score  = beta sum (log p - ref),        u = score of the chosen - score of the rejected,
 *     loss_p = - (1 - smoothing) log sigmoid(u) - smoothing log sigmoid(-u),
 *     a_i    = +- beta g_p [ smoothing sigmoid(u) - (1 - smoothing) sigmoid(-u) ]   (/ number if mean),
 * + for tokens of the chosen answer, - for the rejected one's, g_p = grad_loss[p] (fp32 [n_pairs]; null:
 * 1); the gradient is that of rafiki_token_logp.  out_loss fp32 [n_pairs], out_scores fp32 [n_pairs][2], grad_logits;
 * any may be null, not all.  A pair with g_p = 0 has gradient 0.  A score that is NaN (a row of its tokens that has no
 * distribution, or infinite scores of both answers) makes the loss and the gradient rows of both answers'
 * tokens NaN.  Rows before offsets[0] and from offsets[2 n_pairs] on are not read and their gradient rows are left as
 * they were.  Offsets that decrease or leave [0, n] give wrong values but no access out of the
 * arrays.  log p, scores and the loss are summed in 64 bits.  beta > 0 and finite, 0 <= smoothing <= 0.5,
 * 1 <= n_pairs <= 2^20. */
int rafiki_preference_loss(const void* logits, int dtype, long long ld_row, int n, int n_classes,
                           const int32_t* labels, const int32_t* offsets, int n_pairs, const float* ref_logp,
                           double temperature, double beta, double smoothing, int mean, const float* grad_loss,
                           float* out_loss, float* out_scores, void* grad_logits, long long ld_grad, void* workspace,
                           long long workspace_bytes, void* stream);

/* Bytes of workspace for rafiki_preference_loss. */
int rafiki_preference_workspace(int n, int n_classes, long long* bytes);

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

/* Rows of x [n][c] (dtype, ld_x elements apart, any alignment) in 4 bits: blocks of 32 neighbouring
 * values, each with a scale 2^(b - 127) of one byte b and 32 codes of 4 bits: a sign (8) and one of the
 * magnitudes 0, 0.5, 1, 1.5, 2, 3, 4, 6 (0 .. 7), i.e. E2M1 values with an E8M0 scale.  With e =
 * floor(log2 max |x|) - 2 of the block, b = e + 127 (at least 0; 0 for a block of zeros), and the codes are x / 2^(b - 127)
 * rounded to the nearest magnitude, ties to the even code, above 6 to 6 (so a largest value whose
 * significand exceeds 1.5 is cut to 1.5).  A block with a NaN or an infinity has b = 255 (NaN) and codes 0.
 * A row has ceil(c / 32) blocks, its last one filled up with code 0: q rows of 16 bytes a block, two codes a byte, the
 * even one in the low half, ld_q >= 16 ceil(c / 32) bytes apart; scale rows of a byte a block, ld_scale >=
 * ceil(c / 32) bytes apart (rafiki_fc_mx4 wants both on 16-byte boundaries).  n >= 1, 1 <= c <= 2^30. */
int rafiki_quantize_rows_mx4(const void* x, int dtype, long long ld_x, int n, int c, uint8_t* q, long long ld_q,
                             uint8_t* scale, long long ld_scale, void* stream);

/* FC layer in 4 bits: y[i][o] = act(sum_c x[i][c] w[o][c] + bias[o]) over the values that the codes and scales of
 * x [n] and w [c_out] stand for (layout as above, c_in a multiple of 32: whole blocks), bias fp32 [c_out] or
 * null, act ReLU if relu != 0 (NaN stays NaN).  Products are exact, sums fp32, and y (y_dtype, rows ld_y >= c_out
 * elements apart) is rounded once.  Rows of codes and of scales start on 16-byte boundaries (pointers and
 * distances multiples of 16; the distance of a single row does not matter); rows of scales are readable up to the next multiple of 16, what
 * lies behind c_in / 32 is ignored.  32 <= c_in <= 2^20, 1 <= n, c_out <= 2^24, distances <= 2^22. */
int rafiki_fc_mx4(const uint8_t* x, long long ld_x, const uint8_t* x_scale, long long ld_x_scale, const uint8_t* w,
                  long long ld_w, const uint8_t* w_scale, long long ld_w_scale, const float* bias, int n, int c_in,
                  int c_out, int relu, void* y, int y_dtype, long long ld_y, void* workspace, long long workspace_bytes,
                  void* stream);

/* Bytes of workspace for rafiki_fc_mx4. */
int rafiki_fc_mx4_workspace(int n, int c_in, int c_out, long long* bytes);

#ifdef __cplusplus
}
#endif

#endif /* RAFIKI_TOKENS_H */
