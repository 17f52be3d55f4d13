// C entry points of the vocabulary operators (rafiki_tokens.h): argument checks, then one or
// two launches on the caller's stream.
#include "rafiki_tokens.h"
#include "greedy.h"
#include "tokens.h"

#include <algorithm>
#include <cmath>
#include <string>

using namespace rafiki;

namespace {

int invalid(const char* msg) { return set_error(RAFIKI_ERR_INVALID, msg); }

int launched(hipError_t st, const char* what) {
  if (st == hipSuccess) return RAFIKI_OK;
  return set_error(RAFIKI_ERR_HIP, std::string(what) + " launch: " + hipGetErrorString(st));
}

bool aligned16(const void* p) { return ((uintptr_t)p & 15) == 0; }
bool aligned_to(const void* p, int dtype) { return ((uintptr_t)p & (dtype == RAFIKI_BF16 ? 1 : 3)) == 0; }
bool known(int dtype) { return dtype == RAFIKI_FP32 || dtype == RAFIKI_BF16; }

bool fc_sizes(int n, int c_in, int c_out) {
  return n >= 1 && n <= (1 << 24) && c_out >= 1 && c_out <= (1 << 24) && c_in >= 1 && c_in <= 131071;
}

long long combine_bytes(int n_models, int n, int n_classes) {
  return (long long)n_models * n * token_stat_stride(n_classes) + ((long long)n * 4 + 15) / 16 * 16;
}

bool fc_mx4_sizes(int n, int c_in, int c_out) {
  return n >= 1 && n <= (1 << 24) && c_out >= 1 && c_out <= (1 << 24) && c_in >= 32 && c_in <= (1 << 20) && c_in % 32 == 0;
}
bool row_sizes(int n, int n_classes) { return n >= 1 && n <= (1 << 30) && n_classes >= 1 && n_classes <= kMaxTokenClasses; }
bool bad_workspace(const void* workspace, long long bytes, long long need) {
  return need && (!workspace || bytes < need || !aligned16(workspace));
}

// What the losses over given tokens have alike.
int check_rows(const void* logits, int dtype, long long ld_row, int n, int n_classes, const void* labels, double temperature,
               const void* grad_logits, long long ld_grad, const void* workspace, long long bytes, long long (*need)(int, int)) {
  if (!logits || !labels) return invalid("null pointer");
  if (!known(dtype)) return invalid("dtype must be RAFIKI_FP32 or RAFIKI_BF16");
  if (!row_sizes(n, n_classes)) return invalid("n must be in [1, 2^30] and n_classes in [1, 2^20]");
  if (!(temperature >= 0x1p-20 && temperature <= 0x1p20)) return invalid("temperature must be in [2^-20, 2^20]");
  if (ld_row < 0 || (grad_logits && ld_grad < n_classes)) return invalid("row distances: ld_row >= 0, ld_grad >= n_classes");
  if (!aligned_to(logits, dtype) || !aligned_to(grad_logits, dtype)) return invalid("rows are not aligned to their type");
  if (bad_workspace(workspace, bytes, need(n, n_classes)))
    return invalid("workspace is null, too small or not on a 16-byte boundary");
  return RAFIKI_OK;
}

template <typename Args>
Args row_args(const void* logits, long long ld_row, int n, int n_classes, const int32_t* labels, double temperature,
              void* grad_logits, long long ld_grad) {
  Args a{};
  a.logits = logits;
  a.ld_row = ld_row;
  a.n = n;
  a.C = n_classes;
  a.labels = labels;
  a.inv_t = 1.0 / temperature;
  a.s.s = 1.4426950408889634 / temperature;
  int exponent;
  const double bits = std::frexp(a.s.s, &exponent);          // in [1/2, 1)
  auto first = [&](int n) { return std::ldexp(std::floor(std::ldexp(bits, n)), exponent - n); };
  const double tiny = 0x1p-60;                               // the rests are positive (see token_loss.hip)
  a.s.hi = (float)first(24);
  a.s.lo = (float)std::max(a.s.s - (double)a.s.hi, tiny * a.s.s);
  a.s.hi16 = (float)first(16);
  a.s.rest16 = (float)std::max((a.s.s - (double)a.s.hi16) / (double)a.s.hi16, tiny);
  a.grad = grad_logits;
  a.ld_grad = ld_grad;
  return a;
}

int check_combine(const void* logits, int dtype, long long ld_model, long long ld_row, int n_models, int n,
                  int n_classes, const void* labels, const void* out, const void* workspace, long long bytes) {
  if (!logits || !labels || !out) return invalid("null pointer");
  if (!known(dtype)) return invalid("dtype must be RAFIKI_FP32 or RAFIKI_BF16");
  if (n_models < 1 || n_models > kMaxTokenModels) return invalid("n_models must be in [1, 32]");
  if (n < 1 || n_classes < 1 || n_classes > kMaxTokenClasses)
    return invalid("n must be >= 1 and n_classes in [1, 2^20]");
  if (ld_model < 0 || ld_row < 0) return invalid("row distances must be >= 0");
  if (!aligned_to(logits, dtype)) return invalid("logits are not aligned to their type");
  const long long need = combine_bytes(n_models, n, n_classes);
  if (need && (!workspace || bytes < need || !aligned16(workspace)))
    return invalid("workspace is null, too small or not on a 16-byte boundary");
  return RAFIKI_OK;
}

TokenArgs token_args(const void* logits, long long ld_model, long long ld_row, int n_models, int n, int n_classes,
                     int32_t* labels, float* out, void* workspace) {
  TokenArgs a{};
  a.logits = logits;
  a.ld_model = ld_model;
  a.ld_row = ld_row;
  a.S = n_models;
  a.n = n;
  a.C = n_classes;
  a.units = token_units(n_classes);
  a.stat_stride = token_stat_stride(n_classes);
  a.t_all = 1.f;
  a.stats = (char*)workspace;
  a.flat = (int32_t*)(a.stats + (long long)n_models * n * a.stat_stride);
  a.labels = labels;
  a.out = out;
  return a;
}

}  // namespace

extern "C" {

int rafiki_combine_workspace(int n_models, int n, int n_classes, long long* bytes) {
  if (!bytes) return invalid("null pointer");
  if (n_models < 1 || n_models > kMaxTokenModels || n < 1 || n_classes < 1 || n_classes > kMaxTokenClasses)
    return invalid("n_models must be in [1, 32], n >= 1 and n_classes in [1, 2^20]");
  *bytes = combine_bytes(n_models, n, n_classes);
  return RAFIKI_OK;
}

int rafiki_combine_sample(const void* logits, int dtype, long long ld_model, long long ld_row, int n_models, int n,
                          int n_classes, const float* temperature, const int32_t* top_k, const float* top_p,
                          const float* min_p, const float* uniform, int32_t* out_labels, float* out_probs,
                          void* workspace, long long workspace_bytes, void* stream) {
  const int rc = check_combine(logits, dtype, ld_model, ld_row, n_models, n, n_classes, out_labels, out_probs,
                               workspace, workspace_bytes);
  if (rc) return rc;
  if (!uniform) return invalid("null uniform");
  TokenArgs a = token_args(logits, ld_model, ld_row, n_models, n, n_classes, out_labels, out_probs, workspace);
  a.temperature = temperature;
  a.top_k = top_k;
  a.top_p = top_p;
  a.min_p = min_p;
  a.uniform = uniform;
  return launched(launch_sample(a, dtype == RAFIKI_BF16, (hipStream_t)stream), "sample");
}

int rafiki_combine_topk(const void* logits, int dtype, long long ld_model, long long ld_row, int n_models, int n,
                        int n_classes, float temperature, int k, int32_t* out_labels, float* out_logp,
                        void* workspace, long long workspace_bytes, void* stream) {
  const int rc = check_combine(logits, dtype, ld_model, ld_row, n_models, n, n_classes, out_labels, out_logp,
                               workspace, workspace_bytes);
  if (rc) return rc;
  if (!(temperature > 0.f) || !std::isfinite(temperature)) return invalid("temperature must be positive and finite");
  if (k < 1 || k > kMaxTokenK) return invalid("k must be in [1, 1024]");
  TokenArgs a = token_args(logits, ld_model, ld_row, n_models, n, n_classes, out_labels, out_logp, workspace);
  a.t_all = temperature;
  a.k = k;
  return launched(launch_topk(a, dtype == RAFIKI_BF16, (hipStream_t)stream), "topk");
}

int rafiki_distill_loss(const void* logits, int dtype, long long ld_row, int n, int n_classes,
                        const int32_t* teacher_labels, const float* teacher_logp, int k, float temperature, int rest,
                        const float* grad_loss, float* out_loss, void* grad_logits, long long ld_grad, void* stream) {
  if (!logits || !teacher_labels || !teacher_logp) return invalid("null pointer");
  if (!out_loss && !grad_logits) return invalid("out_loss and grad_logits are both null");
  if (!known(dtype)) return invalid("dtype must be RAFIKI_FP32 or RAFIKI_BF16");
  if (n < 1 || n_classes < 1 || n_classes > kMaxTokenClasses)
    return invalid("n must be >= 1 and n_classes in [1, 2^20]");
  if (k < 1 || k > kMaxTokenK) return invalid("k must be in [1, 1024]");
  if (!(temperature > 0.f) || !std::isfinite(temperature)) return invalid("temperature must be positive and finite");
  if (ld_row < 0 || (grad_logits && ld_grad < n_classes)) return invalid("row distances: ld_row >= 0, ld_grad >= n_classes");
  if (!aligned_to(logits, dtype) || !aligned_to(grad_logits, dtype)) return invalid("rows are not aligned to their type");
  DistillArgs a{};
  a.logits = logits;
  a.ld_row = ld_row;
  a.n = n;
  a.C = n_classes;
  a.k = k;
  a.labels = teacher_labels;
  a.logp = teacher_logp;
  a.t = temperature;
  a.rest = rest != 0;
  a.grad_loss = grad_loss;
  a.loss = out_loss;
  a.grad = grad_logits;
  a.ld_grad = ld_grad;
  return launched(launch_distill(a, dtype == RAFIKI_BF16, (hipStream_t)stream), "distill");
}

int rafiki_token_logp(const void* logits, int dtype, long long ld_row, int n, int n_classes, const int32_t* labels,
                      double temperature, const float* grad_logp, const float* grad_entropy, float* out_logp,
                      float* out_entropy, void* grad_logits, long long ld_grad, void* workspace,
                      long long workspace_bytes, void* stream) {
  const int rc = check_rows(logits, dtype, ld_row, n, n_classes, labels, temperature, grad_logits, ld_grad, workspace,
                            workspace_bytes, token_loss_workspace_bytes);
  if (rc) return rc;
  if (!out_logp && !out_entropy && !grad_logits) return invalid("no output is asked for");
  if (grad_logits && !grad_logp && !grad_entropy) return invalid("grad_logits needs grad_logp or grad_entropy");
  TokenLossArgs a = row_args<TokenLossArgs>(logits, ld_row, n, n_classes, labels, temperature, grad_logits, ld_grad);
  a.grad_logp = grad_logits ? grad_logp : nullptr;
  a.grad_entropy = grad_logits ? grad_entropy : nullptr;
  a.logp = out_logp;
  a.entropy = out_entropy;
  a.parts = workspace;
  return launched(launch_token_loss(a, dtype == RAFIKI_BF16, (hipStream_t)stream), "token_logp");
}

int rafiki_token_workspace(int n, int n_classes, long long* bytes) {
  if (!bytes) return invalid("null pointer");
  if (!row_sizes(n, n_classes)) return invalid("n must be in [1, 2^30] and n_classes in [1, 2^20]");
  *bytes = token_loss_workspace_bytes(n, n_classes);
  return RAFIKI_OK;
}

int rafiki_policy_loss(const void* logits, int dtype, long long ld_row, int n, int n_classes, const int32_t* labels,
                       const float* advantage, const float* old_logp, const float* ref_logp, double temperature,
                       double clip_low, double clip_high, double kl_coef, double entropy_coef, const float* grad_loss,
                       float* out_loss, float* out_logp, float* out_kl, float* out_entropy, void* grad_logits,
                       long long ld_grad, void* workspace, long long workspace_bytes, void* stream) {
  const int rc = check_rows(logits, dtype, ld_row, n, n_classes, labels, temperature, grad_logits, ld_grad, workspace,
                            workspace_bytes, token_loss_workspace_bytes);
  if (rc) return rc;
  if (!advantage) return invalid("null advantage");
  if (!out_loss && !out_logp && !out_kl && !out_entropy && !grad_logits) return invalid("no output is asked for");
  if (!(clip_low >= 0 && clip_low <= 1) || !(clip_high >= 0))
    return invalid("clip_low must be in [0, 1] and clip_high >= 0");
  if (!std::isfinite(kl_coef) || !std::isfinite(entropy_coef)) return invalid("kl_coef and entropy_coef must be finite");
  TokenLossArgs a = row_args<TokenLossArgs>(logits, ld_row, n, n_classes, labels, temperature, grad_logits, ld_grad);
  a.policy = true;
  a.advantage = advantage;
  a.old_logp = old_logp;
  a.ref_logp = ref_logp;
  a.grad_loss = grad_loss;
  a.clip_low = clip_low;
  a.clip_high = clip_high;
  a.kl_coef = kl_coef;
  a.entropy_coef = entropy_coef;
  a.loss = out_loss;
  a.logp = out_logp;
  a.kl = out_kl;
  a.entropy = out_entropy;
  a.parts = workspace;
  return launched(launch_token_loss(a, dtype == RAFIKI_BF16, (hipStream_t)stream), "policy_loss");
}

int rafiki_preference_workspace(int n, int n_classes, long long* bytes) {
  if (!bytes) return invalid("null pointer");
  if (!row_sizes(n, n_classes)) return invalid("n must be in [1, 2^30] and n_classes in [1, 2^20]");
  *bytes = preference_workspace_bytes(n, n_classes);
  return RAFIKI_OK;
}

int rafiki_preference_loss(const void* logits, int dtype, long long ld_row, int n, int n_classes,
                           const int32_t* labels, const int32_t* offsets, int n_pairs, const float* ref_logp,
                           double temperature, double beta, double smoothing, int mean, const float* grad_loss,
                           float* out_loss, float* out_scores, void* grad_logits, long long ld_grad, void* workspace,
                           long long workspace_bytes, void* stream) {
  const int rc = check_rows(logits, dtype, ld_row, n, n_classes, labels, temperature, grad_logits, ld_grad, workspace,
                            workspace_bytes, preference_workspace_bytes);
  if (rc) return rc;
  if (!out_loss && !out_scores && !grad_logits) return invalid("no output is asked for");
  if (n_pairs < 1 || n_pairs > (1 << 20)) return invalid("n_pairs must be in [1, 2^20]");
  if (!offsets && n % (2LL * n_pairs)) return invalid("without offsets n must be a multiple of 2 n_pairs");
  if (!(beta > 0) || !std::isfinite(beta) || !(smoothing >= 0 && smoothing <= 0.5))
    return invalid("beta must be positive and finite, smoothing in [0, 0.5]");
  PreferenceArgs a = row_args<PreferenceArgs>(logits, ld_row, n, n_classes, labels, temperature, grad_logits, ld_grad);
  a.pairs = n_pairs;
  a.offsets = offsets;
  a.ref_logp = ref_logp;
  a.beta = beta;
  a.smoothing = smoothing;
  a.mean = mean != 0;
  a.grad_loss = grad_loss;
  a.loss = out_loss;
  a.scores = out_scores;
  a.rows = (PreferenceRow*)workspace;
  return launched(launch_preference(a, dtype == RAFIKI_BF16, (hipStream_t)stream), "preference_loss");
}

int rafiki_quantize_rows_i8(const void* x, int dtype, long long ld_x, int n, int c, int8_t* q, long long ld_q,
                            float* scale, void* stream) {
  if (!x || !q || !scale) return invalid("null pointer");
  if (!known(dtype)) return invalid("dtype must be RAFIKI_FP32 or RAFIKI_BF16");
  if (n < 1 || c < 1 || c > (1 << 30) || ld_x < 0 || ld_q < c)
    return invalid("n >= 1, c in [1, 2^30], ld_x >= 0 and ld_q >= c");
  if (!aligned_to(x, dtype)) return invalid("rows are not aligned to their type");
  return launched(launch_quantize(x, dtype == RAFIKI_BF16, ld_x, n, c, q, ld_q, scale, (hipStream_t)stream), "quantize");
}

int rafiki_fc_i8_workspace(int n, int c_in, int c_out, long long* bytes) {
  if (!bytes) return invalid("null pointer");
  if (!fc_sizes(n, c_in, c_out)) return invalid("n and c_out must be in [1, 2^24] and c_in in [1, 131071]");
  *bytes = fc_i8_workspace_bytes(n, c_in, c_out);
  return RAFIKI_OK;
}

int rafiki_fc_i8(const int8_t* x, long long ld_x, const float* x_scale, const int8_t* w, long long ld_w,
                 const float* w_scale, const float* bias, int n, int c_in, int c_out, int relu, void* y, int y_dtype,
                 long long ld_y, void* workspace, long long workspace_bytes, void* stream) {
  if (!x || !x_scale || !w || !w_scale || !y) return invalid("null pointer");
  if (!known(y_dtype)) return invalid("y_dtype must be RAFIKI_FP32 or RAFIKI_BF16");
  if (!fc_sizes(n, c_in, c_out)) return invalid("n and c_out must be in [1, 2^24] and c_in in [1, 131071]");
  const long long k16 = (c_in + 15) / 16 * 16;
  if (!aligned16(x) || !aligned16(w) || ld_x % 16 || ld_w % 16 || ld_x < k16 || ld_w < k16 || ld_x > (1 << 22) ||
      ld_w > (1 << 22))
    return invalid("rows of x and w: 16-byte boundaries, at least c_in rounded up to 16 and at most 2^22 bytes apart");
  if (ld_y < c_out || !aligned_to(y, y_dtype)) return invalid("y: ld_y >= c_out, aligned to its type");
  const long long need = fc_i8_workspace_bytes(n, c_in, c_out);
  if (need && (!workspace || workspace_bytes < need || !aligned16(workspace)))
    return invalid("workspace is null, too small or not on a 16-byte boundary");
  FcI8Args a{};
  a.x = x;
  a.w = w;
  a.ld_x = ld_x;
  a.ld_w = ld_w;
  a.ld_y = ld_y;
  a.sx = x_scale;
  a.sw = w_scale;
  a.bias = bias;
  a.n = n;
  a.c_in = c_in;
  a.c_out = c_out;
  a.relu = relu != 0;
  a.out_bf16 = y_dtype == RAFIKI_BF16;
  a.y = y;
  a.partial = (int*)workspace;
  return launched(launch_fc_i8(a, (hipStream_t)stream), "fc_i8");
}

int rafiki_quantize_rows_mx4(const void* x, int dtype, long long ld_x, int n, int c, uint8_t* q, long long ld_q,
                             uint8_t* scale, long long ld_scale, void* stream) {
  if (!x || !q || !scale) return invalid("null pointer");
  if (!known(dtype)) return invalid("dtype must be RAFIKI_FP32 or RAFIKI_BF16");
  if (n < 1 || c < 1 || c > (1 << 30) || ld_x < 0) return invalid("n >= 1, c in [1, 2^30] and ld_x >= 0");
  const long long blocks = ((long long)c + 31) / 32;
  if (ld_q < 16 * blocks || ld_scale < blocks) return invalid("ld_q >= 16 ceil(c / 32) and ld_scale >= ceil(c / 32)");
  if (!aligned_to(x, dtype)) return invalid("rows are not aligned to their type");
  return launched(launch_quantize_mx4(x, dtype == RAFIKI_BF16, ld_x, n, c, q, ld_q, scale, ld_scale, (hipStream_t)stream),
                  "quantize_mx4");
}

int rafiki_fc_mx4_workspace(int n, int c_in, int c_out, long long* bytes) {
  if (!bytes) return invalid("null pointer");
  if (!fc_mx4_sizes(n, c_in, c_out)) return invalid("n and c_out must be in [1, 2^24] and c_in a multiple of 32 up to 2^20");
  *bytes = fc_mx4_workspace_bytes(n, c_in / 32, c_out);
  return RAFIKI_OK;
}

int rafiki_fc_mx4(const uint8_t* x, long long ld_x, const uint8_t* x_scale, long long ld_x_scale, const uint8_t* w,
                  long long ld_w, const uint8_t* w_scale, long long ld_w_scale, const float* bias, int n, int c_in,
                  int c_out, int relu, void* y, int y_dtype, long long ld_y, void* workspace, long long workspace_bytes,
                  void* stream) {
  if (!x || !x_scale || !w || !w_scale || !y) return invalid("null pointer");
  if (!known(y_dtype)) return invalid("y_dtype must be RAFIKI_FP32 or RAFIKI_BF16");
  if (!fc_mx4_sizes(n, c_in, c_out)) return invalid("n and c_out must be in [1, 2^24] and c_in a multiple of 32 up to 2^20");
  const long long row = c_in / 2, scales = ((long long)c_in / 32 + 15) / 16 * 16;
  // a single row has no distance to the next
  if (n == 1) ld_x = row, ld_x_scale = scales;
  if (c_out == 1) ld_w = row, ld_w_scale = scales;
  auto bad = [](const void* p, long long ld, long long least) {
    return !aligned16(p) || ld % 16 || ld < least || ld > (1 << 22);
  };
  if (bad(x, ld_x, row) || bad(w, ld_w, row) || bad(x_scale, ld_x_scale, scales) || bad(w_scale, ld_w_scale, scales))
    return invalid("rows of codes and scales: 16-byte boundaries, at least c_in / 2 and c_in / 32 rounded up to 16, and at most "
                   "2^22 bytes apart");
  if ((n > 1 && ld_y < c_out) || !aligned_to(y, y_dtype)) return invalid("y: ld_y >= c_out, aligned to its type");
  const long long need = fc_mx4_workspace_bytes(n, c_in / 32, c_out);
  if (need && (!workspace || workspace_bytes < need || !aligned16(workspace)))
    return invalid("workspace is null, too small or not on a 16-byte boundary");
  FcMx4Args a{};
  a.x = x;
  a.xs = x_scale;
  a.w = w;
  a.ws = w_scale;
  a.ld_x = ld_x;
  a.ld_xs = ld_x_scale;
  a.ld_w = ld_w;
  a.ld_ws = ld_w_scale;
  a.ld_y = ld_y;
  a.bias = bias;
  a.n = n;
  a.blocks = c_in / 32;
  a.c_out = c_out;
  a.relu = relu != 0;
  a.out_bf16 = y_dtype == RAFIKI_BF16;
  a.y = y;
  a.partial = (float*)workspace;
  return launched(launch_fc_mx4(a, (hipStream_t)stream), "fc_mx4");
}

}  // extern "C"
