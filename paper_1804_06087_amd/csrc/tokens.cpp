// C entry points of the vocabulary operators (rafiki_tokens.h): argument checks, then one or
// two launches on the caller's stream.
#include "rafiki_tokens.h"
#include "greedy.h"
#include "tokens.h"

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

}  // extern "C"
