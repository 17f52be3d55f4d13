// Internal interface of the vocabulary operators (rafiki_tokens.h): launch arguments.
#pragma once
#include "kernels.h"

namespace rafiki {

constexpr int kMaxTokenModels = 32;
constexpr int kMaxTokenClasses = 1 << 20;
constexpr int kMaxTokenK = 1024;
// Statistics of the logits in the workspace: per row and model, the maximum of every 64 classes
// (16 a unit of 1024 classes; +inf throughout a unit that holds NaN or +inf), then a UnitStat of every
// unit: its maximum and its sum of 2^((z - maximum) log2(e) / T).
struct UnitStat {
  double sum;
  float top;
  float pad;
};
constexpr int kUnitClasses = 1024;
constexpr int kUnitTops = kUnitClasses / 64;
inline int token_units(int C) { return (C + kUnitClasses - 1) / kUnitClasses; }
inline long long token_stat_stride(int C) {   // bytes, a multiple of 16
  return (long long)token_units(C) * (kUnitTops * (long long)sizeof(float) + (long long)sizeof(UnitStat));
}

struct TokenArgs {
  const void* logits;
  long long ld_model, ld_row;
  int S, n, C, units, row0;   // row0: the launch's first row
  const float* temperature;   // [n] or null (then t_all)
  float t_all;
  int32_t* flat;              // [n] in the workspace: rows left to the histogram kernels
  char* stats;
  long long stat_stride;
  int32_t* labels;
  float* out;                 // probabilities [n] / log-probabilities [n][k]
  // sample
  const int32_t* top_k;
  const float* top_p;
  const float* min_p;
  const float* uniform;
  // topk
  int k;
};

struct DistillArgs {
  const void* logits;
  long long ld_row;
  int n, C, k, row0;          // row0: the launch's first row
  const int32_t* labels;
  const float* logp;
  float t;
  int rest;
  const float* grad_loss;
  float* loss;
  void* grad;
  long long ld_grad;
};

struct FcI8Args {
  const int8_t* x;
  const int8_t* w;
  long long ld_x, ld_w, ld_y;
  const float* sx;
  const float* sw;
  const float* bias;
  int n, c_in, c_out, relu, out_bf16;
  int kt_per_split;           // K tiles of 128 bytes per split
  void* y;
  int* partial;               // [splits][n][c_out] int32 sums (splits > 1)
};

// log2(e) / T in 64 bits; its first 24 bits and the rest; its first 16 bits and the rest relative to them.
struct Scale {
  double s;
  float hi, lo, hi16, rest16;
};
struct TokenLossArgs {
  const void* logits;
  long long ld_row;
  int n, C, row0;             // row0: the launch's first row
  const int32_t* labels;
  double inv_t;               // 1 / T
  Scale s;
  bool policy;
  const float* grad_logp;     // token_logp
  const float* grad_entropy;
  const float* advantage;     // policy_loss
  const float* old_logp;
  const float* ref_logp;
  const float* grad_loss;
  double clip_low, clip_high, kl_coef, entropy_coef;
  float* loss;
  float* logp;
  float* kl;
  float* entropy;
  void* grad;
  long long ld_grad;
  int n_parts, per_part;      // parts of a row, chunks of a part
  void* parts;                // sums of the parts (n_parts > 1)
};

struct PreferenceRow {        // of the workspace
  float top, share;           // p of a class is 2^((z - top) s) share
  float rest;                 // 1 - p of the label
  float weight;               // dL / d log p over T
};
struct PreferenceArgs {
  const void* logits;
  long long ld_row;
  int n, C, pairs;
  const int32_t* labels;
  const int32_t* offsets;
  const float* ref_logp;
  double inv_t;
  Scale s;
  double beta, smoothing;
  int mean;
  const float* grad_loss;
  float* loss;
  float* scores;
  void* grad;
  long long ld_grad;
  PreferenceRow* rows;        // [n]
  int n_parts, per_part;
  void* parts;                // [n][n_parts]
};

struct FcMx4Args {
  const uint8_t* x;
  const uint8_t* xs;
  const uint8_t* w;
  const uint8_t* ws;
  long long ld_x, ld_xs, ld_w, ld_ws, ld_y;
  const float* bias;
  int n, blocks, c_out, relu, out_bf16;
  int kt_per_split;           // K tiles per split
  void* y;
  float* partial;             // [splits][n][c_out] sums (splits > 1)
};

hipError_t launch_sample(const TokenArgs& a, bool bf16, hipStream_t s);
hipError_t launch_topk(const TokenArgs& a, bool bf16, hipStream_t s);
hipError_t launch_distill(const DistillArgs& a, bool bf16, hipStream_t s);
hipError_t launch_quantize(const void* x, bool bf16, long long ld_x, int n, int c, int8_t* q, long long ld_q,
                           float* scale, hipStream_t s);
hipError_t launch_fc_i8(const FcI8Args& a, hipStream_t s);
long long fc_i8_workspace_bytes(int n, int c_in, int c_out);
hipError_t launch_token_loss(const TokenLossArgs& a, bool bf16, hipStream_t s);
long long token_loss_workspace_bytes(int n, int n_classes);
long long preference_workspace_bytes(int n, int n_classes);
hipError_t launch_preference(const PreferenceArgs& a, bool bf16, hipStream_t s);
hipError_t launch_quantize_mx4(const void* x, bool bf16, long long ld_x, int n, int c, uint8_t* q, long long ld_q,
                               uint8_t* scale, long long ld_scale, hipStream_t s);
hipError_t launch_fc_mx4(const FcMx4Args& a, hipStream_t s);
long long fc_mx4_workspace_bytes(int n, int blocks, int c_out);

}  // namespace rafiki
