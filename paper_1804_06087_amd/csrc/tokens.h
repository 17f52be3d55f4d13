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

hipError_t launch_sample(const TokenArgs& a, bool bf16, hipStream_t s);
hipError_t launch_topk(const TokenArgs& a, bool bf16, hipStream_t s);
hipError_t launch_distill(const DistillArgs& a, bool bf16, hipStream_t s);
hipError_t launch_quantize(const void* x, bool bf16, long long ld_x, int n, int c, int8_t* q, long long ld_q,
                           float* scale, hipStream_t s);
hipError_t launch_fc_i8(const FcI8Args& a, hipStream_t s);
long long fc_i8_workspace_bytes(int n, int c_in, int c_out);

}  // namespace rafiki
