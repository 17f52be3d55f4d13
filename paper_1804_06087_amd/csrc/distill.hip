// Distillation of a teacher's top classes into a student, loss and gradient (rafiki_tokens.h).
//
// With x = z / T, K the row's teacher classes and r the other classes, the row needs the sums of
// exponentials of K and of r; then log p_j = x_j - lse and, for c outside K,
//     dz_c = T g e^(x_c - lse_r) (Q p_r - q_r),
// one exponential and one product per class; K's classes are written after the others.  Without
// rest the split is not needed and dz_c = T g Q e^(x_c - lse).  Taking r's own maximum and sum
// (K's classes are marked in a bitmap in LDS) keeps log p_r exact where p_r is small, which
// 1 - sum p_j does not.
#include "tokens.h"

#include <algorithm>

namespace rafiki {

namespace {

constexpr int kThreads = 1024;
constexpr int kWaves = kThreads / 64;
constexpr float kRestMin = 0x1p-20f;

template <bool BF16>
__device__ __forceinline__ float student(const void* p, long long i) {
  if constexpr (BF16) return __uint_as_float((uint32_t)((const bf16_t*)p)[i] << 16);
  else return ((const float*)p)[i];
}

// Rounded once, to nearest, ties to even; NaN stays NaN.
template <bool BF16>
__device__ __forceinline__ void put(void* p, long long i, float v) {
  if constexpr (BF16) ((__bf16*)p)[i] = (__bf16)v;
  else ((float*)p)[i] = v;
}

// A running maximum and the sum of exponentials below it.
struct MaxSum {
  float top, sum;
  // A NaN in t makes the sum NaN (fmaxf drops it from the maximum).
  __device__ __forceinline__ void join(float t, float s) {
    const float m = fmaxf(top, t);
    sum = sum * (top == m ? 1.f : expf(top - m)) + s * (t == m ? 1.f : expf(t - m));
    top = m;
  }
};

__device__ __forceinline__ MaxSum block_join(MaxSum v, MaxSum* waves) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) v.join(__shfl_xor(v.top, o, 64), __shfl_xor(v.sum, o, 64));
  __syncthreads();
  if ((threadIdx.x & 63) == 0) waves[threadIdx.x >> 6] = v;
  __syncthreads();
  v = waves[0];
  for (int w = 1; w < kWaves; ++w) v.join(waves[w].top, waves[w].sum);
  return v;
}

__device__ __forceinline__ float block_add(float v, float* waves) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o, 64);
  __syncthreads();
  if ((threadIdx.x & 63) == 0) waves[threadIdx.x >> 6] = v;
  __syncthreads();
  v = 0.f;
  for (int w = 0; w < kWaves; ++w) v += waves[w];
  return v;
}

// One workgroup per row.  Thread j < k holds slot j; of the slots of one class the first holds
// the class.
template <bool BF16>
__global__ __launch_bounds__(kThreads) void distill_kernel(DistillArgs a) {
  extern __shared__ uint32_t marks[];                       // rest: one bit per class
  __shared__ MaxSum wave_ms[kWaves];
  __shared__ float wave_f[kWaves];
  __shared__ int ids[kMaxTokenK];
  __shared__ float qs[kMaxTokenK];
  const int tid = threadIdx.x;
  const float inv_t = 1.f / a.t;
  for (int row = blockIdx.x; row < a.n; row += gridDim.x) {
    __syncthreads();
    const long long base = row * a.ld_row, gbase = row * a.ld_grad;
    const float g = a.grad_loss ? a.grad_loss[row] : 1.f;
    int id = -1;
    float t_logp = -INFINITY;
    if (tid < a.k) {
      id = a.labels[(long long)row * a.k + tid];
      if ((unsigned)id >= (unsigned)a.C) id = -1;
      if (id >= 0) t_logp = a.logp[(long long)row * a.k + tid];
      ids[tid] = id;
    }
    // q of this slot
    float q = expf(t_logp);
    if (!a.rest) {
      const MaxSum all = block_join(MaxSum{t_logp, id < 0 ? 0.f : t_logp == -INFINITY ? 0.f : 1.f}, wave_ms);
      const bool any = !(all.top == -INFINITY && all.sum == 0.f);
      if (!any) {                                            // no teacher: nothing to learn
        if (a.loss && tid == 0) a.loss[row] = 0.f;
        if (a.grad)
          for (int c = tid; c < a.C; c += kThreads) put<BF16>(a.grad, gbase + c, 0.f);
        continue;
      }
      q = t_logp == -INFINITY ? 0.f : expf(t_logp - all.top) / all.sum;
    }
    if (tid < a.k) qs[tid] = q;
    if (a.rest)
      for (int w = tid; w < (a.C + 31) / 32; w += kThreads) marks[w] = 0;
    __syncthreads();
    // slots of one class
    bool first = id >= 0;
    float q_class = 0.f;
    if (id >= 0)
      for (int j = 0; j < a.k; ++j)
        if (ids[j] == id) {
          if (j < tid) first = false;
          q_class += qs[j];
        }
    if (a.rest && first) atomicOr(&marks[id >> 5], 1u << (id & 31));
    __syncthreads();
    const float x_member = first ? student<BF16>(a.logits, base + id) * inv_t : -INFINITY;
    const int members = (int)block_add(first ? 1.f : 0.f, wave_f);
    const float q_sum = block_add(first ? q_class : 0.f, wave_f);
    // the sums of exponentials
    MaxSum ms{-INFINITY, 0.f};
    for (int c = tid; c < a.C; c += kThreads) {
      if (a.rest && (marks[c >> 5] >> (c & 31) & 1)) continue;
      const float x = student<BF16>(a.logits, base + c) * inv_t;
      if (x != -INFINITY) ms.join(x, 1.f);
    }
    ms = block_join(ms, wave_ms);
    const float lse_r = ms.top + logf(ms.sum);               // rest = 0: of all classes
    float lse = lse_r;
    float q_r = 0.f;
    if (a.rest) {
      MaxSum k = block_join(MaxSum{x_member, x_member == -INFINITY ? 0.f : 1.f}, wave_ms);
      k.join(ms.top, ms.sum);
      lse = k.top + logf(k.sum);
      q_r = 1.f - q_sum;
      if (q_r < kRestMin || members == a.C) q_r = 0.f;
    }
    const float big_q = a.rest ? q_sum + q_r : q_sum;
    float part = first && q_class != 0.f ? q_class * (logf(q_class) - (x_member - lse)) : 0.f;
    part = block_add(part, wave_f);
    const bool defined = lse > -INFINITY && lse < INFINITY;  // false for NaN too
    if (a.loss && tid == 0) {
      if (q_r > 0.f) part += q_r * (logf(q_r) - (lse_r - lse));
      a.loss[row] = defined ? a.t * a.t * part : NAN;
    }
    if (!a.grad) continue;
    const float scale = defined ? a.t * g : NAN;
    if (g == 0.f) {
      for (int c = tid; c < a.C; c += kThreads) put<BF16>(a.grad, gbase + c, 0.f);
      continue;
    }
    const float p_r = a.rest ? expf(lse_r - lse) : 1.f;
    const float factor = scale * (p_r == 0.f ? 0.f : big_q * p_r - q_r);   // NaN stays
    for (int c = tid; c < a.C; c += kThreads) {
      const float x = student<BF16>(a.logits, base + c) * inv_t;
      put<BF16>(a.grad, gbase + c, x == -INFINITY && defined ? 0.f : factor * expf(x - lse_r));
    }
    __syncthreads();
    if (first) put<BF16>(a.grad, gbase + id, scale * (big_q * expf(x_member - lse) - q_class));
  }
}

}  // namespace

hipError_t launch_distill(const DistillArgs& a, bool bf16, hipStream_t s) {
  const size_t lds = a.rest ? (size_t)(a.C + 31) / 32 * 4 : 0;
  const dim3 grid((unsigned)std::min(a.n, 1 << 20));
  if (bf16) hipLaunchKernelGGL(distill_kernel<true>, grid, dim3(kThreads), lds, s, a);
  else hipLaunchKernelGGL(distill_kernel<false>, grid, dim3(kThreads), lds, s, a);
  return hipGetLastError();
}

}  // namespace rafiki
