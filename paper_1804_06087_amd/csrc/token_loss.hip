// Log-probabilities of given tokens, the clipped policy loss and the preference loss with their
// gradients (rafiki_tokens.h).
//
// With y_c = z_c s, s = log2(e) / T, l the row's label and the sums over all classes but l:
//     R = sum 2^(y_c - r),  r their maximum,   S = R 2^(r - t) + 2^(y_l - t),  t = max(r, y_l),
//     1 - p_l = R 2^(r - t) / S,   log p_l = - log(1 + R 2^(r - y_l))  (y_l > r; otherwise y_l - r - log(R + 2^(y_l - r))),
// which keeps 1 - p_l and log p_l exact where p_l is near 1: a sum over all classes would have lost the others'.
// The gradient is affine in log p under p:  dz_c = 2^(y_c - r) (f + f' (y_c - r)) for c != l, with f' = 0 without entropy.
#include "tokens.h"

#include <algorithm>

namespace rafiki {

namespace {

constexpr float kLn2 = 0.693147180559945f, kLog2e = 1.44269504088896f;

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4_any __attribute__((ext_vector_type(4), aligned(2)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef float f32x2 __attribute__((ext_vector_type(2)));

__device__ __forceinline__ float power2(float t) { return __builtin_amdgcn_exp2f(t); }

template <bool BF16>
__device__ __forceinline__ float element(const void* p, long long i) {
  if constexpr (BF16) return __uint_as_float((uint32_t)((const bf16_t*)p)[i] << 16);
  else return ((const float*)p)[i];
}
// Rounded once, to nearest, ties to even; NaN stays NaN.
template <bool BF16>
__device__ __forceinline__ void put(void* p, long long i, float v) {
  if constexpr (BF16) ((__bf16*)p)[i] = (__bf16)v;
  else ((float*)p)[i] = v;
}
template <bool BF16, int V>
__device__ __forceinline__ void unpack(u32x4 q, float z[V]) {
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    if constexpr (BF16) {
      z[2 * j] = __uint_as_float(q[j] << 16);
      z[2 * j + 1] = __uint_as_float(q[j] & 0xFFFF0000u);
    } else {
      z[j] = __uint_as_float(q[j]);
    }
  }
}
template <bool BF16, int V>
__device__ __forceinline__ u32x4 pack(const float z[V]) {
  u32x4 q;
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    if constexpr (BF16) q[j] = __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2{z[2 * j], z[2 * j + 1]}, bf16x2));
    else q[j] = __float_as_uint(z[j]);
  }
  return q;
}

__device__ __forceinline__ float wave_max(float v) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) v = fmaxf(v, __shfl_xor(v, o, 64));
  return v;
}
template <typename T>
__device__ __forceinline__ T wave_add(T v) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o, 64);
  return v;
}

// The maximum as a reference for powers: an empty row has none and takes 0.
__device__ __forceinline__ float reference(float top) { return top == -INFINITY ? 0.f : top; }
// Exponents of 2 as factors of a power that is 0 below here: -inf would make it NaN.
__device__ __forceinline__ float finite_log2(float x) { return fmaxf(x, -16384.f); }

// A row of C values as chunks of 16 bytes, chunk i from class i V on; the last one, of fewer values, is read from
// class C - V on.  Rows may start anywhere.
template <bool BF16>
struct Row {
  static constexpr int V = BF16 ? 8 : 4;
  const char* x;
  int C, chunks, label;

  __device__ __forceinline__ void init(const void* logits, long long base, int C_, int label_) {
    x = (const char*)logits + base * (16 / V);
    C = C_;
    chunks = (C + V - 1) / V;
    label = label_;
  }
  // Chunk i with -inf in the label's place and in those of classes that it does not have.
  template <bool STREAM>
  __device__ __forceinline__ u32x4 load(int i) const {
    const int c0 = i * V;
    const bool short_chunk = c0 + V > C;
    u32x4 q;
    if (!short_chunk || C >= V) {
      const u32x4_any* p = (const u32x4_any*)(x + (long long)(short_chunk ? C - V : c0) * (16 / V));
      if constexpr (STREAM) q = __builtin_nontemporal_load(p);
      else q = *p;
    }
    if (short_chunk || (unsigned)(label - c0) < (unsigned)V) {
      float z[V];
      if (short_chunk) {
        const int n = C - c0;                                // its classes: the last n of the V that were read
        float t[V];
        if (C >= V) {
          unpack<BF16, V>(q, t);
        } else {
#pragma unroll
          for (int j = 0; j < V; ++j) t[j] = j >= V - n ? element<BF16>(x, j - (V - n)) : -INFINITY;
        }
#pragma unroll
        for (int j = 0; j < V; ++j) {
          z[j] = -INFINITY;
#pragma unroll
          for (int k = 0; k < V; ++k) z[j] = k == j + V - n ? t[k] : z[j];
        }
      } else {
        unpack<BF16, V>(q, z);
      }
#pragma unroll
      for (int j = 0; j < V; ++j) z[j] = c0 + j == label ? -INFINITY : z[j];
      q = pack<BF16, V>(z);
    }
    return q;
  }
  // Chunk i of a row of values; the label's is `at_label`.
  __device__ __forceinline__ void store(char* row, int i, float d[V], float at_label) const {
    const int c0 = i * V;
    if ((unsigned)(label - c0) < (unsigned)V) {
#pragma unroll
      for (int j = 0; j < V; ++j) d[j] = c0 + j == label ? at_label : d[j];
    }
    if (c0 + V <= C) {
      __builtin_nontemporal_store(pack<BF16, V>(d), (u32x4_any*)(row + (long long)c0 * (16 / V)));
    } else {
#pragma unroll
      for (int j = 0; j < V; ++j)
        if (c0 + j < C) put<BF16>(row, c0 + j, d[j]);
    }
  }
  template <int NT>
  __device__ __forceinline__ void zero(char* row) const {
    for (int i = threadIdx.x; i < chunks; i += NT) {
      float d[V];
#pragma unroll
      for (int j = 0; j < V; ++j) d[j] = 0.f;
      store(row, i, d, 0.f);
    }
  }
};

// Sums over classes: 2^(y - top), and of those times (y - top).
struct Sums {
  float top, sum, moment;
};
template <int V, bool ENT>
__device__ __forceinline__ void add_chunk(Sums& a, const float z[V], float s) {
  float now = a.top;
#pragma unroll
  for (int j = 0; j < V; ++j) now = fmaxf(now, z[j]);
  const float ref = reference(now), step = (a.top - ref) * s, grown = power2(step);
  if constexpr (ENT) a.moment = (a.moment + a.sum * finite_log2(step)) * grown;
  a.sum *= grown;
#pragma unroll
  for (int j = 0; j < V; ++j) {
    const float x = (z[j] - ref) * s, e = power2(x);
    a.sum += e;
    if constexpr (ENT) a.moment += e * finite_log2(x);
  }
  a.top = now;
}
// The workgroup's sums in every thread (a barrier).
template <int NW, bool ENT>
__device__ __forceinline__ Sums join(Sums a, float s, Sums (&waves)[NW]) {
  auto to = [&](Sums v, float ref) {
    const float step = (v.top - ref) * s, grown = v.sum == 0.f ? 0.f : power2(step);
    if (ENT) v.moment = (v.moment + v.sum * finite_log2(step)) * grown;
    v.sum *= grown;
    return v;
  };
  const float all = wave_max(a.top);
  a = to(a, reference(all));
  a.sum = wave_add(a.sum);
  if (ENT) a.moment = wave_add(a.moment);
  a.top = all;
  if ((threadIdx.x & 63) == 0) waves[threadIdx.x >> 6] = a;
  __syncthreads();
  float top = -INFINITY;
#pragma unroll
  for (int w = 0; w < NW; ++w) top = fmaxf(top, waves[w].top);
  Sums r{top, 0.f, 0.f};
#pragma unroll
  for (int w = 0; w < NW; ++w) {
    const Sums v = to(waves[w], reference(top));
    r.sum += v.sum;
    r.moment += v.moment;
  }
  return r;
}

// What a row's sums and its label's logit say.
struct RowFacts {
  double logp;
  float entropy;
  float rest, p, share;       // 1 - p of the label, p of the label, p of the class at the others' maximum
  float log2_share;           // log2 of the last (finite)
  bool defined;
};
template <bool ENT>
__device__ __forceinline__ RowFacts row_facts(const Sums& r, float z, float s, double inv_t) {
  RowFacts f;
  const float top = reference(r.top), t = reference(fmaxf(r.top, z));
  const float down = finite_log2((top - t) * s), x = finite_log2((z - t) * s);
  const float e_r = r.sum == 0.f ? 0.f : power2(down), e_y = power2((z - t) * s);
  const float part = r.sum * e_r, total = part + e_y;
  f.defined = total > 0.f && total < INFINITY && t < INFINITY;
  f.rest = part / total;
  f.p = e_y / total;
  f.share = e_r / total;
  const float log2_total = log2f(total);
  f.log2_share = down - log2_total;
  f.entropy = ENT ? kLn2 * (log2_total - ((r.moment + r.sum * down) * e_r + e_y * x) / total) : 0.f;
  // log p in 64 bits: the difference of two logits may exceed fp32, and what follows subtracts it
  const double D = ((double)z - (double)top) * inv_t;
  if (r.sum == 0.f) f.logp = 0.0;
  else if (D > 0) f.logp = -log1p((double)(r.sum * expf((float)-D)));
  else f.logp = D - log((double)r.sum + (double)expf((float)D));
  if (!f.defined) {
    f.logp = NAN;
    f.entropy = NAN;
  }
  return f;
}

// What the gradient pass needs: dz = 2^x (f0 + f1 x) with x = (z - top) s, and the label's.
struct RowGrad {
  float f0, f1, at_label;
};
template <bool ENT>
__device__ __forceinline__ RowGrad row_grad(const RowFacts& f, float a, float h, float inv_t) {
  if (!f.defined || !(fabsf(a) < INFINITY) || h != h) return RowGrad{NAN, 0.f, NAN};
  const float share = f.share * inv_t;
  RowGrad g{share * -a, 0.f, a * f.rest * inv_t};
  if (ENT) {
    g.f0 = share * (-a - h * (kLn2 * f.log2_share + f.entropy));
    g.f1 = -share * h * kLn2;
    if (f.p > 0.f) g.at_label -= h * f.p * ((float)f.logp + f.entropy) * inv_t;
  }
  return g;
}

// One workgroup of NT threads per row.  CH > 0: the row, of at most NT CH chunks, stays in registers from its sums to its
// gradient, so that it is read once; CH = 0: any length, read again for the gradient.
template <bool BF16, bool POLICY, bool ENT, int NT, int CH>
__global__ __launch_bounds__(NT) void token_loss_kernel(TokenLossArgs a) {
  constexpr int V = Row<BF16>::V, NW = NT / 64;
  __shared__ Sums waves[NW];
  __shared__ RowGrad shared_grad;
  const int row = a.row0 + blockIdx.x, tid = threadIdx.x;
  const int label = a.labels[row];
  const bool token = (unsigned)label < (unsigned)a.C;
  const float g = POLICY && a.grad_loss ? a.grad_loss[row] : 1.f;
  const float a_in = !POLICY && a.grad_logp ? a.grad_logp[row] : 0.f;
  const float h_in = !POLICY && a.grad_entropy ? a.grad_entropy[row] : 0.f;
  const bool weightless = POLICY ? g == 0.f : a_in == 0.f && h_in == 0.f;
  const bool outputs = a.loss || a.logp || a.kl || a.entropy;
  Row<BF16> r;
  r.init(a.logits, row * a.ld_row, a.C, label);
  char* const d_row = (char*)a.grad + row * a.ld_grad * (16 / V);
  if (a.grad && (!token || weightless)) r.template zero<NT>(d_row);
  if (!token) {
    if (tid == 0) {
      if (a.loss) a.loss[row] = 0.f;
      if (a.logp) a.logp[row] = 0.f;
      if (a.kl) a.kl[row] = 0.f;
      if (a.entropy) a.entropy[row] = 0.f;
    }
    return;
  }
  if (weightless && !outputs) return;

  u32x4 held[CH > 0 ? CH : 1];
  const u32x4 masked = BF16 ? u32x4{0xFF80FF80u, 0xFF80FF80u, 0xFF80FF80u, 0xFF80FF80u}
                            : u32x4{0xFF800000u, 0xFF800000u, 0xFF800000u, 0xFF800000u};
  Sums sums{-INFINITY, 0.f, 0.f};
  if constexpr (CH > 0) {
#pragma unroll
    for (int i = 0; i < CH; ++i) {
      held[i] = masked;
      if (i * NT + tid < r.chunks) held[i] = r.template load<true>(i * NT + tid);
    }
  }
  const float z_label = element<BF16>(r.x, label);
  float z[V];
  if constexpr (CH > 0) {
#pragma unroll
    for (int i = 0; i < CH; ++i) {
      unpack<BF16, V>(held[i], z);
      add_chunk<V, ENT>(sums, z, a.s);
      __builtin_amdgcn_sched_barrier(0);
    }
  } else {
    constexpr int UN = 4;
    for (int i0 = tid; i0 < r.chunks; i0 += NT * UN) {
      u32x4 q[UN];
#pragma unroll
      for (int u = 0; u < UN; ++u) {
        q[u] = masked;
        if (i0 + u * NT < r.chunks) q[u] = r.template load<true>(i0 + u * NT);
      }
#pragma unroll
      for (int u = 0; u < UN; ++u) {
        unpack<BF16, V>(q[u], z);
        add_chunk<V, ENT>(sums, z, a.s);
      }
    }
  }
  sums = join<NW, ENT>(sums, a.s, waves);
  if (tid < 64) {
    const RowFacts f = row_facts<ENT>(sums, z_label, a.s, a.inv_t);
    float da = a_in, dh = h_in;
    if constexpr (POLICY) {
      // 64 bits: r and exp(d) are powers of differences, and kl is what is left of them
      double loss = 0.0, kl = 0.0, slope = 0.0;
      const double A = a.advantage[row];
      if (A != 0.0) {
        const double ratio = a.old_logp ? (double)(float)exp(f.logp - (double)a.old_logp[row]) : f.logp == f.logp ? 1.0 : f.logp;
        const double kept = fmin(fmax(ratio, 1.0 - (double)a.clip_low), 1.0 + (double)a.clip_high);
        const double plain = ratio * A, cut = kept * A;
        loss = plain != plain ? plain : -fmin(plain, cut);
        slope = plain != plain ? plain : plain <= cut ? -plain : 0.0;
      }
      if (a.ref_logp) {
        const double d = (double)a.ref_logp[row] - f.logp, e = (double)(float)exp(d);
        kl = e < INFINITY || d != d ? expm1(d) - d : INFINITY;
        if (a.kl_coef != 0.f) {
          loss += (double)a.kl_coef * kl;
          slope -= (double)a.kl_coef * (e < INFINITY || d != d ? expm1(d) : INFINITY);
        }
      }
      if (a.entropy_coef != 0.f) loss -= (double)a.entropy_coef * (double)f.entropy;
      if (!f.defined) loss = NAN;
      if (tid == 0) {
        if (a.loss) a.loss[row] = (float)loss;
        if (a.kl) a.kl[row] = f.defined ? (float)kl : NAN;
      }
      da = loss != loss ? NAN : g * (float)slope;
      dh = g * -a.entropy_coef;
    }
    if (tid == 0) {
      if (a.logp) a.logp[row] = (float)f.logp;
      if (a.entropy) a.entropy[row] = f.entropy;
      shared_grad = row_grad<ENT>(f, da, dh, (float)a.inv_t);
    }
  }
  if (!a.grad || weightless) return;
  __syncthreads();
  const RowGrad d = shared_grad;
  const float top = reference(sums.top);
  auto gradient = [&](u32x4 q, int i) {
    unpack<BF16, V>(q, z);
#pragma unroll
    for (int j = 0; j < V; ++j) {
      const float x = (z[j] - top) * a.s;
      z[j] = power2(x) * (ENT ? d.f0 + d.f1 * finite_log2(x) : d.f0);
    }
    r.store(d_row, i, z, d.at_label);
  };
  if constexpr (CH > 0) {
#pragma unroll
    for (int i = 0; i < CH; ++i) {
      // opaque here, or the compiler keeps the first pass's unpacked values
      asm volatile("" : "+v"(held[i][0]), "+v"(held[i][1]), "+v"(held[i][2]), "+v"(held[i][3]));
      if (i * NT + tid < r.chunks) gradient(held[i], i * NT + tid);
      __builtin_amdgcn_sched_barrier(0);
    }
  } else {
    for (int i = tid; i < r.chunks; i += NT) gradient(r.template load<true>(i), i);
  }
}

// ---------------------------------------------------------------- preference

// A sequence's rows [first, last), inside [0, n] whatever the offsets hold.
__device__ __forceinline__ int offset_at(const PreferenceArgs& a, int i) {
  const long long at = a.offsets ? a.offsets[i] : (long long)a.n / (2 * a.pairs) * i;
  return (int)(at < 0 ? 0 : at > a.n ? a.n : at);
}

template <bool BF16, int NT>
__global__ __launch_bounds__(NT) void preference_stats_kernel(PreferenceArgs a) {
  constexpr int V = Row<BF16>::V, NW = NT / 64, UN = 4;
  __shared__ Sums waves[NW];
  const int row = a.row0 + blockIdx.x, tid = threadIdx.x;
  if (row < offset_at(a, 0) || row >= offset_at(a, 2 * a.pairs)) return;
  const int label = a.labels[row];
  if ((unsigned)label >= (unsigned)a.C) return;
  Row<BF16> r;
  r.init(a.logits, row * a.ld_row, a.C, label);
  const u32x4 masked = BF16 ? u32x4{0xFF80FF80u, 0xFF80FF80u, 0xFF80FF80u, 0xFF80FF80u}
                            : u32x4{0xFF800000u, 0xFF800000u, 0xFF800000u, 0xFF800000u};
  const float z_label = element<BF16>(r.x, label);
  Sums sums{-INFINITY, 0.f, 0.f};
  for (int i0 = tid; i0 < r.chunks; i0 += NT * UN) {
    u32x4 q[UN];
#pragma unroll
    for (int u = 0; u < UN; ++u) {
      q[u] = masked;
      if (i0 + u * NT < r.chunks) q[u] = r.template load<false>(i0 + u * NT);
    }
#pragma unroll
    for (int u = 0; u < UN; ++u) {
      float z[V];
      unpack<BF16, V>(q[u], z);
      add_chunk<V, false>(sums, z, a.s);
    }
  }
  sums = join<NW, false>(sums, a.s, waves);
  if (tid < 64) {
    const RowFacts f = row_facts<false>(sums, z_label, a.s, a.inv_t);
    if (tid == 0) {
      PreferenceRow& out = a.rows[row];
      out.delta = f.logp - (a.ref_logp ? (double)a.ref_logp[row] : 0.0);
      out.top = reference(sums.top);
      out.share = f.defined ? f.share : NAN;
      out.rest = f.defined ? f.rest : NAN;
    }
  }
}

// One workgroup per pair: its answers' sums in 64 bits (a thread's rows in their order, then a tree, the same every
// time), the loss, and every row's weight.
__global__ __launch_bounds__(256) void preference_pairs_kernel(PreferenceArgs a) {
  __shared__ double sums[2][4];
  __shared__ int counts[2][4];
  const int p = blockIdx.x, tid = threadIdx.x;
  int at[3];
#pragma unroll
  for (int k = 0; k < 3; ++k) at[k] = offset_at(a, 2 * p + k);
  auto token = [&](int row) { return (unsigned)a.labels[row] < (unsigned)a.C; };
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    double sum = 0.0;
    int count = 0;
    for (int row = at[k] + tid; row < at[k + 1]; row += 256)
      if (token(row)) {
        sum += a.rows[row].delta;
        ++count;
      }
    sum = wave_add(sum);
    count = wave_add(count);
    if ((tid & 63) == 0) {
      sums[k][tid >> 6] = sum;
      counts[k][tid >> 6] = count;
    }
  }
  __syncthreads();
  double score[2], per[2];
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    const int count = counts[k][0] + counts[k][1] + counts[k][2] + counts[k][3];
    per[k] = a.mean && count ? 1.0 / count : 1.0;
    score[k] = (double)a.beta * ((sums[k][0] + sums[k][1] + sums[k][2] + sums[k][3]) * per[k]);
  }
  const double u = score[0] - score[1], smooth = a.smoothing;
  const double soft = log1p(exp(-fabs(u))), up = u > 0 ? 1 / (1 + exp(-u)) : exp(u) / (1 + exp(u));   // sigmoid(u)
  const double down = u > 0 ? exp(-u) / (1 + exp(-u)) : 1 / (1 + exp(u));                            // sigmoid(-u)
  if (tid == 0) {
    double loss = (1 - smooth) * (soft + (u < 0 ? -u : 0.0));
    if (smooth > 0) loss += smooth * (soft + (u > 0 ? u : 0.0));
    if (a.loss) a.loss[p] = u == u ? (float)loss : NAN;
    if (a.scores) {
      a.scores[2 * p] = (float)score[0];
      a.scores[2 * p + 1] = (float)score[1];
    }
  }
  if (!a.grad) return;
  const double g = a.grad_loss ? (double)a.grad_loss[p] : 1.0;
  const double du = g == 0 ? 0.0 : (double)a.beta * g * (smooth * up - (1 - smooth) * down);
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    const float weight = (float)((k ? -du : du) * per[k] * a.inv_t);
    for (int row = at[k] + tid; row < at[k + 1]; row += 256) a.rows[row].weight = token(row) ? weight : 0.f;
  }
}

template <bool BF16, int NT>
__global__ __launch_bounds__(NT) void preference_grad_kernel(PreferenceArgs a) {
  constexpr int V = Row<BF16>::V;
  const int row = a.row0 + blockIdx.x, tid = threadIdx.x;
  if (row < offset_at(a, 0) || row >= offset_at(a, 2 * a.pairs)) return;
  const PreferenceRow f = a.rows[row];
  Row<BF16> r;
  r.init(a.logits, row * a.ld_row, a.C, a.labels[row]);
  char* const d_row = (char*)a.grad + row * a.ld_grad * (16 / V);
  if (f.weight == 0.f) return r.template zero<NT>(d_row);
  const float factor = -f.weight * f.share, at_label = f.weight * f.rest;
  for (int i = tid; i < r.chunks; i += NT) {
    float z[V];
    unpack<BF16, V>(r.template load<false>(i), z);
#pragma unroll
    for (int j = 0; j < V; ++j) z[j] = factor * power2((z[j] - f.top) * a.s);
    r.store(d_row, i, z, at_label);
  }
}

// 2^20 rows a launch at most.
template <typename Args, typename F>
hipError_t launch_row_ranges(const Args& a, F&& launch_rows) {
  Args part = a;
  for (long long row = 0; row < a.n; row += 1 << 20) {
    part.row0 = (int)row;
    launch_rows(part, dim3((unsigned)std::min<long long>(a.n - row, 1 << 20)));
    const hipError_t st = hipGetLastError();
    if (st != hipSuccess) return st;
  }
  return hipSuccess;
}

template <bool BF16, bool POLICY, bool ENT, int NT, int CH>
hipError_t launch_loss_rows(const TokenLossArgs& a, hipStream_t s) {
  return launch_row_ranges(a, [&](const TokenLossArgs& part, dim3 grid) {
    launch(token_loss_kernel<BF16, POLICY, ENT, NT, CH>, grid, dim3(NT), s, part);
  });
}

template <bool BF16, bool POLICY, bool ENT>
hipError_t launch_loss_by_length(const TokenLossArgs& a, hipStream_t s) {
  const int chunks = (a.C + Row<BF16>::V - 1) / Row<BF16>::V;
  if (!a.grad) {
    if (chunks <= 128 * 4) return launch_loss_rows<BF16, POLICY, ENT, 128, 0>(a, s);
    if (chunks <= 256 * 16) return launch_loss_rows<BF16, POLICY, ENT, 256, 0>(a, s);
    return launch_loss_rows<BF16, POLICY, ENT, 1024, 0>(a, s);
  }
  if (chunks <= 128 * 2) return launch_loss_rows<BF16, POLICY, ENT, 128, 2>(a, s);
  if (chunks <= 128 * 8) return launch_loss_rows<BF16, POLICY, ENT, 128, 8>(a, s);
  if (chunks <= 256 * 8) return launch_loss_rows<BF16, POLICY, ENT, 256, 8>(a, s);
  if (chunks <= 256 * 16) return launch_loss_rows<BF16, POLICY, ENT, 256, 16>(a, s);
  if (chunks <= 512 * 16) return launch_loss_rows<BF16, POLICY, ENT, 512, 16>(a, s);
  if (chunks <= 1024 * 16) return launch_loss_rows<BF16, POLICY, ENT, 1024, 16>(a, s);
  if (chunks <= 1024 * 20) return launch_loss_rows<BF16, POLICY, ENT, 1024, 20>(a, s);
  return launch_loss_rows<BF16, POLICY, ENT, 1024, 0>(a, s);
}

template <bool BF16>
hipError_t launch_loss(const TokenLossArgs& a, hipStream_t s) {
  const bool ent = a.entropy || a.grad_entropy || a.entropy_coef != 0.f;
  if (a.policy) return ent ? launch_loss_by_length<BF16, true, true>(a, s) : launch_loss_by_length<BF16, true, false>(a, s);
  return ent ? launch_loss_by_length<BF16, false, true>(a, s) : launch_loss_by_length<BF16, false, false>(a, s);
}

template <bool BF16>
hipError_t launch_preference_of(const PreferenceArgs& a, hipStream_t s) {
  hipError_t st = launch_row_ranges(a, [&](const PreferenceArgs& part, dim3 grid) {
    launch(preference_stats_kernel<BF16, 256>, grid, dim3(256), s, part);
  });
  if (st != hipSuccess) return st;
  launch(preference_pairs_kernel, dim3(a.pairs), dim3(256), s, a);
  st = hipGetLastError();
  if (st != hipSuccess || !a.grad) return st;
  return launch_row_ranges(a, [&](const PreferenceArgs& part, dim3 grid) {
    launch(preference_grad_kernel<BF16, 256>, grid, dim3(256), s, part);
  });
}

}  // namespace

hipError_t launch_token_loss(const TokenLossArgs& a, bool bf16, hipStream_t s) {
  return bf16 ? launch_loss<true>(a, s) : launch_loss<false>(a, s);
}

hipError_t launch_preference(const PreferenceArgs& a, bool bf16, hipStream_t s) {
  return bf16 ? launch_preference_of<true>(a, s) : launch_preference_of<false>(a, s);
}

}  // namespace rafiki
