// Answers over a vocabulary: drawing from an ensemble's combined distribution and listing
// its likeliest classes (rafiki_tokens.h).
//
// The combined probability of class c is p_c = sum_m exp((z_mc - M_m) / T) / (S s_m), with M_m the
// row's maximum and s_m the sum of its exponentials.  Which class is drawn or ranked where
// depends on comparisons of such sums, so everything is taken in 64 bits: MI355X issues a
// 64-bit FMA at the rate of a 32-bit one, and an exponential of about 18 of them costs a
// row no more time than its bytes.  Sums that are compared are sums of integers
// P_c = floor(p_c 2^62), which do not depend on their order, so LDS atomics may add them.
//
// Two launches: the statistics of every group of 256 classes (a wave each), then one
// workgroup per row.
#include "tokens.h"

#include <algorithm>

namespace rafiki {

namespace {

typedef unsigned long long u64;

constexpr int kRowThreads = 1024;
constexpr int kRowWaves = kRowThreads / 64;
constexpr double kUnit = 4611686018427387904.0;            // 2^62
constexpr u64 kLeastKey = (u64)(1023 - 1000) << 52;         // bits of 2^-1000

// e^x for x <= 0 (also -inf; NaN stays NaN): x = n ln 2 + r, |r| <= ln 2 / 2, and the Taylor
// polynomial of e^r to r^12 / 12! (the next term is below 2e-16).
__device__ __forceinline__ double exp_nonpos(double x) {
  x = x < -1100.0 ? -1100.0 : x;
  const double n = __builtin_rint(x * 1.4426950408889634);
  double r = __builtin_fma(-n, 2977044471.0 / 4294967296.0, x);   // ln 2 in two parts: 32 bits, so that
  r = __builtin_fma(-n, 1.9082149292705877e-10, r);          // n times it is exact, and the rest
  double y = 1.0 / 479001600;
  y = __builtin_fma(y, r, 1.0 / 39916800);
  y = __builtin_fma(y, r, 1.0 / 3628800);
  y = __builtin_fma(y, r, 1.0 / 362880);
  y = __builtin_fma(y, r, 1.0 / 40320);
  y = __builtin_fma(y, r, 1.0 / 5040);
  y = __builtin_fma(y, r, 1.0 / 720);
  y = __builtin_fma(y, r, 1.0 / 120);
  y = __builtin_fma(y, r, 1.0 / 24);
  y = __builtin_fma(y, r, 1.0 / 6);
  y = __builtin_fma(y, r, 0.5);
  y = __builtin_fma(y, r, 1.0);
  y = __builtin_fma(y, r, 1.0);
  return __builtin_ldexp(y, (int)n);
}

template <bool BF16>
__device__ __forceinline__ float logit(const void* p, long long i) {
  if constexpr (BF16) return __uint_as_float((uint32_t)((const bf16_t*)p)[i] << 16);
  else return ((const float*)p)[i];
}

// Row i's temperature; 0 and what is no temperature are told apart by the row kernel.
__device__ __forceinline__ float row_temperature(const TokenArgs& a, int row) {
  return a.temperature ? a.temperature[row] : a.t_all;
}
// T = 0 ranks at T = 1.
__device__ __forceinline__ double inverse_temperature(float t) { return t == 0.f ? 1.0 : 1.0 / (double)t; }

// exp((z - top) / T); a masked class has 0 also at T = +inf, where inv is 0.
__device__ __forceinline__ double weight(float z, float top, double inv) {
  return z == -INFINITY ? 0.0 : exp_nonpos(((double)z - (double)top) * inv);
}

// ---------------------------------------------------------------- group statistics
template <bool BF16>
__global__ __launch_bounds__(256) void group_stats_kernel(TokenArgs a) {
  const int lane = threadIdx.x & 63;
  const long long total = (long long)a.n * a.S * a.groups;
  for (long long id = (long long)blockIdx.x * 4 + (threadIdx.x >> 6); id < total; id += (long long)gridDim.x * 4) {
    const int g = (int)(id % a.groups);
    const long long rm = id / a.groups;
    const int m = (int)(rm % a.S), row = (int)(rm / a.S);
    const double inv = inverse_temperature(row_temperature(a, row));
    const long long base = m * a.ld_model + row * a.ld_row;
    float z[4];
    float top = -INFINITY;
    bool bad = false;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int c = g * kGroupClasses + j * 64 + lane;
      z[j] = c < a.C ? logit<BF16>(a.logits, base + c) : -INFINITY;
      bad |= z[j] != z[j];
      top = fmaxf(top, z[j]);
    }
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor(top, o, 64));
    if (__ballot(bad)) top = NAN;
    double sum = 0.0;
    if (top > -INFINITY && top < INFINITY) {
#pragma unroll
      for (int j = 0; j < 4; ++j) sum += weight(z[j], top, inv);
    }
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) sum += __shfl_xor(sum, o, 64);
    if (lane == 0) a.stats[id] = GroupStat{sum, top, 0.f};
  }
}

// ---------------------------------------------------------------- one workgroup per row
struct RowShared {
  float top[kMaxTokenModels];
  double scale[kMaxTokenModels];    // 1 / (S s_m)
  u64 sums[2048];
  uint32_t counts[2048];
  u64 wave_a[kRowWaves], wave_b[kRowWaves];
  double wave_d[kRowWaves];
  float wave_f[kRowWaves];
  u64 found_key, found_count, found_sum;
  int found_class;
  uint32_t n_list;
  u64 list_key[kMaxTokenK];
  int list_class[kMaxTokenK];
};

__device__ __forceinline__ u64 block_sum(u64 v, u64* waves) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o, 64);
  __syncthreads();
  if ((threadIdx.x & 63) == 0) waves[threadIdx.x >> 6] = v;
  __syncthreads();
  u64 t = 0;
#pragma unroll
  for (int w = 0; w < kRowWaves; ++w) t += waves[w];
  return t;
}

// Sum of v over the threads before this one; total = the sum over all.
__device__ __forceinline__ u64 block_scan(u64 v, u64* waves, u64& total) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  u64 s = v;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const u64 t = __shfl_up(s, o, 64);
    if (lane >= o) s += t;
  }
  __syncthreads();
  if (lane == 63) waves[wave] = s;
  __syncthreads();
  u64 before = 0;
  total = 0;
#pragma unroll
  for (int w = 0; w < kRowWaves; ++w) {
    if (w < wave) before += waves[w];
    total += waves[w];
  }
  return before + s - v;
}

template <bool BF16>
struct Row {
  const TokenArgs& a;
  RowShared& sh;
  long long base;
  double inv;

  // Joins the groups' statistics; 0: a distribution, 1: a model without a class above -inf,
  // 2: NaN or +inf somewhere.
  __device__ int init(int row) {
    base = row * a.ld_row;
    int state = 0;
    for (int m = 0; m < a.S; ++m) {
      const GroupStat* st = a.stats + ((long long)row * a.S + m) * a.groups;
      float top = -INFINITY;
      bool bad = false;
      for (int g = threadIdx.x; g < a.groups; g += kRowThreads) {
        const float t = st[g].top;
        bad |= !(t < INFINITY);
        top = fmaxf(top, t);
      }
#pragma unroll
      for (int o = 32; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor(top, o, 64));
      if (__ballot(bad)) top = INFINITY;
      __syncthreads();
      if ((threadIdx.x & 63) == 0) sh.wave_f[threadIdx.x >> 6] = top;
      __syncthreads();
      top = -INFINITY;
#pragma unroll
      for (int w = 0; w < kRowWaves; ++w) top = fmaxf(top, sh.wave_f[w]);
      if (top == INFINITY) return 2;
      if (top == -INFINITY) { state = 1; continue; }
      double s = 0.0;
      for (int g = threadIdx.x; g < a.groups; g += kRowThreads) s += st[g].sum * weight(st[g].top, top, inv);
#pragma unroll
      for (int o = 32; o > 0; o >>= 1) s += __shfl_xor(s, o, 64);
      if ((threadIdx.x & 63) == 0) sh.wave_d[threadIdx.x >> 6] = s;
      __syncthreads();
      s = 0.0;
#pragma unroll
      for (int w = 0; w < kRowWaves; ++w) s += sh.wave_d[w];
      if (threadIdx.x == 0) {
        sh.top[m] = top;
        sh.scale[m] = 1.0 / (s * a.S);
      }
    }
    __syncthreads();
    return state;
  }

  // Bits of p_c (they order as p_c does), 0 for a class without a probability.
  __device__ u64 key(int c) const {
    double p = 0.0;
    for (int m = 0; m < a.S; ++m)
      p = __builtin_fma(weight(logit<BF16>(a.logits, base + m * a.ld_model + c), sh.top[m], inv), sh.scale[m], p);
    const u64 k = (u64)__double_as_longlong(p);
    return k < kLeastKey ? 0 : k;
  }
  static __device__ u64 units(u64 k) { return (u64)(__longlong_as_double((long long)k) * kUnit); }

  // The cut of the ranking: the key at which the number (by_sum: the sum of P) of the classes
  // from the top reaches `target`, by digits of the key from the highest down; above_n and
  // above_sum are those of the larger keys.  False where the whole row stays below target.
  __device__ bool select(bool by_sum, u64 target, u64& cut, u64& above_n, u64& above_sum) {
    constexpr int kShift[6] = {52, 41, 30, 20, 10, 0};
    cut = above_n = above_sum = 0;
    for (int level = 0; level < 6; ++level) {
      const int shift = kShift[level], width = level < 3 ? 11 : 10;
      __syncthreads();
      for (int b = threadIdx.x; b < 2048; b += kRowThreads) {
        sh.sums[b] = 0;
        sh.counts[b] = 0;
      }
      __syncthreads();
      const int up = shift + width;
      for (int c = threadIdx.x; c < a.C; c += kRowThreads) {
        const u64 k = key(c);
        if (k != 0 && k >> up == cut >> up) {
          const int d = (int)(k >> shift) & 2047 & ((1 << width) - 1);
          atomicAdd(&sh.sums[d], units(k));
          atomicAdd(&sh.counts[d], 1u);
        }
      }
      __syncthreads();
      // thread t holds the bins 2047 - 2t and 2046 - 2t, so the scan runs from the top down
      const int b0 = 2047 - 2 * threadIdx.x, b1 = b0 - 1;
      const u64 n0 = sh.counts[b0], n1 = sh.counts[b1], s0 = sh.sums[b0], s1 = sh.sums[b1];
      u64 total_n, total_s;
      const u64 before_n = above_n + block_scan(n0 + n1, sh.wave_a, total_n);
      const u64 before_s = above_sum + block_scan(s0 + s1, sh.wave_b, total_s);
      if ((by_sum ? above_sum + total_s : above_n + total_n) < target) return false;
      const u64 x = by_sum ? before_s : before_n, x0 = by_sum ? s0 : n0, x1 = by_sum ? s1 : n1;
      if (x < target && x + x0 + x1 >= target) {
        const bool first = x + x0 >= target;
        sh.found_key = cut | (u64)(first ? b0 : b1) << shift;
        sh.found_count = before_n + (first ? 0 : n0);
        sh.found_sum = before_s + (first ? 0 : s0);
      }
      __syncthreads();
      cut = sh.found_key;
      above_n = sh.found_count;
      above_sum = sh.found_sum;
    }
    return true;
  }
};

// floor (up = 0) or ceiling (up = 1) of x f, exactly, for 0 < f < 1 (x < 2^63).
__device__ __forceinline__ u64 times_fraction(u64 x, float f, int up) {
  const uint32_t bits = __float_as_uint(f);
  int e = (int)(bits >> 23);
  u64 m = bits & 0x7FFFFF;
  if (e) m |= 0x800000; else e = 1;
  const int sh = 150 - e;                                   // f = m 2^-sh, 24 <= sh <= 149
  const u64 lo = x * m, hi = __umul64hi(x, m);
  u64 q, rest;
  if (sh < 64) {
    q = hi << (64 - sh) | lo >> sh;
    rest = lo & (((u64)1 << sh) - 1);
  } else if (sh < 128) {
    q = sh == 64 ? hi : hi >> (sh - 64);
    rest = lo | (sh == 64 ? 0 : hi & (((u64)1 << (sh - 64)) - 1));
  } else {
    q = 0;
    rest = lo | hi;
  }
  return q + (up && rest ? 1 : 0);
}

template <bool BF16>
__global__ __launch_bounds__(kRowThreads) void sample_kernel(TokenArgs a) {
  __shared__ RowShared sh;
  for (int row = blockIdx.x; row < a.n; row += gridDim.x) {
    __syncthreads();
    const float t = row_temperature(a, row);
    Row<BF16> r{a, sh, 0, inverse_temperature(t)};
    const int state = t >= 0.f ? r.init(row) : 2;
    if (state != 0) {
      if (threadIdx.x == 0) {
        a.labels[row] = -1;
        a.out[row] = state == 1 ? 0.f : NAN;
      }
      continue;
    }
    const bool greedy = t == 0.f;
    int top_k = greedy ? 1 : a.top_k ? a.top_k[row] : 0;
    float top_p = greedy || !a.top_p ? 1.f : a.top_p[row];
    float min_p = greedy || !a.min_p ? 0.f : a.min_p[row];
    float u = greedy ? 0.f : a.uniform[row];
    if (top_p <= 0.f) { top_k = 1; top_p = 1.f; }

    // all classes with key > cut are kept, and the first `ties` with key == cut
    u64 cut = 1, ties = ~(u64)0, above_n, above_sum;
    if (top_k > 0 && top_k < a.C) {
      u64 k;
      if (r.select(false, (u64)top_k, k, above_n, above_sum)) {
        cut = k;
        ties = (u64)top_k - above_n;
      }
    }
    if (top_p < 1.f) {
      u64 mass = 0, equal = 0;
      for (int c = threadIdx.x; c < a.C; c += kRowThreads) {
        const u64 k = r.key(c);
        if (k > cut) mass += r.units(k);
        else if (k == cut) ++equal;
      }
      mass = block_sum(mass, sh.wave_a);
      equal = block_sum(equal, sh.wave_b);
      mass += (equal < ties ? equal : ties) * r.units(cut);
      const u64 target = times_fraction(mass, top_p, 1);
      u64 k;
      if (r.select(true, target, k, above_n, above_sum)) {
        cut = k;
        const u64 each = r.units(k);
        ties = (target - above_sum + each - 1) / each;
      }
    }
    if (min_p > 0.f) {
      u64 best = 0;
      for (int c = threadIdx.x; c < a.C; c += kRowThreads) {
        const u64 k = r.key(c);
        best = k > best ? k : best;
      }
#pragma unroll
      for (int o = 32; o > 0; o >>= 1) {
        const u64 other = __shfl_xor(best, o, 64);
        best = other > best ? other : best;
      }
      __syncthreads();
      if ((threadIdx.x & 63) == 0) sh.wave_a[threadIdx.x >> 6] = best;
      __syncthreads();
      for (int w = 0; w < kRowWaves; ++w) best = sh.wave_a[w] > best ? sh.wave_a[w] : best;
      const u64 least = (u64)__double_as_longlong((double)fminf(min_p, 1.f) * __longlong_as_double((long long)best));
      if (least > cut) { cut = least; ties = ~(u64)0; }
    }
    u64 mass = 0, equal = 0;
    for (int c = threadIdx.x; c < a.C; c += kRowThreads) {
      const u64 k = r.key(c);
      if (k > cut) mass += r.units(k);
      else if (k == cut) ++equal;
    }
    mass = block_sum(mass, sh.wave_a);
    equal = block_sum(equal, sh.wave_b);
    if (equal < ties) ties = equal;
    mass += ties * r.units(cut);

    // the draw: a scan over the classes in their order
    u64 target = u > 0.f ? (u < 1.f ? times_fraction(mass, u, 0) : mass - 1) : 0;
    u64 seen = 0, seen_ties = 0;
    for (int c0 = 0; c0 < a.C; c0 += kRowThreads * 4) {
      u64 k[4];
      u64 n_equal = 0;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int c = c0 + threadIdx.x * 4 + j;
        k[j] = c < a.C ? r.key(c) : 0;
        n_equal += k[j] == cut;
      }
      u64 total_ties, total;
      u64 tie = seen_ties + block_scan(n_equal, sh.wave_a, total_ties);
      u64 part = 0;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        // selects: from a branch on `k < cut || (k == cut && tie++ >= ties)` the compiler of ROCm 7.2
        // drops the assignment of 0 for j = 0 in lanes that take its second half
        const bool equal_cut = k[j] == cut, keep = (k[j] > cut) | (equal_cut & (tie < ties));
        tie += equal_cut;
        k[j] = keep ? k[j] : 0;
        part += r.units(k[j]);
      }
      u64 at = seen + block_scan(part, sh.wave_b, total);
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const u64 p = r.units(k[j]);
        if (at <= target && at + p > target) {
          a.labels[row] = c0 + threadIdx.x * 4 + j;
          a.out[row] = (float)((double)p / (double)mass);
        }
        at += p;
      }
      seen += total;
      seen_ties += total_ties;
      if (seen > target) break;
    }
  }
}

template <bool BF16>
__global__ __launch_bounds__(kRowThreads) void topk_kernel(TokenArgs a) {
  __shared__ RowShared sh;
  for (int row = blockIdx.x; row < a.n; row += gridDim.x) {
    __syncthreads();
    Row<BF16> r{a, sh, 0, inverse_temperature(a.t_all)};
    const int state = r.init(row);
    int32_t* labels = a.labels + (long long)row * a.k;
    float* logp = a.out + (long long)row * a.k;
    if (state != 0) {
      for (int j = threadIdx.x; j < a.k; j += kRowThreads) {
        labels[j] = -1;
        logp[j] = state == 1 ? -INFINITY : NAN;
      }
      continue;
    }
    u64 cut = 1, ties = ~(u64)0, above_n, above_sum, k;
    if (r.select(false, (u64)a.k, k, above_n, above_sum)) {
      cut = k;
      ties = (u64)a.k - above_n;
    }
    if (threadIdx.x == 0) sh.n_list = 0;
    sh.list_key[threadIdx.x] = 0;
    sh.list_class[threadIdx.x] = 0x7fffffff;
    __syncthreads();
    u64 seen_ties = 0;
    for (int c0 = 0; c0 < a.C; c0 += kRowThreads) {
      const int c = c0 + threadIdx.x;
      const u64 key = c < a.C ? r.key(c) : 0;
      u64 total;
      const u64 tie = seen_ties + block_scan(key == cut, sh.wave_a, total);
      if (key > cut || (key == cut && tie < ties)) {
        const uint32_t i = atomicAdd(&sh.n_list, 1u);
        sh.list_key[i] = key;
        sh.list_class[i] = c;
      }
      seen_ties += total;
    }
    __syncthreads();
    // sorted by key down and class up
    int size = 2;
    while (size < (int)sh.n_list) size *= 2;
    for (int span = 2; span <= size; span *= 2)
      for (int d = span / 2; d > 0; d /= 2) {
        const int i = threadIdx.x, j = i ^ d;
        if (i < size && j > i) {
          const u64 ki = sh.list_key[i], kj = sh.list_key[j];
          const int ci = sh.list_class[i], cj = sh.list_class[j];
          const bool after = ki < kj || (ki == kj && ci > cj);    // i belongs behind j
          if (after == ((i & span) == 0)) {
            sh.list_key[i] = kj;
            sh.list_key[j] = ki;
            sh.list_class[i] = cj;
            sh.list_class[j] = ci;
          }
        }
        __syncthreads();
      }
    for (int j = threadIdx.x; j < a.k; j += kRowThreads) {
      const u64 key = sh.list_key[j];
      labels[j] = key ? sh.list_class[j] : -1;
      logp[j] = key ? (float)log(__longlong_as_double((long long)key)) : -INFINITY;
    }
  }
}

template <bool BF16>
hipError_t launch_stats(const TokenArgs& a, hipStream_t s) {
  const long long waves = (long long)a.n * a.S * a.groups;
  launch(group_stats_kernel<BF16>, dim3((unsigned)std::min<long long>((waves + 3) / 4, 1 << 20)), dim3(256), s, a);
  return hipGetLastError();
}

dim3 row_grid(const TokenArgs& a) { return dim3((unsigned)std::min(a.n, 1 << 20)); }

}  // namespace

hipError_t launch_sample(const TokenArgs& a, bool bf16, hipStream_t s) {
  const hipError_t st = bf16 ? launch_stats<true>(a, s) : launch_stats<false>(a, s);
  if (st != hipSuccess) return st;
  if (bf16) launch(sample_kernel<true>, row_grid(a), dim3(kRowThreads), s, a);
  else launch(sample_kernel<false>, row_grid(a), dim3(kRowThreads), s, a);
  return hipGetLastError();
}

hipError_t launch_topk(const TokenArgs& a, bool bf16, hipStream_t s) {
  const hipError_t st = bf16 ? launch_stats<true>(a, s) : launch_stats<false>(a, s);
  if (st != hipSuccess) return st;
  if (bf16) launch(topk_kernel<true>, row_grid(a), dim3(kRowThreads), s, a);
  else launch(topk_kernel<false>, row_grid(a), dim3(kRowThreads), s, a);
  return hipGetLastError();
}

}  // namespace rafiki
