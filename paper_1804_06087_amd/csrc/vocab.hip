// Answers over a vocabulary: drawing from an ensemble's combined distribution and listing
// its likeliest classes (rafiki_tokens.h).
//
// The combined probability of class c is p_c = sum_m 2^((z_mc - M_m) k) / (S s_m), k = log2(e) / T, with
// M_m the row's maximum and s_m its sum of such powers.  Which class is drawn or ranked where
// depends on comparisons of p and of sums of p, so those are taken in 64 bits: MI355X issues a
// 64-bit FMA as fast as a 32-bit one, and a power is about 20 of them.  Sums that are compared
// are sums of integers floor(p 2^62), which do not depend on their order.
//
// Two launches.  stats_kernel reads the logits once: the maximum of every 64 classes and the
// sum of powers of every 1024 (a wave each).  The row kernels, a workgroup per row, then work
// from these: a plain draw locates its unit of 1024 classes by the sums and reads only that;
// top-k and the filters need only the groups of 64 whose maximum reaches a bound.  The bound is the
// k-th largest of the groups' maxima, below which no class can be among the first k (k groups hold
// a class above it each).  The classes above it, hardly more than k, are sorted in LDS.  Rows
// whose kept classes do not fit there (flat distributions) are cut by histograms of the bits of p.
#include "tokens.h"

#include <algorithm>

namespace rafiki {

namespace {

typedef unsigned long long u64;

constexpr int kRowThreads = 512;
constexpr int kRowWaves = kRowThreads / 64;
constexpr int kList = 1024;                                // classes sorted in LDS
constexpr int kBins = 2048;
constexpr int kMaxGroupsListed = 4096;
constexpr double kUnit = 4611686018427387904.0;            // 2^62
constexpr u64 kLeastKey = (u64)(1023 - 1000) << 52;         // bits of 2^-1000
// Scores (log2 p in fp32) are compared with this much slack: they are within 2^-10 of log2 p
// for |log2 p| < 2^11 (a product and a sum rounded to 24 bits, and the fp32 log2).
constexpr float kSlack = 1.f / 64;
constexpr float kBinsPerOctave = 16.f;

// 2^t, t <= 0 (-inf and NaN as -1100: 0): t = n + f, |f| <= 1/2, and 2^f = 1 + f q(f) with q of degree 9
// through (2^f - 1) / f at Chebyshev's nodes: within 6e-16, and exactly 1 at f = 0.
__device__ __forceinline__ double power2(double t) {
  t = __builtin_fmax(t, -1100.0);
  const double n = __builtin_rint(t), f = t - n;
  double y = 7.070977866508138e-09;
  y = __builtin_fma(y, f, 1.0205905413765595e-07);
  y = __builtin_fma(y, f, 1.3215451633221434e-06);
  y = __builtin_fma(y, f, 1.5252672924850737e-05);
  y = __builtin_fma(y, f, 0.00015403530424776529);
  y = __builtin_fma(y, f, 0.0013333558200794592);
  y = __builtin_fma(y, f, 0.009618129107618665);
  y = __builtin_fma(y, f, 0.05550410866465167);
  y = __builtin_fma(y, f, 0.24022650695910075);
  y = __builtin_fma(y, f, 0.6931471805599462);
  y = __builtin_fma(y, f, 1.0);
  return __builtin_ldexp(y, (int)n);
}

// The exact difference of the logits first: the scaled values of two lowest logits do not cancel.
__device__ __forceinline__ double weight(float z, float top, double k) {
  return power2(((double)z - (double)top) * k);
}

template <bool BF16>
__device__ __forceinline__ float logit(const void* p, long long i) {
  if constexpr (BF16) return __uint_as_float((uint32_t)((const bf16_t*)p)[i] << 16);
  else return ((const float*)p)[i];
}

__device__ __forceinline__ float row_temperature(const TokenArgs& a, int row) {
  return a.temperature ? a.temperature[row] : a.t_all;
}
// k = log2(e) / T; T = 0 ranks at T = 1.
__device__ __forceinline__ double log2_scale(float t) { return t == 0.f ? 1.4426950408889634 : 1.4426950408889634 / (double)t; }

__device__ __forceinline__ float* stat_tops(const TokenArgs& a, long long rm) {
  return (float*)(a.stats + rm * a.stat_stride);
}
__device__ __forceinline__ double* stat_sums(const TokenArgs& a, long long rm) {
  return (double*)(a.stats + rm * a.stat_stride + (long long)a.units * kUnitTops * sizeof(float));
}

// Lanes exchanged within 16 by DPP: xor 1, xor 2, then mirrors of 8 and 16, which after those pair
// values as xor 4 and xor 8 would.
template <int CTRL>
__device__ __forceinline__ float dpp(float v) {
  return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), CTRL, 0xF, 0xF, true));
}
template <int CTRL>
__device__ __forceinline__ double dpp(double v) {
  const long long b = __double_as_longlong(v);
  const int lo = __builtin_amdgcn_update_dpp(0, (int)b, CTRL, 0xF, 0xF, true);
  const int hi = __builtin_amdgcn_update_dpp(0, (int)(b >> 32), CTRL, 0xF, 0xF, true);
  return __longlong_as_double((long long)((u64)(uint32_t)hi << 32 | (uint32_t)lo));
}
constexpr int kXor1 = 0xB1, kXor2 = 0x4E, kHalfMirror = 0x141, kMirror = 0x140;

__device__ __forceinline__ double wave_sum(double v) {
  v += dpp<kXor1>(v);
  v += dpp<kXor2>(v);
  v += dpp<kHalfMirror>(v);
  v += dpp<kMirror>(v);
  v += __shfl_xor(v, 16, 64);
  v += __shfl_xor(v, 32, 64);
  return v;
}

// 16 bytes of logits from any element on.
typedef uint32_t u32x4_any __attribute__((ext_vector_type(4), aligned(2)));
typedef float f32x4_any __attribute__((ext_vector_type(4), aligned(4)));

template <bool BF16, int V>
__device__ __forceinline__ void load_logits(const void* p, long long at, int c, int C, float* z) {
  if (c + V <= C) {
    if constexpr (BF16) {
      const u32x4_any q = *(const u32x4_any*)((const bf16_t*)p + at + c);
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        z[2 * j] = __uint_as_float(q[j] << 16);
        z[2 * j + 1] = __uint_as_float(q[j] & 0xFFFF0000u);
      }
    } else {
      const f32x4_any q = *(const f32x4_any*)((const float*)p + at + c);
#pragma unroll
      for (int j = 0; j < 4; ++j) z[j] = q[j];
    }
  } else {
#pragma unroll
    for (int j = 0; j < V; ++j) z[j] = c + j < C ? logit<BF16>(p, at + c + j) : -INFINITY;
  }
}

// ---------------------------------------------------------------- statistics
// A wave per unit of 1024 classes: 16 logits a lane in 16-byte loads, so that 16 (fp32) or 8
// (bf16) neighbouring lanes hold a group of 64.
template <bool BF16>
__global__ __launch_bounds__(256) void stats_kernel(TokenArgs a) {
  constexpr int V = BF16 ? 8 : 4, LOADS = 16 / V;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const long long total = (long long)a.n * a.S * a.units;
  for (long long id = (long long)blockIdx.x * 4 + wave; id < total; id += (long long)gridDim.x * 4) {
    const long long rm = total >> 32 ? id / a.units : (uint32_t)id / (uint32_t)a.units;
    const int u = (int)(id - rm * a.units);
    const int row = (int)(total >> 32 ? rm / a.S : (uint32_t)rm / (uint32_t)a.S), m = (int)(rm - (long long)row * a.S);
    const double k = log2_scale(row_temperature(a, row));
    const long long base = m * a.ld_model + row * a.ld_row;
    float z[16], top[LOADS];
#pragma unroll
    for (int j = 0; j < LOADS; ++j)
      load_logits<BF16, V>(a.logits, base, u * kUnitClasses + (j * 64 + lane) * V, a.C, z + j * V);
    bool bad = false;
    float all = -INFINITY;
#pragma unroll
    for (int j = 0; j < LOADS; ++j) {
      top[j] = z[j * V];
#pragma unroll
      for (int i = 1; i < V; ++i) top[j] = fmaxf(top[j], z[j * V + i]);
#pragma unroll
      for (int i = 0; i < V; ++i) bad |= !(z[j * V + i] < INFINITY);
      top[j] = fmaxf(top[j], dpp<kXor1>(top[j]));
      top[j] = fmaxf(top[j], dpp<kXor2>(top[j]));
      top[j] = fmaxf(top[j], dpp<kHalfMirror>(top[j]));
      if (!BF16) top[j] = fmaxf(top[j], dpp<kMirror>(top[j]));
      all = fmaxf(all, top[j]);
    }
    if (BF16) all = fmaxf(all, dpp<kMirror>(all));
    all = fmaxf(all, __shfl_xor(all, 16, 64));
    all = fmaxf(all, __shfl_xor(all, 32, 64));
    const bool any_bad = __ballot(bad) != 0;
    float* tops = stat_tops(a, rm) + u * kUnitTops;
    constexpr int kLanes = 64 / V;                         // lanes of one group of 64 classes
#pragma unroll
    for (int j = 0; j < LOADS; ++j)
      if (lane % kLanes == 0) tops[j * (64 / kLanes) + lane / kLanes] = any_bad ? INFINITY : top[j];
    double sum = 0.0;
    if (!any_bad && all > -INFINITY) {
#pragma unroll
      for (int i = 0; i < 16; ++i) sum += weight(z[i], all, k);
    }
    sum = wave_sum(sum);
    if (lane == 0) stat_sums(a, rm)[u] = sum;
  }
}

// ---------------------------------------------------------------- one workgroup per row
struct RowShared {
  float top[kMaxTokenModels];       // M_m
  double scale[kMaxTokenModels];    // 1 / (S s_m)
  float log_scale[kMaxTokenModels]; // log2 of it
  int state;                        // as init() returns
  u64 sums[kBins];                  // histogram; also the listed groups, and the units' masses
  uint32_t counts[kBins];
  u64 wave_a[kRowWaves], wave_b[kRowWaves];
  float wave_f[kRowWaves];
  u64 found_a, found_b, found_c;
  int found_class;
  uint32_t n_groups, n_list, overflow;
  u64 list_key[kList];
  int list_class[kList];
};

// Sum of v over the threads before this one; total = the sum over all.
__device__ __forceinline__ u64 block_scan(u64 v, u64* waves, u64& total) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  u64 s = v;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const u64 t = __shfl_up(s, o, 64);
    s += lane >= o ? t : 0;
  }
  __syncthreads();
  if (lane == 63) waves[wave] = s;
  __syncthreads();
  u64 before = 0;
  total = 0;
#pragma unroll
  for (int w = 0; w < kRowWaves; ++w) {
    before += w < wave ? waves[w] : 0;
    total += waves[w];
  }
  return before + s - v;
}

__device__ __forceinline__ float block_max(float v, float* waves) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) v = fmaxf(v, __shfl_xor(v, o, 64));
  __syncthreads();
  if ((threadIdx.x & 63) == 0) waves[threadIdx.x >> 6] = v;
  __syncthreads();
  v = waves[0];
#pragma unroll
  for (int w = 1; w < kRowWaves; ++w) v = fmaxf(v, waves[w]);
  return v;
}

__device__ __forceinline__ u64 units_of(u64 key) { return (u64)(__longlong_as_double((long long)key) * kUnit); }

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

// The position of the draw in a mass of units.
__device__ __forceinline__ u64 draw_target(u64 mass, float u) {
  return u > 0.f ? (u < 1.f ? times_fraction(mass, u, 0) : mass - 1) : 0;
}

// A cut of the ranking: every class with key > cut is kept and the first `ties` with key == cut;
// mass is the sum of their units.
struct Cut {
  u64 key, ties, mass;
};

template <bool BF16>
struct Row {
  const TokenArgs& a;
  RowShared& sh;
  int row;
  double k;

  // Joins the units' statistics, a wave per model; 0: a distribution, 1: a model without a class
  // above -inf, 2: NaN or +inf somewhere.
  __device__ int init() {
    const int lane = threadIdx.x & 63;
    if (threadIdx.x == 0) sh.state = 0;
    __syncthreads();
    for (int m = threadIdx.x >> 6; m < a.S; m += kRowWaves) {
      const long long rm = (long long)row * a.S + m;
      const float4* tops = (const float4*)stat_tops(a, rm);
      const double* sums = stat_sums(a, rm);
      float top = -INFINITY;
      for (int i = lane; i < a.units * 4; i += 64) {
        const float4 t = tops[i];
        top = fmaxf(top, fmaxf(fmaxf(t.x, t.y), fmaxf(t.z, t.w)));
      }
#pragma unroll
      for (int o = 32; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor(top, o, 64));
      double s = 0.0;
      if (top > -INFINITY && top < INFINITY)
        for (int u = lane; u < a.units; u += 64) s += sums[u] * weight(unit_top(tops, u), top, k);
      s = wave_sum(s);
      if (lane == 0) {
        sh.top[m] = top;
        sh.scale[m] = 1.0 / (s * a.S);
        sh.log_scale[m] = __log2f((float)sh.scale[m]);
        if (top == INFINITY) atomicMax(&sh.state, 2);
        else if (top == -INFINITY) atomicMax(&sh.state, 1);
      }
    }
    __syncthreads();
    return sh.state;
  }

  static __device__ __forceinline__ float unit_top(const float4* tops, int u) {
    float v = -INFINITY;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float4 t = tops[u * 4 + i];
      v = fmaxf(v, fmaxf(fmaxf(t.x, t.y), fmaxf(t.z, t.w)));
    }
    return v;
  }

  // Units of the mass of all classes of unit u.
  __device__ u64 unit_mass(int u) const {
    double p = 0.0;
#pragma unroll 1
    for (int m = 0; m < a.S; ++m) {
      const long long rm = (long long)row * a.S + m;
      p += stat_sums(a, rm)[u] * sh.scale[m] * weight(unit_top((const float4*)stat_tops(a, rm), u), sh.top[m], k);
    }
    return (u64)(p * kUnit);
  }

  // Bits of p_c (they order as p_c does), 0 for a class without a probability.
  __device__ __forceinline__ u64 key(int c) const {
    const long long at = row * a.ld_row + c;
    double p = 0.0;
#pragma unroll 1
    for (int m = 0; m < a.S; ++m)
      p = __builtin_fma(weight(logit<BF16>(a.logits, at + m * a.ld_model), sh.top[m], k), sh.scale[m], p);
    const u64 bits = (u64)__double_as_longlong(p);
    return bits < kLeastKey ? 0 : bits;
  }

  // Bounds of log2 p over group g of 64 classes: one of its classes reaches `low`, none exceeds `high`.
  __device__ __forceinline__ void group_scores(int g, float& low, float& high) const {
    const float kf = fminf((float)k, 3e38f);                 // 0 kf stays 0
    if (a.S == 1) {
      low = high = (stat_tops(a, row)[g] - sh.top[0]) * kf + sh.log_scale[0];
      if (!(low > -2048.f)) low = high = -INFINITY;          // also NaN of an infinite product
      return;
    }
    low = -INFINITY;
#pragma unroll 1
    for (int m = 0; m < a.S; ++m) {
      const float t = (stat_tops(a, (long long)row * a.S + m)[g] - sh.top[m]) * kf + sh.log_scale[m];
      if (t > -2048.f) low = fmaxf(low, t);
    }
    high = 0.f;
#pragma unroll 1
    for (int m = 0; m < a.S; ++m) {
      const float t = (stat_tops(a, (long long)row * a.S + m)[g] - sh.top[m]) * kf + sh.log_scale[m];
      if (t > -2048.f) high += exp2f(t - low);
    }
    high = low > -INFINITY ? low + log2f(high) : -INFINITY;
  }

  // A score that at least `need` classes reach (need >= 1; -inf where the groups do not tell):
  // need groups hold a class at least that likely.
  __device__ float bound(int need, float best) {
    const int groups = a.units * kUnitTops;
    __syncthreads();
    for (int b = threadIdx.x; b < kBins; b += kRowThreads) sh.counts[b] = 0;
    if (threadIdx.x == 0) sh.found_a = kBins - 1;
    __syncthreads();
    for (int g = threadIdx.x; g < groups; g += kRowThreads) {
      float low, high;
      group_scores(g, low, high);
      if (low > -INFINITY) atomicAdd(&sh.counts[(int)fminf((best - low) * kBinsPerOctave, (float)(kBins - 1))], 1u);
    }
    __syncthreads();
    constexpr int PER = kBins / kRowThreads;
    u64 n = 0, total;
#pragma unroll
    for (int i = 0; i < PER; ++i) n += sh.counts[threadIdx.x * PER + i];
    u64 at = block_scan(n, sh.wave_a, total);
    if (at < (u64)need && at + n >= (u64)need) {
      int b = threadIdx.x * PER;
      while (at + sh.counts[b] < (u64)need) at += sh.counts[b++];
      sh.found_a = b;
    }
    __syncthreads();
    const int b = (int)sh.found_a;
    return b == kBins - 1 ? -INFINITY : best - (float)(b + 1) / kBinsPerOctave - kSlack;
  }

  __device__ float best_score() {
    float best = -INFINITY;
    for (int g = threadIdx.x; g < a.units * kUnitTops; g += kRowThreads) {
      float low, high;
      group_scores(g, low, high);
      best = fmaxf(best, low);
    }
    return block_max(best, sh.wave_f);
  }

  // Lists every class whose p reaches 2^(score) (and some below it); false where they do not fit.
  __device__ bool list(float score) {
    const int lane = threadIdx.x & 63;
    uint32_t* groups = (uint32_t*)sh.sums;
    __syncthreads();
    if (threadIdx.x == 0) sh.n_groups = sh.n_list = sh.overflow = 0;
    __syncthreads();
    const int n = (a.C + 63) / 64;
    for (int g = threadIdx.x; g < n; g += kRowThreads) {
      float low, high;
      group_scores(g, low, high);
      if (high >= score - kSlack) {
        const uint32_t i = atomicAdd(&sh.n_groups, 1u);
        if (i < kMaxGroupsListed) groups[i] = g;
      }
    }
    __syncthreads();
    const int listed = (int)sh.n_groups;
    if (listed > kMaxGroupsListed) return false;
    const u64 least = score > -1000.f ? (u64)__double_as_longlong((double)exp2f(fmaxf(score - kSlack, -120.f))) : 1;
    for (int i = threadIdx.x >> 6; i < listed; i += kRowWaves) {
      const int c = (int)groups[i] * 64 + lane;
      const u64 x = c < a.C ? key(c) : 0;
      const bool take = x >= (score > -120.f ? least : 1);
      const u64 who = __ballot(take);
      uint32_t at = 0;
      if (lane == 0 && who) at = atomicAdd(&sh.n_list, (uint32_t)__popcll(who));
      at = __shfl(at, 0, 64) + __popcll(who & (((u64)1 << lane) - 1));
      if (take && at < kList) {
        sh.list_key[at] = x;
        sh.list_class[at] = c;
      }
    }
    __syncthreads();
    return sh.n_list <= kList;
  }

  // Sorts the list by key down and class up.
  __device__ void sort() {
    const int n = (int)sh.n_list;
    __syncthreads();
    if (n <= 256) {                                          // by rank: every element against all others
      u64 mine = 0;
      int cls = 0, rank = 0;
      const int i = threadIdx.x % 256, part = threadIdx.x / 256;
      if (threadIdx.x < 256) sh.counts[threadIdx.x] = 0;
      __syncthreads();
      if (i < n) {
        mine = sh.list_key[i];
        cls = sh.list_class[i];
        for (int j = part; j < n; j += kRowThreads / 256) {
          const u64 o = sh.list_key[j];
          rank += (o > mine) | ((o == mine) & (sh.list_class[j] < cls));
        }
        atomicAdd(&sh.counts[i], (uint32_t)rank);
      }
      __syncthreads();
      if (threadIdx.x < n) {
        sh.list_key[sh.counts[threadIdx.x]] = mine;
        sh.list_class[sh.counts[threadIdx.x]] = cls;
      }
      __syncthreads();
      return;
    }
    int size = 512;
    while (size < n) size *= 2;
    for (int i = n + threadIdx.x; i < size; i += kRowThreads) {
      sh.list_key[i] = 0;
      sh.list_class[i] = 0x7fffffff;
    }
    __syncthreads();
    for (int span = 2; span <= size; span *= 2)
      for (int d = span / 2; d > 0; d /= 2) {
        for (int t = threadIdx.x; t < size / 2; t += kRowThreads) {
          const int i = (t & ~(d - 1)) * 2 | (t & (d - 1)), j = i | d;
          const u64 ki = sh.list_key[i], kj = sh.list_key[j];
          const int ci = sh.list_class[i], cj = sh.list_class[j];
          const bool after = (ki < kj) | ((ki == kj) & (ci > cj));    // i belongs behind j
          if (after == ((i & span) == 0)) {
            sh.list_key[i] = kj;
            sh.list_key[j] = ki;
            sh.list_class[i] = cj;
            sh.list_class[j] = ci;
          }
        }
        __syncthreads();
      }
  }

  // Sum of the units of the first n listed classes, and the number of leading classes whose sum
  // reaches target (n + 1 where all n do not).
  __device__ u64 prefix(int n, u64 target, int& reached) {
    constexpr int PER = kList / kRowThreads;
    __syncthreads();
    if (threadIdx.x == 0) sh.found_class = n + 1;
    u64 p[PER], sum = 0, total;
#pragma unroll
    for (int j = 0; j < PER; ++j) {
      const int i = threadIdx.x * PER + j;
      p[j] = i < n ? units_of(sh.list_key[i]) : 0;
      sum += p[j];
    }
    u64 at = block_scan(sum, sh.wave_a, total);
#pragma unroll
    for (int j = 0; j < PER; ++j) {
      if (at < target && at + p[j] >= target) sh.found_class = threadIdx.x * PER + j + 1;
      at += p[j];
    }
    __syncthreads();
    reached = sh.found_class;
    return total;
  }

  // The cut at which the number (by_sum: the sum of the units) of the classes from the top reaches
  // `target`, by histograms of the bits of p: 32 bins an octave from 1 down first (whole: of
  // all the octaves), then 11 bits a level within the bin reached, until its classes fit into the
  // list and are sorted.  False where all classes (those above 2^-63, which have units) stay
  // below target.
  __device__ bool select(bool by_sum, u64 target, bool whole, Cut& cut) {
    constexpr u64 first_bin = (u64)1023 << 5;                 // bits of 1.0 >> 47
    u64 prefix_bits = 0, above_n = 0, above_sum = 0;
    int shift = whole ? 52 : 47, up = 64;
    for (;;) {
      __syncthreads();
      for (int b = threadIdx.x; b < kBins; b += kRowThreads) {
        sh.sums[b] = 0;
        sh.counts[b] = 0;
      }
      if (threadIdx.x == 0) sh.found_a = kBins;
      __syncthreads();
      for (int c = threadIdx.x; c < a.C; c += kRowThreads) {
        const u64 x = key(c);
        if (x != 0 && (up == 64 || x >> up == prefix_bits >> up)) {
          // bins ascend as keys descend
          const u64 top_bin = up == 64 ? (whole ? 2047 : first_bin) : (prefix_bits >> shift) | (((u64)1 << (up - shift)) - 1);
          const u64 below = top_bin - (x >> shift);
          const int b = (x >> shift) > top_bin ? 0 : below < kBins - 1 ? (int)below : kBins - 1;
          atomicAdd(&sh.sums[b], units_of(x));
          atomicAdd(&sh.counts[b], 1u);
        }
      }
      __syncthreads();
      constexpr int PER = kBins / kRowThreads;
      u64 n = 0, s = 0, total_n, total_s;
#pragma unroll
      for (int i = 0; i < PER; ++i) {
        n += sh.counts[threadIdx.x * PER + i];
        s += sh.sums[threadIdx.x * PER + i];
      }
      u64 at_n = above_n + block_scan(n, sh.wave_a, total_n), at_s = above_sum + block_scan(s, sh.wave_b, total_s);
      const u64 at = by_sum ? at_s : at_n, part = by_sum ? s : n;
      if (at < target && at + part >= target) {
        int b = threadIdx.x * PER;
        while ((by_sum ? at_s + sh.sums[b] : at_n + sh.counts[b]) < target) {
          at_n += sh.counts[b];
          at_s += sh.sums[b++];
        }
        sh.found_a = b;
        sh.found_b = at_n;
        sh.found_c = at_s;
      }
      __syncthreads();
      const int b = (int)sh.found_a;
      if (b == kBins) return false;
      if (up == 64 && !whole && b == kBins - 1) return false;         // beyond 63 octaves
      const u64 top_bin = up == 64 ? (whole ? 2047 : first_bin) : (prefix_bits >> shift) | (((u64)1 << (up - shift)) - 1);
      prefix_bits = (top_bin - b) << shift;
      above_n = sh.found_b;
      above_sum = sh.found_c;
      const int count = (int)sh.counts[b];
      if (count <= kList) {
        list_prefix(prefix_bits, shift);
        sort();
        int r;
        if (by_sum) prefix(count, target - above_sum, r);
        else r = (int)(target - above_n);
        cut.key = sh.list_key[r - 1];
        finish(r, above_sum, cut);
        return true;
      }
      if (shift == 0) {                                                // one key, in more classes than the list holds
        cut.key = prefix_bits;
        const u64 each = units_of(cut.key);
        cut.ties = by_sum ? (target - above_sum + each - 1) / each : target - above_n;
        cut.mass = above_sum + cut.ties * each;
        return true;
      }
      up = shift;
      shift = shift > 11 ? shift - 11 : 0;
    }
  }

  // ties and mass of a cut behind the first r listed classes.
  __device__ void finish(int r, u64 above_sum, Cut& cut) {
    __syncthreads();
    if (threadIdx.x == 0) sh.counts[0] = 0;
    __syncthreads();
    int same = 0;
    for (int i = threadIdx.x; i < r; i += kRowThreads) same += sh.list_key[i] == cut.key;
    if (same) atomicAdd(&sh.counts[0], (uint32_t)same);
    __syncthreads();
    cut.ties = sh.counts[0];
    int unused;
    cut.mass = above_sum + prefix(r, ~(u64)0, unused);
  }

  // Lists the classes whose key starts with prefix_bits.
  __device__ void list_prefix(u64 prefix_bits, int shift) {
    __syncthreads();
    if (threadIdx.x == 0) sh.n_list = 0;
    __syncthreads();
    const u64 want = prefix_bits >> shift;
    // with one model the logits themselves tell which classes may be there
    float lo = -INFINITY, hi = INFINITY;
    if (a.S == 1) {
      const float span = shift > 47 ? 1.f : 1.f / 16;         // log2(33 / 32) at most
      lo = log2f((float)__longlong_as_double((long long)prefix_bits)) - kSlack;
      hi = lo + span + 2 * kSlack;
      if (!(lo > -120.f)) lo = -INFINITY, hi = INFINITY;
    }
    const float kf = fminf((float)k, 3e38f);
    for (int c = threadIdx.x; c < a.C; c += kRowThreads) {
      if (a.S == 1) {
        const float t = (logit<BF16>(a.logits, row * a.ld_row + c) - sh.top[0]) * kf + sh.log_scale[0];
        if (t < lo || t > hi) continue;
      }
      const u64 x = key(c);
      if (x != 0 && x >> shift == want) {
        const uint32_t i = atomicAdd(&sh.n_list, 1u);
        if (i < kList) {
          sh.list_key[i] = x;
          sh.list_class[i] = c;
        }
      }
    }
    __syncthreads();
  }

  // The class c of [c0, c0 + kUnitClasses) at which the kept units pass `target`, counted from c0; the
  // first `ties` classes with key == cut are kept.  Where they stay below target (it comes from sums of
  // another rounding) the last kept; false where none has any units.
  __device__ bool draw_in_unit(int c0, u64 target, u64 cut, u64 ties, u64 mass, float u) {
    constexpr int PER = kUnitClasses / kRowThreads;
    u64 x[PER], equal = 0, part = 0, total;
#pragma unroll
    for (int j = 0; j < PER; ++j) {
      const int c = c0 + threadIdx.x * PER + j;
      x[j] = c < a.C ? key(c) : 0;
      equal += x[j] == cut;
    }
    u64 tie = block_scan(equal, sh.wave_a, total);
#pragma unroll
    for (int j = 0; j < PER; ++j) {
      // selects: from a branch on `x < cut || (x == cut && tie++ >= ties)` the compiler of ROCm 7.2
      // drops the assignment of 0 for j = 0 in lanes that take its second half
      const bool at_cut = x[j] == cut, keep = (x[j] > cut) | (at_cut & (tie < ties));
      tie += at_cut;
      x[j] = keep ? units_of(x[j]) : 0;
      part += x[j];
    }
    u64 at = block_scan(part, sh.wave_b, total);
    if (a.units == 1) {                                      // the row's own sum of units decides
      mass = total;
      target = draw_target(total, u);
    }
    const u64 wanted = target < total ? target : total - 1;
#pragma unroll
    for (int j = 0; j < PER; ++j) {
      if (at <= wanted && at + x[j] > wanted) {
        a.labels[row] = c0 + threadIdx.x * PER + j;
        a.out[row] = (float)((double)x[j] / (double)mass);
      }
      at += x[j];
    }
    return total != 0;
  }

  // Draws at `target` of unit `unit`, or where that has no units from the nearest one behind it, or before.
  __device__ void draw(int unit, u64 target, u64 mass, float u) {
    if (draw_in_unit(unit * kUnitClasses, target, 1, ~(u64)0, mass, u)) return;
    for (int next = unit + 1; next < a.units; ++next)
      if (draw_in_unit(next * kUnitClasses, 0, 1, ~(u64)0, mass, u)) return;
    for (int next = unit - 1; next >= 0; --next)
      if (draw_in_unit(next * kUnitClasses, ~(u64)0, 1, ~(u64)0, mass, u)) return;
  }
};

template <bool BF16>
__global__ __launch_bounds__(kRowThreads, 4) void sample_kernel(TokenArgs a) {
  __shared__ RowShared sh;
  for (int row = blockIdx.x; row < a.n; row += gridDim.x) {
    __syncthreads();
    const float t = row_temperature(a, row);
    Row<BF16> r{a, sh, row, log2_scale(t)};
    const int state = t >= 0.f ? r.init() : 2;
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
    const float u = greedy ? 0.f : a.uniform[row];
    if (top_p <= 0.f) { top_k = 1; top_p = 1.f; }
    if (top_k <= 0 || top_k >= a.C) top_k = 0;               // off
    min_p = min_p > 0.f ? fminf(min_p, 1.f) : 0.f;
    const bool by_mass = top_p < 1.f;

    // the units' masses
    u64 total = 0;
    for (int first = 0; first < a.units; first += kRowThreads) {
      const int unit = first + threadIdx.x;
      const u64 mass = unit < a.units ? r.unit_mass(unit) : 0;
      if (unit < a.units) sh.sums[unit] = mass;
      u64 part;
      block_scan(mass, sh.wave_a, part);
      total += part;
    }
    if (!top_k && !by_mass && min_p == 0.f) {
      const u64 target = draw_target(total, u);
      u64 seen = 0;
      __syncthreads();
      for (int first = 0; first < a.units; first += kRowThreads) {
        const int unit = first + threadIdx.x;
        const u64 mass = unit < a.units ? sh.sums[unit] : 0;
        u64 part;
        const u64 at = seen + block_scan(mass, sh.wave_a, part);
        if (at <= target && at + mass > target) {
          sh.found_a = unit;
          sh.found_b = target - at;
        }
        seen += part;
      }
      __syncthreads();
      const int unit = (int)sh.found_a;
      const u64 rest = sh.found_b;
      r.draw(unit, rest, total, u);
      continue;
    }

    // the kept classes, from a list where they fit into one
    const float best = r.best_score();
    float score;
    if (a.C <= kList) score = -INFINITY;
    else if (top_k) score = r.bound(top_k, best);
    else if (by_mass) score = r.bound(256, best);
    else score = best + __log2f(min_p) - kSlack;
    if (r.list(score)) {
      r.sort();
      int kept = (int)sh.n_list;
      if (top_k) kept = min(kept, top_k);
      bool all = true;
      if (by_mass) {
        int unused, reached;
        const u64 mass = top_k || a.C <= kList ? r.prefix(kept, ~(u64)0, unused) : total;
        r.prefix(kept, times_fraction(mass, top_p, 1), reached);
        // past the list: short of the mass, unless the list is everything
        if (reached > kept) all = top_k || a.C <= kList;
        else kept = reached;
      }
      if (all) {
        if (min_p > 0.f) {
          const double least = (double)min_p * __longlong_as_double((long long)sh.list_key[0]);
          __syncthreads();
          if (threadIdx.x == 0) sh.found_class = kept;
          __syncthreads();
          for (int i = threadIdx.x; i < kept; i += kRowThreads)
            if (__longlong_as_double((long long)sh.list_key[i]) < least) atomicMin(&sh.found_class, i);
          __syncthreads();
          kept = sh.found_class;
        }
        int unused;
        const u64 mass = r.prefix(kept, ~(u64)0, unused), target = draw_target(mass, u);
        for (int i = threadIdx.x; i < kept; i += kRowThreads) {
          const int c = sh.list_class[i];
          u64 before = 0;                                    // of the kept classes of lower index
          for (int j = 0; j < kept; ++j) before += sh.list_class[j] < c ? units_of(sh.list_key[j]) : 0;
          const u64 p = units_of(sh.list_key[i]);
          if (before <= target && before + p > target) {
            a.labels[row] = c;
            a.out[row] = greedy ? 1.f : (float)((double)p / (double)mass);
          }
        }
        continue;
      }
    }

    // more classes than a list holds: cut by histograms, then a scan of the units
    Cut cut{1, ~(u64)0, total};
    if (top_k) r.select(false, (u64)top_k, false, cut);
    if (by_mass) r.select(true, times_fraction(cut.mass, top_p, 1), false, cut);
    if (min_p > 0.f) {
      u64 top = 0;
      for (int c = threadIdx.x; c < a.C; c += kRowThreads) {
        const u64 x = r.key(c);
        top = x > top ? x : top;
      }
#pragma unroll
      for (int o = 32; o > 0; o >>= 1) {
        const u64 other = __shfl_xor(top, o, 64);
        top = other > top ? other : top;
      }
      __syncthreads();
      if ((threadIdx.x & 63) == 0) sh.wave_a[threadIdx.x >> 6] = top;
      __syncthreads();
      for (int w = 0; w < kRowWaves; ++w) top = sh.wave_a[w] > top ? sh.wave_a[w] : top;
      const u64 least = (u64)__double_as_longlong((double)min_p * __longlong_as_double((long long)top));
      if (least > cut.key) { cut.key = least; cut.ties = ~(u64)0; }
    }
    __syncthreads();
    // a wave per unit: the units above the cut, and the ties
    const int lane = threadIdx.x & 63;
    for (int unit = threadIdx.x >> 6; unit < a.units; unit += kRowWaves) {
      u64 mass = 0;
      uint32_t equal = 0;
      for (int i = lane; i < kUnitClasses; i += 64) {
        const int c = unit * kUnitClasses + i;
        const u64 x = c < a.C ? r.key(c) : 0;
        mass += x > cut.key ? units_of(x) : 0;
        equal += x == cut.key;
      }
#pragma unroll
      for (int o = 32; o > 0; o >>= 1) {
        mass += __shfl_xor(mass, o, 64);
        equal += __shfl_xor(equal, o, 64);
      }
      if (lane == 0) {
        sh.sums[unit] = mass;
        sh.counts[unit] = equal;
      }
    }
    __syncthreads();
    const u64 each = units_of(cut.key);
    u64 seen_ties = 0;
    total = 0;
    for (int first = 0; first < a.units; first += kRowThreads) {
      const int unit = first + threadIdx.x;
      const u64 equal = unit < a.units ? sh.counts[unit] : 0;
      u64 part_ties, part;
      const u64 before = seen_ties + block_scan(equal, sh.wave_a, part_ties);
      const u64 kept = before >= cut.ties ? 0 : equal < cut.ties - before ? equal : cut.ties - before;
      const u64 mass = unit < a.units ? sh.sums[unit] + kept * each : 0;
      block_scan(mass, sh.wave_b, part);
      if (unit < a.units) {
        sh.sums[unit] = mass;
        sh.counts[unit] = (uint32_t)kept;
      }
      seen_ties += part_ties;
      total += part;
    }
    const u64 target = draw_target(total, u);
    u64 seen = 0;
    for (int first = 0; first < a.units; first += kRowThreads) {
      const int unit = first + threadIdx.x;
      const u64 mass = unit < a.units ? sh.sums[unit] : 0;
      u64 part;
      const u64 at = seen + block_scan(mass, sh.wave_a, part);
      if (at <= target && at + mass > target) {
        sh.found_a = unit;
        sh.found_b = target - at;
      }
      seen += part;
    }
    __syncthreads();
    const int unit = (int)sh.found_a;
    const u64 rest = sh.found_b;
    r.draw_in_unit(unit * kUnitClasses, rest, cut.key, sh.counts[unit], total, u);
  }
}

template <bool BF16>
__global__ __launch_bounds__(kRowThreads, 4) void topk_kernel(TokenArgs a) {
  __shared__ RowShared sh;
  for (int row = blockIdx.x; row < a.n; row += gridDim.x) {
    __syncthreads();
    Row<BF16> r{a, sh, row, log2_scale(a.t_all)};
    const int state = r.init();
    int32_t* labels = a.labels + (long long)row * a.k;
    float* logp = a.out + (long long)row * a.k;
    if (state != 0) {
      for (int j = threadIdx.x; j < a.k; j += kRowThreads) {
        labels[j] = -1;
        logp[j] = state == 1 ? -INFINITY : NAN;
      }
      continue;
    }
    bool listed;
    if (a.C <= kList) listed = r.list(-INFINITY);
    else {
      const float best = r.best_score();
      const float score = r.bound(a.k, best);
      listed = r.list(score);
    }
    if (!listed) {
      // the cut by histograms; the list is then the classes above it and the first ties
      Cut cut{1, ~(u64)0, 0};
      r.select(false, (u64)a.k, true, cut);
      __syncthreads();
      if (threadIdx.x == 0) sh.n_list = 0;
      __syncthreads();
      u64 seen_ties = 0;
      for (int c0 = 0; c0 < a.C; c0 += kRowThreads) {
        const int c = c0 + threadIdx.x;
        const u64 key = c < a.C ? r.key(c) : 0;
        u64 total;
        const u64 tie = seen_ties + block_scan(key == cut.key, sh.wave_a, total);
        if ((key > cut.key) | ((key == cut.key) & (tie < cut.ties))) {
          const uint32_t i = atomicAdd(&sh.n_list, 1u);
          if (i < kList) {
            sh.list_key[i] = key;
            sh.list_class[i] = c;
          }
        }
        seen_ties += total;
      }
    }
    __syncthreads();
    r.sort();
    const int n = (int)sh.n_list;
    for (int j = threadIdx.x; j < a.k; j += kRowThreads) {
      const u64 key = j < n ? sh.list_key[j] : 0;
      labels[j] = key ? sh.list_class[j] : -1;
      logp[j] = key ? (float)log(__longlong_as_double((long long)key)) : -INFINITY;
    }
  }
}

template <bool BF16>
hipError_t launch_stats(const TokenArgs& a, hipStream_t s) {
  const long long waves = (long long)a.n * a.S * a.units;
  launch(stats_kernel<BF16>, dim3((unsigned)std::min<long long>((waves + 3) / 4, 1 << 20)), dim3(256), s, a);
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
