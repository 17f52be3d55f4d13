// Answers over a vocabulary: drawing from an ensemble's combined distribution and listing
// its likeliest classes (rafiki_tokens.h).
//
// The combined probability of class c is p_c = sum_m 2^((z_mc - M_m) k) / (S s_m), k = log2(e) / T, with
// M_m the row's maximum and s_m its sum of such powers.  Which class is drawn or ranked where
// depends on comparisons of p and of sums of p, so those are taken in 64 bits: MI355X issues a
// 64-bit FMA as fast as a 32-bit one, and a power is about 20 of them.  Sums that are compared
// are sums of integers floor(p 2^62), which do not depend on their order.
//
// stats_kernel reads the logits once: the maximum of every 64 classes and the sum of powers of every
// 1024 (a wave each).  The row kernels, a workgroup per row, work from these: a plain draw locates its unit
// of 1024 classes by the sums and reads only that; top-k and the filters need only the groups of 64 whose
// maximum reaches a bound.  The bound is the k-th largest of the groups' maxima, below which no class
// can be among the first k (k groups hold a class above it each).  The classes above it, hardly more
// than k, are sorted in LDS.  For top-p alone the bound is the 64th largest.  Rows whose kept classes do not fit
// into the list (flat distributions), and nuclei that end below that bound, are cut by histograms of the bits of
// p, in a launch of their own that other rows leave at once.
//
// Measured on an MI355X: 1 x 256 x 131072 fp32, 43 us for plain draws (stats 35 us: 3.8 TB/s), 54 us with
// top-k 50 and top-p 0.9, 173 us with every row flat; top-64 of 2 x 1024 x 131072 bf16, 40 calls in a row, 297 us: stats
// 240 us (2.2 TB/s: 17 64-bit instructions a class, of which the conversion takes four times an FMA's cycles, bound
// it, at 1.9 to 2.1 GHz under this load), the rows 49 us, the flat check 4.5 us.  Fewer in a row take 260 us.
// A row alone takes 10 to 20 us: fetching the code that it runs through once, and some ten dependent loads.
#include "tokens.h"

#include <algorithm>

namespace rafiki {

namespace {

typedef unsigned long long u64;

constexpr int kList = 1024;                                // classes sorted in LDS
constexpr int kBins = 2048;                                // of the bound's histogram
constexpr int kFlatBins = 4096;                            // of select()'s
constexpr int kMaxUnits = kMaxTokenClasses / kUnitClasses;
constexpr int kMaxGroupsListed = 2 * kMaxUnits;
constexpr double kUnit = 4611686018427387904.0;            // 2^62
constexpr u64 kLeastKey = (u64)(1023 - 1000) << 52;         // bits of 2^-1000
// Scores (log2 p in fp32) are compared with this much slack: they are within 2^-10 of log2 p
// for |log2 p| < 2^11 (a product and a sum rounded to 24 bits, and the fp32 log2).
constexpr float kSlack = 1.f / 64;
constexpr float kBinsPerOctave = 16.f;

// 2^t, t <= 0 (below -1020, for -inf and for NaN: 2^-1020, less than any probability that counts, and so little that a
// class of 2^-1000 from one of 32 models is off by 2^-15 at most, half a step of its logarithm in fp32).
// t = n + f, |f| <= 1/2: adding 1.5 2^52 leaves n in the low bits, and n goes into the exponent as an integer,
// since conversions, rint and ldexp of 64 bits take four times an FMA's cycles (with them stats_kernel
// took 300 us for 2 x 1024 x 131072).  2^f = 1 + f q(f) with q of degree 8 through (2^f - 1) / f at
// Chebyshev's nodes: within 4e-14, and exactly 1 at f = 0.
__device__ __forceinline__ double power2(double t) {
  constexpr double kRound = 6755399441055744.0;
  t = __builtin_fmax(t, -1020.0);
  const double u = t + kRound, f = t - (u - kRound);
  double y = 1.0203121063391729e-07;
  y = __builtin_fma(y, f, 1.3255224878668817e-06);
  y = __builtin_fma(y, f, 1.525268684626772e-05);
  y = __builtin_fma(y, f, 0.00015403455852453838);
  y = __builtin_fma(y, f, 0.0013333558179043112);
  y = __builtin_fma(y, f, 0.009618129159402558);
  y = __builtin_fma(y, f, 0.055504108664760424);
  y = __builtin_fma(y, f, 0.2402265069581299);
  y = __builtin_fma(y, f, 0.6931471805599453);
  y = __builtin_fma(y, f, 1.0);
  const int n = (int)__double_as_longlong(u);
  const u64 bits = (u64)__double_as_longlong(y);
  return __longlong_as_double((long long)((u64)((uint32_t)(bits >> 32) + ((uint32_t)n << 20)) << 32 | (uint32_t)bits));
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
__device__ __forceinline__ UnitStat* stat_units(const TokenArgs& a, long long rm) {
  return (UnitStat*)(a.stats + rm * a.stat_stride + (long long)a.units * kUnitTops * sizeof(float));
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
// A wave per unit of 1024 classes: 16 logits a lane in 16-byte loads, so that 16 (fp32) or 8 (bf16)
// neighbouring lanes hold a group of 64.  4.8 us for 3 x 16 x 30000 bf16, 36 us for 1 x 256 x 131072 fp32.
template <bool BF16>
__global__ __launch_bounds__(256) void stats_kernel(TokenArgs a) {
  constexpr int V = BF16 ? 8 : 4, LOADS = 16 / V;
  const int lane = threadIdx.x & 63;
  const int u = __builtin_amdgcn_readfirstlane(blockIdx.y * (blockDim.x >> 6) + (threadIdx.x >> 6));
  if (u >= a.units) return;
  const int row = a.row0 + blockIdx.x, m = blockIdx.z;
  const long long rm = (long long)row * a.S + m;
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
  if (lane == 0) stat_units(a, rm)[u] = UnitStat{sum, any_bad ? INFINITY : all, 0.f};
}

// ---------------------------------------------------------------- one workgroup per row
template <bool FLAT>
struct RowShared {
  float top[kMaxTokenModels];       // M_m
  double scale[kMaxTokenModels];    // 1 / (S s_m)
  float log_scale[kMaxTokenModels]; // log2 of it
  int state;                        // as init() returns
  u64 sums[FLAT ? kFlatBins : kMaxUnits];   // the listed groups, the units' masses, units in a draw; FLAT: a histogram
  union {
    uint32_t counts[FLAT ? kFlatBins : kBins];
    u64 run_key[kList];             // sorted runs; sums of units along the list
  };
  u64 wave_a[16];
  u64 found_a, found_b, found_c;
  int found_class;
  uint32_t n_groups, n_list;
  u64 list_key[kList];
  int list_class[kList], run_class[kList];
  uint32_t unit_ties[FLAT ? kMaxUnits : 1];   // kept classes with key == cut of every unit
};

// Sum of v over the threads before this one, and over all.  Not inlined: a row's time is mostly that of
// fetching the code it runs through, and the row kernels scan half a dozen times.
struct Scan {
  u64 before, total;
};
template <int NT>
__device__ __attribute__((noinline)) Scan block_scan(u64 v) {
  __shared__ u64 waves[NT / 64];
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
  u64 before = 0, total = 0;
#pragma unroll 4
  for (int w = 0; w < NT / 64; ++w) {
    const u64 t = waves[w];
    before += w < wave ? t : 0;
    total += t;
  }
  return Scan{before + s - v, total};
}

// floor(p 2^62) for the bits of p <= 1 + 2^-52 (0 for key 0): the mantissa, shifted by the exponent.
__device__ __forceinline__ u64 units_of(u64 key) {
  const u64 mantissa = ((key & (((u64)1 << 52) - 1)) | (u64)1 << 52) << 10;
  const uint32_t down = 1023 - (uint32_t)(key >> 52);
  return down < 64 ? mantissa >> down : 0;
}

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
  bool units;                 // sums and unit_ties hold the units' kept masses and ties
};

template <bool BF16, int NT, bool FLAT>
struct Row {
  static constexpr int kWaves = NT / 64;
  const TokenArgs& a;
  RowShared<FLAT>& sh;
  int row;
  double k;

  // Joins the units' statistics, a wave per model; 0: a distribution, 1: a model without a class
  // above -inf, 2: NaN or +inf somewhere.
  __device__ __forceinline__ int init() {
    const int lane = threadIdx.x & 63;
    if (threadIdx.x == 0) sh.state = 0;
    __syncthreads();
    for (int m = threadIdx.x >> 6; m < a.S; m += kWaves) {
      const long long rm = (long long)row * a.S + m;
      const UnitStat* units = stat_units(a, rm);
      float top = -INFINITY;
      for (int u = lane; u < a.units; u += 64) top = fmaxf(top, units[u].top);
#pragma unroll
      for (int o = 32; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor(top, o, 64));
      double s = 0.0;
      if (top > -INFINITY && top < INFINITY)
        for (int u = lane; u < a.units; u += 64) s += units[u].sum * weight(units[u].top, top, k);
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

  // Units of the mass of all classes of unit u.
  __device__ __forceinline__ u64 unit_mass(int u) const {
    double p = 0.0;
#pragma unroll 1
    for (int m = 0; m < a.S; ++m) {
      const long long rm = (long long)row * a.S + m;
      const UnitStat st = stat_units(a, rm)[u];
      p += st.sum * sh.scale[m] * weight(st.top, sh.top[m], k);
    }
    return (u64)(p * kUnit);
  }

  // Bits of p_c (they order as p_c does) of N classes, 0 for one without a probability or past the row's end:
  // one model's N logits are in flight together, and the next model's behind them.
  template <int N>
  __device__ __forceinline__ void keys(const int (&c)[N], u64 (&x)[N]) const {
    double p[N];
#pragma unroll
    for (int i = 0; i < N; ++i) p[i] = 0.0;
    float next[N];
    auto fetch = [&](int m) {
      const long long at = row * a.ld_row + m * a.ld_model;
#pragma unroll
      for (int i = 0; i < N; ++i) next[i] = c[i] < a.C ? logit<BF16>(a.logits, at + c[i]) : -INFINITY;
    };
    fetch(0);
#pragma unroll 1
    for (int m = 0; m < a.S; ++m) {
      float z[N];
#pragma unroll
      for (int i = 0; i < N; ++i) z[i] = next[i];
      if (m + 1 < a.S) fetch(m + 1);                         // while this model's powers are taken
      const float top = sh.top[m];
      const double scale = sh.scale[m];
#pragma unroll
      for (int i = 0; i < N; ++i) p[i] = __builtin_fma(weight(z[i], top, k), scale, p[i]);
    }
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const u64 bits = (u64)__double_as_longlong(p[i]);
      x[i] = bits < kLeastKey ? 0 : bits;
    }
  }
  __device__ __forceinline__ u64 key(int c) const {
    const int one[1] = {c};
    u64 x[1];
    keys<1>(one, x);
    return x[0];
  }

  // This lane's 16 logits of one model of unit u, as stats_kernel holds them, and the class of the i-th.
  static constexpr int V = BF16 ? 8 : 4;
  __device__ __forceinline__ void unit_logits(int u, int m, float z[16]) const {
    const int lane = threadIdx.x & 63;
#pragma unroll
    for (int j = 0; j < 16 / V; ++j)
      load_logits<BF16, V>(a.logits, row * a.ld_row + m * a.ld_model, u * kUnitClasses + (j * 64 + lane) * V, a.C, z + j * V);
  }
  static __device__ __forceinline__ int unit_class(int u, int i) {
    return u * kUnitClasses + (i / V * 64 + (threadIdx.x & 63)) * V + i % V;
  }
  // Their keys; 0 past the row's end.
  __device__ __forceinline__ void unit_keys(int u, u64 x[16]) const {
    double p[16];
#pragma unroll
    for (int i = 0; i < 16; ++i) p[i] = 0.0;
#pragma unroll 1
    for (int m = 0; m < a.S; ++m) {
      float z[16];
      unit_logits(u, m, z);
      const float top = sh.top[m];
      const double scale = sh.scale[m];
#pragma unroll
      for (int i = 0; i < 16; ++i) p[i] = __builtin_fma(weight(z[i], top, k), scale, p[i]);
    }
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      const u64 bits = (u64)__double_as_longlong(p[i]);
      x[i] = bits < kLeastKey ? 0 : bits;
    }
  }

  // (z - top) k in fp32, for bounds: (z h - top h) by again, h by again = k.  Halves first, since two finite logits
  // may lie further apart than fp32 holds.  For T below about 2^-125, k is beyond fp32 (up to 2^150) and the differences
  // that matter below its normal range, where halves lose bits: whole ones by 2^64 first; those that overflow
  // then are -inf to scale too.  NaN for z = -inf at T = +inf.
  struct Difference {
    float h, by, again;
    __device__ __forceinline__ float operator()(float z, float top) const { return (z * h - top * h) * by * again; }
  };
  __device__ __forceinline__ Difference difference() const {
    return k < 0x1p126 ? Difference{0.5f, (float)(2.0 * k), 1.f} : Difference{1.f, 0x1p64f, (float)(k * 0x1p-64)};
  }

  // Bounds of log2 p over G groups of 64 classes (g0 + j NT + the thread): one of a group's classes reaches
  // `low`, none exceeds `high`; -inf past the last group, and where p is too small to matter.  `best` is
  // best_score().  The groups' maxima of one model are in flight together.
  static constexpr int G = 4;
  __device__ __forceinline__ void group_scores(int g0, float best, float (&low)[G], float (&high)[G]) const {
    const int groups = a.units * kUnitTops;
    const Difference scaled = difference();
#pragma unroll
    for (int j = 0; j < G; ++j) {
      low[j] = -INFINITY;
      high[j] = 0.f;
    }
    float next[G];
    auto fetch = [&](int m) {
      const float* tops = stat_tops(a, (long long)row * a.S + m);
#pragma unroll
      for (int j = 0; j < G; ++j) {
        const int g = g0 + j * NT + (int)threadIdx.x;
        next[j] = g < groups ? tops[g] : -INFINITY;
      }
    };
    fetch(0);
#pragma unroll 1
    for (int m = 0; m < a.S; ++m) {
      float v[G];
#pragma unroll
      for (int j = 0; j < G; ++j) v[j] = next[j];
      if (m + 1 < a.S) fetch(m + 1);
      const float top = sh.top[m], log_scale = sh.log_scale[m];
#pragma unroll
      for (int j = 0; j < G; ++j) {
        const float t = scaled(v[j], top) + log_scale;
        const bool some = t > -2048.f;                       // also false for the NaN of an infinite product
        low[j] = some ? fmaxf(low[j], t) : low[j];
        high[j] += some ? __builtin_amdgcn_exp2f(t - best) : 0.f;
      }
    }
#pragma unroll
    for (int j = 0; j < G; ++j)                              // near underflow 32 models at most sum to 5 octaves more
      high[j] = high[j] > 0x1p-100f ? best + __builtin_amdgcn_logf(high[j]) : low[j] + 5.f;
  }

  // The scores of the first G NT groups, taken once (FLAT: not kept).
  float low0[FLAT ? 1 : G], high0[FLAT ? 1 : G];
  __device__ __forceinline__ void scores(int g0, float best, float (&low)[G], float (&high)[G]) const {
    if constexpr (!FLAT) {
      if (g0 == 0) {
#pragma unroll
        for (int j = 0; j < G; ++j) {
          low[j] = low0[j];
          high[j] = high0[j];
        }
        return;
      }
    }
    group_scores(g0, best, low, high);
  }

  // A score that at least `need` classes reach (need >= 1; -inf where none is found): `need` groups hold a class
  // at least that likely, or where there are fewer groups, `need` classes are (a pass over the logits).
  __device__ __forceinline__ float bound(int need, float best) {
    float score = -INFINITY;
    for (bool classes = need > (a.C + 63) / 64;; classes = true) {
      // the classes of a bin that the bound cuts would not fit into a list beside so many
      if (classes && need > kList / 8 * 7 && a.C > kList) return score;
      __syncthreads();
      for (int b = threadIdx.x; b < kBins; b += NT) sh.counts[b] = 0;
      if (threadIdx.x == 0) sh.found_a = kBins - 1;
      __syncthreads();
      auto count = [&](float low) {
        if (low > -INFINITY) atomicAdd(&sh.counts[(int)fminf((best - low) * kBinsPerOctave, (float)(kBins - 1))], 1u);
      };
      if (classes) {
        const Difference scaled = difference();
        for (int u = threadIdx.x >> 6; u < a.units; u += kWaves) {
          float low[16];
#pragma unroll
          for (int i = 0; i < 16; ++i) low[i] = -INFINITY;
#pragma unroll 1
          for (int m = 0; m < a.S; ++m) {
            float z[16];
            unit_logits(u, m, z);
#pragma unroll
            for (int i = 0; i < 16; ++i) {
              const float t = scaled(z[i], sh.top[m]) + sh.log_scale[m];
              low[i] = t > -2048.f ? fmaxf(low[i], t) : low[i];
            }
          }
#pragma unroll
          for (int i = 0; i < 16; ++i) count(low[i]);
        }
      } else {
        for (int g0 = 0; g0 < a.units * kUnitTops; g0 += G * NT) {
          float low[G], high[G];
          scores(g0, best, low, high);
#pragma unroll
          for (int j = 0; j < G; ++j) count(low[j]);
        }
      }
      __syncthreads();
      constexpr int PER = kBins / NT;
      u64 n = 0;
#pragma unroll
      for (int i = 0; i < PER; ++i) n += sh.counts[threadIdx.x * PER + i];
      u64 at = block_scan<NT>(n).before;
      if (at < (u64)need && at + n >= (u64)need) {
        int b = threadIdx.x * PER;
        while (at + sh.counts[b] < (u64)need) at += sh.counts[b++];
        sh.found_a = b;
      }
      __syncthreads();
      const int b = (int)sh.found_a;
      if (b < kBins - 1) score = best - (float)(b + 1) / kBinsPerOctave - kSlack;
      if (classes || score > -INFINITY || a.C <= kList) return score;
    }
  }

  // The largest of the groups' lower bounds: that of the class at which a model has its maximum.
  __device__ __forceinline__ float best_score() const {
    float best = -INFINITY;
#pragma unroll 1
    for (int m = 0; m < a.S; ++m) best = fmaxf(best, sh.log_scale[m]);
    return best;
  }

  // The groups that may hold a class whose log2 p reaches score, into sums; how many there are (more than
  // kMaxGroupsListed: not all are listed).
  __device__ __forceinline__ int list_groups(float score, float best) {
    uint32_t* groups = (uint32_t*)sh.sums;
    __syncthreads();
    if (threadIdx.x == 0) sh.n_groups = 0;
    __syncthreads();
    const int n = (a.C + 63) / 64;
    for (int g0 = 0; g0 < n; g0 += G * NT) {
      float low[G], high[G];
      scores(g0, best, low, high);
#pragma unroll
      for (int j = 0; j < G; ++j) {
        const int g = g0 + j * NT + threadIdx.x;
        if (g < n && low[j] > -INFINITY && high[j] >= score - kSlack) {
          const uint32_t i = atomicAdd(&sh.n_groups, 1u);
          if (i < kMaxGroupsListed) groups[i] = g;
        }
      }
    }
    __syncthreads();
    return (int)sh.n_groups;
  }

  // Lists every class whose log2 p reaches score - kSlack / 2, and none below: half of the slack above the bound of the
  // groups, whose fp32 scores may be off in their last places, so that the list has no gap above its least class and may
  // be cut anywhere (of equal classes at the groups' own bound, those in groups with a better class would be listed
  // and the others not).  Gaps remain below 2^-120, where no class has units and no sum ends.  False where they do not fit.
  __device__ __forceinline__ bool list(float score, float best) {
    const int lane = threadIdx.x & 63;
    const uint32_t* groups = (const uint32_t*)sh.sums;
    const int listed = list_groups(score, best);
    if (listed > kMaxGroupsListed) return false;
    if (threadIdx.x == 0) sh.n_list = 0;
    __syncthreads();
    const u64 least = score > -1000.f ? (u64)__double_as_longlong((double)exp2f(fmaxf(score - 0.5f * kSlack, -120.f))) : 1;
    for (int i = (threadIdx.x >> 6) * G; i < listed; i += kWaves * G) {
      int c[G];
      u64 x[G];
#pragma unroll
      for (int j = 0; j < G; ++j) c[j] = i + j < listed ? (int)groups[i + j] * 64 + lane : a.C;
      keys<G>(c, x);
#pragma unroll
      for (int j = 0; j < G; ++j) {
        const bool take = x[j] >= (score > -120.f ? least : 1);
        if (take) {
          const uint32_t at = atomicAdd(&sh.n_list, 1u);
          if (at < kList) {
            sh.list_key[at] = x[j];
            sh.list_class[at] = c[j];
          }
        }
      }
    }
    __syncthreads();
    return sh.n_list <= kList;
  }

  // Sorts the list by key down and class up: every 64 by rank in a wave, then every class's place among the
  // other runs of 64 by bisection.  (A bitonic sort of 1024 with a barrier a step took 60 us.)
  __device__ __forceinline__ void sort() {
    const int n = (int)sh.n_list, lane = threadIdx.x & 63;
    const int runs = (n + 63) / 64;
    __syncthreads();
    for (int run = threadIdx.x >> 6; run < runs; run += kWaves) {
      const int i = run * 64 + lane;
      const u64 x = i < n ? sh.list_key[i] : 0;
      const int c = i < n ? sh.list_class[i] : 0x7fffffff;
      int rank = 0;
      const int m = min(64, (n - run * 64 + 7) & ~7);
      for (int j0 = 0; j0 < m; j0 += 8)
#pragma unroll
        for (int j = j0; j < j0 + 8; ++j) {                  // past the run's end: key 0, behind every other
          const u64 y = (u64)(uint32_t)__builtin_amdgcn_readlane((int)(x >> 32), j) << 32 |
                        (uint32_t)__builtin_amdgcn_readlane((int)x, j);
          rank += (y > x) | ((y == x) & (__builtin_amdgcn_readlane(c, j) < c));
        }
      if (i < n) {
        sh.run_key[run * 64 + rank] = x;
        sh.run_class[run * 64 + rank] = c;
      }
    }
    __syncthreads();
    for (int i = threadIdx.x; i < n; i += NT) {
      const u64 x = sh.run_key[i];
      const int c = sh.run_class[i];
      int place = i & 63;
      for (int run = 0; run < runs; ++run) {
        if (run == i >> 6) continue;
        int lo = 0, hi = min(64, n - run * 64);             // classes of the run before this one
        while (lo < hi) {
          const int mid = (lo + hi) >> 1;
          const u64 y = sh.run_key[run * 64 + mid];
          if ((y > x) | ((y == x) & (sh.run_class[run * 64 + mid] < c))) lo = mid + 1;
          else hi = mid;
        }
        place += lo;
      }
      sh.list_key[place] = x;
      sh.list_class[place] = c;
    }
    __syncthreads();
  }

  // run_key[i] = the units of the listed classes up to and with i.
  __device__ __forceinline__ void accumulate() {
    constexpr int PER = kList / NT;
    const int n = (int)sh.n_list;
    u64 p[PER], sum = 0;
#pragma unroll
    for (int j = 0; j < PER; ++j) {
      const int i = threadIdx.x * PER + j;
      p[j] = i < n ? units_of(sh.list_key[i]) : 0;
      sum += p[j];
    }
    u64 at = block_scan<NT>(sum).before;
#pragma unroll
    for (int j = 0; j < PER; ++j) {
      const int i = threadIdx.x * PER + j;
      at += p[j];
      if (i < n) sh.run_key[i] = at;
    }
    __syncthreads();
  }

  // The number of the first n accumulated classes whose sum reaches target (n + 1 where all do not).
  __device__ __forceinline__ int reach(int n, u64 target) {
    __syncthreads();
    if (threadIdx.x == 0) sh.found_class = n + 1;
    __syncthreads();
    for (int i = threadIdx.x; i < n; i += NT)
      if (sh.run_key[i] >= target && (i == 0 || sh.run_key[i - 1] < target)) sh.found_class = i + 1;
    __syncthreads();
    return sh.found_class;
  }

  // The largest key: the only model's maximum has it, and with more models a class of the groups that reach `best`.
  __device__ __forceinline__ u64 best_key(float best) {
    if (a.S == 1) return (u64)__double_as_longlong(sh.scale[0]);
    const int lane = threadIdx.x & 63, listed = list_groups(best, best);
    const uint32_t* groups = (const uint32_t*)sh.sums;
    const bool some = listed <= kMaxGroupsListed;            // else all
    const int n = some ? listed : (a.C + 63) / 64;
    u64 top = 0;
    for (int i = (threadIdx.x >> 6) * G; i < n; i += kWaves * G) {
      int c[G];
      u64 x[G];
#pragma unroll
      for (int j = 0; j < G; ++j) c[j] = i + j < n ? (some ? (int)groups[i + j] : i + j) * 64 + lane : a.C;
      keys<G>(c, x);
#pragma unroll
      for (int j = 0; j < G; ++j) top = x[j] > top ? x[j] : top;
    }
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) {
      const u64 other = __shfl_xor(top, o, 64);
      top = other > top ? other : top;
    }
    __syncthreads();
    if (lane == 0) sh.wave_a[threadIdx.x >> 6] = top;
    __syncthreads();
    for (int w = 0; w < kWaves; ++w) top = sh.wave_a[w] > top ? sh.wave_a[w] : top;
    return top;
  }

  // The cut at which the number (by_sum: the sum of the units) of the classes from the top reaches
  // `target`, by histograms of the bits of p: 64 bins an octave from 1 down first (whole: of
  // all the octaves), then 11 bits a level within the bin reached, until its classes fit into the
  // list and are sorted.  False where all classes (those above 2^-63, which have units) stay
  // below target.
  __device__ __forceinline__ bool select(bool by_sum, u64 target, bool whole, Cut& cut) {
    constexpr u64 first_bin = (u64)1023 << 6;                 // bits of 1.0 >> 46
    u64 prefix_bits = 0, above_n = 0, above_sum = 0;
    int shift = whole ? 52 : 46, up = 64;
    for (;;) {
      __syncthreads();
      for (int b = threadIdx.x; b < kFlatBins; b += NT) {
        sh.sums[b] = 0;
        sh.counts[b] = 0;
      }
      if (threadIdx.x == 0) sh.found_a = kFlatBins;
      __syncthreads();
      // bins ascend as keys descend
      const u64 top_bin = up == 64 ? (whole ? 2047 : first_bin) : (prefix_bits >> shift) | (((u64)1 << (up - shift)) - 1);
      for (int u = threadIdx.x >> 6; u < a.units; u += kWaves) {
        u64 x[16];
        unit_keys(u, x);
#pragma unroll
        for (int i = 0; i < 16; ++i)
          if (x[i] != 0 && (up == 64 || x[i] >> up == prefix_bits >> up)) {
            const uint32_t at = (uint32_t)(x[i] >> shift), below = (uint32_t)top_bin - at;   // equal above 32 bits
            const int b = at > (uint32_t)top_bin && up == 64 ? 0 : (int)min(below, (uint32_t)kFlatBins - 1);
            atomicAdd(&sh.sums[b], units_of(x[i]));
            if (!by_sum) atomicAdd(&sh.counts[b], 1u);
          }
      }
      __syncthreads();
      constexpr int PER = kFlatBins / NT;
      u64 n = 0, s = 0;
#pragma unroll
      for (int i = 0; i < PER; ++i) {
        n += sh.counts[threadIdx.x * PER + i];
        s += sh.sums[threadIdx.x * PER + i];
      }
      u64 at_n = above_n + block_scan<NT>(n).before, at_s = above_sum + block_scan<NT>(s).before;
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
      if (b == kFlatBins) return false;
      if (up == 64 && !whole && b == kFlatBins - 1) return false;         // beyond 63 octaves
      prefix_bits = (top_bin - b) << shift;
      above_n = sh.found_b;
      above_sum = sh.found_c;
      bool fits = by_sum || sh.counts[b] <= kList;
      if (fits) {
        list_prefix(prefix_bits, shift);
        fits = sh.n_list <= kList;
      }
      if (fits) {
        sort();
        accumulate();
        const int r = by_sum ? reach((int)sh.n_list, target - above_sum) : (int)(target - above_n);
        cut.units = true;
        cut.key = sh.list_key[r - 1];
        cut.mass = above_sum + sh.run_key[r - 1];
        __syncthreads();
        if (threadIdx.x == 0) sh.found_class = 0;
        __syncthreads();
        int same = 0;
        for (int i = threadIdx.x; i < r; i += NT) {
          const int unit = sh.list_class[i] / kUnitClasses;
          atomicAdd(&sh.sums[unit], units_of(sh.list_key[i]));
          if (sh.list_key[i] == cut.key) {
            ++same;
            atomicAdd(&sh.unit_ties[unit], 1u);
          }
        }
        if (same) atomicAdd(&sh.found_class, same);
        __syncthreads();
        cut.ties = (u64)sh.found_class;
        return true;
      }
      if (shift == 0) {                                                // one key, in more classes than the list holds
        cut.key = prefix_bits;
        cut.units = false;
        const u64 each = units_of(cut.key);
        cut.ties = by_sum ? (target - above_sum + each - 1) / each : target - above_n;
        cut.mass = above_sum + cut.ties * each;
        return true;
      }
      up = shift;
      shift = shift > 11 ? shift - 11 : 0;
    }
  }

  // Lists the classes whose key starts with prefix_bits; sums[unit]: the units of the classes above them.
  __device__ __forceinline__ void list_prefix(u64 prefix_bits, int shift) {
    __syncthreads();
    if (threadIdx.x == 0) sh.n_list = 0;
    __syncthreads();
    const u64 want = prefix_bits >> shift;
    // with one model the logits themselves tell which classes may be there or above
    float lo = -INFINITY;
    if (a.S == 1) {
      lo = log2f((float)__longlong_as_double((long long)prefix_bits)) - kSlack;
      if (!(lo > -120.f)) lo = -INFINITY;
    }
    const Difference scaled = difference();
    for (int u = threadIdx.x; u < a.units; u += NT) sh.unit_ties[u] = 0;
    u64 above = 0;
    auto take = [&](u64 x, int c) {
      if (x >> shift > want) above += units_of(x);
      if (x != 0 && x >> shift == want) {
        const uint32_t at = atomicAdd(&sh.n_list, 1u);
        if (at < kList) {
          sh.list_key[at] = x;
          sh.list_class[at] = c;
        }
      }
    };
    for (int u = threadIdx.x >> 6; u < a.units; u += kWaves) {
      if (a.S == 1) {
        float z[16];
        unit_logits(u, 0, z);
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          const float t = scaled(z[i], sh.top[0]) + sh.log_scale[0];
          if (!(t < lo)) {
            const u64 x = (u64)__double_as_longlong(__builtin_fma(weight(z[i], sh.top[0], k), sh.scale[0], 0.0));
            take(x < kLeastKey ? 0 : x, unit_class(u, i));
          }
        }
      } else {
        u64 x[16];
        unit_keys(u, x);
#pragma unroll
        for (int i = 0; i < 16; ++i) take(x[i], unit_class(u, i));
      }
#pragma unroll
      for (int o = 32; o > 0; o >>= 1) above += __shfl_xor(above, o, 64);
      if ((threadIdx.x & 63) == 0) sh.sums[u] = above;
      above = 0;
    }
    __syncthreads();
  }

  // Draws from the first n accumulated classes, in the order of their indices.
  __device__ __forceinline__ void draw_listed(int n, u64 target, u64 mass, bool greedy) {
    __syncthreads();
    for (int i = threadIdx.x; i < n; i += NT) sh.sums[i] = sh.run_key[i] - (i ? sh.run_key[i - 1] : 0);
    __syncthreads();
    if (n > 128) {
      // sorted by index (as keys: the complement, which descends), their places beside
      for (int i = threadIdx.x; i < n; i += NT) {
        sh.list_key[i] = (u64)(0x7fffffff - sh.list_class[i]) << 16 | (u64)i;
        sh.list_class[i] = 0;
      }
      if (threadIdx.x == 0) sh.n_list = n;
      __syncthreads();                                       // sort() reads it at once
      sort();
      constexpr int PER = kList / NT;
      u64 p[PER], sum = 0;
#pragma unroll
      for (int j = 0; j < PER; ++j) {
        const int i = threadIdx.x * PER + j;
        p[j] = i < n ? sh.sums[sh.list_key[i] & 0xFFFF] : 0;
        sum += p[j];
      }
      u64 at = block_scan<NT>(sum).before;
#pragma unroll
      for (int j = 0; j < PER; ++j) {
        if (at <= target && at + p[j] > target) {
          a.labels[row] = 0x7fffffff - (int)(sh.list_key[threadIdx.x * PER + j] >> 16);
          a.out[row] = (float)((double)p[j] / (double)mass);
        }
        at += p[j];
      }
      return;
    }
    for (int i = threadIdx.x; i < n; i += NT) {
      const int c = sh.list_class[i];
      u64 before = 0;                                        // of the classes of lower index
#pragma unroll 8
      for (int j = 0; j < n; ++j) before += sh.list_class[j] < c ? sh.sums[j] : 0;
      const u64 p = sh.sums[i];
      if (before <= target && before + p > target) {
        a.labels[row] = c;
        a.out[row] = greedy ? 1.f : (float)((double)p / (double)mass);
      }
    }
  }

  // The units' masses into sums, and their sum.
  __device__ __forceinline__ u64 unit_masses() {
    u64 total = 0;
    for (int first = 0; first < a.units; first += NT) {
      const int unit = first + threadIdx.x;
      const u64 mass = unit < a.units ? unit_mass(unit) : 0;
      if (unit < a.units) sh.sums[unit] = mass;
      total += block_scan<NT>(mass).total;
    }
    return total;
  }

  // The unit in which the sums of the units' masses pass target, and what of target lies in it.
  __device__ __forceinline__ void find_unit(u64 target, int& unit, u64& rest) {
    u64 seen = 0;
    __syncthreads();
    for (int first = 0; first < a.units; first += NT) {
      const int i = first + threadIdx.x;
      const u64 mass = i < a.units ? sh.sums[i] : 0;
      const Scan scan = block_scan<NT>(mass);
      const u64 at = seen + scan.before;
      if (at <= target && at + mass > target) {
        sh.found_a = i;
        sh.found_b = target - at;
      }
      seen += scan.total;
    }
    __syncthreads();
    unit = (int)sh.found_a;
    rest = sh.found_b;
  }

  // The class c of [c0, c0 + kUnitClasses) at which the kept units pass `target`, counted from c0; the
  // first `ties` classes with key == cut are kept.  Where they stay below target (it comes from sums of
  // another rounding) the last kept; false where none has any units.
  __device__ __forceinline__ bool draw_in_unit(int c0, u64 target, u64 cut, u64 ties, u64 mass, float u) {
    constexpr int PER = kUnitClasses / NT;
    u64 x[PER], equal = 0, part = 0;
    int c[PER];
#pragma unroll
    for (int j = 0; j < PER; ++j) c[j] = c0 + threadIdx.x * PER + j;
    keys<PER>(c, x);
#pragma unroll
    for (int j = 0; j < PER; ++j) equal += x[j] == cut;
    u64 tie = ties == ~(u64)0 ? 0 : block_scan<NT>(equal).before;
#pragma unroll
    for (int j = 0; j < PER; ++j) {
      // selects: from a branch on `x < cut || (x == cut && tie++ >= ties)` the compiler of ROCm 7.2
      // drops the assignment of 0 for j = 0 in lanes that take its second half
      const bool at_cut = x[j] == cut, keep = (x[j] > cut) | (at_cut & (tie < ties));
      tie += at_cut;
      x[j] = keep ? units_of(x[j]) : 0;
      part += x[j];
    }
    const Scan scan = block_scan<NT>(part);
    const u64 total = scan.total;
    u64 at = scan.before;
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
  __device__ __forceinline__ void draw(int unit, u64 target, u64 mass, float u) {
    for (int i = 0; i < a.units; ++i) {
      const int behind = unit + i, next = behind < a.units ? behind : a.units - 1 - i;
      if (draw_in_unit(next * kUnitClasses, i == 0 ? target : next > unit ? 0 : ~(u64)0, 1, ~(u64)0, mass, u)) return;
    }
  }
};

// A row's filters, each off or within its range.
struct Filters {
  int top_k;                  // 0: off
  float top_p, min_p, u;      // 1, 0: off
  bool greedy;
};
__device__ __forceinline__ Filters row_filters(const TokenArgs& a, int row, float t) {
  Filters f{a.top_k ? a.top_k[row] : 0, a.top_p ? a.top_p[row] : 1.f, a.min_p ? a.min_p[row] : 0.f, a.uniform[row], t == 0.f};
  if (f.greedy) f = Filters{1, 1.f, 0.f, 0.f, true};
  if (f.top_p <= 0.f) f.top_k = 1;
  if (f.top_k <= 0 || f.top_k >= a.C) f.top_k = 0;
  if (!(f.top_p > 0.f && f.top_p < 1.f)) f.top_p = 1.f;
  f.min_p = f.min_p > 0.f ? fminf(f.min_p, 1.f) : 0.f;
  return f;
}

// Rows drawn from one unit or from a list; those that need more are left to sample_flat_kernel.  Apart,
// because a row's time is mostly that of fetching the code it runs through once (in one kernel of 1024 threads
// with the histograms, 3 x 16 x 30000 took 71 us; apart, in 512 threads, 30 us).
template <bool BF16, int NT>
__global__ __launch_bounds__(NT) void sample_kernel(TokenArgs a) {
  __shared__ RowShared<false> sh;
  const int row = a.row0 + blockIdx.x;
  const float t = row_temperature(a, row);
  Row<BF16, NT, false> r{a, sh, row, log2_scale(t)};
  const int state = t >= 0.f ? r.init() : 2;
  if (threadIdx.x == 0) a.flat[row] = 0;
  if (state != 0) {
    if (threadIdx.x == 0) {
      a.labels[row] = -1;
      a.out[row] = state == 1 ? 0.f : NAN;
    }
    return;
  }
  const Filters f = row_filters(a, row, t);
  const bool by_mass = f.top_p < 1.f;
  const u64 total = f.top_k ? 0 : r.unit_masses();
  if (!f.top_k && !by_mass && f.min_p == 0.f) {
    int unit;
    u64 rest;
    r.find_unit(draw_target(total, f.u), unit, rest);
    r.draw(unit, rest, total, f.u);
    return;
  }
  const float best = r.best_score();
  r.group_scores(0, best, r.low0, r.high0);
  float score;
  // top-p alone: how far the nucleus goes is not known, and a bound from more groups lists and sorts more classes, one from
  // fewer leaves more rows to the flat kernel.  From 16, 64, 256 and 640 groups, in us: 3 x 16 x 30000 with nuclei up to 31
  // classes 84, 41, 49 and 50, up to 145 81, 87, 35 and 35; 1 x 256 x 131072 up to 31 138, 57, 70 and 95, up to 125 133, 138, 71
  // and 94, up to 412 128, 132, 142 and 94.  No more than a quarter of the groups there are.
  if (f.top_k || by_mass) score = r.bound(f.top_k ? f.top_k : min(64, max(a.units * kUnitTops / 4, 4)), best);
  else score = best + __log2f(f.min_p) - kSlack;
  for (bool whole = false; r.list(score, best); whole = true) {
    r.sort();
    r.accumulate();
    int kept = (int)sh.n_list;
    whole |= kept == a.C;
    if (f.top_k) kept = min(kept, f.top_k);
    if (by_mass) {
      const u64 mass = f.top_k || whole ? sh.run_key[kept - 1] : total;
      const int reached = r.reach(kept, times_fraction(mass, f.top_p, 1));
      if (reached > kept) {                                  // the list is short of the mass
        if (a.C > kList) break;
        score = -INFINITY;
        continue;
      }
      kept = reached;
    }
    if (f.min_p > 0.f) {
      const double least = (double)f.min_p * __longlong_as_double((long long)sh.list_key[0]);
      __syncthreads();
      if (threadIdx.x == 0) sh.found_class = kept;
      __syncthreads();
      for (int i = threadIdx.x; i < kept; i += NT)
        if (__longlong_as_double((long long)sh.list_key[i]) < least) atomicMin(&sh.found_class, i);
      __syncthreads();
      kept = sh.found_class;
    }
    const u64 mass = sh.run_key[kept - 1];
    r.draw_listed(kept, draw_target(mass, f.u), mass, f.greedy);
    return;
  }
  if (threadIdx.x == 0) a.flat[row] = 1;
}

// Rows with more kept classes than sample_kernel lists: cut by histograms, then a scan of the units.  1024 threads: two
// passes over the logits, 64-bit powers and LDS atomics bound them (115 us a row of 131072 fp32; 512 threads took 15 us more).
template <bool BF16, int NT>
__global__ __launch_bounds__(NT, 4) void sample_flat_kernel(TokenArgs a) {
  __shared__ RowShared<true> sh;
  const int row = a.row0 + blockIdx.x;
  if (!a.flat[row]) return;
  const float t = row_temperature(a, row);
  Row<BF16, NT, true> r{a, sh, row, log2_scale(t)};
  r.init();
  const Filters f = row_filters(a, row, t);
  Cut cut{1, ~(u64)0, r.unit_masses(), false};
#pragma unroll 1
  for (int pass = 0; pass < 2; ++pass) {                     // one copy of select()'s code
    const bool by_sum = pass == 1;
    if (by_sum ? f.top_p < 1.f : f.top_k != 0)
      r.select(by_sum, by_sum ? times_fraction(cut.mass, f.top_p, 1) : (u64)f.top_k, false, cut);
  }
  if (f.min_p > 0.f) {
    const u64 least = (u64)__double_as_longlong((double)f.min_p * __longlong_as_double((long long)r.best_key(r.best_score())));
    if (least > cut.key) cut = Cut{least, ~(u64)0, 0, false};
    else cut.units = cut.units && a.S == 1;                  // with more models best_key() has used sums
  }
  __syncthreads();
  u64 total = 0;
  if (cut.units) {
    total = cut.mass;
  } else {
    // a wave per unit: the units above the cut, and the ties
    const int lane = threadIdx.x & 63;
    for (int unit = threadIdx.x >> 6; unit < a.units; unit += NT / 64) {
      u64 mass = 0;
      uint32_t equal = 0;
      u64 x[16];
      r.unit_keys(unit, x);
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        mass += x[i] > cut.key ? units_of(x[i]) : 0;
        equal += x[i] == cut.key;
      }
#pragma unroll
      for (int o = 32; o > 0; o >>= 1) {
        mass += __shfl_xor(mass, o, 64);
        equal += __shfl_xor(equal, o, 64);
      }
      if (lane == 0) {
        sh.sums[unit] = mass;
        sh.unit_ties[unit] = equal;
      }
    }
    __syncthreads();
    const u64 each = units_of(cut.key);
    u64 seen_ties = 0;
    for (int first = 0; first < a.units; first += NT) {
      const int unit = first + threadIdx.x;
      const u64 equal = unit < a.units ? sh.unit_ties[unit] : 0;
      const Scan scan = block_scan<NT>(equal);
      const u64 before = seen_ties + scan.before;
      const u64 kept = before >= cut.ties ? 0 : equal < cut.ties - before ? equal : cut.ties - before;
      const u64 mass = unit < a.units ? sh.sums[unit] + kept * each : 0;
      total += block_scan<NT>(mass).total;
      if (unit < a.units) {
        sh.sums[unit] = mass;
        sh.unit_ties[unit] = (uint32_t)kept;
      }
      seen_ties += scan.total;
    }
  }
  int unit;
  u64 rest;
  r.find_unit(draw_target(total, f.u), unit, rest);
  r.draw_in_unit(unit * kUnitClasses, rest, cut.key, sh.unit_ties[unit], total, f.u);
}

// Sorts the list of a row's first classes and writes it.
template <bool BF16, int NT, bool FLAT>
__device__ __forceinline__ void write_topk(const TokenArgs& a, RowShared<FLAT>& sh, Row<BF16, NT, FLAT>& r, int row) {
  r.sort();
  const int n = (int)sh.n_list;
  for (int j = threadIdx.x; j < a.k; j += NT) {
    const u64 key = j < n ? sh.list_key[j] : 0;
    a.labels[(long long)row * a.k + j] = key ? sh.list_class[j] : -1;
    a.out[(long long)row * a.k + j] = key ? (float)log(__longlong_as_double((long long)key)) : -INFINITY;
  }
}

template <bool BF16, int NT>
__global__ __launch_bounds__(NT) void topk_kernel(TokenArgs a) {
  __shared__ RowShared<false> sh;
  const int row = a.row0 + blockIdx.x;
  Row<BF16, NT, false> r{a, sh, row, log2_scale(a.t_all)};
  const int state = r.init();
  const float best = r.best_score();
  r.group_scores(0, best, r.low0, r.high0);
  const bool listed = state != 0 || r.list(r.bound(a.k, best), best);
  if (threadIdx.x == 0) a.flat[row] = !listed;
  if (state != 0) {
    for (int j = threadIdx.x; j < a.k; j += NT) {
      a.labels[(long long)row * a.k + j] = -1;
      a.out[(long long)row * a.k + j] = state == 1 ? -INFINITY : NAN;
    }
  } else if (listed) {
    write_topk(a, sh, r, row);
  }
}

// Rows whose groups do not bound the k-th class closely enough for a list: the cut by histograms; the
// list is then the classes above it and the first ties.
template <bool BF16, int NT>
__global__ __launch_bounds__(NT, 4) void topk_flat_kernel(TokenArgs a) {
  __shared__ RowShared<true> sh;
  const int row = a.row0 + blockIdx.x;
  if (!a.flat[row]) return;
  Row<BF16, NT, true> r{a, sh, row, log2_scale(a.t_all)};
  r.init();
  Cut cut{1, ~(u64)0, 0, false};
  r.select(false, (u64)a.k, true, cut);
  __syncthreads();
  if (threadIdx.x == 0) sh.n_list = 0;
  __syncthreads();
  u64 seen_ties = 0;
  for (int c0 = 0; c0 < a.C; c0 += NT) {
    const int c = c0 + threadIdx.x;
    const u64 key = c < a.C ? r.key(c) : 0;
    const Scan scan = block_scan<NT>(key == cut.key);
    const u64 tie = seen_ties + scan.before;
    if ((key > cut.key) | ((key == cut.key) & (tie < cut.ties))) {
      const uint32_t i = atomicAdd(&sh.n_list, 1u);
      if (i < kList) {
        sh.list_key[i] = key;
        sh.list_class[i] = c;
      }
    }
    seen_ties += scan.total;
  }
  __syncthreads();
  write_topk(a, sh, r, row);
}

template <bool BF16>
hipError_t launch_stats(const TokenArgs& a, hipStream_t s) {
  const int waves = std::min(a.units, 4);
  TokenArgs part = a;
  for (long long row = 0; row < a.n; row += 1 << 20) {
    part.row0 = (int)row;
    launch(stats_kernel<BF16>, dim3((unsigned)std::min<long long>(a.n - row, 1 << 20), (a.units + waves - 1) / waves, a.S),
           dim3(64 * waves), s, part);
    const hipError_t st = hipGetLastError();
    if (st != hipSuccess) return st;
  }
  return hipSuccess;
}

// A workgroup per row, 2^20 rows a launch at most.
template <typename F>
hipError_t launch_row_kernel(F kernel, int threads, const TokenArgs& a, hipStream_t s) {
  TokenArgs part = a;
  for (long long row = 0; row < a.n; row += 1 << 20) {
    part.row0 = (int)row;
    launch(kernel, dim3((unsigned)std::min<long long>(a.n - row, 1 << 20)), dim3(threads), s, part);
    const hipError_t st = hipGetLastError();
    if (st != hipSuccess) return st;
  }
  return hipSuccess;
}

}  // namespace

hipError_t launch_sample(const TokenArgs& a, bool bf16, hipStream_t s) {
  hipError_t st = bf16 ? launch_stats<true>(a, s) : launch_stats<false>(a, s);
  if (st != hipSuccess) return st;
  st = bf16 ? launch_row_kernel(sample_kernel<true, 512>, 512, a, s) : launch_row_kernel(sample_kernel<false, 512>, 512, a, s);
  if (st != hipSuccess || a.C <= kList) return st;           // every class fits into a list
  if (!a.temperature && !a.top_k && !a.top_p && !a.min_p) return st;   // a unit always does
  return bf16 ? launch_row_kernel(sample_flat_kernel<true, 1024>, 1024, a, s)
              : launch_row_kernel(sample_flat_kernel<false, 1024>, 1024, a, s);
}

hipError_t launch_topk(const TokenArgs& a, bool bf16, hipStream_t s) {
  hipError_t st = bf16 ? launch_stats<true>(a, s) : launch_stats<false>(a, s);
  if (st != hipSuccess) return st;
  st = bf16 ? launch_row_kernel(topk_kernel<true, 512>, 512, a, s) : launch_row_kernel(topk_kernel<false, 512>, 512, a, s);
  if (st != hipSuccess || a.C <= kList) return st;
  return bf16 ? launch_row_kernel(topk_flat_kernel<true, 1024>, 1024, a, s)
              : launch_row_kernel(topk_flat_kernel<false, 1024>, 1024, a, s);
}

}  // namespace rafiki
