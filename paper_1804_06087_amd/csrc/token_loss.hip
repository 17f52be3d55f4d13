// Log-probabilities of given tokens, the clipped policy loss and the preference loss with their
// gradients (rafiki_tokens.h).
//
// With x_c = (z_c - top) log2(e) / T, l the row's label, top the row's maximum and the sum over all classes but l:
//     R = sum 2^x_c,   S = R + 2^x_l,   1 - p_l = R / S,   log p_l = ln 2 x_l - log S   (- log(1 + R) where the label is the maximum),
// which keeps 1 - p_l and log p_l exact where p_l is near 1: a sum over all classes would have lost the others'.
// The gradient is affine in log p under p:  dz_c = 2^x_c (f + f' x_c) for c != l, with f' = 0 without entropy.
// The maximum is the largest logit so far, the same in a wave: it grows a few times in a row, and the sums move with it.
//
// Bound by bytes: logits read once and the gradient written once, where the factors f are the row's own; a preference loss
// has them from all rows of a pair and reads the logits twice.  Measured on an MI355X (a device copy moves 4.8 TB/s): 8192 x
// 131072 bf16 log p and entropy 317 us (5.8 TB/s of what has a token; 11 vector instructions a class, so the clock counts too),
// 4096 x 30000 bf16 policy loss with entropy and gradient 103 us (4.4 TB/s; with a maximum of each thread 133), 1500 x 50021
// fp32 125 us (4.5), 3 pairs of 2 x 880 rows of 131071 bf16 740 us, of which the sums take 221 (5.4 TB/s) and the
// gradient 520 (5.1 TB/s).  Pairs in groups that a cache might hold until their gradient is taken were slower (8
// groups of 2 pairs of 2 x 500 x 30000 663 us, all at once 557).
#include "tokens.h"

#include <algorithm>
#include <type_traits>

namespace rafiki {

namespace {

typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4_any __attribute__((ext_vector_type(4), aligned(2)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef float f32x2 __attribute__((ext_vector_type(2)));

// BF16 as a template's parameter: 0 fp32 values, 1 bf16, 2 bf16 in rows that may start off 16-byte boundaries.

__device__ __forceinline__ float power2(float t) { return __builtin_amdgcn_exp2f(t); }

template <int BF16>
__device__ __forceinline__ float element(const void* p, long long i) {
  if constexpr (BF16 != 0) return __uint_as_float((uint32_t)((const bf16_t*)p)[i] << 16);
  else return ((const float*)p)[i];
}
// Rounded once, to nearest, ties to even; NaN stays NaN.
template <int BF16>
__device__ __forceinline__ void put(void* p, long long i, float v) {
  if constexpr (BF16 != 0) ((__bf16*)p)[i] = (__bf16)v;
  else ((float*)p)[i] = v;
}
template <int BF16, int V>
__device__ __forceinline__ void unpack(u32x4 q, float z[V]) {
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    if constexpr (BF16 != 0) {
      z[2 * j] = __uint_as_float(q[j] << 16);
      z[2 * j + 1] = __uint_as_float(q[j] & 0xFFFF0000u);
    } else {
      z[j] = __uint_as_float(q[j]);
    }
  }
}
template <int BF16, int V>
__device__ __forceinline__ u32x4 pack(const float z[V]) {
  u32x4 q;
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    if constexpr (BF16 != 0) q[j] = __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2{z[2 * j], z[2 * j + 1]}, bf16x2));
    else q[j] = __float_as_uint(z[j]);
  }
  return q;
}

// f over W neighbouring lanes, in each of them, all of which call it: neighbours, pairs, fours and eights mirrored, then rows
// of 16 and halves of the wave exchanged.  All by vector instructions: with shuffles, which go through LDS, 20000 x 20000 bf16
// without a gradient took 138 us instead of 134.
template <int CTRL>
__device__ __forceinline__ uint32_t exchanged(uint32_t v) {
  return (uint32_t)__builtin_amdgcn_update_dpp((int)v, (int)v, CTRL, 0xF, 0xF, false);
}
template <int CTRL>
__device__ __forceinline__ float exchanged(float v) { return __uint_as_float(exchanged<CTRL>(__float_as_uint(v))); }
template <int CTRL>
__device__ __forceinline__ int exchanged(int v) { return (int)exchanged<CTRL>((uint32_t)v); }
template <int CTRL>
__device__ __forceinline__ double exchanged(double v) {
  const u32x2 q = __builtin_bit_cast(u32x2, v);
  return __builtin_bit_cast(double, u32x2{exchanged<CTRL>(q[0]), exchanged<CTRL>(q[1])});
}
// The values of both rows (O = 16) or halves (O = 32) of a pair.
template <int O>
__device__ __forceinline__ void both(uint32_t v, uint32_t& a, uint32_t& b) {
  const auto r = O == 16 ? __builtin_amdgcn_permlane16_swap(v, v, false, false) : __builtin_amdgcn_permlane32_swap(v, v, false, false);
  a = r[0];
  b = r[1];
}
template <int O, typename T>
__device__ __forceinline__ void both(T v, T& a, T& b) {
  if constexpr (sizeof(T) == 8) {
    const u32x2 q = __builtin_bit_cast(u32x2, v);
    u32x2 x, y;
    uint32_t lo[2], hi[2];
    both<O>(q[0], lo[0], lo[1]);
    both<O>(q[1], hi[0], hi[1]);
    x = u32x2{lo[0], hi[0]};
    y = u32x2{lo[1], hi[1]};
    a = __builtin_bit_cast(T, x);
    b = __builtin_bit_cast(T, y);
  } else {
    uint32_t x, y;
    both<O>(__builtin_bit_cast(uint32_t, v), x, y);
    a = __builtin_bit_cast(T, x);
    b = __builtin_bit_cast(T, y);
  }
}
template <int W, typename T, typename F>
__device__ __forceinline__ T over_lanes(T v, F f) {
  if constexpr (W >= 2) v = f(v, exchanged<0xB1>(v));
  if constexpr (W >= 4) v = f(v, exchanged<0x4E>(v));
  if constexpr (W >= 8) v = f(v, exchanged<0x141>(v));
  if constexpr (W >= 16) v = f(v, exchanged<0x140>(v));
  T a, b;
  if constexpr (W >= 32) both<16>(v, a, b), v = f(a, b);
  if constexpr (W >= 64) both<32>(v, a, b), v = f(a, b);
  return v;
}
template <int W = 64>
__device__ __forceinline__ float wave_max(float v) {
  return over_lanes<W>(v, [](float a, float b) { return fmaxf(a, b); });
}
template <int W = 64, typename T>
__device__ __forceinline__ T wave_add(T v) {
  return over_lanes<W>(v, [](T a, T b) { return a + b; });
}

// Exponents of 2 as factors of a power that is 0 below here: -inf would make it NaN.
__device__ __forceinline__ float finite_log2(float x) { return fmaxf(x, -16384.f); }

// A row of C values as chunks of 16 bytes, chunk i from class i V - shift on.  Rows may start anywhere; unaligned chunks of bf16
// values were a fifth slower (6000 x 131071 321 us, 6000 x 131072 257; fp32 rows take as long either way), so those are
// taken on 16-byte boundaries of the logits.  The first and the last chunk may have fewer values, and are read from class
// 0 or C - V on.
template <int BF16>
struct Row {
  static constexpr int V = BF16 ? 8 : 4;
  const char* x;
  int C, shift, chunks, label;

  __device__ __forceinline__ void init(const void* logits, long long base, int C_, int label_) {
    x = (const char*)logits + base * (16 / V);
    C = C_;
    shift = BF16 == 2 ? (int)((uintptr_t)x & 15) / 2 : 0;
    chunks = (C + shift + V - 1) / V;
    label = label_;
  }
  __device__ __forceinline__ float at(int c) const { return element<BF16>(x, c); }
  // Chunk i with -inf in the label's place and in those of classes that it does not have.
  template <bool STREAM>
  __device__ __forceinline__ u32x4 load(int i) const {
    const int c0 = i * V - shift, first = min(BF16 == 2 ? max(c0, 0) : c0, C - V);
    u32x4 q;
    if (C >= V) {
      const u32x4_any* p = (const u32x4_any*)(x + (long long)first * (16 / V));
      if constexpr (STREAM) q = __builtin_nontemporal_load(p);
      else q = *p;
    }
    if (c0 != first || (unsigned)(label - c0) < (unsigned)V) {
      float z[V];
      if (C < V) {
#pragma unroll
        for (int j = 0; j < V; ++j) z[j] = (unsigned)(c0 + j) < (unsigned)C ? at(c0 + j) : -INFINITY;
      } else if (c0 != first) {
        float t[V];
        unpack<BF16, V>(q, t);
#pragma unroll
        for (int j = 0; j < V; ++j) {
          z[j] = -INFINITY;
#pragma unroll
          for (int k = 0; k < V; ++k) z[j] = k == j + c0 - first ? t[k] : z[j];
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
    const int c0 = i * V - shift;
    if ((unsigned)(label - c0) < (unsigned)V) {
#pragma unroll
      for (int j = 0; j < V; ++j) d[j] = c0 + j == label ? at_label : d[j];
    }
    if (c0 >= 0 && c0 + V <= C) {
      __builtin_nontemporal_store(pack<BF16, V>(d), (u32x4_any*)(row + (long long)c0 * (16 / V)));
    } else {
#pragma unroll
      for (int j = 0; j < V; ++j)
        if ((unsigned)(c0 + j) < (unsigned)C) put<BF16>(row, c0 + j, d[j]);
    }
  }
  __device__ __forceinline__ void zero_chunk(char* row, int i) const {
    float d[V];
#pragma unroll
    for (int j = 0; j < V; ++j) d[j] = 0.f;
    store(row, i, d, 0.f);
  }
  template <int NT>
  __device__ __forceinline__ void zero(char* row, int tid) const {
    for (int i = tid; i < chunks; i += NT) zero_chunk(row, i);
  }
};

// The exponents x = (z - top) log2(e) / T of a row's classes, with roundings that go either way: log2(e) / T is a number of
// fewer bits and a rest, since a scale rounded to fp32 would move every log p the same way.  log p is off by 1.5e-8 (fp32) to 3e-8
// (bf16 logits) rms, 7e-8 at most; with x relative to the label's logit, up to 40 and in a rounded scale, a label 24 T below
// the top was off by 8e-7 on average and up to 2.4e-6 (T = 0.71, 100 to 200003 classes).
//   fp32: d = z - top,  x = d hi + d lo.
//   bf16: x = y + y rest, y = z hi - top hi, which for hi of 16 bits are exact products.
// lo and rest are positive, so that -inf stays -inf.  Classes 2^80 and more below `top` have no power with any scale.
template <int BF16>
struct Exponent {
  float hi, lo, at;
  __device__ __forceinline__ void relative_to(float top, const Scale& s) {
    if constexpr (BF16 != 0) {
      hi = fabsf(top) > 0x1p100f ? fminf(s.hi16, 1.f) : s.hi16;   // no overflow
      lo = s.rest16;
      at = top * hi;
    } else {
      hi = s.hi;
      lo = s.lo;
      at = top;
    }
  }
  __device__ __forceinline__ float of(float z) const {
    if constexpr (BF16 != 0) {
      const float y = fmaf(z, hi, -at);
      return fmaf(y, lo, y);
    } else {
      const float d = z - at;
      return fmaf(d, hi, d * lo);
    }
  }
};

// Sums over classes, the label's apart: 2^x and of those times x.  A thread adds a chunk's in 32 bits and
// the chunks in 64: unlikely classes by the thousand, each below the last bit of a likely one's sum, would be lost in 32
// (log p of 131071 classes off by 1.4e-6 on average; the additions cost nothing that the loads do not hide).
//
// The entropy of a row that is nearly sure, H = log S - ln 2 sum 2^x x / S, is all in the classes below the maximum, whose power is
// 1 and whose x is 0.  With entropy (ENT) those powers are counted apart, so that nothing is lost beside them: both terms are
// positive, log S = log(1 + the rest), and H keeps its digits however small it is.
struct Sums {
  double sum, moment;
  float top;                  // finite: with no class and no label above -inf, the least number
  float ones;                 // ENT: classes at the top, which `sum` leaves out; otherwise 0
};
constexpr float kLeast = -0x1.fffffep127f;

template <int V>
__device__ __forceinline__ float tree_sum(const float v[V]) {
  if constexpr (V == 8) return ((v[0] + v[1]) + (v[2] + v[3])) + ((v[4] + v[5]) + (v[6] + v[7]));
  else return (v[0] + v[1]) + (v[2] + v[3]);
}
// The compiler's maximum makes NaN of loaded values quiet first, an instruction each.  A row with NaN may have any reference.
__device__ __forceinline__ float max3(float a, float b, float c) {
  asm("v_max3_f32 %0, %0, %1, %2" : "+v"(a) : "v"(b), "v"(c));
  return a;
}
template <int V>
__device__ __forceinline__ float chunk_max(const float v[V]) {
  float top = v[0];
#pragma unroll
  for (int j = 1; j < V; j += 2) top = max3(top, v[j], v[j + 1 < V ? j + 1 : j]);
  return top;
}
// 2^step, step <= 0, with what is rounded off the exponent.
__device__ __forceinline__ double grown(double step) {
  const float x = (float)step;
  return (double)power2(x) * (1.0 + 0.6931471805599453 * (step - (double)x));
}
__device__ __forceinline__ double step_between(float from, float to, double s) { return fmax(((double)from - (double)to) * s, -16384.0); }
// The same sums relative to `top`, at least their own.
template <bool ENT>
__device__ __forceinline__ Sums moved(const Sums& v, float top, double s) {
  if (top == v.top) return v;
  const double sum = v.sum + (ENT ? (double)v.ones : 0.0);
  if (sum == 0.0) return Sums{0.0, 0.0, top, 0.f};
  const double step = step_between(v.top, top, s), factor = grown(step);
  return Sums{sum * factor, ENT ? (v.moment + sum * step) * factor : 0.0, top, 0.f};
}
// A row's sums in W neighbouring lanes, which have the same `top`: the largest logit so far.
// FINE (without entropy): the few chunks of a likely class are added in 64 bits throughout.  Beside it unlikely classes lose more
// than they gain by rounding: log p of bf16 rows of 30000 is 2.5e-8 above its value on average, 1.2e-8 with FINE.
template <int BF16, int W, bool ENT, bool FINE>
struct RowSums {
  static_assert(!(ENT && FINE), "without entropy");
  static constexpr int V = Row<BF16>::V;
  Sums a;
  Exponent<BF16> x;
  __device__ __forceinline__ void start(float top, const Scale& s) {
    a = Sums{0.0, 0.0, top, 0.f};
    x.relative_to(top, s);
  }
  // A chunk in each lane.
  __device__ __forceinline__ void add_any(const float z[V], const Scale& s) {
    const float top = chunk_max<V>(z);
    if (__any(top > a.top)) {
      a = moved<ENT>(a, fmaxf(a.top, wave_max<W>(top)), s.s);
      x.relative_to(a.top, s);
    }
    add(z);
  }
  // The same of classes up to `top`.
  __device__ __forceinline__ void add(const float z[V]) {
    float e[V], m = 0.f;
#pragma unroll
    for (int j = 0; j < V; ++j) {
      const float t = x.of(z[j]);
      e[j] = power2(t);
      if constexpr (ENT) m = fmaf(e[j], finite_log2(t), m);
    }
    float sum = tree_sum<V>(e);
    if constexpr (FINE) {
      if (__any(sum >= 0.25f)) {
        double all[2] = {(double)e[0], (double)e[1]};
#pragma unroll
        for (int j = 2; j < V; ++j) all[j & 1] += (double)e[j];
        a.sum += sum >= 0.25f ? all[0] + all[1] : (double)sum;   // by its own lane's classes, whatever row its neighbours have
        return;
      }
    }
    if constexpr (ENT) {
      a.moment += (double)m;
      asm volatile("" : "+v"(a.moment));                     // or the compiler sinks it behind the branches, with all of its terms
      if (__any(sum >= 1.f)) {                               // else none of them is 1
        float below[V];
#pragma unroll
        for (int j = 0; j < V; ++j) below[j] = __builtin_amdgcn_fractf(e[j]);   // 0 of 1, else e[j]
        const float rest = tree_sum<V>(below);
        a.ones += __builtin_rintf(sum - rest);
        sum = rest;
      }
    }
    a.sum += (double)sum;
  }
};
// The sums of W lanes with tops of their own, in each of them.
template <int W, bool ENT>
__device__ __forceinline__ Sums join_any(Sums a, const Scale& s) {
  a = moved<ENT>(a, wave_max<W>(a.top), s.s);
  a.sum = wave_add<W>(a.sum);
  if (ENT) a.moment = wave_add<W>(a.moment), a.ones = wave_add<W>(a.ones);
  return a;
}
// The sums of NT threads, the same top in a wave: in each of them (NT <= 64), else in the first wave, behind a barrier.
template <int NT, bool ENT>
__device__ __forceinline__ Sums join(Sums a, const Scale& s, Sums* waves) {
  constexpr int W = NT < 64 ? NT : 64;
  a.sum = wave_add<W>(a.sum);
  if (ENT) a.moment = wave_add<W>(a.moment), a.ones = wave_add<W>(a.ones);
  if constexpr (NT > 64) {
    constexpr int NW = NT / 64;
    if ((threadIdx.x & 63) == 0) waves[threadIdx.x >> 6] = a;
    __syncthreads();
    if (threadIdx.x < 64) a = join_any<NW, ENT>(waves[threadIdx.x % NW], s);
  }
  return a;
}

// What a row's sums and its label's logit say.  64 bits: the difference of two logits may exceed fp32, and what follows
// subtracts log p and H.
struct RowFacts {
  double logp, entropy, ln_total;
  double rest, p;             // 1 - p of the label, p of the label
  double share;               // p of any class is 2^x share, x as in the sums; at least 1 / C
  bool defined;
};
template <bool ENT>
__device__ __forceinline__ RowFacts row_facts(const Sums& r, float z, double inv_t) {
  RowFacts f;
  const double D = ((double)z - (double)r.top) * inv_t, e_y = exp(D), sum = r.sum + (double)r.ones, total = sum + e_y;
  f.defined = total > 0.0 && total < INFINITY;
  f.share = 1.0 / total;
  f.rest = sum * f.share;
  f.p = e_y * f.share;
  // S - 1, the power of one class at the top apart: the label's, or one of those that are counted
  const double others = D == 0.0 ? sum : ENT ? r.sum + e_y + ((double)r.ones - 1.0) : total - 1.0;
  // log(1 + others) by the logarithm of the rounded sum and what the rounding left (Kahan); the library's log1p takes longer
  // in one wave (4096 x 30000 bf16 107.5 us, 104.5)
  const double w = 1.0 + others;
  f.ln_total = w == 1.0 ? others : log(w) * (others / (w - 1.0));
  f.logp = f.defined ? D - f.ln_total : NAN;
  f.entropy = 0.0;
  if (ENT) {
    const double own = e_y > 0.0 ? e_y * D : 0.0;
    f.entropy = f.defined ? f.ln_total - (0.6931471805599453 * r.moment + own) * f.share : NAN;
  }
  return f;
}

// What the gradient pass needs: dz = 2^x (f0 + f1 x) with x = (z - top) s, and the label's.
struct RowGrad {
  float f0, f1, at_label, top;
};
template <bool ENT>
__device__ __forceinline__ RowGrad row_grad(const RowFacts& f, float a, float h, float top, double inv_t) {
  if (!f.defined || !(fabsf(a) < INFINITY) || h != h) return RowGrad{NAN, 0.f, NAN, 0.f};
  const double share = f.share * inv_t;
  if (!ENT) return RowGrad{(float)(-a * share), 0.f, (float)(a * f.rest * inv_t), top};
  double at_label = a * f.rest;
  if (f.p > 0.0) at_label -= h * f.p * (f.logp + f.entropy);
  return RowGrad{(float)(share * (-a - h * (f.entropy - f.ln_total))), (float)(share * h * -0.6931471805599453),
                 (float)(at_label * inv_t), top};
}

// What a loss makes of a row's facts: its outputs and the gradient's factors (in every thread that calls it).
template <bool POLICY, bool ENT>
__device__ __forceinline__ RowGrad finish_row(const TokenLossArgs& a, int row, const RowFacts& f, float top, bool writes) {
  float da, dh;
  if constexpr (POLICY) {
    // 64 bits: r and exp(d) are powers of differences, and kl is what is left of them
    double loss = 0.0, kl = 0.0, slope = 0.0;
    const double A = a.advantage[row];
    if (A != 0.0) {
      double ratio = a.old_logp ? exp(f.logp - (double)a.old_logp[row]) : f.logp == f.logp ? 1.0 : f.logp;
      if ((float)ratio == INFINITY) ratio = INFINITY;
      const double kept = fmin(fmax(ratio, 1.0 - a.clip_low), 1.0 + a.clip_high);
      const double plain = ratio * A, cut = kept * A;
      loss = plain != plain ? plain : -fmin(plain, cut);
      slope = plain != plain ? plain : plain <= cut ? -plain : 0.0;
    }
    if (a.ref_logp) {
      const double d = (double)a.ref_logp[row] - f.logp, e = expm1(d);
      const bool beyond = (float)e == INFINITY;
      kl = beyond ? INFINITY : e - d;
      if (a.kl_coef != 0.0) {
        loss += a.kl_coef * kl;
        slope -= a.kl_coef * (beyond ? INFINITY : e);
      }
    }
    if (a.entropy_coef != 0.0) loss -= a.entropy_coef * f.entropy;
    if (!f.defined) loss = kl = NAN;
    if (writes) {
      if (a.loss) a.loss[row] = (float)loss;
      if (a.kl) a.kl[row] = (float)kl;
    }
    const float g = a.grad_loss ? a.grad_loss[row] : 1.f;
    da = loss != loss ? NAN : g * (float)slope;
    dh = g * -(float)a.entropy_coef;
  } else {
    da = a.grad_logp ? a.grad_logp[row] : 0.f;
    dh = a.grad_entropy ? a.grad_entropy[row] : 0.f;
  }
  if (writes) {
    if (a.logp) a.logp[row] = (float)f.logp;
    if (a.entropy) a.entropy[row] = (float)f.entropy;
  }
  return row_grad<ENT>(f, da, dh, top, a.inv_t);
}

template <int BF16>
__device__ __forceinline__ u32x4 masked_chunk() {
  constexpr uint32_t m = BF16 ? 0xFF80FF80u : 0xFF800000u;   // -inf in every place
  return u32x4{m, m, m, m};
}

// f(a chunk's values) for the chunks begin .. last - 1 of a row that is read for it, by NT threads, UN of each in flight (LAST: for
// the last time, one chunk after another).  A wave's lanes call f together, some for a chunk of -inf behind the last.
template <int BF16, bool LAST, int UN, int NT, typename F>
__device__ __forceinline__ void for_chunks(const Row<BF16>& r, int begin, int last, F&& f) {
  constexpr int V = Row<BF16>::V;
  const int lane = threadIdx.x % (NT < 64 ? NT : 64);
  const int wave = NT > 64 ? __builtin_amdgcn_readfirstlane(threadIdx.x / 64) : 0;
  for (int b = begin + wave * 64; b < last; b += NT * UN) {
    u32x4 q[UN];
#pragma unroll
    for (int u = 0; u < UN; ++u) {
      q[u] = masked_chunk<BF16>();
      if (b + u * NT + lane < last) q[u] = r.template load<LAST>(b + u * NT + lane);
    }
#pragma unroll
    for (int u = 0; u < UN; ++u) {
      if (u > 0 && b + u * NT >= last) break;
      float z[V];
      unpack<BF16, V>(q[u], z);
      f(z, b + u * NT + lane);
    }
  }
}

// Chunk i's gradient from its values.
template <int BF16, bool ENT>
__device__ __forceinline__ void store_gradient(const Row<BF16>& r, char* row, int i, float z[Row<BF16>::V], const Exponent<BF16>& x,
                                               const RowGrad& d) {
#pragma unroll
  for (int j = 0; j < Row<BF16>::V; ++j) {
    const float t = x.of(z[j]);
    z[j] = power2(t) * (ENT ? fmaf(d.f1, finite_log2(t), d.f0) : d.f0);
  }
  r.store(row, i, z, d.at_label);
}

// Opens a row: whether it has a token, and whether its gradient is 0 by its weights.
template <int BF16, bool POLICY>
__device__ __forceinline__ bool open_row(const TokenLossArgs& a, int row, Row<BF16>& r, bool& weightless) {
  const int label = a.labels[row];
  r.init(a.logits, row * a.ld_row, a.C, label);
  if (POLICY) weightless = a.grad_loss && a.grad_loss[row] == 0.f;
  else weightless = !((a.grad_logp && a.grad_logp[row] != 0.f) || (a.grad_entropy && a.grad_entropy[row] != 0.f));
  return (unsigned)label < (unsigned)a.C;
}
__device__ __forceinline__ void no_token(const TokenLossArgs& a, int row) {
  if (a.loss) a.loss[row] = 0.f;
  if (a.logp) a.logp[row] = 0.f;
  if (a.kl) a.kl[row] = 0.f;
  if (a.entropy) a.entropy[row] = 0.f;
}

// NT threads per row, G rows a workgroup (G > 1: up to a wave each).  CH > 0: the row, of at most NT CH chunks, stays in registers
// from its sums to its gradient, so that it is read once; CH = 0: any length, read again for the gradient.
template <int BF16, bool POLICY, bool ENT, int NT, int CH, int G, bool REST, int OCC>
__global__ __launch_bounds__(NT * G, OCC) void token_loss_kernel(TokenLossArgs a) {
  constexpr int V = Row<BF16>::V, NW = (NT + 63) / 64, W = NT < 64 ? NT : 64;
  static_assert(G == 1 || NT <= 64, "rows that share a workgroup have no barrier");
  __shared__ Sums waves[NW];
  __shared__ RowGrad shared_grad;
  const int row = a.row0 + blockIdx.x * G + (G > 1 ? threadIdx.x / NT : 0), tid = threadIdx.x % NT;
  if (G > 1 && row >= a.n) return;
  Row<BF16> r;
  bool weightless;
  const bool token = open_row<BF16, POLICY>(a, row, r, weightless);
  char* const d_row = (char*)a.grad + row * a.ld_grad * (16 / V);
  if (a.grad && (!token || weightless)) r.template zero<NT>(d_row, tid);
  if (!token) {
    if (tid == 0) no_token(a, row);
    return;
  }
  if (weightless && !(a.loss || a.logp || a.kl || a.entropy)) return;

  u32x4 held[CH > 0 ? CH : 1];
  if constexpr (CH > 0) {
#pragma unroll
    for (int i = 0; i < CH; ++i) {
      held[i] = masked_chunk<BF16>();
      if (i * NT + tid < r.chunks) held[i] = r.template load<true>(i * NT + tid);
    }
  }
  const float z_label = r.at(r.label);
  auto each = [&](auto last, auto&& f) {
    if constexpr (CH > 0) {
#pragma unroll
      for (int i = 0; i < CH; ++i) {
        float z[V];
        // opaque here, or the compiler keeps every pass's unpacked values for the next one
        asm volatile("" : "+v"(held[i][0]), "+v"(held[i][1]), "+v"(held[i][2]), "+v"(held[i][3]));
        unpack<BF16, V>(held[i], z);
        f(z, i * NT + tid, std::true_type{});
        __builtin_amdgcn_sched_barrier(0);                   // one chunk's values at a time in registers
      }
    }
    if constexpr (REST) {
      for_chunks<BF16, decltype(last)::value, (decltype(last)::value && CH != 0 ? 1 : 4), NT>(
          r, NT * CH, r.chunks, [&](float* z, int i) { f(z, i, std::false_type{}); });
    }
  };
  RowSums<BF16, W, ENT, false> sum;
  float top = fmaxf(z_label, kLeast);
  if constexpr (CH > 0) {
#pragma unroll
    for (int i = 0; i < CH; ++i) {
      float z[V];
      unpack<BF16, V>(held[i], z);
      top = fmaxf(top, chunk_max<V>(z));
    }
    top = wave_max<W>(top);
  }
  sum.start(top, a.s);
  each(std::false_type{}, [&](const float* z, int, auto in_registers) {
    if constexpr (decltype(in_registers)::value) sum.add(z);
    else sum.add_any(z, a.s);
  });
  const Sums sums = join<NT, ENT>(sum.a, a.s, waves);
  RowGrad d{};
  if (NW == 1 || threadIdx.x < 64) {
    d = finish_row<POLICY, ENT>(a, row, row_facts<ENT>(sums, z_label, a.inv_t), sums.top, tid == 0);
    if (NW > 1 && tid == 0) shared_grad = d;
  }
  if (!a.grad || weightless) return;
  if constexpr (NW > 1) {
    __syncthreads();
    d = shared_grad;
  }
  Exponent<BF16> x;
  x.relative_to(d.top, a.s);
  each(std::true_type{}, [&](float* z, int i, auto) {
    if (i < r.chunks) store_gradient<BF16, ENT>(r, d_row, i, z, x, d);
  });
}

// ---------------------------------------------------------------- rows in parts

// The sums over a row's chunks begin .. last - 1, joined over NT threads.
template <int BF16, bool ENT, bool FINE, int NT>
__device__ __forceinline__ Sums row_sums(const Row<BF16>& r, int begin, int last, float z_label, const Scale& s, Sums* waves) {
  RowSums<BF16, (NT < 64 ? NT : 64), ENT, FINE> sum;
  sum.start(fmaxf(z_label, kLeast), s);
  for_chunks<BF16, false, 4, NT>(r, begin, last, [&](const float* z, int) { sum.add_any(z, s); });
  return join<NT, ENT>(sum.a, s, waves);
}
// The sums of a row's part p, chunks p per .. + per - 1, into *out.
template <int BF16, bool ENT, int NT>
__device__ __forceinline__ void part_sums(const Row<BF16>& r, int p, int per, const Scale& s, Sums* out) {
  __shared__ Sums waves[NT / 64];
  const Sums sums = row_sums<BF16, ENT, false, NT>(r, p * per, min(r.chunks, (p + 1) * per), r.at(r.label), s, waves);
  if (threadIdx.x == 0) *out = sums;
}
// A row's sums from its parts', in every lane of a wave.
template <bool ENT>
__device__ __forceinline__ Sums join_parts(const Sums* parts, int n, const Scale& s) {
  Sums a{0.0, 0.0, kLeast, 0.f};
  for (int p = threadIdx.x & 63; p < n; p += 64) {
    const float top = fmaxf(a.top, parts[p].top);
    const Sums b = moved<ENT>(parts[p], top, s.s);
    a = moved<ENT>(a, top, s.s);
    a.sum += b.sum;
    a.moment += b.moment;
    a.ones += b.ones;
  }
  return join_any<64, ENT>(a, s);
}

template <int BF16, bool POLICY, bool ENT, int NT>
__global__ __launch_bounds__(NT) void token_parts_kernel(TokenLossArgs a) {
  const int row = a.row0 + blockIdx.y;
  Row<BF16> r;
  bool weightless;
  const bool token = open_row<BF16, POLICY>(a, row, r, weightless);
  if (!token || (weightless && !(a.loss || a.logp || a.kl || a.entropy))) return;
  part_sums<BF16, ENT, NT>(r, blockIdx.x, a.per_part, a.s, (Sums*)a.parts + (long long)row * a.n_parts + blockIdx.x);
}

// The outputs (by the first part) and a part's gradient.
template <int BF16, bool POLICY, bool ENT, int NT>
__global__ __launch_bounds__(NT) void token_parts_grad_kernel(TokenLossArgs a) {
  constexpr int V = Row<BF16>::V;
  __shared__ RowGrad shared_grad;
  const int row = a.row0 + blockIdx.y, p = blockIdx.x;
  Row<BF16> r;
  bool weightless;
  const bool token = open_row<BF16, POLICY>(a, row, r, weightless);
  const int begin = p * a.per_part, last = min(r.chunks, begin + a.per_part);
  char* const d_row = (char*)a.grad + row * a.ld_grad * (16 / V);
  if (!token || weightless) {
    if (a.grad)
      for (int i = begin + threadIdx.x; i < last; i += NT) r.zero_chunk(d_row, i);
    if (!token) {
      if (p == 0 && threadIdx.x == 0) no_token(a, row);
      return;
    }
    if (p > 0 || !(a.loss || a.logp || a.kl || a.entropy)) return;
  }
  if (threadIdx.x < 64) {
    const Sums sums = join_parts<ENT>((const Sums*)a.parts + (long long)row * a.n_parts, a.n_parts, a.s);
    const RowFacts f = row_facts<ENT>(sums, r.at(r.label), a.inv_t);
    const RowGrad d = finish_row<POLICY, ENT>(a, row, f, sums.top, p == 0 && threadIdx.x == 0);
    if (threadIdx.x == 0) shared_grad = d;
  }
  if (!a.grad || weightless) return;
  __syncthreads();
  const RowGrad d = shared_grad;
  Exponent<BF16> x;
  x.relative_to(d.top, a.s);
  for_chunks<BF16, true, 1, NT>(r, begin, last, [&](float* z, int i) {
    if (i < last) store_gradient<BF16, ENT>(r, d_row, i, z, x, d);
  });
}

// ---------------------------------------------------------------- preference

// A sequence's rows [first, last), inside [0, n] whatever the offsets hold.
__device__ __forceinline__ int offset_at(const PreferenceArgs& a, int i) {
  const long long at = a.offsets ? a.offsets[i] : (long long)a.n / (2 * a.pairs) * i;
  return (int)(at < 0 ? 0 : at > a.n ? a.n : at);
}

// The sums of all rows, NT threads a part of a row in turn, G rows a workgroup (G > 1: up to a wave each).
template <int BF16, int NT, int G>
__global__ __launch_bounds__(NT * G) void preference_sums_kernel(PreferenceArgs a) {
  static_assert(G == 1 || NT <= 64, "rows that share a workgroup have no barrier");
  __shared__ Sums waves[NT > 64 ? NT / 64 : 1];
  const int end = offset_at(a, 2 * a.pairs), tid = threadIdx.x % NT, p = blockIdx.x;
  for (int row = offset_at(a, 0) + blockIdx.y * G + threadIdx.x / NT; row < end; row += gridDim.y * G) {
    const int label = a.labels[row];
    if ((unsigned)label >= (unsigned)a.C) continue;
    Row<BF16> r;
    r.init(a.logits, row * a.ld_row, a.C, label);
    const Sums sums = row_sums<BF16, false, true, NT>(r, p * a.per_part, min(r.chunks, (p + 1) * a.per_part), r.at(label), a.s, waves);
    if (tid == 0) ((Sums*)a.parts)[(long long)row * a.n_parts + p] = sums;
    if (NT > 64) __syncthreads();
  }
}

__device__ __forceinline__ PreferenceRow preference_row(const Sums& sums, const RowFacts& f) {
  return PreferenceRow{sums.top, f.defined ? (float)f.share : NAN, f.defined ? (float)f.rest : NAN, 0.f};
}

// A pair's outputs (where `writes`) and its answers' weights, dL / d log p of a token over T, from NW waves' sums of
// log p - ref and numbers of tokens.
template <int NW>
__device__ __forceinline__ void finish_pair(const PreferenceArgs& a, int p, const double (&sums)[2][NW],
                                            const int (&counts)[2][NW], bool writes, float weight[2]) {
  double score[2], per[2];
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    double total = 0.0;
    int count = 0;
    for (int w = 0; w < NW; ++w) {
      total += sums[k][w];
      count += counts[k][w];
    }
    per[k] = a.mean && count ? 1.0 / count : 1.0;
    score[k] = a.beta * (total * per[k]);
  }
  const double u = score[0] - score[1], smooth = a.smoothing;
  const double e = exp(-fabs(u)), big = 1 / (1 + e), small = e / (1 + e);
  const double up = u > 0 ? big : small, down = u > 0 ? small : big;   // sigmoid(u), sigmoid(-u)
  if (writes) {
    const double soft = log1p(e);
    double loss = (1 - smooth) * (soft + (u < 0 ? -u : 0.0));
    if (smooth > 0) loss += smooth * (soft + (u > 0 ? u : 0.0));
    if (a.loss) a.loss[p] = u == u ? (float)loss : NAN;
    if (a.scores) {
      a.scores[2 * p] = (float)score[0];
      a.scores[2 * p + 1] = (float)score[1];
    }
  }
  const double g = a.grad_loss ? (double)a.grad_loss[p] : 1.0;
  const double du = g == 0 ? 0.0 : u == u ? a.beta * g * (smooth * up - (1 - smooth) * down) : NAN;
#pragma unroll
  for (int k = 0; k < 2; ++k) weight[k] = (float)((k ? -du : du) * per[k] * a.inv_t);
}

// One workgroup per pair: its rows' log p from their sums, its answers' sums in 64 bits (a thread's rows in their order, then
// a tree, the same every time), the loss, and every row's weight.  A chain of a few dependent loads and 64-bit logarithms
// for each 1024 rows: 7 us for 8 pairs of 470 rows, 13 us for 3 of 1760 (11 and 25 in 256 threads).
template <int BF16>
__global__ __launch_bounds__(1024) void preference_pairs_kernel(PreferenceArgs a) {
  constexpr int NW = 16;
  __shared__ double sums[2][NW];
  __shared__ int counts[2][NW];
  const int p = blockIdx.x, tid = threadIdx.x;
  const int begin = offset_at(a, 2 * p), middle = offset_at(a, 2 * p + 1), end = offset_at(a, 2 * p + 2);
  auto token = [&](int row) { return (unsigned)a.labels[row] < (unsigned)a.C; };
  double sum[2] = {0.0, 0.0};
  int tokens[2] = {0, 0};
  for (int row = begin + tid; row < end; row += 1024) {
    const int label = a.labels[row];
    if ((unsigned)label >= (unsigned)a.C) continue;
    const float z = element<BF16>((const char*)a.logits + row * a.ld_row * (BF16 ? 2 : 4), label);
    const Sums* parts = (const Sums*)a.parts + (long long)row * a.n_parts;
    Sums all = parts[0];
    if (a.n_parts > 1) {
#pragma unroll 8
      for (int q = 1; q < a.n_parts; ++q) all.top = fmaxf(all.top, parts[q].top);
      all.sum = 0.0;
#pragma unroll 8
      for (int q = 0; q < a.n_parts; ++q) all.sum += parts[q].sum * grown(step_between(parts[q].top, all.top, a.s.s));
    }
    const RowFacts f = row_facts<false>(all, z, a.inv_t);
    a.rows[row] = preference_row(all, f);
    const double delta = f.logp - (a.ref_logp ? (double)a.ref_logp[row] : 0.0);
    if (row < middle) sum[0] += delta, ++tokens[0];
    else sum[1] += delta, ++tokens[1];
  }
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    sum[k] = wave_add(sum[k]);
    tokens[k] = wave_add(tokens[k]);
    if ((tid & 63) == 0) {
      sums[k][tid >> 6] = sum[k];
      counts[k][tid >> 6] = tokens[k];
    }
  }
  __syncthreads();
  float weight[2];
  finish_pair<NW>(a, p, sums, counts, tid == 0, weight);
  if (!a.grad) return;
  for (int row = begin + tid; row < end; row += 1024)
    a.rows[row].weight = token(row) ? (row < middle ? weight[0] : weight[1]) : 0.f;
}

// Small problems in one launch: a workgroup per pair, a wave a row in turn, whose logits it reads again for the gradient.
template <int BF16>
__global__ __launch_bounds__(1024) void preference_few_kernel(PreferenceArgs a) {
  constexpr int V = Row<BF16>::V, NW = 16;
  __shared__ double sums[2][NW];
  __shared__ int counts[2][NW];
  const int p = blockIdx.x, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int begin = offset_at(a, 2 * p), middle = offset_at(a, 2 * p + 1), end = offset_at(a, 2 * p + 2);
  double sum[2] = {0.0, 0.0};
  int tokens[2] = {0, 0};
  for (int row = begin + wave; row < end; row += NW) {
    Row<BF16> r;
    r.init(a.logits, row * a.ld_row, a.C, a.labels[row]);
    if ((unsigned)r.label >= (unsigned)a.C) continue;
    const float z_label = r.at(r.label);
    const Sums all = row_sums<BF16, false, true, 64>(r, 0, r.chunks, z_label, a.s, nullptr);
    const RowFacts f = row_facts<false>(all, z_label, a.inv_t);
    if (lane == 0) a.rows[row] = preference_row(all, f);
    const double delta = f.logp - (a.ref_logp ? (double)a.ref_logp[row] : 0.0);
    if (row < middle) sum[0] += delta, ++tokens[0];
    else sum[1] += delta, ++tokens[1];
  }
  if (lane < 2) {
    sums[lane][wave] = lane ? sum[1] : sum[0];
    counts[lane][wave] = lane ? tokens[1] : tokens[0];
  }
  __syncthreads();
  float weight[2];
  finish_pair<NW>(a, p, sums, counts, threadIdx.x == 0, weight);
  if (!a.grad) return;
  __threadfence_block();                                     // the wave's own rows' facts
  for (int row = begin + wave; row < end; row += NW) {
    Row<BF16> r;
    r.init(a.logits, row * a.ld_row, a.C, a.labels[row]);
    char* const d_row = (char*)a.grad + row * a.ld_grad * (16 / V);
    const float w = row < middle ? weight[0] : weight[1];
    if ((unsigned)r.label >= (unsigned)a.C || w == 0.f) {
      r.template zero<64>(d_row, lane);
      continue;
    }
    const PreferenceRow f = a.rows[row];
    const RowGrad d{-w * f.share, 0.f, w * f.rest, f.top};
    Exponent<BF16> x;
    x.relative_to(f.top, a.s);
    for_chunks<BF16, true, 1, 64>(r, 0, r.chunks, [&](float* z, int i) {
      if (i < r.chunks) store_gradient<BF16, false>(r, d_row, i, z, x, d);
    });
  }
}

template <int BF16, int NT, int G>
__global__ __launch_bounds__(NT * G) void preference_grad_kernel(PreferenceArgs a) {
  constexpr int V = Row<BF16>::V;
  const int end = offset_at(a, 2 * a.pairs), tid = threadIdx.x % NT;
  for (int row = offset_at(a, 0) + blockIdx.y * G + threadIdx.x / NT; row < end; row += gridDim.y * G) {
    const PreferenceRow f = a.rows[row];
    Row<BF16> r;
    r.init(a.logits, row * a.ld_row, a.C, a.labels[row]);
    char* const d_row = (char*)a.grad + row * a.ld_grad * (16 / V);
    const int begin = blockIdx.x * a.per_part, last = min(r.chunks, begin + a.per_part);
    if (f.weight == 0.f) {
      for (int i = begin + tid; i < last; i += NT) r.zero_chunk(d_row, i);
      continue;
    }
    const RowGrad d{-f.weight * f.share, 0.f, f.weight * f.rest, f.top};
    Exponent<BF16> x;
    x.relative_to(f.top, a.s);
    for_chunks<BF16, true, 1, NT>(r, begin, last, [&](float* z, int i) {
      if (i < last) store_gradient<BF16, false>(r, d_row, i, z, x, d);
    });
  }
}

// Workgroups of a launch's second axis at most.
constexpr int kGridRows = 1 << 15, kUnits = 256;
constexpr long long kFewBytes = 4 << 20;                     // bounds what uneven answers leave to one workgroup

template <int BF16, bool POLICY, bool ENT, int NT, int CH, int G, bool REST, int OCC = 1>
hipError_t launch_loss_rows(const TokenLossArgs& args, hipStream_t s) {
  TokenLossArgs a = args;
  for (long long row = 0; row < args.n; row += (1 << 20) * G) {   // 2^20 workgroups a launch at most
    a.row0 = (int)row;
    const long long rows = std::min<long long>(args.n - row, (1 << 20) * G);
    launch(token_loss_kernel<BF16, POLICY, ENT, NT, CH, G, REST, OCC>, dim3((unsigned)((rows + G - 1) / G)), dim3(NT * G), s, a);
    const hipError_t st = hipGetLastError();
    if (st != hipSuccess) return st;
  }
  return hipSuccess;
}

// Parts of a row of so many chunks, so that n rows give work to the whole GPU; 1: rows stay whole.  In us, whole and in parts:
// 1 x 131072 fp32 27 and 13, 16 x 100000 fp32 21 and 13, 100 x 50000 bf16 13.7 and 12.9 (12 of them the path to two launches).
int parts_of(long long n, int chunks) {
  constexpr int kLeast = 512, kGroups = 512;                 // chunks of a part at least; workgroups to aim at
  return (int)std::max<long long>(1, std::min<long long>(kGroups / std::max<long long>(n, 1), chunks / kLeast));
}

// Chunks of the longest row: one more where bf16 rows may start off 16-byte boundaries.
template <int BF16>
int most_chunks(int C) {
  constexpr int V = Row<BF16>::V;
  return (C + (BF16 == 2 ? 2 * V - 2 : V - 1)) / V;
}
bool on_boundaries(const void* logits, long long ld_row) { return ((uintptr_t)logits & 15) == 0 && ld_row % 8 == 0; }

template <int BF16, bool POLICY, bool ENT>
hipError_t launch_loss_parts(const TokenLossArgs& a, hipStream_t s) {
  constexpr int NT = 256;
  launch(token_parts_kernel<BF16, POLICY, ENT, NT>, dim3(a.n_parts, a.n), dim3(NT), s, a);
  const hipError_t st = hipGetLastError();
  if (st != hipSuccess) return st;
  launch(token_parts_grad_kernel<BF16, POLICY, ENT, NT>, dim3(a.grad ? a.n_parts : 1, a.n), dim3(NT), s, a);
  return hipGetLastError();
}

// Short rows share a wave, up to 256 chunks stay in registers; of longer ones a part does, so that more rows run at once, and
// the rest is read again from a cache.  What bounds all of these is how many bytes are on their way, so registers are given
// to the threads up to 8, 6 or 5 waves a SIMD (OCC); rows of one wave need no barrier and are faster up to
// longer rows with entropy and where there is no gradient.  In us, taken and otherwise (threads a row x chunks held in each), bf16:
//                            with entropy and gradient           without entropy             with entropy, no gradient
//   40000 x 1000, 125 chunks   32 x 4 47.7, 16 x 8 48.1            32 x 4 42.1, 16 x 8 44.4
//   40000 x 3200, 400          64 x 8 124, 128 x 4 143             64 x 8 116, 128 x 4 118
//   4096 x 2600, 325           64 x 8 17.8, 128 x 4 18.4           64 x 8 15.8, 128 x 4 15.6   64 x 8 13.8, 128 x 4 14.2
//   2000 x 5000, 625           128 x 4 15.3, 64 x 8 16.0           128 x 4 13.0, 64 x 8 14.2   128 x 4 11.3, 64 x 8 12.2
//   16000 x 5000, 625          64 x 8 73.2, 128 x 4 79.0           128 x 4 66.9, 64 x 8 70.2   64 x 8 46.1, 128 x 4 53.4
//   40000 x 8000, 1000         64 x 8 255, 128 x 4 271             128 x 4 236, 64 x 8 242     64 x 8 134, 128 x 4 154
//   8000 x 12000, 1500         256 x 4 85.9, 256 x 8 88.2          256 x 4 74.8, 256 x 8 81.5
//   8000 x 20000, 2500         256 x 8 130, 256 x 4 134, 512 x 4 148
//   4096 x 30000, 3750         256 x 8 103.4, 512 x 4 104.9, 256 x 4 108                       256 x 0 50.4, 512 x 0 56.7
//   4096 x 64000, 8000         512 x 6 212.6, 512 x 4 212.6, 512 x 8 in 5 waves a SIMD 237     512 x 0 (50000) 81.2, 256 x 0 78.8
// and fp32: 2000 x 30001, 7501 chunks, 512 x 8 91.3, 512 x 6 94.0; 900 x 30001 512 x 3 49.1 (in 8 waves: four rows a unit at
// once, so all of them), 512 x 8 50.4; 4096 x 30000 without a gradient 512 x 0 86.0, 256 x 0 88.8.
template <int BF16, bool POLICY, bool ENT>
hipError_t launch_loss_by_length(const TokenLossArgs& args, hipStream_t s) {
  TokenLossArgs a = args;
  const int chunks = most_chunks<BF16>(a.C);
  a.n_parts = parts_of(a.n, chunks);
  a.per_part = (chunks + a.n_parts - 1) / a.n_parts;
  if (a.n_parts > 1) return launch_loss_parts<BF16, POLICY, ENT>(a, s);
  if (chunks <= 8 * 4) return launch_loss_rows<BF16, POLICY, ENT, 8, 4, 32, false>(a, s);
  if (chunks <= 16 * 4) return launch_loss_rows<BF16, POLICY, ENT, 16, 4, 16, false>(a, s);
  if (chunks <= 32 * 4) return launch_loss_rows<BF16, POLICY, ENT, 32, 4, 8, false, 8>(a, s);
  if (chunks <= 32 * 8) return launch_loss_rows<BF16, POLICY, ENT, 32, 8, 8, false, ENT ? 5 : 1>(a, s);
  if (chunks <= (ENT || !a.grad ? 64 * 16 : 64 * 7) && a.n >= 16 * kUnits)
    return launch_loss_rows<BF16, POLICY, ENT, 64, 8, 1, true, 6>(a, s);
  if (chunks <= 128 * 8) return launch_loss_rows<BF16, POLICY, ENT, 128, 4, 1, true, 8>(a, s);
  if (!a.grad && chunks <= 256 * 16) return launch_loss_rows<BF16, POLICY, ENT, 256, 0, 1, true, 8>(a, s);
  if (!a.grad) return launch_loss_rows<BF16, POLICY, ENT, 512, 0, 1, true>(a, s);
  if (chunks <= 256 * 8) return launch_loss_rows<BF16, POLICY, ENT, 256, 4, 1, true, 8>(a, s);
  if (chunks <= 256 * 16) return launch_loss_rows<BF16, POLICY, ENT, 256, 8, 1, true, 6>(a, s);
  if (a.n > 3 * kUnits && a.n <= 4 * kUnits) return launch_loss_rows<BF16, POLICY, ENT, 512, 3, 1, true, 8>(a, s);
  return launch_loss_rows<BF16, POLICY, ENT, 512, BF16 ? 6 : 8, 1, true, 6>(a, s);
}

template <int BF16>
hipError_t launch_loss(const TokenLossArgs& a, hipStream_t s) {
  const bool ent = a.entropy || a.grad_entropy || a.entropy_coef != 0.0;
  if (a.policy) return ent ? launch_loss_by_length<BF16, true, true>(a, s) : launch_loss_by_length<BF16, true, false>(a, s);
  return ent ? launch_loss_by_length<BF16, false, true>(a, s) : launch_loss_by_length<BF16, false, false>(a, s);
}

template <int BF16, int NT, int G>
hipError_t launch_preference_sums(const PreferenceArgs& a, hipStream_t s) {
  launch(preference_sums_kernel<BF16, NT, G>, dim3(a.n_parts, std::min((a.n + G - 1) / G, kGridRows)), dim3(NT * G), s, a);
  return hipGetLastError();
}
template <int BF16, int NT, int G>
hipError_t launch_preference_grad(const PreferenceArgs& a, hipStream_t s) {
  launch(preference_grad_kernel<BF16, NT, G>, dim3(a.n_parts, std::min((a.n + G - 1) / G, kGridRows)), dim3(NT * G), s, a);
  return hipGetLastError();
}

template <int BF16>
hipError_t launch_preference_of(const PreferenceArgs& args, hipStream_t s) {
  PreferenceArgs a = args;
  const int chunks = most_chunks<BF16>(a.C);
  a.n_parts = parts_of(a.n, chunks);
  a.per_part = (chunks + a.n_parts - 1) / a.n_parts;
  // One launch for few short rows.  In us, and in three launches: 2 pairs of 2 x 5 rows of 1000 fp32 8.9 and 15.2, 64 of 2 x 4
  // 9.8 and 15.7, 2 of 2 x 16 15.6 and 15.4, 1 of 2 x 32 rows of 500 22 and 15.6.
  const long long turns = (a.n / a.pairs + 15) / 16;         // rows of a wave, as answers go on average
  if (turns * (256 + chunks) <= 1024 && a.n * (chunks * 16LL) <= kFewBytes) {
    launch(preference_few_kernel<BF16>, dim3(a.pairs), dim3(1024), s, a);
    return hipGetLastError();
  }
  // Threads of a row (and rows a workgroup) by its chunks.  Sums and gradient, in us for all three kernels, taken and otherwise:
  // 64 pairs of 2 x 250 rows of 1000 bf16 52, with 256 and 512 threads 128; 32 of 5000 99 and 124, 16 of 10000 92 and 105, 16 of 2 x
  // 100 of 10000 45 and 49; 16 of 8000 fp32 129, with 64 and 256 threads 134; 8 of 30000 bf16 132, with 64 threads for sums
  // 135 and for both 140.
  const bool short_rows = a.n_parts == 1 && chunks <= 1536;
  hipError_t st = !short_rows ? launch_preference_sums<BF16, 256, 1>(a, s)
                  : chunks <= 256 ? launch_preference_sums<BF16, 32, 8>(a, s) : launch_preference_sums<BF16, 64, 1>(a, s);
  if (st != hipSuccess) return st;
  launch(preference_pairs_kernel<BF16>, dim3(a.pairs), dim3(1024), s, a);
  st = hipGetLastError();
  if (st != hipSuccess || !a.grad) return st;
  if (!short_rows) return launch_preference_grad<BF16, 512, 1>(a, s);
  return chunks <= 1024 ? launch_preference_grad<BF16, 64, 4>(a, s) : launch_preference_grad<BF16, 256, 1>(a, s);
}

// Parts of a row at most: of fp32 values, which has more chunks.
int most_parts(int n, int n_classes) { return parts_of(n, (n_classes + 3) / 4); }

}  // namespace

long long token_loss_workspace_bytes(int n, int n_classes) {
  const int parts = most_parts(n, n_classes);
  return parts > 1 ? ((long long)n * parts * (long long)sizeof(Sums) + 15) / 16 * 16 : 0;
}
long long preference_workspace_bytes(int n, int n_classes) {
  return ((long long)n * (long long)sizeof(PreferenceRow) + 15) / 16 * 16 +
         ((long long)n * most_parts(n, n_classes) * (long long)sizeof(Sums) + 15) / 16 * 16;
}

hipError_t launch_token_loss(const TokenLossArgs& a, bool bf16, hipStream_t s) {
  if (!bf16) return launch_loss<0>(a, s);
  return on_boundaries(a.logits, a.ld_row) ? launch_loss<1>(a, s) : launch_loss<2>(a, s);
}

hipError_t launch_preference(const PreferenceArgs& args, bool bf16, hipStream_t s) {
  PreferenceArgs a = args;
  a.parts = (char*)a.rows + ((long long)a.n * (long long)sizeof(PreferenceRow) + 15) / 16 * 16;
  if (!bf16) return launch_preference_of<0>(a, s);
  return on_boundaries(a.logits, a.ld_row) ? launch_preference_of<1>(a, s) : launch_preference_of<2>(a, s);
}

}  // namespace rafiki
