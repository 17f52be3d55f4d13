// Distillation of a teacher's top classes into a student, loss and gradient (rafiki_tokens.h).
//
// With y_c = z_c s, s = log2(e) / T, K the row's teacher classes and r the other classes:
//     S_r = sum_{c not in K} 2^(y_c - y_r),  y_r their maximum,   S the same sum over all classes,
//     p_c = 2^(y_c - y) / S,  p_r = S_r 2^(y_r - y) / S,
//     dz_c = T g (Q p_c - q_c) in K,  T g (Q p_r - q_r) 2^(y_c - y_r) / S_r otherwise,
// one power and one product per class outside K; K's classes are written after the others.  K's classes
// are marked in a bitmap in LDS and left out of r's sum, which keeps p_r exact where it is small
// (1 - sum p_j does not).  Without rest nothing is marked, r is all classes and q_r = 0.
//
// One workgroup per row, the row in its registers: the logits are read once and the gradient written
// once, which is the floor.  Chunks of 16 bytes lie on 16-byte boundaries of the logits, so a row may
// start anywhere.  Rows too long for the registers are read again for each pass (CH = 0), from the L2
// or the memory-side cache.
//
// Measured on an MI355X: 4096 x 30000 bf16 127 us (3.9 TB/s of the floor's bytes; a device copy moves 4.7), 2047 x
// 131071 bf16 294 us (3.6 TB/s): one such row fills a compute unit's registers, so its arithmetic (two powers a
// class, 15 us) overlaps only with its own loads and stores and those of other units.
#include "tokens.h"

#include <algorithm>

namespace rafiki {

namespace {

constexpr float kRestMin = 0x1p-20f;
constexpr float kLn2 = 0.693147180559945f, kLog2e = 1.44269504088896f;

typedef unsigned long long u64;
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4_any __attribute__((ext_vector_type(4), aligned(2)));

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

// A 16-byte chunk of V values: unpacked, packed.
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
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
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
__device__ __forceinline__ float wave_add(float v) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o, 64);
  return v;
}

// A barrier for what goes through LDS alone: __syncthreads() would also wait for every load from memory.
__device__ __forceinline__ void lds_barrier() {
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_waitcnt(0xC07F);                        // lgkmcnt(0)
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
}

// The maximum as a reference for powers: an empty row has none and takes 0.
__device__ __forceinline__ float reference(float top) { return top == -INFINITY ? 0.f : top; }

// NT threads hold a row of up to NT CH + 2 chunks, the two edges among them (CH = 0: any length, not held).
// WIDE: the logits are halved as they are read, and T with them, since two finite ones may lie further apart than fp32
// holds.  It is for T above 2^120: below, such a difference is more than 2^8 T, whose power is 0 in fp32 as that of
// -inf is.  (Halves in the differences of every row instead: 300 us for 2047 x 131071, against 292 without
// either.)
template <bool BF16, bool REST, int NT, int CH, int OCC, bool WIDE>
__global__ __launch_bounds__(NT, OCC) void distill_kernel(DistillArgs a) {
  constexpr int V = BF16 ? 8 : 4, NW = NT / 64;
  extern __shared__ uint32_t marks[];                        // rest: bit c + shift is set for c in K
  __shared__ float w_top[NW], w_member_top[NW], w_members[NW], w_q[NW], w_sum[NW], w_member_sum[NW], w_part[NW];
  __shared__ int ids[kMaxTokenK];
  __shared__ float slot_q[kMaxTokenK];                       // teacher_logp, then q of the slot
  constexpr uint32_t kMasked = BF16 ? 0xFF80FF80u : 0xFF800000u;     // -inf in every place
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  // Powers are of (z - top) s, not of z s - top s: masks of the type's lowest value overflow the products,
  // and a row of nothing else is a uniform one.  T below log2(e) 2^-127 (no normal T is) counts as that, which
  // keeps 0 s at 0.
  const float s = fminf(kLog2e / (WIDE ? 0.5f * a.t : a.t), 0x1p127f);
  const int row = a.row0 + blockIdx.x;
  const float g = a.grad_loss ? a.grad_loss[row] : 1.f;
  const long long base = row * a.ld_row, gbase = row * a.ld_grad;
  const int shift = (int)((((uintptr_t)a.logits / (16 / V)) + base) & (V - 1));   // classes behind a boundary
  const int chunks = (a.C + shift + V - 1) / V;
  // Chunk c: classes c V - shift .. + V - 1, on a 16-byte boundary.  The first and the last may stand out of
  // the row: thread 0 and thread 1 hold, beside the others, the row's first and last V classes instead (the
  // edges), of which those that another chunk has too count there.  Gradients are the same from both.
  const char* const x_row = (const char*)a.logits + (base - shift) * (16 / V);
  char* const d_row = (char*)a.grad + (gbase - shift) * (16 / V);
  const int edge_at = tid == 0 ? 0 : a.C - V;              // its first class, where C >= V
  const bool has_edge = tid == 0 || (tid == 1 && chunks > 1);
  // the edge's classes that count: a bit each (a row shorter than a chunk is thread 0's)
  const uint32_t edge_own = a.C < V ? (tid == 0 ? (1u << a.C) - 1 : 0u)
                            : tid == 0 ? (1u << (V - shift)) - 1
                                       : ~0u << (chunks * V - shift - a.C) & ((1u << V) - 1);
  auto halved = [&](u32x4 q) {
    if constexpr (WIDE) {
      float z[V];
      unpack<BF16, V>(q, z);
#pragma unroll
      for (int j = 0; j < V; ++j) z[j] *= 0.5f;
      q = pack<BF16, V>(z);
    }
    return q;
  };
  auto load = [&](int i) {
    return halved(__builtin_nontemporal_load((const u32x4*)(x_row + (long long)i * NT * 16 + (unsigned)(tid + 1) * 16u)));
  };
  auto store = [&](int i, const float d[V]) {
    __builtin_nontemporal_store(pack<BF16, V>(d), (u32x4_any*)(d_row + (long long)i * NT * 16 + (unsigned)(tid + 1) * 16u));
  };
  auto load_edge = [&]() {
    u32x4 q = {kMasked, kMasked, kMasked, kMasked};
    if (has_edge) {
      if (a.C >= V) {
        q = *(const u32x4_any*)(x_row + (shift + edge_at) * (16 / V));
      } else {
        float z[V];
#pragma unroll
        for (int j = 0; j < V; ++j) z[j] = tid == 0 && j < a.C ? element<BF16>(a.logits, base + j) : -INFINITY;
        q = pack<BF16, V>(z);
      }
    }
    return halved(q);
  };
  auto store_edge = [&](const float d[V]) {
    if (has_edge && a.C >= V) {
      *(u32x4_any*)(d_row + (shift + edge_at) * (16 / V)) = pack<BF16, V>(d);
    } else if (tid == 0) {
#pragma unroll
      for (int j = 0; j < V; ++j)
        if (j < a.C) put<BF16>(a.grad, gbase + j, d[j]);
    }
  };
  auto zero_row = [&]() {
    float d[V];
#pragma unroll
    for (int j = 0; j < V; ++j) d[j] = 0.f;
    for (int i = 0; i * NT + tid + 1 < chunks - 1; ++i) store(i, d);
    store_edge(d);
  };
  if (g == 0.f && !a.loss) {                               // of no weight: the row is not read
    if (a.grad) zero_row();
    return;
  }
  u32x4 held[CH > 0 ? CH : 1], edge = load_edge();
  if constexpr (CH > 0) {
#pragma unroll
    for (int i = 0; i < CH; ++i) {
      held[i] = u32x4{kMasked, kMasked, kMasked, kMasked};
      if (i * NT + tid + 1 < chunks - 1) held[i] = load(i);
    }
  }
  // K's classes as -inf in the V classes whose first has bit `at` of the marks
  auto without_members = [&](u32x4 q, int at) {
    const u64 two = (u64)marks[(at >> 5) + 1] << 32 | marks[at >> 5];
    const uint32_t m = (uint32_t)(two >> (at & 31)) & ((1u << V) - 1);
    if (m) {
      float z[V];
      unpack<BF16, V>(q, z);
#pragma unroll
      for (int j = 0; j < V; ++j) z[j] = m >> j & 1 ? -INFINITY : z[j];
      q = pack<BF16, V>(z);
    }
    return q;
  };
  // f(a chunk's logits, the bits that count) for every chunk of this thread; store_chunk(d) puts its gradient
  auto for_chunks = [&](auto&& f) {
    float z[V];
    constexpr uint32_t kAll = (1u << V) - 1;
    if constexpr (CH > 0) {
#pragma unroll
      for (int i = 0; i < CH; ++i) {
        // opaque here, or the compiler keeps every pass's unpacked values for the next one
        asm volatile("" : "+v"(held[i][0]), "+v"(held[i][1]), "+v"(held[i][2]), "+v"(held[i][3]));
        unpack<BF16, V>(held[i], z);
        f(z, kAll, [&](const float* d) { if (i * NT + tid + 1 < chunks - 1) store(i, d); });
        __builtin_amdgcn_sched_barrier(0);                 // one chunk's values at a time in registers
      }
    } else {
      for (int i = 0; i * NT + tid + 1 < chunks - 1; ++i) {
        unpack<BF16, V>(REST ? without_members(load(i), (i * NT + tid + 1) * V) : load(i), z);
        f(z, kAll, [&](const float* d) { store(i, d); });
      }
    }
    if (has_edge) {
      unpack<BF16, V>(edge, z);
      f(z, edge_own, store_edge);
    }
  };

  // ---- the teacher's slots
  for (int j = tid; j < a.k; j += NT) {
    const int id = a.labels[(long long)row * a.k + j];
    const bool valid = (unsigned)id < (unsigned)a.C;
    ids[j] = valid ? id : -1;
    slot_q[j] = valid ? a.logp[(long long)row * a.k + j] : -INFINITY;
  }
  if (REST)
    for (int w = tid; w < (chunks * V + 31) / 32 + 1; w += NT) marks[w] = 0;
  lds_barrier();
  float t_top = 0.f, t_sum = 1.f;                          // rest = 0: q = 2^(..) / sum, in every wave
  if (!REST) {
    t_top = -INFINITY;
    for (int j = lane; j < a.k; j += 64) t_top = fmaxf(t_top, slot_q[j]);
    t_top = reference(wave_max(t_top));
    t_sum = 0.f;
    for (int j = lane; j < a.k; j += 64) t_sum += expf(slot_q[j] - t_top);   // NaN stays NaN
    t_sum = wave_add(t_sum);
    if (t_sum == 0.f) {                                    // no teacher: nothing to learn
      if (a.loss && tid == 0) a.loss[row] = 0.f;
      if (a.grad) zero_row();
      return;
    }
  }
  lds_barrier();
  for (int j = tid; j < a.k; j += NT) {
    const int id = ids[j];
    slot_q[j] = expf(slot_q[j] - t_top) / t_sum;
    if (REST && id >= 0) atomicOr(&marks[(id + shift) >> 5], 1u << ((id + shift) & 31));
  }
  lds_barrier();
  if (REST) {
    if constexpr (CH > 0) {
#pragma unroll
      for (int i = 0; i < CH; ++i)
        if (i * NT + tid + 1 < chunks - 1) held[i] = without_members(held[i], (i * NT + tid + 1) * V);
    }
    if (has_edge) edge = without_members(edge, a.C >= V ? shift + edge_at : shift);
  }
  // of the slots of one class the first holds the class: its logit, and the sum of their q
  constexpr int SLOTS = kMaxTokenK / NT;
  float z_class[SLOTS], q_class[SLOTS];
  float member_top = -INFINITY, members = 0.f, q_sum = 0.f;
#pragma unroll
  for (int i = 0; i < SLOTS; ++i) {
    const int j = tid + i * NT;
    z_class[i] = -INFINITY;
    q_class[i] = -1.f;                                     // no class
    const int id = j < a.k ? ids[j] : -1;
    if (id >= 0) {
      float q = 0.f;
      bool first = true;
#pragma unroll 1
      for (int o = 0; o < a.k; ++o)
        if (ids[o] == id) {
          first &= o >= j;
          q += slot_q[o];
        }
      if (first) {
        z_class[i] = element<BF16>(a.logits, base + id) * (WIDE ? 0.5f : 1.f);
        q_class[i] = q;
        member_top = fmaxf(member_top, z_class[i]);
        members += 1.f;
        q_sum += q;
      }
    }
  }

  // ---- maxima and sums of powers, in one pass: a thread's sum follows its maximum, so that it grows while the row
  // is still arriving (with a pass for the maximum first, loading, computing and storing took turns on all
  // compute units at once, 339 us for 2047 x 131071)
  float top = -INFINITY, sum = 0.f;
  for_chunks([&](const float* z, uint32_t own, auto&&) {
    float now = top;
#pragma unroll
    for (int j = 0; j < V; ++j) now = fmaxf(now, z[j]);
    const float ref = reference(now);
    sum *= power2((top - ref) * s);
#pragma unroll
    for (int j = 0; j < V; ++j) sum += own >> j & 1 ? power2((z[j] - ref) * s) : 0.f;
    top = now;
  });
  // the wave's, then the workgroup's
  auto join = [&](float& t, float& v) {
    const float all = wave_max(t);
    v = wave_add(v * power2((t - reference(all)) * s));
    t = all;
  };
  join(top, sum);
  float member_sum = 0.f;
#pragma unroll
  for (int i = 0; i < SLOTS; ++i)
    if (q_class[i] >= 0.f || q_class[i] != q_class[i]) member_sum += power2((z_class[i] - reference(member_top)) * s);
  join(member_top, member_sum);
  members = wave_add(members);
  q_sum = wave_add(q_sum);
  if (lane == 0) {
    w_top[wave] = top;
    w_sum[wave] = sum;
    w_member_top[wave] = member_top;
    w_member_sum[wave] = member_sum;
    w_members[wave] = members;
    w_q[wave] = q_sum;
  }
  lds_barrier();
  top = member_top = -INFINITY;
  members = q_sum = 0.f;
#pragma unroll
  for (int w = 0; w < NW; ++w) {
    top = fmaxf(top, w_top[w]);
    member_top = fmaxf(member_top, w_member_top[w]);
    members += w_members[w];
    q_sum += w_q[w];
  }
  const float top_r = reference(top), top_all = REST ? reference(fmaxf(top, member_top)) : top_r;
  sum = member_sum = 0.f;
#pragma unroll
  for (int w = 0; w < NW; ++w) {
    sum += w_sum[w] * power2((w_top[w] - top_r) * s);
    member_sum += w_member_sum[w] * power2((w_member_top[w] - top_all) * s);
  }
  // r's share of the sum over all; none where nothing is above -inf outside K (top_r is then no maximum, and its power
  // may be infinite).  A NaN sum stays NaN.
  const float part_r = sum == 0.f ? 0.f : sum * power2((top_r - top_all) * s);
  const float sum_all = REST ? part_r + member_sum : sum;
  const bool defined = sum_all > 0.f && sum_all < INFINITY && top_all < INFINITY && member_top < INFINITY;
  float q_r = 0.f;
  if (REST) {
    q_r = 1.f - q_sum;
    if (q_r < kRestMin || members == (float)a.C) q_r = 0.f;
  }
  const float big_q = q_sum + (sum == 0.f ? 0.f : q_r);       // where p_r = 0, q_r has a part in the loss alone
  const float log_all = log2f(sum_all);

  // ---- loss: a wave's part of the sum over K.  A logarithm stays finite as long as fp32 holds it.
  auto log2_ratio = [&](float z, float top) { return (0.5f * z - 0.5f * top) * s * 2.f; };
  if (a.loss) {
    float part = 0.f;
#pragma unroll
    for (int i = 0; i < SLOTS; ++i) {
      const float q = q_class[i];
      if (q > 0.f || q != q) part += q * (logf(q) - kLn2 * (log2_ratio(z_class[i], top_all) - log_all));
    }
    part = wave_add(part);
    if (lane == 0) w_part[wave] = part;
  }
  // ---- gradient outside K
  const float scale = defined ? a.t * g : NAN;
  if (a.grad) {
    if (g == 0.f) {
      zero_row();
    } else {
      const float p_r = REST ? part_r / sum_all : 1.f;
      const bool nan = !defined || big_q != big_q;           // of the student, of the teacher
      const float factor = sum == 0.f ? (nan ? NAN : 0.f) : scale * (big_q * p_r - q_r) / sum;
      for_chunks([&](const float* z, uint32_t, auto&& store_chunk) {
        float d[V];
#pragma unroll
        for (int j = 0; j < V; ++j) d[j] = factor * power2((z[j] - top_r) * s);
        store_chunk(d);
      });
      __builtin_amdgcn_s_waitcnt(0x0F70);                  // vmcnt(0): K's classes are written after these
    }
  }
  lds_barrier();
  if (a.loss && tid == 0) {
    float part = 0.f;
#pragma unroll
    for (int w = 0; w < NW; ++w) part += w_part[w];
    if (q_r > 0.f) part += sum == 0.f ? INFINITY : q_r * (logf(q_r) - kLn2 * (log2f(sum) + log2_ratio(top_r, top_all) - log_all));
    a.loss[row] = defined ? a.t * (a.t * part) : NAN;      // T^2 alone may be beyond fp32 where its product is not
  }
  if (a.grad && g != 0.f) {
#pragma unroll
    for (int i = 0; i < SLOTS; ++i) {
      const float q = q_class[i];
      if (q >= 0.f || q != q)
        put<BF16>(a.grad, gbase + ids[tid + i * NT], scale * (big_q * (power2((z_class[i] - top_all) * s) / sum_all) - q));
    }
  }
}

template <bool BF16, bool REST, int NT, int CH, int OCC, bool WIDE = false>
hipError_t launch_rows(const DistillArgs& a, hipStream_t s) {
  const size_t lds = REST ? ((size_t)a.C + 16 + 31) / 32 * 4 + 4 : 0;   // and a word behind
  DistillArgs part = a;
  for (long long row = 0; row < a.n; row += 1 << 20) {       // 2^20 rows a launch at most
    part.row0 = (int)row;
    const int rows = (int)std::min<long long>(a.n - row, 1 << 20);
    launch_lds(distill_kernel<BF16, REST, NT, CH, OCC, WIDE>, dim3(rows), dim3(NT), lds, s, part);
    const hipError_t st = hipGetLastError();
    if (st != hipSuccess) return st;
  }
  return hipSuccess;
}

template <bool BF16, bool REST>
hipError_t launch_by_length(const DistillArgs& a, hipStream_t s) {
  constexpr int V = BF16 ? 8 : 4;
  const int held = a.C + V - 1 - 2 * V;                      // classes between the edges, with the longest shift
  if (a.t > 0x1p120f) return launch_rows<BF16, REST, 1024, 0, 4, true>(a, s);
  // Few threads with many chunks each: more rows share a compute unit, and one's loads run beside another's
  // arithmetic (30000 bf16 classes: 151 us in 512 threads of 8 chunks, 129 us in 256 of 16).
  if (held <= 128 * 2 * V) return launch_rows<BF16, REST, 128, 2, 4>(a, s);
  if (held <= 128 * 8 * V) return launch_rows<BF16, REST, 128, 8, 4>(a, s);
  if (held <= 256 * 8 * V) return launch_rows<BF16, REST, 256, 8, 4>(a, s);
  if (held <= 256 * 16 * V) return launch_rows<BF16, REST, 256, 16, 4>(a, s);
  if (held <= 512 * 16 * V) return launch_rows<BF16, REST, 512, 16, 4>(a, s);
  if (held <= 1024 * 16 * V) return launch_rows<BF16, REST, 1024, 16, 4>(a, s);
  if (held <= 1024 * 20 * V) return launch_rows<BF16, REST, 1024, 20, 4>(a, s);
  return launch_rows<BF16, REST, 1024, 0, 4>(a, s);
}

}  // namespace

hipError_t launch_distill(const DistillArgs& a, bool bf16, hipStream_t s) {
  if (bf16) return a.rest ? launch_by_length<true, true>(a, s) : launch_by_length<true, false>(a, s);
  return a.rest ? launch_by_length<false, true>(a, s) : launch_by_length<false, false>(a, s);
}

}  // namespace rafiki
