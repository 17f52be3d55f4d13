// FC layer in 8-bit integers on the matrix cores, and the quantisation of its rows
// (rafiki_tokens.h).
#include "tokens.h"

#include <algorithm>

namespace rafiki {

namespace {

typedef int i32x4 __attribute__((ext_vector_type(4)));

template <bool BF16>
__device__ __forceinline__ float value(const void* p, long long i) {
  if constexpr (BF16) return __uint_as_float((uint32_t)((const bf16_t*)p)[i] << 16);
  else return ((const float*)p)[i];
}

// x / s rounded to the nearest integer, ties to even, exactly: the candidate may be one off or
// on the wrong side of a tie; its residual r = x - q s is exact in one FMA (q has 7 bits, and
// |r| <= s leaves no more than 24), so comparing it with s / 2 decides.
__device__ __forceinline__ int nearest_quotient(float x, float s, float inv) {
  float q = __builtin_rintf(x * inv);
  const float r = __builtin_fmaf(-q, s, x), h = 0.5f * s;
  const bool odd = ((int)q & 1) != 0;
  if (r > h || (r == h && odd)) q += 1.f;
  else if (r < -h || (r == -h && odd)) q -= 1.f;
  return (int)q;
}

typedef uint32_t u32x4_any __attribute__((ext_vector_type(4), aligned(2)));
typedef uint32_t u32x2_byte __attribute__((ext_vector_type(2), aligned(1)));
typedef uint32_t u32_byte __attribute__((aligned(1)));

// One workgroup per row, which its NT threads hold in CH chunks of 16 bytes each (CH = 0: any length, read
// twice): the largest magnitude, then the quotients.  The bound is the row's bytes, and with few rows
// their latency: 64 rows of 25088 fp32 take 7 us (50 us in 256 threads that read single values), 4096 of
// 4096 bf16 16 us.
template <bool BF16, int NT, int CH>
__global__ __launch_bounds__(NT) void quantize_kernel(const void* x, long long ld_x, int row0, int c, int8_t* q,
                                                      long long ld_q, float* scale) {
  constexpr int V = BF16 ? 8 : 4, NW = NT / 64, HELD = CH > 0 ? CH : 1;
  __shared__ float waves[NW];
  const int row = row0 + blockIdx.x, tid = threadIdx.x;
  const long long base = row * ld_x;
  const int chunks = c / V;                                 // whole ones; then c % V values
  auto load = [&](int i, float z[V]) {
    const u32x4_any w = *(const u32x4_any*)((const char*)x + (base + (long long)i * V) * (16 / V));
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      if constexpr (BF16) {
        z[2 * j] = __uint_as_float(w[j] << 16);
        z[2 * j + 1] = __uint_as_float(w[j] & 0xFFFF0000u);
      } else {
        z[j] = __uint_as_float(w[j]);
      }
    }
  };
  float held[HELD][V];
  float top = 0.f;
  bool bad = false;
#pragma unroll
  for (int i = 0; i < (CH > 0 ? CH : 1); ++i)
#pragma unroll
    for (int j = 0; j < V; ++j) held[i][j] = 0.f;
  if constexpr (CH > 0) {
#pragma unroll
    for (int i = 0; i < CH; ++i)
      if (i * NT + tid < chunks) load(i * NT + tid, held[i]);
#pragma unroll
    for (int i = 0; i < CH; ++i)
#pragma unroll
      for (int j = 0; j < V; ++j) {
        bad |= !(fabsf(held[i][j]) < INFINITY);
        top = fmaxf(top, fabsf(held[i][j]));
      }
  } else {
    for (int i = tid; i < chunks; i += NT) {
      load(i, held[0]);
#pragma unroll
      for (int j = 0; j < V; ++j) {
        bad |= !(fabsf(held[0][j]) < INFINITY);
        top = fmaxf(top, fabsf(held[0][j]));
      }
    }
  }
  const int last = chunks * V + tid;                         // this thread's value of the last c % V
  const float tail = last < c ? value<BF16>(x, base + last) : 0.f;
  bad |= !(fabsf(tail) < INFINITY);
  top = bad ? INFINITY : fmaxf(top, fabsf(tail));
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor(top, o, 64));
  if ((tid & 63) == 0) waves[tid >> 6] = top;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < NW; ++w) top = fmaxf(top, waves[w]);
  float s = top / 127.f;
  if (s < 0x1p-126f) s = 0.f;
  const bool zero = s == 0.f || top == INFINITY;
  const float inv = zero ? 0.f : 1.f / s;
  int8_t* out = q + row * ld_q;
  auto put = [&](int i, const float z[V]) {
    uint32_t w[V / 4];
#pragma unroll
    for (int j = 0; j < V / 4; ++j) {
      w[j] = 0;
#pragma unroll
      for (int b = 0; b < 4; ++b) w[j] |= (uint32_t)((zero ? 0 : nearest_quotient(z[4 * j + b], s, inv)) & 255) << (8 * b);
    }
    if constexpr (BF16) *(u32x2_byte*)(out + (long long)i * V) = u32x2_byte{w[0], w[V / 4 - 1]};
    else *(u32_byte*)(out + (long long)i * V) = w[0];
  };
  if constexpr (CH > 0) {
#pragma unroll
    for (int i = 0; i < CH; ++i)
      if (i * NT + tid < chunks) put(i * NT + tid, held[i]);
  } else {
    for (int i = tid; i < chunks; i += NT) {
      load(i, held[0]);
      put(i, held[0]);
    }
  }
  if (last < c) out[last] = zero ? 0 : (int8_t)nearest_quotient(tail, s, inv);
  if (tid == 0) scale[row] = top == INFINITY ? NAN : s;
}

typedef int i32x16 __attribute__((ext_vector_type(16)));
typedef __attribute__((address_space(3))) void lds_void;

// s_waitcnt with only the vector-memory counter constrained (gfx9 encoding).
template <int N>
__device__ __forceinline__ void wait_vmcnt() {
  static_assert(N >= 0 && N < 64, "vmcnt range");
  __builtin_amdgcn_s_waitcnt((N & 0xF) | ((N >> 4) << 14) | (0x7 << 4) | (0xF << 8));
}
// Waits until at most `ahead` tiles of PER loads each are in flight.
template <int PER, int MAX>
__device__ __forceinline__ void wait_tiles(int ahead) {
  if constexpr (MAX > 0) {
    if (ahead >= MAX) {
      wait_vmcnt<PER * MAX>();
      return;
    }
    wait_tiles<PER, MAX - 1>(ahead);
  } else {
    wait_vmcnt<0>();
  }
}

// Row r of an LDS tile (128 bytes, 8 chunks of 16) keeps chunk c in slot c ^ swz(r): 16 rows' equal
// chunks then lie on 64 different banks.
__device__ __forceinline__ int swz(int r) { return (r & 7) ^ ((r >> 3) & 1); }

typedef float f32x4_any __attribute__((ext_vector_type(4), aligned(4)));
typedef int i32x4_any __attribute__((ext_vector_type(4), aligned(4)));
typedef __bf16 bf16x8_any __attribute__((ext_vector_type(8), aligned(2)));

__device__ __forceinline__ float finish(int acc, float scale, float bias, int relu) {
  float v = (float)acc * scale + bias;
  return relu && v < 0.f ? 0.f : v;                          // NaN stays NaN
}

// One wave's loads of a K tile: instruction j of wave w fills rows (j NW + w) 8 .. + 7, lane l slot l % 8 of
// row l / 8 of those.  Rows and 16-byte chunks past the operands get an offset past the buffer's end,
// for which the hardware writes zeros.
template <int BM, int BN, int NW>
struct TileLoader {
  static constexpr int RA = BM / (8 * NW), RB = BN / (8 * NW), PER = RA + RB;
  static constexpr unsigned kOut = 0x60000000u;              // past every tile (at most 2^30 bytes and a row)
  static_assert(RA >= 1 && RB >= 1 && NW % 2 == 0, "tile shape");
  __amdgpu_buffer_rsrc_t xr, wr;
  unsigned xo[RA], wo[RB];
  int chunk, wave, kt_begin, k16;

  __device__ __forceinline__ void init(const FcI8Args& a, int m0, int n0, int wave_, int lane, int kt_begin_, int k16_) {
    wave = wave_;
    kt_begin = kt_begin_;
    k16 = k16_;
    const int lrow = lane >> 3;
    chunk = (lane & 7) ^ lrow ^ (wave & 1);
    const int x_rows = min(BM, a.n - m0), w_rows = min(BN, a.c_out - n0);
    xr = __builtin_amdgcn_make_buffer_rsrc((void*)(a.x + m0 * a.ld_x), (short)0, (int)((x_rows - 1) * a.ld_x) + k16,
                                           0x00020000);
    wr = __builtin_amdgcn_make_buffer_rsrc((void*)(a.w + n0 * a.ld_w), (short)0, (int)((w_rows - 1) * a.ld_w) + k16,
                                           0x00020000);
#pragma unroll
    for (int j = 0; j < RA; ++j) {
      const int r = (j * NW + wave) * 8 + lrow;
      xo[j] = r < x_rows ? (unsigned)(r * a.ld_x) + chunk * 16 : kOut;
    }
#pragma unroll
    for (int j = 0; j < RB; ++j) {
      const int r = (j * NW + wave) * 8 + lrow;
      wo[j] = r < w_rows ? (unsigned)(r * a.ld_w) + chunk * 16 : kOut;
    }
  }

  // K tile t of this split into `base` (x's rows, then w's).
  __device__ __forceinline__ void issue(int t, uint4* base) const {
    const int k0 = (kt_begin + t) * 128;
    const bool inside = k0 + chunk * 16 < k16;
#pragma unroll
    for (int j = 0; j < RA; ++j)
      __builtin_amdgcn_raw_ptr_buffer_load_lds(xr, (lds_void*)(base + (j * NW + wave) * 64), 16, inside ? xo[j] : kOut,
                                               k0, 0, 0);
#pragma unroll
    for (int j = 0; j < RB; ++j)
      __builtin_amdgcn_raw_ptr_buffer_load_lds(wr, (lds_void*)(base + BM * 8 + (j * NW + wave) * 64), 16,
                                               inside ? wo[j] : kOut, k0, 0, 0);
  }
};

// Tiled product: BM rows of x by BN rows of w per workgroup of WM x WN waves, K in tiles of 128 bytes
// that go from memory to an LDS ring of STAGES tiles without registers (buffer loads ... lds);
// v_mfma_i32_32x32x32_i8 with w as the first operand, so that a lane sums 4 neighbouring outputs of
// one row.  Splits (grid y) each sum a range of K tiles; with more than one the
// int32 sums go to the workspace and fc_i8_reduce_kernel joins them.
//
// Measured on an MI355X: 4096 x 4096 x 30000 515 to 610 us by the values (1.65 to 1.95 POP/s; the library's int8 product,
// without scales and bias, 530 us on random values).  The matrix cores are busy for 47 % of the cycles at the
// 1.95 GHz that this load leaves them; without the products the loads, fragment reads and stores alone take
// 443 us, without the loads the rest takes 500 us, without the stores 536 us: LDS, which takes both operands'
// tiles and gives each wave 192 rows for 128 x 64 outputs, is shared by all of them.  Deeper rings of 64-byte K tiles,
// 4 waves of 128 x 128 and two workgroups of 128 x 256 a unit were 5 to 20 % slower.
template <int BM, int BN, int WM, int WN, int STAGES, int OCC>
__global__ __launch_bounds__(WM * WN * 64, OCC) void fc_i8_tile_kernel(FcI8Args a) {
  constexpr int NW = WM * WN;
  constexpr int WTM = BM / WM, WTN = BN / WN, TM = WTM / 32, TN = WTN / 32;
  constexpr int PER = TileLoader<BM, BN, NW>::PER;
  constexpr int STAGE = (BM + BN) * 8;                       // 16-byte chunks
  static_assert(TM >= 1 && TN >= 1, "tile shape");
  static_assert(STAGES >= 2 && STAGE * 16 * STAGES <= 160 * 1024, "LDS budget");
  constexpr int CW = TN >= 2 ? 64 : 32;                      // outputs of a row staged at once
  static_assert(NW * 32 * CW * 4 <= STAGE * 16 * STAGES, "epilogue staging fits in LDS");
  __shared__ uint4 lds[STAGE * STAGES];

  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wm = wave % WM, wn = wave / WM;
  // Workgroups are dealt round-robin to the 8 XCDs: each XCD takes a contiguous range of tiles, walked in
  // bands of `band` row tiles, rows fastest, so that the tiles running together on one XCD share
  // rows of x and of w in its L2.
  const int G = gridDim.x, q = G >> 3, r8 = G & 7, xcd = blockIdx.x & 7, loc = blockIdx.x >> 3;
  const int tile = (xcd < r8 ? xcd * (q + 1) : r8 * (q + 1) + (xcd - r8) * q) + loc;
  const int tiles_m = (a.n + BM - 1) / BM, tiles_n = (a.c_out + BN - 1) / BN;
  constexpr int kBand = 8;
  const int band = tile / (kBand * tiles_n), in_band = tile - band * kBand * tiles_n;
  const int rows = min(kBand, tiles_m - band * kBand);
  const int m0 = (band * kBand + in_band % rows) * BM, n0 = in_band / rows * BN;

  const int k16 = (a.c_in + 15) / 16 * 16, ktiles = (k16 + 127) / 128;
  const int kt_begin = blockIdx.y * a.kt_per_split;
  const int nk = min(a.kt_per_split, ktiles - kt_begin);

  TileLoader<BM, BN, NW> loader;
  loader.init(a, m0, n0, wave, lane, kt_begin, k16);
  auto issue = [&](int t, int stage) { loader.issue(t, lds + stage * STAGE); };

  i32x16 acc[TN][TM];
#pragma unroll
  for (int i = 0; i < TN; ++i)
#pragma unroll
    for (int j = 0; j < TM; ++j)
#pragma unroll
      for (int e = 0; e < 16; ++e) acc[i][j][e] = 0;

  const int frow = lane & 31, fk = lane >> 5;
  auto frag = [&](const uint4* base, int r, int c) { return __builtin_bit_cast(i32x4, base[r * 8 + (c ^ swz(r))]); };
  // Bytes of x behind c_in in the last K tile's last chunk become 0 (a barrier for all waves).
  const int tail = a.c_in & 15;
  auto clear_tail = [&](int t, uint4* tile_x) {
    if (tail == 0 || kt_begin + t != ktiles - 1) return;
    const int c = (a.c_in & 127) >> 4;
    for (int r = threadIdx.x; r < BM; r += NW * 64) {
      uint4& v = tile_x[r * 8 + (c ^ swz(r))];
      uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int left = tail - 4 * i;
        w[i] = left <= 0 ? 0u : left < 4 ? w[i] & ((1u << (8 * left)) - 1u) : w[i];
      }
      v = make_uint4(w[0], w[1], w[2], w[3]);
    }
    __syncthreads();
  };

  i32x4 xf[2][TM], wf[2][TN];
  if (nk > 0) {
#pragma unroll
    for (int s = 0; s < STAGES; ++s)
      if (s < nk) issue(s, s);
    wait_tiles<PER, STAGES - 1>(min(STAGES, nk) - 1);
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
    clear_tail(0, lds);
#pragma unroll
    for (int tm = 0; tm < TM; ++tm) xf[0][tm] = frag(lds, wm * WTM + tm * 32 + frow, fk);
#pragma unroll
    for (int tn = 0; tn < TN; ++tn) wf[0][tn] = frag(lds + BM * 8, wn * WTN + tn * 32 + frow, fk);
  }
  for (int kt = 0; kt < nk; ++kt) {
    const int cur = kt % STAGES;
    const uint4* As = lds + cur * STAGE;
    const uint4* Bs = As + BM * 8;
#pragma unroll
    for (int s = 0; s < 4; ++s) {
      const int b = s & 1;
      if (s < 3) {
#pragma unroll
        for (int tm = 0; tm < TM; ++tm) xf[b ^ 1][tm] = frag(As, wm * WTM + tm * 32 + frow, 2 * (s + 1) + fk);
#pragma unroll
        for (int tn = 0; tn < TN; ++tn) wf[b ^ 1][tn] = frag(Bs, wn * WTN + tn * 32 + frow, 2 * (s + 1) + fk);
      }
      __builtin_amdgcn_sched_barrier(0);                     // the next step's reads ahead of this one's products
#pragma unroll
      for (int tn = 0; tn < TN; ++tn)
#pragma unroll
        for (int tm = 0; tm < TM; ++tm)
          acc[tn][tm] = __builtin_amdgcn_mfma_i32_32x32x32_i8(wf[b][tn], xf[b][tm], acc[tn][tm], 0, 0, 0);
      __builtin_amdgcn_sched_barrier(0);
    }
    if (kt + 1 < nk) {
      // tile kt's fragments are in registers; wait for tile kt + 1, then stage `cur` takes tile kt + STAGES
      asm volatile("" ::: "memory");
      wait_tiles<PER, STAGES - 2>(min(STAGES - 2, nk - 2 - kt));
      __builtin_amdgcn_s_barrier();
      asm volatile("" ::: "memory");
      if (kt + STAGES < nk) issue(kt + STAGES, cur);
      uint4* An = lds + ((kt + 1) % STAGES) * STAGE;
      clear_tail(kt + 1, An);
#pragma unroll
      for (int tm = 0; tm < TM; ++tm) xf[0][tm] = frag(An, wm * WTM + tm * 32 + frow, fk);
#pragma unroll
      for (int tn = 0; tn < TN; ++tn) wf[0][tn] = frag(An + BM * 8, wn * WTN + tn * 32 + frow, fk);
    }
  }

  // ---- epilogue: each wave transposes 32 rows by CW outputs at a time through its own part of LDS (slots
  // swizzled by the row), and lanes then hold 8 neighbouring outputs of a row: CW / 8 lanes write one run.
  constexpr int OL = CW / 8, RP = 64 / OL;                   // lanes per row, rows per pass
  __syncthreads();
  int4* stg = (int4*)lds + wave * (32 * CW / 4);
  const int oct = lane % OL, prow = lane / OL;
#pragma unroll
  for (int t0 = 0; t0 < TN; t0 += CW / 32) {
    const int o = n0 + wn * WTN + t0 * 32 + oct * 8;
    float sw[8], bias[8];
    if (gridDim.y == 1) {
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const int c = min(o + j, a.c_out - 1);
        sw[j] = a.sw[c];
        bias[j] = a.bias ? a.bias[c] : 0.f;
      }
    }
#pragma unroll
    for (int tm = 0; tm < TM; ++tm) {
#pragma unroll
      for (int tn = 0; tn < CW / 32; ++tn)
#pragma unroll
        for (int g = 0; g < 4; ++g) {
          const i32x16& v = acc[t0 + tn][tm];
          stg[frow * (CW / 4) + ((tn * 8 + 2 * g + fk) ^ (frow & (CW / 4 - 1)))] =
              make_int4(v[4 * g], v[4 * g + 1], v[4 * g + 2], v[4 * g + 3]);
        }
      __builtin_amdgcn_s_waitcnt(0xC07F);                    // lgkmcnt(0): this wave's writes have landed
      __builtin_amdgcn_wave_barrier();
#pragma unroll
      for (int p = 0; p < 32; p += RP) {
        const int r = p + prow, row = m0 + wm * WTM + tm * 32 + r;
        const int4 lo = stg[r * (CW / 4) + ((2 * oct) ^ (r & (CW / 4 - 1)))];
        const int4 hi = stg[r * (CW / 4) + ((2 * oct + 1) ^ (r & (CW / 4 - 1)))];
        const int v[8] = {lo.x, lo.y, lo.z, lo.w, hi.x, hi.y, hi.z, hi.w};
        if (row >= a.n || o >= a.c_out) continue;
        if (gridDim.y > 1) {
          int* out = a.partial + ((long long)blockIdx.y * a.n + row) * a.c_out + o;
          if (o + 8 <= a.c_out) {
            *(i32x4_any*)out = i32x4_any{v[0], v[1], v[2], v[3]};
            *(i32x4_any*)(out + 4) = i32x4_any{v[4], v[5], v[6], v[7]};
          } else {
            for (int j = 0; j < a.c_out - o; ++j) out[j] = v[j];
          }
          continue;
        }
        const float sx = a.sx[row];
        float f[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) f[j] = finish(v[j], sx * sw[j], bias[j], a.relu);
        const long long at = row * a.ld_y + o;
        if (o + 8 <= a.c_out) {
          if (a.out_bf16) {
            bf16x8_any h;
#pragma unroll
            for (int j = 0; j < 8; ++j) h[j] = (__bf16)f[j];
            *(bf16x8_any*)((__bf16*)a.y + at) = h;
          } else {
            *(f32x4_any*)((float*)a.y + at) = f32x4_any{f[0], f[1], f[2], f[3]};
            *(f32x4_any*)((float*)a.y + at + 4) = f32x4_any{f[4], f[5], f[6], f[7]};
          }
        } else {
#pragma unroll
          for (int j = 0; j < 8; ++j)
            if (o + j < a.c_out) {
              if (a.out_bf16) ((__bf16*)a.y)[at + j] = (__bf16)f[j];
              else ((float*)a.y)[at + j] = f[j];
            }
        }
      }
      __builtin_amdgcn_s_waitcnt(0xC07F);                    // reads done before the region is rewritten
      __builtin_amdgcn_wave_barrier();
    }
  }
}

// 16 bytes of a row from k on; chunks behind the row's last are 0, and bytes behind c_in.
__device__ __forceinline__ i32x4 x_chunk(const int8_t* p, int k, int c_in) {
  i32x4 v = {0, 0, 0, 0};
  if (k < c_in) v = *(const i32x4*)(p + k);
  if (k + 16 > c_in) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int left = c_in - (k + 4 * i);
      v[i] = left <= 0 ? 0 : left < 4 ? v[i] & ((1 << (8 * left)) - 1) : v[i];
    }
  }
  return v;
}

// Few rows (up to 16 NB): one launch whose bound is the bytes of w, each read once, by one wave, without LDS.
// A workgroup takes 16 rows of w and its WAVES waves the 64-byte steps of K in turn, UNROLL steps in flight;
// v_mfma_i32_16x16x64_i8 sums them (lane l holds 16 bytes from 16 (l / 16) of row l % 16 of either operand,
// and outputs 4 (l / 16) .. + 3 of w's rows for row l % 16 of x), and the waves' sums meet in LDS.
// 1 x 4096 x 4096: 5.6 us, 3.0 TB/s.
template <int NB, int WAVES, int UNROLL>
__global__ __launch_bounds__(WAVES * 64) void fc_i8_rows_kernel(FcI8Args a) {
  __shared__ int4 sums[WAVES][NB][64];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int o0 = blockIdx.x * 16, r = lane & 15, q = lane >> 4;
  const int8_t* wp = a.w + min(o0 + r, a.c_out - 1) * a.ld_w;
  const int8_t* xp[NB];
#pragma unroll
  for (int b = 0; b < NB; ++b) xp[b] = a.x + min(b * 16 + r, a.n - 1) * a.ld_x;
  i32x4 acc[NB];
#pragma unroll
  for (int b = 0; b < NB; ++b) acc[b] = i32x4{0, 0, 0, 0};
  const int steps = (a.c_in + 63) / 64;
  for (int s0 = wave; s0 < steps; s0 += WAVES * UNROLL) {
    i32x4 w[UNROLL], x[UNROLL][NB];
#pragma unroll
    for (int i = 0; i < UNROLL; ++i) {
      const int k = (s0 + i * WAVES) * 64 + q * 16;
      w[i] = i32x4{0, 0, 0, 0};
      if (k < a.c_in) w[i] = __builtin_nontemporal_load((const i32x4*)(wp + k));
#pragma unroll
      for (int b = 0; b < NB; ++b) x[i][b] = x_chunk(xp[b], k, a.c_in);
    }
#pragma unroll
    for (int i = 0; i < UNROLL; ++i)
#pragma unroll
      for (int b = 0; b < NB; ++b) acc[b] = __builtin_amdgcn_mfma_i32_16x16x64_i8(w[i], x[i][b], acc[b], 0, 0, 0);
  }
#pragma unroll
  for (int b = 0; b < NB; ++b) sums[wave][b][lane] = make_int4(acc[b][0], acc[b][1], acc[b][2], acc[b][3]);
  __syncthreads();
  for (int t = threadIdx.x; t < NB * 64; t += WAVES * 64) {
    const int b = t >> 6, l = t & 63;
    int v[4] = {0, 0, 0, 0};
#pragma unroll
    for (int w = 0; w < WAVES; ++w) {
      const int4 p = sums[w][b][l];
      v[0] += p.x;
      v[1] += p.y;
      v[2] += p.z;
      v[3] += p.w;
    }
    const int row = b * 16 + (l & 15), o = o0 + 4 * (l >> 4);
    if (row >= a.n) continue;
    const float sx = a.sx[row];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      if (o + j >= a.c_out) continue;
      const float f = finish(v[j], sx * a.sw[o + j], a.bias ? a.bias[o + j] : 0.f, a.relu);
      if (a.out_bf16) ((__bf16*)a.y)[row * a.ld_y + o + j] = (__bf16)f;
      else ((float*)a.y)[row * a.ld_y + o + j] = f;
    }
  }
}

// Joins the splits' sums: a thread per 4 outputs of a row.  Bound by its launch and the sums' bytes: 4 us for 8 splits
// of 64 x 4096.
__global__ __launch_bounds__(256) void fc_i8_reduce_kernel(FcI8Args a, int splits) {
  const int quads = (a.c_out + 3) / 4;
  const long long total = (long long)a.n * quads, plane = (long long)a.n * a.c_out;
  for (long long i = (long long)blockIdx.x * 256 + threadIdx.x; i < total; i += (long long)gridDim.x * 256) {
    const int row = (int)(total >> 32 ? i / quads : (uint32_t)i / (uint32_t)quads), o = (int)(i - (long long)row * quads) * 4;
    const int* p = a.partial + (long long)row * a.c_out + o;
    i32x4 acc = {0, 0, 0, 0};
    if (o + 4 <= a.c_out) {
#pragma unroll 4
      for (int s = 0; s < splits; ++s) acc += *(const i32x4_any*)(p + s * plane);
    } else {
      for (int s = 0; s < splits; ++s)
#pragma unroll
        for (int j = 0; j < 3; ++j) acc[j] += o + j < a.c_out ? p[s * plane + j] : 0;
    }
    const float sx = a.sx[row];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      if (o + j >= a.c_out) continue;
      const float v = finish(acc[j], sx * a.sw[o + j], a.bias ? a.bias[o + j] : 0.f, a.relu);
      if (a.out_bf16) ((__bf16*)a.y)[row * a.ld_y + o + j] = (__bf16)v;
      else ((float*)a.y)[row * a.ld_y + o + j] = v;
    }
  }
}

template <bool BF16, int NT, int CH>
hipError_t launch_quantize_rows(const void* x, long long ld_x, int n, int c, int8_t* q, long long ld_q, float* scale,
                                hipStream_t s) {
  for (long long row = 0; row < n; row += 1 << 20) {         // 2^20 rows a launch at most
    launch(quantize_kernel<BF16, NT, CH>, dim3((unsigned)std::min<long long>(n - row, 1 << 20)), dim3(NT), s, x, ld_x,
           (int)row, c, q, ld_q, scale);
    const hipError_t st = hipGetLastError();
    if (st != hipSuccess) return st;
  }
  return hipSuccess;
}

template <bool BF16>
hipError_t launch_quantize_by_length(const void* x, long long ld_x, int n, int c, int8_t* q, long long ld_q, float* scale,
                                     hipStream_t s) {
  constexpr int V = BF16 ? 8 : 4;
  if (c <= 256 * 2 * V) return launch_quantize_rows<BF16, 256, 2>(x, ld_x, n, c, q, ld_q, scale, s);
  if (c <= 1024 * 2 * V) return launch_quantize_rows<BF16, 1024, 2>(x, ld_x, n, c, q, ld_q, scale, s);
  if (c <= 1024 * 7 * V) return launch_quantize_rows<BF16, 1024, 7>(x, ld_x, n, c, q, ld_q, scale, s);
  return launch_quantize_rows<BF16, 1024, 0>(x, ld_x, n, c, q, ld_q, scale, s);
}

}  // namespace

hipError_t launch_quantize(const void* x, bool bf16, long long ld_x, int n, int c, int8_t* q, long long ld_q,
                           float* scale, hipStream_t s) {
  return bf16 ? launch_quantize_by_length<true>(x, ld_x, n, c, q, ld_q, scale, s)
              : launch_quantize_by_length<false>(x, ld_x, n, c, q, ld_q, scale, s);
}

// The tile configurations, largest first.
struct FcConfig {
  int bm, bn;
};
constexpr FcConfig kConfigs[] = {{256, 256}, {128, 128}, {64, 128}};
constexpr int kUnitsOfGpu = 256;

struct FcPlan {
  int cfg, splits, kt_per_split;
};

// The largest tile that still gives every compute unit one (2048 x 1024 x 8192: 26.8 us in 256 x 256, 29.0 in 128 x 128,
// 35.2 in 64 x 128; 1000 x 4096 x 4096: 53, 28 and 28 us), else the smallest, with K split over the idle units
// in runs of at least 8 K tiles (64 x 25088 x 4096: 78 us unsplit, 24 in 8, 27 in 16; 128 x 2048 x 1000: 10.3
// unsplit, 10.7 in 2, 12.3 in 4): the splits' sums go through memory and a second launch.
FcPlan plan_fc(int n, int c_in, int c_out) {
  const int ktiles = (c_in + 127) / 128;
  auto tiles = [&](int c) {
    return ((long long)n + kConfigs[c].bm - 1) / kConfigs[c].bm * (((long long)c_out + kConfigs[c].bn - 1) / kConfigs[c].bn);
  };
  int cfg = 0;
  while (cfg < 2 && tiles(cfg) < kUnitsOfGpu) ++cfg;
  const int splits = (int)std::max<long long>(1, std::min<long long>(kUnitsOfGpu / tiles(cfg), ktiles / 8));
  FcPlan p{cfg, 1, (ktiles + splits - 1) / splits};
  p.splits = (ktiles + p.kt_per_split - 1) / p.kt_per_split;
  return p;
}

template <int BM, int BN, int WM, int WN, int STAGES, int OCC>
hipError_t launch_tile(const FcI8Args& a, int splits, hipStream_t s) {
  const long long tiles = (long long)((a.n + BM - 1) / BM) * ((a.c_out + BN - 1) / BN);
  if (tiles > (1 << 22)) return hipErrorInvalidValue;
  launch(fc_i8_tile_kernel<BM, BN, WM, WN, STAGES, OCC>, dim3((unsigned)tiles, splits), dim3(WM * WN * 64), s, a);
  return hipGetLastError();
}

// What fc_i8_rows_kernel takes: its waves read x again for every 16 outputs, so it suits products whose x and w are
// small.  In us, and in tiles: 1 x 4096 x 4096 7.8 and 12.0, 16 x 8192 x 4096 10.9 and 11.4, 32 x 4096 x 4096 8.7 and 12.1;
// but 32 x 8192 x 4096 15.1 and 12.4, 16 x 12288 x 1000 15.2 and 11.6, 16 x 1024 x 30000 11.3 and 7.3.
bool few_rows(int n, int c_in, int c_out) {
  if (n > 32) return false;
  const int blocks = (n + 15) / 16;
  return c_in * blocks <= 8192 && c_out <= 16384 && (long long)c_in * c_out * blocks <= 1 << 25;
}

long long fc_i8_workspace_bytes(int n, int c_in, int c_out) {
  if (few_rows(n, c_in, c_out)) return 0;
  const FcPlan p = plan_fc(n, c_in, c_out);
  return p.splits > 1 ? (long long)p.splits * n * c_out * 4 : 0;
}

hipError_t launch_fc_i8(const FcI8Args& args, hipStream_t s) {
  FcI8Args a = args;
  if (few_rows(a.n, a.c_in, a.c_out)) {
    const dim3 grid((a.c_out + 15) / 16);
    if (a.n <= 16) launch(fc_i8_rows_kernel<1, 8, 4>, grid, dim3(512), s, a);
    else launch(fc_i8_rows_kernel<2, 8, 4>, grid, dim3(512), s, a);
    return hipGetLastError();
  }
  const FcPlan p = plan_fc(a.n, a.c_in, a.c_out);
  a.kt_per_split = p.kt_per_split;
  hipError_t st;
  switch (p.cfg) {
    case 0: st = launch_tile<256, 256, 2, 4, 2, 2>(a, p.splits, s); break;
    case 1: st = launch_tile<128, 128, 2, 2, 2, 2>(a, p.splits, s); break;
    default: st = launch_tile<64, 128, 1, 4, 3, 2>(a, p.splits, s); break;
  }
  if (st != hipSuccess || p.splits == 1) return st;
  const long long total = (long long)a.n * ((a.c_out + 3) / 4);
  launch(fc_i8_reduce_kernel, dim3((unsigned)std::min<long long>((total + 255) / 256, 1 << 16)), dim3(256), s, a, p.splits);
  return hipGetLastError();
}

}  // namespace rafiki
