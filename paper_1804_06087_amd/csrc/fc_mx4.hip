// FC layer in 4-bit floating point with a scale for every 32 values, on the matrix cores, and the quantisation
// of its rows (rafiki_tokens.h).
//
// v_mfma_scale_f32_*_f8f6f4 takes 32 codes of one block a lane (16 bytes) and the block's scale byte from a
// register's byte that the instruction names, the same for all lanes.  A lane that holds 4 neighbouring blocks of a row
// thus needs one 4-byte load of scales for 4 instructions, and since sums over K may take blocks in any order
// that both operands agree on, neighbouring blocks of a lane need not be neighbours in the instruction's K.
#include "tokens.h"

#include <algorithm>

namespace rafiki {

namespace {

typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef int i32x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef uint32_t u32x4_any __attribute__((ext_vector_type(4), aligned(2)));
typedef uint32_t u32_byte __attribute__((aligned(1)));

template <bool BF16>
__device__ __forceinline__ float value(const void* p, long long i) {
  if constexpr (BF16) return __uint_as_float((uint32_t)((const bf16_t*)p)[i] << 16);
  else return ((const float*)p)[i];
}

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));

// Two values over `scale` as codes in byte `at` of `codes`: to the nearest magnitude, ties to even, above 6 to 6, the sign kept.
__device__ __forceinline__ uint32_t two_codes(uint32_t codes, bf16x2 v, float scale, int at) {
  switch (at) {
    case 0: return __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(codes, v, scale, 0);
    case 1: return __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(codes, v, scale, 1);
    case 2: return __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(codes, v, scale, 2);
    default: return __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(codes, v, scale, 3);
  }
}
__device__ __forceinline__ uint32_t two_codes(uint32_t codes, float lo, float hi, float scale, int at) {
  switch (at) {
    case 0: return __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(codes, lo, hi, scale, 0);
    case 1: return __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(codes, lo, hi, scale, 1);
    case 2: return __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(codes, lo, hi, scale, 2);
    default: return __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(codes, lo, hi, scale, 3);
  }
}

// A thread per 8 values of a block, 4 threads a block: its largest magnitude, then the codes.  Bits of magnitudes order as the
// magnitudes, NaN above +inf.  Bound by bytes: 30001 x 2050 bf16 30 us (5.1 TB/s; with codes from comparisons and a 64-bit
// division 45), 4096 x 25088 fp32 81 us (5.8 TB/s).
template <bool BF16>
__global__ __launch_bounds__(256) void quantize_mx4_kernel(const void* x, long long ld_x, int n, int c, uint8_t* q,
                                                           long long ld_q, uint8_t* scale, long long ld_scale) {
  constexpr int W = BF16 ? 4 : 8;                            // registers of 8 values
  const int quarters = (c + 31) / 32 * 4;
  const long long total = (long long)n * quarters;
  for (long long i = (long long)blockIdx.x * 256 + threadIdx.x; i < total; i += (long long)gridDim.x * 256) {
    const long long row = total >> 32 ? i / quarters : (uint32_t)i / (uint32_t)quarters;
    const int part = (int)(i - row * quarters), c0 = part * 8;
    const long long base = row * ld_x + c0;
    uint32_t v[W];
    if (c0 + 8 <= c) {
#pragma unroll
      for (int h = 0; h < W / 4; ++h) {
        const u32x4_any w = *(const u32x4_any*)((const char*)x + base * (BF16 ? 2 : 4) + 16 * h);
#pragma unroll
        for (int j = 0; j < 4; ++j) v[4 * h + j] = w[j];
      }
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const uint32_t b = c0 + j < c ? __float_as_uint(value<BF16>(x, base + j)) : 0u;
        if constexpr (!BF16) v[j] = b;
        else v[j / 2] = j & 1 ? v[j / 2] | b : b >> 16;
      }
    }
    uint32_t top = 0;
#pragma unroll
    for (int j = 0; j < W; ++j) {
      if constexpr (BF16) top = max(top, max(v[j] << 16 & 0x7FFF0000u, v[j] & 0x7FFF0000u));
      else top = max(top, v[j] & 0x7FFFFFFFu);
    }
    top = max(top, (uint32_t)__shfl_xor((int)top, 1, 64));
    top = max(top, (uint32_t)__shfl_xor((int)top, 2, 64));
    const bool bad = top >= 0x7F800000u;
    const int e = max((int)(top >> 23) - 127 - 2, -127);     // of a value below 2^-126, at most -127 too
    const float s = e == -127 ? 0x1p-127f : __uint_as_float((uint32_t)(127 + e) << 23);
    uint32_t codes = 0;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      if constexpr (BF16) codes = two_codes(codes, __builtin_bit_cast(bf16x2, v[j]), s, j);
      else codes = two_codes(codes, __uint_as_float(v[2 * j]), __uint_as_float(v[2 * j + 1]), s, j);
    }
    *(u32_byte*)(q + row * ld_q + part * 4) = bad ? 0u : codes;
    if ((part & 3) == 0) scale[row * ld_scale + part / 4] = bad ? 255 : (uint8_t)(e + 127);
  }
}

__device__ __forceinline__ float finish(float acc, float bias, int relu) {
  const float v = acc + bias;
  return relu && v < 0.f ? 0.f : v;                          // NaN stays NaN
}

// The builtins take 8 registers for every 8-, 6- and 4-bit type; of 4-bit codes the instruction reads 4.
__device__ __forceinline__ i32x8 wide(i32x4 v) { return __builtin_shufflevector(v, v, 0, 1, 2, 3, -1, -1, -1, -1); }

// Products of one step, whose scales are byte `s` of the registers.
__device__ __forceinline__ f32x16 mfma32(i32x4 w, i32x4 x, f32x16 acc, int s, int sw, int sx) {
  switch (s) {
    case 0: return __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(wide(w), wide(x), acc, 4, 4, 0, sw, 0, sx);
    case 1: return __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(wide(w), wide(x), acc, 4, 4, 1, sw, 1, sx);
    case 2: return __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(wide(w), wide(x), acc, 4, 4, 2, sw, 2, sx);
    default: return __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(wide(w), wide(x), acc, 4, 4, 3, sw, 3, sx);
  }
}
__device__ __forceinline__ f32x4 mfma16(i32x4 w, i32x4 x, f32x4 acc, int s, int sw, int sx) {
  switch (s) {
    case 0: return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(wide(w), wide(x), acc, 4, 4, 0, sw, 0, sx);
    case 1: return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(wide(w), wide(x), acc, 4, 4, 1, sw, 1, sx);
    case 2: return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(wide(w), wide(x), acc, 4, 4, 2, sw, 2, sx);
    default: return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(wide(w), wide(x), acc, 4, 4, 3, sw, 3, sx);
  }
}

// Up to 16 rows: 16 rows of w a workgroup, whose 8 waves take the steps of 16 blocks in turn.  Lane l holds blocks 4 (l / 16) ..
// + 3 of a step of row l % 16 of either operand; outputs are 4 (l / 16) .. + 3 of w's rows for row l % 16 of x, and the
// waves' sums meet in LDS.  Bound by w's bytes and the launch: 1 x 4096 x 4096 4.5 us, 1 x 25088 x 4096 12 us (4.5 TB/s; in 4 waves
// 16).
__global__ __launch_bounds__(512) void fc_mx4_rows_kernel(FcMx4Args a) {
  constexpr int NW = 8;
  __shared__ f32x4 sums[NW][64];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int o0 = blockIdx.x * 16, r = lane & 15, q = lane >> 4;
  const long long wr = min(o0 + r, a.c_out - 1), xr = min(r, a.n - 1);
  const uint8_t *wp = a.w + wr * a.ld_w, *wsp = a.ws + wr * a.ld_ws, *xp = a.x + xr * a.ld_x, *xsp = a.xs + xr * a.ld_xs;
  f32x4 acc = {0.f, 0.f, 0.f, 0.f};
  const int steps = (a.blocks + 15) / 16;
  for (int s = wave; s < steps; s += NW) {
    const int b0 = s * 16 + q * 4, left = a.blocks - b0;     // blocks of the row from this lane's first on
    // scales behind the row's blocks are 0 (2^-127), not what lies there: NaN times code 0 is NaN
    const uint32_t mask = left >= 4 ? ~0u : left <= 0 ? 0u : (1u << (8 * left)) - 1;
    i32x4 w[4], x[4];
    const int sw = (int)(*(const uint32_t*)(wsp + b0) & mask), sx = (int)(*(const uint32_t*)(xsp + b0) & mask);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      w[i] = x[i] = i32x4{0, 0, 0, 0};
      if (i < left) w[i] = *(const i32x4*)(wp + (long long)(b0 + i) * 16);
      if (i < left) x[i] = *(const i32x4*)(xp + (long long)(b0 + i) * 16);
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) acc = mfma16(w[i], x[i], acc, i, sw, sx);
  }
  sums[wave][lane] = acc;
  __syncthreads();
  if (threadIdx.x >= 64) return;
  f32x4 v = sums[0][lane];
#pragma unroll
  for (int w = 1; w < NW; ++w) v += sums[w][lane];
  const int o = o0 + 4 * q;
  if (r >= a.n) return;
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    if (o + j >= a.c_out) continue;
    const float f = finish(v[j], a.bias ? a.bias[o + j] : 0.f, a.relu);
    if (a.out_bf16) ((__bf16*)a.y)[r * a.ld_y + o + j] = (__bf16)f;
    else ((float*)a.y)[r * a.ld_y + o + j] = f;
  }
}

// s_waitcnt with only the vector-memory counter constrained (gfx9 encoding).
template <int N>
__device__ __forceinline__ void wait_vmcnt() {
  static_assert(N >= 0 && N < 64, "vmcnt range");
  __builtin_amdgcn_s_waitcnt((N & 0xF) | ((N >> 4) << 14) | (0x7 << 4) | (0xF << 8));
}

typedef float f32x4_any __attribute__((ext_vector_type(4), aligned(4)));
typedef __bf16 bf16x8_any __attribute__((ext_vector_type(8), aligned(2)));
typedef __attribute__((address_space(3))) void lds_void;
typedef __attribute__((address_space(3))) i32x4 lds_i32x4;
typedef __attribute__((address_space(3))) uint32_t lds_u32;

// Row r of an LDS tile (128 bytes, 8 blocks) keeps block c in slot c ^ swz(r): 16 rows' equal blocks then lie on 64
// different banks.
__device__ __forceinline__ int swz(int r) { return (r & 7) ^ ((r >> 3) & 1); }

// One wave's loads of a K tile.  Codes: instruction j of wave w fills rows (j NW + w) 8 .. + 7 of an operand's 128 bytes a
// row, lane l slot l % 8 of row l / 8 of those.  Scales: 16 bytes a row for two K tiles, row 64 i + l in
// instruction i.  Rows and blocks past the operands get an offset past the buffer's end, for which the hardware
// writes zeros.
template <int BM, int BN, int NW>
struct MxTileLoader {
  static constexpr int RA = BM / (8 * NW), RB = BN / (8 * NW), SA = BM / 64, SB = BN / 64, S = (SA + SB + NW - 1) / NW;
  static constexpr unsigned kOut = 0x60000000u;              // past every tile (at most 2^30 bytes and a row)
  static_assert(RA >= 1 && RB >= 1 && SA >= 1 && SB >= 1 && NW % 2 == 0, "tile shape");
  __amdgpu_buffer_rsrc_t xr, wr, xsr, wsr;
  unsigned xo[RA], wo[RB], so[S];
  int chunk, wave, blocks, scale_bytes;

  __device__ __forceinline__ void init(const FcMx4Args& a, int m0, int n0, int wave_, int lane) {
    wave = wave_;
    blocks = a.blocks;
    scale_bytes = (blocks + 15) / 16 * 16;
    const int lrow = lane >> 3, x_rows = min(BM, a.n - m0), w_rows = min(BN, a.c_out - n0);
    chunk = (lane & 7) ^ lrow ^ (wave & 1);
    xr = __builtin_amdgcn_make_buffer_rsrc((void*)(a.x + m0 * a.ld_x), (short)0, (int)((x_rows - 1) * a.ld_x) + blocks * 16,
                                           0x00020000);
    wr = __builtin_amdgcn_make_buffer_rsrc((void*)(a.w + n0 * a.ld_w), (short)0, (int)((w_rows - 1) * a.ld_w) + blocks * 16,
                                           0x00020000);
    xsr = __builtin_amdgcn_make_buffer_rsrc((void*)(a.xs + m0 * a.ld_xs), (short)0, (int)((x_rows - 1) * a.ld_xs) + scale_bytes,
                                            0x00020000);
    wsr = __builtin_amdgcn_make_buffer_rsrc((void*)(a.ws + n0 * a.ld_ws), (short)0, (int)((w_rows - 1) * a.ld_ws) + scale_bytes,
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
#pragma unroll
    for (int i = 0; i < S; ++i) {
      const int k = i * NW + wave;                           // x's SA instructions, then w's
      const int r = (k < SA ? k : k - SA) * 64 + lane;
      so[i] = k < SA ? (r < x_rows ? (unsigned)(r * a.ld_xs) : kOut) : (r < w_rows ? (unsigned)(r * a.ld_ws) : kOut);
    }
  }
  // K tile kt's codes into `base` (x's rows, then w's).
  __device__ __forceinline__ void issue(int kt, uint4* base) const {
    const bool inside = kt * 8 + chunk < blocks;
#pragma unroll
    for (int j = 0; j < RA; ++j)
      __builtin_amdgcn_raw_ptr_buffer_load_lds(xr, (lds_void*)(base + (j * NW + wave) * 64), 16, inside ? xo[j] : kOut, kt * 128,
                                               0, 0);
#pragma unroll
    for (int j = 0; j < RB; ++j)
      __builtin_amdgcn_raw_ptr_buffer_load_lds(wr, (lds_void*)(base + BM * 8 + (j * NW + wave) * 64), 16, inside ? wo[j] : kOut,
                                               kt * 128, 0, 0);
  }
  // The scales of K tiles kt and kt + 1 (kt even) into `base` (x's rows, then w's).
  __device__ __forceinline__ void issue_scales(int kt, uint4* base) const {
#pragma unroll
    for (int i = 0; i < S; ++i) {
      const int k = i * NW + wave;
      if (k < SA) __builtin_amdgcn_raw_ptr_buffer_load_lds(xsr, (lds_void*)(base + k * 64), 16, so[i], kt * 8, 0, 0);
      else if (k < SA + SB) __builtin_amdgcn_raw_ptr_buffer_load_lds(wsr, (lds_void*)(base + k * 64), 16, so[i], kt * 8, 0, 0);
    }
  }
};

// Tiled product: BM rows of x by BN rows of w per workgroup of WM x WN waves, K in tiles of 256 codes (128
// bytes) that go from memory to two LDS buffers in turn without registers (buffer loads ... lds); v_mfma_scale_f32_32x32x64
// with w as the first operand, so that a lane sums 4 neighbouring outputs of one row.  Splits (grid y) each sum a
// range of K tiles (an even number of them, since scales come for two); with more than one the sums go to the
// workspace and fc_mx4_reduce_kernel joins them in their order.
//
// Measured on an MI355X: 4096 x 4096 x 30000 306 to 338 us by the values (3.0 to 3.3 PFLOP/s), 8192 x 8192 x 8192 272 us (4.0; the
// library's product of the same types 359 us).  Matrix cores are busy for 47 % of the cycles at the 2.04 GHz that the load leaves
// them; products from registers alone reach 6.7 PFLOP/s on random codes and 9.1 on zeros.  8192^3 without the loads takes
// 216 us, without the products 184, without the stores 252, on zeros 222: LDS, which takes both operands' tiles and gives
// each wave 192 rows for 128 x 64 outputs, and the power of all that share the time.  Slower: 4 waves of 128 x 128 (296 us),
// loads between the products (285), a ring of four 64-byte tiles (316), outputs exchanged between lanes instead of through
// LDS (273, but 4096 x 4096 x 30000 338, 320 with the next tile's loads beside them), scales for four tiles at once (287).
template <int BM, int BN, int WM, int WN, int OCC>
__global__ __launch_bounds__(WM * WN * 64, OCC) void fc_mx4_tile_kernel(FcMx4Args a) {
  constexpr int NW = WM * WN;
  constexpr int WTM = BM / WM, WTN = BN / WN, TM = WTM / 32, TN = WTN / 32;
  constexpr int STAGE = (BM + BN) * 8, SCALES = BM + BN;     // 16-byte chunks
  static_assert(TM >= 1 && TN >= 1, "tile shape");
  static_assert((STAGE + SCALES) * 2 * 16 <= 160 * 1024, "LDS budget");
  constexpr int CW = TN >= 2 ? 64 : 32;                      // outputs of a row staged at once
  static_assert(NW * 32 * CW * 4 <= STAGE * 2 * 16, "epilogue staging fits in LDS");
  __shared__ __align__(128) uint4 lds[(STAGE + SCALES) * 2];
  uint4* const lds_scales = lds + STAGE * 2;

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

  const int ktiles = (a.blocks + 7) / 8;
  const int kt0 = blockIdx.y * a.kt_per_split, nk = min(a.kt_per_split, ktiles - kt0);

  MxTileLoader<BM, BN, NW> loader;
  loader.init(a, m0, n0, wave, lane);
  auto issue = [&](int t) {
    loader.issue(kt0 + t, lds + (t & 1) * STAGE);
    if ((t & 1) == 0) loader.issue_scales(kt0 + t, lds_scales + (t >> 1 & 1) * SCALES);
  };

  f32x16 acc[TN][TM];
#pragma unroll
  for (int i = 0; i < TN; ++i)
#pragma unroll
    for (int j = 0; j < TM; ++j)
#pragma unroll
      for (int e = 0; e < 16; ++e) acc[i][j][e] = 0.f;

  // Lane l holds block 4 (l / 32) + s of its row in step s of a K tile: of a block in slot c ^ swz(r), s is two bits of the
  // address.  Addresses are bytes of LDS, so that one register a tile serves an operand's reads.
  const int frow = lane & 31, fk = lane >> 5;
  const uint32_t lds_at = (uint32_t)(uintptr_t)(lds_void*)lds;
  const uint32_t slot = ((4 * fk) ^ swz(frow)) * 16;
  const uint32_t x_at = lds_at + (wm * WTM + frow) * 128 + slot, w_at = lds_at + (BM + wn * WTN + frow) * 128 + slot;
  const uint32_t xs_at = lds_at + STAGE * 32 + (wm * WTM + frow) * 16 + fk * 4;
  const uint32_t ws_at = lds_at + STAGE * 32 + (BM + wn * WTN + frow) * 16 + fk * 4;

  i32x4 xf[2][TM], wf[2][TN];
  int sx[TM], sw[TN];
  auto read = [&](int b, uint32_t stage, int s) {
    const uint32_t xa = (x_at + stage) ^ (s * 16), wa = (w_at + stage) ^ (s * 16);
#pragma unroll
    for (int tm = 0; tm < TM; ++tm) xf[b][tm] = *(const lds_i32x4*)(xa + tm * 4096);
#pragma unroll
    for (int tn = 0; tn < TN; ++tn) wf[b][tn] = *(const lds_i32x4*)(wa + tn * 4096);
  };
  auto first_step = [&](int t) {
    read(0, (t & 1) * STAGE * 16, 0);
    // scales behind the rows' blocks are 0 (2^-127), not what lies there: NaN times code 0 is NaN
    const int left = a.blocks - (kt0 + t) * 8 - 4 * fk;
    const uint32_t mask = left >= 4 ? ~0u : left <= 0 ? 0u : (1u << (8 * left)) - 1;
    const uint32_t at = (t >> 1 & 1) * SCALES * 16 + (t & 1) * 8;
#pragma unroll
    for (int tm = 0; tm < TM; ++tm) sx[tm] = (int)(*(const lds_u32*)(xs_at + at + tm * 512) & mask);
#pragma unroll
    for (int tn = 0; tn < TN; ++tn) sw[tn] = (int)(*(const lds_u32*)(ws_at + at + tn * 512) & mask);
  };
  if (nk > 0) {
    issue(0);
    if (nk > 1) issue(1);
    wait_vmcnt<0>();
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
    first_step(0);
  }
  for (int t = 0; t < nk; ++t) {
    uint32_t stage = (t & 1) * STAGE * 16;
    asm volatile("" : "+s"(stage));                          // or the addresses of both buffers stay in registers
#pragma unroll
    for (int s = 0; s < 4; ++s) {
      const int b = s & 1;
      if (s < 3) read(b ^ 1, stage, s + 1);
      __builtin_amdgcn_sched_barrier(0);                     // the next step's reads ahead of this one's products
#pragma unroll
      for (int tn = 0; tn < TN; ++tn)
#pragma unroll
        for (int tm = 0; tm < TM; ++tm) acc[tn][tm] = mfma32(wf[b][tn], xf[b][tm], acc[tn][tm], s, sw[tn], sx[tm]);
      __builtin_amdgcn_sched_barrier(0);
    }
    // or the compiler sinks the products behind the barrier, with all of the tile's fragments held for them
#pragma unroll
    for (int tn = 0; tn < TN; ++tn)
#pragma unroll
      for (int tm = 0; tm < TM; ++tm) asm volatile("" : "+v"(acc[tn][tm]));
    if (t + 1 < nk) {
      // tile t's fragments are in registers; wait for tile t + 1, then t's buffer takes tile t + 2
      asm volatile("" ::: "memory");
      wait_vmcnt<0>();
      __builtin_amdgcn_s_barrier();
      asm volatile("" ::: "memory");
      if (t + 2 < nk) issue(t + 2);
      first_step(t + 1);
    }
  }

  // ---- epilogue: each wave transposes 32 rows by CW outputs at a time through its own part of LDS (slots
  // swizzled by the row), and lanes then hold 8 neighbouring outputs of a row: CW / 8 lanes write one run.
  constexpr int OL = CW / 8, RP = 64 / OL;                   // lanes per row, rows per pass
  __syncthreads();
  f32x4* stg = (f32x4*)lds + wave * (32 * CW / 4);
  const int oct = lane % OL, prow = lane / OL;
#pragma unroll
  for (int t0 = 0; t0 < TN; t0 += CW / 32) {
    const int o = n0 + wn * WTN + t0 * 32 + oct * 8;
    float bias[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) bias[j] = gridDim.y == 1 && a.bias ? a.bias[min(o + j, a.c_out - 1)] : 0.f;
#pragma unroll
    for (int tm = 0; tm < TM; ++tm) {
#pragma unroll
      for (int tn = 0; tn < CW / 32; ++tn)
#pragma unroll
        for (int g = 0; g < 4; ++g) {
          const f32x16& v = acc[t0 + tn][tm];
          stg[frow * (CW / 4) + ((tn * 8 + 2 * g + fk) ^ (frow & (CW / 4 - 1)))] =
              f32x4{v[4 * g], v[4 * g + 1], v[4 * g + 2], v[4 * g + 3]};
        }
      __builtin_amdgcn_s_waitcnt(0xC07F);                    // lgkmcnt(0): this wave's writes have landed
      __builtin_amdgcn_wave_barrier();
#pragma unroll
      for (int p = 0; p < 32; p += RP) {
        const int r = p + prow, row = m0 + wm * WTM + tm * 32 + r;
        const f32x4 lo = stg[r * (CW / 4) + ((2 * oct) ^ (r & (CW / 4 - 1)))];
        const f32x4 hi = stg[r * (CW / 4) + ((2 * oct + 1) ^ (r & (CW / 4 - 1)))];
        if (row >= a.n || o >= a.c_out) continue;
        float f[8] = {lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
        float* out_f = (float*)a.y + row * a.ld_y + o;
        bool out_bf16 = a.out_bf16;
        if (gridDim.y > 1) {
          out_f = a.partial + ((long long)blockIdx.y * a.n + row) * a.c_out + o;
          out_bf16 = false;
        } else {
#pragma unroll
          for (int j = 0; j < 8; ++j) f[j] = finish(f[j], bias[j], a.relu);
        }
        __bf16* out_h = (__bf16*)a.y + row * a.ld_y + o;
        if (o + 8 <= a.c_out) {
          if (out_bf16) {
            bf16x8_any h;
#pragma unroll
            for (int j = 0; j < 8; ++j) h[j] = (__bf16)f[j];
            *(bf16x8_any*)out_h = h;
          } else {
            *(f32x4_any*)out_f = f32x4_any{f[0], f[1], f[2], f[3]};
            *(f32x4_any*)(out_f + 4) = f32x4_any{f[4], f[5], f[6], f[7]};
          }
        } else {
#pragma unroll
          for (int j = 0; j < 8; ++j)
            if (o + j < a.c_out) {
              if (out_bf16) out_h[j] = (__bf16)f[j];
              else out_f[j] = f[j];
            }
        }
      }
      __builtin_amdgcn_s_waitcnt(0xC07F);                    // reads done before the region is rewritten
      __builtin_amdgcn_wave_barrier();
    }
  }
}

// Joins the splits' sums in their order: a thread per 4 outputs of a row.  Bound by its launch and the sums' bytes: 4 us for 7
// splits of 64 x 4096.
__global__ __launch_bounds__(256) void fc_mx4_reduce_kernel(FcMx4Args a, int splits) {
  const int quads = (a.c_out + 3) / 4;
  const long long total = (long long)a.n * quads, plane = (long long)a.n * a.c_out;
  for (long long i = (long long)blockIdx.x * 256 + threadIdx.x; i < total; i += (long long)gridDim.x * 256) {
    const int row = (int)(total >> 32 ? i / quads : (uint32_t)i / (uint32_t)quads), o = (int)(i - (long long)row * quads) * 4;
    const float* p = a.partial + (long long)row * a.c_out + o;
    f32x4 acc = {0.f, 0.f, 0.f, 0.f};
    if (o + 4 <= a.c_out) {
#pragma unroll 4
      for (int s = 0; s < splits; ++s) acc += *(const f32x4_any*)(p + s * plane);
    } else {
      for (int s = 0; s < splits; ++s)
#pragma unroll
        for (int j = 0; j < 3; ++j) acc[j] += o + j < a.c_out ? p[s * plane + j] : 0.f;
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      if (o + j >= a.c_out) continue;
      const float v = finish(acc[j], a.bias ? a.bias[o + j] : 0.f, a.relu);
      if (a.out_bf16) ((__bf16*)a.y)[row * a.ld_y + o + j] = (__bf16)v;
      else ((float*)a.y)[row * a.ld_y + o + j] = v;
    }
  }
}

// The tile configurations, largest first.
struct MxConfig {
  int bm, bn;
};
constexpr MxConfig kMxConfigs[] = {{256, 256}, {128, 128}, {64, 64}};
constexpr int kUnitsOfGpu = 256;

struct MxPlan {
  int cfg, splits, kt_per_split;
};

// The largest tile that still gives every compute unit one (2048 x 1024 x 8192: 20.0 us in 256 x 256, 21.6 in 128 x 128; 1000 x
// 4096 x 4096: 33, 17.7 and 19.5 in 64 x 64; 512 x 4096 x 4096: 32, 16.0 and 11.6), else the smallest, with K split
// where two workgroups a unit leave room for it, in runs of at least 12 K tiles (64 x 25088 x 4096: 49 us unsplit,
// 18.1 in 8; 300 x 25088 x 500: 52.8 unsplit, 16.8 in 8; 40 x 4096 x 4096: 10.8 unsplit, 13.8 in 2): the splits' sums go
// through memory and a second launch.
MxPlan plan_mx4(int n, int blocks, int c_out) {
  const int pairs = (blocks + 15) / 16;                      // of K tiles
  auto tiles = [&](int c) {
    return ((long long)n + kMxConfigs[c].bm - 1) / kMxConfigs[c].bm * (((long long)c_out + kMxConfigs[c].bn - 1) / kMxConfigs[c].bn);
  };
  int cfg = 0;
  while (cfg < 2 && tiles(cfg) < kUnitsOfGpu) ++cfg;
  const int splits = cfg < 2 ? 1 : (int)std::max<long long>(1, std::min<long long>(2 * kUnitsOfGpu / tiles(cfg), pairs / 6));
  const int per = (pairs + splits - 1) / splits;
  return MxPlan{cfg, (pairs + per - 1) / per, 2 * per};
}

template <int BM, int BN, int WM, int WN, int OCC>
hipError_t launch_mx4_tile(const FcMx4Args& a, int splits, hipStream_t s) {
  const long long tiles = (long long)((a.n + BM - 1) / BM) * ((a.c_out + BN - 1) / BN);
  if (tiles > (1 << 22)) return hipErrorInvalidValue;
  launch(fc_mx4_tile_kernel<BM, BN, WM, WN, OCC>, dim3((unsigned)tiles, splits), dim3(WM * WN * 64), s, a);
  return hipGetLastError();
}

// What fc_mx4_rows_kernel takes: its workgroups read x again for every 16 outputs.  In us, and in tiles: 1 x 25088 x 4096 12.1 and
// 14.7, 2 x 8192 x 8192 10.9 and 13.6, 1 x 25088 x 100 12.4 and 13.3; but 16 x 25088 x 4096 17.1 and 15.4, 1 x 4096 x
// 30000 14.4 and 12.4, 16 x 4096 x 30000 21.6 and 12.5.
bool few_rows_mx4(int n, int blocks, int c_out) { return n <= 16 && n * blocks <= 4096 && c_out <= 8192; }

}  // namespace

hipError_t launch_quantize_mx4(const void* x, bool bf16, long long ld_x, int n, int c, uint8_t* q, long long ld_q,
                               uint8_t* scale, long long ld_scale, hipStream_t s) {
  const long long total = (long long)n * ((c + 31) / 32 * 4LL);
  const dim3 grid((unsigned)std::min<long long>((total + 255) / 256, 1 << 22));
  if (bf16) launch(quantize_mx4_kernel<true>, grid, dim3(256), s, x, ld_x, n, c, q, ld_q, scale, ld_scale);
  else launch(quantize_mx4_kernel<false>, grid, dim3(256), s, x, ld_x, n, c, q, ld_q, scale, ld_scale);
  return hipGetLastError();
}

long long fc_mx4_workspace_bytes(int n, int blocks, int c_out) {
  if (few_rows_mx4(n, blocks, c_out)) return 0;
  const MxPlan p = plan_mx4(n, blocks, c_out);
  return p.splits > 1 ? (long long)p.splits * n * c_out * 4 : 0;
}

hipError_t launch_fc_mx4(const FcMx4Args& args, hipStream_t s) {
  FcMx4Args a = args;
  if (few_rows_mx4(a.n, a.blocks, a.c_out)) {
    launch(fc_mx4_rows_kernel, dim3((a.c_out + 15) / 16), dim3(512), s, a);
    return hipGetLastError();
  }
  const MxPlan p = plan_mx4(a.n, a.blocks, a.c_out);
  a.kt_per_split = p.kt_per_split;
  hipError_t st;
  switch (p.cfg) {
    case 0: st = launch_mx4_tile<256, 256, 2, 4, 2>(a, p.splits, s); break;
    case 1: st = launch_mx4_tile<128, 128, 2, 2, 2>(a, p.splits, s); break;
    default: st = launch_mx4_tile<64, 64, 2, 2, 2>(a, p.splits, s); break;
  }
  if (st != hipSuccess || p.splits == 1) return st;
  const long long total = (long long)a.n * ((a.c_out + 3) / 4);
  launch(fc_mx4_reduce_kernel, dim3((unsigned)std::min<long long>((total + 255) / 256, 1 << 16)), dim3(256), s, a, p.splits);
  return hipGetLastError();
}

}  // namespace rafiki
