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
typedef uint32_t u32x4_any __attribute__((ext_vector_type(4), aligned(2)));
typedef uint32_t u32_byte __attribute__((aligned(1)));

template <bool BF16>
__device__ __forceinline__ float value(const void* p, long long i) {
  if constexpr (BF16) return __uint_as_float((uint32_t)((const bf16_t*)p)[i] << 16);
  else return ((const float*)p)[i];
}

// The code of v (already over its scale): magnitudes are multiples of 1/2 below 2, of 1 below 4 and of 2 above, and rounding up
// to the next such range gives its first code.
__device__ __forceinline__ uint32_t code_of(float v) {
  const float m = fminf(fabsf(v), 6.f);
  const float code = m < 2.f ? __builtin_rintf(2.f * m) : m < 4.f ? 2.f + __builtin_rintf(m) : 4.f + __builtin_rintf(0.5f * m);
  return (uint32_t)code | (__float_as_uint(v) >> 31 << 3);
}

// A thread per 8 values of a block, 4 threads a block.
template <bool BF16>
__global__ __launch_bounds__(256) void quantize_mx4_kernel(const void* x, long long ld_x, int n, int c, uint8_t* q,
                                                           long long ld_q, uint8_t* scale, long long ld_scale) {
  const int quarters = (c + 31) / 32 * 4;
  const long long total = (long long)n * quarters;
  for (long long i = (long long)blockIdx.x * 256 + threadIdx.x; i < total; i += (long long)gridDim.x * 256) {
    const long long row = i / quarters;
    const int part = (int)(i - row * quarters), c0 = part * 8;
    const long long base = row * ld_x + c0;
    float v[8];
    if (c0 + 8 <= c) {
      if constexpr (BF16) {
        const u32x4_any w = *(const u32x4_any*)((const bf16_t*)x + base);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          v[2 * j] = __uint_as_float(w[j] << 16);
          v[2 * j + 1] = __uint_as_float(w[j] & 0xFFFF0000u);
        }
      } else {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const u32x4_any w = *(const u32x4_any*)((const float*)x + base + 4 * h);
#pragma unroll
          for (int j = 0; j < 4; ++j) v[4 * h + j] = __uint_as_float(w[j]);
        }
      }
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j) v[j] = c0 + j < c ? value<BF16>(x, base + j) : 0.f;
    }
    uint32_t top = 0;                                        // bits of magnitudes order as the magnitudes, NaN above +inf
#pragma unroll
    for (int j = 0; j < 8; ++j) top = max(top, __float_as_uint(v[j]) & 0x7FFFFFFFu);
    top = max(top, (uint32_t)__shfl_xor((int)top, 1, 64));
    top = max(top, (uint32_t)__shfl_xor((int)top, 2, 64));
    const bool bad = top >= 0x7F800000u;
    const int e = max((int)(top >> 23) - 127 - 2, -127);     // of a value below 2^-126, at most -127 too
    const float inverse = __uint_as_float((uint32_t)(127 - e) << 23);   // 2^-e: e is in [-127, 125]
    uint32_t codes = 0;
#pragma unroll
    for (int j = 0; j < 8; ++j) codes |= (bad ? 0u : code_of(v[j] * inverse)) << (4 * j);
    *(u32_byte*)(q + row * ld_q + part * 4) = codes;
    if ((part & 3) == 0) scale[row * ld_scale + part / 4] = bad ? 255 : (uint8_t)(e + 127);
  }
}

__device__ __forceinline__ float finish(float acc, float bias, int relu) {
  const float v = acc + bias;
  return relu && v < 0.f ? 0.f : v;                          // NaN stays NaN
}

__device__ __forceinline__ i32x8 wide(i32x4 v) { return i32x8{v[0], v[1], v[2], v[3], 0, 0, 0, 0}; }

// Few rows (16 NB a workgroup): 16 rows of w and its WAVES waves the steps of 16 blocks in turn.  Lane l holds blocks
// 4 (l / 16) .. + 3 of a step of row l % 16 of either operand; outputs are 4 (l / 16) .. + 3 of w's rows for row l % 16 of x,
// and the waves' sums meet in LDS.
template <int NB, int WAVES>
__global__ __launch_bounds__(WAVES * 64) void fc_mx4_rows_kernel(FcMx4Args a) {
  __shared__ f32x4 sums[WAVES][NB][64];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int o0 = blockIdx.x * 16, n0 = blockIdx.y * 16 * NB, r = lane & 15, q = lane >> 4;
  const long long wr = min(o0 + r, a.c_out - 1);
  const uint8_t* wp = a.w + wr * a.ld_w;
  const uint8_t* wsp = a.ws + wr * a.ld_ws;
  const uint8_t* xp[NB];
  const uint8_t* xsp[NB];
#pragma unroll
  for (int b = 0; b < NB; ++b) {
    const long long xr = min(n0 + b * 16 + r, a.n - 1);
    xp[b] = a.x + xr * a.ld_x;
    xsp[b] = a.xs + xr * a.ld_xs;
  }
  f32x4 acc[NB];
#pragma unroll
  for (int b = 0; b < NB; ++b) acc[b] = f32x4{0.f, 0.f, 0.f, 0.f};
  const int steps = (a.blocks + 15) / 16;
  for (int s = wave; s < steps; s += WAVES) {
    const int b0 = s * 16 + q * 4, left = a.blocks - b0;     // blocks of the row from this lane's first on
    // scales behind the row's blocks are 0 (2^-127), not what lies there: NaN times code 0 is NaN
    const uint32_t mask = left >= 4 ? ~0u : left <= 0 ? 0u : (1u << (8 * left)) - 1;
    i32x4 w[4], x[NB][4];
    int sw, sx[NB];
    sw = (int)(*(const uint32_t*)(wsp + b0) & mask);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      w[i] = i32x4{0, 0, 0, 0};
      if (i < left) w[i] = *(const i32x4*)(wp + (long long)(b0 + i) * 16);
    }
#pragma unroll
    for (int b = 0; b < NB; ++b) {
      sx[b] = (int)(*(const uint32_t*)(xsp[b] + b0) & mask);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        x[b][i] = i32x4{0, 0, 0, 0};
        if (i < left) x[b][i] = *(const i32x4*)(xp[b] + (long long)(b0 + i) * 16);
      }
    }
#pragma unroll
    for (int b = 0; b < NB; ++b) {
      acc[b] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(wide(w[0]), wide(x[b][0]), acc[b], 4, 4, 0, sw, 0, sx[b]);
      acc[b] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(wide(w[1]), wide(x[b][1]), acc[b], 4, 4, 1, sw, 1, sx[b]);
      acc[b] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(wide(w[2]), wide(x[b][2]), acc[b], 4, 4, 2, sw, 2, sx[b]);
      acc[b] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(wide(w[3]), wide(x[b][3]), acc[b], 4, 4, 3, sw, 3, sx[b]);
    }
  }
#pragma unroll
  for (int b = 0; b < NB; ++b) sums[wave][b][lane] = acc[b];
  __syncthreads();
  for (int t = threadIdx.x; t < NB * 64; t += WAVES * 64) {
    const int b = t >> 6, l = t & 63;
    f32x4 v = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int w = 0; w < WAVES; ++w) v += sums[w][b][l];
    const int row = n0 + b * 16 + (l & 15), o = o0 + 4 * (l >> 4);
    if (row >= a.n) continue;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      if (o + j >= a.c_out) continue;
      const float f = finish(v[j], a.bias ? a.bias[o + j] : 0.f, a.relu);
      if (a.out_bf16) ((__bf16*)a.y)[row * a.ld_y + o + j] = (__bf16)f;
      else ((float*)a.y)[row * a.ld_y + o + j] = f;
    }
  }
}

}  // namespace

hipError_t launch_quantize_mx4(const void* x, bool bf16, long long ld_x, int n, int c, uint8_t* q, long long ld_q,
                               uint8_t* scale, long long ld_scale, hipStream_t s) {
  const long long total = (long long)n * ((c + 31) / 32 * 4LL);
  const dim3 grid((unsigned)std::min<long long>((total + 255) / 256, 1 << 22));
  if (bf16) launch(quantize_mx4_kernel<true>, grid, dim3(256), s, x, ld_x, n, c, q, ld_q, scale, ld_scale);
  else launch(quantize_mx4_kernel<false>, grid, dim3(256), s, x, ld_x, n, c, q, ld_q, scale, ld_scale);
  return hipGetLastError();
}

long long fc_mx4_workspace_bytes(int, int, int) { return 0; }

hipError_t launch_fc_mx4(const FcMx4Args& args, hipStream_t s) {
  // 2^15 times 16 rows a launch at most (a grid's second axis)
  for (long long n0 = 0; n0 < args.n; n0 += 1 << 19) {
    FcMx4Args a = args;
    a.n = (int)std::min<long long>(args.n - n0, 1 << 19);
    a.x += n0 * a.ld_x;
    a.xs += n0 * a.ld_xs;
    a.y = (char*)a.y + n0 * a.ld_y * (a.out_bf16 ? 2 : 4);
    const unsigned cols = (a.c_out + 15) / 16;
    if (a.n <= 16) launch(fc_mx4_rows_kernel<1, 4>, dim3(cols, 1), dim3(256), s, a);
    else launch(fc_mx4_rows_kernel<2, 4>, dim3(cols, (a.n + 31) / 32), dim3(256), s, a);
    const hipError_t st = hipGetLastError();
    if (st != hipSuccess) return st;
  }
  return hipSuccess;
}

}  // namespace rafiki
