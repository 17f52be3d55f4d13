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

// One workgroup per row: the largest magnitude, then the quotients.
template <bool BF16>
__global__ __launch_bounds__(256) void quantize_kernel(const void* x, long long ld_x, int n, int c, int8_t* q,
                                                       long long ld_q, float* scale) {
  __shared__ float waves[4];
  for (int row = blockIdx.x; row < n; row += gridDim.x) {
    const long long base = row * ld_x;
    float top = 0.f;
    bool bad = false;
    for (int i = threadIdx.x; i < c; i += 256) {
      const float v = fabsf(value<BF16>(x, base + i));
      bad |= !(v < INFINITY);
      top = fmaxf(top, v);
    }
    if (bad) top = INFINITY;
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor(top, o, 64));
    __syncthreads();
    if ((threadIdx.x & 63) == 0) waves[threadIdx.x >> 6] = top;
    __syncthreads();
    top = fmaxf(fmaxf(waves[0], waves[1]), fmaxf(waves[2], waves[3]));
    float s = top / 127.f;
    if (s < 0x1p-126f) s = 0.f;
    const bool zero = s == 0.f || top == INFINITY;
    const float inv = zero ? 0.f : 1.f / s;
    for (int i = threadIdx.x; i < c; i += 256)
      q[row * ld_q + i] = zero ? 0 : (int8_t)nearest_quotient(value<BF16>(x, base + i), s, inv);
    if (threadIdx.x == 0) scale[row] = top == INFINITY ? NAN : s;
  }
}

__device__ __forceinline__ void store_out(const FcI8Args& a, int row, int o, int acc) {
  float v = (float)acc * (a.sx[row] * a.sw[o]);
  if (a.bias) v += a.bias[o];
  if (a.relu && v < 0.f) v = 0.f;                            // NaN stays NaN
  if (a.out_bf16) ((__bf16*)a.y)[row * a.ld_y + o] = (__bf16)v;
  else ((float*)a.y)[row * a.ld_y + o] = v;
}

// 16 bytes of a row from k on; bytes behind c_in are 0.
__device__ __forceinline__ i32x4 chunk16(const int8_t* p, int k, int c_in) {
  i32x4 v = {0, 0, 0, 0};
  if (k >= c_in) return v;
  v = *(const i32x4*)(p + k);
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int left = c_in - (k + 4 * i);                     // valid bytes from this word on
    if (left <= 0) v[i] = 0;
    else if (left < 4) v[i] &= (1 << (8 * left)) - 1;
  }
  return v;
}

// A wave per 16 rows of x by 16 rows of w, fragments straight from memory.  v_mfma_i32_16x16x64_i8:
// lane l holds 16 consecutive k (from 16 (l / 16)) of row l % 16 of either operand, and sums 4 (l / 16) .. + 3
// of the first operand's rows for row l % 16 of the second.
__global__ __launch_bounds__(256) void fc_i8_kernel(FcI8Args a) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int tiles_o = (a.c_out + 63) / 64;
  const int o0 = (int)(blockIdx.x % tiles_o) * 64 + wave * 16;
  const int r0 = (int)(blockIdx.x / tiles_o) * 16;
  if (o0 >= a.c_out) return;
  const int xr = std::min(r0 + (lane & 15), a.n - 1), wr = std::min(o0 + (lane & 15), a.c_out - 1);
  const int8_t* xp = a.x + xr * a.ld_x;
  const int8_t* wp = a.w + wr * a.ld_w;
  i32x4 acc = {0, 0, 0, 0};
  for (int k = 16 * (lane >> 4); k - 16 * (lane >> 4) < a.c_in; k += 64) {
    const i32x4 wv = chunk16(wp, k, a.c_in), xv = chunk16(xp, k, a.c_in);
    acc = __builtin_amdgcn_mfma_i32_16x16x64_i8(wv, xv, acc, 0, 0, 0);
  }
  const int row = r0 + (lane & 15);
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int o = o0 + 4 * (lane >> 4) + i;
    if (row < a.n && o < a.c_out) store_out(a, row, o, acc[i]);
  }
}

}  // namespace

hipError_t launch_quantize(const void* x, bool bf16, long long ld_x, int n, int c, int8_t* q, long long ld_q,
                           float* scale, hipStream_t s) {
  const dim3 grid((unsigned)std::min(n, 1 << 20));
  if (bf16) launch(quantize_kernel<true>, grid, dim3(256), s, x, ld_x, n, c, q, ld_q, scale);
  else launch(quantize_kernel<false>, grid, dim3(256), s, x, ld_x, n, c, q, ld_q, scale);
  return hipGetLastError();
}

long long fc_i8_workspace_bytes(int, int, int) { return 0; }

hipError_t launch_fc_i8(const FcI8Args& a, hipStream_t s) {
  const long long tiles = (long long)((a.c_out + 63) / 64) * ((a.n + 15) / 16);
  if (tiles > (1 << 23)) return hipErrorInvalidValue;
  launch(fc_i8_kernel, dim3((unsigned)tiles), dim3(256), s, a);
  return hipGetLastError();
}

}  // namespace rafiki
