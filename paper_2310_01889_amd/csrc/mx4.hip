// Products of a few rows with weights in 4 bits (MX format: e2m1 elements, one power-of-two scale
// for every 32 inputs of an output), and the packing of bf16 weights into them.
//
// y [T, d_out] = x [T, d_in] W (+ residual).  The weights lie in blocks of 16 outputs x 128
// inputs, 1 KB of codes each: lane l of a wave loads 16 bytes, output l % 16, whose bytes
// 4s .. 4s + 3 are the 8 inputs 32 s + 8 (l / 16) ..., the A operand of one 16x16x32 product.
#include <math.h>

#include "ra_common.h"
#include "ra_runtime.h"
#include "ringattn.h"

namespace ra {
namespace {

constexpr int kMxMaxT = 512;  // rows of one call

// ---- packing -------------------------------------------------------------------------------
// A thread a (group of 32 inputs, output); consecutive threads take consecutive outputs.  Scale:
// the smallest power of two with which every element of the group is at most 6 in magnitude;
// codes rounded to nearest, ties to the even code.
__global__ __launch_bounds__(256) void mx4_pack_kernel(const bf16* w, uint8_t* w4, uint8_t* scales, int K, int N,
                                                       int kb) {
  const int n = blockIdx.x * 256 + threadIdx.x, g = blockIdx.y;
  if (n >= (N + 15) / 16 * 16) return;
  const int k0 = 32 * g;
  float x[32];
  float top = 0.f;
  bool finite = true;
#pragma unroll
  for (int j = 0; j < 32; ++j) {
    x[j] = n < N && k0 + j < K ? (float)w[(long long)(k0 + j) * N + n] : 0.f;
    top = fmaxf(top, fabsf(x[j]));
    finite &= fabsf(x[j]) < INFINITY;
  }
  // 6 = 1.5 * 2^2: the exponent less 2, one more where the mantissa is past 1.5
  const uint32_t mag = __float_as_uint(top);
  int e2 = (int)(mag >> 23) - 127 - 2 + ((mag & 0x7fffffu) > 0x400000u);
  e2 = mag == 0 || !finite ? 0 : max(e2, -126);
  const float inv = ldexpf(1.f, -e2);
  const long long block = (long long)(n / 16) * kb + g / 4;
#pragma unroll
  for (int c = 0; c < 4; ++c) {
    uint32_t word = 0;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const float v = x[8 * c + j] * inv, m = fabsf(v);
      uint32_t code = (m > 0.25f) + (m >= 0.75f) + (m > 1.25f) + (m >= 1.75f) + (m > 2.5f) + (m >= 3.5f) + (m > 5.f);
      if (v < 0.f && code) code |= 8;
      word |= code << (4 * j);
    }
    *(uint32_t*)(w4 + (block * 64 + c * 16 + n % 16) * 16 + 4 * (g % 4)) = word;
  }
  scales[(block * 16 + n % 16) * 4 + g % 4] = finite ? (uint8_t)(e2 + 127) : 255;
}

// ---- product -------------------------------------------------------------------------------
struct MxArgs {
  const bf16* x;
  const uint8_t *w4, *scales;
  const bf16* residual;
  bf16* y;
  int T, K, N, kb;
};

__device__ __forceinline__ float mx_scale(uint8_t b) { return b == 255 ? NAN : ldexpf(1.f, (int)b - 127); }
__device__ __forceinline__ float e2m1(uint32_t c) {
  const uint32_t m = c & 7;
  const float v = m < 2 ? 0.5f * m : (1.f + 0.5f * (m & 1)) * (float)(1u << (m >> 1)) * 0.5f;
  return c & 8 ? -v : v;
}

// A workgroup a block of 16 outputs and a row: 16 threads an output, each a share of the groups.
__global__ __launch_bounds__(256) void mx4_simple_kernel(const MxArgs a) {
  __shared__ float s_sum[16][17];
  const int i = blockIdx.x, t = blockIdx.y, r = threadIdx.x % 16, part = threadIdx.x / 16;
  float acc = 0.f;
  for (int g = part; g < a.K / 32; g += 16) {
    const long long block = (long long)i * a.kb + g / 4;
    const float s = mx_scale(a.scales[(block * 16 + r) * 4 + g % 4]);
    for (int c = 0; c < 4; ++c) {
      const uint32_t word = *(const uint32_t*)(a.w4 + (block * 64 + c * 16 + r) * 16 + 4 * (g % 4));
      const bf16* xr = a.x + (long long)t * a.K + 32 * g + 8 * c;
      for (int j = 0; j < 8; ++j) acc = fmaf((float)xr[j], e2m1(word >> (4 * j) & 15) * s, acc);
    }
  }
  s_sum[part][r] = acc;
  __syncthreads();
  const int n = 16 * i + r;
  if (part != 0 || n >= a.N) return;
  for (int p = 1; p < 16; ++p) acc += s_sum[p][r];
  const long long at = (long long)t * a.N + n;
  a.y[at] = (bf16)(acc + (a.residual ? (float)a.residual[at] : 0.f));
}

int check_mx(int K, int N) {
  if (K <= 0 || N <= 0) return set_err(RA_EINVAL, "sizes must be positive (d_in=%d d_out=%d)", K, N);
  if (K % 32) return set_err(RA_EUNSUPPORTED, "d_in=%d must be a multiple of 32", K);
  if ((long long)K * N >= (1ll << 31)) return set_err(RA_EUNSUPPORTED, "d_in*d_out exceeds 2^31-1 elements");
  return RA_OK;
}

}  // namespace
}  // namespace ra

using namespace ra;

extern "C" int mx4_pack(const void* w, void* w4, unsigned char* scales, int d_in, int d_out, hipStream_t stream) {
  g_err.clear();
  if (!w || !w4 || !scales) return set_err(RA_EINVAL, "null pointer argument");
  if (int e = check_aligned({w, w4}, {scales})) return e;
  if (int e = check_mx(d_in, d_out)) return e;
  const int kb = (d_in + 127) / 128;
  hipLaunchKernelGGL(mx4_pack_kernel, dim3((d_out + 255) / 256, 4 * kb), dim3(256), 0, stream, (const bf16*)w,
                     (uint8_t*)w4, scales, d_in, d_out, kb);
  RA_HIP(hipGetLastError());
  return RA_OK;
}

extern "C" int mx4_linear(const void* x, const void* w4, const unsigned char* scales, const void* residual, void* y,
                          int T, int d_in, int d_out, hipStream_t stream) {
  g_err.clear();
  if (!x || !w4 || !scales || !y) return set_err(RA_EINVAL, "null pointer argument");
  if (int e = check_aligned({x, w4, residual, y}, {scales})) return e;
  if (T <= 0) return set_err(RA_EINVAL, "sizes must be positive (T=%d)", T);
  if (int e = check_mx(d_in, d_out)) return e;
  if (T > kMxMaxT) return set_err(RA_EUNSUPPORTED, "T=%d exceeds %d rows", T, kMxMaxT);
  MxArgs a{(const bf16*)x, (const uint8_t*)w4, scales, (const bf16*)residual, (bf16*)y, T, d_in, d_out,
           (d_in + 127) / 128};
  hipLaunchKernelGGL(mx4_simple_kernel, dim3((d_out + 15) / 16, T), dim3(256), 0, stream, a);
  RA_HIP(hipGetLastError());
  return RA_OK;
}
