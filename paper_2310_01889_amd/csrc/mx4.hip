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

// Eight codes (one dword) as a bf16 operand, exactly.  A scale byte of 255 makes an infinite scale,
// under which the conversion gives NaN for every code (checked on the device).
__device__ __forceinline__ bf16x8 from_e2m1(uint32_t codes, float scale) {
  typedef __bf16 bf16x2_t __attribute__((ext_vector_type(2)));
  const bf16x2_t a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 0);
  const bf16x2_t b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 1);
  const bf16x2_t c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 2);
  const bf16x2_t d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 3);
  return bf16x8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}

// A workgroup of 8 waves takes a block of 16 outputs for NT tiles of 16 rows; its waves take turns
// of U weight blocks along the inputs, their sums are added in wave order through LDS.  Every
// weight is read once a launch and becomes a bf16 operand once for all NT tiles; x comes from L2.
constexpr int kMxWaves = 8;

template <int NT, int U>
__global__ __launch_bounds__(64 * kMxWaves) void mx4_linear_kernel(const MxArgs a) {
  __shared__ f32x4 s_sum[kMxWaves][NT][64];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, l16 = lane & 15, c = lane >> 4;
  const int i = blockIdx.x, t0 = blockIdx.y * NT * 16;
  const uint8_t* w4 = a.w4 + (long long)i * a.kb * 1024 + lane * 16;
  const uint8_t* sc = a.scales + (long long)i * a.kb * 64 + l16 * 4;
  f32x4 acc[NT];
#pragma unroll
  for (int n = 0; n < NT; ++n) acc[n] = f32x4{0.f, 0.f, 0.f, 0.f};
  for (int b0 = wave * U; b0 < a.kb; b0 += kMxWaves * U) {
    u32x4 w[U];
    uint32_t e[U];
    bf16x8 x[U][4][NT];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int b = min(b0 + u, a.kb - 1);
      w[u] = *(const u32x4*)(w4 + (long long)b * 1024);
      e[u] = *(const uint32_t*)(sc + (long long)b * 64);
    }
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int s = 0; s < 4; ++s)
#pragma unroll
        for (int n = 0; n < NT; ++n) {
          // (places past the ends read others' elements: for rows that are not stored, or unused)
          const int k = min(128 * (b0 + u) + 32 * s, a.K - 32) + 8 * c, t = min(t0 + 16 * n + l16, a.T - 1);
          x[u][s][n] = *(const bf16x8*)(a.x + (long long)t * a.K + k);
        }
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int s = 0; s < 4; ++s) {
        if (128 * (b0 + u) + 32 * s >= a.K) break;
        const bf16x8 wv = from_e2m1(w[u][s], __uint_as_float((e[u] >> (8 * s) & 255u) << 23));
#pragma unroll
        for (int n = 0; n < NT; ++n) acc[n] = mfma16(wv, x[u][s][n], acc[n]);
      }
  }
#pragma unroll
  for (int n = 0; n < NT; ++n) s_sum[wave][n][lane] = acc[n];
  __syncthreads();
  if (wave >= NT) return;
  f32x4 y = s_sum[0][wave][lane];
#pragma unroll
  for (int v = 1; v < kMxWaves; ++v) y += s_sum[v][wave][lane];
  const int t = t0 + 16 * wave + l16, n0 = 16 * i + 4 * c;
  if (t >= a.T) return;
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const long long at = (long long)t * a.N + n0 + j;
    if (n0 + j < a.N) a.y[at] = (bf16)(y[j] + (a.residual ? (float)a.residual[at] : 0.f));
  }
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
  const int tiles = (T + 15) / 16;
  auto run = [&](auto kernel, int nt) {
    hipLaunchKernelGGL(kernel, dim3((d_out + 15) / 16, (tiles + nt - 1) / nt), dim3(64 * kMxWaves), 0, stream, a);
  };
  if (tiles == 1) run(mx4_linear_kernel<1, 4>, 1);
  else if (tiles == 2) run(mx4_linear_kernel<2, 2>, 2);
  else if (tiles == 3) run(mx4_linear_kernel<3, 2>, 3);
  else run(mx4_linear_kernel<4, 2>, 4);
  RA_HIP(hipGetLastError());
  return RA_OK;
}
