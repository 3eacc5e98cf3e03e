// Products of a few rows with weights in 4 bits (MX format: e2m1 elements, one power-of-two scale
// for every 32 inputs of an output), and the packing of bf16 weights into them.
//
// y [T, d_out] = x [T, d_in] W (+ residual).  The weights lie in blocks of 16 outputs x 128
// inputs, 1 KB of codes each: lane l of a wave loads 16 bytes, output l % 16, whose bytes
// 4s .. 4s + 3 are the 8 inputs 32 s + 8 (l / 16) ..., the A operand of one 16x16x32 product.
#include <math.h>

#include "ra_common.h"
#include "ra_dma.h"
#include "ra_runtime.h"
#include "ringattn.h"

namespace ra {
namespace {

constexpr int kMxMaxT = 512;  // rows of one call

// ---- packing -------------------------------------------------------------------------------
// A thread a (group of 32 inputs, output); consecutive threads take consecutive outputs, blockIdx.x
// counts 256 of them and the groups (of whole blocks) together.  Scale:
// the smallest power of two with which every element of the group is at most 6 in magnitude;
// codes rounded to nearest, ties to the even code.
__global__ __launch_bounds__(256) void mx4_pack_kernel(const bf16* w, uint8_t* w4, uint8_t* scales, int K, int N,
                                                       int kb) {
  const int g = blockIdx.x % (4 * kb), n = blockIdx.x / (4 * kb) * 256 + threadIdx.x;
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

// A workgroup of WV waves takes NB blocks of 16 outputs for NT tiles of 16 rows; its waves take
// turns along the inputs, 128 at a time, and their sums are added in wave order through LDS.
// Every weight is read once for NT tiles, straight from memory into the lane that needs it, and
// becomes a bf16 operand once.  The rows' 128 inputs go through a slab of LDS of the wave's own:
// an operand's neighbouring lanes are neighbouring rows, and a load of 64 lanes from 16 rows
// takes the address unit four times as long as the slab's loads of whole 256-byte pieces (48 x
// 11008 x 4096: 33 us without the slab, 16 with it; 7 x 4096 x 11008: 9 and 7).  Workgroups start
// at different inputs: the rows' pieces at one place lie in few channels of the L2 where the row
// length is a multiple of 4 KB (32 x 4096 x 4096: 7.6 us without, 6.7).
// Bound by latency for few weights; by the weights' bytes and, for many rows, by x, which every
// workgroup reads whole from L2.
template <int NT, int NB, int WV>
__global__ __launch_bounds__(64 * WV) void mx4_linear_kernel(const MxArgs a) {
  constexpr int SLAB = NT * 4096, SUMS = NT * NB * 1024;
  __shared__ __attribute__((aligned(1024))) uint8_t s_mem[WV][SLAB > SUMS ? SLAB : SUMS];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int l16 = lane & 15, c = lane >> 4;
  const int nb = (a.N + 15) / 16, i0 = blockIdx.x * NB, t0 = blockIdx.y * NT * 16;
  const int rows = min(NT * 16, a.T - t0);
  uint8_t* slab = s_mem[wave];
  const int xoff = l16 * 256 + 16 * (c ^ swz<128>(l16));
  const int start = (int)(blockIdx.x * 7u % (unsigned)a.kb);
  const uint8_t *w4[NB], *sc[NB];
#pragma unroll
  for (int j = 0; j < NB; ++j) {
    const int i = min(i0 + j, nb - 1);  // (past the end: computed, not stored)
    w4[j] = a.w4 + (long long)i * a.kb * 1024 + lane * 16;
    sc[j] = a.scales + (long long)i * a.kb * 64 + l16 * 4;
  }
  f32x4 acc[NB][NT];
#pragma unroll
  for (int j = 0; j < NB; ++j)
#pragma unroll
    for (int n = 0; n < NT; ++n) acc[j][n] = f32x4{0.f, 0.f, 0.f, 0.f};
  for (int at = wave; at < a.kb; at += WV) {
    const int b = at + start < a.kb ? at + start : at + start - a.kb;
#pragma unroll
    for (int j = 0; j < NT * 4; ++j) {
      if (4 * j >= rows) break;
      // four rows a load; rows and inputs past the ends read others, which nothing uses
      const int r = 4 * j + c, k = min(128 * b + 8 * (l16 ^ swz<128>(r)), a.K - 8);
      dma_lds16_at(a.x + (long long)min(t0 + r, a.T - 1) * a.K + k, lds_addr(slab) + j * 1024);
    }
    u32x4 w[NB];
    uint32_t e[NB];
#pragma unroll
    for (int j = 0; j < NB; ++j) {
      w[j] = *(const u32x4*)(w4[j] + (long long)b * 1024);
      e[j] = *(const uint32_t*)(sc[j] + (long long)b * 64);
    }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    auto product = [&](int s) __attribute__((always_inline)) {  // of 32 inputs
      bf16x8 x[NT];
#pragma unroll
      for (int n = 0; n < NT; ++n) x[n] = *(const bf16x8*)(slab + n * 4096 + (xoff ^ (64 * s)));
#pragma unroll
      for (int j = 0; j < NB; ++j) {
        const bf16x8 wv = from_e2m1(w[j][s], __uint_as_float((e[j] >> (8 * s) & 255u) << 23));
#pragma unroll
        for (int n = 0; n < NT; ++n) acc[j][n] = mfma16(wv, x[n], acc[j][n]);
      }
    };
    if (128 * (b + 1) <= a.K) {  // (branches between the steps would keep their reads apart)
#pragma unroll
      for (int s = 0; s < 4; ++s) {
        if (NT * NB >= 16 && s == 2) __builtin_amdgcn_sched_barrier(0);  // not all reads at once: registers
        product(s);
      }
    } else {
#pragma unroll
      for (int s = 0; s < 3; ++s)
        if (128 * b + 32 * s < a.K) product(s);
    }
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");  // the slab has been read
  }
#pragma unroll
  for (int j = 0; j < NB; ++j)
#pragma unroll
    for (int n = 0; n < NT; ++n) ((f32x4*)slab)[(j * NT + n) * 64 + lane] = acc[j][n];
  __syncthreads();
  for (int q = wave; q < NT * NB; q += WV) {
    f32x4 y = ((const f32x4*)s_mem[0])[q * 64 + lane];
#pragma unroll
    for (int v = 1; v < WV; ++v) y += ((const f32x4*)s_mem[v])[q * 64 + lane];
    const int t = t0 + 16 * (q % NT) + l16, n0 = 16 * (i0 + q / NT) + 4 * c;
    if (t >= a.T) continue;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const long long o = (long long)t * a.N + n0 + j;
      if (n0 + j < a.N) a.y[o] = (bf16)(y[j] + (a.residual ? (float)a.residual[o] : 0.f));
    }
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
  hipLaunchKernelGGL(mx4_pack_kernel, dim3((unsigned)((d_out + 255) / 256) * 4 * kb), dim3(256), 0, stream, (const bf16*)w,
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
  // NT: a pass over the weights for up to 64 rows.  Blocks a workgroup: as many as leave one
  // workgroup a compute unit (of 256), for then x is read least often.  us with one, two, four
  // blocks: 64 x 4096 x 11008 (688 blocks) -, 19.3, 15.4; 20 x 2048 x 6000 (375) 5.9, 5.2, 6.2; 32 x
  // 4096 x 4096 (256) 6.7, 7.3, 8.3.  For one tile x is little: one block, with 16 waves where the
  // blocks are no more than the compute units (1 x 11008 x 4096: 6.4 us, 8 waves 8.3; 7 x 4096 x
  // 11008, 688 blocks: 8.4, 8 waves 6.9).
  const int tiles = (T + 15) / 16, blocks = (d_out + 15) / 16;
  auto run = [&](auto kernel, int nt, int nb, int wv) {
    hipLaunchKernelGGL(kernel, dim3((blocks + nb - 1) / nb, (tiles + nt - 1) / nt), dim3(64 * wv), 0, stream, a);
  };
  const int nb = blocks <= 256 ? 1 : blocks <= 512 ? 2 : 4;
  if (tiles == 1 && nb == 1) run(mx4_linear_kernel<1, 1, 16>, 1, 1, 16);
  else if (tiles == 1) run(mx4_linear_kernel<1, 1, 8>, 1, 1, 8);
  else if (tiles == 2 && nb == 1) run(mx4_linear_kernel<2, 1, 8>, 2, 1, 8);
  else if (tiles == 2 && nb == 2) run(mx4_linear_kernel<2, 2, 8>, 2, 2, 8);
  else if (tiles == 2) run(mx4_linear_kernel<2, 4, 8>, 2, 4, 8);
  else if (tiles == 3 && nb == 1) run(mx4_linear_kernel<3, 1, 8>, 3, 1, 8);
  else if (tiles == 3 && nb == 2) run(mx4_linear_kernel<3, 2, 8>, 3, 2, 8);
  else if (tiles == 3) run(mx4_linear_kernel<3, 4, 8>, 3, 4, 8);
  else if (nb == 1) run(mx4_linear_kernel<4, 1, 8>, 4, 1, 8);
  else if (nb == 2) run(mx4_linear_kernel<4, 2, 8>, 4, 2, 8);
  else run(mx4_linear_kernel<4, 4, 8>, 4, 4, 8);
  RA_HIP(hipGetLastError());
  return RA_OK;
}
