// Products of a few rows with weights in 4 bits (MX format: e2m1 elements, one power-of-two scale
// for every 32 inputs of an output), and the packing of bf16 weights into them.
//
// y [T, d_out] = x [T, d_in] W (+ residual).  The weights lie in blocks of 16 outputs x 128
// inputs, 1 KB of codes each: lane l of a wave loads 16 bytes, output l % 16, whose bytes
// 4s .. 4s + 3 are the 8 inputs 32 s + 8 (l / 16) ..., the A operand of one 16x16x32 product.
#include <limits.h>
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
// codes rounded to nearest, ties to the even code.  Once a weight: 4096 x 11008 57 us (2.0 TB/s read and
// written, 32 loads a thread of a row's length apart; a floor of 20).
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

// A workgroup of WV waves takes NB blocks of 16 outputs for NT tiles of 16 rows (of one tile: for 4 XL
// rows); its waves take turns along the inputs, 128 at a time, and their sums are added in wave order
// through LDS.  Every weight becomes a bf16 operand once.  The rows' 128 inputs go through a slab of
// LDS of the wave's own: an operand's neighbouring lanes are neighbouring rows, and a load of 64 lanes
// from 16 rows takes the address unit four times as long as the slab's loads of whole 256-byte
// pieces (48 x 11008 x 4096: 33 us without the slab, 16 with it; 7 x 4096 x 11008: 9 and 7).
// PIPE: codes and scales go through LDS as well and a wave has two stages, one in flight while the
// other is computed; else weights go straight to registers and other waves hide the loads, eight
// of them where their slabs are large (64 x 4096 x 4096 in 2 x 2 tiles: 6.7 us with two stages, 7.8 with
// one; 24 x 4096 x 11008 in 2 x 4: 11.3 and 10.9).  A wave of one stage waits for its own loads at
// every 128 inputs.
// Workgroups start at different inputs: the rows' pieces at one place lie in few channels of the L2
// where the row length is a multiple of 4 KB (32 x 4096 x 4096: 7.6 us without, 6.7).
// Bound by latency for few weights; by the weights' bytes; for many rows by what the compute units take
// from L2, x being read whole by every column of workgroups: 47 to 55 bytes a ns each with two stages (48 x
// 11008 x 4096 in 2 x 2 0.89 MB in 16.2 us, in 1 x 4 0.73 in 15.5), 29 to 47 with one, where the loads are
// waited for (24 x 4096 x 11008 in 2 x 3 0.30 MB in 10.3, 48 rows in 3 x 3 0.50 in 13.0).
template <int NT, int NB, int WV, bool PIPE, int XL = 4 * NT>
__global__ __launch_bounds__(64 * WV) void mx4_linear_kernel(const MxArgs a) {
  constexpr int SLAB = XL * 1024, STAGE = SLAB + (PIPE ? NB * 1280 : 0), LOADS = XL + 2 * NB;
  constexpr int SUMS = NT * NB * 1024, MEM = PIPE ? 2 * STAGE : STAGE;
  __shared__ __attribute__((aligned(1024))) uint8_t s_mem[WV][MEM > SUMS ? MEM : SUMS];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int l16 = lane & 15, c = lane >> 4;
  const int nb = (a.N + 15) / 16, i0 = blockIdx.x * NB, t0 = blockIdx.y * NT * 16;
  const int rows = min(NT * 16, a.T - t0);
  uint8_t* slab = s_mem[wave];
  const int xr = XL < 4 ? l16 % (4 * XL) : l16;  // (rows past the last are others again; nothing uses them)
  const int xoff = xr * 256 + 16 * (c ^ swz<128>(xr));
  const int start = (int)(blockIdx.x * 7u % (unsigned)a.kb);
  const uint8_t *w4[NB], *sc[NB];
#pragma unroll
  for (int j = 0; j < NB; ++j) {
    const int i = min(i0 + j, nb - 1);  // (past the end: computed, not stored)
    w4[j] = a.w4 + (long long)i * a.kb * 1024 + lane * 16;
    sc[j] = a.scales + (long long)i * a.kb * 64 + l16 * 4;
  }
  auto block_of = [&](int at) { return at + start < a.kb ? at + start : at + start - a.kb; };
  auto load = [&](int at, uint8_t* to) __attribute__((always_inline)) {
    const int b = block_of(at);
    if constexpr (PIPE) {
#pragma unroll
      for (int j = 0; j < NB; ++j) {
        dma_lds16_at(w4[j] + (long long)b * 1024, lds_addr(to) + SLAB + j * 1280);
        dma_lds4_at(sc[j] + (long long)b * 64, lds_addr(to) + SLAB + j * 1280 + 1024);
      }
    }
#pragma unroll
    for (int j = 0; j < XL; ++j) {
      if (!PIPE && 4 * j >= rows) break;  // (PIPE counts its loads)
      // four rows a load; rows and inputs past the ends read others, which nothing uses
      const int r = 4 * j + c, k = min(128 * b + 8 * (l16 ^ swz<128>(r)), a.K - 8);
      dma_lds16_at(a.x + (long long)min(t0 + r, a.T - 1) * a.K + k, lds_addr(to) + j * 1024);
    }
  };
  f32x4 acc[NB][NT];
#pragma unroll
  for (int j = 0; j < NB; ++j)
#pragma unroll
    for (int n = 0; n < NT; ++n) acc[j][n] = f32x4{0.f, 0.f, 0.f, 0.f};
  if (PIPE && wave < a.kb) load(wave, slab);
#pragma unroll 1
  for (int at = wave, st = 0; at < a.kb; at += WV, st ^= 1) {
    const int b = block_of(at);
    uint8_t* here = slab + (PIPE ? st * STAGE : 0);
    u32x4 w[NB];
    uint32_t e[NB];
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");  // what is loaded into has been read
    if constexpr (PIPE) {
      if (at + WV < a.kb) {
        load(at + WV, slab + (st ^ 1) * STAGE);
        asm volatile("s_waitcnt vmcnt(%0)" ::"n"(LOADS) : "memory");  // this stage has landed
      } else {
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
      }
#pragma unroll
      for (int j = 0; j < NB; ++j) {
        w[j] = *(const u32x4*)(here + SLAB + j * 1280 + lane * 16);
        e[j] = *(const uint32_t*)(here + SLAB + j * 1280 + 1024 + lane * 4);
      }
    } else {
      load(at, slab);
#pragma unroll
      for (int j = 0; j < NB; ++j) {
        w[j] = *(const u32x4*)(w4[j] + (long long)b * 1024);
        e[j] = *(const uint32_t*)(sc[j] + (long long)b * 64);
      }
      asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    }
    auto product = [&](int s) __attribute__((always_inline)) {  // of 32 inputs
      bf16x8 x[NT];
#pragma unroll
      for (int n = 0; n < NT; ++n) x[n] = *(const bf16x8*)(here + n * 4096 + (xoff ^ (64 * s)));
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
  }
  asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");  // the slab has been read
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
  // (the packing's grid: fewer than 2^24 workgroups of 256 threads)
  if (K > (1 << 29) - 128) return set_err(RA_EUNSUPPORTED, "d_in=%d exceeds 2^29-128", K);
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
  if (x == y) return set_err(RA_EINVAL, "y must not be x");
  if (T > kMxMaxT) return set_err(RA_EUNSUPPORTED, "T=%d exceeds %d rows", T, kMxMaxT);
  MxArgs a{(const bf16*)x, (const uint8_t*)w4, scales, (const bf16*)residual, (bf16*)y, T, d_in, d_out,
           (d_in + 127) / 128};
  // Tiles NT and blocks NB a workgroup: the pair with which a compute unit (of 256) takes the fewest
  // bytes, counting for every input 8 of x for four rows and 17 a block of weights, twice what
  // they are, for they come from memory and not from L2.  us of a call among others, 512 MB of weights taken
  // in turn so that they come from memory, by pair 1x1, 1x2, 1x4, 2x2, 2x4, 3x4 (a call alone is 5.7):
  //   32 x 4096 x 4096   8.4  6.1  7.7  8.1  -     -        20 x 4096 x 2048   5.9  5.9  7.3  7.1  -  -
  //   48 x 11008 x 4096  22.3 19.3 15.5 16.2 22.0  28.6     48 x 4096 x 11008  28.7 20.9 19.8 19.0 17.1 14.0
  //   96 x 4096 x 11008  48.4 34.9 31.5 28.3 20.5  21.7
  // 4x4 for 64 x 4096 x 11008: 17.4 us, 2x4 18.2.  Three blocks where two need two rounds of the chip and
  // four leave units idle: 7 x 4096 x 11008 7.1 us, 1x4 7.8; 24 x 4096 x 11008 10.3, 2x4 11.2; 48 rows 13.0, 3x4
  // 14.0.  Several tiles of three and more blocks, one stage: eight waves where every workgroup has a compute
  // unit of its own (24 x 4096 x 11008 10.3 us, four waves 15.0), else four, two workgroups a unit (300 x
  // 4096 x 4096 21.1, eight waves 22.7).  1x1 and up to eight rows: 16 waves (1 x 11008 x 4096 6.7 us, eight
  // waves 8.1).
  const int tiles = (T + 15) / 16, blocks = (d_out + 15) / 16;
  const int xl = T <= 4 ? 1 : T <= 8 ? 2 : 4;
  auto groups = [&](int nt, int nb) { return (long long)((blocks + nb - 1) / nb) * ((tiles + nt - 1) / nt); };
  static constexpr int kPairs[][2] = {{4, 4}, {3, 4}, {3, 3}, {2, 4}, {2, 3}, {2, 2}, {1, 4}, {1, 3}, {1, 2}, {1, 1}};
  int nt = 1, nb = 1;
  long long least = LLONG_MAX;
  for (const auto& p : kPairs) {
    if (p[0] > tiles) continue;
    const long long cost = (groups(p[0], p[1]) + 255) / 256 * (8 * (p[0] == 1 ? xl : 4 * p[0]) + 17 * p[1]);
    if (cost < least) least = cost, nt = p[0], nb = p[1];
  }
  const bool wide = groups(nt, nb) <= 256;
  auto run = [&](auto* kernel, int wv) {
    hipLaunchKernelGGL(kernel, dim3((blocks + nb - 1) / nb, (tiles + nt - 1) / nt), dim3(64 * wv), 0, stream, a);
  };
  auto one_tile = [&](auto* four, auto* eight, auto* sixteen) { run(xl == 1 ? four : xl == 2 ? eight : sixteen, 8); };
  if (nt == 1 && nb == 1 && xl == 4) run(mx4_linear_kernel<1, 1, 8, true>, 8);
  else if (nt == 1 && nb == 1)
    run(xl == 1 ? mx4_linear_kernel<1, 1, 16, true, 1> : mx4_linear_kernel<1, 1, 16, true, 2>, 16);
  else if (nt == 1 && nb == 2)
    one_tile(mx4_linear_kernel<1, 2, 8, true, 1>, mx4_linear_kernel<1, 2, 8, true, 2>, mx4_linear_kernel<1, 2, 8, true>);
  else if (nt == 1 && nb == 3)
    one_tile(mx4_linear_kernel<1, 3, 8, true, 1>, mx4_linear_kernel<1, 3, 8, true, 2>, mx4_linear_kernel<1, 3, 8, true>);
  else if (nt == 1)
    one_tile(mx4_linear_kernel<1, 4, 8, true, 1>, mx4_linear_kernel<1, 4, 8, true, 2>, mx4_linear_kernel<1, 4, 8, true>);
  else if (nt == 2 && nb == 2) run(mx4_linear_kernel<2, 2, 7, true>, 7);
  else if (nt == 4) run(mx4_linear_kernel<4, 4, 8, false>, 8);
  else if (wide)
    run(nt == 2 ? (nb == 3 ? mx4_linear_kernel<2, 3, 8, false> : mx4_linear_kernel<2, 4, 8, false>)
                : (nb == 3 ? mx4_linear_kernel<3, 3, 8, false> : mx4_linear_kernel<3, 4, 8, false>), 8);
  else
    run(nt == 2 ? (nb == 3 ? mx4_linear_kernel<2, 3, 4, false> : mx4_linear_kernel<2, 4, 4, false>)
                : (nb == 3 ? mx4_linear_kernel<3, 3, 4, false> : mx4_linear_kernel<3, 4, 4, false>), 4);
  RA_HIP(hipGetLastError());
  return RA_OK;
}
