// Attention of the newest tokens of many requests over a paged key/value cache.
//
// o = softmax(q K^T / sqrt(D)) V over the keys of each request, read page by page through its
// row of the block table; the new tokens are the last of the cache and see keys up to their own.
#include <math.h>

#include "ra_common.h"
#include "ra_paged.h"
#include "ra_runtime.h"
#include "ringattn.h"

namespace ra {
namespace {

constexpr int kMaxNew = 32;  // new tokens a request

struct PagedArgs {
  const bf16* q;  // [T, Hq, D]
  const void *k, *v;
  const uint8_t *ks, *vs;
  const int *table, *lens, *cu;
  bf16* o;     // [T, Hq, D]
  float* lse;  // [T, Hq]
  int T, R, Hq, Hkv, n_pages, page_shift, max_pages, max_new;
  float scale;
};

__device__ __forceinline__ float wave_sum(float v) {
#pragma unroll
  for (int off = 32; off >= 1; off >>= 1) v += __shfl_xor(v, off);
  return v;
}

// A workgroup of four waves a (request, new token, query head); a wave takes every fourth key,
// its lanes the head dims, with the online softmax recurrence; the four states are joined in LDS.
template <int D, bool E4M3>
__global__ __launch_bounds__(256) void paged_simple_kernel(const PagedArgs a) {
  constexpr int E = D / 64;
  __shared__ float s_part[4][D + 2];
  const int hq = blockIdx.x % a.Hq, t = blockIdx.x / a.Hq % a.max_new, r = blockIdx.x / a.Hq / a.max_new;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int row0 = a.cu ? min(max(a.cu[r], 0), a.T) : r, row1 = a.cu ? min(max(a.cu[r + 1], row0), a.T) : r + 1;
  if (t >= row1 - row0) return;
  const int h = hq / (a.Hq / a.Hkv);
  const int len = a.lens[r];
  const long long cap = (long long)a.max_pages << a.page_shift;
  const int end = (int)max(0ll, min(min((long long)len, cap), (long long)len - (row1 - row0) + t + 1));
  float qv[E], acc[E];
  const long long qrow = (long long)(row0 + t) * a.Hq + hq;
#pragma unroll
  for (int e = 0; e < E; ++e) {
    qv[e] = (float)a.q[qrow * D + lane * E + e] * a.scale;
    acc[e] = 0.f;
  }
  float m = -INFINITY, l = 0.f;
  for (int p = wave; p < end; p += 4) {
    const int page = a.table[(long long)r * a.max_pages + (p >> a.page_shift)];
    if (page < 0 || page >= a.n_pages) continue;
    const long long row = (((long long)page << a.page_shift) + (p & ((1 << a.page_shift) - 1))) * a.Hkv + h;
    float kv[E], vv[E];
#pragma unroll
    for (int e = 0; e < E; ++e) {
      const long long i = row * D + lane * E + e;
      if constexpr (E4M3) {
        kv[e] = __builtin_amdgcn_cvt_f32_fp8(((const uint8_t*)a.k)[i], 0) * ldexpf(1.f, a.ks[row] - 127);
        vv[e] = __builtin_amdgcn_cvt_f32_fp8(((const uint8_t*)a.v)[i], 0) * ldexpf(1.f, a.vs[row] - 127);
      } else {
        kv[e] = (float)((const bf16*)a.k)[i];
        vv[e] = (float)((const bf16*)a.v)[i];
      }
    }
    float s = 0.f;
#pragma unroll
    for (int e = 0; e < E; ++e) s = fmaf(qv[e], kv[e], s);
    s = wave_sum(s);
    if (s == -INFINITY) continue;  // weighs nothing
    const float mn = s == s ? fmaxf(m, s) : INFINITY;  // a NaN makes everything after it NaN
    const float alpha = m == -INFINITY ? 0.f : expf(m - mn), w = expf(s - mn);
    l = l * alpha + w;
#pragma unroll
    for (int e = 0; e < E; ++e) acc[e] = fmaf(w, vv[e], acc[e] * alpha);
    m = mn;
  }
#pragma unroll
  for (int e = 0; e < E; ++e) s_part[wave][lane * E + e] = acc[e];
  if (lane == 0) {
    s_part[wave][D] = m;
    s_part[wave][D + 1] = l;
  }
  __syncthreads();
  if (wave != 0) return;
  float mt = -INFINITY, lt = 0.f, ot[E] = {};
  for (int w = 0; w < 4; ++w) mt = fmaxf(mt, s_part[w][D]);
  for (int w = 0; w < 4; ++w) {
    const float f = s_part[w][D] == -INFINITY ? 0.f : expf(s_part[w][D] - mt);
    lt = fmaf(s_part[w][D + 1], f, lt);
#pragma unroll
    for (int e = 0; e < E; ++e) ot[e] += f == 0.f ? 0.f : s_part[w][lane * E + e] * f;
  }
#pragma unroll
  for (int e = 0; e < E; ++e) a.o[qrow * D + lane * E + e] = (bf16)(mt == -INFINITY ? 0.f : ot[e] / lt);
  if (lane == 0) a.lse[qrow] = mt == -INFINITY ? -INFINITY : mt + logf(lt);
}

}  // namespace
}  // namespace ra

using namespace ra;

static int paged_check_heads(int R, int Hq, int Hkv, int D, int max_new) {
  if (R <= 0 || Hq <= 0 || Hkv <= 0 || D <= 0 || max_new <= 0)
    return set_err(RA_EINVAL, "sizes must be positive (R=%d Hq=%d Hkv=%d D=%d max_new=%d)", R, Hq, Hkv, D, max_new);
  if (D != 64 && D != 128) return set_err(RA_EUNSUPPORTED, "head dim D=%d not supported (64 or 128)", D);
  if (max_new > kMaxNew) return set_err(RA_EUNSUPPORTED, "max_new=%d exceeds %d new tokens", max_new, kMaxNew);
  if (Hq % Hkv) return set_err(RA_EUNSUPPORTED, "Hq=%d is not a multiple of Hkv=%d", Hq, Hkv);
  if (Hq > kMaxHeads) return set_err(RA_EUNSUPPORTED, "Hq=%d exceeds %d heads", Hq, kMaxHeads);
  if (R > kMaxRequests) return set_err(RA_EUNSUPPORTED, "R=%d exceeds %d requests", R, kMaxRequests);
  return RA_OK;
}

static int paged_check(const void* q, const void* k_pages, const void* v_pages, const unsigned char* k_scales,
                       const unsigned char* v_scales, const int* block_table, const int* lens, const int* cu_rows,
                       const void* o, const float* lse, int T, int R, int Hq, int Hkv, int D, int n_pages,
                       int page_size, int max_pages, int max_new, int kv_type) {
  if (!q || !k_pages || !v_pages || !block_table || !lens || !o || !lse)
    return set_err(RA_EINVAL, "null pointer argument");
  if (int e = check_aligned({q, k_pages, v_pages, o}, {block_table, lens, cu_rows, lse})) return e;
  if (int e = check_kv(kv_type, k_scales, v_scales)) return e;
  if (T <= 0 || max_pages <= 0)
    return set_err(RA_EINVAL, "sizes must be positive (T=%d max_pages=%d)", T, max_pages);
  if (int e = paged_check_heads(R, Hq, Hkv, D, max_new)) return e;
  if (int e = check_pages(page_size, n_pages, Hkv, D)) return e;
  if (!cu_rows && (T < R || max_new != 1))
    return set_err(RA_EINVAL, "without cu_rows row r is request r's one new token (T=%d R=%d max_new=%d)", T, R,
                   max_new);
  if ((long long)max_pages * page_size >= (1ll << 30))
    return set_err(RA_EUNSUPPORTED, "max_pages*page_size = %lld tokens of a request exceeds 2^30-1",
                   (long long)max_pages * page_size);
  return RA_OK;
}

extern "C" int paged_attn_workspace(int R, int Hq, int Hkv, int D, int max_new, size_t* bytes) {
  g_err.clear();
  if (!bytes) return set_err(RA_EINVAL, "null pointer argument");
  if (int e = paged_check_heads(R, Hq, Hkv, D, max_new)) return e;
  *bytes = 0;
  return RA_OK;
}

extern "C" int paged_attn_decode(const void* q, const void* k_pages, const void* v_pages,
                                 const unsigned char* k_scales, const unsigned char* v_scales, const int* block_table,
                                 const int* lens, const int* cu_rows, void* o, float* lse, void* workspace,
                                 size_t workspace_bytes, int T, int R, int Hq, int Hkv, int D, int n_pages,
                                 int page_size, int max_pages, int max_new, int kv_type, hipStream_t stream) {
  g_err.clear();
  int rc = paged_check(q, k_pages, v_pages, k_scales, v_scales, block_table, lens, cu_rows, o, lse, T, R, Hq, Hkv, D,
                       n_pages, page_size, max_pages, max_new, kv_type);
  if (rc) return rc;
  if (int e = check_aligned({workspace})) return e;
  PagedArgs a{(const bf16*)q, k_pages, v_pages, k_scales, v_scales, block_table, lens, cu_rows, (bf16*)o, lse, T, R,
              Hq, Hkv, n_pages, 0, max_pages, max_new, 1.f / sqrtf((float)D)};
  while ((1 << a.page_shift) < page_size) ++a.page_shift;
  auto* kern = D == 128 ? (k_scales ? paged_simple_kernel<128, true> : paged_simple_kernel<128, false>)
                        : (k_scales ? paged_simple_kernel<64, true> : paged_simple_kernel<64, false>);
  RA_HIP(timed_launch(RA_KERNEL_DECODE, stream, [&] {
    hipLaunchKernelGGL(kern, dim3((unsigned)R * max_new * Hq), dim3(256), 0, stream, a);
    return hipGetLastError();
  }));
  return RA_OK;
}
