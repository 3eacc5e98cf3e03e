// A decode step over a paged key/value cache: the plan (pages, slots and positions of the new
// tokens), and the append that rotates q and k and writes keys and values into their pages.
//
// The cache is n_pages pages of page_size tokens; request r owns the pages its row of
// block_table lists, in order, so its token at position p lies in slot
//   block_table[r][p / page_size] * page_size + p % page_size.
// The attention over these pages is in paged_attn.hip.
#include <math.h>

#include "ra_common.h"
#include "ra_paged.h"
#include "ra_runtime.h"
#include "ringattn.h"

namespace ra {
namespace {

// ---- plan ----------------------------------------------------------------------------------
constexpr int kPlanThreads = 256;
constexpr int kPlanRows = 4;  // rows a thread

struct PlanArgs {
  const int *lens, *n_new, *free_pages, *free_head;
  int *table, *cu, *new_lens, *slots, *positions, *counts;
  int R, page_shift, max_pages, n_pages, n_free, T;
  int vector;  // slots and positions on 16-byte boundaries
};

// Exclusive prefix sums of two values over the workgroup's threads, and the sums of all.
struct Scan2 {
  long long a, b, all_a, all_b;
};
__device__ __forceinline__ Scan2 block_scan(long long a, long long b, long long (*s_wave)[2]) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  long long x = a, y = b;
#pragma unroll
  for (int off = 1; off < 64; off <<= 1) {
    const long long u = __shfl_up(x, off), v = __shfl_up(y, off);
    if (lane >= off) x += u, y += v;
  }
  __syncthreads();  // an earlier scan's sums have been read
  if (lane == 63) s_wave[wave][0] = x, s_wave[wave][1] = y;
  __syncthreads();
  Scan2 r{x - a, y - b, 0, 0};
#pragma unroll
  for (int w = 0; w < kPlanThreads / 64; ++w) {
    if (w < wave) r.a += s_wave[w][0], r.b += s_wave[w][1];
    r.all_a += s_wave[w][0], r.all_b += s_wave[w][1];
  }
  return r;
}

// Every workgroup forms the prefix sums of all requests' rows and pages (R is small and the
// lengths stay in L2), then fills its share of the rows: one launch, no order between workgroups.
// A new page's id is free_pages[head + its number in request order], so nothing here depends on
// what another workgroup writes; its table entry is written by the row that opens it (a page is
// only taken for a token).  Bound by latency: a handful of dependent loads and barriers (8 requests
// of one token 4.5 us; 512 of up to 1024 tokens 6.1, 7.0 with a row's loads after the last row's).
__global__ __launch_bounds__(kPlanThreads) void paged_plan_kernel(const PlanArgs a) {
  extern __shared__ int s_req[];
  int* s_cu = s_req;                   // [R + 1] first row of each request
  int* s_page = s_req + a.R + 1;       // [R] number of its first new page (at most n_free)
  int* s_len = s_page + a.R;           // [R] tokens it has in the cache
  __shared__ long long s_wave[kPlanThreads / 64][2];
  const int tid = threadIdx.x;
  const int per = (a.R + kPlanThreads - 1) / kPlanThreads;
  const int r0 = min(a.R, tid * per), r1 = min(a.R, r0 + per);
  const int P = 1 << a.page_shift;
  const long long cap = (long long)a.max_pages << a.page_shift;
  int flags = 0;
  const int head_in = a.free_head ? *a.free_head : 0;

  auto held = [&](long long tokens) { return (int)((min(tokens, cap) + P - 1) >> a.page_shift); };
  long long rows_sum = 0, page_sum = 0;
#pragma unroll 4
  for (int r = r0; r < r1; ++r) {
    const int n = a.n_new[r], len = a.lens[r];
    if (n < 0 || len < 0) flags |= RA_PLAN_BAD_INPUT;
    s_cu[r] = max(n, 0);  // its number of rows, for now
    s_len[r] = max(len, 0);
    rows_sum += max(n, 0);
    page_sum += held((long long)max(len, 0) + max(n, 0)) - held(max(len, 0));
    if ((long long)max(len, 0) + max(n, 0) > cap) flags |= RA_PLAN_CAPACITY;
  }
  Scan2 at = block_scan(rows_sum, page_sum, s_wave);
  const bool clipped = at.all_a > a.T;
  if (clipped) {  // a request takes no more rows than T holds, and pages for those alone
    flags = RA_PLAN_ROWS | (flags & RA_PLAN_BAD_INPUT);
    long long row = at.a;
    page_sum = 0;
    for (int r = r0; r < r1; ++r) {
      const int n = (int)min((long long)s_cu[r], max(0ll, a.T - row));
      row += s_cu[r];
      s_cu[r] = n;
      const long long before = s_len[r], after = before + n;
      page_sum += held(after) - held(before);
      if (after > cap) flags |= RA_PLAN_CAPACITY;
    }
    const long long first = min(at.a, (long long)a.T);
    at = block_scan(0, page_sum, s_wave);
    at.a = first;
    at.all_a = a.T;
  }
  long long row = at.a, page = at.b;
  for (int r = r0; r < r1; ++r) {
    const int n = s_cu[r];
    s_cu[r] = (int)row;
    s_page[r] = (int)min(page, (long long)a.n_free);
    row += n;
    page += held((long long)s_len[r] + n) - held(s_len[r]);
  }
  const int rows = (int)at.all_a;
  if (tid == 0) s_cu[a.R] = rows;
  if (head_in < 0) flags |= RA_PLAN_BAD_INPUT;
  const int head = min(max(head_in, 0), a.n_free);
  const long long left = a.n_free - head;
  if (at.all_b > left) flags |= RA_PLAN_PAGES;
  __syncthreads();

  // this workgroup's share of the requests' offsets and lengths
  for (int r = blockIdx.x * kPlanThreads + tid; r < a.R; r += gridDim.x * kPlanThreads) {
    a.cu[r] = s_cu[r];
    a.new_lens[r] = (int)min((long long)s_len[r] + s_cu[r + 1] - s_cu[r], 0x7fffffffll);
  }

  // slots and positions of its rows, and the entries of the pages that they open: four rows a thread,
  // their loads in flight together
  const uint32_t i0 = (blockIdx.x * (uint32_t)kPlanThreads + tid) * kPlanRows;
  if (i0 < (uint32_t)a.T) {
    int r = 0;  // the last request that starts at or before the row
    for (int step = 1 << (31 - __clz(a.R)); step > 0; step >>= 1)
      if (r + step < a.R && (uint32_t)s_cu[r + step] <= i0) r += step;
    int slot[kPlanRows], pos[kPlanRows], in_page[kPlanRows], *entry[kPlanRows];  // entry: of a page that the row opens
#pragma unroll
    for (int e = 0; e < kPlanRows; ++e) {
      const uint32_t i = i0 + e;
      const int* from = nullptr;
      pos[e] = -1;
      in_page[e] = 0;
      entry[e] = nullptr;
      if (i < (uint32_t)rows) {
        while ((uint32_t)s_cu[r + 1] <= i) ++r;
        const long long before = s_len[r], p = before + i - s_cu[r];
        pos[e] = (int)min(p, 0x7fffffffll);
        in_page[e] = (int)(p & (P - 1));
        if (p < cap) {
          const int j = (int)(p >> a.page_shift), h0 = held(before);
          int* own = a.table + (long long)r * a.max_pages + j;
          const long long k = (long long)head + s_page[r] + (j - h0);
          if (j < h0) from = own;
          else if (k < a.n_free) from = a.free_pages + k;
          if (j >= h0 && in_page[e] == 0) entry[e] = own;
        }
      }
      slot[e] = from ? *from : -1;  // the page's id
    }
#pragma unroll
    for (int e = 0; e < kPlanRows; ++e) {
      const bool there = slot[e] >= 0 && slot[e] < a.n_pages;
      if (entry[e]) *entry[e] = there ? slot[e] : -1;
      slot[e] = there ? (slot[e] << a.page_shift) + in_page[e] : -1;
    }
    typedef int i32x4 __attribute__((ext_vector_type(4)));
    if (a.vector && i0 + kPlanRows <= (uint32_t)a.T) {
      *(i32x4*)(a.slots + i0) = i32x4{slot[0], slot[1], slot[2], slot[3]};
      *(i32x4*)(a.positions + i0) = i32x4{pos[0], pos[1], pos[2], pos[3]};
    } else {
#pragma unroll
      for (int e = 0; e < kPlanRows; ++e) {
        if (i0 + e >= (uint32_t)a.T) break;
        a.slots[i0 + e] = slot[e];
        a.positions[i0 + e] = pos[e];
      }
    }
  }

  if (blockIdx.x == 0) {
    __shared__ int s_flags[kPlanThreads / 64];
#pragma unroll
    for (int off = 32; off >= 1; off >>= 1) flags |= __shfl_xor(flags, off);
    if ((tid & 63) == 0) s_flags[tid >> 6] = flags;
    __syncthreads();
    if (tid == 0) {
      for (int w = 1; w < kPlanThreads / 64; ++w) flags |= s_flags[w];
      const int took = (int)min(at.all_b, left);
      a.cu[a.R] = rows;
      a.counts[0] = rows;
      a.counts[1] = took;
      a.counts[2] = head + took;
      a.counts[3] = flags;
    }
  }
}

// ---- append --------------------------------------------------------------------------------
constexpr double kRopeBase = 10000.0;
constexpr double kTwoPi = 6.283185307179586476925286766559;

struct RopeFreq {
  double turns[64];  // base^(-2i/D) / (2 pi), i < D/2: turns a position
};

struct AppendArgs {
  const bf16 *q, *k, *v;
  bf16* q_out;
  void *k_pages, *v_pages;
  uint8_t *k_scales, *v_scales;
  const int *slots, *positions;
  int T, Hq, Hkv, q_stride, k_stride, v_stride, rotate;
  long long n_slots;
};

// A workgroup of 256 threads takes one token, 8 elements a thread of every head.  A thread's loads
// (of kAppendLoads elements at a time) are issued before the token's cosines and sines are formed
// into LDS, which hides one behind the other.  Angles: the turns position * freq in double, the
// whole turns dropped, sine and cosine of the rest in double, rounded once (positions reach 10^6
// radians and more); with the rotation's products in the order that rope_apply's have, keys of one
// token are the same from either.  HBM-bound: 16384 tokens of 32 + 2 x 32 heads of 128 in bf16 (805 MB) 150 us.
constexpr int kAppendLoads = 4;

template <int D, bool E4M3>
__global__ __launch_bounds__(256) void paged_append_kernel(const AppendArgs a, const RopeFreq f) {
  constexpr int CPR = D / 8;  // threads a head
  __shared__ float s_rope[D];  // cos, sin of each pair
  const int t = blockIdx.x, heads = a.Hq + 2 * a.Hkv, items = heads * CPR;
  const int ch = threadIdx.x % CPR;
  const long long step = 256 / CPR;  // heads a pass of the workgroup
  const int pos = a.positions[t], slot = a.slots[t];
  const bool stored = slot >= 0 && slot < a.n_slots;
  auto source = [&](int hh) {  // the elements of this thread of head hh of q, k, v in a row
    const bf16* src = hh < a.Hq ? a.q + (long long)t * a.q_stride + hh * D
                                : hh < a.Hq + a.Hkv ? a.k + (long long)t * a.k_stride + (hh - a.Hq) * D
                                                    : a.v + (long long)t * a.v_stride + (hh - a.Hq - a.Hkv) * D;
    return (const bf16x8*)(src + ch * 8);
  };
  // whole waves run the loop, so that the lanes of a head reduce together
  for (int base = 0; base < items; base += 256 * kAppendLoads) {
    const int h0 = (base + threadIdx.x) / CPR;
    bf16x8 in[kAppendLoads];
#pragma unroll
    for (int u = 0; u < kAppendLoads; ++u) in[u] = *source(min(h0 + u * (int)step, heads - 1));
    if (base == 0 && a.rotate) {
      if (threadIdx.x < D / 2) {
        const double turns = (double)pos * f.turns[threadIdx.x];
        double sn, cs;
        sincospi(2.0 * (turns - rint(turns)), &sn, &cs);
        s_rope[2 * threadIdx.x] = (float)cs;
        s_rope[2 * threadIdx.x + 1] = (float)sn;
      }
      __syncthreads();
    }
#pragma unroll
    for (int u = 0; u < kAppendLoads; ++u) {
      const int hh = h0 + u * (int)step;
      const bool is_q = hh < a.Hq, is_k = !is_q && hh < a.Hq + a.Hkv;
      const int h = is_q ? hh : is_k ? hh - a.Hq : hh - a.Hq - a.Hkv;
      const bool live = hh < heads && pos >= 0 && (is_q || stored);
      float x[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) x[e] = (float)in[u][e];
      if (a.rotate && (is_q || is_k)) {
        const float* cs = s_rope + ch * 8;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float x0 = x[2 * e], x1 = x[2 * e + 1], c = cs[2 * e], s = cs[2 * e + 1];
          x[2 * e] = fmaf(x0, c, -(x1 * s));
          x[2 * e + 1] = fmaf(x0, s, x1 * c);
        }
      }
      const long long row = (long long)slot * a.Hkv + h;
      if (E4M3 && !is_q) {
        // scale: the smallest power of two that brings every finite element to at most 448
        float top = 0.f;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const float m = fabsf(x[e]);
          if (m < INFINITY) top = fmaxf(top, m);
        }
        uint32_t mag = __float_as_uint(top);
#pragma unroll
        for (int off = CPR / 2; off >= 1; off >>= 1) mag = max(mag, (uint32_t)__shfl_xor((int)mag, off));
        if (live) {
          // 448 = 1.75 * 2^8: the exponent less 8, one more where the mantissa is past 1.75
          int e2 = (int)(mag >> 23) - 127 - 8 + ((mag & 0x7fffffu) > 0x600000u);
          e2 = mag == 0 ? 0 : max(e2, -126);
          const float inv = ldexpf(1.f, -e2);
          uint32_t w[2];
#pragma unroll
          for (int j = 0; j < 2; ++j) {
            int p = 0;
            p = __builtin_amdgcn_cvt_pk_fp8_f32(x[4 * j] * inv, x[4 * j + 1] * inv, p, false);
            p = __builtin_amdgcn_cvt_pk_fp8_f32(x[4 * j + 2] * inv, x[4 * j + 3] * inv, p, true);
            w[j] = (uint32_t)p;
#pragma unroll
            for (int e = 0; e < 4; ++e)  // e4m3 has no infinity: NaN
              if (!(fabsf(x[4 * j + e]) < INFINITY)) w[j] |= 0x7fu << (8 * e);
          }
          uint8_t* out = (uint8_t*)(is_k ? a.k_pages : a.v_pages) + row * D + ch * 8;
          *(u32x2*)out = u32x2{w[0], w[1]};
          if (ch == 0) (is_k ? a.k_scales : a.v_scales)[row] = (uint8_t)(e2 + 127);
        }
      } else if (live) {
        bf16* out = is_q ? a.q_out + ((long long)t * a.Hq + h) * D + ch * 8
                         : (bf16*)(is_k ? a.k_pages : a.v_pages) + row * D + ch * 8;
        *(u32x4*)out = u32x4{pack_bf16x2(x[0], x[1]), pack_bf16x2(x[2], x[3]), pack_bf16x2(x[4], x[5]),
                             pack_bf16x2(x[6], x[7])};
      }
    }
  }
}

const RopeFreq& rope_freq(int D) {
  struct Tables {
    RopeFreq f[2];
    Tables() {
      for (int d = 0; d < 2; ++d)
        for (int i = 0; i < 64; ++i) f[d].turns[i] = pow(kRopeBase, -2.0 * i / (64 << d)) / kTwoPi;
    }
  };
  static const Tables t;
  return t.f[D == 128];
}

}  // namespace

int check_pages(int page_size, int n_pages, int Hkv, int D) {
  if (page_size <= 0 || n_pages <= 0 || Hkv <= 0 || D <= 0)
    return set_err(RA_EINVAL, "sizes must be positive (page_size=%d n_pages=%d Hkv=%d D=%d)", page_size, n_pages, Hkv,
                   D);
  if (page_size > kMaxPage || (page_size & (page_size - 1)))
    return set_err(RA_EUNSUPPORTED, "page_size=%d must be a power of two of at most %d", page_size, kMaxPage);
  if ((long long)n_pages * page_size >= (1ll << 31))
    return set_err(RA_EUNSUPPORTED, "n_pages*page_size = %lld slots exceeds 2^31-1", (long long)n_pages * page_size);
  return RA_OK;
}

int check_kv(int kv_type, const void* k_scales, const void* v_scales) {
  if (kv_type != RA_KV_BF16 && kv_type != RA_KV_E4M3)
    return set_err(RA_EINVAL, "kv_type=%d must be RA_KV_BF16 or RA_KV_E4M3", kv_type);
  if (kv_type == RA_KV_E4M3 && (!k_scales || !v_scales)) return set_err(RA_EINVAL, "an e4m3 cache needs scales");
  if (kv_type == RA_KV_BF16 && (k_scales || v_scales)) return set_err(RA_EINVAL, "a bf16 cache has no scales");
  return RA_OK;
}

}  // namespace ra

using namespace ra;

extern "C" int paged_plan(const int* lens, const int* n_new, const int* free_pages, const int* free_head,
                          int* block_table, int* cu_rows, int* new_lens, int* slots, int* positions, int* counts, int R,
                          int page_size, int max_pages, int n_pages, int n_free, int T, hipStream_t stream) {
  g_err.clear();
  if (!lens || !n_new || !free_pages || !block_table || !cu_rows || !new_lens || !slots || !positions || !counts)
    return set_err(RA_EINVAL, "null pointer argument");
  if (int e = check_aligned({}, {lens, n_new, free_pages, free_head, block_table, cu_rows, new_lens, slots, positions,
                                 counts}))
    return e;
  if (lens == new_lens || n_new == new_lens) return set_err(RA_EINVAL, "new_lens must not be lens or n_new");
  if (free_head && free_head >= counts && free_head < counts + 4)
    return set_err(RA_EINVAL, "free_head must not lie in counts");
  if (R <= 0 || max_pages <= 0 || n_free <= 0 || T <= 0)
    return set_err(RA_EINVAL, "sizes must be positive (R=%d max_pages=%d n_free=%d T=%d)", R, max_pages, n_free, T);
  if (int e = check_pages(page_size, n_pages, 1, 1)) return e;
  if (R > kMaxRequests) return set_err(RA_EUNSUPPORTED, "R=%d exceeds %d requests", R, kMaxRequests);
  PlanArgs a{lens, n_new, free_pages, free_head, block_table, cu_rows, new_lens, slots, positions, counts, R, 0,
             max_pages, n_pages, n_free, T, (((uintptr_t)slots | (uintptr_t)positions) & 15) == 0};
  while ((1 << a.page_shift) < page_size) ++a.page_shift;
  const int per = kPlanThreads * kPlanRows;
  const unsigned grid = (unsigned)(((long long)T + per - 1) / per);
  hipLaunchKernelGGL(paged_plan_kernel, dim3(grid), dim3(kPlanThreads), (3 * R + 1) * sizeof(int), stream, a);
  RA_HIP(hipGetLastError());
  return RA_OK;
}

extern "C" int paged_append(const void* q, const void* k, const void* v, void* q_out, void* k_pages, void* v_pages,
                            unsigned char* k_scales, unsigned char* v_scales, const int* slots, const int* positions,
                            int T, int Hq, int Hkv, int D, int q_stride, int k_stride, int v_stride, int n_pages,
                            int page_size, int kv_type, int rotate, hipStream_t stream) {
  g_err.clear();
  if (!k || !v || !k_pages || !v_pages || !slots || !positions) return set_err(RA_EINVAL, "null pointer argument");
  if (!q != !q_out) return set_err(RA_EINVAL, "q and q_out are given together or not at all");
  if (int e = check_aligned({q, k, v, q_out, k_pages, v_pages}, {slots, positions})) return e;
  if (int e = check_kv(kv_type, k_scales, v_scales)) return e;
  if (rotate != 0 && rotate != 1) return set_err(RA_EINVAL, "rotate must be 0 or 1 (got %d)", rotate);
  if (T <= 0 || Hq < 0 || (q && Hq == 0)) return set_err(RA_EINVAL, "sizes must be positive (T=%d Hq=%d)", T, Hq);
  if (int e = check_pages(page_size, n_pages, Hkv, D)) return e;
  if (D != 64 && D != 128) return set_err(RA_EUNSUPPORTED, "head dim D=%d not supported (64 or 128)", D);
  if (T >= 1 << 24) return set_err(RA_EUNSUPPORTED, "T=%d rows exceeds 2^24-1", T);  // of 256 threads each
  if (!q) Hq = 0;
  if (Hq > kMaxHeads || Hkv > kMaxHeads)
    return set_err(RA_EUNSUPPORTED, "Hq=%d, Hkv=%d: at most %d heads", Hq, Hkv, kMaxHeads);
  if ((q && (q_stride < Hq * D || q_stride % 8)) || k_stride < Hkv * D || k_stride % 8 || v_stride < Hkv * D ||
      v_stride % 8)
    return set_err(RA_EINVAL, "row strides %d, %d, %d must hold the heads and be multiples of 8", q_stride, k_stride,
                   v_stride);
  if (q == q_out && q && q_stride != Hq * D) return set_err(RA_EINVAL, "q_out is dense: it can be q only where q is");
  AppendArgs a{(const bf16*)q, (const bf16*)k, (const bf16*)v, (bf16*)q_out, k_pages, v_pages, k_scales, v_scales,
               slots, positions, T, Hq, Hkv, q_stride, k_stride, v_stride, rotate, (long long)n_pages * page_size};
  auto* kern = D == 128 ? (kv_type == RA_KV_E4M3 ? paged_append_kernel<128, true> : paged_append_kernel<128, false>)
                        : (kv_type == RA_KV_E4M3 ? paged_append_kernel<64, true> : paged_append_kernel<64, false>);
  hipLaunchKernelGGL(kern, dim3(T), dim3(256), 0, stream, a, rope_freq(D));
  RA_HIP(hipGetLastError());
  return RA_OK;
}
