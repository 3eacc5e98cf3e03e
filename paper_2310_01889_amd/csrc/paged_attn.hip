// Attention of the newest tokens of many requests over a paged key/value cache, for gfx950.
//
// o = softmax(q K^T / sqrt(D)) V over the keys of each request, read page by page through its
// row of the block table; the new tokens are the last of the cache and see keys up to their own.
// A step reads every key and value once, 2 D bytes a key and head each (D and a scale in 8 bits):
// it is bound by HBM bandwidth, as long as the reads are spread evenly over the chip.
//
// Work is counted in units: one tile of KT keys of one request, for up to 32 query slots a key
// head (slot n = new token n / G, query head n % G of the G that share the key head; requests of
// more slots take several rounds over their keys).  The units of all requests stand in one row,
// and teams of Hkv waves, a wave a key head, take equal shares of it, so the lengths of a batch do
// not matter for the balance; the heads of one token, neighbours in memory, are read at about the
// same time.  The lengths are on the device: each wave finds its team's share from their prefix
// sums itself.  A wave whose share holds a whole (request, round) writes its result; the others
// leave partial softmax states that a second launch joins.
#include <limits.h>
#include <math.h>

#include <algorithm>

#include "ra_common.h"
#include "ra_dma.h"
#include "ra_paged.h"
#include "ra_runtime.h"
#include "ringattn.h"

namespace ra {
namespace {

constexpr int kMaxNew = 32;      // new tokens a request
constexpr int kSlots = 32;       // query slots a wave

// Keys a tile, and the waves that share all tiles, four a workgroup: neighbouring key heads read pieces of
// one token, so their waves stay close to one another in time and place (24 requests of 700 to 16001
// tokens, one new each, us with one, two and four waves a workgroup: 8 heads of 128 dims in bf16 167, 159,
// 157; 16 heads of 64 dims 177, 167, 162, in 8 bits 119, 121, 100; 8 heads of 128 in 8 bits 91, 92, 92).
// bf16: tiles of 8 KB, four of them (32 KB of LDS) a wave, one workgroup a compute unit (768 waves in
// place of 1024: 16 heads of 64 190 us for 162; 262144 tokens of 32 heads 728 for 707).
// 8 bits: rows have half the bytes and the same products: 4 KB tiles, so that a SIMD's second wave
// converts and multiplies while the first one waits (8 KB tiles and 1024 waves: 8 heads of 128 97 us
// for 92, of 64 59 for 49).  Two workgroups fit a compute unit's LDS: 2048 waves fill the chip; for 128 dims
// 1792 (448 workgroups: most units have two, some one), with which the partial states of 32 slots
// stay below the 64 MB of a workspace that the library keeps (us with 1280, 1536, 1792, 2048 waves:
// 8 heads of 128 112, 97, 90, 87; of 64 64, 59, 53, 49).
// Four waves that join in LDS take 64 keys at a time in 8 bits as well, which is the room their states
// need.
constexpr int kShareWaves = 4;
constexpr int workers(int D, bool f8) { return !f8 ? 1024 : D == 128 ? 1792 : 2048; }
constexpr int max_workers(int D) { return workers(D, true); }
constexpr int tile_keys(int D, bool f8, int gw) { return D == 64 || (f8 && gw > 1) ? 64 : 32; }

// What the second launch joins: the parts of a group of units (request, key head, round) that
// several waves share, written by the first of them.  parts = 0: nothing to join.
struct Split {
  int row0;   // first q row of the request
  int h;      // key head
  int slot0;  // first query slot (of the request's n * G)
  int slots;  // query slots
  int first;  // index of the first wave's part; the next teams' follow, 2 Hkv apart
  int parts;
};

struct PagedArgs {
  const bf16* q;  // [T, Hq, D]
  const void *k, *v;
  const uint8_t *ks, *vs;
  const int *table, *lens, *cu;
  bf16* o;          // [T, Hq, D]
  float* lse;       // [T, Hq]
  float* part_acc;  // [waves][2][M][D] unnormalised outputs: of a wave's first group, of its last
  float* part_ml;   // [waves][2][M][2] maxima (log2 units) and denominators
  Split* split;     // one a group where the groups are fewer than the waves, else one a wave
  int T, R, Hq, Hkv, n_pages, page_shift, max_pages, max_new;
  int M;            // query slots of a group at most
  int rounds;       // rounds of slots of a request at most
  int by_group;     // entries of split: 1 a group, 0 a wave
  int teams;        // workers / Hkv
  int round_rows;   // one launch: rows a round holds at least, or 0: rounds of each request to a workgroup each
  int rounds_row;   // rounds that a row takes at most
  float scale;
};

// The requests' shape as every wave reads it, whatever the arrays hold.
struct Request {
  int row0, n, keys, first;  // first q row, new tokens, keys to read, position of the first new token
};
// (The arrays are constant while the kernel runs: scalar loads where r is uniform.)
typedef __attribute__((address_space(4))) const int const_int;
__device__ __forceinline__ Request request(const PagedArgs& a, int r) {
  Request q;
  int row1 = r + 1;
  q.row0 = r;
  if (a.cu) {
    q.row0 = min(max(((const_int*)a.cu)[r], 0), a.T);
    row1 = min(max(((const_int*)a.cu)[r + 1], q.row0), a.T);
  }
  const int len = max(((const_int*)a.lens)[r], 0), rows = row1 - q.row0;
  q.n = min(rows, a.max_new);
  q.first = len - rows;
  q.keys = (int)min((long long)len, (long long)a.max_pages << a.page_shift);
  return q;
}

__device__ const uint8_t g_zero_row[256] __attribute__((aligned(256))) = {};  // read in place of masked rows

// A value that is the same in every lane, to scalar registers.
__device__ __forceinline__ long long uniform(long long x) {
  const uint32_t lo = __builtin_amdgcn_readfirstlane((int)x), up = __builtin_amdgcn_readfirstlane((int)(x >> 32));
  return (long long)((unsigned long long)up << 32 | lo);
}

// XOR swizzle of the 16-byte chunks of an LDS row of RB bytes.
template <int RB>
__device__ __forceinline__ int row_swz(int r) {
  if constexpr (RB == 256) return swz<128>(r);
  else if constexpr (RB == 128) return swz<64>(r);
  else return (r >> 2) & 3;
}

__device__ __forceinline__ bf16x8 from_e4m3(uint32_t lo, uint32_t hi, float scale) {
  typedef __bf16 bf16x2_t __attribute__((ext_vector_type(2)));
  const bf16x2_t a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, scale, false);
  const bf16x2_t b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, scale, true);
  const bf16x2_t c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, scale, false);
  const bf16x2_t d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, scale, true);
  return bf16x8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}

// Whether any of 16 bytes of values is not finite (8 bits: NaN), and the bytes with those zeroed.
template <bool F8>
__device__ __forceinline__ bool any_not_finite(u32x4 x) {
  bool odd = false;
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    if constexpr (F8) odd |= (((x[e] & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u) != 0;  // 0x7f becomes 0x80
    else odd |= (x[e] & 0x7f80u) == 0x7f80u || (x[e] & 0x7f800000u) == 0x7f800000u;
  }
  return odd;
}
template <bool F8>
__device__ __forceinline__ u32x4 only_finite(u32x4 x) {
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    if constexpr (F8) {
      const uint32_t hit = (((x[e] & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u) >> 7;
      x[e] &= ~(hit * 0xffu);
    } else {
      if ((x[e] & 0x7f80u) == 0x7f80u) x[e] &= 0xffff0000u;
      if ((x[e] & 0x7f800000u) == 0x7f800000u) x[e] &= 0xffffu;
    }
  }
  return x;
}

// GW = 0: each wave its team's share of all units.  GW > 0: short requests; GW waves take
// the tiles of one group (request, key head, round) in turns and join their states in LDS, so that
// one launch does.  Per tile the arithmetic of the decode kernel over a contiguous cache, but for the
// probabilities' parts:
// S^T = K Q^T on the matrix cores (K rows with bits 2 and 3 of the row index swapped as the A
// operand, a lane one query slot), lazy online softmax, O^T += V^T P^T with V^T from the
// transpose reads of LDS.  Tiles are double buffered: the direct-to-LDS loads of tile i + 1,
// every row at an address of its own (pages of any size), are in flight while tile i is computed.
// 8-bit tiles become bf16 operands in registers, exactly: key rows under their scales, values as
// they are, their scales (powers of two) going into the probabilities before those are split.
template <int D, bool F8, int GW>
__global__ __launch_bounds__(64 * (GW ? GW : kShareWaves), GW > 1 ? 1 : 2) void paged_attn_kernel(const PagedArgs a) {
  constexpr int NW = GW ? GW : 1, WAVES = GW ? GW : kShareWaves;  // waves of a group, of a workgroup
  constexpr int RB = F8 ? D : 2 * D;              // bytes a row
  constexpr int CPR = RB / 16, RPL = 64 / CPR;    // chunks a row; rows one 1 KB wave load fills
  constexpr int KT = tile_keys(D, F8, GW);        // keys a tile
  constexpr int LOADS = KT / RPL, NS = KT / 32, NKK = D / 16, NDT = D / 32;
  constexpr float kTau = F8 ? 7.f : 8.f;          // lazy-rescale threshold (log2 units); 2^7 times a scale of 2^120 is finite
  constexpr int TB = KT * RB;                     // bytes of a tile; its scales: a dword a key
  __shared__ __attribute__((aligned(1024))) uint8_t s_tiles[WAVES][2][2][TB];  // wave, K or V, buffer
  __shared__ __attribute__((aligned(256))) uint32_t s_scales[WAVES][2][2][F8 ? 64 : 1];
  const int lane = threadIdx.x & 63, l32 = lane & 31, hi = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  uint8_t(*sK)[TB] = s_tiles[wave][0];
  uint8_t(*sV)[TB] = s_tiles[wave][1];
  uint32_t(*sKS)[F8 ? 64 : 1] = s_scales[wave][0];
  uint32_t(*sVS)[F8 ? 64 : 1] = s_scales[wave][1];
  const int G = a.Hq / a.Hkv;
  auto quotient = [&](long long x, long long y) {  // x / y, seldom past 32 bits
    return (x | y) >> 31 ? x / y : (long long)((uint32_t)x / (uint32_t)y);
  };
  // neighbours of one XCD: what the heads of a request read side by side (ids, scales) shares an L2
  const int id = xcd_swizzle(blockIdx.x, gridDim.x);
  int w = 0, team = 0, h, r, round = 0;
  long long share = 0, u0 = 0, u1 = 1, r_at = 0;  // r_at: first unit of request r
  Request q;                                      // request r
  if constexpr (GW > 0) {
    if (a.round_rows == 0) {  // a workgroup a (request, key head, round), whether the request has it or not
      const int g = id / a.rounds;
      r = g / a.Hkv;
      h = g - r * a.Hkv;
      round = id - g * a.rounds;
    } else {  // request r's rounds from number first(r) on: the largest r with first(r) <= u, 64 tried at a time
      const int u = id / a.Hkv;
      h = id - u * a.Hkv;
      auto first = [&](int r) {
        const int row = min(max(a.cu[r], 0), a.T);
        return G <= kSlots ? r + row / a.round_rows : row * a.rounds_row;
      };
      auto last = [](bool on) -> int {  // of the lanes from 0 on where it is true; 0 if it is nowhere
        const int n = (int)__popcll(__builtin_amdgcn_ballot_w64(on));  // (unsigned as it comes)
        return n > 0 ? n - 1 : 0;
      };
      const int stride = (a.R + 63) / 64, from = lane * stride;
      r = last(from < a.R && first(from) <= u) * stride;
      if (stride > 1) {
        const int at = r + lane;
        r += last(lane < stride && at < a.R && first(at) <= u);
      }
      r = __builtin_amdgcn_readfirstlane(min(r, a.R - 1));
      round = u - __builtin_amdgcn_readfirstlane(first(r));
      if (round < 0) return;
    }
    q = request(a, r);
  } else {
    w = id * kShareWaves + wave;
    team = w / a.Hkv;
    h = w - team * a.Hkv;

    // ---- this team's share of the units ----
    auto units = [&](int r, Request& q) -> long long {  // of request r
      q = Request{};
      if (r >= a.R) return 0;
      q = request(a, r);
      const int rounds = (q.n * G + kSlots - 1) / kSlots, tiles = max(1, (q.keys + KT - 1) / KT);
      return (long long)rounds * tiles;
    };
    auto scan = [&](long long v) {  // inclusive prefix sum over the lanes
#pragma unroll
      for (int off = 1; off < 64; off <<= 1) {
        const long long y = __shfl_up(v, off);
        if (lane >= off) v += y;
      }
      return v;
    };
    const int per = (a.R + 63) / 64;  // requests a lane sums
    long long mine = 0;
    for (int j = 0; j < per; ++j) mine += units(lane * per + j, q);
    const long long upto = scan(mine), total = uniform(__shfl(upto, 63));
    share = max(1ll, quotient(total + a.teams - 1, a.teams));
    u0 = share * team;
    u1 = min(total, u0 + share);
    if (!a.by_group && lane == 0) a.split[w].parts = 0;
    if (team >= a.teams || u0 >= u1) return;
    // the request of unit u0: the lane whose sums reach past it, then the request among that lane's
    r = __ffsll((unsigned long long)__builtin_amdgcn_ballot_w64(upto > u0)) - 1;
    r_at = __shfl(upto - mine, r);
    int at = r;
    if (per > 1) {
      r *= per;
      const long long v = lane < per ? units(r + lane, q) : 0, s = scan(v);
      at = __ffsll((unsigned long long)__builtin_amdgcn_ballot_w64(r_at + s > u0)) - 1;
      r_at += __shfl(s - v, at);
      r += at;
    }
    r = __builtin_amdgcn_readfirstlane(r);
    r_at = uniform(r_at);
    at = __builtin_amdgcn_readfirstlane(at);  // the lane that has read request r
    q.row0 = __builtin_amdgcn_readlane(q.row0, at);
    q.n = __builtin_amdgcn_readlane(q.n, at);
    q.keys = __builtin_amdgcn_readlane(q.keys, at);
    q.first = __builtin_amdgcn_readlane(q.first, at);
  }

  // ---- constants of the tile loop ----
  const float sl2 = a.scale * kLog2e;
  const int rs = a.Hkv * RB;  // bytes a token
  const int page_mask = (1 << a.page_shift) - 1;
  // Offsets in a tile.  The swizzle is an XOR of the chunk's number, so the steps over chunks are
  // XORs as well; a step over rows that changes the swizzle (loads) is one of a constant.
  const int load_row = lane / CPR, load_off = 16 * ((lane % CPR) ^ row_swz<RB>(load_row));
  auto chunk = [&](int j) { return load_off ^ (16 * (row_swz<RB>(j * RPL) ^ row_swz<RB>(0))); };
  const int krow = swap_bits23(l32), koff = krow * RB + 16 * (hi ^ row_swz<RB>(krow));
  const int g16 = lane >> 4, li = lane & 15;
  int voff[2];
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const int row = F8 ? 8 * hi + (li >> 1) : 8 * hi + 4 * i + (li >> 2);
    const int byte = F8 ? 16 * (g16 & 1) + 8 * (li & 1) : 2 * (16 * (g16 & 1) + 4 * (li & 3));
    voff[i] = row * RB + 16 * ((byte >> 4) ^ row_swz<RB>(row)) + (byte & 15);
  }

  for (long long u = u0; u < u1;) {
    // ---- the group of unit u: request r, round of slots; its tiles [t0, t1) ----
    int tiles, t0, t1;
    if constexpr (GW > 0) {
      tiles = max(1, (q.keys + KT - 1) / KT);
      if (round * kSlots >= q.n * G) return;
      t0 = wave;
      t1 = tiles;
    } else {
      int rounds;
      for (;;) {
        rounds = (q.n * G + kSlots - 1) / kSlots;
        tiles = max(1, (q.keys + KT - 1) / KT);
        const long long end = r_at + (long long)rounds * tiles;
        if (u < end) break;
        r_at = end;
        q = request(a, ++r);
      }
      const long long in_r = u - r_at;
      round = rounds == 1 ? 0 : (int)quotient(in_r, tiles);
      t0 = (int)(in_r - (long long)round * tiles);
      t1 = (int)min((long long)tiles, t0 + (u1 - u));
    }
    const int slot0 = round * kSlots, slots = min(kSlots, q.n * G - slot0);
    const int n = slot0 + min(l32, slots - 1), t = n / G;  // this lane's slot
    const long long qrow = (long long)(q.row0 + t) * a.Hq + h * G + (n - t * G);
    const int qpos = q.first + t;

    f32x16 oacc[NDT];
#pragma unroll
    for (int dt = 0; dt < NDT; ++dt)
#pragma unroll
      for (int i = 0; i < 16; ++i) oacc[dt][i] = 0.f;
    float m_run = -INFINITY, l_run = 0.f, m_eff = 0.f, thr = -INFINITY;
    uint64_t hit_nan = 0, hit_up = 0, hit_down = 0;  // this lane's sums that a value not finite joins
    // slot of key row `lane` of tile i in the cache, or -1; the ids of 64 pages are at hand
    const int* trow = a.table + (long long)r * a.max_pages;
    int ids = -1, ids_at = -1;
    auto slot_of = [&](int i) __attribute__((always_inline)) {
      const int p = i * KT + lane, page = p >> a.page_shift, at = (i * KT >> a.page_shift) & ~63;
      if (at != ids_at) {  // pages of a tile are 64 at most and aligned: of one such run
        ids = at + lane < a.max_pages ? trow[at + lane] : -1;
        ids_at = at;
        asm volatile("s_waitcnt vmcnt(0)" : "+v"(ids));  // here, not at every tile's use of ids
      }
      const int id = __shfl(ids, page & 63);
      const bool there = lane < KT && p < q.keys && id >= 0 && id < a.n_pages;
      return there ? (id << a.page_shift) + (p & page_mask) : -1;
    };
    const uint8_t* kb = (const uint8_t*)a.k + h * RB;
    const uint8_t* vb = (const uint8_t*)a.v + h * RB;
    auto load_tile = [&](int s, int b) __attribute__((always_inline)) {  // into buffer b
      if constexpr (F8) {
        const long long i = (long long)max(s, 0) * a.Hkv + h;
        dma_lds1_at(a.ks + i, lds_addr(sKS[b]));
        dma_lds1_at(a.vs + i, lds_addr(sVS[b]));
      }
#pragma unroll
      for (int j = 0; j < LOADS; ++j) {
        const int row = __shfl(s, j * RPL + load_row);
        const long long off = (long long)row * rs + chunk(j);
        dma_lds16_at(row >= 0 ? kb + off : g_zero_row + chunk(j), lds_addr(sK[b]) + j * 1024);
        dma_lds16_at(row >= 0 ? vb + off : g_zero_row + chunk(j), lds_addr(sV[b]) + j * 1024);
      }
    };

    int s_cur = -1;
    if (GW <= 1 || t0 < t1) {
      s_cur = slot_of(t0);
      load_tile(s_cur, 0);
    }
    // (lanes past the slots repeat the last one; nothing of theirs is kept)
    bf16x8 qreg[NKK];
#pragma unroll
    for (int kk = 0; kk < NKK; ++kk)
      qreg[kk] = *(const bf16x8*)(a.q + qrow * D + (F8 ? 32 * (kk / 2) + 16 * hi + 8 * (kk & 1) : 16 * kk + 8 * hi));

#pragma unroll 1
    for (int it = t0, b = 0; it < t1; it += NW, b ^= 1) {
      const uint64_t present = __builtin_amdgcn_ballot_w64(s_cur >= 0);  // keys of the tile that exist
      // the previous tile's LDS reads have all returned before its buffer is refilled
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
      if (it + NW < t1) {
        s_cur = slot_of(it + NW);
        load_tile(s_cur, b ^ 1);
        asm volatile("s_waitcnt vmcnt(%0)" ::"n"(2 * LOADS + (F8 ? 2 : 0)) : "memory");  // tile it landed
      } else {
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
      }
      const uint8_t* kt = sK[b];
      uint8_t* vt = sV[b];
      const int k0 = it * KT;
      // keys that some row of the request does not see, or none does
      const bool diagonal = k0 + KT - 1 > q.first;
      const bool masked = diagonal || present != (KT == 64 ? ~0ull : (1ull << KT) - 1);
      if (diagonal && q.first + 1 < q.keys) {  // (none such: every key is there for every row)
        // A value that is not finite, in a row that some slots see and some do not, would make NaN
        // of zero probabilities: its slots are noted, and it is overwritten by zero.
        bool odd = false;
#pragma unroll 1
        for (int i = 0; i < TB / 1024; ++i) odd |= any_not_finite<F8>(*(const u32x4*)(vt + i * 1024 + lane * 16));
        if (__builtin_amdgcn_ballot_w64(odd)) {
#pragma unroll 1
          for (int row = 0; row < KT; ++row) {
            if (k0 + row > qpos) continue;
#pragma unroll 1
            for (int g = 0; g < NDT * 4; ++g) {  // elements 4 g ... of this lane's part of a row
              const int byte = (F8 ? 1 : 2) * (8 * g + 4 * hi);
              const uint8_t* at = vt + row * RB + 16 * ((byte >> 4) ^ row_swz<RB>(row)) + (byte & 15);
#pragma unroll
              for (int e = 0; e < 4; ++e) {
                const float x = F8 ? ((at[e] & 0x7f) == 0x7f ? NAN : 0.f) : (float)((const bf16*)at)[e];
                const uint64_t bit = 1ull << (4 * g + e);
                if (x != x) hit_nan |= bit;
                else if (x == INFINITY) hit_up |= bit;
                else if (x == -INFINITY) hit_down |= bit;
              }
            }
          }
          asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
#pragma unroll 1
          for (int i = 0; i < TB / 1024; ++i) {
            u32x4* at = (u32x4*)(vt + i * 1024 + lane * 16);
            *at = only_finite<F8>(*at);
          }
          asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        }
      }
#pragma unroll
      for (int sub = 0; sub < NS; ++sub) {
        f32x16 s;
#pragma unroll
        for (int i = 0; i < 16; ++i) s[i] = 0.f;
        if constexpr (F8) {
          const float ksc = __uint_as_float(sKS[b][32 * sub + krow] << 23);
#pragma unroll
          for (int kk = 0; kk < NKK; kk += 2) {
            const u32x4 x = *(const u32x4*)(kt + 32 * sub * RB + (koff ^ (16 * kk)));
            s = mfma32(from_e4m3(x[0], x[1], ksc), qreg[kk], s);
            s = mfma32(from_e4m3(x[2], x[3], ksc), qreg[kk + 1], s);
          }
        } else {
#pragma unroll
          for (int kk = 0; kk < NKK; ++kk)
            s = mfma32(*(const bf16x8*)(kt + 32 * sub * RB + (koff ^ (32 * kk))), qreg[kk], s);
        }
#pragma unroll
        for (int i = 0; i < 16; ++i) s[i] = fmaf(s[i], sl2, -m_eff);  // log2 units
        if (masked) {
#pragma unroll
          for (int i = 0; i < 16; ++i) {
            const int key = 32 * sub + 16 * (i >> 3) + 8 * hi + (i & 7);
            if (k0 + key > qpos || !(present >> key & 1)) s[i] = -INFINITY;
          }
        }
        // lazy rescale: raise the running maximum only when a score exceeds it by kTau
        float mx = -INFINITY;
#pragma unroll
        for (int i = 0; i < 16; ++i) mx = fmaxf(mx, s[i]);
        const float mx2 = pair_max(mx);
        if (__builtin_amdgcn_ballot_w64(mx2 > thr)) {
          const float m_new = fmaxf(m_run, m_eff + mx2);
          const float m_new_eff = (m_new == -INFINITY) ? 0.f : m_new;
          const float alpha = (m_run == -INFINITY) ? 0.f : fast_exp2(m_run - m_new);
          const float delta = m_new_eff - m_eff;
          // (a slot that has seen no key keeps zero sums: 0 * alpha; NaN sums stay NaN)
          l_run *= alpha;
#pragma unroll
          for (int dt = 0; dt < NDT; ++dt)
#pragma unroll
            for (int i = 0; i < 16; ++i) oacc[dt][i] *= alpha;
#pragma unroll
          for (int i = 0; i < 16; ++i) s[i] -= delta;
          m_run = m_new;
          m_eff = m_new_eff;
          thr = (m_new == -INFINITY) ? -INFINITY : kTau;
        }
        // Probabilities; the denominator sums them as they are, the products take them as the sum of
        // three bf16 numbers, the upper 8 bits of what the ones before leave: exact.  (With two they are
        // off by up to 2^-16, which outputs that nearly cancel show.)  None is zero, but 2^-133 at least,
        // where the probability is not: an infinite value has an infinite sum (8 bits hold none).
#pragma unroll
        for (int i = 0; i < 16; ++i) s[i] = fast_exp2(s[i]);
#pragma unroll
        for (int i = 0; i < 16; i += 4) l_run += (s[i] + s[i + 1]) + (s[i + 2] + s[i + 3]);
        if constexpr (F8) {
#pragma unroll
          for (int g = 0; g < 2; ++g) {
            const uint32_t* sc = sVS[b] + 32 * sub + 16 * g + 8 * hi;
            const u32x4 lo = *(const u32x4*)sc, up = *(const u32x4*)(sc + 4);
#pragma unroll
            for (int e = 0; e < 8; ++e)  // (0 stays 0 under any scale)
              s[8 * g + e] = __builtin_ldexpf(s[8 * g + e], (int)(e < 4 ? lo[e & 3] : up[e & 3]) - 127);
          }
        }
        bf16x8 pb[3][2];
#pragma unroll
        for (int g = 0; g < 2; ++g) {
          u32x4 w[3];
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            float p0 = s[8 * g + 2 * j], p1 = s[8 * g + 2 * j + 1];
#pragma unroll
            for (int e = 0; e < 3; ++e) {
              const uint32_t x = __float_as_uint(p0), y = __float_as_uint(p1);
              w[e][j] = __builtin_amdgcn_perm(y, x, 0x07060302u);
              p0 -= __uint_as_float(x & 0xffff0000u);
              p1 -= __uint_as_float(y & 0xffff0000u);
            }
            if constexpr (!F8) {
              const uint32_t least = min_u16x2(w[0][j], 0x10001u);
              w[1][j] = max_u16x2(w[1][j], least);
              w[2][j] = max_u16x2(w[2][j], least);
            }
          }
#pragma unroll
          for (int e = 0; e < 3; ++e) pb[e][g] = __builtin_bit_cast(bf16x8, w[e]);
        }
        const uint8_t* vs = vt + 32 * sub * RB;
        auto values = [&](int g, int dt) __attribute__((always_inline)) {  // 16 keys x 32 dims of V^T
          const uint8_t* vg = vs + 16 * g * RB;
          if constexpr (F8) {
            typedef int i32x2_t __attribute__((ext_vector_type(2)));
            const i32x2_t x = __builtin_amdgcn_ds_read_tr8_b64_v2i32(
                (__attribute__((address_space(3))) i32x2_t*)((lds_void*)(vg + (voff[0] ^ (32 * dt)))));
            return from_e4m3((uint32_t)x[0], (uint32_t)x[1], 1.f);
          } else {
            const bf16x4 lo = lds_read_tr16((const bf16*)(vg + (voff[0] ^ (64 * dt))));
            const bf16x4 up = lds_read_tr16((const bf16*)(vg + (voff[1] ^ (64 * dt))));
            return bf16x8{lo[0], lo[1], lo[2], lo[3], up[0], up[1], up[2], up[3]};
          }
        };
#pragma unroll
        for (int g = 0; g < 2; ++g)
#pragma unroll
          for (int dt = 0; dt < NDT; ++dt) {
            const bf16x8 vv = values(g, dt);
#pragma unroll
            for (int e = 0; e < 3; ++e) oacc[dt] = mfma32(vv, pb[e][g], oacc[dt]);
          }
      }
    }

    if (__builtin_amdgcn_ballot_w64((hit_nan | hit_up | hit_down) != 0)) {
#pragma unroll
      for (int dt = 0; dt < NDT; ++dt)
#pragma unroll
        for (int i = 0; i < 16; ++i) {  // bit 16 dt + i: dims 32 dt + 8 (i / 4) + 4 hi + i % 4
          const uint64_t bit = 1ull << (16 * dt + i);
          if (hit_up & bit) oacc[dt][i] += INFINITY;
          if (hit_down & bit) oacc[dt][i] -= INFINITY;
          if (hit_nan & bit) oacc[dt][i] = NAN;
        }
    }

    // ---- the result, or this wave's part of it ----
    const float l = pair_sum(l_run);
    if constexpr (GW > 1) {
      // the waves' states through LDS: a slot's sums in a row of its own, 4 floats apart from the next
      constexpr int ROW = D + 4;
      static_assert(kSlots * ROW * 4 <= 4 * TB, "the states fit the tiles");
      __shared__ float s_ml[GW][kSlots][2];
      float* acc = (float*)s_tiles[wave];
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
      if (l32 < slots) {
#pragma unroll
        for (int dt = 0; dt < NDT; ++dt)
#pragma unroll
          for (int g = 0; g < 4; ++g)
            *(f32x4*)(acc + l32 * ROW + 32 * dt + 8 * g + 4 * hi) =
                f32x4{oacc[dt][4 * g], oacc[dt][4 * g + 1], oacc[dt][4 * g + 2], oacc[dt][4 * g + 3]};
        if (!hi) s_ml[wave][l32][0] = m_run, s_ml[wave][l32][1] = l;
      }
      __syncthreads();
      for (int sl = wave; sl < slots; sl += GW) {
        float mx = -INFINITY, lt = 0.f, wt[GW], x[D / 64];
#pragma unroll
        for (int v = 0; v < GW; ++v) mx = fmaxf(mx, s_ml[v][sl][0]);
        const float top = mx == -INFINITY ? 0.f : mx;
#pragma unroll
        for (int e = 0; e < D / 64; ++e) x[e] = 0.f;
#pragma unroll
        for (int v = 0; v < GW; ++v) {
          const float lv = s_ml[v][sl][1];
          wt[v] = lv == 0.f ? 0.f : fast_exp2(s_ml[v][sl][0] - top);
          lt = fmaf(lv, wt[v], lt);
#pragma unroll
          for (int e = 0; e < D / 64; ++e)
            x[e] = fmaf(((const float*)s_tiles[v])[sl * ROW + lane + 64 * e], wt[v], x[e]);
        }
        const int nn = slot0 + sl, tt = nn / G;
        const long long row = (long long)(q.row0 + tt) * a.Hq + h * G + (nn - tt * G);
        const float inv = lt == 0.f ? 0.f : 1.f / lt;
#pragma unroll
        for (int e = 0; e < D / 64; ++e) a.o[row * D + lane + 64 * e] = (bf16)(x[e] * inv);
        if (lane == 0) a.lse[row] = lt == 0.f ? -INFINITY : top * kLn2 + logf(lt);
      }
      return;
    }
    const bool whole = GW == 1 || (t0 == 0 && t1 == tiles);
    if (l32 < slots) {
      if (whole) {
        const float inv = l == 0.f ? 0.f : 1.f / l;
        bf16* out = a.o + qrow * D;
#pragma unroll
        for (int dt = 0; dt < NDT; ++dt)
#pragma unroll
          for (int g = 0; g < 4; ++g) {
            const f32x4 x{oacc[dt][4 * g], oacc[dt][4 * g + 1], oacc[dt][4 * g + 2], oacc[dt][4 * g + 3]};
            *(u32x2*)(out + 32 * dt + 8 * g + 4 * hi) =
                u32x2{pack_bf16x2(x[0] * inv, x[1] * inv), pack_bf16x2(x[2] * inv, x[3] * inv)};
          }
        if (!hi) a.lse[qrow] = l == 0.f ? -INFINITY : m_eff * kLn2 + logf(l);
      } else {
        const long long part = ((long long)2 * w + (u == u0 ? 0 : 1)) * a.M + l32;
        float* acc = a.part_acc + part * D;
#pragma unroll
        for (int dt = 0; dt < NDT; ++dt)
#pragma unroll
          for (int g = 0; g < 4; ++g)
            *(f32x4*)(acc + 32 * dt + 8 * g + 4 * hi) =
                f32x4{oacc[dt][4 * g], oacc[dt][4 * g + 1], oacc[dt][4 * g + 2], oacc[dt][4 * g + 3]};
        if (!hi) *(f32x2*)(a.part_ml + 2 * part) = f32x2{m_run, l};
      }
    }
    if (GW == 1) return;
    if (t0 == 0 && lane == 0 && (a.by_group || !whole)) {
      const long long last = u + tiles - 1;  // the group's last unit
      a.split[a.by_group ? (r * a.Hkv + h) * a.rounds + round : w] =
          Split{q.row0, h, slot0, slots, 2 * w + (u == u0 ? 0 : 1), whole ? 0 : (int)quotient(last, share) - team + 1};
    }
    u += t1 - t0;
    // the buffers are refilled by the next group's first loads
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
  }
}

// Joins the parts of the groups that several waves share.  WPS waves take one query slot of one
// entry: each sums every WPS-th part, kBatch loads of them in flight together, and their sums are added
// in order.  A workgroup is 8 waves: one slot or eight (see the choice at the launch).  The weights
// 2^(m - M) are formed by the lanes, 64 parts at a time.
constexpr int kJoinWaves = 8;
constexpr int kEarly = 8;   // parts whose loads do not wait for the weights
constexpr int kBatch = 16;  // (8 slots of 940 parts, a wave each: 257 us with one load after the other, 90 so)
constexpr int kLongParts = 64;  // (see the launch)

template <int D, int WPS>
__device__ __forceinline__ void join_slot(const PagedArgs& a, const Split& sp, int slot, float (*s_sum)[D + 2]) {
  constexpr int E = D / 64;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), G = a.Hq / a.Hkv;
  const int w = wave % WPS;
  const bool on = slot < sp.slots;  // (the waves of a workgroup meet at its barriers)
  auto part = [&](int i) { return ((long long)(i == 0 ? sp.first : (sp.first & ~1) + 2 * i * a.Hkv)) * a.M + slot; };
  // the largest maximum of this wave's parts, then their sums relative to it
  const int mine = on ? (sp.parts - w + WPS - 1) / WPS : 0;  // parts w, w + WPS, ...
  float acc[E], x[kEarly][E];
#pragma unroll
  for (int i = 0; i < kEarly; ++i)  // the first parts are on their way while their weights are formed
#pragma unroll
    for (int e = 0; e < E; ++e)
      x[i][e] = i < mine ? a.part_acc[part(w + i * WPS) * D + lane + 64 * e] : 0.f;
  const f32x2 none = {-INFINITY, 0.f};
  const f32x2 ml0 = lane < mine ? *(const f32x2*)(a.part_ml + 2 * part(w + lane * WPS)) : none;
  float m = ml0[0];
  for (int i = lane + 64; i < mine; i += 64) m = fmaxf(m, a.part_ml[2 * part(w + i * WPS)]);
#pragma unroll
  for (int off = 32; off >= 1; off >>= 1) m = fmaxf(m, __shfl_xor(m, off));
  const float m_eff = m == -INFINITY ? 0.f : m;
  float l = 0.f;
#pragma unroll
  for (int e = 0; e < E; ++e) acc[e] = 0.f;
  for (int i0 = 0; i0 < mine; i0 += 64) {
    const f32x2 ml = i0 == 0 ? ml0 : i0 + lane < mine ? *(const f32x2*)(a.part_ml + 2 * part(w + (i0 + lane) * WPS)) : none;
    const float wt = ml[1] == 0.f ? 0.f : exp2f(ml[0] - m_eff);
    l = fmaf(ml[1], wt, l);
    const int n = min(64, mine - i0);
    auto weight = [&](int i) { return __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(wt), i)); };
    if (i0 == 0) {
#pragma unroll
      for (int i = 0; i < kEarly; ++i)
        if (i < n)
#pragma unroll
          for (int e = 0; e < E; ++e) acc[e] = fmaf(x[i][e], weight(i), acc[e]);
    }
#pragma unroll 1
    for (int i = i0 == 0 ? kEarly : 0; i < n; i += kBatch) {
      float y[kBatch][E];
#pragma unroll
      for (int j = 0; j < kBatch; ++j) {
        const float* at = a.part_acc + part(w + (i0 + min(i + j, n - 1)) * WPS) * D + lane;
#pragma unroll
        for (int e = 0; e < E; ++e) y[j][e] = at[64 * e];
      }
#pragma unroll
      for (int j = 0; j < kBatch; ++j)
        if (i + j < n)
#pragma unroll
          for (int e = 0; e < E; ++e) acc[e] = fmaf(y[j][e], weight(i + j), acc[e]);
    }
  }
#pragma unroll
  for (int off = 32; off >= 1; off >>= 1) l += __shfl_xor(l, off);
  float top = m_eff;
  if constexpr (WPS > 1) {
#pragma unroll
    for (int e = 0; e < E; ++e) s_sum[wave][lane + 64 * e] = acc[e];
    if (lane == 0) {
      s_sum[wave][D] = m;
      s_sum[wave][D + 1] = l;
    }
    __syncthreads();
    if (w != 0) return;
#pragma unroll
    for (int v = 1; v < WPS; ++v) m = fmaxf(m, s_sum[wave + v][D]);
    top = m == -INFINITY ? 0.f : m;
    l = 0.f;
#pragma unroll
    for (int e = 0; e < E; ++e) acc[e] = 0.f;
#pragma unroll
    for (int v = 0; v < WPS; ++v) {
      const float mv = s_sum[wave + v][D], lv = s_sum[wave + v][D + 1];
      const float wv = lv == 0.f ? 0.f : exp2f((mv == -INFINITY ? 0.f : mv) - top);
      l = fmaf(lv, wv, l);
#pragma unroll
      for (int e = 0; e < E; ++e) acc[e] = fmaf(s_sum[wave + v][lane + 64 * e], wv, acc[e]);
    }
  }
  if (!on) return;
  const int n = sp.slot0 + slot, t = n / G;
  const long long qrow = (long long)(sp.row0 + t) * a.Hq + sp.h * G + (n - t * G);
  const float inv = l == 0.f ? 0.f : 1.f / l;
#pragma unroll
  for (int e = 0; e < E; ++e) a.o[qrow * D + lane + 64 * e] = (bf16)(acc[e] * inv);
  if (lane == 0) a.lse[qrow] = l == 0.f ? -INFINITY : top * kLn2 + logf(l);
}

// FEW: eight waves a slot.  Else a wave a slot, but for entries of more than `longer` parts.
template <int D, bool FEW>
__global__ __launch_bounds__(64 * kJoinWaves) void paged_join_kernel(const PagedArgs a, int longer) {
  __shared__ float s_sum[kJoinWaves][D + 2];
  const Split sp = a.split[blockIdx.x];
  if (a.by_group) {  // an entry is there if its request has such a round
    const int g = blockIdx.x / a.rounds, round = blockIdx.x - g * a.rounds;
    if (request(a, g / a.Hkv).n * (a.Hq / a.Hkv) <= round * kSlots) return;
  }
  if (sp.parts == 0) return;
  const int y = blockIdx.y;
  if (FEW || sp.parts > longer) {
    for (int slot = y; slot < sp.slots; slot += gridDim.y) {
      if (slot != y) __syncthreads();  // the last slot's sums have been read
      join_slot<D, kJoinWaves>(a, sp, slot, s_sum);
    }
  } else if (y * kJoinWaves < sp.slots) {
    join_slot<D, 1>(a, sp, y * kJoinWaves + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), s_sum);
  }
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

// Query slots of a group at most, and the bytes of the partial states and entries of `waves` waves.
static int paged_slots(int Hq, int Hkv, int max_new) { return std::min(kSlots, max_new * (Hq / Hkv)); }
static size_t paged_bytes(int waves, int M, int D) {
  return (size_t)waves * (2 * (size_t)M * (D + 2) * sizeof(float) + sizeof(Split));
}

extern "C" int paged_attn_workspace(int R, int Hq, int Hkv, int D, int max_new, size_t* bytes) {
  g_err.clear();
  if (!bytes) return set_err(RA_EINVAL, "null pointer argument");
  if (int e = paged_check_heads(R, Hq, Hkv, D, max_new)) return e;
  *bytes = paged_bytes(max_workers(D), paged_slots(Hq, Hkv, max_new), D);
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
  const bool f8 = kv_type == RA_KV_E4M3;
  const int M = paged_slots(Hq, Hkv, max_new);
  const int rounds = (int)(((long long)max_new * (Hq / Hkv) + kSlots - 1) / kSlots);
  const size_t need = paged_bytes(max_workers(D), M, D);
  static_assert(workers(64, false) >= kMaxHeads && workers(128, false) >= kMaxHeads, "a team at least");
  const int nw = workers(D, f8);
  if (workspace && workspace_bytes < need)
    return set_err(RA_EINVAL, "workspace of %zu bytes, %zu needed", workspace_bytes, need);
  const long long groups = (long long)R * Hkv * rounds;
  // Groups that the rows can make, whatever max_new allows (by rounds of slots): rounds hold round_rows
  // rows or more, so that n rows take 1 + (n - 1) / round_rows at most (a row of more slots than a round
  // holds, rounds_row).  One launch gives request r as many as lie between first(r) and first(r + 1) in the
  // kernel, which its first row says and which is no fewer.
  const int some = std::min(R, T), G = Hq / Hkv;
  const int round_rows = std::max(1, kSlots / G), rounds_row = (G + kSlots - 1) / kSlots;
  const long long real = std::min(groups, Hkv * (long long)rounds_row * (some + (T - some) / round_rows));
  const long long numbers = Hkv * (G <= kSlots ? (long long)R + T / round_rows : (long long)T * rounds_row);
  const bool by_rows = numbers < groups;  // (never without cu_rows: max_new is 1 then)
  // Short requests, by what their tables can hold: one launch, a workgroup a group.  One wave each
  // where the groups fill the chip or the tiles (64 keys, 32 of 256-byte rows) are few, four waves where
  // they do not and their turns take no longer than a second launch; else shares of all tiles and that
  // second launch.  us with one wave, four, shares; one token a request, of a quarter of the keys to all:
  //   1024 groups of 128 dims in bf16: 120 keys 14.5, 22.4, 22.4; 500 39.2, 47.1, 40.2; 1000 78.4, 88.0,
  //   72.0.  512 groups: 120 9.8, 10.6, 15.9; 500 31.1, 26.0, 26.6; 1000 55.7, 41.3, 35.8; 1500 79.3, 55.4,
  //   45.7.  128 groups: 250 14.5, 8.1, 11.2; 1000 52.0, 18.7, 19.9; 1500 75.3, 25.2, 22.6; in 8 bits 1000
  //   43.5, 15.8, 18.5; 2000 83.5, 28.2, 22.1.  16 groups: 120 8.8, 8.0, 11.4; 500 25.9, 10.7, 12.0; 1000
  //   48.3, 17.4, 12.0.  256 groups of 64 dims in bf16: 500 17.6, 9.1, 14.6; 2000 61.4, 26.3, 25.6.
  // Four waves, shares; of a third of the keys to all:  58 groups, one token 1000 18.3, 18.0; 1500 25.1, 17.6;
  //   four tokens of 8 heads 1000 21.3, 33.4; 1500 27.9, 32.6.  32 groups 600 12.4, 12.5; 1000 17.3, 13.1.
  //   320 groups, four tokens of 4 heads 600 30.0, 29.1; 1000 41.3, 33.4; in 8 bits 600 28.2, 27.2.
  const long long keys = (long long)max_pages * page_size, kt = f8 || D == 64 ? 64 : 32, tiles = (keys + kt - 1) / kt;
  int gw = 0;
  if (real >= 1024) gw = keys <= 768 ? 1 : 0;
  else if (real > 256) gw = tiles <= 8 ? 1 : keys <= 768 ? 4 : 0;
  else gw = tiles <= 2 ? 1 : keys <= (real > 48 ? 1152 : 640) ? 4 : 0;
  CallResources res(stream);
  if (!workspace && gw == 0) {  // (one launch keeps nothing in it)
    if ((rc = res.alloc(paged_bytes(nw, M, D)))) return rc;
    workspace = res.ws;
  }
  PagedArgs a{(const bf16*)q, k_pages, v_pages, k_scales, v_scales, block_table, lens, cu_rows, (bf16*)o, lse, nullptr,
              nullptr, nullptr, T, R, Hq, Hkv, n_pages, 0, max_pages, max_new, M, rounds, groups <= nw, nw / Hkv,
              by_rows ? round_rows : 0, rounds_row, 1.f / sqrtf((float)D)};
  if (gw == 0) {
    a.part_acc = (float*)workspace;
    a.part_ml = a.part_acc + (size_t)nw * 2 * M * D;
    a.split = (Split*)(a.part_ml + (size_t)nw * 2 * M * 2);
  }
  while ((1 << a.page_shift) < page_size) ++a.page_shift;
  auto launch = [&](auto* share, auto* one, auto* four) {
    auto* kern = gw == 0 ? share : gw == 1 ? one : four;
    const unsigned grid = gw == 0 ? nw / kShareWaves : (unsigned)(by_rows ? numbers : groups);
    return timed_launch(RA_KERNEL_DECODE, stream, [&] {
      hipLaunchKernelGGL(kern, dim3(grid), dim3(64 * (gw ? gw : kShareWaves)), 0, stream, a);
      return hipGetLastError();
    });
  };
  RA_HIP(D == 128 ? (f8 ? launch(paged_attn_kernel<128, true, 0>, paged_attn_kernel<128, true, 1>,
                                 paged_attn_kernel<128, true, 4>)
                        : launch(paged_attn_kernel<128, false, 0>, paged_attn_kernel<128, false, 1>,
                                 paged_attn_kernel<128, false, 4>))
                  : (f8 ? launch(paged_attn_kernel<64, true, 0>, paged_attn_kernel<64, true, 1>,
                                 paged_attn_kernel<64, true, 4>)
                        : launch(paged_attn_kernel<64, false, 0>, paged_attn_kernel<64, false, 1>,
                                 paged_attn_kernel<64, false, 4>)));
  if (gw) return RA_OK;
  // Few groups: many parts each, a workgroup a slot.  Many: few parts, a wave a slot; but of requests of
  // very different lengths one may still have a part of every team.  Where the teams are many, the slots of
  // entries of more than kLongParts parts are dealt to workgroups of their own, 2048 in all at most, for
  // most find nothing to do (400 entries of 32 slots: 124 us with a workgroup a slot, 96 so); with up to
  // 256 parts a wave a slot will do.  One request of 60000 tokens alone, 8 heads over one key head: 27 us;
  // among 69 of five tokens 104 with a wave a slot, 30 so; among 900 84 and 62.
  const bool few = groups <= 64, long_lists = !few && a.teams > 256;
  const int entries = a.by_group ? (int)groups : nw, least = (M + kJoinWaves - 1) / kJoinWaves;
  const dim3 grid(entries, few ? M : long_lists ? std::min(M, std::max(least, 2048 / entries)) : least);
  auto* join = D == 128 ? (few ? paged_join_kernel<128, true> : paged_join_kernel<128, false>)
                        : (few ? paged_join_kernel<64, true> : paged_join_kernel<64, false>);
  hipLaunchKernelGGL(join, grid, dim3(64 * kJoinWaves), 0, stream, a, long_lists ? kLongParts : INT_MAX);
  RA_HIP(hipGetLastError());
  return RA_OK;
}
