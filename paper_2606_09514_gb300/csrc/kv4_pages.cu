// The pages of a 4-bit cache that a query is likely to need: each page's bounds of the keys
// (buddy_kv4_bounds) and each query's best pages by them (buddy_kv4_select).  Attention
// over those lists is a form of the few-row kernel (kv4_attn.cu), or a kernel of its own (kv4_lists.cu).
//
// For a channel c of a page's keys let lo_c <= k_pc <= hi_c.  Then for any position p
//   q . k_p <= sum_c max(q_c, 0) hi_c + min(q_c, 0) lo_c,
// and, summed over the query heads of a KV head, which share a selection,
//   score = sum_c a_c hi_c + sum_c b_c lo_c,   a_c = sum_h max(q_hc, 0), b_c = sum_h min(q_hc, 0):
// two products of vectors per page, whatever the number of heads.  A selection is whole
// numbers, in which the last bit of a score shows; so the order of every sum is fixed, without
// fused multiply-adds (include/buddy.h), and any program can follow it bit by bit.
#include <cuda_runtime.h>

#include <algorithm>
#include <type_traits>

#include "common.cuh"
#include "internal.h"
#include "kv4_attn.cuh"

namespace buddy {

bool kv4_cache_ok(const buddy_kv4_cache* c);
kv4::Pages kv4_pages(const buddy_kv4_cache* c);

namespace kv4 {

// A sequence's tokens t0 .. t0 + m - 1 and its n positions; false where they are bad.
__device__ __forceinline__ bool rows_of(const buddy_kv4_seqs& S, int shift, int i, Rows* s) {
  s->t0 = S.row_start ? S.row_start[i] : i;
  const int t1 = S.row_start ? S.row_start[i + 1] : i + 1;
  s->n = S.kv_len[i];
  s->m = t1 - s->t0;
  return s->t0 >= 0 && t1 >= s->t0 && t1 <= S.n_tok && s->m <= S.max_new && s->n >= 0 &&
         s->n <= (int64_t)S.max_pages << shift;
}

// ------------------------------------------------------------------ bounds
constexpr int kBoundWarps = 4;

struct BoundArgs {
  buddy_kv4_seqs s;
  Pages p;
  __half* bounds;
  int32_t* flags;
  int cols;                             // pages that the new tokens of a sequence can lie in
};

__device__ __forceinline__ __half2 shfl_xor(__half2 v, int o) {
  return as_h2(__shfl_xor_sync(0xffffffffu, h2(v), o));
}

// A warp has a page's keys of one head: HD / 16 lanes a position, 16 channels a lane, smallest
// and largest of them in registers, then over the lanes.  The values are exact in half
// (kv4.cuh), and so are the bounds. What is recomputed is the page as it stands, not what the
// call has added to it: no order of writes and no earlier bounds show in the result.
//
// Bound by instructions: 120,001 positions of 8 KV heads (77 MB) take 19.4 us, 4.0 TB/s, of which a word of
// eight channels costs thirteen logical or comparing instructions and six of the products'. (Up to 16
// positions per lane on their way; with 8 20.0 us. Comparisons of three fp32 values at once: 29.8 us.)
// The last pages of 250 sequences take 3.7 us, the chain of length, page id and keys.  There are CTAs for as many pages of every
// sequence as the longest piece of the call may have, which find that they have none: 249 single tokens next to a prompt of
// 2,000 take 19 us, of 100,000 800 (the prompt alone: 15).
template <int HD>
__global__ void __launch_bounds__(32 * kBoundWarps) kv4_bounds_kernel(const BoundArgs A) {
  constexpr int LPR = HD / 16, RPL = 32 / LPR;     // lanes per position, positions per load
  const int lane = threadIdx.x & 31, tl = lane % LPR, row = lane / LPR;
  pdl_wait();
  pdl_trigger();
  const int64_t unit = (int64_t)blockIdx.x * kBoundWarps + (threadIdx.x >> 5);
  const int g = (int)(unit % A.p.nkv);
  const int64_t x = unit / A.p.nkv;
  const int i = (int)(x / A.cols), col = (int)(x % A.cols);
  if (i >= A.s.batch) return;
  Rows s;
  const bool ok = rows_of(A.s, A.p.shift, i, &s);
  if (!ok) {
    if (col == 0 && g == 0 && lane == 0 && A.flags) atomicOr(A.flags, BUDDY_DEV_BAD_POSITION);
    return;
  }
  const int page = (max(0, s.n - s.m) >> A.p.shift) + col;
  if (s.m == 0 || (int64_t)page << A.p.shift >= s.n) return;
  const int id = A.s.table[(int64_t)i * A.s.max_pages + page];
  if ((uint32_t)id >= (uint32_t)A.p.n_pages) {
    if (g == 0 && lane == 0 && A.flags) atomicOr(A.flags, BUDDY_DEV_BAD_PAGE);
    return;
  }
  const uint8_t* const blk = A.p.k + block_at<HD>(A.p, id, g);
  const uint8_t* const codes = blk + 8 * tl;
  const __half* const scales = reinterpret_cast<const __half*>(blk + ((int64_t)code_bytes(HD) << A.p.shift)) + tl / 2;
  const int end = min(1 << A.p.shift, s.n - (page << A.p.shift));
  __half2 lo[8], hi[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) lo[e] = __half2half2(__ushort_as_half(0x7C00)), hi[e] = __half2half2(__ushort_as_half(0xFC00));
  // N positions of the lane's, the first of them r0; CHECK: up to the sequence's end
  auto take = [&](auto number, auto check, int r0) {
    constexpr int N = decltype(number)::value;
    constexpr bool CHECK = decltype(check)::value;
    const uint8_t* const c = codes + r0 * code_bytes(HD);
    const __half* const sc = scales + r0 * (scale_bytes(HD) / 2);
    uint2 w[N];
    __half s0[N];
#pragma unroll
    for (int j = 0; j < N; ++j) {
      if (CHECK && r0 + j * RPL >= end) continue;
      w[j] = *reinterpret_cast<const uint2*>(c + j * RPL * code_bytes(HD));
      s0[j] = sc[j * RPL * (scale_bytes(HD) / 2)];
    }
#pragma unroll
    for (int j = 0; j < N; ++j) {
      if (CHECK && r0 + j * RPL >= end) continue;
      const __half2 s1 = __half2half2(s0[j]), s72 = __hmul2(s1, __float2half2_rn(-72.f));
      uint32_t v[8];
      dequant4(w[j].x, s1, s72, v);
      dequant4(w[j].y, s1, s72, v + 4);
#pragma unroll
      for (int e = 0; e < 8; ++e) lo[e] = __hmin2_nan(lo[e], as_h2(v[e])), hi[e] = __hmax2_nan(hi[e], as_h2(v[e]));
    }
  };
  auto whole = [&](auto number) {                  // a page in one go, or in several
    constexpr int N = decltype(number)::value;
#pragma unroll 1
    for (int r0 = row; r0 < end; r0 += N * RPL) take(number, std::false_type(), r0);
  };
  constexpr int FEW = 16 / RPL;                    // 16 positions of the warp
  const int loads = (1 << A.p.shift) / RPL;
  if (end < 1 << A.p.shift) {
#pragma unroll 1
    for (int r0 = row; r0 < end; r0 += FEW * RPL) take(std::integral_constant<int, FEW>(), std::true_type(), r0);
  } else if (loads >= 16) {
    whole(std::integral_constant<int, 16>());
  } else if (loads == 8) {
    whole(std::integral_constant<int, 8>());
  } else if (loads == 4) {
    whole(std::integral_constant<int, 4>());
  } else {
    whole(std::integral_constant<int, 2>());
  }
#pragma unroll
  for (int o = LPR; o < 32; o <<= 1)
#pragma unroll
    for (int e = 0; e < 8; ++e) lo[e] = __hmin2_nan(lo[e], shfl_xor(lo[e], o)), hi[e] = __hmax2_nan(hi[e], shfl_xor(hi[e], o));
  if (row < 2) {
    uint4* const d = reinterpret_cast<uint4*>(A.bounds + (((int64_t)id * A.p.nkv + g) * 2 + row) * HD + 16 * tl);
    uint32_t y[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) y[e] = row ? h2(hi[e]) : h2(lo[e]);
    d[0] = make_uint4(y[0], y[1], y[2], y[3]);
    d[1] = make_uint4(y[4], y[5], y[6], y[7]);
  }
}

// ------------------------------------------------------------------ selection
constexpr int kSelWarps = 8;            // of a CTA at most
constexpr int kSelMaxPages = 40000;     // a score each in shared memory, next to the copies in flight (a multiple of 32)
constexpr int kSelCluster = 16;         // most CTAs of a (token, KV head)
constexpr int kSelTokens = 4;           // most tokens of a sequence that share a walk
constexpr int kSelShared = 8192;        // scores of a token up to which they do
constexpr int kSelPairs = 512;          // up to which they do so over two heads' bounds
constexpr int kSelBins = 256;

struct SelectArgs {
  buddy_kv4_select_args a;
  Pages p;
  int G;
  int slots;                            // scores of a token: entries of a table row that may be among them
  int chunks;                           // CTAs per head of a sequence, TT tokens each; 0: a CTA for each token
  float minus_zero;
  int32_t* flags;
};

// Scores in an order of whole numbers: a NaN above all, what has no page (0) below all.
__device__ __forceinline__ uint32_t key_of(float s) {
  if (isnan(s)) return 0xFFFFFFFFu;
  const uint32_t u = __float_as_uint(__fadd_rn(s, 0.f));    // (-0 is 0)
  return u & 0x80000000u ? ~u : u | 0x80000000u;
}

// The sequence of token t: the last one that begins at t or before, over the warp; -1: none.
__device__ __forceinline__ int seq_of(const buddy_kv4_seqs& S, int t, int lane) {
  if (!S.row_start) return t;
  int lo = 0, hi = S.batch + 1;
  while (hi - lo > 1) {
    const int step = (hi - lo + 31) / 32, at = lo + lane * step;
    const int c = __popc(__ballot_sync(0xffffffffu, at < hi && S.row_start[min(at, S.batch)] <= t));
    if (c == 0) return -1;
    lo += (c - 1) * step;
    hi = min(hi, lo + step);
  }
  return lo < S.batch ? lo : -1;
}

// The same by one thread.
__device__ __forceinline__ int seq_of(const buddy_kv4_seqs& S, int t) {
  int lo = -1, hi = S.batch + 1;
  while (hi - lo > 1) {
    const int mid = (lo + hi) / 2;
    if (S.row_start[mid] <= t) lo = mid;
    else hi = mid;
  }
  return lo < S.batch ? lo : -1;
}

// A word of the first CTA's shared memory, from any CTA of its cluster.
__device__ __forceinline__ void put_first(uint32_t* at, uint32_t v) {
  asm volatile("st.shared::cluster.u32 [%0], %1;" ::"r"(ptx::dsmem_addr(at, 0)), "r"(v) : "memory");
}

// Two fp32 at once, each rounded as alone.  A product is a fused multiply-add with a -0 that the
// compiler does not know: of a packed product and a packed sum it would make one operation with
// one rounding.
using F2 = uint64_t;
__device__ __forceinline__ F2 pair(float a, float b) {
  F2 r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(a), "f"(b));
  return r;
}
__device__ __forceinline__ F2 product2(F2 a, F2 b, F2 minus_zero) {
  F2 r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(minus_zero));
  return r;
}
__device__ __forceinline__ F2 sum2(F2 a, F2 b) {
  F2 r;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}

// Sums over the lanes of a page, in the order of the scores: the eights of lo and of hi by
// halves, then both. Of V values a lane gives half away at each step, as long as it has two, so
// that there is about one exchange per sum; it is left with those from first_sum() on, in the
// first places.
template <int HD>
__device__ __forceinline__ constexpr int sum_steps() { return HD == 128 ? 4 : 3; }
template <int HD>
__device__ __forceinline__ constexpr int sum_bit(int step) {   // 4 2 1 8, or 2 1 4
  return step < sum_steps<HD>() - 1 ? HD / 32 >> step : HD / 16;
}
template <int HD, int V>
__device__ __forceinline__ int first_sum(int lane) {
  int at = 0, n = V;
#pragma unroll
  for (int step = 0; step < sum_steps<HD>(); ++step)
    if (n > 1) n /= 2, at += lane & sum_bit<HD>(step) ? n : 0;
  return at;
}
template <int HD, int V>
__device__ __forceinline__ void sum_lanes(float (&v)[V], int lane) {
  int n = V;
#pragma unroll
  for (int step = 0; step < sum_steps<HD>(); ++step) {
    const int bit = sum_bit<HD>(step);
    if (n > 1) {
      n /= 2;
      const bool up = lane & bit;
#pragma unroll
      for (int i = 0; i < V / 2; ++i) {
        if (i < n) {
          const float give = up ? v[i] : v[i + n], keep = up ? v[i + n] : v[i];
          v[i] = __fadd_rn(keep, __shfl_xor_sync(0xffffffffu, give, bit));
        }
      }
    } else {
      v[0] = __fadd_rn(v[0], __shfl_xor_sync(0xffffffffu, v[0], bit));
    }
  }
}

// The warps that look for a token's best pages: WARPS of a CTA's, the bar-th such group.
template <int WARPS>
struct Group {
  int tid, lane, warp, bar;
  __device__ __forceinline__ void sync() const {
    if constexpr (WARPS == 1) __syncwarp();
    else asm volatile("bar.sync %0, %1;" ::"r"(bar + 1), "n"(32 * WARPS) : "memory");
  }
};

// What a thread has of M keys, and the ids of their pages: a warp those from `first` on, 32 at a
// time. Up to KEPT of them stay in registers, more in shared memory.
template <int WARPS, int KEPT>
struct Keys {
  const uint32_t* all;
  const int32_t* ids;
  int first, end;                                  // of the warp
  bool few;
  uint32_t kept[KEPT];
  int32_t page[KEPT];
  __device__ __forceinline__ Keys(const uint32_t* keys, const int32_t* row, int M, const Group<WARPS>& G) : all(keys), ids(row) {
    const int run = (M + 32 * WARPS - 1) / (32 * WARPS) * 32;
    first = G.warp * run;
    end = min(M, first + run);
    few = run <= KEPT * 32;
    if (few) {
#pragma unroll
      for (int k = 0; k < KEPT; ++k) page[k] = there(k, G.lane) ? row[first + 32 * k + G.lane] : 0;
#pragma unroll
      for (int k = 0; k < KEPT; ++k) kept[k] = there(k, G.lane) ? keys[first + 32 * k + G.lane] : 0u;
    }
  }
  __device__ __forceinline__ bool there(int k, int lane) const { return first + 32 * k + lane < end; }
  // smallest and largest of the warp's
  __device__ __forceinline__ void range(int lane, uint32_t* lo, uint32_t* hi) const {
    uint32_t a = 0xFFFFFFFFu, b = 0u;
    if (few) {
#pragma unroll
      for (int k = 0; k < KEPT; ++k)
        if (there(k, lane)) a = min(a, kept[k]), b = max(b, kept[k]);
    } else {
#pragma unroll 4
      for (int j = first + lane; j < end; j += 32) a = min(a, all[j]), b = max(b, all[j]);
    }
    *lo = __reduce_min_sync(0xffffffffu, a);
    *hi = __reduce_max_sync(0xffffffffu, b);
  }
  // f(key) of those in [lo, hi]
  template <typename F>
  __device__ __forceinline__ void within(uint32_t lo, uint32_t hi, int lane, F&& f) const {
    if (few) {
#pragma unroll
      for (int k = 0; k < KEPT; ++k)
        if (there(k, lane) && kept[k] - lo <= hi - lo) f(kept[k]);
    } else {
#pragma unroll 4
      for (int j = first + lane; j < end; j += 32) {
        const uint32_t k = all[j];
        if (k - lo <= hi - lo) f(k);
      }
    }
  }
};

// A group's scratch.
constexpr int kSelFew = 64;
struct Search {
  __align__(16) int bins[kSelBins];                // zeros before and after
  __align__(16) uint32_t few[kSelFew];
  int n_few;                                       // as bins
  int above[kSelWarps], equal[kSelWarps];          // of each warp
  uint32_t lo[kSelWarps], hi[kSelWarps];
};

// The r-th largest of n <= kSelFew keys (16-byte aligned, readable to a multiple of four), by every warp.
__device__ __forceinline__ uint32_t rank_few(const uint32_t* few, int n, int r, int lane) {
  const uint32_t k0 = lane < n ? few[lane] : 0u, k1 = lane + 32 < n ? few[lane + 32] : 0u;
  int g0 = 0, g1 = 0, e0 = 0, e1 = 0;              // larger ones, equal ones
  auto count = [&](uint32_t k) { g0 += k > k0, e0 += k == k0, g1 += k > k1, e1 += k == k1; };
#pragma unroll 2
  for (int x = 0; x < n; x += 4) {
    const uint4 k = *reinterpret_cast<const uint4*>(few + x);
    count(k.x);
    if (x + 1 < n) count(k.y);
    if (x + 2 < n) count(k.z);
    if (x + 3 < n) count(k.w);
  }
  const uint32_t h0 = __ballot_sync(0xffffffffu, lane < n && g0 < r && g0 + e0 >= r);
  const uint32_t h1 = __ballot_sync(0xffffffffu, lane + 32 < n && g1 < r && g1 + e1 >= r);
  return h0 ? __shfl_sync(0xffffffffu, k0, __ffs(h0) - 1) : __shfl_sync(0xffffffffu, k1, __ffs(h1) - 1);
}

// How many of m keys (16-byte aligned, zeros behind them up to a multiple of 32) come before that of
// index j0 + lane: larger ones, and of the equal ones those with a lower index.
constexpr int kSelRanked = 64;       // keys up to which each is ranked by itself
__device__ __forceinline__ int rank_of(const uint32_t* keys, int m, uint32_t mine, int j0, int lane) {
  int n = 0;
  auto block = [&](int b, auto before) {
#pragma unroll
    for (int x = 0; x < 32; x += 4) {
      const uint4 k = *reinterpret_cast<const uint4*>(keys + b + x);
      n += before(k.x, x) + before(k.y, x + 1) + before(k.z, x + 2) + before(k.w, x + 3);
    }
  };
#pragma unroll 1
  for (int b = 0; b < j0; b += 32) block(b, [&](uint32_t k, int) { return (int)(k >= mine); });
  block(j0, [&](uint32_t k, int x) { return (int)(k > mine || (k == mine && x < lane)); });
#pragma unroll 1
  for (int b = j0 + 32; b < m; b += 32) block(b, [&](uint32_t k, int) { return (int)(k > mine); });
  return n;
}

// Where the best r of the keys end: just r of them are above what is returned, or these and the first
// of those equal to it. By counts of the keys in 256 parts of the range [lo, hi] that holds the r-th,
// from the top, until a part's keys are all wanted, are few, or are one value.
template <int WARPS, int KEPT>
__device__ __forceinline__ uint32_t threshold(const Keys<WARPS, KEPT>& keys, int r, Search& S, const Group<WARPS>& G) {
  uint32_t lo, hi;
  keys.range(G.lane, &lo, &hi);
  if (WARPS > 1) {
    if (G.lane == 0) S.lo[G.warp] = lo, S.hi[G.warp] = hi;
    G.sync();
#pragma unroll
    for (int w = 0; w < WARPS; ++w) lo = min(lo, S.lo[w]), hi = max(hi, S.hi[w]);
  }
  for (;;) {
    const int shift = max(0, 32 - __clz(hi - lo) - 8);       // ((hi - lo) >> shift) < 256
    keys.within(lo, hi, G.lane, [&](uint32_t k) { atomicAdd(&S.bins[(k - lo) >> shift], 1); });
    G.sync();
    // every warp: lane x has the parts from 255 - 8 x down
    const int4* const mine = reinterpret_cast<const int4*>(S.bins + 248 - 8 * G.lane);
    const int4 y0 = mine[1], y1 = mine[0];
    const int c[8] = {y0.w, y0.z, y0.y, y0.x, y1.w, y1.z, y1.y, y1.x};
    int sum = 0;
#pragma unroll
    for (int e = 0; e < 8; ++e) sum += c[e];
    int upto = sum;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int y = __shfl_up_sync(0xffffffffu, upto, o);
      if (G.lane >= o) upto += y;
    }
    const int src = __ffs(__ballot_sync(0xffffffffu, upto >= r)) - 1;
    int before = upto - sum, part = 255 - 8 * G.lane, in = c[0];
#pragma unroll
    for (int e = 1; e < 8; ++e)
      if (before + in < r) before += in, in = c[e], part = 255 - 8 * G.lane - e;
    before = __shfl_sync(0xffffffffu, before, src);
    part = __shfl_sync(0xffffffffu, part, src);
    in = __shfl_sync(0xffffffffu, in, src);
    r -= before;
    lo += (uint32_t)part << shift;
    hi = lo + min(hi - lo, (1u << shift) - 1);
    G.sync();                                      // (the counts have been read)
    for (int b = G.tid; b < kSelBins; b += 32 * WARPS) S.bins[b] = 0;
    if (shift == 0) return lo;
    if (in == r) return lo - 1;                    // (lo > 0: not all of the keys are wanted)
    if (in <= kSelFew) {
      int n = 0;
      keys.within(lo, hi, G.lane, [&](uint32_t) { ++n; });
      if (n > 0) {
        uint32_t* to = S.few + atomicAdd(&S.n_few, n);
        keys.within(lo, hi, G.lane, [&](uint32_t k) { *to++ = k; });
      }
      G.sync();
      if (G.tid == 0) S.n_few = 0;
      return rank_few(S.few, in, r, G.lane);
    }
    G.sync();
  }
}

__device__ __forceinline__ void copy16(uint32_t dst, const void* src, bool there) {   // zeros where there is nothing
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(there ? 16 : 0) : "memory");
}

// The forms of the kernel: one token by a CTA, one by a cluster (CL), up to TT = 4 of a sequence by a
// CTA, for one KV head or two (HG). Warps and those that look for the pages of one token and head;
// loads of a turn of a warp (two copies of 16 bytes per lane each) and turns in flight.
template <int TT, int HG, bool CL>
struct Form {
  static constexpr int kWarps = TT == 1 && !CL ? 4 : 8, kThreads = 32 * kWarps, kLoads = TT == 1 ? 4 : 2, kTurns = TT == 1 ? 2 : 4;
  // (kCtas by registers: with the ring's shared memory a CTA of one token is there six times an SM at most)
  static constexpr int kGroup = kWarps / (TT * HG), kKept = TT == 1 ? (CL ? 8 : 4) : 16, kCtas = TT == 1 && !CL ? 7 : 2;
  static constexpr int kRing = kWarps * kTurns * kLoads * 1024;   // bytes
  // shared memory of a call with so many scores per token, and of any call
  static constexpr int smem(int slots) { return kRing + (int)sizeof(uint32_t) * HG * TT * slots; }
  static constexpr int kMostSmem = smem(TT == 1 ? kSelMaxPages : HG == 1 ? kSelShared : kSelPairs);
};

// Up to TT tokens of a sequence share a walk over its pages' bounds; the CTA of the first of
// them does the work of all. CL: a cluster has one token, its CTAs the pages in turn, and the first
// one the scores. A page has HD / 8 lanes: the lower ones two eights each of the smallest of its
// channels, by b, the upper ones of the largest, by a; the two eights are those that the
// score's sum takes first, and go side by side through packed instructions. Every lane reads what
// it has copied itself, so that the turns in flight need neither registers nor barriers. Two heads'
// bounds of a page lie next to each other and go to neighbouring lanes.
//
// Bound by latencies where tokens are few: one token of 32 heads over 8 takes 7.7 us over 1,876 pages
// (7.7 MB); time stamps of the clusters' first CTAs (medians, after the wait for the work before): lengths and page ids 0.7,
// copies on their way 1.3, scores 3.2, the cluster's barrier 3.8, search 5.9, output 6.7. 250 sequences of 8 to 128
// pages, 28 heads over 4 (18 MB), 8.1. By instructions where several tokens share a walk: 31 sequences of up to 750 pages and
// five tokens, 40 KV heads (115 MB), 45 us, 2.5 TB/s; of a CTA's 13.8 us (median) the walk is 8.4, what comes before it 2.1,
// search and output 3.3. What it gained: a search by counts 64.8 -> 11.8 with the clusters (one token), copies
// that need no registers instead of loads 11.8 -> 9.5, packed instructions over pairs of eights and code for
// each number of tokens 62 -> 55 us (31 sequences), the longest sequences first 55 -> 45.
template <typename T, int HD, int TT, int HG, bool CL>
__global__ void __launch_bounds__(Form<TT, HG, CL>::kThreads, Form<TT, HG, CL>::kCtas) kv4_select_kernel(const SelectArgs A) {
  using F = Form<TT, HG, CL>;
  extern __shared__ __align__(128) uint8_t sel_smem[];
  uint32_t* const keys = reinterpret_cast<uint32_t*>(sel_smem + F::kRing);   // [HG][TT][slots, a multiple of 32]
  constexpr int WARPS = F::kWarps, THREADS = F::kThreads;
  __shared__ Search search[HG * TT];
  __shared__ __align__(16) float s_q[HG * TT][2][HD];   // a token's b, then its a
  __shared__ __align__(16) int s_len[TT > 1 ? THREADS : 4];
  __shared__ int4 s_seq;
  static_assert((!CL || TT == 1) && (HG == 1 || TT > 1), "");
  constexpr int LPP = HD / 8, PPW = 32 / LPP / HG; // lanes of a head's page, pages of a warp's load
  constexpr int LOADS = F::kLoads;
  constexpr int TURNS = F::kTurns, PAGES = LOADS * PPW, IDS = 32 / PAGES;   // turns whose ids a warp reads at once
  const buddy_kv4_select_args& a = A.a;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const uint32_t rank = CL ? ptx::cluster_rank() : 0, C = CL ? ptx::cluster_size() : 1;
  const unsigned unit = blockIdx.x / C;
  const int gs = A.p.nkv / HG, g = (int)(unit % (unsigned)gs) * HG;   // (the first of HG heads)
  int t = (int)(unit / (unsigned)gs), i = 0, chunk = 0;
  const bool by_seq = TT > 1 && A.chunks > 0;
  if (by_seq) {
    i = t / A.chunks, chunk = t % A.chunks;
    if (i >= a.s.batch) {                          // behind the sequences' CTAs: the tokens that are in none
      const int64_t x = ((int64_t)unit - (int64_t)a.s.batch * A.chunks * gs) * THREADS + tid;
      pdl_wait();
      pdl_trigger();
      if (x >= a.s.n_tok) return;
      t = (int)x, i = seq_of(a.s, t);
      Rows s{};
      const bool ok = i >= 0 && rows_of(a.s, A.p.shift, i, &s) && t >= s.t0 && t < s.t0 + s.m;
      if (!ok) a.visible[t] = -1;
      if (!ok && i >= 0 && A.flags) atomicOr(A.flags, BUDDY_DEV_BAD_POSITION);
      return;
    }
  }
  if (!by_seq && t >= a.s.n_tok) {                 // behind the tokens' CTAs: the sequences, of which some have no token
    const int64_t j = (int64_t)(unit - (unsigned)a.s.n_tok * (unsigned)gs) * THREADS + tid;
    pdl_wait();
    pdl_trigger();
    Rows s{};
    if (rank == 0 && j < a.s.batch && !rows_of(a.s, A.p.shift, (int)j, &s) && A.flags) atomicOr(A.flags, BUDDY_DEV_BAD_POSITION);
    return;
  }
  for (int b = tid; b < HG * TT * kSelBins; b += THREADS) search[b / kSelBins].bins[b % kSelBins] = 0;
  if (tid < HG * TT) search[tid].n_few = 0;
  constexpr int PER = (HG * TT * HD + THREADS - 1) / THREADS;
  auto query = [&](int t, int e) {                 // of a head and token
    const int hu = (tid + e * THREADS) / HD;
    return (const T*)a.q + min(t + hu % TT, a.s.n_tok - 1) * a.q_stride + (int64_t)(g + hu / TT) * A.G * HD + tid % HD;
  };
  T x[PER][8];
  auto read_queries = [&](const T* const (&q)[PER]) {
#pragma unroll
    for (int e = 0; e < PER; ++e)
#pragma unroll
      for (int h = 0; h < 8; ++h)
        if ((tid + e * THREADS) / HD < HG * TT && h < A.G) x[e][h] = q[e][h * HD];
  };
  Rows s{};
  bool ok = true;
  if (by_seq) {
    pdl_wait();
    pdl_trigger();
    if (a.s.batch <= THREADS) {                    // the longest sequences first: theirs would be waited for at the end
      ok = tid < a.s.batch && rows_of(a.s, A.p.shift, tid, &s);
      s_len[tid] = tid < a.s.batch ? s.n : INT32_MIN;
      __syncthreads();
      if (tid < a.s.batch) {
        int rank = 0;
        for (int j = 0; j < a.s.batch; j += 4) {
          const int4 y = *reinterpret_cast<const int4*>(s_len + j);
          rank += (y.x > s.n || (y.x == s.n && j < tid)) + (y.y > s.n || (y.y == s.n && j + 1 < tid)) +
                  (y.z > s.n || (y.z == s.n && j + 2 < tid)) + (y.w > s.n || (y.w == s.n && j + 3 < tid));
        }
        if (rank == i) s_seq = make_int4(ok ? tid : -1, s.t0, s.m, s.n);
      }
      __syncthreads();
      const int4 y = s_seq;
      i = y.x;
      s = Rows{y.y, y.z, y.w};
      ok = i >= 0;
    } else {
      ok = rows_of(a.s, A.p.shift, i, &s);
    }
    t = s.t0 + chunk * TT;
    if (!ok && chunk == 0 && g == 0 && tid == 0 && A.flags) atomicOr(A.flags, BUDDY_DEV_BAD_POSITION);
    if (!ok || chunk * TT >= s.m) return;          // (the CTAs behind see to the tokens)
    const T* q[PER];
#pragma unroll
    for (int e = 0; e < PER; ++e) q[e] = query(t, e);
    read_queries(q);
  } else {
    const T* q[PER];
#pragma unroll
    for (int e = 0; e < PER; ++e) q[e] = query(t, e);
    // (the arguments that are wanted first come from memory while the work before this kernel ends)
    asm volatile("" ::"l"(a.s.kv_len), "l"(a.s.table), "l"(a.bounds), "l"(A.flags), "r"(A.G), "r"(A.slots));
    pdl_wait();
    pdl_trigger();
    read_queries(q);                               // (on their way while the token's sequence is looked for)
    i = seq_of(a.s, t, lane);
  }
  // turn n of the warp has the pages from (n C WARPS + rank WARPS + warp) PAGES on; their ids,
  // of IDS turns at once, by lanes (what lies behind the sequence's pages may be anything)
  const int32_t* const row = a.s.table + (int64_t)max(i, 0) * a.s.max_pages;
  const int turn = (int)C * WARPS * PAGES, j_first = ((int)rank * WARPS + warp) * PAGES;
  auto ids_of = [&](int n) {
    const int64_t j = (int64_t)(n + lane / PAGES) * turn + j_first + lane % PAGES;
    return j < A.slots && a.first + j < a.s.max_pages ? row[a.first + j] : -1;
  };
  int ids = ids_of(0), ids_next = ids_of(IDS);
  if (!by_seq) {
    ok = i >= 0;
    if (ok) {
      ok = rows_of(a.s, A.p.shift, i, &s) && t >= s.t0 && t < s.t0 + s.m;
      if (!ok && g == 0 && tid == 0 && rank == 0 && A.flags) atomicOr(A.flags, BUDDY_DEV_BAD_POSITION);
    }
    if (!ok) {
      if (g == 0 && tid == 0 && rank == 0) a.visible[t] = -1;
      return;
    }
    if (TT > 1 && (t - s.t0) % TT != 0) return;    // (the CTA of another token sees to this one)
  }
  const int p0 = s.n - s.m + (t - s.t0);           // of token t; the next ones follow
  const int in_page = (1 << A.p.shift) - 1;
  auto pages_of = [&](int p) { return p < 0 ? 0 : (p >> A.p.shift) + 1; };
  const int tokens = min(TT, s.t0 + s.m - t);
  if (g == 0 && tid < tokens && rank == 0) {
    const int p = p0 + tid, N = pages_of(p);
    a.visible[t + tid] = N == 0 ? 0 : ((min(N, a.budget) - 1) << A.p.shift) + (p & in_page) + 1;
  }
  auto list_of = [&](int u, int hl) { return a.pages + ((int64_t)(t + u) * A.p.nkv + g + hl) * a.budget; };
  const int r = a.budget - a.first - a.last;
  auto scored = [&](int u) { const int N = pages_of(p0 + u); return u < tokens && N > a.budget ? N - a.first - a.last : 0; };
  const int M = scored(tokens - 1);                // of the last token: the most
  // what is in without a score: the ends of long lists, of which a thread reads its first one early, and all of short ones
  // (a list that is too short for a sequence's pages has fewer entries than a table may have: no count passes 32 bits)
  const int ends = min(a.first + a.last, kSelMaxPages);
  auto end_of = [&](int x) {                       // the x-th of all tokens' ends
    const int u = TT == 1 ? 0 : x / ends, j = x - u * ends, N = pages_of(p0 + u);
    return N > a.budget ? row[j < a.first ? j : N - ends + j] : 0;
  };
  const int32_t early = (TT > 1 || CL) && tid < tokens * ends && rank == 0 ? end_of(tid) : 0;
  auto always = [&]() {
    for (int x = tid; x < tokens * ends; x += THREADS) {
      const int u = TT == 1 ? 0 : x / ends, j = x - u * ends;
      if (pages_of(p0 + u) <= a.budget) continue;
      const int32_t id = (TT > 1 || CL) && x == tid ? early : end_of(x);
#pragma unroll
      for (int hl = 0; hl < HG; ++hl) list_of(u, hl)[j < a.first ? j : a.budget - ends + j] = id;
    }
    for (int u = 0; u < tokens && pages_of(p0 + u) <= a.budget; ++u) {
      const int N = pages_of(p0 + u);
      for (unsigned j = tid; j < (unsigned)a.budget; j += THREADS) {   // (a step may pass 2^31)
        const int32_t id = j < (unsigned)N ? row[j] : -1;
#pragma unroll
        for (int hl = 0; hl < HG; ++hl) list_of(u, hl)[j] = id;
      }
    }
  };
  if (M == 0 || r == 0) {                          // (the same in the whole cluster)
    if (rank == 0) always();
    return;
  }
  if (CL) ptx::cluster_arrive_started();

  // ---- scores
  const int turns = M > j_first ? (M - j_first + turn - 1) / turn : 0;
  const uint32_t ring = ptx::smem_u32(sel_smem) + (uint32_t)(warp * TURNS * LOADS * 1024 + lane * 16);
  const int eight = lane % (LPP / 2), high = lane / (LPP / 2) % 2;   // the lane's first of two; of lo or of hi
  const int hl = lane / LPP % HG, pl = lane / LPP / HG;              // its head, and its page of a load's
  const __half* const bounds = (const __half*)a.bounds + ((int64_t)(g + hl) * 2 + high) * HD + eight * 8;
  const int64_t per_page = (int64_t)A.p.nkv * 2 * HD;
  uint32_t gone = 0;                               // of the loads in flight and the one at hand, LOADS bits a turn, the newest lowest
  auto issue = [&](int n, int at) {                // (a turn that is not there copies nothing: the counts of groups go on)
    gone <<= LOADS;
    if (n < turns) {
      if (n > 0 && n % IDS == 0) ids = ids_next, ids_next = ids_of(n + IDS);
      int id[LOADS];
#pragma unroll
      for (int k = 0; k < LOADS; ++k) id[k] = __shfl_sync(0xffffffffu, ids, n % IDS * PAGES + k * PPW + pl);
#pragma unroll
      for (int k = 0; k < LOADS; ++k) {
        const bool there = (uint32_t)id[k] < (uint32_t)A.p.n_pages;
        gone |= there ? 0u : 1u << k;
        const __half* const src = bounds + (there ? id[k] : 0) * per_page;
        copy16(ring + (at * LOADS + k) * 1024, src, there);
        copy16(ring + (at * LOADS + k) * 1024 + 512, src + HD / 2, there);
      }
    }
    asm volatile("cp.async.commit_group;" ::: "memory");
  };
#pragma unroll
  for (int n = 0; n < TURNS; ++n) issue(n, n);
  // (Written out here, the first warp waits for the ids: one token over 1,876 pages 7.9 us instead of 7.7. With many CTAs that
  // wait is filled, and what is kept until later costs: 250 sequences 8.3 instead of 8.0.)
  constexpr bool LATE = TT > 1 || CL;
  if (!LATE) always();
#pragma unroll
  for (int e = 0; e < PER; ++e) {
    const int u = (tid + e * THREADS) / HD, c = tid % HD;
    if (u >= HG * TT) continue;
    float up = 0.f, down = 0.f;
#pragma unroll
    for (int h = 0; h < 8; ++h) {
      if (h >= A.G) continue;
      const float y = to_f(x[e][h]), y0 = isnan(y) ? y : fminf(y, 0.f), y1 = isnan(y) ? y : fmaxf(y, 0.f);
      down = h == 0 ? y0 : __fadd_rn(down, y0);
      up = h == 0 ? y1 : __fadd_rn(up, y1);
    }
    s_q[u][0][c] = down;
    s_q[u][1][c] = up;
  }
  __syncthreads();
  const F2 minus_zero = pair(A.minus_zero, A.minus_zero);
  bool lost = false;
  if (CL) ptx::cluster_wait_started();
  auto score = [&](auto number) {
    constexpr int NT = decltype(number)::value, NP = NT == 3 ? 4 : NT, V = LOADS * NP;   // tokens; scores of a turn
    F2 f[NT][8];                                   // this lane's channels of both eights
#pragma unroll
    for (int u = 0; u < NT; ++u) {
      const float4* const y = reinterpret_cast<const float4*>(&s_q[hl * TT + u][high][eight * 8]);
      const float4 a0 = y[0], a1 = y[1], b0 = y[HD / 8], b1 = y[HD / 8 + 1];
      f[u][0] = pair(a0.x, b0.x), f[u][1] = pair(a0.y, b0.y), f[u][2] = pair(a0.z, b0.z), f[u][3] = pair(a0.w, b0.w);
      f[u][4] = pair(a1.x, b1.x), f[u][5] = pair(a1.y, b1.y), f[u][6] = pair(a1.z, b1.z), f[u][7] = pair(a1.w, b1.w);
    }
    // what a lane is left with of a turn: its page in the first turn, where its token's pages end, and the token
    constexpr int LEFT = V > LPP ? V / LPP : 1;
    // (lanes that differ in these bits only are left with the same)
    constexpr int TWINS = V >= LPP ? 0 : V == LPP / 2 ? LPP / 2 : LPP / 2 + LPP / (2 * V) - 1;
    const int mine_at = first_sum<HD, V>(lane);
    int j_mine[LEFT], j_end[LEFT], u_mine[LEFT];
#pragma unroll
    for (int e = 0; e < LEFT; ++e) {
      u_mine[e] = (mine_at + e) % NP;
      j_mine[e] = j_first + (mine_at + e) / NP * PPW + pl;
      j_end[e] = lane & TWINS ? 0 : scored(u_mine[e]);
    }
    for (int n = 0, at = 0; n < turns; ++n, at = at + 1 == TURNS ? 0 : at + 1) {
      asm volatile("cp.async.wait_group %0;" ::"n"(TURNS - 1) : "memory");
      float v[V];
#pragma unroll
      for (int k = 0; k < LOADS; ++k) {
        const uint8_t* const src = sel_smem + ((warp * TURNS + at) * LOADS + k) * 1024 + lane * 16;
        const uint4 w0 = *reinterpret_cast<const uint4*>(src), w1 = *reinterpret_cast<const uint4*>(src + 512);
        const uint32_t x0[4] = {w0.x, w0.y, w0.z, w0.w}, x1[4] = {w1.x, w1.y, w1.z, w1.w};
        F2 y[8];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float2 y0 = __half22float2(as_h2(x0[e])), y1 = __half22float2(as_h2(x1[e]));
          y[2 * e] = pair(y0.x, y1.x), y[2 * e + 1] = pair(y0.y, y1.y);
        }
#pragma unroll
        for (int u = 0; u < NP; ++u) {
          if (u >= NT) {
            v[k * NP + u] = 0.f;
            continue;
          }
          F2 z[8];
#pragma unroll
          for (int e = 0; e < 8; ++e) z[e] = product2(f[min(u, NT - 1)][e], y[e], minus_zero);
#pragma unroll
          for (int h = 4; h > 0; h /= 2)
#pragma unroll
            for (int e = 0; e < h; ++e) z[e] = sum2(z[e], z[e + h]);
          float s0, s1;
          asm("mov.b64 {%0, %1}, %2;" : "=f"(s0), "=f"(s1) : "l"(z[0]));
          v[k * NP + u] = __fadd_rn(s0, s1);
        }
      }
      sum_lanes<HD, V>(v, lane);
      const uint32_t missing = gone >> ((TURNS - 1) * LOADS);
      issue(n + TURNS, at);                        // (what this turn has read has been used)
#pragma unroll
      for (int e = 0; e < LEFT; ++e) {
        const int j = j_mine[e] + n * turn;
        if (j >= j_end[e]) continue;
        const bool there = !(missing >> ((mine_at + e) / NP) & 1);
        const uint32_t key = there ? key_of(v[e]) : 0u;
        lost |= !there;
        if (CL) put_first(&keys[j], key);
        else keys[(hl * TT + u_mine[e]) * A.slots + j] = key;
      }
    }
  };
  if (TT == 1 || tokens == 1) score(std::integral_constant<int, 1>());
  else if (TT > 1 && tokens == 2) score(std::integral_constant<int, TT == 1 ? 1 : 2>());
  else if (TT > 1 && tokens == 3) score(std::integral_constant<int, TT == 1 ? 1 : 3>());
  else if (TT > 1) score(std::integral_constant<int, TT>());
  if (lost && A.flags) atomicOr(A.flags, BUDDY_DEV_BAD_PAGE);
  if (LATE && rank == 0) always();
  if (rank == 0)                                   // (behind the keys zeros, up to a multiple of 32)
    for (int x = tid; x < HG * TT * 32; x += THREADS) {
      const int end = scored(x / 32 % TT), j = end + x % 32;
      if (j < (end + 31) / 32 * 32) keys[x / 32 * A.slots + j] = 0u;
    }
  if (CL) {
    ptx::cluster_sync();
    if (rank != 0) return;
  } else {
    __syncthreads();
  }

  // ---- the best r, in their order: each token by a group of warps
  const int hu = warp / F::kGroup, u = hu % TT, m = scored(u);
  if (m == 0) return;
  const Group<F::kGroup> G{tid % (32 * F::kGroup), lane, warp % F::kGroup, hu};
  Search& S = search[hu];
  const Keys<F::kGroup, F::kKept> mine(keys + hu * A.slots, row + a.first, m, G);
  // (A key of each lane's; where the groups are many the counts' round trips cost less than all these comparisons: 250
  // tokens of 16 pages 7.3 us, 7.9 by ranks; of 64 pages 9.7 and 10.9; 100 sequences of three tokens, 16 pages, 8.8 and 8.0.)
  const bool ranked = TT > 1 && m <= min(kSelRanked, 32 * F::kGroup);
  const uint32_t at = ranked ? 0u : threshold(mine, r, S, G);
  // pages above it in each 32, pages with it; then where these of the warp begin
  const uint32_t below = (1u << lane) - 1;
  int32_t* const out = list_of(u, hu / TT) + a.first;
  int above = 0, equal = 0;
  uint32_t up[F::kKept], eq[F::kKept];
  if (ranked) {
#pragma unroll
    for (int k = 0; k < F::kKept; ++k) {
      up[k] = eq[k] = 0u;
      if (k == 0 && mine.first < mine.end)
        up[k] = __ballot_sync(0xffffffffu, mine.there(k, lane) && rank_of(mine.all, m, mine.kept[k], mine.first, lane) < r);
      above += __popc(up[k]);
    }
  } else if (mine.few) {
#pragma unroll
    for (int k = 0; k < F::kKept; ++k) {
      up[k] = __ballot_sync(0xffffffffu, mine.there(k, lane) && mine.kept[k] > at);
      eq[k] = __ballot_sync(0xffffffffu, mine.there(k, lane) && mine.kept[k] == at);
    }
#pragma unroll
    for (int k = 0; k < F::kKept; ++k) above += __popc(up[k]), equal += __popc(eq[k]);
  } else {
#pragma unroll 4
    for (int j = mine.first + lane; j - lane < mine.end; j += 32) {
      const uint32_t k = j < mine.end ? mine.all[j] : 0u;
      above += __popc(__ballot_sync(0xffffffffu, j < mine.end && k > at));
      equal += __popc(__ballot_sync(0xffffffffu, j < mine.end && k == at));
    }
  }
  if (lane == 0) S.above[G.warp] = above, S.equal[G.warp] = equal;
  G.sync();
  int n_above = 0, n_equal = 0, all_above = 0;
#pragma unroll
  for (int w = 0; w < F::kGroup; ++w) {
    if (w == G.warp) n_above = all_above;
    if (w < G.warp) n_equal += S.equal[w];
    all_above += S.above[w];
  }
  const int left = r - all_above;                  // of those with the r-th score
  auto put = [&](uint32_t ups, uint32_t eqs, int32_t id) {
    const int n = n_above + __popc(ups & below), e = n_equal + __popc(eqs & below);
    if ((ups >> lane & 1) || ((eqs >> lane & 1) && e < left)) out[n + min(e, left)] = id;
    n_above += __popc(ups);
    n_equal += __popc(eqs);
  };
  if (mine.few) {
#pragma unroll
    for (int k = 0; k < F::kKept; ++k) put(up[k], eq[k], mine.page[k]);
  } else {
    for (int j = mine.first + lane; j - lane < mine.end; j += 32) {
      const uint32_t k = j < mine.end ? mine.all[j] : 0u;
      put(__ballot_sync(0xffffffffu, j < mine.end && k > at), __ballot_sync(0xffffffffu, j < mine.end && k == at),
          j < mine.end ? mine.ids[j] : 0);
    }
  }
}

}  // namespace kv4

using namespace kv4;

static bool seqs_ok(const buddy_kv4_cache* c, const buddy_kv4_seqs& s) {
  return s.batch >= 1 && s.batch <= 16384 && s.n_tok >= 0 && s.max_new >= 1 && s.max_pages >= 1 &&
         (int64_t)s.max_pages * c->page_size <= INT32_MAX && s.kv_len && s.table &&
         (s.row_start || (s.n_tok == s.batch && s.max_new == 1));
}

template <typename T, int HD, int TT, int HG, bool CL>
static int launch_select(SelectArgs A, int C, cudaStream_t s) {
  using F = Form<TT, HG, CL>;
  int64_t ctas = (int64_t)A.a.s.n_tok * (A.p.nkv / HG) * C;
  if (TT > 1) {                                    // by sequences, unless few of them have as many tokens as the longest
    const int64_t chunks = (A.a.s.max_new + TT - 1) / TT;
    if (A.a.s.batch * chunks <= A.a.s.n_tok) {
      A.chunks = (int)chunks;
      ctas = A.a.s.batch * chunks * (A.p.nkv / HG) + (A.a.s.n_tok + F::kThreads - 1) / F::kThreads;
    }
  }
  if (A.chunks == 0 && A.a.s.row_start) ctas += (int64_t)(A.a.s.batch + F::kThreads - 1) / F::kThreads * C;
  if (ctas > INT32_MAX) return BUDDY_ERR_RANGE;
  auto* const kern = kv4_select_kernel<T, HD, TT, HG, CL>;
  const int smem = F::smem(A.slots);
  // the largest size any call uses: the attribute belongs to the function on the device, and a call's
  // own would take it from another host thread's launch
  if (smem > 40 * 1024 &&
      cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, F::kMostSmem) != cudaSuccess)
    return BUDDY_ERR_CUDA;
  if (!CL) return launch_k(kern, (unsigned)ctas, F::kThreads, smem, s, true, A) == cudaSuccess ? BUDDY_OK : BUDDY_ERR_CUDA;
  if (C > 8 && cudaFuncSetAttribute(kern, cudaFuncAttributeNonPortableClusterSizeAllowed, 1) != cudaSuccess) return BUDDY_ERR_CUDA;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = (unsigned)ctas;
  cfg.blockDim = F::kThreads;
  cfg.dynamicSmemBytes = smem;
  cfg.stream = s;
  cudaLaunchAttribute at[2];
  at[0].id = cudaLaunchAttributeClusterDimension;
  at[0].val.clusterDim.x = C;
  at[0].val.clusterDim.y = at[0].val.clusterDim.z = 1;
  at[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  at[1].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = at;
  cfg.numAttrs = 2;
  return cudaLaunchKernelEx(&cfg, kern, A) == cudaSuccess ? BUDDY_OK : BUDDY_ERR_CUDA;
}

// Several tokens of a sequence share a walk where there may be such, over two heads' bounds where the table
// is short, so that what a CTA does before and after its walk counts (31 sequences of up to five tokens, 40 KV
// heads, 256 pages: 47.5 us, one head each 57.7; 9 prompts of up to 1,500 tokens, 8 KV heads, 60 pages: 142 and
// 246; 750 pages, 25 to 750 in use: 54.8 and 45.4, the longest walk being the last to end; widths between 256 and 750
// were not measured). Clusters, where a table has more pages than a CTA's warps take at once, as large as leaves every warp
// a turn, and up to 608 CTAs: twice as many as are resident at once by registers (two an SM; one by shared memory, from some
// 12,000 pages on), a number that was not measured against smaller ones (one token of 8 KV heads over 1,876 pages 7.6 us,
// 64 with a CTA for each head; four such sequences 14.5).
//
// Form and shared memory go by the table's width, not by what is in use: 250 sequences of 8 to 128 pages take 8.2 us
// under tables of 129 to 2,048 entries, 9.8 of 8,192, 19 of 40,000; 31 sequences of several tokens and up to 750 pages 45 under
// 751 to 2,048, 71 under 8,000. And tokens that share a walk have no clusters: one sequence over 1,876 pages, 8 KV heads,
// takes 37 us with two tokens and 47 with four to eight, over 7,500 pages 128 and 172 (one token: 7.6 and 20).
template <typename T, int HD>
static int dispatch_select(SelectArgs A, cudaStream_t s) {
  A.slots = (std::max(1, A.a.s.max_pages - A.a.first - A.a.last) + 31) / 32 * 32;
  if (A.a.s.max_new > 1 && A.slots <= kSelShared) {
    if (A.p.nkv % 2 == 0 && A.slots <= kSelPairs) return launch_select<T, HD, kSelTokens, 2, false>(A, 1, s);
    return launch_select<T, HD, kSelTokens, 1, false>(A, 1, s);
  }
  const int64_t units = (int64_t)A.a.s.n_tok * A.p.nkv;
  int C = 1;
  while (C < kSelCluster && 2 * C * Form<1, 1, true>::kWarps * Form<1, 1, true>::kLoads * (256 / HD) <= A.slots && units * 2 * C <= 4 * 152) C *= 2;
  return C > 1 ? launch_select<T, HD, 1, 1, true>(A, C, s) : launch_select<T, HD, 1, 1, false>(A, 1, s);
}

}  // namespace buddy

using namespace buddy;

extern "C" int buddy_kv4_bounds(const buddy_kv4_cache* cache, const buddy_kv4_seqs* seqs, void* bounds, int32_t* flags,
                                void* stream) {
  if (!kv4_cache_ok(cache) || !seqs || !seqs_ok(cache, *seqs) || !bounds || !aligned16(bounds)) return BUDDY_ERR_ARG;
  const int P = cache->page_size;
  const int cols = (int)std::min<int64_t>(seqs->max_pages, ((int64_t)seqs->max_new + P - 2) / P + 1);
  const BoundArgs A{*seqs, kv4_pages(cache), (__half*)bounds, flags, cols};
  const int64_t units = (int64_t)seqs->batch * cols * cache->n_kv_heads, ctas = (units + kBoundWarps - 1) / kBoundWarps;
  if (ctas > INT32_MAX) return BUDDY_ERR_RANGE;
  auto* const kern = cache->head_dim == 128 ? kv4_bounds_kernel<128> : kv4_bounds_kernel<64>;
  return launch_k(kern, (unsigned)ctas, 32 * kBoundWarps, 0, (cudaStream_t)stream, true, A) == cudaSuccess ? BUDDY_OK
                                                                                                           : BUDDY_ERR_CUDA;
}

extern "C" int buddy_kv4_select(const buddy_kv4_cache* cache, const buddy_kv4_select_args* a, int32_t* flags,
                                void* stream) {
  if (!kv4_cache_ok(cache) || !a || !seqs_ok(cache, a->s) || a->n_q_heads < cache->n_kv_heads ||
      a->n_q_heads % cache->n_kv_heads || a->n_q_heads / cache->n_kv_heads > 8 ||
      (a->q_dtype != BUDDY_DTYPE_F32 && a->q_dtype != BUDDY_DTYPE_BF16) || a->first < 0 || a->last < 1 ||
      (int64_t)a->first + a->last > a->budget)
    return BUDDY_ERR_ARG;
  if (a->s.max_pages > kSelMaxPages) return BUDDY_ERR_RANGE;
  if (a->s.n_tok == 0) return BUDDY_OK;
  if (!a->q || !aligned16(a->q) || a->q_stride * (a->q_dtype == BUDDY_DTYPE_F32 ? 4 : 2) % 16 || !a->bounds ||
      !aligned16(a->bounds) || !a->pages || !a->visible)
    return BUDDY_ERR_ARG;
  const SelectArgs A{*a, kv4_pages(cache), a->n_q_heads / cache->n_kv_heads, 0, 0, -0.f, flags};
  cudaStream_t s = (cudaStream_t)stream;
  if (a->q_dtype == BUDDY_DTYPE_F32)
    return cache->head_dim == 128 ? dispatch_select<float, 128>(A, s) : dispatch_select<float, 64>(A, s);
  return cache->head_dim == 128 ? dispatch_select<bf16, 128>(A, s) : dispatch_select<bf16, 64>(A, s);
}
