// The pages of a 4-bit cache that a query is likely to need: each page's bounds of the keys
// (buddy_kv4_bounds) and each query's best pages by them (buddy_kv4_select).  Attention
// over those lists is a form of the few-row kernel (kv4_attn.cu).
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
constexpr int kBoundLoads = 8;          // rows of codes in flight per lane

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
// (kv4.cuh), and so are the bounds.
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
#pragma unroll 1
  for (int r0 = row; r0 < end; r0 += kBoundLoads * RPL) {
    uint2 w[kBoundLoads];
    __half sc[kBoundLoads];
#pragma unroll
    for (int j = 0; j < kBoundLoads; ++j) {
      const int r = r0 + j * RPL;
      if (r < end) {
        w[j] = *reinterpret_cast<const uint2*>(codes + r * code_bytes(HD));
        sc[j] = scales[r * (scale_bytes(HD) / 2)];
      }
    }
#pragma unroll
    for (int j = 0; j < kBoundLoads; ++j) {
      if (r0 + j * RPL >= end) break;
      const __half2 s1 = __half2half2(sc[j]), s72 = __hmul2(s1, __float2half2_rn(-72.f));
      uint32_t v[8];
      dequant4(w[j].x, s1, s72, v);
      dequant4(w[j].y, s1, s72, v + 4);
#pragma unroll
      for (int e = 0; e < 8; ++e) lo[e] = __hmin2_nan(lo[e], as_h2(v[e])), hi[e] = __hmax2_nan(hi[e], as_h2(v[e]));
    }
  }
#pragma unroll
  for (int o = LPR; o < 32; o <<= 1)
#pragma unroll
    for (int e = 0; e < 8; ++e) lo[e] = __hmin2_nan(lo[e], shfl_xor(lo[e], o)), hi[e] = __hmax2_nan(hi[e], shfl_xor(hi[e], o));
  if (row < 2) {
    uint4* const d = reinterpret_cast<uint4*>(A.bounds + (((int64_t)id * A.p.nkv + g) * 2 + row) * HD + 16 * tl);
    const __half2* const y = row ? hi : lo;
    d[0] = make_uint4(h2(y[0]), h2(y[1]), h2(y[2]), h2(y[3]));
    d[1] = make_uint4(h2(y[4]), h2(y[5]), h2(y[6]), h2(y[7]));
  }
}

// ------------------------------------------------------------------ selection
constexpr int kSelWarps = 8;
constexpr int kSelThreads = 32 * kSelWarps;
constexpr int kSelMaxPages = 49152;     // a score each in shared memory
constexpr int kSelCluster = 16;         // most CTAs of a (token, KV head)
constexpr int kSelBins = 256;

struct SelectArgs {
  buddy_kv4_select_args a;
  Pages p;
  int G;
  int slots;                            // scores of a token: entries of a table row that may be among them
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

// A word of the first CTA's shared memory, from any CTA of its cluster.
__device__ __forceinline__ void put_first(uint32_t* at, uint32_t v) {
  asm volatile("st.shared::cluster.u32 [%0], %1;" ::"r"(ptx::dsmem_addr(at, 0)), "r"(v) : "memory");
}

// Sums over the lanes of a page, in the order of the scores: the eights of lo and of hi by
// halves, then both. Of V values a lane gives half away at each step, as long as it has two, so
// that there is about one exchange per sum; it is left with those from *base on.
template <int HD, int V>
__device__ __forceinline__ void sum_lanes(float (&v)[V], int lane, int* base) {
  constexpr int EIGHTS = HD / 8;
  int n = V, at = 0;
#pragma unroll
  for (int o = EIGHTS / 2; o >= 0; o = o > 1 ? o / 2 : o - 1) {
    const int bit = o > 0 ? o : EIGHTS;            // (last: lo and hi)
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
      at += up ? n : 0;
    } else {
      v[0] = __fadd_rn(v[0], __shfl_xor_sync(0xffffffffu, v[0], bit));
    }
  }
  *base = at;
}

// Where the best r of M keys end: just r of them are above *at, or these and the first of those
// equal to it. By counts of the keys in 256 parts of the range [lo, hi] that holds the r-th, from the
// top, until a part is one value or its keys are all wanted. bins: two sets, zeros.
__device__ __forceinline__ uint32_t threshold(const uint32_t* keys, int M, int r, uint32_t lo, uint32_t hi,
                                              int (*bins)[kSelBins], int tid, int lane) {
  for (int set = 0;; set ^= 1) {
    const int shift = max(0, 32 - __clz(hi - lo) - 8);       // ((hi - lo) >> shift) < 256
    for (int j = tid; j < M; j += kSelThreads) {
      const uint32_t k = keys[j];
      if (k >= lo && k <= hi) atomicAdd(&bins[set][(k - lo) >> shift], 1);
    }
    __syncthreads();
    bins[set ^ 1][tid] = 0;
    // every warp: lane x has the parts 255 - 8 x and below
    int c[8], sum = 0;
#pragma unroll
    for (int e = 0; e < 8; ++e) sum += c[e] = bins[set][255 - 8 * lane - e];
    int upto = sum;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int y = __shfl_up_sync(0xffffffffu, upto, o);
      if (lane >= o) upto += y;
    }
    const int src = __ffs(__ballot_sync(0xffffffffu, upto >= r)) - 1;
    int before = upto - sum, part = 255 - 8 * lane, in = c[0];
#pragma unroll
    for (int e = 1; e < 8; ++e)
      if (before + in < r) before += in, in = c[e], part = 255 - 8 * lane - e;
    before = __shfl_sync(0xffffffffu, before, src);
    part = __shfl_sync(0xffffffffu, part, src);
    in = __shfl_sync(0xffffffffu, in, src);
    r -= before;
    lo += (uint32_t)part << shift;
    hi = lo + min(hi - lo, (1u << shift) - 1);
    __syncthreads();                               // (the other set is zero, this one has been read)
    if (shift == 0) return lo;
    if (in == r) return lo - 1;                    // (lo > 0: no score lies below the parts' range)
  }
}

// Up to TT tokens of a sequence share a walk over its pages' bounds; the CTA of the first of
// them does the work of all. CL: a cluster has one token, its CTAs the pages in turn, and the first
// one the scores. A page's bounds are HD / 4 loads of 16 bytes, one per lane: the smallest
// of eight channels, by b, or the largest, by a.
template <typename T, int HD, int TT, bool CL>
__global__ void __launch_bounds__(kSelThreads, TT == 1 ? 4 : 2) kv4_select_kernel(const SelectArgs A) {
  extern __shared__ uint32_t keys[];               // [TT][slots]
  __shared__ int bins[2][kSelBins];
  __shared__ uint32_t s_lo[TT][kSelCluster * kSelWarps], s_hi[TT][kSelCluster * kSelWarps];
  __shared__ int s_above[kSelWarps], s_equal[kSelWarps];
  static_assert(!CL || TT == 1, "");
  constexpr int LPP = HD / 4, PPW = 32 / LPP;      // lanes of a page, pages of a warp's load
  constexpr int LOADS = TT == 1 ? 8 : 4;           // in flight
  constexpr int V = LOADS * TT;
  const buddy_kv4_select_args& a = A.a;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const uint32_t rank = CL ? ptx::cluster_rank() : 0, C = CL ? ptx::cluster_size() : 1;
  const unsigned unit = blockIdx.x / C;
  const int g = (int)(unit % (unsigned)A.p.nkv), t = (int)(unit / (unsigned)A.p.nkv);
  bins[0][tid] = bins[1][tid] = 0;
  pdl_wait();
  pdl_trigger();
  const int i = seq_of(a.s, t, lane);
  Rows s{};
  bool ok = i >= 0;
  if (ok) {
    ok = rows_of(a.s, A.p.shift, i, &s) && t >= s.t0 && t < s.t0 + s.m;
    if (!ok && g == 0 && tid == 0 && rank == 0 && A.flags) atomicOr(A.flags, BUDDY_DEV_BAD_POSITION);
  }
  if (!ok) {
    if (g == 0 && tid == 0 && rank == 0) a.visible[t] = -1;
    return;
  }
  const int p0 = s.n - s.m + (t - s.t0);           // of token t; the next ones follow
  const int in_page = (1 << A.p.shift) - 1;
  auto pages_of = [&](int p) { return p < 0 ? 0 : (p >> A.p.shift) + 1; };
  if (g == 0 && tid == 0 && rank == 0) {
    const int N = pages_of(p0);
    a.visible[t] = N == 0 ? 0 : ((min(N, a.budget) - 1) << A.p.shift) + (p0 & in_page) + 1;
  }
  if (TT > 1 && (t - s.t0) % TT != 0) return;
  const int tokens = min(TT, s.t0 + s.m - t);
  const int32_t* const row = a.s.table + (int64_t)i * a.s.max_pages;
  auto list_of = [&](int u) { return a.pages + ((int64_t)(t + u) * A.p.nkv + g) * a.budget; };
  // what is in without a score
  const int r = a.budget - a.first - a.last;
  if (rank == 0) {
    for (int u = 0; u < tokens; ++u) {
      const int N = pages_of(p0 + u);
      int32_t* const out = list_of(u);
      if (N <= a.budget) {
        for (int j = tid; j < a.budget; j += kSelThreads) out[j] = j < N ? row[j] : -1;
      } else {
        for (int j = tid; j < a.first; j += kSelThreads) out[j] = row[j];
        for (int j = tid; j < a.last; j += kSelThreads) out[a.budget - a.last + j] = row[N - a.last + j];
      }
    }
  }
  auto scored = [&](int u) { const int N = pages_of(p0 + u); return u < tokens && N > a.budget ? N - a.first - a.last : 0; };
  const int M = scored(tokens - 1);                // of the last token: the most
  if (M == 0 || r == 0) return;                    // (the same in the whole cluster)
  if (CL) ptx::cluster_arrive_started();

  // ---- scores
  float f[TT][8];
#pragma unroll
  for (int u = 0; u < TT; ++u) {
    const bool high = lane % LPP >= LPP / 2;
    const T* q = (const T*)a.q + (t + min(u, tokens - 1)) * a.q_stride + (int64_t)g * A.G * HD + lane % (LPP / 2) * 8;
    for (int h = 0; h < A.G; ++h) {
      float x[8];
      load8(q + h * HD, x);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float y = isnan(x[e]) ? x[e] : high ? fmaxf(x[e], 0.f) : fminf(x[e], 0.f);
        f[u][e] = h == 0 ? y : __fadd_rn(f[u][e], y);
      }
    }
  }
  const __half* const bounds = (const __half*)a.bounds + (int64_t)g * 2 * HD + lane % LPP * 8;
  const int64_t per_page = (int64_t)A.p.nkv * 2 * HD;
  bool lost = false;
  uint32_t low[TT], top[TT];
#pragma unroll
  for (int u = 0; u < TT; ++u) low[u] = 0xFFFFFFFFu, top[u] = 0u;
  if (CL) ptx::cluster_wait_started();
  for (int j0 = ((int)rank * kSelWarps + warp) * LOADS * PPW; j0 < M; j0 += (int)C * kSelWarps * LOADS * PPW) {
    uint4 w[LOADS];
    uint32_t gone = 0;                             // loads whose page is not there
#pragma unroll
    for (int k = 0; k < LOADS; ++k) {
      const int j = j0 + k * PPW + lane / LPP;
      const int id = j < M ? row[a.first + j] : 0;
      const bool there = (uint32_t)id < (uint32_t)A.p.n_pages;
      gone |= there ? 0u : 1u << k;
      w[k] = there ? __ldg(reinterpret_cast<const uint4*>(bounds + id * per_page)) : make_uint4(0, 0, 0, 0);
    }
    float v[V];
#pragma unroll
    for (int k = 0; k < LOADS; ++k) {
      const float2 y[4] = {__half22float2(as_h2(w[k].x)), __half22float2(as_h2(w[k].y)), __half22float2(as_h2(w[k].z)),
                           __half22float2(as_h2(w[k].w))};
#pragma unroll
      for (int u = 0; u < TT; ++u) {
        float x[8];
#pragma unroll
        for (int e = 0; e < 4; ++e) x[2 * e] = __fmul_rn(f[u][2 * e], y[e].x), x[2 * e + 1] = __fmul_rn(f[u][2 * e + 1], y[e].y);
#pragma unroll
        for (int e = 0; e < 4; ++e) x[e] = __fadd_rn(x[e], x[e + 4]);
        v[k * TT + u] = __fadd_rn(__fadd_rn(x[0], x[2]), __fadd_rn(x[1], x[3]));
      }
    }
    int base;
    sum_lanes<HD, V>(v, lane, &base);
    constexpr int LEFT = V > LPP ? V / LPP : 1;    // values that a lane is left with
    // lanes that differ in these bits only are left with the same
    constexpr int TWINS = V >= LPP ? 0 : V == LPP / 2 ? LPP / 2 : LPP / 2 + LPP / (2 * V) - 1;
#pragma unroll
    for (int x = 0; x < LEFT; ++x) {
      const int k = (base + x) / TT, u = (base + x) % TT, j = j0 + k * PPW + lane / LPP;
      if (j >= scored(u) || (lane & TWINS)) continue;
      const bool there = !(gone >> k & 1);
      const uint32_t key = there ? key_of(v[x]) : 0u;
      lost |= !there;
      if (CL) put_first(&keys[j], key);
      else keys[u * A.slots + j] = key;
#pragma unroll
      for (int y = 0; y < TT; ++y)
        if (y == u) low[y] = min(low[y], key), top[y] = max(top[y], key);
    }
  }
  if (lost && A.flags) atomicOr(A.flags, BUDDY_DEV_BAD_PAGE);
#pragma unroll
  for (int u = 0; u < TT; ++u) {
    low[u] = __reduce_min_sync(0xffffffffu, low[u]);
    top[u] = __reduce_max_sync(0xffffffffu, top[u]);
    if (lane == 0) {
      const int at = (int)rank * kSelWarps + warp;
      if (CL) put_first(&s_lo[u][at], low[u]), put_first(&s_hi[u][at], top[u]);
      else s_lo[u][at] = low[u], s_hi[u][at] = top[u];
    }
  }
  if (CL) {
    ptx::cluster_sync();
    if (rank != 0) return;
  } else {
    __syncthreads();
  }

  // ---- the best r, in their order
  for (int u = 0; u < tokens; ++u) {
    const int m = scored(u);
    if (m == 0) continue;
    const uint32_t* const mine = keys + u * A.slots;
    uint32_t lo = 0xFFFFFFFFu, hi = 0;
    for (int x = lane; x < (int)C * kSelWarps; x += 32) lo = min(lo, s_lo[u][x]), hi = max(hi, s_hi[u][x]);
    lo = __reduce_min_sync(0xffffffffu, lo);
    hi = __reduce_max_sync(0xffffffffu, hi);
    const uint32_t at = threshold(mine, m, r, lo, hi, bins, tid, lane);
    const int run = (m + kSelThreads - 1) / kSelThreads * 32, end = min(m, (warp + 1) * run);   // of a warp
    int above = 0, equal = 0;
    for (int j = warp * run + lane; j - lane < end; j += 32) {
      const uint32_t k = j < end ? mine[j] : 0u;
      above += __popc(__ballot_sync(0xffffffffu, j < end && k > at));
      equal += __popc(__ballot_sync(0xffffffffu, j < end && k == at));
    }
    if (lane == 0) s_above[warp] = above, s_equal[warp] = equal;
    bins[0][tid] = bins[1][tid] = 0;               // for the next token
    __syncthreads();
    int n_above = 0, n_equal = 0, all_above = 0;
#pragma unroll
    for (int w = 0; w < kSelWarps; ++w) {
      if (w == warp) n_above = all_above;
      if (w < warp) n_equal += s_equal[w];
      all_above += s_above[w];
    }
    const int left = r - all_above;                // of those with the r-th score
    const uint32_t below = (1u << lane) - 1;
    int32_t* const out = list_of(u) + a.first;
    for (int j = warp * run + lane; j - lane < end; j += 32) {
      const uint32_t k = j < end ? mine[j] : 0u;
      const uint32_t up = __ballot_sync(0xffffffffu, j < end && k > at), eq = __ballot_sync(0xffffffffu, j < end && k == at);
      const int ups = n_above + __popc(up & below), eqs = n_equal + __popc(eq & below);
      if ((up >> lane & 1) || ((eq >> lane & 1) && eqs < left)) out[ups + min(eqs, left)] = row[a.first + j];
      n_above += __popc(up);
      n_equal += __popc(eq);
    }
    if (TT > 1) __syncthreads();                   // (the warps' counts have been read)
  }
}

}  // namespace kv4

using namespace kv4;

static bool seqs_ok(const buddy_kv4_cache* c, const buddy_kv4_seqs& s) {
  return s.batch >= 1 && s.batch <= 16384 && s.n_tok >= 0 && s.max_new >= 1 && s.max_pages >= 1 &&
         (int64_t)s.max_pages * c->page_size <= INT32_MAX && s.kv_len && s.table &&
         (s.row_start || (s.n_tok == s.batch && s.max_new == 1));
}

template <typename T, int HD, int TT, bool CL>
static int launch_select(SelectArgs A, int C, cudaStream_t s) {
  const int64_t ctas = (int64_t)A.a.s.n_tok * A.p.nkv * C;
  if (ctas > INT32_MAX) return BUDDY_ERR_RANGE;
  auto* const kern = kv4_select_kernel<T, HD, TT, CL>;
  const size_t smem = sizeof(uint32_t) * (size_t)TT * A.slots;
  if (smem > 32 * 1024 && cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem) != cudaSuccess)
    return BUDDY_ERR_CUDA;
  if (!CL) return launch_k(kern, (unsigned)ctas, kSelThreads, smem, s, true, A) == cudaSuccess ? BUDDY_OK : BUDDY_ERR_CUDA;
  if (C > 8 && cudaFuncSetAttribute(kern, cudaFuncAttributeNonPortableClusterSizeAllowed, 1) != cudaSuccess) return BUDDY_ERR_CUDA;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = (unsigned)ctas;
  cfg.blockDim = kSelThreads;
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

// Several tokens of a sequence share a walk where there may be such; clusters, where a table has more pages than a
// CTA's warps take at once, as large as leaves every warp a turn and the GPU (four CTAs
// an SM) room for all.
constexpr int kSelTokens = 4;
template <typename T, int HD>
static int dispatch_select(SelectArgs A, cudaStream_t s) {
  A.slots = std::max(1, A.a.s.max_pages - A.a.first - A.a.last);
  if (A.a.s.max_new > 1 && (int64_t)A.slots * kSelTokens <= kSelMaxPages) return launch_select<T, HD, kSelTokens, false>(A, 1, s);
  const int64_t units = (int64_t)A.a.s.n_tok * A.p.nkv;
  int C = 1;
  while (C < kSelCluster && 2 * C * kSelWarps * 8 * (128 / HD) <= A.slots && units * 2 * C <= 4 * 152) C *= 2;
  return C > 1 ? launch_select<T, HD, 1, true>(A, C, s) : launch_select<T, HD, 1, false>(A, 1, s);
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
  const SelectArgs A{*a, kv4_pages(cache), a->n_q_heads / cache->n_kv_heads, 0, flags};
  cudaStream_t s = (cudaStream_t)stream;
  if (a->q_dtype == BUDDY_DTYPE_F32)
    return cache->head_dim == 128 ? dispatch_select<float, 128>(A, s) : dispatch_select<float, 64>(A, s);
  return cache->head_dim == 128 ? dispatch_select<bf16, 128>(A, s) : dispatch_select<bf16, 64>(A, s);
}
