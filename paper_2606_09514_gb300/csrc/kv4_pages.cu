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
constexpr int kSelMaxPages = 40000;     // a score each in shared memory, next to the copies in flight
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

// What a thread has of M keys: warp w those from w * run on, 32 at a time. Up to kSelKept of them
// stay in registers, more in shared memory.
constexpr int kSelKept = 8;
struct Keys {
  const uint32_t* all;
  int first, end;                                  // of the warp
  bool few;
  uint32_t kept[kSelKept];
  __device__ __forceinline__ Keys(const uint32_t* keys, int M, int warp, int lane) : all(keys) {
    const int run = (M + kSelThreads - 1) / kSelThreads * 32;
    first = warp * run;
    end = min(M, first + run);
    few = run <= kSelKept * 32;
    if (few) {
#pragma unroll
      for (int k = 0; k < kSelKept; ++k) kept[k] = first + 32 * k + lane < end ? keys[first + 32 * k + lane] : 0u;
    }
  }
  // f(key, index, true where there is one), a warp together
  template <typename F>
  __device__ __forceinline__ void each(int lane, F&& f) const {
    if (few) {
#pragma unroll
      for (int k = 0; k < kSelKept; ++k)
        if (first + 32 * k < end) f(kept[k], first + 32 * k + lane, first + 32 * k + lane < end);
    } else {
#pragma unroll 4
      for (int j = first + lane; j - lane < end; j += 32) f(j < end ? all[j] : 0u, j, j < end);
    }
  }
};

// Where the best r of the keys end: just r of them are above what is returned, or these and the first
// of those equal to it. By counts of the keys in 256 parts of the range [lo, hi] that holds the r-th,
// from the top, until a part is one value or its keys are all wanted. bins: two sets, zeros.
__device__ __forceinline__ uint32_t threshold(const Keys& keys, int r, uint32_t lo, uint32_t hi, int (*bins)[kSelBins],
                                              int tid, int lane) {
  for (int set = 0;; set ^= 1) {
    const int shift = max(0, 32 - __clz(hi - lo) - 8);       // ((hi - lo) >> shift) < 256
    keys.each(lane, [&](uint32_t k, int, bool there) {
      if (there && k >= lo && k <= hi) atomicAdd(&bins[set][(k - lo) >> shift], 1);
    });
    __syncthreads();
    bins[set ^ 1][tid] = 0;
    // every warp: lane x has the parts from 255 - 8 x down
    const int4* const mine = reinterpret_cast<const int4*>(bins[set] + 248 - 8 * lane);
    const int4 y0 = mine[1], y1 = mine[0];
    const int c[8] = {y0.w, y0.z, y0.y, y0.x, y1.w, y1.z, y1.y, y1.x};
    int sum = 0;
#pragma unroll
    for (int e = 0; e < 8; ++e) sum += c[e];
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
    if (in == r) return lo - 1;                    // (lo > 0: not all of the keys are wanted)
  }
}

__device__ __forceinline__ void copy16(uint32_t dst, const void* src, bool there) {   // zeros where there is nothing
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(there ? 16 : 0) : "memory");
}

// Pages of a warp's turn, as loads of 16 bytes per lane; turns in flight.
constexpr int kSelLoads = 4;
template <int TT, bool CL>
__host__ __device__ constexpr int sel_turns() { return TT == 1 && !CL ? 2 : 4; }
template <int TT, bool CL>
__host__ __device__ constexpr int sel_ring() { return kSelWarps * sel_turns<TT, CL>() * kSelLoads * 512; }   // bytes
template <int TT>
__host__ __device__ constexpr int sel_ctas() { return TT == 1 ? 4 : 2; }                                      // per SM

// Up to TT tokens of a sequence share a walk over its pages' bounds; the CTA of the first of
// them does the work of all. CL: a cluster has one token, its CTAs the pages in turn, and the first
// one the scores. A page's bounds are HD / 4 copies of 16 bytes, one per lane: the smallest
// of eight channels, by b, or the largest, by a. Every lane reads what it has copied itself, so
// that the turns in flight need neither registers nor barriers.
template <typename T, int HD, int TT, bool CL>
__global__ void __launch_bounds__(kSelThreads, sel_ctas<TT>()) kv4_select_kernel(const SelectArgs A) {
  extern __shared__ __align__(128) uint8_t sel_smem[];
  uint32_t* const keys = reinterpret_cast<uint32_t*>(sel_smem + sel_ring<TT, CL>());   // [TT][slots]
  __shared__ __align__(16) int bins[2][kSelBins];
  __shared__ uint32_t s_lo[TT][kSelCluster * kSelWarps], s_hi[TT][kSelCluster * kSelWarps];
  __shared__ int s_above[kSelWarps], s_equal[kSelWarps];
  __shared__ __align__(16) float s_q[TT][2][HD];   // a token's b, then its a
  static_assert(!CL || TT == 1, "");
  constexpr int LPP = HD / 4, PPW = 32 / LPP;      // lanes of a page, pages of a warp's load
  constexpr int LOADS = kSelLoads, V = LOADS * TT; // of a turn, and their scores
  constexpr int TURNS = sel_turns<TT, CL>(), PAGES = LOADS * PPW, IDS = 32 / PAGES;   // turns whose ids a warp reads at once
  const buddy_kv4_select_args& a = A.a;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const uint32_t rank = CL ? ptx::cluster_rank() : 0, C = CL ? ptx::cluster_size() : 1;
  const unsigned unit = blockIdx.x / C;
  const int g = (int)(unit % (unsigned)A.p.nkv), t = (int)(unit / (unsigned)A.p.nkv);
  bins[0][tid] = bins[1][tid] = 0;
  pdl_wait();
  pdl_trigger();
  // (the queries are on their way while the token's sequence is looked for)
  constexpr int PER = (TT * HD + kSelThreads - 1) / kSelThreads;
  T x[PER][8];
#pragma unroll
  for (int e = 0; e < PER; ++e) {
    const int u = (tid + e * kSelThreads) / HD, c = tid % HD;
    const T* const q = (const T*)a.q + min(t + u, a.s.n_tok - 1) * a.q_stride + (int64_t)g * A.G * HD + c;
#pragma unroll
    for (int h = 0; h < 8; ++h)
      if (u < TT && h < A.G) x[e][h] = q[h * HD];
  }
  const int i = seq_of(a.s, t, lane);
  // turn n of the warp has the pages from (n C kSelWarps + rank kSelWarps + warp) PAGES on; their ids,
  // of IDS turns at once, by lanes (what lies behind the sequence's pages may be anything)
  const int32_t* const row = a.s.table + (int64_t)max(i, 0) * a.s.max_pages;
  const int turn = (int)C * kSelWarps * PAGES, j_first = ((int)rank * kSelWarps + warp) * PAGES;
  auto ids_of = [&](int n) {
    const int64_t j = (int64_t)(n + lane / PAGES) * turn + j_first + lane % PAGES;
    return j < A.slots && a.first + j < a.s.max_pages ? row[a.first + j] : -1;
  };
  int ids = ids_of(0), ids_next = ids_of(IDS);
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
  auto list_of = [&](int u) { return a.pages + ((int64_t)(t + u) * A.p.nkv + g) * a.budget; };
  const int r = a.budget - a.first - a.last;
  auto scored = [&](int u) { const int N = pages_of(p0 + u); return u < tokens && N > a.budget ? N - a.first - a.last : 0; };
  const int M = scored(tokens - 1);                // of the last token: the most
  // what is in without a score
  auto always = [&]() {
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
  };
  if (M == 0 || r == 0) {                          // (the same in the whole cluster)
    if (rank == 0) always();
    return;
  }
  if (CL) ptx::cluster_arrive_started();

  // ---- scores
  const int turns = M > j_first ? (M - j_first + turn - 1) / turn : 0;
  const uint32_t ring = ptx::smem_u32(sel_smem) + (uint32_t)(warp * TURNS * LOADS * 512 + lane * 16);
  const __half* const bounds = (const __half*)a.bounds + (int64_t)g * 2 * HD + lane % LPP * 8;
  const int64_t per_page = (int64_t)A.p.nkv * 2 * HD;
  uint32_t gone = 0;                               // of the loads in flight and the one at hand, LOADS bits a turn, the newest lowest
  auto issue = [&](int n, int at) {                // (a turn that is not there copies nothing: the counts of groups go on)
    gone <<= LOADS;
    if (n < turns) {
      if (n > 0 && n % IDS == 0) ids = ids_next, ids_next = ids_of(n + IDS);
#pragma unroll
      for (int k = 0; k < LOADS; ++k) {
        const int id = __shfl_sync(0xffffffffu, ids, n % IDS * PAGES + k * PPW + lane / LPP);
        const bool there = (uint32_t)id < (uint32_t)A.p.n_pages;
        gone |= there ? 0u : 1u << k;
        copy16(ring + (at * LOADS + k) * 512, bounds + (there ? id : 0) * per_page, there);
      }
    }
    asm volatile("cp.async.commit_group;" ::: "memory");
  };
#pragma unroll
  for (int n = 0; n < TURNS; ++n) issue(n, n);
#pragma unroll
  for (int e = 0; e < PER; ++e) {
    const int u = (tid + e * kSelThreads) / HD, c = tid % HD;
    if (u >= TT) continue;
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
  float f[TT][8];                                  // this lane's eight channels, of lo or of hi
#pragma unroll
  for (int u = 0; u < TT; ++u) {
    const float4* const y = reinterpret_cast<const float4*>(&s_q[u][0][0] + lane % LPP * 8);
    const float4 y0 = y[0], y1 = y[1];
    f[u][0] = y0.x, f[u][1] = y0.y, f[u][2] = y0.z, f[u][3] = y0.w;
    f[u][4] = y1.x, f[u][5] = y1.y, f[u][6] = y1.z, f[u][7] = y1.w;
  }
  bool lost = false;
  uint32_t low[TT], top[TT];
#pragma unroll
  for (int u = 0; u < TT; ++u) low[u] = 0xFFFFFFFFu, top[u] = 0u;
  if (CL) ptx::cluster_wait_started();
  for (int n = 0, at = 0; n < turns; ++n, at = at + 1 == TURNS ? 0 : at + 1) {
    asm volatile("cp.async.wait_group %0;" ::"n"(TURNS - 1) : "memory");
    float v[V];
#pragma unroll
    for (int k = 0; k < LOADS; ++k) {
      const uint4 w = *reinterpret_cast<const uint4*>(sel_smem + ((warp * TURNS + at) * LOADS + k) * 512 + lane * 16);
      const float2 y[4] = {__half22float2(as_h2(w.x)), __half22float2(as_h2(w.y)), __half22float2(as_h2(w.z)),
                           __half22float2(as_h2(w.w))};
#pragma unroll
      for (int u = 0; u < TT; ++u) {
        float z[8];
#pragma unroll
        for (int e = 0; e < 4; ++e) z[2 * e] = __fmul_rn(f[u][2 * e], y[e].x), z[2 * e + 1] = __fmul_rn(f[u][2 * e + 1], y[e].y);
#pragma unroll
        for (int e = 0; e < 4; ++e) z[e] = __fadd_rn(z[e], z[e + 4]);
        v[k * TT + u] = __fadd_rn(__fadd_rn(z[0], z[2]), __fadd_rn(z[1], z[3]));
      }
    }
    int base;
    sum_lanes<HD, V>(v, lane, &base);
    const uint32_t missing = gone >> ((TURNS - 1) * LOADS);
    issue(n + TURNS, at);                          // (what this turn has read has been used)
    constexpr int LEFT = V > LPP ? V / LPP : 1;    // values that a lane is left with
    // lanes that differ in these bits only are left with the same
    constexpr int TWINS = V >= LPP ? 0 : V == LPP / 2 ? LPP / 2 : LPP / 2 + LPP / (2 * V) - 1;
#pragma unroll
    for (int e = 0; e < LEFT; ++e) {
      const int k = (base + e) / TT, u = (base + e) % TT, j = n * turn + j_first + k * PPW + lane / LPP;
      if (j >= scored(u) || (lane & TWINS)) continue;
      const bool there = !(missing >> k & 1);
      const uint32_t key = there ? key_of(v[e]) : 0u;
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
  if (rank == 0) always();
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
    const Keys mine(keys + u * A.slots, m, warp, lane);
    uint32_t lo = 0xFFFFFFFFu, hi = 0;
    for (int y = lane; y < (int)C * kSelWarps; y += 32) lo = min(lo, s_lo[u][y]), hi = max(hi, s_hi[u][y]);
    lo = __reduce_min_sync(0xffffffffu, lo);
    hi = __reduce_max_sync(0xffffffffu, hi);
    const uint32_t at = threshold(mine, r, lo, hi, bins, tid, lane);
    int above = 0, equal = 0;
    mine.each(lane, [&](uint32_t k, int, bool there) {
      above += __popc(__ballot_sync(0xffffffffu, there && k > at));
      equal += __popc(__ballot_sync(0xffffffffu, there && k == at));
    });
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
    mine.each(lane, [&](uint32_t k, int j, bool there) {
      const uint32_t up = __ballot_sync(0xffffffffu, there && k > at), eq = __ballot_sync(0xffffffffu, there && k == at);
      const int ups = n_above + __popc(up & below), eqs = n_equal + __popc(eq & below);
      if ((up >> lane & 1) || ((eq >> lane & 1) && eqs < left)) out[ups + min(eqs, left)] = row[a.first + j];
      n_above += __popc(up);
      n_equal += __popc(eq);
    });
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
  const size_t smem = sel_ring<TT, CL>() + sizeof(uint32_t) * (size_t)TT * A.slots;
  if (smem > 24 * 1024 && cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem) != cudaSuccess)
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
  if (A.a.s.max_new > 1 && (int64_t)A.slots * kSelTokens <= 32768) return launch_select<T, HD, kSelTokens, false>(A, 1, s);
  const int64_t units = (int64_t)A.a.s.n_tok * A.p.nkv;
  int C = 1;
  while (C < kSelCluster && 2 * C * kSelWarps * kSelLoads * (128 / HD) <= A.slots && units * 2 * C <= 4 * 152) C *= 2;
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
