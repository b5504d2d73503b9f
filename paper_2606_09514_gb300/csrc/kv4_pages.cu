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
constexpr int kSelLoads = 8;            // pages in flight per warp or half a warp
constexpr int kSelMaxPages = 49152;     // a score each in shared memory

struct SelectArgs {
  buddy_kv4_select_args a;
  Pages p;
  int G;
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

// A CTA has a token's pages of one KV head.  A page's bounds are 32 HD / 128 loads of 16 bytes,
// a lane each: the smallest of eight channels, or the largest, by b or a.  Scores lie in
// shared memory; the r-th best is found by bits from the top, two at a time, and the pages
// above it, and as many with its score as are left, go out in their order.
template <typename T, int HD>
__global__ void __launch_bounds__(kSelThreads) kv4_select_kernel(const SelectArgs A) {
  extern __shared__ uint32_t keys[];
  __shared__ int s_count[2][kSelWarps][3];
  constexpr int LPP = HD / 4;                      // lanes of a page: HD / 8 for lo, as many for hi
  const buddy_kv4_select_args& a = A.a;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int g = (int)(blockIdx.x % (unsigned)A.p.nkv), t = (int)(blockIdx.x / (unsigned)A.p.nkv);
  pdl_wait();
  pdl_trigger();
  const int i = seq_of(a.s, t, lane);
  Rows s{};
  bool ok = i >= 0;
  if (ok) {
    ok = rows_of(a.s, A.p.shift, i, &s) && t >= s.t0 && t < s.t0 + s.m;
    if (!ok && g == 0 && tid == 0 && A.flags) atomicOr(A.flags, BUDDY_DEV_BAD_POSITION);
  }
  if (!ok) {
    if (g == 0 && tid == 0) a.visible[t] = -1;
    return;
  }
  const int p = s.n - s.m + (t - s.t0);
  const int N = p < 0 ? 0 : (p >> A.p.shift) + 1, count = min(N, a.budget);
  if (g == 0 && tid == 0) a.visible[t] = N == 0 ? 0 : ((count - 1) << A.p.shift) + (p & ((1 << A.p.shift) - 1)) + 1;
  const int32_t* const row = a.s.table + (int64_t)i * a.s.max_pages;
  int32_t* const out = a.pages + ((int64_t)t * A.p.nkv + g) * a.budget;
  if (N <= a.budget) {
    for (int j = tid; j < a.budget; j += kSelThreads) out[j] = j < N ? row[j] : -1;
    return;
  }
  for (int j = tid; j < a.first; j += kSelThreads) out[j] = row[j];
  for (int j = tid; j < a.last; j += kSelThreads) out[a.budget - a.last + j] = row[N - a.last + j];
  const int M = N - a.first - a.last, r = a.budget - a.first - a.last;
  if (r == 0) return;

  // ---- scores
  float f[8];
  {
    const bool high = lane % LPP >= LPP / 2;
    const T* q = (const T*)a.q + t * a.q_stride + (int64_t)g * A.G * HD + lane % (LPP / 2) * 8;
#pragma unroll
    for (int e = 0; e < 8; ++e) f[e] = 0.f;
    for (int h = 0; h < A.G; ++h) {
      float x[8];
      load8(q + h * HD, x);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float y = isnan(x[e]) ? x[e] : high ? fmaxf(x[e], 0.f) : fminf(x[e], 0.f);
        f[e] = h == 0 ? y : __fadd_rn(f[e], y);
      }
    }
  }
  constexpr int PPW = 32 / LPP;                    // pages of a load of the warp
  const __half* const bounds = (const __half*)a.bounds + (int64_t)g * 2 * HD + lane % LPP * 8;
  const int64_t per_page = (int64_t)A.p.nkv * 2 * HD;
  bool lost = false;
  for (int j0 = warp * kSelLoads * PPW; j0 < M; j0 += kSelWarps * kSelLoads * PPW) {
    uint4 w[kSelLoads];
    bool there[kSelLoads];
#pragma unroll
    for (int k = 0; k < kSelLoads; ++k) {
      const int j = j0 + k * PPW + lane / LPP;
      const int id = j < M ? row[a.first + j] : 0;
      there[k] = (uint32_t)id < (uint32_t)A.p.n_pages;
      w[k] = there[k] ? *reinterpret_cast<const uint4*>(bounds + id * per_page) : make_uint4(0, 0, 0, 0);
    }
#pragma unroll
    for (int k = 0; k < kSelLoads; ++k) {
      const uint32_t u[4] = {w[k].x, w[k].y, w[k].z, w[k].w};
      float x[8];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const float2 y = __half22float2(as_h2(u[e]));
        x[2 * e] = __fmul_rn(f[2 * e], y.x);
        x[2 * e + 1] = __fmul_rn(f[2 * e + 1], y.y);
      }
#pragma unroll
      for (int e = 0; e < 4; ++e) x[e] = __fadd_rn(x[e], x[e + 4]);
      float sum = __fadd_rn(__fadd_rn(x[0], x[2]), __fadd_rn(x[1], x[3]));
#pragma unroll
      for (int o = LPP / 4; o > 0; o >>= 1) sum = __fadd_rn(sum, __shfl_xor_sync(0xffffffffu, sum, o));
      sum = __fadd_rn(sum, __shfl_xor_sync(0xffffffffu, sum, LPP / 2));
      const int j = j0 + k * PPW + lane / LPP;
      if (lane % LPP == 0 && j < M) keys[j] = there[k] ? key_of(sum) : 0u;
      lost |= !there[k];
    }
  }
  if (lost && A.flags) atomicOr(A.flags, BUDDY_DEV_BAD_PAGE);
  __syncthreads();

  // ---- the r-th largest key: `at` is the largest value that r keys or more reach
  uint32_t at = 0;
  int step = 0;
  bool exact = false;                              // just r keys reach it
  for (int b = 30; b >= 0 && !exact; b -= 2, step ^= 1) {
    int c[3] = {0, 0, 0};
    for (int j = tid; j < M; j += kSelThreads) {
      const uint32_t k = keys[j];
#pragma unroll
      for (int v = 0; v < 3; ++v) c[v] += k >= (at | ((uint32_t)(v + 1) << b));
    }
#pragma unroll
    for (int v = 0; v < 3; ++v) c[v] = __reduce_add_sync(0xffffffffu, c[v]);
    if (lane < 3) s_count[step][warp][lane] = lane == 0 ? c[0] : lane == 1 ? c[1] : c[2];
    __syncthreads();
    uint32_t to = at;
#pragma unroll
    for (int v = 0; v < 3; ++v) {
      int all = 0;
#pragma unroll
      for (int w = 0; w < kSelWarps; ++w) all += s_count[step][w][v];
      if (all >= r) to = at | ((uint32_t)(v + 1) << b), exact = all == r;
    }
    at = to;
  }

  // ---- in their order: a warp has a run of pages
  const int run = (M + kSelThreads - 1) / kSelThreads * 32, j_end = min(M, (warp + 1) * run);
  int above = 0, equal = 0;
  for (int j0 = warp * run; j0 < j_end; j0 += 32) {
    const uint32_t k = j0 + lane < j_end ? keys[j0 + lane] : 0u;
    const bool in = j0 + lane < j_end;
    above += __popc(__ballot_sync(0xffffffffu, in && k > at));
    equal += __popc(__ballot_sync(0xffffffffu, in && k == at));
  }
  __syncthreads();                                 // (the last step's counts have been read)
  if (lane == 0) s_count[0][warp][0] = above, s_count[0][warp][1] = equal;
  __syncthreads();
  int n_above = 0, n_equal = 0, all_above = 0;
  for (int w = 0; w < kSelWarps; ++w) {
    if (w == warp) n_above = all_above;
    if (w < warp) n_equal += s_count[0][w][1];
    all_above += s_count[0][w][0];
  }
  const int left = r - all_above;                  // of those with the r-th score
  const uint32_t below = (1u << lane) - 1;
  for (int j0 = warp * run; j0 < j_end; j0 += 32) {
    const bool in = j0 + lane < j_end;
    const uint32_t k = in ? keys[j0 + lane] : 0u;
    const uint32_t up = __ballot_sync(0xffffffffu, in && k > at), eq = __ballot_sync(0xffffffffu, in && k == at);
    const int ups = n_above + __popc(up & below), eqs = n_equal + __popc(eq & below);
    if ((up >> lane & 1) || ((eq >> lane & 1) && eqs < left)) out[a.first + ups + min(eqs, left)] = row[a.first + j0 + lane];
    n_above += __popc(up);
    n_equal += __popc(eq);
  }
}

}  // namespace kv4

using namespace kv4;

static bool seqs_ok(const buddy_kv4_cache* c, const buddy_kv4_seqs& s) {
  return s.batch >= 1 && s.batch <= 16384 && s.n_tok >= 0 && s.max_new >= 1 && s.max_pages >= 1 &&
         (int64_t)s.max_pages * c->page_size <= INT32_MAX && s.kv_len && s.table &&
         (s.row_start || (s.n_tok == s.batch && s.max_new == 1));
}

template <typename T, int HD>
static int launch_select(const SelectArgs& A, cudaStream_t s) {
  const size_t smem = sizeof(uint32_t) * (size_t)std::max(1, A.a.s.max_pages - A.a.first - A.a.last);
  if (smem > 40 * 1024 && cudaFuncSetAttribute(kv4_select_kernel<T, HD>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                               (int)smem) != cudaSuccess)
    return BUDDY_ERR_CUDA;
  const int64_t ctas = (int64_t)A.a.s.n_tok * A.p.nkv;
  if (ctas > INT32_MAX) return BUDDY_ERR_RANGE;
  return launch_k(kv4_select_kernel<T, HD>, (unsigned)ctas, kSelThreads, smem, s, true, A) == cudaSuccess ? BUDDY_OK
                                                                                                          : BUDDY_ERR_CUDA;
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
  const SelectArgs A{*a, kv4_pages(cache), a->n_q_heads / cache->n_kv_heads, flags};
  cudaStream_t s = (cudaStream_t)stream;
  if (a->q_dtype == BUDDY_DTYPE_F32)
    return cache->head_dim == 128 ? launch_select<float, 128>(A, s) : launch_select<float, 64>(A, s);
  return cache->head_dim == 128 ? launch_select<bf16, 128>(A, s) : launch_select<bf16, 64>(A, s);
}
