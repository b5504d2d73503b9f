// Attention over lists of pages of the 4-bit cache (buddy_kv4_attention_pages) where there are
// many streams, a stream being the list of one (token, KV head): up to eight query rows, all of
// which see all of its positions.
//
// The products are those of kv4_attn.cu (kv4_few.cuh). There the four warps of a CTA take the chunks
// of a stream in turn and join what they have; lists are short (some tens of chunks), so that a
// warp comes to two or three beginnings, barriers and joins for twenty chunks. Here all streams end to
// end, each as its chunks and kListOpen chunks' worth for its beginning, go in equal shares over
// the warps, and a warp works alone: a stream within its share is written out, of one that is cut
// the warps write partials, and the last of them to arrive joins these in order.
//
// Bound by instructions, as there: 250 sequences (209 MB of entries) 52.8 us, 4.0 TB/s, 58% of HBM's rate, with
// 700 instructions of a warp per chunk issued in 54% of the cycles; CTAs' turns took 60.2 us. Many short
// lists, 31 sequences of up to five tokens and 40 KV heads with a list each: 63.9 us, 77.3.
#include <cuda_runtime.h>

#include <algorithm>

#include "gemm_common.cuh"
#include "internal.h"
#include "kv4_few.cuh"

namespace buddy {
namespace kv4 {

constexpr int kListWarps = 4;
constexpr int kListThreads = 32 * kListWarps;
// (Lists of 32 pages of 64 positions of 250 sequences, 4 KV heads: 52.8 us with two stages, 54.2 with three, 54.9
// with four; with kListOpen 1, 2 and 3 55.0, 52.8 and 53.8.)
constexpr int kListStages = 2;
constexpr int kListOpen = 2;     // what beginning and ending a stream costs, in chunks
constexpr int kListWhole = 4;    // streams of at most this many chunks are not cut
constexpr int kListMaxGrid = 512;   // two partials of eight rows and an arrival counter per warp in the workspace
template <bool WIDE>
__host__ __device__ constexpr int list_ctas() { return WIDE ? 2 : 3; }   // per SM
template <int HD>
__host__ __device__ constexpr int list_smem() { return kListWarps * kListStages * stage_bytes<HD>(); }
template <int HD>
__host__ __device__ constexpr int64_t list_part() { return 8 * (HD + 2); }   // floats: maxima, sums, outputs

// Positions of token i's lists; -1: none to work on.
__device__ __forceinline__ int list_len(const AttnArgs4& A, int i, bool* bad) {
  const int n = A.a.kv_len[i];
  *bad = n > (int64_t)A.a.max_pages << A.p.shift;
  return *bad || n < 0 ? -1 : n;
}
__device__ __forceinline__ int64_t list_cost(const AttnArgs4& A, int n) {
  return n < 0 ? 0 : (int64_t)(chunks_of(n) + kListOpen) * A.p.nkv;
}

// A walk over the streams of a warp's share.
struct ListWalk {
  int i, n, g, c, c1;         // token, its positions, KV head, chunks [c, c1) of the stream in this share
  int rem;                    // what is left of the share behind this stream
  // to the next stream; false at the share's end
  __device__ __forceinline__ bool next(const AttnArgs4& A) {
    rem -= kListOpen;
    if (rem <= 0) return false;
    if (++g >= A.p.nkv) {
      g = 0;
      bool bad;
      do {
        n = list_len(A, ++i, &bad);      // (with some of the share left there is another stream)
      } while (n < 0);
    }
    c = 0;
    c1 = chunks_of(n);
    if (c1 > kListWhole) c1 = min(c1, rem);
    rem -= c1;
    return true;
  }
};

template <int HD, bool WIDE>
__global__ void __launch_bounds__(kListThreads, list_ctas<WIDE>()) kv4_lists_kernel(const AttnArgs4 A) {
  extern __shared__ __align__(128) uint8_t smem[];
  __shared__ __align__(8) uint64_t full[kListWarps * kListStages];
  __shared__ volatile int abort_flag;
  __shared__ int64_t s_sum[kListWarps], s_at[kListWarps];
  __shared__ int s_first[kListWarps];
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, lg = lane >> 2, lc = lane & 3;
  const int B = A.a.batch, G = A.G;
  if (tid < kListWarps * kListStages) ptx::mbar_init(&full[tid], 1);
  if (tid == 0) abort_flag = 0;
  ptx::fence_mbar_init();
  pdl_wait();
  pdl_trigger();

  // ---- the share of each warp: [lo, lo + share) of all streams' beginnings and chunks
  const int per = (B + kListThreads - 1) / kListThreads, b0 = min(B, tid * per), b1 = min(B, b0 + per);
  int64_t mine = 0;
  bool any_bad = false;
#pragma unroll 4
  for (int i = b0; i < b1; ++i) {
    bool bad;
    mine += list_cost(A, list_len(A, i, &bad));
    any_bad |= bad;
  }
  if (any_bad && blockIdx.x == 0 && A.flags) atomicOr(A.flags, BUDDY_DEV_BAD_POSITION);
  int64_t upto = mine, total = 0;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int64_t v = __shfl_up_sync(0xffffffffu, upto, o);
    if (lane >= o) upto += v;
  }
  if (lane == 31) s_sum[warp] = upto;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < kListWarps; ++w) {
    if (w == warp) upto += total;
    total += s_sum[w];
  }
  const int64_t warps = (int64_t)gridDim.x * kListWarps;
  const int share = (int)min((int64_t)INT32_MAX / 2, (total + warps - 1) / warps);
#pragma unroll 1
  for (int w = 0; w < kListWarps; ++w) {
    const int64_t lo = ((int64_t)blockIdx.x * kListWarps + w) * share;
    if (upto - mine <= lo && lo < upto) {
      int64_t x = upto - mine;
#pragma unroll 1
      for (int i = b0; i < b1; ++i) {
        bool bad;
        const int64_t n = list_cost(A, list_len(A, i, &bad));
        if (lo < x + n) {
          s_first[w] = i;
          s_at[w] = lo - x;
          break;
        }
        x += n;
      }
    }
  }
  __syncthreads();
  const int W = (int)blockIdx.x * kListWarps + warp;
  const int64_t lo = (int64_t)W * share;
  if (lo >= total) return;
  ListWalk use;
  int start;                        // where the stream's first chunk is, from the share's beginning on
  {
    bool bad;
    use.i = s_first[warp];
    use.n = list_len(A, use.i, &bad);
    const int64_t at = s_at[warp];
    const int nc = chunks_of(use.n);
    use.g = (int)(at / (nc + kListOpen));
    const int x = (int)(at - (int64_t)use.g * (nc + kListOpen)) - kListOpen;   // chunk of the stream; below 0: its beginning
    start = -x;
    use.rem = (int)min((int64_t)share, total - lo) + min(x, 0);
    use.c = max(x, 0);
    if (use.rem <= 0) return;
    if (x > 0 && nc <= kListWhole) {     // the warp before has it all
      use.rem -= nc - x;
      start += nc + kListOpen;
      if (!use.next(A)) return;
    } else {
      use.c1 = nc <= kListWhole ? nc : min(nc, use.c + use.rem);
      use.rem -= use.c1 - use.c;
    }
  }
  ListWalk ld = use;
  bool more = true;                 // (the walk's, until a copy does not come)
  const uint32_t ring = ptx::smem_u32(smem) + warp * kListStages * stage_bytes<HD>();

  // The load walk stands on the chunk to copy next; its page ids, of the lower and the upper
  // 16 positions, are read a chunk early.  (A chunk of nothing reads the list's first.)
  int id0 = -1, id1 = -1;
  auto fetch_ids = [&]() {
    if (ld.c >= ld.c1) {
      more = ld.next(A);
      if (!more) return;
    }
    const int p0 = ld.c * kChunk;
    const int32_t* row = A.a.table + ((int64_t)ld.i * A.p.nkv + ld.g) * A.a.max_pages;
    id0 = id1 = row[p0 >> A.p.shift];
    if (A.p.shift == 4 && p0 + 16 < ld.n) id1 = row[(p0 >> 4) + 1];
  };
  uint32_t gone = 0;                // two bits per chunk in flight, the oldest lowest: 16 positions without a page
  int take = 0, issued = 0;         // the stage to take, and its phase
  uint32_t phase = 0;
  auto issue = [&](int stage, int ahead) {
    if (!more) return;
    const int p0 = ld.c * kChunk;
    uint32_t lost = 0;
    if (max((uint32_t)id0, (uint32_t)id1) >= (uint32_t)A.p.n_pages) {
      lost = ((uint32_t)id0 < (uint32_t)A.p.n_pages ? 0 : 1) + ((uint32_t)id1 < (uint32_t)A.p.n_pages ? 0 : 2);
      if (lane == 0 && A.flags && p0 < ld.n) atomicOr(A.flags, BUDDY_DEV_BAD_PAGE);
      gone |= lost << (2 * ahead);
    }
    __syncwarp();
    if (ptx::elect_one()) {
      uint64_t* const bar = &full[warp * kListStages + stage];
      const uint32_t dst = ring + stage * stage_bytes<HD>(), b = ptx::smem_u32(bar);
      ptx::mbar_arrive_expect_tx(bar, (2 - __popc(lost)) * 16 * 2 * entry_bytes(HD));
      if (A.p.shift > 4) {
        if (lost == 0) load_piece<HD, kChunk>(A.p, dst, b, id0, ld.g, p0 & ((1 << A.p.shift) - 1), 0);
      } else {
        if (!(lost & 1)) load_piece<HD, 16>(A.p, dst, b, id0, ld.g, 0, 0);
        if (!(lost & 2)) load_piece<HD, 16>(A.p, dst, b, id1, ld.g, 0, 16);
      }
    }
    ++ld.c;
    ++issued;
    fetch_ids();
  };
  fetch_ids();
#pragma unroll 1
  for (int s = 0; s < kListStages - 1; ++s) issue(s, s);

  const Places<HD> places(lane);
  for (bool go = true; go;) {
    // ---- one stream (or the part of it in this share)
    const int n = use.n, nc = chunks_of(n);
    // queries: row lg, this lane's HD / 4 channels (rows that are not there repeat the last)
    uint32_t qf[1][HD / 16][2], ql[1][HD / 16][2];
    float fac[1][2], o[1][HD / 16][4], m[1][2], l[1][2];
    const int seen[1][2] = {{n, n}};
    {
      const int64_t at = use.i * A.a.q_stride + (int64_t)(use.g * G + min(lg, G - 1)) * HD + lc * (HD / 4);
      float x[HD / 4], top = 0.f;
#pragma unroll
      for (int e = 0; e < HD / 4; e += 8) {
        if (WIDE && A.a.q_dtype == BUDDY_DTYPE_F32) load8((const float*)A.a.q + at + e, x + e);
        else load8((const bf16*)A.a.q + at + e, x + e);
      }
#pragma unroll
      for (int e = 0; e < HD / 4; ++e) top = fmaxf(top, fabsf(x[e]));
      top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 1));
      top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 2));
      float down, f;
      row_scale<WIDE>(top, (A.a.scale != 0.f ? A.a.scale : rsqrtf((float)HD)) * 1.4426950408889634f, &down, &f);
#pragma unroll
      for (int e = 0; e < HD / 4; e += 2) {
        const Halves<WIDE> y(x[e] * down, x[e + 1] * down);
        qf[0][e / 4][(e / 2) & 1] = y.hi;
        if constexpr (WIDE) ql[0][e / 4][(e / 2) & 1] = y.lo;
      }
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        fac[0][e] = __shfl_sync(0xffffffffu, f, (2 * lc + e) * 4);
        m[0][e] = -INFINITY, l[0][e] = 0.f;
      }
#pragma unroll
      for (int t = 0; t < HD / 16; ++t)
#pragma unroll
        for (int e = 0; e < 4; ++e) o[0][t][e] = 0.f;
    }
    for (int c = use.c; c < use.c1; ++c) {
      if (!__all_sync(0xffffffffu, ptx::mbar_wait_bounded(&full[warp * kListStages + take], phase, kWaitLimitNs, &abort_flag)))
        more = false;
      const uint8_t* st = smem + (warp * kListStages + take) * stage_bytes<HD>();
      const uint32_t lost = gone & 3u;
      gone >>= 2;
      issue(take == 0 ? kListStages - 1 : take - 1, kListStages - 2);   // to the stage that the chunk before this one has left
      take_chunk<HD, 1, WIDE>(st, places, c * kChunk, n, n, lost, lg, lc, qf, ql, fac, seen, o, m, l);
      take = take + 1 == kListStages ? 0 : take + 1;
      phase ^= take == 0;
    }
#pragma unroll
    for (int e = 0; e < 2; ++e)
#pragma unroll
      for (int x = 4; x < 32; x <<= 1) l[0][e] += __shfl_xor_sync(0xffffffffu, l[0][e], x);
    const bool whole = use.c == 0 && use.c1 == nc;
    const int64_t at = (int64_t)use.i * A.a.out_stride + (int64_t)use.g * G * HD;
    const int first = W - (start < 0 ? (share - 1 - start) / share : 0), last = W + (start + nc - 1) / share;   // warps of the stream
    auto slot = [&](int w) { return A.part + (2 * (int64_t)w + (w == first ? 1 : 0)) * list_part<HD>(); };
    float* const part = slot(W);
    // a lane has rows 2 lc and 2 lc + 1, HD / 8 channels from lg * HD / 8 on
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      const int r = 2 * lc + e;
      if (r >= G) continue;
      const float inv = !whole ? 1.f : m[0][e] == -INFINITY ? 0.f : 1.f / l[0][e];
      if (!whole && lg == 0) part[r] = m[0][e], part[8 + r] = l[0][e];
#pragma unroll
      for (int t = 0; t < HD / 16; t += 2) {
        const int ch = lg * (HD / 8) + 2 * t;
        const float4 v = make_float4(o[0][t][e] * inv, o[0][t][e + 2] * inv, o[0][t + 1][e] * inv, o[0][t + 1][e + 2] * inv);
        if (!whole) *reinterpret_cast<float4*>(part + 16 + r * HD + ch) = v;
        else if (A.a.out_dtype == BUDDY_DTYPE_F32) *reinterpret_cast<float4*>((float*)A.a.out + at + r * HD + ch) = v;
        else *reinterpret_cast<uint2*>((bf16*)A.a.out + at + r * HD + ch) = make_uint2(tca::pack_bf16(v.x, v.y), tca::pack_bf16(v.z, v.w));
      }
    }
    if (!whole) {
      __syncwarp();      // the partial's writes come before the arrival, which releases them
      int arrived = 0;
      if (lane == 0) {
        arrived = ptx::atom_add_acq_rel(A.arrive + first, 1) == last - first;
        if (arrived) A.arrive[first] = 0;
      }
      if (__shfl_sync(0xffffffffu, arrived, 0)) {
        __syncwarp();
        // all rows at once, span by span: HD / 32 channels of each row per lane
        constexpr int CH = HD / 32;
        float M[8], L[8], v[8][CH];
#pragma unroll
        for (int r = 0; r < 8; ++r) {
          M[r] = -INFINITY, L[r] = 0.f;
#pragma unroll
          for (int x = 0; x < CH; ++x) v[r][x] = 0.f;
        }
#pragma unroll 2
        for (int w = first; w <= last; ++w) {
          const float* const p = slot(w);
          float pm[8], pl[8], y[8][CH];
#pragma unroll
          for (int r = 0; r < 8; ++r) {
            pm[r] = -INFINITY, pl[r] = 0.f;
#pragma unroll
            for (int x = 0; x < CH; ++x) y[r][x] = 0.f;
            if (r < G) {
              pm[r] = __ldcg(p + r), pl[r] = __ldcg(p + 8 + r);
              if constexpr (CH == 4) {
                const float4 z = __ldcg(reinterpret_cast<const float4*>(p + 16 + r * HD) + lane);
                y[r][0] = z.x, y[r][1] = z.y, y[r][CH - 2] = z.z, y[r][CH - 1] = z.w;
              } else {
                const float2 z = __ldcg(reinterpret_cast<const float2*>(p + 16 + r * HD) + lane);
                y[r][0] = z.x, y[r][1] = z.y;
              }
            }
          }
#pragma unroll
          for (int r = 0; r < 8; ++r) {
            const float to = fmaxf(M[r], pm[r]), ref = to == -INFINITY ? 0.f : to;
            const float a = tca::exp2a(M[r] - ref), b = tca::exp2a(pm[r] - ref);
            L[r] = a * L[r] + b * pl[r];
#pragma unroll
            for (int x = 0; x < CH; ++x) v[r][x] = a * v[r][x] + b * y[r][x];
            M[r] = to;
          }
        }
#pragma unroll
        for (int r = 0; r < 8; ++r) {
          if (r >= G) continue;
          const float inv = M[r] == -INFINITY ? 0.f : 1.f / L[r];
          const int64_t to = at + r * HD + lane * CH;
#pragma unroll
          for (int x = 0; x < CH; ++x) v[r][x] *= inv;
          if (A.a.out_dtype == BUDDY_DTYPE_F32) {
            if constexpr (CH == 4) *reinterpret_cast<float4*>((float*)A.a.out + to) = make_float4(v[r][0], v[r][1], v[r][CH - 2], v[r][CH - 1]);
            else *reinterpret_cast<float2*>((float*)A.a.out + to) = make_float2(v[r][0], v[r][1]);
          } else if constexpr (CH == 4) {
            *reinterpret_cast<uint2*>((bf16*)A.a.out + to) = make_uint2(tca::pack_bf16(v[r][0], v[r][1]), tca::pack_bf16(v[r][CH - 2], v[r][CH - 1]));
          } else {
            *reinterpret_cast<uint32_t*>((bf16*)A.a.out + to) = tca::pack_bf16(v[r][0], v[r][1]);
          }
        }
      }
    }
    start += nc + kListOpen;
    go = use.next(A);
  }
  if (abort_flag) {      // a copy did not come: the results are not whole; the others' writes are waited for
    volatile int ignored = 0;
    for (int s = 0; s < kListStages; ++s)
      if (issued > s)
        ptx::mbar_wait_bounded(&full[warp * kListStages + s], ((issued - s - 1) / kListStages) & 1, kWaitLimitNs, &ignored);
    if (lane == 0 && A.flags) atomicOr(A.flags, BUDDY_DEV_TIMEOUT);
  }
}

template <int HD, bool WIDE>
static int launch(const AttnArgs4& A, int sms, cudaStream_t s) {
  constexpr int64_t warps = (int64_t)kListMaxGrid * kListWarps;
  static_assert(warps * sizeof(int32_t) <= kWsCounters, "");
  static_assert(2 * warps * list_part<HD>() * sizeof(float) <= few_bytes(HD) - kWsCounters, "");
  auto* const kern = kv4_lists_kernel<HD, WIDE>;
  constexpr int smem = list_smem<HD>();
  if (cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, smem) != cudaSuccess) return BUDDY_ERR_CUDA;
  const int grid = std::min(kListMaxGrid, list_ctas<WIDE>() * sms);
  return launch_k(kern, grid, kListThreads, smem, s, true, A) == cudaSuccess ? BUDDY_OK : BUDDY_ERR_CUDA;
}

int launch_lists(const AttnArgs4& A, int head_dim, bool wide, int sms, cudaStream_t s) {
  if (head_dim == 128) return wide ? launch<128, true>(A, sms, s) : launch<128, false>(A, sms, s);
  return wide ? launch<64, true>(A, sms, s) : launch<64, false>(A, sms, s);
}

}  // namespace kv4
}  // namespace buddy
