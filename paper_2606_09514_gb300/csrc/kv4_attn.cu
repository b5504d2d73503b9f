// Causal attention over the paged 4-bit cache: few query rows per KV head (single
// tokens, proposed tokens checked at once).
//
// The rows of a (sequence, KV head) are (query token, head of the group) pairs, row
// r = token r / G, head r % G; up to 8 NB of them share a walk over the keys and
// values (a stream).  With so few rows the work is
// reading the cache and turning codes into numbers, which the tensor cores' mma.sync
// takes from registers: nothing goes back to shared memory.
//
//   S^T = K Q^T   m16n8k16, half: 16 positions x 8 rows.  The order of the channels
//                 in the contraction is free, so a lane takes HD / 4 consecutive
//                 ones: one wide load of codes is its A operand of all K steps.
//   softmax       base 2, per row (a column here): running reference m, which follows
//                 the maximum when that rises by more than 8 (p is 2^7 times that of the
//                 reference, 2^15 at most in half).
//   O^T += V^T P^T  16 channels x 8 rows; a lane takes HD / 8 consecutive channels of
//                 four positions, whose code words are put side by side by halves; P^T
//                 is S^T's accumulator transposed in registers (movmatrix).
//
// Codes become halves in one logical and one or two arithmetic instructions per pair
// (kv4_attn.cuh), exactly.  Queries are scaled by a power of two per row to 1 .. 2 and
// rounded to half (11 bits, below 2^-14 of the row's largest 2^-25 of it), the power goes
// into the softmax's factor.  Probabilities are rounded to half for the product only (their sum is taken
// before): each by 2^-11 of it at most, or 2^-32 of the row's largest where that is more.  With fp32
// queries or outputs (WIDE) both are sums of two halves: twice the MMAs and a CTA less per SM
// (64 sequences of 8,192 positions 148 us instead of 121; errors of 2^-12 become 2^-21).
//
// Work: all streams end to end, each as its chunks of 32 positions and kOpen chunks'
// worth for its beginning and end, in equal shares per CTA.  (With kOpen 4, 8, 10 and 12:
// 250 sequences of 512 to 8,192 positions and 4 KV heads 98.9, 93.0, 89.5 and 90.5 us; 31
// of 100 to 4,096 with up to five new tokens and 40 KV heads 76, 60, 60 and 61.)  A short
// stream belongs to the share where it begins: what a CTA saves by passing on a part of it,
// the partials cost again.  In a share, four warps take the chunks of a stream in turn or,
// where there are several short streams, a warp the whole of every fourth, without barriers
// and joins (250 sequences of 50 to 200 positions, 8 KV heads: 19.0 us, 25.5 with their
// chunks in turn; 1,000 of 20 to 250: 54 and 76; with long streams among them it loses, 250 of
// 30 to 1,000 take 40 us instead of 37, and a sixth more with up to 16 chunks instead of 12).
// Each warp has its own ring of stages, which runs on across streams: one lane copies a
// chunk in four bulk copies, in whole halves of 16 positions, and what lies behind the
// sequence's end, or has no page, is masked.  A stream within a share is written out; the CTAs of one
// that is cut write partials, which are joined in order by the last of them to arrive or,
// where they are many, by teams first (one sequence of 120,001 positions, 4 KV heads, 152
// CTAs each: 49 us with one join, 32 with teams).
//
// Bound by instructions: 64 sequences of 8,192 positions and 8 KV heads (567 MB) take 121 us,
// their copies alone 91 us (94% of HBM's rate), the arithmetic alone 100; a chunk is about
// 700 instructions of a warp, 350 of them codes to halves.  One token over 2,048 positions
// takes 9.0 us a call: 1 for the lengths and shares, 2 for the page ids and the first chunk, 1.5
// for two chunks, 4 for partials, arrival and join.
#include <cuda_runtime.h>

#include <algorithm>

#include "gemm_common.cuh"
#include "internal.h"
#include "kv4_attn.cuh"

namespace buddy {

bool kv4_cache_ok(const buddy_kv4_cache* c);
kv4::Pages kv4_pages(const buddy_kv4_cache* c);

namespace kv4 {

constexpr int kChunk = 32;
constexpr int kWarps = 4;
constexpr int kThreads = 32 * kWarps;
constexpr int kStages = 3;
// CTAs per SM: by registers (128 a thread with one block of eight rows, 168 with two; WIDE
// 168 and 255).
template <int NB, bool WIDE>
__host__ __device__ constexpr int ctas_per_sm() { return (NB == 1 ? 4 : 3) - (WIDE ? 1 : 0); }
constexpr int kWhole = 12;       // streams of at most this many chunks are not cut
constexpr int kOpen = 10;        // what beginning and ending a stream costs, in chunks
constexpr int kMany = 2 * kOpen; // shares from this on hold several short streams
constexpr int kMaxGrid = 1024;   // CTAs: four on each of at most 256 SMs
constexpr int kJoin = 8;         // partials in flight when a cut stream is joined
constexpr int kOneTeam = 24;     // spans up to which one CTA joins them all
constexpr int kTeam = 4;         // spans of a team: a multiple of this
// Rows of a KV head up to which these kernels take a sequence.  (With a limit of 32, 28 rows
// over 4 KV heads took, 16 sequences of 4,096 positions, 57 us here and 45 us with the
// prompts' kernel; one of 30,000 43 and 32; 100 of 600 67 and 68.)
constexpr int kFewRows = 16;

template <int HD>
__host__ __device__ constexpr int stage_bytes() { return 2 * kChunk * entry_bytes(HD); }
// A warp's outputs, maxima and sums when the warps are joined: with one block of rows in
// the stage that it has used last, which is free until its next copy.
template <int HD, int NB>
__host__ __device__ constexpr int join_bytes() { return 8 * NB * (HD + 4 + 2) * 4; }
template <int HD, int NB>
__host__ __device__ constexpr bool join_in_stage() { return join_bytes<HD, NB>() <= stage_bytes<HD>(); }
template <int HD, int NB>
__host__ __device__ constexpr int smem_bytes() {
  return kWarps * (kStages * stage_bytes<HD>() + (join_in_stage<HD, NB>() ? 0 : join_bytes<HD, NB>()));
}
// Arrival counters, then two partials per CTA: m and l of 8 NB rows, then their outputs.
template <int HD, int NB>
__host__ __device__ constexpr int64_t partial_floats() { return 8 * NB * (HD + 2); }

// Chunks of a stream of n positions.  (A sequence without positions: one of nothing.)
__device__ __forceinline__ int chunks_of(int n) { return max(1, (n + kChunk - 1) / kChunk); }
// A sequence with m = 0 where it has no rows here.
__device__ __forceinline__ Rows few_rows(const AttnArgs4& A, int i, bool* bad) {
  Rows q = rows_of(A, i, bad);
  if (q.m * A.G > A.row_limit) q.m = 0;
  return q;
}

// A walk over the streams of a CTA's share.
struct Walk {
  Rows q;
  int i, g, c, c1;            // sequence, KV head, chunks [c, c1) of the stream in this share
  int k;                      // streams of the share before this one
  int rem;                    // what is left of the share behind this stream
  // to the next stream; false at the share's end
  __device__ __forceinline__ bool next(const AttnArgs4& A) {
    rem -= kOpen;
    if (rem <= 0) return false;
    ++k;
    if (++g >= A.p.nkv) {
      g = 0;
      bool bad;
      do {
        q = few_rows(A, ++i, &bad);   // (with some of the share left there is another stream)
      } while (q.m == 0);
    }
    c = 0;
    c1 = chunks_of(q.n);
    if (c1 > kWhole) c1 = min(c1, rem);
    rem -= c1;
    return true;
  }
};

__device__ __forceinline__ void mma_f16(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0,
                                        uint32_t b1) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
      : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
      : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

__device__ __forceinline__ void bulk_load(uint32_t dst, const void* src, uint32_t bytes, uint32_t bar) {
  asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(dst),
               "l"(src), "r"(bytes), "r"(bar)
               : "memory");
}

// Position (of 16) of row r of S^T: odd and even neighbours, so that neither the key nor the
// value loads meet in a bank more than they have to.
__device__ __forceinline__ int place(int r) { return r ^ ((r >> 1) & 1); }

// Copies of a chunk's 16 or 32 positions from in_page on into a stage from position `at`
// on, by one lane: K codes, V codes, K scales, V scales (what lies behind the sequence's
// end is in the block too).
template <int HD, int N>
__device__ __forceinline__ void load_piece(const Pages& P, uint32_t dst, uint32_t bar, int page, int g, int in_page, int at) {
  constexpr int CB = code_bytes(HD), SB = scale_bytes(HD);
  // (the blocks' count fits in 32 bits: one has 576 bytes at least)
  const uint32_t block = (uint32_t)page * (uint32_t)P.nkv + (uint32_t)g;
  const uint8_t* const k = P.k + (uint64_t)block * (uint32_t)(entry_bytes(HD) << P.shift) + (uint32_t)(in_page * CB);
  const uint8_t* const v = k + (P.v - P.k);
  const uint32_t to_scales = (uint32_t)((CB << P.shift) - in_page * (CB - SB));
  bulk_load(dst + at * CB, k, N * CB, bar);
  bulk_load(dst + (kChunk + at) * CB, v, N * CB, bar);
  bulk_load(dst + 2 * kChunk * CB + at * SB, k + to_scales, N * SB, bar);
  bulk_load(dst + 2 * kChunk * CB + (kChunk + at) * SB, v + to_scales, N * SB, bar);
}

template <int HD, int NB, bool WIDE>
__global__ void __launch_bounds__(kThreads, ctas_per_sm<NB, WIDE>()) kv4_decode_kernel(const AttnArgs4 A) {
  extern __shared__ __align__(128) uint8_t smem[];
  __shared__ __align__(8) uint64_t full[kWarps * kStages];
  __shared__ volatile int abort_flag;
  constexpr int ROWS = 8 * NB, KS = HD / 16, LDO = HD + 4;
  __shared__ int s_stage[kWarps];
  // where warp w's part is: [row][LDO] outputs, then maxima and sums
  auto part_of = [&](int w) {
    return reinterpret_cast<float*>(smem + (join_in_stage<HD, NB>()
                                                ? (w * kStages + s_stage[w]) * stage_bytes<HD>()
                                                : kWarps * kStages * stage_bytes<HD>() + w * join_bytes<HD, NB>()));
  };
  constexpr int PM = ROWS * LDO, PL = PM + ROWS;
  __shared__ int64_t s_sum[kWarps], s_at;
  __shared__ int s_first, s_last;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, lg = lane >> 2, lc = lane & 3;
  const int B = A.a.batch, G = A.G;
  if (tid < kWarps * kStages) ptx::mbar_init(&full[tid], 1);
  if (tid == 0) abort_flag = 0;
  ptx::fence_mbar_init();
  __syncthreads();
  pdl_wait();
  pdl_trigger();   // (the prompts of the same call may start where there is room)

  // ---- this CTA's share: [lo, lo + share) of all streams' openings and chunks.  Where it
  // begins: sequence use.i and how far into that one's streams
  auto cost = [&](const Rows& q) { return q.m > 0 ? (int64_t)(chunks_of(q.n) + kOpen) * A.p.nkv : 0; };
  auto scan = [&](int64_t x) {      // over the warp
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int64_t v = __shfl_up_sync(0xffffffffu, x, o);
      if (lane >= o) x += v;
    }
    return x;
  };
  auto share_of = [&](int64_t total) {
    return (int)min((int64_t)INT32_MAX / 2, ((total + gridDim.x - 1) / gridDim.x + kWarps - 1) / kWarps * kWarps);
  };
  Walk use;
  int64_t total = 0, lo, at;
  int share;
  if (B <= 32) {                    // every warp by itself
    Rows q{0, 0, 0};
    bool bad = false;
    if (lane < B) q = few_rows(A, lane, &bad);
    if (__any_sync(0xffffffffu, bad) && blockIdx.x == 0 && tid == 0 && A.flags) atomicOr(A.flags, BUDDY_DEV_BAD_POSITION);
    const int64_t mine = cost(q), upto = scan(mine);
    total = __shfl_sync(0xffffffffu, upto, 31);
    if (total == 0) return;
    share = share_of(total);
    lo = (int64_t)blockIdx.x * share;
    if (lo >= total) return;
    use.i = __ffs(__ballot_sync(0xffffffffu, lo < upto)) - 1;
    at = lo - __shfl_sync(0xffffffffu, upto - mine, use.i);
    use.q.t0 = __shfl_sync(0xffffffffu, q.t0, use.i);
    use.q.m = __shfl_sync(0xffffffffu, q.m, use.i);
    use.q.n = __shfl_sync(0xffffffffu, q.n, use.i);
  } else {
    const int per = (B + kThreads - 1) / kThreads;
    const int b0 = min(B, tid * per), b1 = min(B, b0 + per);
    int64_t mine = 0;
    bool any_bad = false;
#pragma unroll 1
    for (int i = b0; i < b1; ++i) {
      bool bad;
      mine += cost(few_rows(A, i, &bad));
      any_bad |= bad;
    }
    if (any_bad && blockIdx.x == 0 && A.flags) atomicOr(A.flags, BUDDY_DEV_BAD_POSITION);
    int64_t upto = scan(mine);
    if (lane == 31) s_sum[warp] = upto;
    __syncthreads();
    for (int w = 0; w < kWarps; ++w) {
      if (w == warp) upto += total;
      total += s_sum[w];
    }
    if (total == 0) return;
    share = share_of(total);
    lo = (int64_t)blockIdx.x * share;
    if (lo >= total) return;
    if (upto - mine <= lo && lo < upto) {
      int64_t x = upto - mine;
#pragma unroll 1
      for (int i = b0; i < b1; ++i) {
        bool bad;
        const int64_t n = cost(few_rows(A, i, &bad));
        if (lo < x + n) {
          s_first = i;
          s_at = lo - x;
          break;
        }
        x += n;
      }
    }
    __syncthreads();
    bool bad;
    use.i = s_first;
    at = s_at;
    use.q = few_rows(A, use.i, &bad);
  }
  use.k = 0;
  int start;                        // where the stream's first chunk is, from the share's beginning on
  {
    const int nc = chunks_of(use.q.n);
    use.g = (int)(at / (nc + kOpen));
    const int x = (int)(at - (int64_t)use.g * (nc + kOpen)) - kOpen;   // chunk of the stream; below 0: its opening
    start = -x;
    use.rem = (int)min((int64_t)share, total - lo) + min(x, 0);
    use.c = max(x, 0);
    if (use.rem <= 0) return;
    if (x > 0 && nc <= kWhole) {         // the CTA before has it all
      use.rem -= nc - x;
      start += nc + kOpen;
      if (!use.next(A)) return;
    } else {
      use.c1 = nc <= kWhole ? nc : min(nc, use.c + use.rem);
      use.rem -= use.c1 - use.c;
    }
  }
  Walk ld = use;
  bool more = true;                 // (the walk's, until a copy does not come)
  // Where a share holds several short streams, a warp takes the whole of every fourth.
  const bool many = share >= kMany;
  auto owned = [&](const Walk& w) { return NB == 1 && many && w.q.n <= kWhole * kChunk; };
  auto enter = [&](const Walk& w) { return owned(w) ? (w.k % kWarps == warp ? 0 : w.c1) : w.c + warp; };
  ld.c = enter(ld);
  int ld_step = owned(ld) ? 1 : kWarps;
  const uint32_t ring = ptx::smem_u32(smem) + warp * kStages * stage_bytes<HD>();

  // The load walk stands on the chunk to copy next; its page ids, of the lower and the upper
  // 16 positions, are read a chunk early.  (A chunk of nothing reads the row's first.)
  int id0 = -1, id1 = -1;
  auto fetch_ids = [&]() {
    if (ld.c >= ld.c1) {
      do {
        more = ld.next(A);
        ld.c = enter(ld);
        ld_step = owned(ld) ? 1 : kWarps;
      } while (more && ld.c >= ld.c1);
      if (!more) return;
    }
    const int p0 = ld.c * kChunk;
    const int32_t* row = A.a.table + (int64_t)ld.i * A.a.max_pages;
    id0 = id1 = row[p0 >> A.p.shift];
    if (A.p.shift == 4 && p0 + 16 < ld.q.n) id1 = row[(p0 >> 4) + 1];
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
      if (lane == 0 && A.flags && p0 < ld.q.n) atomicOr(A.flags, BUDDY_DEV_BAD_PAGE);
      gone |= lost << (2 * ahead);
    }
    __syncwarp();
    if (ptx::elect_one()) {
      uint64_t* const bar = &full[warp * kStages + stage];
      const uint32_t dst = ring + stage * stage_bytes<HD>(), b = ptx::smem_u32(bar);
      ptx::mbar_arrive_expect_tx(bar, (2 - __popc(lost)) * 16 * 2 * entry_bytes(HD));
      if (A.p.shift > 4) {
        if (lost == 0) load_piece<HD, kChunk>(A.p, dst, b, id0, ld.g, p0 & ((1 << A.p.shift) - 1), 0);
      } else {
        if (!(lost & 1)) load_piece<HD, 16>(A.p, dst, b, id0, ld.g, 0, 0);
        if (!(lost & 2)) load_piece<HD, 16>(A.p, dst, b, id1, ld.g, 0, 16);
      }
    }
    ld.c += ld_step;
    ++issued;
    fetch_ids();
  };
  fetch_ids();
#pragma unroll 1
  for (int s = 0; s < kStages - 1; ++s) issue(s, s);

  // where a lane's codes and scales are in a stage: keys of row lg, values of rows 2 lc and 2 lc + 1
  constexpr int VC = kChunk * code_bytes(HD), KSC = 2 * VC, VSC = KSC + kChunk * scale_bytes(HD);
  const int k_at = place(lg) * code_bytes(HD) + lc * (HD / 8);
  const int ks_at = KSC + place(lg) * scale_bytes(HD) + (lc * (HD / 4) / 32) * 2;
  int v_at[2], vs_at[2];
#pragma unroll
  for (int u = 0; u < 2; ++u) {
    v_at[u] = VC + place(2 * lc + u) * code_bytes(HD) + lg * (HD / 16);
    vs_at[u] = VSC + place(2 * lc + u) * scale_bytes(HD) + (lg * (HD / 8) / 32) * 2;
  }

  for (bool go = true; go;) {
    // ---- one stream (or the part of it in this share)
    const int g = use.g, rows = use.q.m * G, n = use.q.n, nc = chunks_of(n);
    const bool whole = use.c == 0 && use.c1 == nc, own = owned(use);
    const int c0 = enter(use), step = own ? 1 : kWarps;
    if (own && c0 == use.c1) {      // another warp's
      start += nc + kOpen;
      go = use.next(A);
      continue;
    }
    // queries: rows lg of each block of eight, this lane's HD / 4 channels
    uint32_t qf[NB][KS][2], ql[WIDE ? NB : 1][KS][2];
    float fac[NB][2];               // of the scores of rows 2 lc and 2 lc + 1
    int seen[NB][2];
#pragma unroll
    for (int b = 0; b < NB; ++b) {
      const int r = min(8 * b + lg, rows - 1);
      const int64_t at = (use.q.t0 + r / G) * A.a.q_stride + (int64_t)(g * G + r % G) * HD + lc * (HD / 4);
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
        qf[b][e / 4][(e / 2) & 1] = y.hi;
        if constexpr (WIDE) ql[b][e / 4][(e / 2) & 1] = y.lo;
      }
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        fac[b][e] = __shfl_sync(0xffffffffu, f, (2 * lc + e) * 4);
        // (rows that are not there repeat the last)
        seen[b][e] = n - use.q.m + min(8 * b + 2 * lc + e, rows - 1) / G + 1;
      }
    }
    const int all_seen = n - use.q.m + 1;   // positions that every row sees
    float o[NB][HD / 16][4], m[NB][2], l[NB][2];
#pragma unroll
    for (int b = 0; b < NB; ++b) {
      m[b][0] = m[b][1] = -INFINITY;
      l[b][0] = l[b][1] = 0.f;
#pragma unroll
      for (int t = 0; t < HD / 16; ++t)
#pragma unroll
        for (int e = 0; e < 4; ++e) o[b][t][e] = 0.f;
    }

    for (int c = c0; c < use.c1; c += step) {
      if (!__all_sync(0xffffffffu, ptx::mbar_wait_bounded(&full[warp * kStages + take], phase, kWaitLimitNs, &abort_flag)))
        more = false;
      const uint8_t* st = smem + (warp * kStages + take) * stage_bytes<HD>();
      const uint32_t lost = gone & 3u;
      gone >>= 2;
      issue(take == 0 ? kStages - 1 : take - 1, kStages - 2);   // to the stage that the chunk before this one has left
      const int p0 = c * kChunk;

      // ---- S^T
      float s[NB][2][4];
#pragma unroll
      for (int b = 0; b < NB; ++b)
#pragma unroll
        for (int t = 0; t < 2; ++t) s[b][t][0] = s[b][t][1] = s[b][t][2] = s[b][t][3] = 0.f;
      {
        uint32_t w[2][2][HD / 32];                   // codes of positions 16 t + 8 u + place(lg)
        __half2 sc[2][2], s72[2][2];
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
          for (int u = 0; u < 2; ++u) {
            const uint8_t* src = st + k_at + (16 * t + 8 * u) * code_bytes(HD);
            if constexpr (HD == 128) {
              const uint4 v = *reinterpret_cast<const uint4*>(src);
              w[t][u][0] = v.x, w[t][u][1] = v.y, w[t][u][HD / 32 - 2] = v.z, w[t][u][HD / 32 - 1] = v.w;
            } else {
              const uint2 v = *reinterpret_cast<const uint2*>(src);
              w[t][u][0] = v.x, w[t][u][1] = v.y;
            }
            sc[t][u] = __half2half2(*reinterpret_cast<const __half*>(st + ks_at + (16 * t + 8 * u) * scale_bytes(HD)));
            s72[t][u] = __hmul2(sc[t][u], __float2half2_rn(-72.f));
          }
#pragma unroll
        for (int i = 0; i < HD / 32; ++i)
#pragma unroll
          for (int t = 0; t < 2; ++t) {
            uint32_t x[4], y[4];
            dequant4(w[t][0][i], sc[t][0], s72[t][0], x);
            dequant4(w[t][1][i], sc[t][1], s72[t][1], y);
#pragma unroll
            for (int b = 0; b < NB; ++b) {
              mma_f16(s[b][t], x[0], y[0], x[1], y[1], qf[b][2 * i][0], qf[b][2 * i][1]);
              mma_f16(s[b][t], x[2], y[2], x[3], y[3], qf[b][2 * i + 1][0], qf[b][2 * i + 1][1]);
              if constexpr (WIDE) {
                mma_f16(s[b][t], x[0], y[0], x[1], y[1], ql[b][2 * i][0], ql[b][2 * i][1]);
                mma_f16(s[b][t], x[2], y[2], x[3], y[3], ql[b][2 * i + 1][0], ql[b][2 * i + 1][1]);
              }
            }
          }
      }
      // ---- mask and softmax
      uint32_t pt[NB][2][2], pl[WIDE ? NB : 1][2][2];
      const bool cut = p0 + kChunk > all_seen || lost != 0;
#pragma unroll
      for (int b = 0; b < NB; ++b) {
        if (cut) {
#pragma unroll
          for (int t = 0; t < 2; ++t)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const int p = p0 + 16 * t + place(lg) + 8 * (e >> 1);
              if (p >= seen[b][e & 1] || ((lost >> t) & 1)) s[b][t][e] = -INFINITY;
            }
        }
        float mx[2];
#pragma unroll
        for (int e = 0; e < 2; ++e)
          mx[e] = fmaxf(fmaxf(s[b][0][e], s[b][0][e + 2]), fmaxf(s[b][1][e], s[b][1][e + 2])) * fac[b][e];
        if (__any_sync(0xffffffffu, mx[0] > m[b][0] + 8.f || mx[1] > m[b][1] + 8.f)) {
          float al[2];
#pragma unroll
          for (int e = 0; e < 2; ++e) {
#pragma unroll
            for (int x = 4; x < 32; x <<= 1) mx[e] = fmaxf(mx[e], __shfl_xor_sync(0xffffffffu, mx[e], x));
            const float to = fmaxf(m[b][e], mx[e]);
            al[e] = to == -INFINITY ? 1.f : tca::exp2a(m[b][e] - to);
            m[b][e] = to;
            l[b][e] *= al[e];
          }
#pragma unroll
          for (int t = 0; t < HD / 16; ++t)
#pragma unroll
            for (int e = 0; e < 4; ++e) o[b][t][e] *= al[e & 1];
        }
        const float ref[2] = {m[b][0] == -INFINITY ? 0.f : m[b][0] - kHigh, m[b][1] == -INFINITY ? 0.f : m[b][1] - kHigh};
#pragma unroll
        for (int t = 0; t < 2; ++t) {
          float p[4];
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            p[e] = tca::exp2a(fmaf(s[b][t][e], fac[b][e & 1], -ref[e & 1]));
            l[b][e & 1] += p[e];
          }
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            const Halves<WIDE> y(p[2 * e], p[2 * e + 1]);
            pt[b][t][e] = tca::movt(y.hi);
            if constexpr (WIDE) pl[b][t][e] = tca::movt(y.lo);
          }
        }
      }
      // ---- O^T: this lane's four positions of each 16, channels lg * HD / 8 on
      // scales of pairs of positions, [16 positions][pairs 0 1, 8 9 of the contraction]
      __half2 vsc[2][2];
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int u = 0; u < 2; ++u)
          vsc[t][u] = __halves2half2(*reinterpret_cast<const __half*>(st + vs_at[0] + (16 * t + 8 * u) * scale_bytes(HD)),
                                     *reinterpret_cast<const __half*>(st + vs_at[1] + (16 * t + 8 * u) * scale_bytes(HD)));
      int nan_at = INT32_MAX;                         // first position whose values here are NaN
      bool has_nan = false;
      if (cut) {
        // What lies behind the sequence's end, or was not copied, counts as zeros.  And a NaN
        // must not meet the zero probabilities of rows that do not see its position: its
        // values count as zeros, and the rows that do see it become NaN below.
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
          for (int u = 0; u < 2; ++u) {
            __half x[2] = {__low2half(vsc[t][u]), __high2half(vsc[t][u])};
#pragma unroll
            for (int e = 0; e < 2; ++e) {
              const int pos = p0 + 16 * t + place(2 * lc + e) + 8 * u;
              const bool real = pos < n && !((lost >> t) & 1), nan = __hisnan(x[e]);
              if (real && nan) nan_at = min(nan_at, pos);
              if (!real || nan) x[e] = __float2half_rn(0.f);
            }
            vsc[t][u] = __halves2half2(x[0], x[1]);
          }
        has_nan = __any_sync(0xffffffffu, nan_at != INT32_MAX);
      }
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        const __half2 k72 = __float2half2_rn(-72.f);
        const __half2 sa = vsc[t][0], sb = vsc[t][1], sa72 = __hmul2(sa, k72), sb72 = __hmul2(sb, k72);
        uint32_t w[4][HD / 64];
#pragma unroll
        for (int u = 0; u < 4; ++u) {
          const uint32_t* src =
              reinterpret_cast<const uint32_t*>(st + v_at[u & 1] + (16 * t + 8 * (u >> 1)) * code_bytes(HD));
          if constexpr (HD == 128) {
            const uint2 v = *reinterpret_cast<const uint2*>(src);
            w[u][0] = v.x;
            w[u][HD / 64 - 1] = v.y;
          } else {
            w[u][0] = *src;
          }
        }
#pragma unroll
        for (int x = 0; x < HD / 64; ++x) {
          uint32_t a[4][4];
          dequant4(__byte_perm(w[0][x], w[1][x], 0x5410), sa, sa72, a[0]);
          dequant4(__byte_perm(w[0][x], w[1][x], 0x7632), sa, sa72, a[1]);
          dequant4(__byte_perm(w[2][x], w[3][x], 0x5410), sb, sb72, a[2]);
          dequant4(__byte_perm(w[2][x], w[3][x], 0x7632), sb, sb72, a[3]);
#pragma unroll
          for (int j = 0; j < 4; ++j) {
#pragma unroll
            for (int b = 0; b < NB; ++b) {
              mma_f16(o[b][4 * x + j], a[0][j], a[1][j], a[2][j], a[3][j], pt[b][t][0], pt[b][t][1]);
              if constexpr (WIDE) mma_f16(o[b][4 * x + j], a[0][j], a[1][j], a[2][j], a[3][j], pl[b][t][0], pl[b][t][1]);
            }
          }
        }
      }
      if (has_nan) {
        nan_at = min(nan_at, __shfl_xor_sync(0xffffffffu, nan_at, 1));
        nan_at = min(nan_at, __shfl_xor_sync(0xffffffffu, nan_at, 2));
#pragma unroll
        for (int b = 0; b < NB; ++b)
#pragma unroll
          for (int t = 0; t < HD / 16; ++t)
#pragma unroll
            for (int e = 0; e < 4; ++e)
              if (nan_at < seen[b][e & 1]) o[b][t][e] = __uint_as_float(0x7FC00000u);
      }
      take = take + 1 == kStages ? 0 : take + 1;
      phase ^= take == 0;
    }

    auto out4 = [&](int r, int ch, float4 v) {
      const int64_t at = (use.q.t0 + r / G) * A.a.out_stride + (int64_t)(g * G + r % G) * HD + ch;
      if (A.a.out_dtype == BUDDY_DTYPE_F32) {
        *reinterpret_cast<float4*>((float*)A.a.out + at) = v;
      } else {
        *reinterpret_cast<uint2*>((bf16*)A.a.out + at) = make_uint2(tca::pack_bf16(v.x, v.y), tca::pack_bf16(v.z, v.w));
      }
    };
    if (own) {
#pragma unroll
      for (int b = 0; b < NB; ++b)
#pragma unroll
        for (int e = 0; e < 2; ++e) {
#pragma unroll
          for (int x = 4; x < 32; x <<= 1) l[b][e] += __shfl_xor_sync(0xffffffffu, l[b][e], x);
          const int r = 8 * b + 2 * lc + e;
          if (r < rows) {
            const float inv = m[b][e] == -INFINITY ? 0.f : 1.f / l[b][e];
#pragma unroll
            for (int t = 0; t < HD / 16; t += 2)
              out4(r, lg * (HD / 8) + 2 * t, make_float4(o[b][t][e] * inv, o[b][t][e + 2] * inv, o[b][t + 1][e] * inv,
                                                         o[b][t + 1][e + 2] * inv));
          }
        }
      start += nc + kOpen;
      go = use.next(A);
      continue;
    }
    // ---- join the warps, in the stages taken last: a lane has rows 2 lc, 2 lc + 1 of each block,
    // HD / 8 channels from lg * HD / 8 on
    if (lane == 0) s_stage[warp] = take == 0 ? kStages - 1 : take - 1;
    __syncwarp();
    float* const mine = part_of(warp);
#pragma unroll
    for (int b = 0; b < NB; ++b)
#pragma unroll
      for (int e = 0; e < 2; ++e) {
#pragma unroll
        for (int x = 4; x < 32; x <<= 1) l[b][e] += __shfl_xor_sync(0xffffffffu, l[b][e], x);
        const int r = 8 * b + 2 * lc + e;
        if (r < rows) {
          if (lg == 0) mine[PM + r] = m[b][e], mine[PL + r] = l[b][e];
          float4* d = reinterpret_cast<float4*>(mine + r * LDO + lg * (HD / 8));
#pragma unroll
          for (int t = 0; t < HD / 16; t += 2)
            d[t / 2] = make_float4(o[b][t][e], o[b][t][e + 2], o[b][t + 1][e], o[b][t + 1][e + 2]);
        }
      }
    __syncthreads();
    // the CTAs that have parts of the stream: from the one of its first chunk (start may lie
    // before this share) to the one of its last
    const int first_cta = (int)blockIdx.x - (start < 0 ? (share - 1 - start) / share : 0);
    const int last_cta = (int)blockIdx.x + (start + nc - 1) / share;
    float* part = A.part + (2 * (int64_t)blockIdx.x + ((int)blockIdx.x == first_cta ? 1 : 0)) * partial_floats<HD, NB>();
    for (int x = tid; x < rows * (HD / 4); x += kThreads) {
      const int r = x / (HD / 4), ch = x % (HD / 4) * 4;
      float M = -INFINITY, L = 0.f;
      float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
      for (int w = 0; w < kWarps; ++w) M = fmaxf(M, part_of(w)[PM + r]);
#pragma unroll
      for (int w = 0; w < kWarps; ++w) {
        const float* const pw = part_of(w);
        const float mw = pw[PM + r], a = mw == -INFINITY ? 0.f : tca::exp2a(mw - M);
        const float4 y = *reinterpret_cast<const float4*>(pw + r * LDO + ch);
        L += a * pw[PL + r];
        v.x += a * y.x, v.y += a * y.y, v.z += a * y.z, v.w += a * y.w;
      }
      if (whole) {
        const float inv = M == -INFINITY ? 0.f : 1.f / L;
        out4(r, ch, make_float4(v.x * inv, v.y * inv, v.z * inv, v.w * inv));
      } else {
        if (ch == 0) part[r] = M, part[ROWS + r] = L;
        *reinterpret_cast<float4*>(part + 2 * ROWS + r * HD + ch) = v;
      }
    }
    if (!whole) {
      constexpr int64_t PF = partial_floats<HD, NB>();
      const int spans = last_cta - first_cta + 1, span = (int)blockIdx.x - first_cta;
      const int items = rows * (HD / 4);
      // few rows: the spans go over as many groups of threads as there are
      const int groups = items < kThreads ? kThreads / items : 1, grp = items < kThreads ? tid / items : 0;
      auto slot = [&](int cta, int which) { return A.part + (2 * (int64_t)cta + which) * PF; };
      // `count` partials, partial k at from(k), kJoin at a time into a running log-sum-exp
      auto join = [&](int count, auto from, auto emit) {
#pragma unroll 1
        for (int x = tid - grp * items; x < items && grp < groups; x += kThreads) {
          const int r = x / (HD / 4), ch = x % (HD / 4) * 4;
          float M = -INFINITY, L = 0.f;
          float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 1
          for (int k0 = grp; k0 < count; k0 += kJoin * groups) {
            float m[kJoin], l[kJoin], to = M;
            float4 y[kJoin];
#pragma unroll
            for (int i = 0; i < kJoin; ++i) {
              const int k = k0 + i * groups;
              m[i] = -INFINITY, l[i] = 0.f, y[i] = make_float4(0.f, 0.f, 0.f, 0.f);
              if (k < count) {
                const float* p = from(k);
                m[i] = __ldcg(p + r), l[i] = __ldcg(p + ROWS + r);
                y[i] = __ldcg(reinterpret_cast<const float4*>(p + 2 * ROWS + x * 4));
              }
            }
#pragma unroll
            for (int i = 0; i < kJoin; ++i) to = fmaxf(to, m[i]);
            const float at = to == -INFINITY ? 0.f : to, a = tca::exp2a(M - at);
            L *= a, v.x *= a, v.y *= a, v.z *= a, v.w *= a;
#pragma unroll
            for (int i = 0; i < kJoin; ++i) {
              const float b = tca::exp2a(m[i] - at);
              L += b * l[i];
              v.x += b * y[i].x, v.y += b * y[i].y, v.z += b * y[i].z, v.w += b * y[i].w;
            }
            M = to;
          }
          if (groups == 1) {
            emit(r, ch, M, L, v);
          } else {
            reinterpret_cast<float4*>(part_of(0))[grp * items + x] = v;
            if (ch == 0) part_of(0)[PM + grp * rows + r] = M, part_of(0)[PL + grp * rows + r] = L;
          }
        }
        if (groups > 1) {
          __syncthreads();
          if (tid < items) {
            const int r = tid / (HD / 4), ch = tid % (HD / 4) * 4;
            float M = -INFINITY, L = 0.f;
            float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
            const float* const pw = part_of(0);
            for (int k = 0; k < groups; ++k) M = fmaxf(M, pw[PM + k * rows + r]);
            const float at = M == -INFINITY ? 0.f : M;
            for (int k = 0; k < groups; ++k) {
              const float a = tca::exp2a(pw[PM + k * rows + r] - at);
              const float4 y = reinterpret_cast<const float4*>(pw)[k * items + tid];
              L += a * pw[PL + k * rows + r];
              v.x += a * y.x, v.y += a * y.y, v.z += a * y.z, v.w += a * y.w;
            }
            emit(r, ch, M, L, v);
          }
        }
      };
      auto finish = [&](int r, int ch, float M, float L, float4 v) {
        const float inv = M == -INFINITY ? 0.f : 1.f / L;
        out4(r, ch, make_float4(v.x * inv, v.y * inv, v.z * inv, v.w * inv));
      };
      // True in the last of `count` CTAs that come here with this counter.
      auto last_of = [&](int counter, int count) {
        __syncthreads();   // the partial's writes come before the arrival, which releases them
        if (tid == 0) {
          s_last = ptx::atom_add_acq_rel(A.arrive + counter, 1) == count - 1;
          if (s_last) A.arrive[counter] = 0;
        }
        __syncthreads();
        return s_last != 0;
      };
      // The first span's partial is its CTA's second one, the others are their CTAs' first.
      auto span_at = [&](int k) { return slot(first_cta + k, k == 0 ? 1 : 0); };
      if (spans <= kOneTeam) {
        if (last_of(first_cta, spans)) join(spans, span_at, finish);
      } else {
        // Many spans: in about as many teams as a team has spans, then the teams.  What a team
        // has joined goes to the second partial of a CTA that begins no stream, its first one
        // (of the first team: its second), whose counter is the team's.
        int team = kTeam;
        while (team * team < spans) team += kTeam;
        const int teams = (spans + team - 1) / team, mine_k = span / team;
        auto host = [&](int t) { return first_cta + (t == 0 ? 1 : t * team); };
        const int in_team = min(team, spans - mine_k * team);
        bool go_on = true;
        if (in_team > 1) {
          go_on = last_of(host(mine_k), in_team);
          if (go_on) {
            float* const to = slot(host(mine_k), 1);
            join(in_team, [&](int k) { return span_at(mine_k * team + k); },
                 [&](int r, int ch, float M, float L, float4 v) {
                   if (ch == 0) to[r] = M, to[ROWS + r] = L;
                   *reinterpret_cast<float4*>(to + 2 * ROWS + r * HD + ch) = v;
                 });
          }
        }
        if (go_on && last_of(first_cta, teams))
          join(teams, [&](int t) { return t * team + 1 == spans ? span_at(t * team) : slot(host(t), 1); }, finish);
      }
    }
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    __syncthreads();     // the warps' parts are free again
    start += nc + kOpen;
    go = use.next(A);
  }
  if (abort_flag) {      // a copy did not come: the results are not whole; the others' writes are waited for
    volatile int ignored = 0;
    for (int s = 0; s < kStages; ++s)
      if (issued > s)
        ptx::mbar_wait_bounded(&full[warp * kStages + s], ((issued - s - 1) / kStages) & 1, kWaitLimitNs, &ignored);
    if (lane == 0 && A.flags) atomicOr(A.flags, BUDDY_DEV_TIMEOUT);
  }
}

}  // namespace kv4

using namespace kv4;

static int sm_count() {
  int dev = 0, n = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess)
    return 0;
  return n;
}

template <int HD, int NB, bool WIDE>
static int launch_decode(const AttnArgs4& A, int64_t most, int sms, cudaStream_t s) {
  constexpr int smem = smem_bytes<HD, NB>();
  const int grid = (int)std::min<int64_t>(most, std::min(kMaxGrid, ctas_per_sm<NB, WIDE>() * sms));
  if (cudaFuncSetAttribute(kv4_decode_kernel<HD, NB, WIDE>, cudaFuncAttributeMaxDynamicSharedMemorySize, smem) != cudaSuccess)
    return BUDDY_ERR_CUDA;
  return launch_k(kv4_decode_kernel<HD, NB, WIDE>, grid, kThreads, smem, s, true, A) == cudaSuccess ? BUDDY_OK : BUDDY_ERR_CUDA;
}
template <int HD, bool WIDE>
static int launch_few(const AttnArgs4& A, bool two, int64_t most, int sms, cudaStream_t s) {
  return two ? launch_decode<HD, 2, WIDE>(A, most, sms, s) : launch_decode<HD, 1, WIDE>(A, most, sms, s);
}

}  // namespace buddy

using namespace buddy;

constexpr int64_t kWsCounters = 4096;   // bytes of arrival counters in front of a workspace
static int64_t few_bytes(int head_dim) { return kWsCounters + (int64_t)kMaxGrid * 2 * 16 * (head_dim + 2) * 4; }

static bool sizes_ok(int32_t n_q_heads, int32_t n_kv_heads, int32_t head_dim, int32_t max_new) {
  return n_kv_heads >= 1 && n_kv_heads <= 1024 && n_q_heads >= n_kv_heads && n_q_heads % n_kv_heads == 0 &&
         n_q_heads / n_kv_heads <= 8 && (head_dim == 64 || head_dim == 128) && max_new >= 1;
}
static int64_t workspace_bytes(int group, int head_dim, int max_new, int sms) {
  return few_bytes(head_dim) + ((int64_t)max_new * group > kFewRows ? prompt_workspace(head_dim, sms) : 0);
}

extern "C" int64_t buddy_kv4_attention_workspace(int32_t n_q_heads, int32_t n_kv_heads, int32_t head_dim,
                                                 int32_t max_new) {
  if (!sizes_ok(n_q_heads, n_kv_heads, head_dim, max_new)) return -1;
  const int sms = sm_count();
  return sms > 0 ? workspace_bytes(n_q_heads / n_kv_heads, head_dim, max_new, sms) : -1;
}

extern "C" int buddy_kv4_attention(const buddy_kv4_cache* cache, const buddy_kv4_attention_args* a, int32_t* flags,
                                   void* stream) {
  if (!kv4_cache_ok(cache) || !a || a->batch < 1 || a->batch > 16384 || a->n_tok < 0 || a->max_pages < 1 ||
      (int64_t)a->max_pages * cache->page_size > INT32_MAX || !(a->scale >= 0.f) || a->scale > 2.3e38f)   // (times log2(e) it is finite)
    return BUDDY_ERR_ARG;
  if (!sizes_ok(a->n_q_heads, cache->n_kv_heads, cache->head_dim, a->max_new) ||
      (a->q_dtype != BUDDY_DTYPE_F32 && a->q_dtype != BUDDY_DTYPE_BF16) ||
      (a->out_dtype != BUDDY_DTYPE_F32 && a->out_dtype != BUDDY_DTYPE_BF16) || !a->kv_len || !a->table)
    return BUDDY_ERR_ARG;
  if (!a->row_start && (a->n_tok != a->batch || a->max_new != 1)) return BUDDY_ERR_ARG;
  if (!a->workspace || a->workspace_bytes < few_bytes(cache->head_dim) ||
      (reinterpret_cast<uintptr_t>(a->workspace) & 255))
    return BUDDY_ERR_ARG;
  if (a->n_tok == 0) return BUDDY_OK;
  // rows are counted in 32 bits, up to the end of their last tile
  if ((int64_t)a->n_tok * a->n_q_heads >= (int64_t)INT32_MAX - 511) return BUDDY_ERR_RANGE;
  if (!a->q || !a->out || !aligned16(a->q) || !aligned16(a->out) ||
      a->q_stride * (a->q_dtype == BUDDY_DTYPE_F32 ? 4 : 2) % 16 || a->out_stride * (a->out_dtype == BUDDY_DTYPE_F32 ? 4 : 2) % 16)
    return BUDDY_ERR_ARG;
  const int sms = sm_count();
  if (sms == 0) return BUDDY_ERR_CUDA;
  if (a->workspace_bytes < workspace_bytes(a->n_q_heads / cache->n_kv_heads, cache->head_dim, a->max_new, sms))
    return BUDDY_ERR_ARG;
  AttnArgs4 A{*a, kv4_pages(cache), a->n_q_heads / cache->n_kv_heads, kFewRows, flags, (int32_t*)a->workspace,
              (float*)((uint8_t*)a->workspace + kWsCounters)};
  // The form by the most rows that a sequence may have here: a prompt in the call, too, sends
  // its single tokens through the form for 16 rows (not measured next to many of them).  One CTA
  // for every four chunks there can be, as many as run at once at most.
  const int64_t most_rows = (int64_t)a->max_new * A.G;
  const bool two = most_rows > 8;
  const int64_t chunks = ((int64_t)a->max_pages * cache->page_size + kv4::kChunk - 1) / kv4::kChunk;
  const int64_t most = (int64_t)a->batch * cache->n_kv_heads * (chunks + kOpen) / kWarps + 1;
  const bool wide = a->q_dtype == BUDDY_DTYPE_F32 || a->out_dtype == BUDDY_DTYPE_F32;
  cudaStream_t s = (cudaStream_t)stream;
  const int rc = cache->head_dim == 128
                     ? (wide ? launch_few<128, true>(A, two, most, sms, s) : launch_few<128, false>(A, two, most, sms, s))
                     : (wide ? launch_few<64, true>(A, two, most, sms, s) : launch_few<64, false>(A, two, most, sms, s));
  if (rc != BUDDY_OK || most_rows <= kFewRows) return rc;
  return launch_prompt(A, cache->head_dim, wide, sms, (uint8_t*)a->workspace + few_bytes(cache->head_dim), s);
}
