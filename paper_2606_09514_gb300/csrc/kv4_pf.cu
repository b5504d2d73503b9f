// Causal attention over the paged 4-bit cache: many query rows per KV head (prompts
// and pieces of prompts behind a prefix).
//
// The rows of a (sequence, KV head) are (query token, head of the group) pairs, row
// r = token r / G, head r % G; two tiles of 128 of them (an item) walk the same
// key/value tiles of 128 positions.  On the 5th-generation tensor cores, in half:
//   S = Q K^T   tcgen05.mma M = 128, N = 128, K = HD: queries and keys from shared memory, S in TMEM;
//   softmax     four warps per tile, a row per thread, base 2: running reference m,
//               which follows the maximum when that rises by more than 8; p, 2^7 times
//               that of the reference, back into TMEM as half over S's columns;
//   O += P V    M = 128, N = HD, K = 128: P from TMEM, V from shared memory (MN-major),
//               O in TMEM.
// Four producer warps take the codes of a tile's positions from the pages (a position per
// thread, in registers while the tile before is worked on) and write them
// as halves into the 128-byte-swizzled layout, two buffers each for keys and values.
// Positions past the end and pages that are not there become zeros and are masked.
// With fp32 queries or outputs (WIDE) queries and P are sums of two halves: an item is one tile
// of 128 rows, whose second halves take the second tile's place (the nine requests below 634 us
// instead of 257).
//
// Work: the items' tiles end to end, each item with kPfOpen tiles' worth for its
// beginning and end, in equal shares for one CTA per SM.  What an item that is cut
// has gathered (m, l, O of its rows) goes to the workspace, and a second kernel joins
// the parts in order.  Every wait is bounded.
//
// Nine requests of 1 to 1,500 new tokens behind 300 to 6,000 positions, 32 heads over 8:
// 257 us, 960 TFLOP/s, the tensor pipe busy for half of the time.  A tile of 256 rows and
// 128 positions takes about 3,500 cycles, 3,100 of them in its 32 MMAs of N = 128, 97 cycles each
// where the pipe alone would need 64.  What they wait for was not told apart: their issue (two
// issuing warps were slower), or shared memory, whose whole rate the operands of 64 cycles
// take, with 64 KB of producers' writes per tile next to them.
#include <cuda_runtime.h>

#include <algorithm>

#include "gemm_common.cuh"
#include "internal.h"
#include "kv4_attn.cuh"

namespace buddy {
namespace kv4 {

constexpr int kPfRows = 128, kPfKeys = 128;
constexpr int kPfSoftWarps = 8, kPfProducers = 128;
constexpr int kPfThreads = 512;          // four warpgroups: two of softmax, producers, the MMA warp's
// Registers: 128 a thread at launch (65,536 in all), then by setmaxnreg 2 x 128 x 184 +
// 128 x 80 + 128 x 64 = 65,536.  (What spills, in any role, is felt: nine requests take 260 us so, 275
// with 176, 88 and 72, 287 with 168, 96 and 80, 294 with 192, 72 and 56.)
constexpr int kPfRegsSoft = 184, kPfRegsProduce = 80, kPfRegsMma = 64, kPfRegs = 128;
static_assert(256 * kPfRegsSoft + kPfProducers * kPfRegsProduce + 128 * kPfRegsMma <= kPfThreads * kPfRegs,
              "the roles' registers come out of the launch's");
constexpr int kPfOpen = 4;               // what beginning and ending an item costs, in tiles
constexpr int kPfWhole = 4;              // items of at most this many tiles are not cut
constexpr uint32_t kPfRegion = 128u * 128u;   // 128 rows x 64 channels of half

template <int HD>
__host__ __device__ constexpr size_t pf_smem() {
  return (size_t)(HD / 64) * kPfRegion * 6 + 1024;   // two tiles of queries, two of keys, two of values; alignment
}
template <int HD>
__host__ __device__ constexpr int64_t pf_part_floats() { return 2 * kPfRows * (HD + 2); }

// Byte offset of 16-byte piece c of row r in a tile of 64-channel regions (128-byte
// rows, 128-byte swizzle).
__device__ __forceinline__ uint32_t pf_piece(int r, int c) {
  return (uint32_t)(c >> 3) * kPfRegion + (uint32_t)r * 128u + (uint32_t)(((c ^ r) & 7) << 4);
}

// A cut item, written by the CTA where it begins.
struct CutItem {
  int spans, t0, g, row0, rows;   // spans 0: none
  int pad[3];
};

struct PfItem {
  int seq, t0, m, n, g, R, row0, nt, j0, j1;
  int64_t start;                  // where the item's first tile is
  int go;                         // 0: the share's end, no item

  template <int IR>
  __device__ __forceinline__ int tiles() const { return IR > kPfRows && R - row0 > kPfRows ? 2 : 1; }   // tiles of rows
  __device__ __forceinline__ int len() const { return j1 - j0; }
};

template <int IR>
__device__ __forceinline__ int pf_tiles(int n, int m, int G, int R, int qp) {
  const int last = min(R, (qp + 1) * IR) - 1;
  return max(1, (max(n - m + last / G + 1, 0) + kPfKeys - 1) / kPfKeys);
}
// Cost of one KV head of a sequence (whole warp).
template <int IR>
__device__ __forceinline__ int64_t pf_head_cost(int n, int m, int G, int R, int lane) {
  const int nqp = (R + IR - 1) / IR;
  int64_t c = 0;
#pragma unroll 1
  for (int qp = lane; qp < nqp; qp += 32) c += pf_tiles<IR>(n, m, G, R, qp) + kPfOpen;
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) c += __shfl_xor_sync(0xffffffffu, c, o);
  return c;
}
// Cost of a KV head of sequence i0 + lane (0: not this kernel's, or not below end): a lane for
// itself where there are few items, the whole warp for the longer ones.
template <int IR>
__device__ __forceinline__ int64_t pf_block_costs(const AttnArgs4& A, int i0, int end, int lane, Rows* q) {
  *q = {0, 0, 0};
  bool bad;
  if (i0 + lane < end) *q = rows_of(A, i0 + lane, &bad);
  const int R = q->m * A.G, nqp = (R + IR - 1) / IR;
  int64_t c = 0;
  if (R > A.row_limit && nqp <= 4)
#pragma unroll 1
    for (int qp = 0; qp < nqp; ++qp) c += pf_tiles<IR>(q->n, q->m, A.G, R, qp) + kPfOpen;
  uint32_t longer = __ballot_sync(0xffffffffu, R > A.row_limit && nqp > 4);
#pragma unroll 1
  while (longer) {
    const int x = __ffs(longer) - 1;
    longer &= longer - 1;
    const int m = __shfl_sync(0xffffffffu, q->m, x);
    const int64_t v = pf_head_cost<IR>(__shfl_sync(0xffffffffu, q->n, x), m, A.G, m * A.G, lane);
    if (lane == x) c = v;
  }
  return c;
}
// First sequence from i on (below end) that is this kernel's; end if none (whole warp).
__device__ __forceinline__ int pf_next_seq(const AttnArgs4& A, int i, int end, int lane, Rows* q) {
#pragma unroll 1
  for (; i < end; i += 32) {
    Rows s{0, 0, 0};
    bool bad;
    if (i + lane < end) s = rows_of(A, i + lane, &bad);
    const uint32_t hit = __ballot_sync(0xffffffffu, s.m * A.G > A.row_limit);
    if (hit) {
      const int at = __ffs(hit) - 1;
      q->t0 = __shfl_sync(0xffffffffu, s.t0, at);
      q->m = __shfl_sync(0xffffffffu, s.m, at);
      q->n = __shfl_sync(0xffffffffu, s.n, at);
      return i + at;
    }
  }
  return end;
}

// The walk over a CTA's items, by one warp.
template <int IR>
struct PfWalk {
  Rows q;
  int i, g, qp, nt, j0, j1;
  int64_t rem, start;
  __device__ __forceinline__ bool next(const AttnArgs4& A, int lane) {
    start += nt + kPfOpen;
    rem -= kPfOpen;
    if (rem <= 0) return false;
    if (++qp * IR >= q.m * A.G) {
      qp = 0;
      if (++g == A.p.nkv) {
        g = 0;
        i = pf_next_seq(A, i + 1, A.a.batch, lane, &q);   // (with some of the share left there is another)
      }
    }
    nt = pf_tiles<IR>(q.n, q.m, A.G, q.m * A.G, qp);
    j0 = 0;
    j1 = nt <= kPfWhole ? nt : (int)min((int64_t)nt, rem);
    rem -= j1;
    return true;
  }
};

// Two fp32 at once.
__device__ __forceinline__ uint64_t pair(float a, float b) {
  uint64_t r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(a), "f"(b));
  return r;
}
__device__ __forceinline__ void unpair(uint64_t v, float& a, float& b) { asm("mov.b64 {%0, %1}, %2;" : "=f"(a), "=f"(b) : "l"(v)); }
__device__ __forceinline__ uint64_t fma2(uint64_t a, uint64_t b, uint64_t c) {
  uint64_t r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
  return r;
}
__device__ __forceinline__ uint64_t add2(uint64_t a, uint64_t b) {
  uint64_t r;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}

template <int N>
__device__ __forceinline__ void regs_up() { asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(N)); }
template <int N>
__device__ __forceinline__ void regs_down() { asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(N)); }

template <int HD, bool WIDE>
__global__ void __launch_bounds__(kPfThreads, 1) kv4_prompt_kernel(const AttnArgs4 A, CutItem* cuts) {
  extern __shared__ uint8_t smem_raw[];
  constexpr uint32_t TILE = (HD / 64) * kPfRegion;      // bytes of a 128-row tile
  constexpr int GR = HD / kGroup;                       // scale groups of a head
  // Rows of an item.  WIDE: one tile, the second buffer of queries holds their second halves, and
  // the second halves of P lie behind the first ones over S's columns.
  constexpr int IR = WIDE ? kPfRows : 2 * kPfRows;
  // TMEM columns: S of tile q at 128 q (P over their first half), O of tile q at 256 + 128 q
  constexpr uint32_t kO = 256;
  __shared__ __align__(8) uint64_t q_ready[2], k_full[2], k_empty[2], v_full[2], v_empty[2];
  __shared__ __align__(8) uint64_t s_full[2], p_ready[2][2], o_full[2], drained;
  __shared__ uint32_t tmem_slot;
  __shared__ volatile int abort_flag;
  __shared__ int64_t s_sum[kPfSoftWarps];
  __shared__ __align__(8) uint64_t item_full[2], item_empty[2];
  __shared__ PfItem s_first, s_item[2];                 // [item % 2]
  __shared__ int s_nan[2][GR];                          // [item % 2] first position whose values are NaN, by group
  __shared__ __align__(4) uint8_t s_ok[4][4];           // [tile % 4][32 positions]: two bits, pages that are there

  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int B = A.a.batch, G = A.G;
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  uint8_t* sQ = smem;                                   // [tile]
  uint8_t* sK = smem + 2 * TILE;                        // [2]
  uint8_t* sV = sK + 2 * TILE;                          // [2]
  constexpr int kMmaWarp = kPfSoftWarps + kPfProducers / 32;

  // ---- this CTA's share of all items' openings and tiles
  const int per = (B + kPfSoftWarps - 1) / kPfSoftWarps;
  const int b0 = min(B, warp * per), b1 = min(B, b0 + per);
  int64_t mine = 0;
  if (warp < kPfSoftWarps) {
    Rows q;
#pragma unroll 1
    for (int i0 = b0; i0 < b1; i0 += 32) mine += pf_block_costs<IR>(A, i0, b1, lane, &q);
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) mine += __shfl_xor_sync(0xffffffffu, mine, o);
    mine *= A.p.nkv;
    if (lane == 0) s_sum[warp] = mine;
  }
  if (tid == 0) {
    for (int b = 0; b < 2; ++b) {
      ptx::mbar_init(&q_ready[b], 128);
      ptx::mbar_init(&k_full[b], kPfProducers);
      ptx::mbar_init(&v_full[b], kPfProducers);
      ptx::mbar_init(&k_empty[b], 1);
      ptx::mbar_init(&v_empty[b], 1);
      ptx::mbar_init(&s_full[b], 1);
      ptx::mbar_init(&p_ready[b][0], 128);
      ptx::mbar_init(&p_ready[b][1], 128);
      ptx::mbar_init(&o_full[b], 1);
      ptx::mbar_init(&item_full[b], 1);
      ptx::mbar_init(&item_empty[b], kPfSoftWarps + kPfProducers / 32 + 1);
    }
    ptx::mbar_init(&drained, 1);
    abort_flag = 0;
    cuts[blockIdx.x].spans = 0;
    ptx::fence_mbar_init();
  }
  __syncthreads();
  int64_t total = 0, before = 0;
  for (int w = 0; w < kPfSoftWarps; ++w) {
    if (w < warp) before += s_sum[w];
    total += s_sum[w];
  }
  const int64_t share = max((int64_t)kPfWhole, (total + gridDim.x - 1) / gridDim.x);
  const int64_t lo = blockIdx.x * share;
  if (lo >= total) {
    pdl_wait();
    return;
  }
  if (warp < kPfSoftWarps && before <= lo && lo < before + mine) {
    // the sequence, its head, the item of it and the tile where the share begins
    PfWalk<IR> w;
    int64_t at = before, cost = 0;
#pragma unroll 1
    for (int i0 = b0;; i0 += 32) {
      const int64_t c = pf_block_costs<IR>(A, i0, b1, lane, &w.q);
      int64_t upto = c * A.p.nkv;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const int64_t v = __shfl_up_sync(0xffffffffu, upto, o);
        if (lane >= o) upto += v;
      }
      const uint32_t hit = __ballot_sync(0xffffffffu, lo < at + upto);
      if (hit || i0 + 32 >= b1) {
        const int x = hit ? __ffs(hit) - 1 : 31;
        w.i = i0 + x;
        cost = __shfl_sync(0xffffffffu, c, x);
        at += __shfl_sync(0xffffffffu, upto - c * A.p.nkv, x);
        w.q = {__shfl_sync(0xffffffffu, w.q.t0, x), __shfl_sync(0xffffffffu, w.q.m, x), __shfl_sync(0xffffffffu, w.q.n, x)};
        break;
      }
      at += __shfl_sync(0xffffffffu, upto, 31);
    }
    w.g = 0;
#pragma unroll 1
    for (; lo >= at + cost; at += cost) ++w.g;
    const int R = w.q.m * G, nqp = (R + IR - 1) / IR;
#pragma unroll 1
    for (int q0 = 0;; q0 += 32) {
      const int64_t c = q0 + lane < nqp ? pf_tiles<IR>(w.q.n, w.q.m, G, R, q0 + lane) + kPfOpen : 0;
      int64_t upto = c;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const int64_t v = __shfl_up_sync(0xffffffffu, upto, o);
        if (lane >= o) upto += v;
      }
      const uint32_t hit = __ballot_sync(0xffffffffu, lo < at + upto);
      if (hit || q0 + 32 >= nqp) {
        const int x = hit ? __ffs(hit) - 1 : 31;
        w.qp = q0 + x;
        at += __shfl_sync(0xffffffffu, upto - c, x);
        break;
      }
      at += __shfl_sync(0xffffffffu, upto, 31);
    }
    if (lane == 0)
      s_first = {w.i, w.q.t0, w.q.m, w.q.n, w.g, R, w.qp * IR, pf_tiles<IR>(w.q.n, w.q.m, G, R, w.qp), 0, 0,
                 at + kPfOpen, 1};
  }
  if (warp == kMmaWarp) {
    ptx::tmem_alloc(&tmem_slot, 512);
    ptx::tmem_relinquish();
  }
  ptx::tc_fence_before();
  __syncthreads();
  ptx::tc_fence_after();
  const uint32_t tmem = tmem_slot;

  // A warp walks the items and hands them to the roles, two at a time; a role gives an item
  // back when it is done with it, so that the producers are at the next item's keys and the
  // softmax warps have its queries on the way while this one's outputs are written.  The
  // counts of tiles and items so far give the mbarriers' phases: of all tiles and items,
  // and of those with a second tile of rows.
  uint32_t T = 0, I = 0, T1 = 0, I1 = 0;
  auto take = [&](uint32_t i) {    // whether there is an item i: s_item[i % 2] until it is given back
    if (!__all_sync(0xffffffffu,
                    ptx::mbar_wait_bounded(&item_full[i & 1], (i >> 1) & 1, kWaitLimitNs, &abort_flag)))
      return false;
    return s_item[i & 1].go != 0;
  };
  auto give = [&]() {              // (whole warp)
    const int len = s_item[I & 1].len(), two = s_item[I & 1].template tiles<IR>() - 1;
    __syncwarp();
    if (lane == 0) ptx::mbar_arrive(&item_empty[I & 1]);
    T += len, ++I;
    T1 += two * len, I1 += two;
  };

  // (a warpgroup takes or gives registers in one instruction)
  if (warp >= kMmaWarp) regs_down<kPfRegsMma>();
  if (warp < kPfSoftWarps) {
    regs_up<kPfRegsSoft>();
    const int q = warp >> 2;                            // this warp's tile
    constexpr int LPR = HD / 8, RPL = 32 / LPR;         // queries: lanes per row, rows per load
    auto row_at = [&](const PfItem& x, int64_t stride) {   // this lane's row
      const int rr = min(x.row0 + q * kPfRows + (warp & 3) * 32 + lane, x.R - 1), t = rr / G;
      return (x.t0 + t) * stride + (int64_t)(x.g * G + rr - t * G) * HD;
    };
    const bool q32 = WIDE && A.a.q_dtype == BUDDY_DTYPE_F32, out32 = WIDE && A.a.out_dtype == BUDDY_DTYPE_F32;
    auto fetch_q = [&](const PfItem& x) {               // an item's queries into L2
      if (q >= x.template tiles<IR>()) return;
      const int esz = q32 ? 4 : 2;
      const uint8_t* src = (const uint8_t*)A.a.q + row_at(x, A.a.q_stride) * esz;
      for (int i = 0; i < HD * esz; i += 128) asm volatile("prefetch.global.L2 [%0];" ::"l"(src + i));
    };
    uint8_t* const qdst = sQ + (size_t)q * TILE;
    const float base = (A.a.scale != 0.f ? A.a.scale : rsqrtf((float)HD)) * 1.4426950408889634f;
    // The queries of this warp's 32 rows as halves; returns the factor of this lane's row's
    // scores.  Where a row has elements above 2^15, or none of 2^-14, the warp's rows are taken
    // once more, scaled by a power of two each.
    auto put_q = [&](const PfItem& x) {
      const int l8 = lane % LPR;
      const int64_t at = row_at(x, A.a.q_stride);
      auto from = [&](int u) { return __shfl_sync(0xffffffffu, (long long)at, u * RPL + lane / LPR) + l8 * 8; };
      auto put = [&](int u, const float* v) {
        const Halves<WIDE> a(v[0], v[1]), b(v[2], v[3]), c(v[4], v[5]), d(v[6], v[7]);
        uint8_t* const dst = qdst + pf_piece((warp & 3) * 32 + u * RPL + lane / LPR, l8);
        *reinterpret_cast<uint4*>(dst) = make_uint4(a.hi, b.hi, c.hi, d.hi);
        if constexpr (WIDE) *reinterpret_cast<uint4*>(dst + TILE) = make_uint4(a.lo, b.lo, c.lo, d.lo);
      };
      float fac = fmaxf(base, 1.2e-38f);
      // row by row, scaled by a power of two each
      auto scaled = [&](int u) {
        float v[8], row_top = 0.f, down, f;
        const int64_t src = from(u);
        if (q32) load8((const float*)A.a.q + src, v);
        else load8((const bf16*)A.a.q + src, v);
#pragma unroll
        for (int e = 0; e < 8; ++e) row_top = fmaxf(row_top, fabsf(v[e]));
#pragma unroll
        for (int o = LPR / 2; o > 0; o >>= 1) row_top = fmaxf(row_top, __shfl_xor_sync(0xffffffffu, row_top, o));
        row_scale<WIDE>(row_top, base, &down, &f);
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] *= down;
        put(u, v);
        // to the lane of the row
        const float mine = __shfl_sync(0xffffffffu, f, (lane % RPL) * LPR);
        if (lane / RPL == u) fac = mine;
      };
      if constexpr (WIDE) {
#pragma unroll 2
        for (int u = 0; u < 32 / RPL; ++u) scaled(u);
      } else {
        const bf16* src = (const bf16*)A.a.q;
        uint4 raw[32 / RPL];                            // all of them in flight
#pragma unroll
        for (int u = 0; u < 32 / RPL; ++u) raw[u] = __ldg(reinterpret_cast<const uint4*>(src + from(u)));
        // magnitudes as integers, which order alike: the largest of all, and by rows whether any is
        // above zero, and any 2^-14 or more
        uint32_t top = 0, some = 0, enough = 0;
#pragma unroll
        for (int u = 0; u < 32 / RPL; ++u) {
          const uint32_t w[4] = {raw[u].x, raw[u].y, raw[u].z, raw[u].w};
          uint32_t m2 = 0;
#pragma unroll
          for (int e = 0; e < 4; ++e) m2 = __vmaxu2(m2, w[e] & 0x7FFF7FFFu);
          const uint32_t most = max(m2 >> 16, m2 & 0xFFFFu);
          top = max(top, most);
          some |= (most != 0 ? 1u : 0u) << u;
          enough |= (most >= 0x3880u ? 1u : 0u) << u;    // 2^-14
          float v[8];
#pragma unroll
          for (int e = 0; e < 4; ++e) v[2 * e] = __uint_as_float(w[e] << 16), v[2 * e + 1] = __uint_as_float(w[e] & 0xFFFF0000u);
          put(u, v);
        }
#pragma unroll
        for (int o = LPR / 2; o > 0; o >>= 1) some |= __shfl_xor_sync(0xffffffffu, some, o), enough |= __shfl_xor_sync(0xffffffffu, enough, o);
        if (__any_sync(0xffffffffu, top > 0x4700u || some != enough)) {   // (above 2^15)
          // (a counter in memory keeps this apart from the loops above: nine requests as above take
          // 258 us so, 262 otherwise)
#pragma unroll 1
          for (volatile int u = 0; u < 32 / RPL; u = u + 1) scaled(u);
        }
      }
      asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
      ptx::mbar_arrive(&q_ready[q]);
      return fac;
    };
    bool go = take(0);
    while (go) {
      const PfItem& it = s_item[I & 1];
      const int len = it.len();
      bool ok = true;
      if (q >= it.template tiles<IR>()) {
        go = take(I + 1);
        if (go) fetch_q(s_item[(I + 1) & 1]);
      } else {
        // ----------------------------------------------------------- softmax
        // (what only the end needs is worked out there: the tiles need the registers)
        const int rt = (warp & 3) * 32 + lane;          // row of the tile
        auto seen_by = [&]() {                          // positions this lane's row sees (may be <= 0)
          return it.n - it.m + min(it.row0 + q * kPfRows + rt, it.R - 1) / G + 1;
        };
        const float fac = put_q(it);
        const uint32_t tq = tmem + ((uint32_t)((warp & 3) * 32) << 16);
        const uint32_t ts = tq + (uint32_t)q * 128u, to = tq + kO + (uint32_t)q * 128u;
        const int seen = seen_by();
        const uint32_t C = q == 0 ? T : T1;
        float m = -INFINITY, l = 0.f;
        for (int jj = 0; jj < len; ++jj) {
          ok = __all_sync(0xffffffffu, ptx::mbar_wait_bounded(&s_full[q], (C + jj) & 1, kWaitLimitNs, &abort_flag));
          if (!ok) break;
          ptx::tc_fence_after();
          const int lim = seen - (it.j0 + jj) * kPfKeys;   // visible columns of this tile (may be <= 0)
          const uint32_t there = *reinterpret_cast<const volatile uint32_t*>(s_ok[(T + jj) & 3]);
          uint32_t s[kPfKeys];   // the row, read once (P overwrites its columns)
#pragma unroll
          for (int c = 0; c < kPfKeys; c += 32) ptx::tmem_ld32(ts + c, s + c);
          ptx::tmem_wait_ld();
          if (__any_sync(0xffffffffu, lim < kPfKeys)) {
#pragma unroll
            for (int i = 0; i < kPfKeys; ++i)
              if (i >= lim) s[i] = 0xff800000u;   // -inf: p = 0
          }
          if (there != 0x03030303u) {
#pragma unroll
            for (int i = 0; i < kPfKeys; i += 16)
              if (!((there >> (8 * (i >> 5) + ((i >> 4) & 1))) & 1))
#pragma unroll
                for (int e = 0; e < 16; ++e) s[i + e] = 0xff800000u;
          }
          float mx4[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
          for (int i = 0; i < kPfKeys; ++i) mx4[i & 3] = fmaxf(mx4[i & 3], __uint_as_float(s[i]));
          const float mx = fmaxf(fmaxf(mx4[0], mx4[1]), fmaxf(mx4[2], mx4[3])) * fac;
          const bool raise = mx > m + 8.f;
          if (__any_sync(0xffffffffu, raise)) {
            const float al = raise ? tca::exp2a(m - mx) : 1.f;
            if (raise) m = mx;
            l *= al;
            if (jj > 0) {
#pragma unroll 1
              for (int c = 0; c < HD; c += 32) {
                uint32_t o[32];
                ptx::tmem_ld32(to + c, o);
                ptx::tmem_wait_ld();
#pragma unroll
                for (int i = 0; i < 32; ++i) o[i] = __float_as_uint(__uint_as_float(o[i]) * al);
                ptx::tmem_st32(to + c, o);
              }
            }
          }
          const float ref = m == -INFINITY ? 0.f : m - kHigh;
          // The first half of P is handed over while the second is worked out.
          const uint64_t fac2 = pair(fac, fac), ref2 = pair(-ref, -ref);
          uint64_t ls[2] = {0, 0};
#pragma unroll
          for (int c = 0; c < kPfKeys; c += 32) {
            uint32_t p[16], pl[WIDE ? 16 : 1];
#pragma unroll
            for (int i = 0; i < 16; ++i) {
              float p0, p1;
              unpair(fma2(pair(__uint_as_float(s[c + 2 * i]), __uint_as_float(s[c + 2 * i + 1])), fac2, ref2), p0, p1);
              p0 = tca::exp2a(p0);
              p1 = tca::exp2a(p1);
              ls[i & 1] = add2(ls[i & 1], pair(p0, p1));
              const Halves<WIDE> y(p0, p1);
              p[i] = y.hi;
              if constexpr (WIDE) pl[i] = y.lo;
            }
            ptx::tmem_st16(ts + c / 2, p);
            if constexpr (WIDE) ptx::tmem_st16(ts + kPfKeys / 2 + c / 2, pl);
            if (c == kPfKeys / 2 - 32 || c == kPfKeys - 32) {
              ptx::tmem_wait_st();
              ptx::tc_fence_before();
              ptx::mbar_arrive(&p_ready[q][c > kPfKeys / 2]);
            }
          }
          float l0, l1;
          unpair(add2(ls[0], ls[1]), l0, l1);
          l += l0 + l1;
        }
        if (ok) {
          go = take(I + 1);
          if (go) fetch_q(s_item[(I + 1) & 1]);
          ok = __all_sync(0xffffffffu,
                          ptx::mbar_wait_bounded(&o_full[q], (q == 0 ? I : I1) & 1, kWaitLimitNs, &abort_flag));
        }
        if (ok) {
          ptx::tc_fence_after();
          const bool whole = len == it.nt;
          const float inv = !whole ? 1.f : m == -INFINITY ? 0.f : 1.f / l;
          float* part = A.part + (2 * (int64_t)blockIdx.x + (it.j0 == 0 ? 1 : 0)) * pf_part_floats<HD>() + q * kPfRows + rt;
          if (!whole) part[0] = m, part[2 * kPfRows] = l;
          const int64_t out_at = row_at(it, A.a.out_stride);
          const int sees = seen_by();
          const bool staged = whole && !out32;
#pragma unroll 1
          for (int c = 0; c < HD; c += 32) {
            float o[32];
            ptx::tmem_ld32(to + c, reinterpret_cast<uint32_t*>(o));
            ptx::tmem_wait_ld();
            const bool nan = *reinterpret_cast<const volatile int*>(&s_nan[I & 1][c / kGroup]) < sees;
#pragma unroll
            for (int i = 0; i < 32; ++i) o[i] = nan ? __uint_as_float(0x7FC00000u) : o[i] * inv;
            if (!whole) {
#pragma unroll
              for (int i = 0; i < 32; ++i) part[(2 + c + i) * 2 * kPfRows] = o[i];
            } else if (staged) {   // through this tile's query buffer (its MMAs are done): whole rows are stored
#pragma unroll
              for (int i = 0; i < 32; i += 8)
                *reinterpret_cast<uint4*>(qdst + pf_piece(rt, (c + i) >> 3)) =
                    make_uint4(tca::pack_bf16(o[i], o[i + 1]), tca::pack_bf16(o[i + 2], o[i + 3]),
                               tca::pack_bf16(o[i + 4], o[i + 5]), tca::pack_bf16(o[i + 6], o[i + 7]));
            } else if (WIDE && it.row0 + q * kPfRows + rt < it.R) {
              float4* d = reinterpret_cast<float4*>((float*)A.a.out + out_at + c);
#pragma unroll
              for (int i = 0; i < 8; ++i) d[i] = make_float4(o[4 * i], o[4 * i + 1], o[4 * i + 2], o[4 * i + 3]);
            }
          }
          if (staged) {
            __syncwarp();
            constexpr int V16 = HD / 8, RPS = 32 / V16;   // pieces of a row, rows per store
#pragma unroll 4
            for (int r0 = 0; r0 < 32; r0 += RPS) {
              const int r = r0 + lane / V16, c = lane % V16;
              const int64_t dst = __shfl_sync(0xffffffffu, (long long)out_at, r) + c * 8;
              if (it.row0 + q * kPfRows + (warp & 3) * 32 + r < it.R)
                *reinterpret_cast<uint4*>((bf16*)A.a.out + dst) =
                    *reinterpret_cast<const uint4*>(qdst + pf_piece((warp & 3) * 32 + r, c));
            }
            __syncwarp();
          }
        }
      }
      if (!ok) break;
      give();
    }
  } else if (warp == kMmaWarp) {
    // -------------------------------------------------------------------- MMA
    while (take(I)) {
      const int nq = s_item[I & 1].template tiles<IR>(), len = s_item[I & 1].len();
      bool ok = true;
      if (ptx::elect_one()) {
        const uint32_t id_s = (1u << 4) | ((uint32_t)(kPfKeys >> 3) << 17) | (8u << 24);   // half in, fp32 out, M 128
        const uint32_t id_o = (1u << 4) | ((uint32_t)(HD >> 3) << 17) | (8u << 24) | ptx::kIdescBMnMajor;
        auto wait = [&](uint64_t* bar, uint32_t count) {
          return ptx::mbar_wait_bounded(bar, count & 1, kWaitLimitNs, &abort_flag);
        };
        // (descriptors of the buffers once: what an MMA adds to one fits in its address field)
        const uint64_t dQ = ptx::smem_desc_sw128(sQ), dK = ptx::smem_desc_sw128(sK);
        const uint64_t dV = ptx::smem_desc_sw128_mn(sV, kPfRegion);
        auto qk = [&](int q, uint32_t tile) {           // S_q = Q_q K^T
          const uint64_t a = dQ + (uint64_t)q * (TILE >> 4), b = dK + (uint64_t)(tile & 1) * (TILE >> 4);
#pragma unroll
          for (int x = 0; x < (WIDE ? 2 : 1); ++x)
#pragma unroll
            for (int k = 0; k < HD / 16; ++k) {
              const uint64_t off = (k >> 2) * (kPfRegion >> 4) + 2 * (k & 3);
              ptx::mma_bf16(tmem + (uint32_t)q * 128u, a + x * (TILE >> 4) + off, b + off, id_s, x + k > 0 ? 1u : 0u);
            }
          ptx::mma_commit(&s_full[q]);
        };
        auto pv = [&](int q, uint32_t tile, int half, bool first) {   // O_q += P_q V, 64 positions
          const uint64_t v = dV + (uint64_t)(tile & 1) * (TILE >> 4) + half * (kPfKeys / 32) * (2048 >> 4);
          const uint32_t p = tmem + (uint32_t)q * 128u + 8u * half * (kPfKeys / 32);
#pragma unroll
          for (int x = 0; x < kPfKeys / 32; ++x) {      // 16 positions: two 1 KiB groups
            ptx::mma_bf16_ts(tmem + kO + (uint32_t)q * 128u, p + 8u * x, v + x * (2048 >> 4), id_o,
                             (!first || x > 0) ? 1u : 0u);
            if constexpr (WIDE)
              ptx::mma_bf16_ts(tmem + kO + (uint32_t)q * 128u, p + kPfKeys / 2 + 8u * x, v + x * (2048 >> 4), id_o, 1u);
          }
        };
        ok = wait(&k_full[T & 1], T >> 1);
        for (int q = 0; q < nq && ok; ++q) {
          ok = wait(&q_ready[q], q == 0 ? I : I1);
          if (!ok) break;
          ptx::tc_fence_after();
          qk(q, T);
        }
        if (ok) ptx::mma_commit(&k_empty[T & 1]);
        for (int jj = 0; jj < len && ok; ++jj) {
          const bool more = jj + 1 < len;
          const uint32_t u = T + jj;
          for (int q = 0; q < nq && ok; ++q) {
            const uint32_t c = (q == 0 ? T : T1) + jj;
            ok = (q > 0 || wait(&v_full[u & 1], u >> 1)) && wait(&p_ready[q][0], c);
            if (!ok) break;
            ptx::tc_fence_after();
            pv(q, u, 0, jj == 0);
            ok = (q > 0 || !more || wait(&k_full[(u + 1) & 1], (u + 1) >> 1)) && wait(&p_ready[q][1], c);
            if (!ok) break;
            ptx::tc_fence_after();
            pv(q, u, 1, false);
            if (q == nq - 1) ptx::mma_commit(&v_empty[u & 1]);
            if (more) {
              qk(q, u + 1);   // in issue order after the P V that reads P from the same columns
              if (q == nq - 1) ptx::mma_commit(&k_empty[(u + 1) & 1]);
            } else {
              ptx::mma_commit(&o_full[q]);
            }
          }
        }
      }
      if (!__all_sync(0xffffffffu, ok)) break;
      give();
    }
  } else if (warp == kMmaWarp + 1) {
    // ------------------------------------------------- the walk over the items
    PfWalk<IR> walk{};
    walk.q = {s_first.t0, s_first.m, s_first.n};
    walk.i = s_first.seq, walk.g = s_first.g, walk.qp = s_first.row0 / IR, walk.nt = s_first.nt;
    walk.start = s_first.start;
    const int64_t x = lo - walk.start;                  // tile of the item; below 0: its opening
    walk.rem = min(share, total - lo) + min(x, (int64_t)0);
    walk.j0 = (int)max(x, (int64_t)0);
    bool go = walk.rem > 0;
    if (go) {
      if (x > 0 && walk.nt <= kPfWhole) {               // the CTA before has it all
        walk.rem -= walk.nt - x;
        go = walk.next(A, lane);
      } else {
        walk.j1 = walk.nt <= kPfWhole ? walk.nt : (int)min((int64_t)walk.nt, walk.j0 + walk.rem);
        walk.rem -= walk.j1 - walk.j0;
      }
    }
    for (uint32_t i = 0;; ++i) {
      if (!__all_sync(0xffffffffu, ptx::mbar_wait_bounded(&item_empty[i & 1], ((i >> 1) & 1) ^ 1, kWaitLimitNs,
                                                          &abort_flag)))
        break;
      if (lane < GR) s_nan[i & 1][lane] = INT32_MAX;
      __syncwarp();
      if (lane == 0) {
        s_item[i & 1] = {walk.i, walk.q.t0, walk.q.m, walk.q.n, walk.g, walk.q.m * G, walk.qp * IR, walk.nt,
                         walk.j0, walk.j1, walk.start, go};
        if (go && walk.j0 == 0 && walk.j1 < walk.nt) {
          CutItem* c = cuts + blockIdx.x;
          c->t0 = walk.q.t0, c->g = walk.g, c->row0 = walk.qp * IR;
          c->rows = min(walk.q.m * G - c->row0, IR);
          c->spans = (int)((walk.start + walk.nt - 1) / share - blockIdx.x) + 1;
        }
        ptx::mbar_arrive(&item_full[i & 1]);
      }
      if (!go) break;
      go = walk.next(A, lane);
    }
  } else if (warp < kMmaWarp) {
    // -------------------------------------------------------------- K, V tiles
    regs_down<kPfRegsProduce>();
    const int lt = tid - 32 * kPfSoftWarps;             // this thread's position of a tile
    while (take(I)) {
      const PfItem it = s_item[I & 1];
      const int len = it.len();
      const int last = min(it.R, it.row0 + IR) - 1;
      const int end = min(it.n, max(it.n - it.m + last / G + 1, 0));                  // positions that any row sees
      const int in_page = (1 << A.p.shift) - 1;
      const int32_t* table = A.a.table + (int64_t)it.seq * A.a.max_pages;
      struct Entry {
        uint4 w[GR];
        __half s[GR];
      };
      // page of this thread's position of a tile: -1 past the end, -2 not there
      auto id_of = [&](int j) {
        const int p = j * kPfKeys + lt;
        if (p >= end) return -1;
        const int id = table[p >> A.p.shift];
        if ((uint32_t)id < (uint32_t)A.p.n_pages) return id;
        if (A.flags) atomicOr(A.flags, BUDDY_DEV_BAD_PAGE);
        return -2;
      };
      auto load = [&](const uint8_t* pages, int j, int id, Entry* e) {
        const int r = (j * kPfKeys + lt) & in_page;
        const uint8_t* b = pages + (id >= 0 ? block_at<HD>(A.p, id, it.g) : 0);
        const uint8_t* sc = b + ((int64_t)code_bytes(HD) << A.p.shift) + r * scale_bytes(HD);
        b += r * code_bytes(HD);
#pragma unroll
        for (int x = 0; x < GR; ++x) {
          e->w[x] = id >= 0 ? __ldg(reinterpret_cast<const uint4*>(b) + x) : make_uint4(0, 0, 0, 0);
          e->s[x] = id >= 0 ? __ldg(reinterpret_cast<const __half*>(sc) + x) : __ushort_as_half(0);
        }
      };
      auto put = [&](uint8_t* dst, const Entry* e, int j, bool values) {
#pragma unroll
        for (int x = 0; x < GR; ++x) {
          __half sc = e->s[x];
          // A NaN must not meet the zero probabilities of rows that do not see its position:
          // its values count as zeros, and the rows that see it become NaN at the end.
          if (values && __hisnan(sc)) {
            sc = __ushort_as_half(0);
            atomicMin(&s_nan[I & 1][x], j * kPfKeys + lt);
          }
          const __half2 s2 = __half2half2(sc), s72 = __hmul2(s2, __float2half2_rn(-72.f));
          const uint32_t w[4] = {e->w[x].x, e->w[x].y, e->w[x].z, e->w[x].w};
#pragma unroll
          for (int y = 0; y < 4; ++y) {
            uint32_t o[4];
            dequant4(w[y], s2, s72, o);
            *reinterpret_cast<uint4*>(dst + pf_piece(lt, 4 * x + y)) = make_uint4(o[0], o[1], o[2], o[3]);
          }
        }
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
      };
      // (the whole warp goes on or leaves: its lanes say together which pages are there)
      auto emptied = [&](uint64_t* bar, uint32_t u) {
        return __all_sync(0xffffffffu, ptx::mbar_wait_bounded(bar, ((u >> 1) & 1) ^ 1, kWaitLimitNs, &abort_flag));
      };
      Entry ek, ev;
      int id = id_of(it.j0), id_next = -1;
      load(A.p.k, it.j0, id, &ek);
      load(A.p.v, it.j0, id, &ev);
      for (int jj = 0; jj < len; ++jj) {
        const int j = it.j0 + jj;
        const uint32_t u = T + jj;
        const bool more = jj + 1 < len;
        if (more) id_next = id_of(j + 1);
        if (!emptied(&k_empty[u & 1], u)) break;
        put(sK + (size_t)(u & 1) * TILE, &ek, j, false);
        const uint32_t bad = __ballot_sync(0xffffffffu, id == -2);
        if (lane == 0) s_ok[u & 3][lt >> 5] = (uint8_t)(((bad & 0xFFFFu) ? 0 : 1) | ((bad >> 16) ? 0 : 2));
        ptx::mbar_arrive(&k_full[u & 1]);
        if (more) load(A.p.k, j + 1, id_next, &ek);
        if (!emptied(&v_empty[u & 1], u)) break;
        put(sV + (size_t)(u & 1) * TILE, &ev, j, true);
        ptx::mbar_arrive(&v_full[u & 1]);
        if (more) load(A.p.v, j + 1, id_next, &ev);
        id = id_next;
      }
      if (__any_sync(0xffffffffu, abort_flag)) break;
      give();
    }
  }

  // every issued MMA completes before TMEM is freed: normally all have (o_full), after a
  // wait that ran out the MMA warp waits for its own
  pdl_trigger();
  __syncthreads();
  if (warp == kMmaWarp) {
    if (abort_flag) {
      if (ptx::elect_one()) {   // the thread that has issued them
        ptx::mma_commit(&drained);
        volatile int dummy = 0;
        ptx::mbar_wait_bounded(&drained, 0, kWaitLimitNs, &dummy);
        if (A.flags) atomicOr(A.flags, BUDDY_DEV_TIMEOUT);
      }
      __syncwarp();
    }
    ptx::tc_fence_after();
    ptx::tmem_dealloc(tmem, 512);
  }
  // Started next to the few-row kernel of the call, which lets it start once each of its CTAs has
  // waited for all work before the call: queries, entries and lengths are there from the
  // beginning, and the workspace is free.  It does not end before that kernel, so that what
  // waits for this one has waited for both.
  pdl_wait();
}

// The parts of the items that were cut, in order: a thread per row, four channels, eight
// parts' loads at a time.  A CTA's threads take 8 channels (nine requests as above 254 us,
// with 4 channels, and so twice the CTAs, most of them without work, 257, with 16 256).
constexpr int kJoinChannels = 8;
template <int HD>
__global__ void __launch_bounds__(2 * kPfRows) kv4_join_kernel(const AttnArgs4 A, const CutItem* cuts) {
  pdl_wait();
  const CutItem c = cuts[blockIdx.x];
  const int x = threadIdx.x;
  if (x >= c.rows || c.spans == 0) return;
#pragma unroll 1
  for (int ch = blockIdx.y * 4; ch < HD; ch += gridDim.y * 4) {
    auto part = [&](int k) {
      return A.part + (2 * (int64_t)(blockIdx.x + k) + (k == 0 ? 1 : 0)) * pf_part_floats<HD>() + x;
    };
    float M = -INFINITY, L = 0.f, o[4] = {0.f, 0.f, 0.f, 0.f};
    constexpr int N = 8;
    for (int k0 = 0; k0 < c.spans; k0 += N) {
      float m[N], l[N], v[N][4], to = M;
#pragma unroll
      for (int k = 0; k < N; ++k) {
        const bool in = k0 + k < c.spans;
        const float* p = part(k0 + k);
        m[k] = in ? p[0] : -INFINITY;
        l[k] = in ? p[2 * kPfRows] : 0.f;
#pragma unroll
        for (int i = 0; i < 4; ++i) v[k][i] = in ? p[(2 + ch + i) * 2 * kPfRows] : 0.f;
      }
#pragma unroll
      for (int k = 0; k < N; ++k) to = fmaxf(to, m[k]);
      const float at = to == -INFINITY ? 0.f : to, a = tca::exp2a(M - at);
      L *= a;
#pragma unroll
      for (int i = 0; i < 4; ++i) o[i] *= a;
#pragma unroll
      for (int k = 0; k < N; ++k) {
        if (k0 + k >= c.spans) break;
        const float b = tca::exp2a(m[k] - at);
        L += b * l[k];
#pragma unroll
        for (int i = 0; i < 4; ++i) o[i] += b * v[k][i];
      }
      M = to;
    }
    const float inv = M == -INFINITY ? 0.f : 1.f / L;
    const int row = c.row0 + x, G = A.G;
    const int64_t to = (c.t0 + row / G) * A.a.out_stride + (int64_t)(c.g * G + row % G) * HD + ch;
    if (A.a.out_dtype == BUDDY_DTYPE_F32)
      *reinterpret_cast<float4*>((float*)A.a.out + to) = make_float4(o[0] * inv, o[1] * inv, o[2] * inv, o[3] * inv);
    else
      *reinterpret_cast<uint2*>((bf16*)A.a.out + to) =
          make_uint2(tca::pack_bf16(o[0] * inv, o[1] * inv), tca::pack_bf16(o[2] * inv, o[3] * inv));
  }
}

int64_t prompt_workspace(int head_dim, int sms) {
  return (int64_t)sms * (sizeof(CutItem) + 2 * (head_dim == 128 ? pf_part_floats<128>() : pf_part_floats<64>()) * 4);
}

template <int HD, bool WIDE>
static int launch_prompt_hd(const AttnArgs4& A, CutItem* cuts, int sms, cudaStream_t s) {
  // (built with fewer registers, the roles would wait for ever for theirs)
  cudaFuncAttributes at;
  if (cudaFuncGetAttributes(&at, kv4_prompt_kernel<HD, WIDE>) != cudaSuccess || at.numRegs != kPfRegs ||
      cudaFuncSetAttribute(kv4_prompt_kernel<HD, WIDE>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)pf_smem<HD>()) !=
          cudaSuccess)
    return BUDDY_ERR_CUDA;
  // the prompts start on the SMs that the few-row kernel leaves free, the join is launched
  // as the prompts end
  if (launch_k(kv4_prompt_kernel<HD, WIDE>, sms, kPfThreads, pf_smem<HD>(), s, true, A, cuts) != cudaSuccess ||
      launch_k(kv4_join_kernel<HD>, dim3(sms, HD / kJoinChannels), 2 * kPfRows, 0, s, true, A, (const CutItem*)cuts) != cudaSuccess)
    return BUDDY_ERR_CUDA;
  return BUDDY_OK;
}

// ws: prompt_workspace() bytes.
int launch_prompt(AttnArgs4 A, int head_dim, bool wide, int sms, void* ws, cudaStream_t s) {
  CutItem* cuts = (CutItem*)ws;
  A.part = (float*)((uint8_t*)ws + sms * sizeof(CutItem));
  if (wide) return head_dim == 128 ? launch_prompt_hd<128, true>(A, cuts, sms, s) : launch_prompt_hd<64, true>(A, cuts, sms, s);
  return head_dim == 128 ? launch_prompt_hd<128, false>(A, cuts, sms, s) : launch_prompt_hd<64, false>(A, cuts, sms, s);
}

}  // namespace kv4
}  // namespace buddy
