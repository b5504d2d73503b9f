// What the kernels with few query rows per KV head share: a warp's stage of a chunk, and the walk
// of a stream's rows over it (kv4_attn.cu says how the products are laid out).
#pragma once

#include "kv4_attn.cuh"

namespace buddy {
namespace kv4 {

constexpr int kChunk = 32;
// The workspace of these kernels: arrival counters, then partials.
constexpr int kMaxGrid = 1024;          // CTAs that have two partials of sixteen rows each: four on each of at most 256 SMs
constexpr int64_t kWsCounters = 8192;   // bytes of counters
constexpr int64_t few_bytes(int head_dim) { return kWsCounters + (int64_t)kMaxGrid * 2 * 16 * (head_dim + 2) * 4; }
template <int HD>
__host__ __device__ constexpr int stage_bytes() { return 2 * kChunk * entry_bytes(HD); }
// Chunks of a stream of n positions.  (A sequence without positions: one of nothing.)
__device__ __forceinline__ int chunks_of(int n) { return max(1, (n + kChunk - 1) / kChunk); }

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

// Where a lane's codes and scales are in a stage: keys of row lg, values of rows 2 lc and 2 lc + 1.
template <int HD>
struct Places {
  static constexpr int VC = kChunk * code_bytes(HD), KSC = 2 * VC, VSC = KSC + kChunk * scale_bytes(HD);
  int k_at, ks_at, v_at[2], vs_at[2];
  __device__ __forceinline__ explicit Places(int lane) {
    const int lg = lane >> 2, lc = lane & 3;
    k_at = place(lg) * code_bytes(HD) + lc * (HD / 8);
    ks_at = KSC + place(lg) * scale_bytes(HD) + (lc * (HD / 4) / 32) * 2;
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      v_at[u] = VC + place(2 * lc + u) * code_bytes(HD) + lg * (HD / 16);
      vs_at[u] = VSC + place(2 * lc + u) * scale_bytes(HD) + (lg * (HD / 8) / 32) * 2;
    }
  }
};

// The chunk of positions from p0 on in stage st, of a sequence of n, for a warp's rows of a stream
// (up to 8 NB): their queries as halves (ql: what the halves leave of them), factors of the scores of
// rows 2 lc and 2 lc + 1 and the positions that these see, outputs, running maxima and sums.
// all_seen: positions that every row sees; lost: 16 positions without a page.
template <int HD, int NB, bool WIDE>
__device__ __forceinline__ void take_chunk(const uint8_t* st, const Places<HD>& P, int p0, int n, int all_seen,
                                           uint32_t lost, int lg, int lc,
                                           const uint32_t (&qf)[NB][HD / 16][2],
                                           const uint32_t (&ql)[WIDE ? NB : 1][HD / 16][2],
                                           const float (&fac)[NB][2],
                                           const int (&seen)[NB][2],
                                           float (&o)[NB][HD / 16][4],
                                           float (&m)[NB][2],
                                           float (&l)[NB][2]) {
  constexpr int KS = HD / 16;
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
        const uint8_t* src = st + P.k_at + (16 * t + 8 * u) * code_bytes(HD);
        if constexpr (HD == 128) {
          const uint4 v = *reinterpret_cast<const uint4*>(src);
          w[t][u][0] = v.x, w[t][u][1] = v.y, w[t][u][HD / 32 - 2] = v.z, w[t][u][HD / 32 - 1] = v.w;
        } else {
          const uint2 v = *reinterpret_cast<const uint2*>(src);
          w[t][u][0] = v.x, w[t][u][1] = v.y;
        }
        sc[t][u] = __half2half2(*reinterpret_cast<const __half*>(st + P.ks_at + (16 * t + 8 * u) * scale_bytes(HD)));
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
      vsc[t][u] = __halves2half2(*reinterpret_cast<const __half*>(st + P.vs_at[0] + (16 * t + 8 * u) * scale_bytes(HD)),
                                 *reinterpret_cast<const __half*>(st + P.vs_at[1] + (16 * t + 8 * u) * scale_bytes(HD)));
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
          reinterpret_cast<const uint32_t*>(st + P.v_at[u & 1] + (16 * t + 8 * (u >> 1)) * code_bytes(HD));
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
}

}  // namespace kv4
}  // namespace buddy
