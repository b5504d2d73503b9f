// Rows of queries, keys and values between a block's QKV projection and its
// attention: norm of each head and rotation (buddy_qk_norm_rope), the same with the
// entries quantised into the paged 4-bit cache (buddy_kv4_append), both with one position
// or with several axes of them (.._axes), and entries read back (buddy_kv4_read).
//
// A team of HD / 16 lanes holds a head: a lane has eight neighbours of the lower half and
// the eight of the upper half that the rotation pairs them with, each in one 16-byte load
// (bf16).  A scale's 32 channels are four lanes, a lane's eight codes are one word.  A
// team takes consecutive heads of a token, one loaded while the one before is worked on, so
// that the token's position, slot and rotation factors are read once for them.
//
// The sum of squares: within the eights halves onto each other, then halves of the
// eights; products and sums rounded one by one (no fused multiply-adds), so that a plain
// program can follow it bit by bit, which the codes need: where a value lies between two
// codes, one bit decides.
//
// Bound by HBM from thousands of tokens on (8,297 of 40 heads, 174 MB: 29.8 us a call, 5.9
// TB/s, with instructions issued in 63% of the cycles; in fp32, 348 MB, 53.9 us, 6.4 TB/s); below by the latency of position,
// rotation factors and rows, one after the other: one token 2.5 us, an append of 64 and
// their read 4.8.  With three axes in runs of frequencies 7,901 tokens take 31.0 us, in turn 34.0.
#include <cuda_runtime.h>

#include <algorithm>
#include <type_traits>

#include "common.cuh"
#include "internal.h"
#include "kv4.cuh"
#include "ptx.cuh"

namespace buddy {

constexpr int kRowThreads = 128;

struct RowArgs {
  buddy_qk_rows r;
  const void* v;
  int64_t v_stride;
  kv4::Pages pages;
  const int64_t* slot;
  int32_t* flags;
  int per, groups;             // heads of a team, teams of a token
};

// Which position turns a frequency: two bits each, the first of a word lowest.
struct Axes {
  uint32_t of[4];
  int n;
  int64_t stride;              // from axis to axis of the positions
};
struct OneAxis {};

// bf16: heads of a team on their way at once (copied to shared memory, which takes no registers: a lane
// reads what it has copied itself).  Of fp32 a lane's eight channels are two pieces of 16 bytes, which its
// neighbours' lie between: their sectors would be fetched twice (8,297 tokens 79 us, with loads of
// the head after this one 54).
constexpr int kRowAhead = 3;
constexpr int kRowHead = kRowThreads * 32, kRowRing = kRowAhead * kRowHead;   // bytes of a CTA
__device__ __forceinline__ void copy16(uint32_t dst, const void* src) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
}

__device__ __forceinline__ void store8(float* p, const float* x) {
  reinterpret_cast<float4*>(p)[0] = make_float4(x[0], x[1], x[2], x[3]);
  reinterpret_cast<float4*>(p)[1] = make_float4(x[4], x[5], x[6], x[7]);
}
__device__ __forceinline__ void store8(bf16* p, const float* x) {
  __nv_bfloat162 h[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) h[i] = __floats2bfloat162_rn(x[2 * i], x[2 * i + 1]);
  *reinterpret_cast<uint4*>(p) = *reinterpret_cast<const uint4*>(h);
}
__device__ __forceinline__ void store8(__half* p, const float* x) {
  __half2 h[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) h[i] = __floats2half2_rn(x[2 * i], x[2 * i + 1]);
  *reinterpret_cast<uint4*>(p) = *reinterpret_cast<const uint4*>(h);
}

// Two fp32 at once, each rounded as alone.
struct F2 {
  uint64_t v;
  __device__ __forceinline__ F2() {}
  __device__ __forceinline__ F2(float a, float b) { asm("mov.b64 %0, {%1, %2};" : "=l"(v) : "f"(a), "f"(b)); }
  __device__ __forceinline__ void get(float& a, float& b) const { asm("mov.b64 {%0, %1}, %2;" : "=f"(a), "=f"(b) : "l"(v)); }
};
__device__ __forceinline__ F2 operator*(F2 a, F2 b) {
  F2 r;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r.v) : "l"(a.v), "l"(b.v));
  return r;
}
__device__ __forceinline__ F2 operator+(F2 a, F2 b) {
  F2 r;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r.v) : "l"(a.v), "l"(b.v));
  return r;
}
// Products that a sum takes, one by one: the assembler makes fused multiply-adds of a packed
// product and a packed sum, rounding modifiers or not.
__device__ __forceinline__ F2 products(F2 a, F2 b) {
  float a0, a1, b0, b1;
  a.get(a0, a1);
  b.get(b0, b1);
  return F2(__fmul_rn(a0, b0), __fmul_rn(a1, b1));
}
__device__ __forceinline__ F2 fma2(F2 a, F2 b, F2 c) {
  F2 r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r.v) : "l"(a.v), "l"(b.v), "l"(c.v));
  return r;
}
__device__ __forceinline__ F2 neg(F2 a) {
  F2 r;
  r.v = a.v ^ 0x8000000080000000ull;
  return r;
}
__device__ __forceinline__ float max_nan(float a, float b) {   // NaN if one is
  float r;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
  return r;
}

// Eight consecutive elements of a row as they lie in memory.  (Ordinary loads: in place, the
// kernel writes what it has read, which the path of read-only data does not allow.)
template <typename T> struct Raw8;
template <> struct Raw8<bf16> {
  uint4 a;
  __device__ __forceinline__ void load(const bf16* p) { a = *reinterpret_cast<const uint4*>(p); }
  __device__ __forceinline__ void get(F2* o) const {
    const uint32_t w[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) o[i] = F2(__uint_as_float(w[i] << 16), __uint_as_float(w[i] & 0xFFFF0000u));
  }
};
template <> struct Raw8<float> {
  float4 a, b;
  __device__ __forceinline__ void load(const float* p) {
    a = reinterpret_cast<const float4*>(p)[0];
    b = reinterpret_cast<const float4*>(p)[1];
  }
  __device__ __forceinline__ void get(F2* o) const {
    o[0] = F2(a.x, a.y), o[1] = F2(a.z, a.w), o[2] = F2(b.x, b.y), o[3] = F2(b.z, b.w);
  }
};
// Eight values that no kernel of the call writes (gains, rotation factors).
__device__ __forceinline__ void load8(const float* p, F2* o) {
  const float4 a = __ldg(reinterpret_cast<const float4*>(p)), b = __ldg(reinterpret_cast<const float4*>(p) + 1);
  o[0] = F2(a.x, a.y), o[1] = F2(a.z, a.w), o[2] = F2(b.x, b.y), o[3] = F2(b.z, b.w);
}
template <typename T>
__device__ __forceinline__ void store8(T* p, const F2* x) {
  float y[8];
#pragma unroll
  for (int i = 0; i < 4; ++i) x[i].get(y[2 * i], y[2 * i + 1]);
  store8(p, y);
}

// Sum of the squares of eight values, halves onto each other.
__device__ __forceinline__ float squares8(const F2* x) {
  const F2 a = products(x[0], x[0]) + products(x[2], x[2]), b = products(x[1], x[1]) + products(x[3], x[3]), c = a + b;
  float u, v;
  c.get(u, v);
  return __fadd_rn(u, v);
}

// Eight channels of a group of 32 (four lanes, all of `mask`) into code word and scale.
// The quotients are the correctly rounded ones: with y = 1 / s correctly rounded, q = x y
// and r = x - q s, q + r y rounds to x / s (P. Markstein, IBM J. Res. Dev. 34 (1990), theorem
// on the last step of a division by multiplications).  Adding 1.5 * 2^23 + 8 rounds one to an integer (ties
// to even) and leaves its code in the low bits.
__device__ __forceinline__ uint32_t encode8(const F2* x, uint32_t mask, __half* scale) {
  float v[8], m = 0.f;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    x[i].get(v[2 * i], v[2 * i + 1]);
    m = max_nan(m, max_nan(fabsf(v[2 * i]), fabsf(v[2 * i + 1])));
  }
  m = max_nan(m, __shfl_xor_sync(mask, m, 1));
  m = max_nan(m, __shfl_xor_sync(mask, m, 2));
  *scale = kv4::scale_of(__float_as_uint(m));
  const float s = __half2float(*scale);
  if (!(s > 0.f)) return 0x88888888u;
  const float y = __frcp_rn(s);
  // a scale at its limit, or rounded among the smallest halves: larger quotients than 7 are there
  const bool clamp = s >= kv4::kMaxScale || s < 7.62939453125e-6f;
  const F2 s2(-s, -s), y2(y, y), magic(12582920.f, 12582920.f);
  uint32_t w = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    F2 z = x[i];
    if (clamp) {
      const float top = 7.f * s;
      z = F2(fminf(fmaxf(v[2 * i], -top), top), fminf(fmaxf(v[2 * i + 1], -top), top));
    }
    const F2 q = z * y2, n = fma2(fma2(q, s2, z), y2, q) + magic;
    float lo, hi;
    n.get(lo, hi);
    w |= (__byte_perm(__float_as_uint(lo), __float_as_uint(hi), 0x5410) & 0x000F000Fu) << (4 * i);
  }
  return w;
}

// AX: OneAxis, or Axes.  With several axes a lane's eight frequencies mostly have the same (runs
// of a multiple of eight frequencies per axis): rows of the tables in wide loads, as with one
// axis. Where they have not, each value is loaded by itself.  (In wide loads of every axis, and a
// choice between them, 64 tokens whose frequencies go round three axes took 3.8 us instead of 3.4.)
enum class Team {
  One,        // one head, which the team loads itself (with the copies' code 64 tokens appended and read took 5.0 us instead of 4.8)
  Next,       // several, the next one in registers while one is worked on
  Ring        // several, kRowAhead of them in shared memory
};
template <typename T, int HD, bool CACHE, typename AX, Team TEAM>
__global__ void __launch_bounds__(kRowThreads) qk_rows_kernel(const RowArgs A, const AX ax) {
  constexpr bool AXES = std::is_same<AX, Axes>::value, ONE = TEAM == Team::One, RING = TEAM == Team::Ring;
  constexpr int LPH = HD / 16, HALF = HD / 2;
  const buddy_qk_rows& R = A.r;
  const int kq = R.n_q_heads, kk = kq + R.n_kv_heads, heads = kk + (CACHE ? R.n_kv_heads : 0);
  const int tl = threadIdx.x % LPH;
  const uint32_t team = ((1u << LPH) - 1) << (threadIdx.x % 32 / LPH * LPH);   // this team's lanes
  pdl_wait();
  pdl_trigger();
  // (the teams of a warp take the same heads of neighbouring tokens: queries, keys and
  // values go different ways)
  const int grp = (int)(blockIdx.x % (unsigned)A.groups);
  const int64_t t = (int64_t)(blockIdx.x / (unsigned)A.groups) * (kRowThreads / LPH) + threadIdx.x / LPH;
  if (t >= R.n_tok) return;                     // (whole teams)
  const int h0 = ONE ? grp : grp * A.per, h1 = ONE ? h0 + 1 : min(h0 + A.per, heads);

  const int c = tl * 8;                         // this lane's channels: c .. c + 7 of both halves
  auto row = [&](int h) -> const T* {
    if (h < kq) return (const T*)R.q + t * R.q_stride + (int64_t)h * HD + c;
    if (!CACHE || h < kk) return (const T*)R.k + t * R.k_stride + (int64_t)(h - kq) * HD + c;
    return (const T*)A.v + t * A.v_stride + (int64_t)(h - kk) * HD + c;
  };
  Raw8<T> lo, hi;
  // a lane's pieces of 16 bytes of a head's halves, those of the other threads between them
  extern __shared__ __align__(16) uint8_t rows_smem[];
  const uint32_t ring = ptx::smem_u32(rows_smem) + threadIdx.x * 16;
  uint32_t held = 0;                            // where in the ring the head at hand is
  auto ahead = [&](int h, uint32_t at) {
    if (h < h1) {
      const T* src = row(h);
      const uint32_t to = ring + at;
      copy16(to, src);
      copy16(to + kRowThreads * 16, src + HALF);
    }
    asm volatile("cp.async.commit_group;" ::: "memory");
  };
  static_assert(!RING || sizeof(T) == 2, "");
  if constexpr (!RING) {
    lo.load(row(h0));
    hi.load(row(h0) + HALF);
  } else {
    for (int j = 0; j < kRowAhead - 1; ++j) ahead(h0 + j, j * kRowHead);
  }
  int p = R.pos[t], most = p, least = p;        // (of all axes)
  int q[4] = {p, p, p, p};                      // positions on the axes
  auto place_of = [&](uint32_t a) { return a & 2 ? (a & 1 ? q[3] : q[2]) : (a & 1 ? q[1] : q[0]); };
  uint32_t mix = 0, axis = 0;                   // two bits of each of the lane's frequencies, the first one's axis
  if constexpr (AXES) {
#pragma unroll
    for (int a = 1; a < 4; ++a)
      if (a < ax.n) q[a] = R.pos[a * ax.stride + t];
    mix = (ax.of[tl / 2] >> (tl % 2 * 16)) & 0xFFFFu;
    axis = mix & 3u;
    most = max(max(q[0], q[1]), max(q[2], q[3]));
    least = min(min(q[0], q[1]), min(q[2], q[3]));
    p = place_of(axis);
  }
  int64_t slot = -1;
  if (CACHE) slot = A.slot[t];
  const bool ok = least >= 0 && most < R.max_pos;
  const int64_t end = (int64_t)A.pages.n_pages << A.pages.shift;
  if (tl == 0 && h0 == 0 && A.flags) {
    const int bad = (most >= R.max_pos ? BUDDY_DEV_BAD_POSITION : 0) | (CACHE && ok && slot >= end ? BUDDY_DEV_BAD_PAGE : 0);
    if (bad) atomicOr(A.flags, bad);
  }
  if (!ok) {
    if constexpr (RING) asm volatile("cp.async.wait_all;" ::: "memory");
    return;
  }
  const bool keep = CACHE && slot >= 0 && slot < end;
  F2 co[4], si[4];
  if (h0 < kk) {
    if (!AXES || mix == axis * 0x5555u) {
      load8(R.rope_cos + (int64_t)p * HALF + c, co);
      load8(R.rope_sin + (int64_t)p * HALF + c, si);
    } else {                                    // value by value, all on their way at once
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int64_t u = (int64_t)place_of(mix >> (4 * e)) * HALF + c + 2 * e;
        const int64_t v = (int64_t)place_of(mix >> (4 * e + 2)) * HALF + c + 2 * e + 1;
        co[e] = F2(__ldg(R.rope_cos + u), __ldg(R.rope_cos + v));
        si[e] = F2(__ldg(R.rope_sin + u), __ldg(R.rope_sin + v));
      }
    }
  }
#pragma unroll 1
  for (int h = h0; h < h1; ++h) {
    F2 a[4], b[4];                              // lower and upper half
    if constexpr (RING) {
      ahead(h + kRowAhead - 1, held == 0 ? kRowRing - kRowHead : held - kRowHead);   // to where the head before this one was
      asm volatile("cp.async.wait_group %0;" ::"n"(kRowAhead - 1) : "memory");
      const uint8_t* const at = rows_smem + held + threadIdx.x * 16;
      held = held == kRowRing - kRowHead ? 0 : held + kRowHead;
      lo.load(reinterpret_cast<const T*>(at));
      hi.load(reinterpret_cast<const T*>(at + kRowThreads * 16));
    }
    lo.get(a);
    hi.get(b);
    if (!RING && h + 1 < h1) {
      lo.load(row(h + 1));
      hi.load(row(h + 1) + HALF);
    }
    if (!CACHE || h < kk) {
      const float* gains = h < kq ? R.q_gain : R.k_gain;
      if (gains) {
        float sum = __fadd_rn(squares8(a), squares8(b));
#pragma unroll
        for (int o = LPH / 2; o > 0; o >>= 1) sum = __fadd_rn(sum, __shfl_xor_sync(team, sum, o));
        const float r = __fdiv_rn(1.f, __fsqrt_rn(__fadd_rn(__fmul_rn(sum, 1.f / HD), R.eps)));
        const F2 r2(r, r);
        F2 ga[4], gb[4];
        load8(gains + c, ga);
        load8(gains + HALF + c, gb);
#pragma unroll
        for (int i = 0; i < 4; ++i) a[i] = a[i] * r2 * ga[i], b[i] = b[i] * r2 * gb[i];
      }
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const F2 ac = products(a[i], co[i]), bs = products(b[i], si[i]);
        b[i] = products(b[i], co[i]) + products(a[i], si[i]);
        a[i] = ac + neg(bs);
      }
      if (h < kq) {
        T* d = (T*)R.q_out + t * R.q_out_stride + (int64_t)h * HD + c;
        store8(d, a);
        store8(d + HALF, b);
        continue;
      }
      if (R.k_out) {
        T* d = (T*)R.k_out + t * R.k_out_stride + (int64_t)(h - kq) * HD + c;
        store8(d, a);
        store8(d + HALF, b);
      }
    }
    if (CACHE && keep) {
      __half sa, sb;
      const uint32_t wa = encode8(a, team, &sa), wb = encode8(b, team, &sb);
      const int in_page = (int)(slot & ((1 << A.pages.shift) - 1));
      uint8_t* blk = (h < kk ? A.pages.k : A.pages.v) + kv4::block_at<HD>(A.pages, slot >> A.pages.shift, h < kk ? h - kq : h - kk);
      uint32_t* codes = reinterpret_cast<uint32_t*>(blk + in_page * kv4::code_bytes(HD)) + tl;
      codes[0] = wa;
      codes[HD / 16] = wb;
      if (tl % 4 == 0) {
        __half* sc = reinterpret_cast<__half*>(blk + ((int64_t)kv4::code_bytes(HD) << A.pages.shift) +
                                               in_page * kv4::scale_bytes(HD)) + tl / 4;
        sc[0] = sa;
        sc[HD / 64] = sb;
      }
    }
  }
}

template <typename T, int HD>
__global__ void __launch_bounds__(kRowThreads) kv4_read_kernel(const kv4::Pages P, int n, const int64_t* slots, T* k_out,
                                                               T* v_out, int32_t* flags) {
  constexpr int LPH = HD / 8;
  const int64_t u = ((int64_t)blockIdx.x * kRowThreads + threadIdx.x) / LPH;   // (entry, head)
  const int tl = threadIdx.x % LPH;
  pdl_wait();
  pdl_trigger();
  if (u >= (int64_t)n * P.nkv) return;
  const int64_t j = u / P.nkv;
  const int g = (int)(u - j * P.nkv);
  const int64_t slot = slots[j];
  if (slot < 0) return;
  if (slot >= (int64_t)P.n_pages << P.shift) {
    if (flags && g == 0 && tl == 0) atomicOr(flags, BUDDY_DEV_BAD_PAGE);
    return;
  }
  const int64_t block = kv4::block_at<HD>(P, slot >> P.shift, g);
  const int row = (int)(slot & ((1 << P.shift) - 1));
  const int64_t code_at = block + row * kv4::code_bytes(HD) + 4 * tl;
  const int64_t scale_at = block + ((int64_t)kv4::code_bytes(HD) << P.shift) + row * kv4::scale_bytes(HD) + (tl >> 2) * 2;
  uint32_t w[2] = {0, 0};
  float s[2] = {0.f, 0.f};
#pragma unroll
  for (int i = 0; i < 2; ++i) {   // both before the first is stored
    if (!(i ? v_out : k_out)) continue;
    const uint8_t* b = i ? P.v : P.k;
    w[i] = *reinterpret_cast<const uint32_t*>(b + code_at);
    s[i] = __half2float(*reinterpret_cast<const __half*>(b + scale_at));
  }
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    T* out = i ? v_out : k_out;
    if (!out) continue;
    float y[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) y[e] = kv4::decode(w[i], e, s[i]);
    store8(out + u * HD + tl * 8, y);
  }
}

static bool aligned_rows(const void* p, int64_t stride, int esz) {
  return p && aligned16(p) && stride * esz % 16 == 0;
}

static bool rows_ok(const buddy_qk_rows* r, bool k_out_needed) {
  if (!r || r->n_tok < 0 || r->n_q_heads < 0 || r->n_kv_heads < 1 || r->n_q_heads > 65536 || r->n_kv_heads > 65536 ||
      (r->head_dim != 64 && r->head_dim != 128) || (r->dtype != BUDDY_DTYPE_F32 && r->dtype != BUDDY_DTYPE_BF16) ||
      r->max_pos < 1 || !(r->eps > 0.f) || !r->rope_cos || !r->rope_sin || !aligned16(r->rope_cos) ||
      !aligned16(r->rope_sin))
    return false;
  if ((r->q_gain && !aligned16(r->q_gain)) || (r->k_gain && !aligned16(r->k_gain))) return false;
  if (r->n_tok == 0) return true;
  const int e = r->dtype == BUDDY_DTYPE_F32 ? 4 : 2;
  if (!r->pos || !aligned_rows(r->k, r->k_stride, e)) return false;
  if (r->n_q_heads > 0 && (!aligned_rows(r->q, r->q_stride, e) || !aligned_rows(r->q_out, r->q_out_stride, e)))
    return false;
  return (!k_out_needed && !r->k_out) || aligned_rows(r->k_out, r->k_out_stride, e);
}

bool kv4_cache_ok(const buddy_kv4_cache* c) {
  return c && c->n_pages >= 1 && (c->page_size == 16 || c->page_size == 32 || c->page_size == 64 || c->page_size == 128) &&
         c->n_kv_heads >= 1 && c->n_kv_heads <= 1024 && (c->head_dim == 64 || c->head_dim == 128) && c->k_pages &&
         c->v_pages && aligned16(c->k_pages) && aligned16(c->v_pages);
}

kv4::Pages kv4_pages(const buddy_kv4_cache* c) {
  int shift = 4;
  while ((1 << shift) < c->page_size) ++shift;
  return {(uint8_t*)c->k_pages, (uint8_t*)c->v_pages, c->n_pages, shift, c->n_kv_heads};
}

// Heads of a team: one while there are few rows, for the shortest chain; more as they fill
// the GPU (kRowTeams), up to eight, which share the reads of position and rotation
// (8,297 tokens of 40 heads 29.8 us, a fifth more with four; append of 4,999 tokens of
// 36 heads and their read 22.4, 12% more with four).
// Where the axes change within a lane's frequencies the reads are many and narrow, and shared from fewer rows
// on: 250 tokens of 40 heads 4.6 us instead of 5.3, 1,000 8.5 instead of 9.4 (an append does more with what it
// has read: 250 tokens of fp32 7.4 instead of 6.9, so it does not).
constexpr int64_t kRowTeams = 16384;
// Heads of a call from which on bf16 appends with one axis take the ring. Below, with rows that a projection has left
// in L2, its turns cost more than the registers that it saves (32 + 16 heads, in registers and by the ring: 3,000 tokens
// with norms 19.9 and 21.5 us, 8,297 44.0 and 42.8; without norms 2,200 12.5 and 13.8, 6,000 31.2 and 28.5). Rows from HBM
// gain by the ring earlier: 3,000 tokens without norms 20.4 and 19.9, with norms 23.0 and 23.6. With several axes it is the
// ring throughout (3,000 tokens with norms, three axes in runs: 20.7 and 22.1 us, from HBM 25.8 and 24.6).
constexpr int64_t kRingNorms = 17 * kRowTeams, kRingPlain = 9 * kRowTeams;
// Whether a lane's eight frequencies have different axes somewhere.
static bool mixed(const OneAxis&) { return false; }
static bool mixed(const Axes& a) {
  for (int j = 0; j < 8; ++j) {
    const uint32_t w = a.of[j / 2] >> (j % 2 * 16) & 0xFFFFu;
    if (w != (w & 3u) * 0x5555u) return true;
  }
  return false;
}
template <typename T, int HD, bool CACHE, typename AX>
static int launch_rows(RowArgs A, const AX& ax, cudaStream_t s) {
  const int heads = A.r.n_q_heads + A.r.n_kv_heads * (CACHE ? 2 : 1);
  A.per = (int)std::min<int64_t>(8, std::max<int64_t>(1, (int64_t)A.r.n_tok * heads / (!CACHE && mixed(ax) ? kRowTeams / 4 : kRowTeams)));
  A.groups = (heads + A.per - 1) / A.per;
  const int64_t ctas = ((int64_t)A.r.n_tok * (HD / 16) + kRowThreads - 1) / kRowThreads * A.groups;
  if (ctas > INT32_MAX) return BUDDY_ERR_RANGE;
  auto launch = [&](auto* kern, int smem) {
    return launch_k(kern, (unsigned)ctas, kRowThreads, smem, s, true, A, ax) == cudaSuccess ? BUDDY_OK : BUDDY_ERR_CUDA;
  };
  if (A.per == 1) return launch(qk_rows_kernel<T, HD, CACHE, AX, Team::One>, 0);
  if constexpr (sizeof(T) == 4) {
    return launch(qk_rows_kernel<T, HD, CACHE, AX, Team::Next>, 0);
  } else {
    if constexpr (CACHE && std::is_same<AX, OneAxis>::value) {
      if ((int64_t)A.r.n_tok * heads < (A.r.q_gain || A.r.k_gain ? kRingNorms : kRingPlain))
        return launch(qk_rows_kernel<T, HD, CACHE, AX, Team::Next>, 0);
    }
    return launch(qk_rows_kernel<T, HD, CACHE, AX, Team::Ring>, kRowRing);
  }
}
template <bool CACHE, typename AX>
static int dispatch_rows(const RowArgs& A, const AX& ax, cudaStream_t s) {
  if (A.r.n_tok == 0) return BUDDY_OK;
  if (A.r.dtype == BUDDY_DTYPE_F32)
    return A.r.head_dim == 128 ? launch_rows<float, 128, CACHE>(A, ax, s) : launch_rows<float, 64, CACHE>(A, ax, s);
  return A.r.head_dim == 128 ? launch_rows<bf16, 128, CACHE>(A, ax, s) : launch_rows<bf16, 64, CACHE>(A, ax, s);
}

// The axes of a call's frequencies; false where they are not those of head_dim / 2 frequencies.
static bool axes_ok(const buddy_rope_axes* a, int head_dim, Axes* out) {
  if (!a || a->n_axes < 1 || a->n_axes > 4 || a->pos_stride < 0) return false;
  *out = Axes{{0, 0, 0, 0}, a->n_axes, a->pos_stride};
  for (int j = 0; j < head_dim / 2; ++j) {
    if (a->axis[j] >= a->n_axes) return false;
    out->of[j / 16] |= (uint32_t)a->axis[j] << (j % 16 * 2);
  }
  return true;
}

template <typename T>
static int launch_read(const buddy_kv4_cache* c, int n, const int64_t* slot, void* k, void* v, int32_t* flags,
                       cudaStream_t s) {
  const int64_t ctas = ((int64_t)n * c->n_kv_heads * (c->head_dim / 8) + kRowThreads - 1) / kRowThreads;
  if (ctas > INT32_MAX) return BUDDY_ERR_RANGE;
  auto* const kern = c->head_dim == 128 ? kv4_read_kernel<T, 128> : kv4_read_kernel<T, 64>;
  return launch_k(kern, (unsigned)ctas, kRowThreads, 0, s, true, kv4_pages(c), n, slot, (T*)k, (T*)v, flags) == cudaSuccess
             ? BUDDY_OK : BUDDY_ERR_CUDA;
}

}  // namespace buddy

using namespace buddy;

extern "C" int buddy_rope_table(float* rope_cos, float* rope_sin, int32_t max_pos, int32_t head_dim, float rope_theta,
                                void* stream) {
  if (!rope_cos || !rope_sin || max_pos < 1 || (head_dim != 64 && head_dim != 128) || !(rope_theta > 0.f))
    return BUDDY_ERR_ARG;
  launch_rope_table(rope_cos, rope_sin, max_pos, head_dim, (double)rope_theta, (cudaStream_t)stream);
  return cudaGetLastError() == cudaSuccess ? BUDDY_OK : BUDDY_ERR_CUDA;
}

extern "C" int buddy_qk_norm_rope(const buddy_qk_rows* rows, int32_t* flags, void* stream) {
  if (!rows_ok(rows, true)) return BUDDY_ERR_ARG;
  RowArgs A{};
  A.r = *rows;
  A.flags = flags;
  return dispatch_rows<false>(A, OneAxis{}, (cudaStream_t)stream);
}

extern "C" int buddy_qk_norm_rope_axes(const buddy_qk_rows* rows, const buddy_rope_axes* axes, int32_t* flags,
                                       void* stream) {
  Axes ax;
  if (!rows_ok(rows, true) || !axes_ok(axes, rows->head_dim, &ax)) return BUDDY_ERR_ARG;
  RowArgs A{};
  A.r = *rows;
  A.flags = flags;
  return dispatch_rows<false>(A, ax, (cudaStream_t)stream);
}

static bool append_ok(const buddy_kv4_cache* cache, const buddy_qk_rows* rows, const void* v, int64_t v_stride,
                      const int64_t* slot) {
  if (!kv4_cache_ok(cache) || !rows_ok(rows, false) || rows->n_kv_heads != cache->n_kv_heads ||
      rows->head_dim != cache->head_dim)
    return false;
  return rows->n_tok == 0 || (slot && aligned_rows(v, v_stride, rows->dtype == BUDDY_DTYPE_F32 ? 4 : 2));
}

extern "C" int buddy_kv4_append(const buddy_kv4_cache* cache, const buddy_qk_rows* rows, const void* v,
                                int64_t v_stride, const int64_t* slot, int32_t* flags, void* stream) {
  if (!append_ok(cache, rows, v, v_stride, slot)) return BUDDY_ERR_ARG;
  const RowArgs A{*rows, v, v_stride, kv4_pages(cache), slot, flags, 0, 0};
  return dispatch_rows<true>(A, OneAxis{}, (cudaStream_t)stream);
}

extern "C" int buddy_kv4_append_axes(const buddy_kv4_cache* cache, const buddy_qk_rows* rows, const buddy_rope_axes* axes,
                                     const void* v, int64_t v_stride, const int64_t* slot, int32_t* flags, void* stream) {
  Axes ax;
  if (!append_ok(cache, rows, v, v_stride, slot) || !axes_ok(axes, rows->head_dim, &ax)) return BUDDY_ERR_ARG;
  const RowArgs A{*rows, v, v_stride, kv4_pages(cache), slot, flags, 0, 0};
  return dispatch_rows<true>(A, ax, (cudaStream_t)stream);
}

extern "C" int buddy_kv4_read(const buddy_kv4_cache* cache, int32_t n, const int64_t* slot, int32_t dtype, void* k_out,
                              void* v_out, int32_t* flags, void* stream) {
  if (!kv4_cache_ok(cache) || n < 0 || (n > 0 && !slot) || (k_out && !aligned16(k_out)) || (v_out && !aligned16(v_out)))
    return BUDDY_ERR_ARG;
  if (dtype != BUDDY_DTYPE_F32 && dtype != BUDDY_DTYPE_BF16 && dtype != BUDDY_DTYPE_F16) return BUDDY_ERR_ARG;
  if (n == 0 || (!k_out && !v_out)) return BUDDY_OK;
  cudaStream_t s = (cudaStream_t)stream;
  if (dtype == BUDDY_DTYPE_F32) return launch_read<float>(cache, n, slot, k_out, v_out, flags, s);
  if (dtype == BUDDY_DTYPE_BF16) return launch_read<bf16>(cache, n, slot, k_out, v_out, flags, s);
  return launch_read<__half>(cache, n, slot, k_out, v_out, flags, s);
}
