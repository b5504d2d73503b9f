// What the attention kernels over the 4-bit cache share: arguments, the sequences'
// checks, and codes to halves.
#pragma once

#include "attn_tc.cuh"
#include "common.cuh"
#include "kv4.cuh"
#include "ptx.cuh"

namespace buddy {
namespace kv4 {

struct AttnArgs4 {
  buddy_kv4_attention_args a;
  Pages p;
  int G, row_limit;           // sequences of at most this many rows are the few-row kernel's
  int32_t* flags;
  int32_t* arrive;            // few rows: [grid], zero between calls
  float* part;                // partials of streams or items that are cut
};

// A sequence's query tokens t0 .. t0 + m - 1 and its n positions; m = 0 where they are bad.
struct Rows {
  int t0, m, n;
};
__device__ __forceinline__ Rows rows_of(const AttnArgs4& A, int i, bool* bad) {
  Rows s;
  s.t0 = A.a.row_start ? A.a.row_start[i] : i;
  const int t1 = A.a.row_start ? A.a.row_start[i + 1] : i + 1;
  s.n = A.a.kv_len[i];
  *bad = s.t0 < 0 || t1 < s.t0 || t1 > A.a.n_tok || t1 - s.t0 > A.a.max_new || s.n < 0 ||
         s.n > (int64_t)A.a.max_pages << A.p.shift;
  s.m = *bad ? 0 : t1 - s.t0;
  return s;
}

// Probabilities enter the products as halves, 2^kHigh times what the running reference makes
// them: a row's largest is 2^7 at least, and 2^15 at most, since the reference follows the
// maximum when that is more than 8 above.  With eleven bits down to 2^-21 of the largest, and
// below that steps of 2^-31 of it, a million small ones behind a few large ones still add up.  (At
// 1 to 2^8 they would be rounded to steps of 2^-24 of the largest, or to nothing: 4,092
// positions with 2^-23.4 of it each came out a third too small.)
constexpr float kHigh = 7.f;

// Numbers of the products.  A product takes halves, eleven bits of a query's element or of a
// probability, which is what bf16 queries have and bf16 outputs can hold.  Where the queries or
// the outputs are fp32 (WIDE), each is the sum of two halves, the second one what the first
// leaves: 22 bits, for twice as many MMAs.
template <bool WIDE>
struct Halves {
  uint32_t hi, lo;
  __device__ __forceinline__ Halves(float a, float b) {
    const __half2 h = __floats2half2_rn(a, b);
    hi = *reinterpret_cast<const uint32_t*>(&h);
    if constexpr (WIDE) {
      const __half2 l = __floats2half2_rn(a - __low2float(h), b - __high2float(h));
      lo = *reinterpret_cast<const uint32_t*>(&l);
    }
  }
};

// For query rows that enter the products as halves of 1 .. 2 (WIDE: 2^14 .. 2^15, so that the
// second halves are not among the smallest): the power of two that takes the row's largest
// magnitude there, and the factor that takes a score of the halves to base 2 (base: log2(e)
// times the scores' scale; above zero, so that it takes -inf to -inf).
template <bool WIDE>
__device__ __forceinline__ void row_scale(float top, float base, float* down, float* fac) {
  constexpr int UP = WIDE ? 14 : 0;
  const int ex = min(max((int)(__float_as_uint(top) >> 23) - 127, UP - 126), 126);
  *down = __uint_as_float((uint32_t)(127 + UP - ex) << 23);
  *fac = fmaxf(base * __uint_as_float((uint32_t)(127 - UP + ex) << 23), 1.2e-38f);
}

__device__ __forceinline__ uint32_t h2(__half2 v) { return *reinterpret_cast<uint32_t*>(&v); }
__device__ __forceinline__ __half2 as_h2(uint32_t v) { return *reinterpret_cast<__half2*>(&v); }

// Codes in bits 4 .. 7 of both halves -> (code - 8) s, with s72 = -72 s.
__device__ __forceinline__ uint32_t dequant(uint32_t w, __half2 s, __half2 s72) {
  uint32_t x;
  asm("lop3.b32 %0, %1, 0x00F000F0, 0x54005400, 0xEA;" : "=r"(x) : "r"(w));   // (w & mask) | 64.0
  return h2(__hfma2(as_h2(x), s, s72));
}
// Codes in bits 0 .. 3: 1024 + n needs a subtraction of its own (1032 s would be rounded), but no
// shift, and shifts share their pipe with the logical instructions.
__device__ __forceinline__ uint32_t dequant_low(uint32_t w, __half2 s) {
  uint32_t x;
  asm("lop3.b32 %0, %1, 0x000F000F, 0x64006400, 0xEA;" : "=r"(x) : "r"(w));
  return h2(__hmul2(__hadd2(as_h2(x), __float2half2_rn(-1032.f)), s));
}
__device__ __forceinline__ void dequant2(uint32_t w, __half2 s, __half2 s72, uint32_t* o) {
  o[0] = dequant_low(w, s);
  o[1] = dequant(w, s, s72);
}
// The four pairs (codes j of both halves) of a word.  (With shifts for all four, 250 sequences
// take 96.6 us instead of 93.9; with shifts as high halves of products 4 to 10% more.)
__device__ __forceinline__ void dequant4(uint32_t w, __half2 s, __half2 s72, uint32_t* o) {
  dequant2(w, s, s72, o);
  dequant2(w >> 8, s, s72, o + 2);
}

// Sequences of more than row_limit rows per KV head (kv4_pf.cu).
int64_t prompt_workspace(int head_dim, int sms);
int launch_prompt(AttnArgs4 A, int head_dim, bool wide, int sms, void* ws, cudaStream_t s);

// Lists of pages of so many (token, KV head) streams that a warp takes them alone (kv4_lists.cu).
int launch_lists(const AttnArgs4& A, int head_dim, bool wide, int sms, cudaStream_t s);

}  // namespace kv4
}  // namespace buddy
