// Layout of the paged 4-bit cache (include/buddy.h) and its arithmetic.
//
// A scale has 7 significant bits so that a code becomes its value in one
// half-precision instruction without a rounding: a code n in bits 4..7 of a half
// whose exponent field says 64 .. 127 is 64 + n; 72 s has 7 + 4 bits and is exact,
// and fma(64 + n, s, -72 s) = (n - 8) s has 4 + 7 bits and is exact.  The scale's
// limit of 896 keeps 72 s finite.
#pragma once

#include <cuda_fp16.h>

#include "common.cuh"

namespace buddy {
namespace kv4 {

constexpr int kGroup = 32;              // channels that share a scale
constexpr float kMaxScale = 896.f;

__host__ __device__ constexpr int code_bytes(int hd) { return hd / 2; }
__host__ __device__ constexpr int scale_bytes(int hd) { return hd / 16; }
__host__ __device__ constexpr int entry_bytes(int hd) { return code_bytes(hd) + scale_bytes(hd); }

struct Pages {
  uint8_t* k;
  uint8_t* v;
  int n_pages, shift, nkv;              // page size 1 << shift
};

// Byte offset of block (page, head).
template <int HD>
__device__ __forceinline__ int64_t block_at(const Pages& p, int64_t page, int g) {
  return ((page * p.nkv + g) << p.shift) * entry_bytes(HD);
}

// Scale of a group from the bit pattern of its largest magnitude (as integers,
// magnitudes order like the numbers and a NaN is above infinity).
__device__ __forceinline__ __half scale_of(uint32_t amax_bits) {
  if (amax_bits > 0x7F800000u) return __ushort_as_half(0x7E00);
  uint32_t u = __float_as_uint(__fdiv_rn(__uint_as_float(amax_bits), 7.f));
  u = (u + 0xFFFFu + ((u >> 17) & 1u)) & ~0x1FFFFu;   // 24 -> 7 significant bits, ties to even
  return __float2half_rn(fminf(__uint_as_float(u), kMaxScale));
}

// Nibble of the code word that holds channel e of eight.
__host__ __device__ constexpr int nibble_of(int e) { return (e & 1) ? 4 + (e >> 1) : e >> 1; }

__device__ __forceinline__ float decode(uint32_t w, int e, float s) {
  return (float)((int)((w >> (4 * nibble_of(e))) & 15u) - 8) * s;
}

}  // namespace kv4
}  // namespace buddy
