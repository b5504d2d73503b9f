// Rows of queries, keys and values between a block's QKV projection and its
// attention: norm of each head and rotation (buddy_qk_norm_rope), the same with the
// entries quantised into the paged 4-bit cache (buddy_kv4_append), and entries read
// back (buddy_kv4_read).
//
// A team of HD / 8 lanes holds a head, eight channels per lane in one 16-byte load:
// the channel that the rotation pairs with is in the lane HD / 16 further on, a
// scale's 32 channels are four lanes, and a lane's eight codes are one word.  A team
// takes kRowHeads consecutive heads of a token, all loaded before the first is used,
// so that the token's position and rotation factors are read once for them.
//
// The sum of squares: within a lane halves of the eight onto each other, then
// halves of the lanes; products and sums rounded one by one (no fused
// multiply-adds), so that a plain program can follow it bit by bit, which the codes
// need: where a value lies between two codes, one bit decides.
#include <cuda_runtime.h>

#include "common.cuh"
#include "internal.h"
#include "kv4.cuh"

namespace buddy {

constexpr int kRowThreads = 256;
constexpr int kRowHeads = 4;

struct RowArgs {
  buddy_qk_rows r;
  const void* v;
  int64_t v_stride;
  kv4::Pages pages;
  const int64_t* slot;
  int32_t* flags;
};

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

// Every lane's x of the head becomes x / sqrt(mean(x^2) + eps) * gain.
template <int HD>
__device__ __forceinline__ void norm_head(float* x, const float* gain, float eps) {
  float q[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) q[e] = __fmul_rn(x[e], x[e]);
#pragma unroll
  for (int n = 4; n > 0; n >>= 1)
#pragma unroll
    for (int e = 0; e < n; ++e) q[e] = __fadd_rn(q[e], q[e + n]);
#pragma unroll
  for (int o = HD / 16; o > 0; o >>= 1) q[0] = __fadd_rn(q[0], __shfl_xor_sync(0xffffffffu, q[0], o));
  const float r = __fdiv_rn(1.f, __fsqrt_rn(__fadd_rn(__fmul_rn(q[0], 1.f / HD), eps)));
#pragma unroll
  for (int e = 0; e < 8; ++e) x[e] = __fmul_rn(__fmul_rn(x[e], r), gain[e]);
}

template <int HD>
__device__ __forceinline__ void turn_head(float* x, const float* co, const float* si, bool low) {
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const float y = __shfl_xor_sync(0xffffffffu, x[e], HD / 16);
    const float a = __fmul_rn(x[e], co[e]), b = __fmul_rn(y, si[e]);
    x[e] = low ? __fsub_rn(a, b) : __fadd_rn(a, b);
  }
}

// The lane's eight channels into an entry at byte `at` of `pages`; whole teams call it.
template <int HD>
__device__ __forceinline__ void store_entry(uint8_t* pages, int64_t block, int row, int shift, int tl, const float* x,
                                            bool real) {
  uint32_t m = 0;
#pragma unroll
  for (int e = 0; e < 8; ++e) m = max(m, __float_as_uint(x[e]) & 0x7FFFFFFFu);
  m = max(m, __shfl_xor_sync(0xffffffffu, m, 1));
  m = max(m, __shfl_xor_sync(0xffffffffu, m, 2));
  const __half s = kv4::scale_of(m);
  if (!real) return;
  uint8_t* b = pages + block;
  *reinterpret_cast<uint32_t*>(b + row * kv4::code_bytes(HD) + 4 * tl) = kv4::encode8(x, __half2float(s));
  if ((tl & 3) == 0)
    *reinterpret_cast<__half*>(b + ((int64_t)kv4::code_bytes(HD) << shift) + row * kv4::scale_bytes(HD) + (tl >> 1)) = s;
}

template <typename T, int HD, bool CACHE>
__global__ void __launch_bounds__(kRowThreads) qk_rows_kernel(const RowArgs A) {
  constexpr int LPH = HD / 8, TEAMS = kRowThreads / LPH;
  const buddy_qk_rows& R = A.r;
  const int heads = R.n_q_heads + R.n_kv_heads * (CACHE ? 2 : 1);
  const int groups = (heads + kRowHeads - 1) / kRowHeads;
  const int tl = threadIdx.x % LPH;
  const int64_t u = (int64_t)blockIdx.x * TEAMS + threadIdx.x / LPH;
  const int t = (int)min(u / groups, (int64_t)R.n_tok - 1);
  const bool there = u < (int64_t)R.n_tok * groups;
  const int h0 = (int)(u % groups) * kRowHeads;

  const int p = R.pos[t];
  const bool ok = there && p >= 0 && p < R.max_pos;
  int64_t slot = -1;
  if (CACHE) slot = A.slot[t];
  const int64_t end = (int64_t)A.pages.n_pages << A.pages.shift;
  if (there && tl == 0 && h0 == 0 && A.flags) {
    const int bad = (p >= R.max_pos ? BUDDY_DEV_BAD_POSITION : 0) |
                    (CACHE && p >= 0 && slot >= end ? BUDDY_DEV_BAD_PAGE : 0);
    if (bad) atomicOr(A.flags, bad);
  }
  const bool keep = CACHE && ok && slot >= 0 && slot < end;

  float x[kRowHeads][8];
#pragma unroll
  for (int i = 0; i < kRowHeads; ++i) {
    int h = min(h0 + i, heads - 1);
    const T* src;
    if (h < R.n_q_heads) src = (const T*)R.q + t * R.q_stride;
    else if ((h -= R.n_q_heads) < R.n_kv_heads) src = (const T*)R.k + t * R.k_stride;
    else h -= R.n_kv_heads, src = (const T*)A.v + t * A.v_stride;
    load8(src + (int64_t)h * HD + tl * 8, x[i]);
  }
  float co[8], si[8];
  const bool low = tl < LPH / 2;
  {
    const int64_t at = (int64_t)(ok ? p : 0) * (HD / 2) + (low ? tl : tl - LPH / 2) * 8;
    load8(R.rope_cos + at, co);
    load8(R.rope_sin + at, si);
  }
#pragma unroll
  for (int i = 0; i < kRowHeads; ++i) {
    const int h = h0 + i;
    const bool is_q = h < R.n_q_heads, is_v = h >= R.n_q_heads + R.n_kv_heads;
    const bool real = ok && h < heads;
    const float* gains = is_q ? R.q_gain : R.k_gain;
    // (a warp may hold teams of both kinds: all lanes take part in the shuffles)
    float y[8], gain[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) y[e] = x[i][e], gain[e] = 1.f;
    if (gains) load8(gains + tl * 8, gain);
    norm_head<HD>(y, gain, R.eps);
#pragma unroll
    for (int e = 0; e < 8; ++e) y[e] = gains ? y[e] : x[i][e];
    turn_head<HD>(y, co, si, low);
    if (is_q) {
      if (real) store8((T*)R.q_out + t * R.q_out_stride + (int64_t)h * HD + tl * 8, y);
    } else if (!is_v) {
      if (real && R.k_out) store8((T*)R.k_out + t * R.k_out_stride + (int64_t)(h - R.n_q_heads) * HD + tl * 8, y);
    }
    if (CACHE) {
      const int g = is_v ? h - R.n_q_heads - R.n_kv_heads : h - R.n_q_heads;
#pragma unroll
      for (int e = 0; e < 8; ++e) y[e] = is_v ? x[i][e] : y[e];
      const bool put = keep && real && !is_q;
      const int64_t block = put ? kv4::block_at<HD>(A.pages, slot >> A.pages.shift, g) : 0;
      store_entry<HD>(is_v ? A.pages.v : A.pages.k, block, (int)(slot & ((1 << A.pages.shift) - 1)), A.pages.shift, tl,
                      y, put);
    }
  }
}

template <typename T, int HD>
__global__ void __launch_bounds__(kRowThreads) kv4_read_kernel(const kv4::Pages P, int n, const int64_t* slots, T* k_out,
                                                               T* v_out, int32_t* flags) {
  constexpr int LPH = HD / 8;
  const int64_t u = ((int64_t)blockIdx.x * kRowThreads + threadIdx.x) / LPH;   // (entry, head)
  const int tl = threadIdx.x % LPH;
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
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    T* out = i ? v_out : k_out;
    if (!out) continue;
    const uint8_t* b = (i ? P.v : P.k) + block;
    const uint32_t w = *reinterpret_cast<const uint32_t*>(b + row * kv4::code_bytes(HD) + 4 * tl);
    const float s = __half2float(*reinterpret_cast<const __half*>(b + ((int64_t)kv4::code_bytes(HD) << P.shift) +
                                                                  row * kv4::scale_bytes(HD) + (tl >> 2) * 2));
    float y[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) y[e] = kv4::decode(w, e, s);
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

template <typename T, int HD, bool CACHE>
static int launch_rows(const RowArgs& A, cudaStream_t s) {
  const int heads = A.r.n_q_heads + A.r.n_kv_heads * (CACHE ? 2 : 1);
  const int64_t teams = (int64_t)A.r.n_tok * ((heads + kRowHeads - 1) / kRowHeads);
  const int64_t ctas = (teams * (HD / 8) + kRowThreads - 1) / kRowThreads;
  if (ctas > INT32_MAX) return BUDDY_ERR_RANGE;
  qk_rows_kernel<T, HD, CACHE><<<(unsigned)ctas, kRowThreads, 0, s>>>(A);
  return cudaGetLastError() == cudaSuccess ? BUDDY_OK : BUDDY_ERR_CUDA;
}
template <bool CACHE>
static int dispatch_rows(const RowArgs& A, cudaStream_t s) {
  if (A.r.n_tok == 0) return BUDDY_OK;
  if (A.r.dtype == BUDDY_DTYPE_F32)
    return A.r.head_dim == 128 ? launch_rows<float, 128, CACHE>(A, s) : launch_rows<float, 64, CACHE>(A, s);
  return A.r.head_dim == 128 ? launch_rows<bf16, 128, CACHE>(A, s) : launch_rows<bf16, 64, CACHE>(A, s);
}

template <typename T>
static int launch_read(const buddy_kv4_cache* c, int n, const int64_t* slot, void* k, void* v, int32_t* flags,
                       cudaStream_t s) {
  const int64_t ctas = ((int64_t)n * c->n_kv_heads * (c->head_dim / 8) + kRowThreads - 1) / kRowThreads;
  if (ctas > INT32_MAX) return BUDDY_ERR_RANGE;
  if (c->head_dim == 128)
    kv4_read_kernel<T, 128><<<(unsigned)ctas, kRowThreads, 0, s>>>(kv4_pages(c), n, slot, (T*)k, (T*)v, flags);
  else
    kv4_read_kernel<T, 64><<<(unsigned)ctas, kRowThreads, 0, s>>>(kv4_pages(c), n, slot, (T*)k, (T*)v, flags);
  return cudaGetLastError() == cudaSuccess ? BUDDY_OK : BUDDY_ERR_CUDA;
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
  return dispatch_rows<false>(A, (cudaStream_t)stream);
}

extern "C" int buddy_kv4_append(const buddy_kv4_cache* cache, const buddy_qk_rows* rows, const void* v,
                                int64_t v_stride, const int64_t* slot, int32_t* flags, void* stream) {
  if (!kv4_cache_ok(cache) || !rows_ok(rows, false) || rows->n_kv_heads != cache->n_kv_heads ||
      rows->head_dim != cache->head_dim)
    return BUDDY_ERR_ARG;
  if (rows->n_tok > 0 && (!slot || !aligned_rows(v, v_stride, rows->dtype == BUDDY_DTYPE_F32 ? 4 : 2)))
    return BUDDY_ERR_ARG;
  const RowArgs A{*rows, v, v_stride, kv4_pages(cache), slot, flags};
  return dispatch_rows<true>(A, (cudaStream_t)stream);
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
