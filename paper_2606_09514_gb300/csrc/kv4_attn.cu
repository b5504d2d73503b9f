// Causal attention over the paged 4-bit cache.
//
// One CTA per (sequence, place of the query token in it, KV head): its warps take the positions in turn, a lane
// holding four channels of the group's query heads; running maximum and sum per
// head, joined over the warps at the end.
#include <cuda_runtime.h>

#include "common.cuh"
#include "internal.h"
#include "kv4.cuh"

namespace buddy {

bool kv4_cache_ok(const buddy_kv4_cache* c);
kv4::Pages kv4_pages(const buddy_kv4_cache* c);

constexpr int kSimpleWarps = 4;

template <int HD>
__global__ void __launch_bounds__(32 * kSimpleWarps) kv4_attn_simple_kernel(const buddy_kv4_attention_args A,
                                                                            const kv4::Pages P, int32_t* flags) {
  constexpr int C = HD / 32;
  const int i = blockIdx.x / A.max_new, j = blockIdx.x % A.max_new;
  const int g = blockIdx.y, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int G = A.n_q_heads / P.nkv;
  const int t0 = A.row_start ? A.row_start[i] : i, t1 = A.row_start ? A.row_start[i + 1] : i + 1;
  const int n = A.kv_len[i], m = t1 - t0;
  if (t0 < 0 || t1 < t0 || t1 > A.n_tok || m > A.max_new || n < 0 || n > (int64_t)A.max_pages << P.shift) {
    if (flags && threadIdx.x == 0) atomicOr(flags, BUDDY_DEV_BAD_POSITION);
    return;
  }
  if (j >= m) return;
  const int t = t0 + j;
  const int seen = min(n, n - m + j + 1);
  const float scale = A.scale != 0.f ? A.scale : rsqrtf((float)HD);
  float q[8][C], acc[8][C], mx[8], sum[8];
#pragma unroll
  for (int h = 0; h < 8; ++h) {
    mx[h] = -INFINITY, sum[h] = 0.f;
    for (int c = 0; c < C; ++c) {
      acc[h][c] = 0.f;
      const int64_t at = t * A.q_stride + (int64_t)(g * G + min(h, G - 1)) * HD + lane * C + c;
      q[h][c] = (A.q_dtype == BUDDY_DTYPE_F32 ? ((const float*)A.q)[at] : to_f(((const bf16*)A.q)[at])) * scale;
    }
  }
  for (int p = warp; p < seen; p += kSimpleWarps) {
    const int page = A.table[(int64_t)i * A.max_pages + (p >> P.shift)];
    if (page < 0 || page >= P.n_pages) {
      if (flags && lane == 0) atomicOr(flags, BUDDY_DEV_BAD_PAGE);
      continue;
    }
    const int row = p & ((1 << P.shift) - 1);
    float kv[2][C];
#pragma unroll
    for (int x = 0; x < 2; ++x) {
      const uint8_t* b = (x ? P.v : P.k) + kv4::block_at<HD>(P, page, g);
      const int ch = lane * C;
      const uint32_t w = *reinterpret_cast<const uint32_t*>(b + row * kv4::code_bytes(HD) + (ch / 8) * 4);
      const float s = __half2float(*reinterpret_cast<const __half*>(b + ((int64_t)kv4::code_bytes(HD) << P.shift) +
                                                                    row * kv4::scale_bytes(HD) + ch / 32 * 2));
      for (int c = 0; c < C; ++c) kv[x][c] = kv4::decode(w, (ch + c) & 7, s);
    }
#pragma unroll
    for (int h = 0; h < 8; ++h) {
      float d = 0.f;
      for (int c = 0; c < C; ++c) d += q[h][c] * kv[0][c];
      d = warp_sum(d);
      const float m1 = fmaxf(mx[h], d);
      const float a = expf(mx[h] - m1), e = expf(d - m1);
      mx[h] = m1;
      sum[h] = sum[h] * a + e;
      for (int c = 0; c < C; ++c) acc[h][c] = acc[h][c] * a + e * kv[1][c];
    }
  }
  __shared__ float s_m[kSimpleWarps][8], s_l[kSimpleWarps][8], s_o[kSimpleWarps][8][HD];
#pragma unroll
  for (int h = 0; h < 8; ++h) {
    if (lane == 0) s_m[warp][h] = mx[h], s_l[warp][h] = sum[h];
    for (int c = 0; c < C; ++c) s_o[warp][h][lane * C + c] = acc[h][c];
  }
  __syncthreads();
  for (int x = threadIdx.x; x < G * HD; x += blockDim.x) {
    const int h = x / HD, c = x % HD;
    float M = -INFINITY, L = 0.f, O = 0.f;
    for (int w = 0; w < kSimpleWarps; ++w) M = fmaxf(M, s_m[w][h]);
    for (int w = 0; w < kSimpleWarps; ++w) {
      const float a = s_l[w][h] != 0.f ? expf(s_m[w][h] - M) : 0.f;
      if (a != 0.f) L += a * s_l[w][h], O += a * s_o[w][h][c];
    }
    const float o = L != 0.f ? O / L : 0.f;
    const int64_t at = t * A.out_stride + (int64_t)(g * G + h) * HD + c;
    if (A.out_dtype == BUDDY_DTYPE_F32) ((float*)A.out)[at] = o;
    else ((bf16*)A.out)[at] = from_f<bf16>(o);
  }
}

}  // namespace buddy

using namespace buddy;

extern "C" int64_t buddy_kv4_attention_workspace(int32_t n_q_heads, int32_t n_kv_heads, int32_t head_dim,
                                                 int32_t max_new) {
  if (n_kv_heads < 1 || n_kv_heads > 1024 || n_q_heads < n_kv_heads || n_q_heads % n_kv_heads ||
      n_q_heads / n_kv_heads > 8 || (head_dim != 64 && head_dim != 128) || max_new < 1)
    return -1;
  return 256;
}

extern "C" int buddy_kv4_attention(const buddy_kv4_cache* cache, const buddy_kv4_attention_args* a, int32_t* flags,
                                   void* stream) {
  if (!kv4_cache_ok(cache) || !a || a->batch < 1 || a->batch > 16384 || a->n_tok < 0 || a->max_pages < 1 ||
      (int64_t)a->max_pages * cache->page_size > INT32_MAX || !(a->scale >= 0.f) || a->scale > 3e38f)
    return BUDDY_ERR_ARG;
  const int64_t need =
      buddy_kv4_attention_workspace(a->n_q_heads, cache->n_kv_heads, cache->head_dim, a->max_new);
  if (need < 0 || (a->q_dtype != BUDDY_DTYPE_F32 && a->q_dtype != BUDDY_DTYPE_BF16) ||
      (a->out_dtype != BUDDY_DTYPE_F32 && a->out_dtype != BUDDY_DTYPE_BF16) || !a->kv_len || !a->table)
    return BUDDY_ERR_ARG;
  if (!a->row_start && (a->n_tok != a->batch || a->max_new != 1)) return BUDDY_ERR_ARG;
  if (!a->workspace || a->workspace_bytes < need || (reinterpret_cast<uintptr_t>(a->workspace) & 255)) return BUDDY_ERR_ARG;
  if (a->n_tok == 0) return BUDDY_OK;
  if ((int64_t)a->batch * a->max_new > INT32_MAX) return BUDDY_ERR_RANGE;
  if (!a->q || !a->out || !aligned16(a->q) || !aligned16(a->out) ||
      a->q_stride * (a->q_dtype == BUDDY_DTYPE_F32 ? 4 : 2) % 16 || a->out_stride * (a->out_dtype == BUDDY_DTYPE_F32 ? 4 : 2) % 16)
    return BUDDY_ERR_ARG;
  dim3 grid((unsigned)((int64_t)a->batch * a->max_new), cache->n_kv_heads);
  if (cache->head_dim == 128)
    kv4_attn_simple_kernel<128><<<grid, 32 * kSimpleWarps, 0, (cudaStream_t)stream>>>(*a, kv4_pages(cache), flags);
  else
    kv4_attn_simple_kernel<64><<<grid, 32 * kSimpleWarps, 0, (cudaStream_t)stream>>>(*a, kv4_pages(cache), flags);
  return cudaGetLastError() == cudaSuccess ? BUDDY_OK : BUDDY_ERR_CUDA;
}
