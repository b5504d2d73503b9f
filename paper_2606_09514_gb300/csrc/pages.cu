// Block tables and slot maps from request lengths.
//
// One launch: every CTA scans the whole batch (8 bytes per sequence, from L2) into
// the running counts of new tokens and new pages in its shared memory, so that no
// CTA waits for another; then it writes its part of the table entries and slots,
// each found by bisection in those counts.  The checks come out of the same scan,
// before anything is written.  Latency only: 250 sequences of a token each 3.4 us a call,
// 61 prompts of 128 to 1,024 tokens 3.1; two launches, counts first, would cost another
// 2 us.
#include <cuda_runtime.h>

#include "common.cuh"
#include "internal.h"

namespace buddy {

// A thread has a token, up to the largest grid.  (When it was chosen, 61 prompts took 2.9 us, with four tokens each 4.5,
// with CTAs of 128 threads 3.3; 16,000 sequences 34 us, with CTAs of 1,024 threads 51.)
constexpr int kPlanThreads = 256;
constexpr int kPlanMaxBatch = 16384;    // two counts per sequence in shared memory
constexpr size_t plan_smem_bytes(int batch) { return 2 * ((size_t)batch + 1) * sizeof(int32_t); }

// Largest i < n with a[i] <= x, for ascending a with a[0] <= x.
__device__ __forceinline__ int last_at_most(const int32_t* a, int n, int x) {
  int lo = 0, hi = n;
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (a[mid] <= x) lo = mid;
    else hi = mid;
  }
  return lo;
}

__global__ void __launch_bounds__(kPlanThreads) page_plan_kernel(const buddy_page_plan_args A, int shift,
                                                                 int32_t* flags) {
  extern __shared__ int32_t plan_smem[];
  int32_t* tok = plan_smem;               // [batch + 1] new tokens before each sequence
  int32_t* page = plan_smem + A.batch + 1;
  __shared__ int64_t warp_tok[kPlanThreads / 32], warp_page[kPlanThreads / 32];
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int64_t mask = ((int64_t)1 << shift) - 1, room = (int64_t)A.max_pages << shift;
  pdl_wait();
  pdl_trigger();
  const int64_t head = *A.free_head;

  // consecutive sequences per thread: their sums, then a scan over the threads
  const int per = (A.batch + kPlanThreads - 1) / kPlanThreads;
  const int i0 = min(A.batch, tid * per), i1 = min(A.batch, i0 + per);
  int64_t nt = 0, np = 0;
  bool off = false;
  for (int i = i0; i < i1; ++i) {
    const int64_t n = A.len[i], m = A.n_new[i];
    off |= n < 0 || m < 0 || n + m > room;
    nt += m;
    np += ((n + m + mask) >> shift) - ((n + mask) >> shift);
  }
  int64_t st = nt, sp = np;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int64_t a = __shfl_up_sync(0xffffffffu, st, o), b = __shfl_up_sync(0xffffffffu, sp, o);
    if (lane >= o) st += a, sp += b;
  }
  if (lane == 31) warp_tok[warp] = st, warp_page[warp] = sp;
  off = __syncthreads_or(off);
  int64_t all_tok = 0, all_page = 0;
  for (int w = 0; w < kPlanThreads / 32; ++w) {
    if (w == warp) st += all_tok, sp += all_page;
    all_tok += warp_tok[w];
    all_page += warp_page[w];
  }
  int bad = 0;   // (with bad lengths the counts say nothing)
  if (off || all_tok > A.n_tok) bad = BUDDY_DEV_BAD_POSITION;
  else if (head < 0 || head + all_page > A.n_free) bad = BUDDY_DEV_NO_PAGES;
  if (bad) {   // the same in every CTA
    if (flags && blockIdx.x == 0 && tid == 0) atomicOr(flags, bad);
    return;
  }
  st -= nt, sp -= np;
  for (int i = i0; i < i1; ++i) {
    const int64_t n = A.len[i], m = A.n_new[i];
    tok[i] = (int32_t)st;
    page[i] = (int32_t)sp;
    st += m;
    sp += ((n + m + mask) >> shift) - ((n + mask) >> shift);
    if (blockIdx.x == 0) {
      A.kv_len[i] = (int32_t)(n + m);
      A.row_start[i] = tok[i];
    }
  }
  const int T = (int)all_tok, NP = (int)all_page;
  if (tid == 0) {
    tok[A.batch] = T;
    page[A.batch] = NP;
    if (blockIdx.x == 0) {
      A.row_start[A.batch] = T;
      *A.free_head_out = (int32_t)(head + NP);
    }
  }
  __syncthreads();

  // (counted in 64 bits: both ends may be next to 2^31)
  const int stride = gridDim.x * kPlanThreads, first = blockIdx.x * kPlanThreads + tid;
  for (int64_t x = first; x < NP; x += stride) {
    const int i = last_at_most(page, A.batch, (int)x);
    const int64_t held = ((int64_t)A.len[i] + mask) >> shift;
    A.table[(int64_t)i * A.max_pages + held + (x - page[i])] = A.free_pages[head + x];
  }
  for (int64_t t = first; t < A.n_tok; t += stride) {
    int64_t slot = -1;
    int p = -1;
    if (t < T) {
      const int i = last_at_most(tok, A.batch, (int)t);
      const int n = A.len[i];
      p = n + ((int)t - tok[i]);
      const int64_t at = p >> shift, held = ((int64_t)n + mask) >> shift;
      const int32_t id = at < held ? A.table[(int64_t)i * A.max_pages + at] : A.free_pages[head + page[i] + (at - held)];
      slot = ((int64_t)id << shift) + (p & mask);
    }
    A.slot[t] = slot;
    A.pos[t] = p;
  }
}

struct Range {
  const void* p;
  int64_t bytes;
};
static bool overlap(const Range& a, const Range& b) {
  const auto x = reinterpret_cast<uintptr_t>(a.p), y = reinterpret_cast<uintptr_t>(b.p);
  return a.bytes > 0 && b.bytes > 0 && x < y + (uintptr_t)b.bytes && y < x + (uintptr_t)a.bytes;
}

}  // namespace buddy

using namespace buddy;

extern "C" int buddy_page_plan(const buddy_page_plan_args* a, int32_t* flags, void* stream) {
  if (!a || a->batch < 1 || a->batch > kPlanMaxBatch || a->page_size < 1 || a->page_size > 65536 ||
      (a->page_size & (a->page_size - 1)) || a->max_pages < 1 || a->n_free < 0 || a->n_tok < 0 || !a->len ||
      !a->n_new || !a->table || !a->free_head || !a->kv_len || !a->row_start || !a->free_head_out ||
      (a->n_free > 0 && !a->free_pages) || (a->n_tok > 0 && (!a->slot || !a->pos)))
    return BUDDY_ERR_ARG;
  // every CTA reads the inputs while others write: nothing that is written may overlap anything else
  const auto batch = (int64_t)a->batch;
  const Range written[] = {{a->table, batch * a->max_pages * 4}, {a->kv_len, batch * 4},
                           {a->row_start, (batch + 1) * 4},      {a->slot, (int64_t)a->n_tok * 8},
                           {a->pos, (int64_t)a->n_tok * 4},      {a->free_head_out, 4}};
  const Range read[] = {{a->len, batch * 4}, {a->n_new, batch * 4}, {a->free_pages, (int64_t)a->n_free * 4}, {a->free_head, 4}};
  for (const Range& w : written) {
    for (const Range& r : read)
      if (overlap(w, r)) return BUDDY_ERR_ARG;
    for (const Range& o : written)
      if (&o != &w && overlap(w, o)) return BUDDY_ERR_ARG;
  }
  int shift = 0;
  while ((1 << shift) < a->page_size) ++shift;
  const size_t smem = plan_smem_bytes(a->batch);
  // the largest size any call uses: the attribute belongs to the function on the device, and a call's
  // own would take it from another host thread's launch
  if (smem > 40 * 1024 && cudaFuncSetAttribute(page_plan_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                               (int)plan_smem_bytes(kPlanMaxBatch)) != cudaSuccess)
    return BUDDY_ERR_CUDA;
  const int grid = min(max(1, a->n_tok / kPlanThreads + (a->n_tok % kPlanThreads != 0)), 152);
  return launch_k(page_plan_kernel, grid, kPlanThreads, smem, (cudaStream_t)stream, true, *a, shift, flags) == cudaSuccess
             ? BUDDY_OK : BUDDY_ERR_CUDA;
}
