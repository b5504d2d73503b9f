/*
 * libbuddy — budget-routed batched decode (BUDDY, arXiv 2606.09514) on one
 * NVIDIA GB300 (sm_103a).
 *
 * One decode step, for every sequence i of a batch:
 *   1. runs the first decoder block (always executed, Sec. 4.2.1) -- blocks
 *      0..c with a context layer c > 0 (App. D, Start Layer ablation);
 *   2. pools the context layer's cache (value states by default, or key states,
 *      or their sum, Sec. 5.4), including the newest token, and concatenates
 *      the newest token's hidden state (KV-aware planner, Sec. 4.3);
 *   3. scores the routed blocks c+1 .. L-2 with the Decision Module, a
 *      Linear-SiLU-Linear MLP (App. C.1), fused with an optional prior
 *      s' = s + omega * p~ (Eq. 2); a sequence without a budget (k_i = 0)
 *      takes the Budget Predictor's k^ (Sec. 4.4);
 *   4. executes the k_i highest-scoring routed blocks (Eq. 2, ties to the lower
 *      layer index), each block on the sub-batch of sequences that selected it
 *      (grouping by mask, App. C.1), skipped blocks being the identity (Eq. 1)
 *      and storing zero K/V at the new position (Sec. 6) -- or nothing, in the
 *      masked variant;
 *   5. runs the last block (always executed) and advances every sequence's
 *      position by one (KV cache update, Eq. 9).
 *
 * buddy_prefill does the same for whole prompts: one route per prompt, every
 * prompt token through the selected blocks (Sec. 4.1, App. E).
 *
 * Conventions for every entry point:
 *   - Pointers marked "device" are device pointers owned by the caller; the
 *     library never frees them.  Weight pointers are retained (not copied) by
 *     buddy_set_weights and must stay valid while the context is used.
 *   - Weight matrices (of the Decision Module and the Budget Predictor: w1) and
 *     norm gains, the K/V caches, the pooled sums and the hidden-state buffers
 *     (h_in, h_out, prefill x, route h1) must be 16-byte aligned (the kernels
 *     access them with 16-byte vectors and TMA); a misaligned one is rejected
 *     with BUDDY_ERR_ARG.
 *   - `stream` is a cudaStream_t passed as void* (NULL = legacy default stream).
 *     Calls are asynchronous on that stream unless stated otherwise.
 *   - Return value: BUDDY_OK or a BUDDY_ERR_* code.  On a host-detected error
 *     nothing is launched and nothing is written.  Conditions that only the
 *     device can see (a budget or position stored in device memory out of
 *     range) make every kernel of that call return without writing; the flag
 *     is reported by buddy_device_status().
 *   - The library allocates device memory only in buddy_create (scratch sized
 *     by max_batch, max_pos and max_prefill_tokens), in buddy_set_weights
 *     (tensor descriptors, split-K workspace; with max_prefill_tokens > 0 also
 *     40 MB for the parts of cut prefill units) and in
 *     buddy_set_budget_predictor (its hidden units).  With max_prefill_tokens
 *     > 0 buddy_create also pins host memory, as much as the device holds of a
 *     call's tables: about n_layers * (max_prefill_tokens * (4 + n_q_heads / 4)
 *     + max_batch * n_q_heads * 16) bytes (30 MB for 32 layers, 32 heads, 256
 *     sequences and 65,536 tokens).
 */
#ifndef BUDDY_H_
#define BUDDY_H_

#include <stdint.h>

#if defined(__GNUC__)
#define BUDDY_API __attribute__((visibility("default")))
#else
#define BUDDY_API
#endif

#ifdef __cplusplus
extern "C" {
#endif

enum {
  BUDDY_OK = 0,
  BUDDY_ERR_ARG = 1,      /* null pointer, bad size, unsupported shape */
  BUDDY_ERR_RANGE = 2,    /* value outside its documented range (host-visible) */
  BUDDY_ERR_CUDA = 3,     /* a CUDA runtime call failed */
  BUDDY_ERR_DEVICE = 4,   /* a kernel raised the device error flag */
  BUDDY_ERR_STATE = 5     /* call order: e.g. weights not set */
};

enum { BUDDY_DTYPE_F32 = 0, BUDDY_DTYPE_BF16 = 1, BUDDY_DTYPE_F16 = 2 /* buddy_kv4_read only */ };

/* Planner feature G_t pooled from the context layer's cache (Sec. 4.3; the
 * Sec. 5.4 ablation "Hidden-State Features"): value states (the paper's
 * default), key states (as cached, after RoPE), or their element-wise sum. */
enum { BUDDY_FEATURE_V = 0, BUDDY_FEATURE_K = 1, BUDDY_FEATURE_KV = 2 };

/* KV of a sequence at a block it skips (Sec. 6): zero-filled K and V at the
 * new position, which later attention includes with logit 0 (the paper's
 * design); or nothing stored, so that block's later attention reads only the
 * positions at which it executed (the KV-cache strategy Sec. 6 leaves to
 * future work). */
enum { BUDDY_SKIP_ZERO = 0, BUDDY_SKIP_MASKED = 1 };

/* Bits of the device error flag (buddy_device_status). */
enum {
  BUDDY_DEV_BAD_BUDGET = 1,    /* k_i outside [1, L-2-c] (0 without a Budget Predictor) */
  BUDDY_DEV_BAD_POSITION = 2,  /* len_i + new positions > cap_i or > max_pos */
  BUDDY_DEV_BAD_SEQ = 4,       /* a sequence id outside [0, batch) */
  BUDDY_DEV_TIMEOUT = 8,       /* a bounded wait inside a kernel ran out */
  BUDDY_DEV_NO_PAGES = 16,     /* the list of free pages is shorter than what a plan needs */
  BUDDY_DEV_BAD_PAGE = 32      /* a page id outside [0, n_pages) (a slot's or a table's) */
};

typedef struct buddy_ctx buddy_ctx;

/* Model shape.  The decoder block is Llama-style (App. "Background"):
 * RMSNorm, Q/K/V projections (optional bias, Qwen2.5), rotate-half RoPE,
 * grouped-query attention, output projection, RMSNorm, SwiGLU MLP d->F->d.
 * Requirements: n_layers >= 3; head_dim 64 or 128; n_q_heads a multiple of
 * n_kv_heads (group of at most 8); d_model == n_q_heads * head_dim, a
 * multiple of 64; ffn_dim a multiple of 8; dm_hidden >= 1;
 * 1 <= max_batch <= 1024 (<= 256 for bf16, which needs an sm_103 device);
 * max_pos >= 1; 0 <= ctx_layer <= n_layers - 3; 0 <= max_prefill_tokens
 * <= 65536.  The routed blocks are ctx_layer+1 .. n_layers-2: their number
 * n_cand = n_layers - 2 - ctx_layer sizes the Decision Module's output. */
typedef struct {
  int32_t n_layers;     /* L */
  int32_t d_model;      /* d */
  int32_t n_q_heads;
  int32_t n_kv_heads;
  int32_t head_dim;
  int32_t ffn_dim;      /* F */
  int32_t dm_hidden;    /* r: Decision Module hidden width */
  int32_t dtype;        /* BUDDY_DTYPE_F32 or BUDDY_DTYPE_BF16: weights, KV cache, GEMM inputs */
  int32_t max_batch;    /* largest B of any call */
  int32_t max_pos;      /* every position p written or read satisfies p < max_pos */
  int32_t qkv_bias;     /* 1: Q/K/V projections carry a bias */
  int32_t feature;      /* BUDDY_FEATURE_*: planner feature */
  int32_t ctx_layer;    /* c: blocks 0..c always run, the planner reads block c's cache */
  int32_t skip_kv;      /* BUDDY_SKIP_*: what a skipped block stores */
  int32_t max_prefill_tokens;  /* 0: no buddy_prefill; else the largest sum of prompt lengths */
  float rms_eps;
  float rope_theta;
} buddy_config;

/* One decoder layer; matrices row-major in nn.Linear layout [out, in],
 * element type = config dtype; gains and biases fp32. */
typedef struct {
  const float* attn_norm;   /* device [d] */
  const void* w_qkv;        /* device [(n_q + 2 n_kv) * hd, d]: Q rows, then K rows, then V rows */
  const float* b_qkv;       /* device [(n_q + 2 n_kv) * hd], or NULL when qkv_bias == 0 */
  const void* w_o;          /* device [d, n_q * hd] */
  const float* ffn_norm;    /* device [d] */
  const void* w_gate_up;    /* device [2F, d]: rows [0, F) gate, rows [F, 2F) up */
  const void* w_down;       /* device [d, F] */
} buddy_layer_weights;

/* Decision Module (App. C.1): s' = W2 SiLU(W1 x + b1) + b2 + omega * prior,
 * x = [pool expanded to d ; h] of width 2d (Sec. 4.3).  All fp32.
 * n_cand = n_layers - 2 - ctx_layer. */
typedef struct {
  const float* w1;      /* device [r, 2d] */
  const float* b1;      /* device [r] */
  const float* w2;      /* device [n_cand, r] */
  const float* b2;      /* device [n_cand] */
  const float* prior;   /* device [n_cand] normalised prior p~ (Eq. 2), or NULL */
  float omega;          /* prior weight (ignored when prior == NULL) */
} buddy_dm_weights;

/* Budget Predictor (Sec. 4.4): a categorical policy pi(k | G_t) over
 * A = {1..n_cand} on the Decision Module's input x, here the same
 * Linear-SiLU-Linear form: logits = W2 SiLU(W1 x + b1) + b2; k^ = argmax
 * (ties to the smaller k), i.e. budget b^ = (k^ + 2 + ctx_layer) / L (Eq. 3).
 * All fp32. */
typedef struct {
  const float* w1;      /* device [hidden, 2d] */
  const float* b1;      /* device [hidden] */
  const float* w2;      /* device [n_cand, hidden] */
  const float* b2;      /* device [n_cand] */
  int32_t hidden;       /* >= 1 */
} buddy_predictor_weights;

/* Per-layer KV caches and per-sequence positions (Eq. 9).
 * Element (sequence i, kv head g, position p, channel e) of layer l's K cache
 * is at  k_cache[l] + ((seq_off[i] * n_kv + g * cap[i] + p) * head_dim + e)
 * elements (same for V): each sequence owns a head-major block of cap[i]
 * positions; blocks must not overlap.  len[i] = tokens n_i of sequence i (the
 * RoPE position of its next token).  With BUDDY_SKIP_ZERO every layer holds
 * len[i] cached positions; with BUDDY_SKIP_MASKED layer l holds
 * layer_len[l * batch + i] <= len[i] (the positions at which it executed).
 * pool_sum[i] = running fp32 sum over the context layer's cached positions of
 * the planner feature (the KV-aware planner's context, Sec. 4.3). */
typedef struct {
  void* const* k_cache;     /* host array [L] of device pointers (config dtype) */
  void* const* v_cache;     /* host array [L] of device pointers */
  const int64_t* seq_off;   /* device [batch] */
  const int32_t* cap;       /* device [batch] */
  int32_t* len;             /* device [batch] */
  float* pool_sum;          /* device [batch, n_kv * hd] */
  int32_t batch;            /* number of sequences the state holds */
  int32_t* layer_len;       /* device [L, batch] with BUDDY_SKIP_MASKED, else NULL */
} buddy_kv_state;

/* Creates a context on the current device; allocates its scratch. */
BUDDY_API int buddy_create(const buddy_config* cfg, buddy_ctx** out);
BUDDY_API void buddy_destroy(buddy_ctx* ctx);

/* Registers the model: layers[0..L-1] and the Decision Module.  Pointers are
 * retained.  Builds the TMA tensor descriptors of the bf16 weight matrices.
 * BUDDY_ERR_ARG for a bf16 context the tensor-core path cannot serve (a
 * device other than sm_103). */
BUDDY_API int buddy_set_weights(buddy_ctx* ctx, const buddy_layer_weights* layers, const buddy_dm_weights* dm);

/* Registers (bp != NULL) or removes (NULL) the Budget Predictor (Sec. 4.4).
 * With one registered, a budget k_i = 0 in buddy_decode_step, buddy_route or
 * buddy_prefill means "no budget given": the sequence executes the
 * predictor's k^ routed blocks.  Pointers are retained.  Allocates the
 * predictor's hidden units (max_batch * hidden fp32). */
BUDDY_API int buddy_set_budget_predictor(buddy_ctx* ctx, const buddy_predictor_weights* bp);

/* Bulk append of n_new given positions to layer `layer` for n_seq sequences
 * (KV cache update, Eq. 9), e.g. to load a prefilled cache.  k_new, v_new:
 * device [n_seq, n_new, n_kv, hd] (config dtype), written at positions
 * p0 .. p0 + n_new - 1 of sequence s = seq_ids[j], p0 = len[s]
 * (BUDDY_SKIP_MASKED: p0 = layer_len[layer][s], which then grows by n_new).
 * For the context layer the pooled context pool_sum[s] is recomputed as the
 * full sum of the planner feature over positions 0 .. p0 + n_new - 1.
 * advance != 0 adds n_new to len[s] afterwards (pass it on the last layer
 * appended).  seq_ids must be distinct.  Device-checked: s < kv->batch,
 * p0 + n_new <= cap[s] and <= max_pos. */
BUDDY_API int buddy_kv_append(buddy_ctx* ctx, const buddy_kv_state* kv, int32_t layer, int32_t n_seq,
                    const int32_t* seq_ids, int32_t n_new, const void* k_new, const void* v_new,
                    int32_t advance, void* stream);

/* The router alone (KV-aware planner + Decision Module + top-k, Sec. 4.2-4.3):
 * for i < batch, pool = pool_sum[i] / len[i] (the cache must already hold the
 * newest token at position len[i]-1), x = [pool expanded; h1[i]],
 * s' as in buddy_dm_weights, selection = the k[i] largest s' (ties to the lower
 * index; k[i] = 0: the Budget Predictor's k^).  h1: device [batch, d] fp32,
 * the newest token's state after block c; k: device [batch] int32 in
 * [1, n_cand] (or 0).  Outputs (device, any may be NULL): sel_out
 * [batch, n_cand] int32 — executed layer ids (c+1..L-2, ascending) then -1;
 * mask_out [batch, L] uint8 (blocks 0..c and the last set); scores_out
 * [batch, n_cand] fp32. */
BUDDY_API int buddy_route(buddy_ctx* ctx, const buddy_kv_state* kv, int32_t batch, const float* h1,
                const int32_t* k, int32_t* sel_out, uint8_t* mask_out, float* scores_out,
                void* stream);

/* Allocation-free router, for callers that cannot allocate device memory and
 * therefore cannot create a buddy_ctx: for example a process whose device
 * memory is all owned by its own pool allocator, or code that runs where
 * cudaMalloc (which may synchronise the device) is not allowed.  The paper
 * has no counterpart; this is a deployment variant of buddy_route.
 *
 * Computes what buddy_route computes for a context with ctx_layer 0 and no
 * Budget Predictor, from explicit arguments instead of a context: shape
 * (n_layers, d_model, n_q_heads, n_kv_heads, head_dim, dm_hidden, same rules
 * as buddy_config), Decision Module `dm` (n_cand = n_layers - 2), and device
 * arrays pool_sum [batch, n_kv*hd], len [batch] (>= 1, the cache already holds
 * the newest token), h1 [batch, d] fp32, k [batch].  Outputs as buddy_route;
 * flags_out (device int32, may be NULL) receives the BUDDY_DEV_* bits of this
 * call (0 when valid; on a nonzero value nothing else was written).
 *
 * Scratch: one static device array of the library (256 KiB of hidden units
 * plus a small header), held by every GPU that loads the library until the
 * process exits.  batch * dm_hidden must not exceed 65536, else
 * BUDDY_ERR_RANGE.  The first call on each device looks up the array's
 * device address (cudaGetSymbolAddress); make that first call outside any
 * stream capture.  The address is cached for the life of the process: after
 * cudaDeviceReset (or anything else that recreates the device's primary
 * context) the library must be reloaded before this entry is called again.
 * All calls share the array: calls whose kernels overlap on the GPU
 * (different streams without ordering) race.  Allocates nothing. */
BUDDY_API int buddy_route_noalloc(int32_t n_layers, int32_t d_model, int32_t n_q_heads,
                                  int32_t n_kv_heads, int32_t head_dim, int32_t dm_hidden,
                                  const buddy_dm_weights* dm, int32_t batch, const float* pool_sum,
                                  const int32_t* len, const float* h1, const int32_t* k,
                                  int32_t* sel_out, uint8_t* mask_out, float* scores_out,
                                  int32_t* flags_out, void* stream);

/* One budget-routed decode step for sequences 0..batch-1 of `kv`.
 * h_in: device [batch, d] fp32 (input of the first block); k: device [batch]
 * int32 budgets in [1, n_cand] (0: predicted); h_out: device [batch, d] fp32,
 * the hidden state after the last block (must not alias h_in).  Optional
 * device outputs (NULL to skip): mask_out [batch, L] uint8; rows_out [L,
 * batch] int32 (for layer l the ascending ids of the sequences that execute
 * it, then unspecified); count_out [L] int32 (their number); scores_out
 * [batch, n_cand] fp32.  Every layer's cache receives one position per
 * sequence (zeros for skipped layers; with BUDDY_SKIP_MASKED only executed
 * layers store one, and layer_len counts them) and len[i] += 1.
 * Device-checked: k[i] in range, len[i] + 1 <= cap[i] and <= max_pos, and
 * with BUDDY_SKIP_MASKED 0 <= layer_len[l][i] <= len[i]; on failure nothing is
 * written. */
BUDDY_API int buddy_decode_step(buddy_ctx* ctx, const buddy_kv_state* kv, int32_t batch, const float* h_in,
                      const int32_t* k, float* h_out, uint8_t* mask_out, int32_t* rows_out,
                      int32_t* count_out, float* scores_out, void* stream);

/* Routed prefill of one prompt per sequence (Sec. 4.1; App. E "Prefill vs.
 * Decode"), bf16 contexts created with max_prefill_tokens > 0.
 * n_tok: HOST [batch] prompt lengths (>= 1, sum <= max_prefill_tokens);
 * x: device [sum n_tok, d] fp32, the prompts' input hidden states, sequence
 * by sequence (rows off_i .. off_i + n_tok[i] - 1 for sequence i, off_i the
 * sum of the earlier lengths); k: device [batch] budgets as in
 * buddy_decode_step; h_out: device [sum n_tok, d] fp32, every token's hidden
 * state after the last block (must not alias x).  Optional device outputs:
 * mask_out [batch, L] uint8, scores_out [batch, n_cand] fp32.
 * Sequence i's tokens take positions len[i] .. len[i] + n_tok[i] - 1.  Blocks
 * 0..c run on every token with causal attention; each sequence is routed once
 * from its pooled context-layer cache (prompt included) and its last token's
 * state after block c; each routed block runs on all tokens of the sequences
 * that selected it; a skipped block stores zero K/V at every prompt position
 * (BUDDY_SKIP_MASKED: nothing).  Then len[i] += n_tok[i].  The call
 * synchronises `stream` once, after the routing, to size the later launches;
 * it returns BUDDY_ERR_DEVICE (nothing written) when the device checks of
 * buddy_decode_step fail (budgets, len[i] + n_tok[i] <= cap[i], <= max_pos). */
BUDDY_API int buddy_prefill(buddy_ctx* ctx, const buddy_kv_state* kv, int32_t batch, const int32_t* n_tok,
                            const float* x, const int32_t* k, float* h_out, uint8_t* mask_out,
                            float* scores_out, void* stream);

/* buddy_decode_step with HOST buffers: h_in_host [batch, d] fp32, k_host
 * [batch] int32, h_out_host [batch, d] fp32, mask_host [batch, L] uint8 (or
 * NULL).  Copies the inputs to device staging buffers, runs the step, copies
 * the outputs back and synchronises the stream before returning.  Pinned host
 * memory gives asynchronous copies; pageable memory works but is slower. */
BUDDY_API int buddy_decode_step_host(buddy_ctx* ctx, const buddy_kv_state* kv, int32_t batch,
                           const float* h_in_host, const int32_t* k_host, float* h_out_host,
                           uint8_t* mask_host, void* stream);

/* Execution options.  use_graph != 0: buddy_decode_step replays a CUDA graph
 * of the step's launches, captured per (batch, kv state, stream) on first use;
 * the kernels of a layer that no sequence selected exit as soon as they start.
 * The graph bakes in the pointers of that call; a call with other pointers
 * re-captures. */
BUDDY_API int buddy_set_options(buddy_ctx* ctx, int32_t use_graph);

/* Which kernels a context runs (valid after buddy_set_weights), so that a
 * measurement can state them: paths[0] GEMM (0 CUDA-core fp32, 1 tcgen05
 * bf16), paths[1] attention (0 CUDA-core, 1 mma.sync tensor-core loop over
 * the whole GPU, 2 the same contractions with one thread-block cluster per
 * (row, KV head) stream, for small batches),
 * paths[2] RMSNorm computed inside the QKV and gate/up GEMMs (0/1; fp32: by
 * the rows of each call, here for max_batch rows),
 * paths[3] split-K sums in a separate fixup kernel (0/1).  n <= 4 entries. */
BUDDY_API int buddy_get_paths(buddy_ctx* ctx, int32_t* paths, int32_t n);

/* Limit of every bounded wait inside the tensor-core GEMM pipelines (TMA
 * stages, MMA completion, accumulator hand-over), in nanoseconds; ns <= 0
 * restores the default of 4 s.  A wait that runs out makes its kernel stop
 * (after its copies and MMAs in flight have completed), raise
 * BUDDY_DEV_TIMEOUT and leave its outputs incomplete; buddy_device_status
 * then reports the bit and re-arms the kernels' arrival counters, so the
 * context stays usable.  Synchronises the device; drops captured graphs. */
BUDDY_API int buddy_set_wait_limit(buddy_ctx* ctx, int64_t ns);

/* Kernel classes reported by the profiler. */
enum {
  BUDDY_PROF_CHECK = 0, BUDDY_PROF_RMSNORM, BUDDY_PROF_GEMM_QKV, BUDDY_PROF_QKV_FINALIZE,
  BUDDY_PROF_ATTENTION, BUDDY_PROF_GEMM_O, BUDDY_PROF_GEMM_GATE_UP, BUDDY_PROF_GEMM_DOWN,
  BUDDY_PROF_ROUTE, BUDDY_PROF_COMPACT, BUDDY_PROF_OTHER,
  BUDDY_PROF_GEMM_FIXUP,   /* split-K sums + epilogues of the GEMMs (larger batches) */
  BUDDY_PROF_PF_GEMM,      /* prefill: projections (tcgen05, M-tiled) */
  BUDDY_PROF_PF_ATTENTION, /* prefill: causal attention */
  BUDDY_PROF_PF_OTHER,     /* prefill: RMSNorm, zero fill, advance */
  BUDDY_PROF_NCLASS
};

/* Per-kernel-class timing.  With on != 0, direct-launch decode steps
 * (use_graph == 0) record a CUDA event pair on the launching stream around
 * every kernel launch, and count the launches.  buddy_profile_read
 * synchronises those events, writes per class the summed milliseconds and the
 * launch count (arrays of n_cls entries, n_cls <= BUDDY_PROF_NCLASS), and
 * clears the records.  buddy_profile_class_name gives a class's name. */
BUDDY_API int buddy_set_profiling(buddy_ctx* ctx, int32_t on);
BUDDY_API int buddy_profile_read(buddy_ctx* ctx, int32_t n_cls, float* ms, int32_t* launches);
BUDDY_API const char* buddy_profile_class_name(int32_t cls);

/* Synchronises `stream`, stores the device error flag bits (BUDDY_DEV_*) in
 * *flags and clears them.  Returns BUDDY_ERR_DEVICE if any bit was set. */
BUDDY_API int buddy_device_status(buddy_ctx* ctx, void* stream, int32_t* flags);

/* Budget b in (0, 1] to middle-layer count: k = round(b * L) - 2 (Eq. 2,
 * ties to even), clamped to the action space [1, L-2] (Sec. 4.4).
 * Returns -1 if n_layers < 3 or b is not finite. */
BUDDY_API int32_t buddy_budget_to_k(float b, int32_t n_layers);

/* ---------------------------------------------------------------------------
 * Paged KV cache in 4 bits.  The paper has no counterpart; it is the cache of
 * deployments whose batches are bound by the bytes of keys and values, or whose
 * sequences (and the blocks that skip them) grow at different rates.  The
 * entries below need no context and allocate nothing.
 *
 * One layer's cache is n_pages pages of page_size positions for the keys and as
 * many for the values.  A page holds one block per KV head; block (page p, head
 * g) starts at byte (p * n_kv_heads + g) * page_size * (hd/2 + hd/16) and holds
 *   codes   [page_size][hd/2]   4 bits per channel,
 *   scales  [page_size][hd/32]  IEEE half, one per 32 channels.
 * Channels 8w .. 8w + 7 are the 32-bit little-endian word w of the position's
 * codes: bits 4j .. 4j + 3 hold channel 8w + 2j (j < 4) or 8w + 2(j - 4) + 1
 * (j >= 4).  The value of a channel is (code - 8) * scale, code 1 .. 15.
 *
 * An entry x of 32 channels is stored with
 *   scale = max|x| / 7 rounded to 7 significant bits (ties to even), then to
 *           half, at most 896,
 *   code  = 8 + x / scale rounded to the nearest integer (ties to even), kept in
 *           [-7, 7]; 8 where the scale is 0.
 * A NaN among the 32 makes the scale NaN, and so the 32 values; an infinite
 * channel takes the largest value of the largest scale (6272).
 *
 * Position p of a sequence is at slot table[p / page_size] * page_size +
 * p % page_size.  Pages belong to one sequence each.  What a cache holds behind
 * a sequence's last position may be anything.
 *
 * `flags` of the entries below: device int32, or NULL.  A kernel that meets a
 * bad value in device memory sets its BUDDY_DEV_* bit there and leaves out what
 * the entry says; nothing clears the word.  (BUDDY_DEV_TIMEOUT: a wait of an
 * attention kernel has run out after 4 s; its outputs are incomplete.)
 *
 * Launches of the entries below may begin while the work before them on their
 * stream ends; they read and write memory only after it. */
typedef struct {
  void* k_pages;        /* device, n_pages * n_kv_heads blocks; 16-byte aligned */
  void* v_pages;        /* device, as k_pages */
  int32_t n_pages;      /* >= 1 */
  int32_t page_size;    /* positions of a page: 16, 32, 64 or 128 */
  int32_t n_kv_heads;   /* 1 .. 1024 */
  int32_t head_dim;     /* 64 or 128 */
} buddy_kv4_cache;

/* Block tables and slot maps from request lengths.  Sequence i holds len[i]
 * positions in the first ceil(len[i] / page_size) pages of its table row and is
 * to take n_new[i] >= 0 more (len[i] = 0: a request that starts).  The pages it
 * lacks come from free_pages, in order, from index *free_head on: first those of
 * sequence 0, then of sequence 1, ...
 * Written: those table entries (others are left as they are); kv_len[i] = len[i]
 * + n_new[i]; row_start[i] = new tokens before sequence i, row_start[batch] =
 * their number; for token t of the call its slot and its position; -1 for both
 * behind the last token, up to n_tok; *free_head_out = the index after the last
 * page taken.  What is written (`table` among it) overlaps neither an input nor
 * anything else that is written (else BUDDY_ERR_ARG).
 * Device-checked: lengths >= 0, len[i] + n_new[i] <= max_pages * page_size, at
 * most n_tok new tokens (BUDDY_DEV_BAD_POSITION); 0 <= *free_head and as many free
 * pages left as the call needs (BUDDY_DEV_NO_PAGES); on failure nothing is
 * written. */
typedef struct {
  int32_t batch;              /* 1 .. 16384 */
  int32_t page_size;          /* a power of two, 1 .. 65536 */
  int32_t max_pages;          /* entries of a table row */
  int32_t n_free;             /* entries of free_pages */
  int32_t n_tok;              /* entries of slot and pos */
  const int32_t* len;         /* device [batch] */
  const int32_t* n_new;       /* device [batch] */
  int32_t* table;             /* device [batch, max_pages] page ids */
  const int32_t* free_pages;  /* device [n_free] page ids (may be NULL when n_free is 0) */
  const int32_t* free_head;   /* device */
  int32_t* kv_len;            /* device [batch] */
  int32_t* row_start;         /* device [batch + 1] */
  int64_t* slot;              /* device [n_tok] (may be NULL when n_tok is 0) */
  int32_t* pos;               /* device [n_tok], as slot */
  int32_t* free_head_out;     /* device */
} buddy_page_plan_args;
BUDDY_API int buddy_page_plan(const buddy_page_plan_args* args, int32_t* flags, void* stream);

/* Rotary tables: cos and sin of p * theta^(-2j / head_dim), device [max_pos,
 * head_dim / 2] each, evaluated in double and stored fp32. */
BUDDY_API int buddy_rope_table(float* rope_cos, float* rope_sin, int32_t max_pos, int32_t head_dim,
                               float rope_theta, void* stream);

/* Query and key heads of n_tok tokens.  Head h of token t is head_dim
 * consecutive elements from element t * stride + h * head_dim on.  All rows
 * 16-byte aligned: pointers, and strides in bytes. */
typedef struct {
  int32_t n_tok;         /* >= 0 */
  int32_t n_q_heads;     /* >= 0 (0: no queries; q, q_out unused) */
  int32_t n_kv_heads;    /* >= 1 */
  int32_t head_dim;      /* 64 or 128 */
  int32_t dtype;         /* BUDDY_DTYPE_F32 or _BF16: q, k, v and the outputs */
  int32_t max_pos;       /* rows of the rotary tables */
  float eps;             /* of the norms, > 0 */
  const void* q;         /* device */
  const void* k;         /* device */
  int64_t q_stride;      /* elements from token to token */
  int64_t k_stride;
  const float* q_gain;   /* device [head_dim], or NULL: no norm of the queries */
  const float* k_gain;   /* device [head_dim], or NULL: no norm of the keys */
  const int32_t* pos;    /* device [n_tok] positions; negative: the token is left out */
  const float* rope_cos; /* device [max_pos, head_dim / 2] */
  const float* rope_sin;
  void* q_out;           /* device; may be q with q's stride */
  void* k_out;           /* device; may be k with k's stride */
  int64_t q_out_stride;
  int64_t k_out_stride;
} buddy_qk_rows;

/* The norm of every query and key head and its rotation, in one pass:
 *   y = x / sqrt(mean(x^2) + eps) * gain,
 *   out[j] = y[j] cos_j - y[j + hd/2] sin_j,  out[j + hd/2] = y[j + hd/2] cos_j + y[j] sin_j,
 * in fp32, rounded once.  The sum of squares is taken in a fixed order (halves
 * onto each other inside eight neighbours, then over the eights), without fused
 * multiply-adds, so that equal inputs give equal bits in any batch.
 * Device-checked: pos[t] < max_pos (BUDDY_DEV_BAD_POSITION; the token's outputs
 * are left as they were, as for a negative position, which sets no bit). */
BUDDY_API int buddy_qk_norm_rope(const buddy_qk_rows* rows, int32_t* flags, void* stream);

/* The same for a block that keeps its entries in a 4-bit cache: queries to
 * q_out; keys, normalised and rotated, and values v (device, rows as k's with
 * stride v_stride) into the cache at slot[t]; keys also to rows->k_out unless
 * that is NULL.  Keys are quantised from their fp32 values.  A token with a
 * negative slot stores no entry (its queries are written).  The slots of a call
 * must be distinct.  Device-checked: positions as above (the token is left out
 * as a whole); slot[t] < n_pages * page_size (BUDDY_DEV_BAD_PAGE; no entry is
 * stored). */
BUDDY_API int buddy_kv4_append(const buddy_kv4_cache* cache, const buddy_qk_rows* rows, const void* v,
                               int64_t v_stride, const int64_t* slot, int32_t* flags, void* stream);

/* Both with several position axes (time, height and width of a video's patches; text
 * has the same position on every axis).  Frequency j, the pair of channels j and
 * j + hd/2, turns by the tables' row of axis axis[j]'s position: row pos[a] for a =
 * axis[j], where axis a's positions are rows->pos[a * pos_stride + t], t < n_tok.
 * Everything else is as above; a token that is negative on any axis is left out, one
 * with a position >= max_pos on any axis too (BUDDY_DEV_BAD_POSITION). */
typedef struct {
  int32_t n_axes;        /* 1 .. 4 */
  uint8_t axis[64];      /* of frequency j < head_dim / 2; each < n_axes */
  int64_t pos_stride;    /* elements from axis to axis of rows->pos, >= 0 */
} buddy_rope_axes;
BUDDY_API int buddy_qk_norm_rope_axes(const buddy_qk_rows* rows, const buddy_rope_axes* axes, int32_t* flags,
                                      void* stream);
BUDDY_API int buddy_kv4_append_axes(const buddy_kv4_cache* cache, const buddy_qk_rows* rows,
                                    const buddy_rope_axes* axes, const void* v, int64_t v_stride,
                                    const int64_t* slot, int32_t* flags, void* stream);

/* The values that the cache holds at n slots: k_out, v_out device [n,
 * n_kv_heads, head_dim] of dtype BUDDY_DTYPE_F32 or _F16 (both exact) or _BF16
 * (rounded), 16-byte aligned; either may be NULL.  Rows of negative slots are
 * left as they were, and those of slots past the last page (BUDDY_DEV_BAD_PAGE). */
BUDDY_API int buddy_kv4_read(const buddy_kv4_cache* cache, int32_t n, const int64_t* slot, int32_t dtype,
                             void* k_out, void* v_out, int32_t* flags, void* stream);

/* Causal attention over a 4-bit cache.  Sequence i's query tokens are rows
 * row_start[i] .. row_start[i + 1] - 1 of q, and the last of them is the
 * sequence's position kv_len[i] - 1 (the entries of the tokens are in the cache
 * already: append first).  Query head h reads KV head h / (n_q_heads /
 * n_kv_heads).  A token's output is
 *   sum_p softmax_p(scale * q . k_p) v_p   over positions 0 .. its own;
 * a token without any position (kv_len[i] = 0, or more query tokens than
 * positions) gets zeros.  Rows of q behind row_start[batch] are not written.
 * Query elements enter the products as halves, scaled by a power of two per row
 * where that is needed: 11 significant bits (a bf16 element whole), fewer for the
 * smallest of a row, which are rounded at 2^-25 of its largest element, or at 2^-25
 * where that is in 2^-14 .. 2^15.  Probabilities enter with 11 bits, below 2^-21 of the
 * row's largest rounded at 2^-32 of that; keys and values exactly; sums and
 * statistics are fp32.  With fp32 queries or fp32 outputs both enter as the sum of
 * two halves, with 22 bits (queries rounded at 2^-39 of the row's largest element
 * or less).
 * Device-checked: 0 <= kv_len[i] <= max_pages * page_size and row_start
 * ascending from >= 0 to <= n_tok with at most max_new rows each
 * (BUDDY_DEV_BAD_POSITION: the sequence's rows are not written); page ids
 * (BUDDY_DEV_BAD_PAGE: the page's positions count as not there). */
typedef struct {
  int32_t batch;              /* 1 .. 16384 */
  int32_t n_tok;              /* rows of q and out; n_tok * n_q_heads < 2^31 - 512 (else BUDDY_ERR_RANGE) */
  int32_t max_new;            /* >= 1: most query tokens of one sequence */
  int32_t n_q_heads;          /* a multiple of n_kv_heads, at most 8 times */
  int32_t q_dtype;            /* BUDDY_DTYPE_F32 or _BF16 */
  int32_t out_dtype;          /* BUDDY_DTYPE_F32 or _BF16 */
  int32_t max_pages;          /* entries of a table row, max_pages * page_size < 2^31 */
  float scale;                /* of the scores, 0 .. 2.3e38; 0: 1 / sqrt(head_dim) */
  const void* q;              /* device [n_tok, n_q_heads, head_dim], tokens q_stride elements apart */
  void* out;                  /* device, as q with out_stride; must not overlap q */
  int64_t q_stride;           /* rows 16-byte aligned */
  int64_t out_stride;
  const int32_t* row_start;   /* device [batch + 1]; NULL: one token per sequence (n_tok == batch) */
  const int32_t* kv_len;      /* device [batch], the query tokens' own positions among them */
  const int32_t* table;       /* device [batch, max_pages] */
  void* workspace;            /* device, 256-byte aligned */
  int64_t workspace_bytes;    /* at least buddy_kv4_attention_workspace() */
} buddy_kv4_attention_args;
BUDDY_API int buddy_kv4_attention(const buddy_kv4_cache* cache, const buddy_kv4_attention_args* args,
                                  int32_t* flags, void* stream);

/* Bytes of workspace that any buddy_kv4_attention call with these sizes takes on
 * the current device; -1 for sizes that it rejects.  The caller zeroes it once;
 * every call leaves it ready for the next.  Calls that may overlap on the GPU
 * need workspaces of their own. */
BUDDY_API int64_t buddy_kv4_attention_workspace(int32_t n_q_heads, int32_t n_kv_heads, int32_t head_dim,
                                                int32_t max_new);

/* ---------------------------------------------------------------------------
 * Attention over the pages that a score selects for each query: for contexts so
 * long that reading all of them for every token costs too much.  After an append,
 *   buddy_kv4_bounds            bounds of the keys of the pages that it wrote to,
 *   buddy_kv4_select            each query's best pages by those bounds,
 *   buddy_kv4_attention_pages   attention over them.
 *
 * Sequences of a call, as in buddy_kv4_attention: tokens row_start[i] ..
 * row_start[i + 1] - 1 are the last positions of sequence i's kv_len[i]. */
typedef struct {
  int32_t batch;              /* 1 .. 16384 */
  int32_t n_tok;              /* rows of the call */
  int32_t max_new;            /* >= 1: most tokens of one sequence */
  int32_t max_pages;          /* entries of a table row, max_pages * page_size < 2^31 */
  const int32_t* row_start;   /* device [batch + 1]; NULL: one token per sequence (n_tok == batch) */
  const int32_t* kv_len;      /* device [batch], the call's tokens among them */
  const int32_t* table;       /* device [batch, max_pages] */
} buddy_kv4_seqs;

/* Bounds of the keys: device half [n_pages, n_kv_heads, 2, head_dim], 16-byte
 * aligned: of each page, KV head and channel the smallest of the stored keys, then
 * the largest; exact, and NaN where one of them is.  Written are those of the pages
 * that the call's tokens lie in, from everything these pages hold up to kv_len[i]
 * (so the bounds of a sequence with as many tokens as positions are made anew; a
 * call may be repeated); others are left as they were.
 * Device-checked: lengths and row starts as in buddy_kv4_attention
 * (BUDDY_DEV_BAD_POSITION: the sequence is left out); page ids (BUDDY_DEV_BAD_PAGE:
 * the page is). */
BUDDY_API int buddy_kv4_bounds(const buddy_kv4_cache* cache, const buddy_kv4_seqs* seqs, void* bounds,
                               int32_t* flags, void* stream);

/* Of each query token and KV head at most `budget` pages.  A token at position p has
 * pages 0 .. p / page_size.  Where they are `budget` or fewer, all are selected;
 * else the `first` first ones, the `last` last ones (its own the last of them), and
 * of the others those with the highest scores, ties to the lower position:
 *   score = sum_c a_c hi_c + sum_c b_c lo_c,
 *   a_c = sum_h max(q_hc, 0), b_c = sum_h min(q_hc, 0),
 * over the query heads h of the KV head and the page's bounds: the sum over these
 * heads of a bound of q . k over the page.  A NaN counts as the highest score, a page
 * that is not there (BUDDY_DEV_BAD_PAGE) as the lowest.  fp32, every product and sum
 * rounded by itself, in this order: over h from the first head on; the products over
 * c halves onto each other inside eight neighbours, then so over the eights; then the
 * sum over hi plus that over lo.
 * Written for each token t: to pages[t][g] the page ids, in the order of their
 * positions, -1 behind them; to visible[t] how many positions they hold up to the
 * token (all pages but the last are whole), the same for every KV head: 0 for a
 * token without any position, -1, with its pages left as they were, for one that is
 * in no sequence, or in one whose length or row starts are bad
 * (BUDDY_DEV_BAD_POSITION, also for a sequence without tokens). What is written
 * overlaps no input. */
typedef struct {
  buddy_kv4_seqs s;           /* max_pages <= 40000 (else BUDDY_ERR_RANGE) */
  int32_t n_q_heads;          /* a multiple of n_kv_heads, at most 8 times */
  int32_t q_dtype;            /* BUDDY_DTYPE_F32 or _BF16 */
  int32_t budget;             /* >= first + last */
  int32_t first;              /* >= 0 */
  int32_t last;               /* >= 1 */
  const void* q;              /* device [n_tok, n_q_heads, head_dim], tokens q_stride elements apart */
  int64_t q_stride;           /* rows 16-byte aligned */
  const void* bounds;         /* device, of buddy_kv4_bounds */
  int32_t* pages;             /* device [n_tok, n_kv_heads, budget] */
  int32_t* visible;           /* device [n_tok] */
} buddy_kv4_select_args;
BUDDY_API int buddy_kv4_select(const buddy_kv4_cache* cache, const buddy_kv4_select_args* args, int32_t* flags,
                               void* stream);

/* buddy_kv4_attention of single tokens, each KV head over pages of its own: batch ==
 * n_tok, 0 .. 16384 tokens, max_new 1, row_start NULL; table is device [n_tok,
 * n_kv_heads, max_pages], kv_len[t] the positions of token t's lists that it sees
 * (the first kv_len[t] in the order of the lists).  A token with none gets zeros, one
 * with a negative number is left as it was.  Numerics, workspace
 * (buddy_kv4_attention_workspace with max_new 1) and device checks as above. */
BUDDY_API int buddy_kv4_attention_pages(const buddy_kv4_cache* cache, const buddy_kv4_attention_args* args,
                                        int32_t* flags, void* stream);

BUDDY_API const char* buddy_error_string(int32_t code);
BUDDY_API int32_t buddy_version(void);

#ifdef __cplusplus
}
#endif

#endif /* BUDDY_H_ */
