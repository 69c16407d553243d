/*
 * tlf.h - C ABI of libtlf: routed prefill and decode of a looped, weight-shared
 * transformer with token-level depth and a recursion-wise KV cache
 * (T-LoopFormer, Section 3.2 and Section 3.3), for AMD Instinct MI355X (gfx950).
 *
 * Model
 *   h0 = E[x] + P[pos] (token plus learned absolute position, added once;
 *   Section 3 and Section 3.2).  A router maps h0 to R logits (Eq. 2) and a
 *   depth rule turns them into the token's loop count m in [1, R] (Eq. 3-5, or
 *   argmax, or a fixed depth).  Loop i (1..R) applies the shared block of J
 *   pre-norm layers (RMSNorm without affine, multi-head attention, SwiGLU FFN,
 *   residuals inside each layer; Appendix A) to the tokens with m >= i only
 *   (gather, Eq. 6; scatter, Eq. 7).  Exited tokens keep h^(m).  Logits are
 *   RMSNorm(h^(m)) times the LM head (tied to E unless a head is given).
 *
 * Recursion-wise KV cache (Eq. 8-11)
 *   Every (sequence b, loop i) owns its own cache, shared by the J layers'
 *   K/V planes.  A token that executes loop i writes its k, v there (Eq. 11);
 *   a query at loop i attends only to the entries of that cache (Eq. 10): the
 *   earlier tokens of the sequence whose depth is >= i, and itself.  Entries
 *   are stored compactly in position order in 16-token pages, with the
 *   original position of every entry recorded; tokens that never reached loop
 *   i occupy no slot, so the validity mask of Eq. 10 is implicit.
 *
 * Conventions
 *   - Every function returns an int status (TLF_OK or a negative TLF_E_*
 *     code); no C++ exception crosses this boundary.
 *   - Device pointers ("d_") are HIP device memory on the device that is
 *     current when tlf_init is called.  Host pointers ("h_") are host memory.
 *   - Weights and the workspace are borrowed: the caller keeps them alive and
 *     unchanged until tlf_destroy.  Outputs are caller-allocated.  The context
 *     owns only host-side state.  tlf_init also writes a copy of every
 *     layer's block weights into the workspace, reordered for the decode
 *     projections' matrix-core loads (counted in the workspace size).
 *   - Work is enqueued asynchronously on the stream given to tlf_init; only
 *     tlf_cache_stats waits for the stream.  A context is not thread-safe.
 *   - Arguments are validated on the host before any device work; an argument
 *     error (TLF_E_INVALID_ARG, TLF_E_STATE) leaves the context unchanged.
 *   - A HIP error (TLF_E_HIP) poisons the context: later calls return
 *     TLF_E_STATE.  Errors found on the device (a token id out of range, the
 *     page pool exhausted) are sticky and are returned by tlf_cache_stats and
 *     by every call after it.
 */
#ifndef TLF_H
#define TLF_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

#define TLF_ABI_VERSION 5
#define TLF_MAX_LOOPS 16
#define TLF_MAX_LAYERS 8
#define TLF_MAX_BATCH 4096
#define TLF_PAGE_TOKENS 16

/* Status codes. */
#define TLF_OK 0
#define TLF_E_INVALID_ARG (-1)    /* bad argument: no valid model, call or buffer */
#define TLF_E_NEED_WORKSPACE (-2) /* tlf_init size query: *ws_needed is set */
#define TLF_E_OUT_OF_PAGES (-3)   /* the KV page pool (max_pages) is exhausted */
#define TLF_E_STATE (-4)          /* call not valid in this state (e.g. decode before prefill) */
#define TLF_E_HIP (-5)            /* a HIP runtime call failed; the context is poisoned */
#define TLF_E_DEVICE (-6)         /* the device found a bad input (token id out of range) */
#define TLF_E_UNSUPPORTED (-7)    /* a valid config outside this build's shapes and sizes (tlf_init) */

/* Storage dtype of embeddings, block weights and the KV cache.  The residual
 * stream, the activations passed between kernels (normalised rows, q,
 * attention output, SwiGLU output), router, softmax, accumulators and logits
 * are float32 in both cases; with bf16 weights each float32 activation enters
 * a matrix product as the sum of two bf16 parts (hi + lo), so only the weights,
 * the cached k and v, and the attention probabilities are rounded to bf16. */
#define TLF_DTYPE_F32 0
#define TLF_DTYPE_BF16 1

/* Depth rules (Section 3.2). */
#define TLF_ROUTE_ARGMAX 0  /* m = 1 + index of the largest router logit (lowest on ties) */
#define TLF_ROUTE_CUMPROB 1 /* m = max{i : sum_{l>=i} softmax(z)_l > threshold} (Eq. 2-5) */
#define TLF_ROUTE_FIXED 2   /* m = fixed_depth for every token (fixed-depth looped model) */

/* tlf_prefill flags. */
#define TLF_PREFILL_ALL_LOGITS 1u /* logits for every position ([B][T][V]) instead of the last */
#define TLF_PREFILL_APPEND 2u     /* continue the current batch: the tokens are its next positions */

typedef struct tlf_config {
  int32_t abi_version;   /* must be TLF_ABI_VERSION */
  int32_t dtype;         /* TLF_DTYPE_F32 or TLF_DTYPE_BF16 */
  int32_t vocab;         /* V >= 1 */
  int32_t d_model;       /* d <= 4096, multiple of 128 (bf16) or 64 (float32) */
  int32_t n_heads;       /* H, n_heads * head_dim == d_model */
  int32_t head_dim;      /* D: 64 or 128 (16 for float32 models only) */
  int32_t d_ff;          /* F, SwiGLU hidden width, multiple of 128 (bf16) or 64 (float32) */
  int32_t n_layers;      /* J in [1, TLF_MAX_LAYERS], layers of the shared block */
  int32_t max_loops;     /* R = M in [1, TLF_MAX_LOOPS], router width and loop cap */
  int32_t max_pos;       /* rows of the position table, <= 65536; prompt + decode steps <= max_pos */
  int32_t max_batch;     /* sequences per call, in [1, TLF_MAX_BATCH] */
  int32_t page_tokens;   /* tokens per KV page, must be TLF_PAGE_TOKENS */
  int32_t max_pages;     /* KV pages in the pool (all sequences and loops) */
  int32_t max_prefill_tokens; /* activation rows for prefill; larger prefills run in sequence groups */
  int32_t route_rule;    /* TLF_ROUTE_* */
  float route_threshold; /* CUMPROB threshold in (0, 1); the paper uses 0.5 */
  int32_t fixed_depth;   /* FIXED depth in [1, R] */
  float rms_eps;         /* RMSNorm epsilon (> 0) */
  int32_t decode_graph;  /* 1: each decode step replays a captured HIP graph; a graph belongs to
                            the batch and the step's token and output pointers, the graphs of
                            the last 4 distinct ones are kept (a step whose tokens are the
                            previous step's next_tokens alternates between two) and a new one
                            is captured in place of the least recently used;
                            0: kernels are launched one by one */
  int32_t router_hidden; /* 0: linear router z = W_r h0 + b_r; Hr > 0 (<= 4096, multiple of 64): the
                            two-layer MLP router z = W_r silu(W_1 h0 + b_1) + b_r (Section 3.2) */
  int32_t dense_decode;  /* 0: each decode loop runs on the gathered active rows (Eq. 6-7);
                            1: gather-scatter off (the ablation of Section 4's latency study):
                            every loop up to the step's deepest token runs on all rows of the
                            batch, exited rows are computed and discarded at the scatter and
                            write no cache entry, attention keeps the validity mask of Eq. 10.
                            Same results as 0; prefill is not affected */
  int32_t adaln;         /* 0: unconditioned block; 1: AdaLN time/step conditioning (Section 3.1,
                            Appendix A; weights in tlf_weights.adaln): a token of depth m at
                            loop i has cumulative time (i-1)/m and step 1/m, and layer j's
                            modulation (alpha_msa, alpha_mlp, gamma_msa, gamma_mlp) enters as
                            x += (1 + alpha) * F(RMSNorm(x) * (1 + gamma)) */
  int32_t prefill_act_bf16; /* bf16 models: 0: the float32 activations enter the block's matrix
                               products and the attention scores of a prefill as bf16 hi + lo parts;
                               1: as one bf16 part (round to nearest even), half the matrix-core
                               work.  Two parts whatever this says: decode steps, every LM head, and
                               a prefill group (the sequences that fit max_prefill_tokens together)
                               of one sequence of at most 2048 tokens or of at most 256 x 768 row
                               elements (tokens x d_model).  An exact bf16 implementation with
                               every activation rounded stays within 1.9e-2 of float64 on the
                               logits at d_model 1024 but reaches 4.1e-2 at 2048 */
} tlf_config;

/* Weights of layer j of the shared block, row-major [out][in] (y = x W^T),
 * in the storage dtype. */
typedef struct tlf_layer_weights {
  const void* w_qkv;     /* [3d][d]: rows q | k | v, each head-major (head h = rows h*D..h*D+D-1) */
  const void* w_o;       /* [d][d] */
  const void* w_gate_up; /* [2F][d]: rows gate | up; FFN(y) = W_down (silu(W_gate y) * (W_up y)) */
  const void* w_down;    /* [d][F] */
} tlf_layer_weights;

/* AdaLN conditioning weights (config.adaln = 1), row-major [out][in]:
 * matrices in the storage dtype, biases float32.  Each conditioning scalar
 * s becomes 256 Fourier features [cos(s w_1), sin(s w_1), ..., cos(s w_128),
 * sin(s w_128)], w_k = 10000^(-(k-1)/128), then phi(s) = W_2 silu(W_1 f + b_1)
 * + b_2; the embedding is phi_time(c) + phi_step(Delta), and layer j's
 * modulation is mod_w[j] silu(embedding) + mod_b[j].  Read by tlf_init only:
 * the modulation of every (layer, loop, depth) is tabulated there. */
typedef struct tlf_adaln_weights {
  const void* time_w1;  /* [d][256] */
  const float* time_b1; /* [d] */
  const void* time_w2;  /* [d][d] */
  const float* time_b2; /* [d] */
  const void* step_w1;  /* [d][256] */
  const float* step_b1; /* [d] */
  const void* step_w2;  /* [d][d] */
  const float* step_b2; /* [d] */
  const void* const* mod_w;  /* host array of n_layers device pointers: [4d][d], output rows
                                alpha_msa | alpha_mlp | gamma_msa | gamma_mlp */
  const float* const* mod_b; /* host array of n_layers device pointers: [4d] */
} tlf_adaln_weights;

typedef struct tlf_weights {
  const void* tok_emb;      /* [V][d] storage dtype; also the LM head when lm_head is NULL */
  const void* pos_emb;      /* [max_pos][d] storage dtype */
  const float* router_w;    /* [R][d] float32 ([R][Hr], the output layer, for an MLP router) */
  const float* router_b;    /* [R] float32 */
  const void* lm_head;      /* [V][d] storage dtype, or NULL for a head tied to tok_emb */
  int32_t n_layers;         /* must equal config.n_layers */
  const tlf_layer_weights* layers; /* host array of n_layers entries (copied by tlf_init) */
  const void* router_w1;    /* MLP router hidden layer [Hr][d] storage dtype; NULL for a linear router */
  const float* router_b1;   /* [Hr] float32; NULL for a linear router */
  const tlf_adaln_weights* adaln; /* host pointer; required when config.adaln = 1, else NULL */
} tlf_weights;

typedef struct tlf_cache_stats_t {
  int64_t slots_per_loop[TLF_MAX_LOOPS];  /* sum over sequences of cache entries of loop i */
  int64_t pages_per_loop[TLF_MAX_LOOPS];  /* pages held by loop i's caches */
  int64_t depth_hist[TLF_MAX_LOOPS];      /* routed depth counts of every token seen (index m-1) */
  int64_t pages_used;                     /* pages in use (free pages: pages_total - pages_used) */
  int64_t pages_total;
  int64_t kv_bytes_resident;              /* pages_used * bytes per page */
  int64_t batch;                          /* sequences in the current batch */
  int64_t seq_len;                        /* tokens per sequence so far */
  /* Algorithmic bytes of the last decode step (exact, from the step's depths):
   * kv_read counts only valid entries (cache entries plus the step's own);
   * kv_write the appended k, v; weight bytes count the shared block once per
   * executed loop plus the LM head and router. */
  int64_t last_step_kv_read_bytes;
  int64_t last_step_kv_write_bytes;
  int64_t last_step_weight_bytes;
  int64_t last_step_loops_executed;       /* #{i : some token of the step has m >= i} */
  int64_t last_step_active_rows[TLF_MAX_LOOPS]; /* rows run at loop i in the last step: n_i = #{b : m_b >= i}
                                                   (dense_decode: the batch, up to the deepest loop) */
  /* Totals since profiling was last enabled (tlf_set_profiling): */
  int64_t decode_steps;                   /* decode steps enqueued */
  int64_t attn_launches;                  /* decode-attention launches timed */
  int64_t attn_algo_bytes;                /* their algorithmic bytes: valid K/V entries read, q read, o written */
  double attn_ms;                         /* their summed duration (HIP events on the context's stream) */
  int64_t kv_write_bytes_total;           /* bytes of appended k, v */
  int64_t loops_executed_total;           /* shared-block applications (each streams the block weights once) */
  double block_ms;                        /* summed duration of the loop-and-layer region of each step */
  int32_t device_error;                   /* sticky device-side status (TLF_OK if none) */
  int32_t reserved;
} tlf_cache_stats_t;

typedef struct tlf_ctx tlf_ctx;

/* Create a context (Section 3.3 inference state).
 *   cfg, w:       model description; w's device pointers are borrowed.
 *   d_workspace:  device memory for the KV page pool, page tables, positions,
 *                 activations and split-K partials; NULL to query the size.
 *   ws_bytes:     size of d_workspace.
 *   ws_needed:    out (may be NULL unless d_workspace is NULL): bytes needed.
 *   hip_stream:   hipStream_t on which all work is enqueued (NULL = default).
 *   out:          receives the context.
 * Returns TLF_E_NEED_WORKSPACE (with *ws_needed set) when d_workspace is NULL
 * or ws_bytes is too small, TLF_E_INVALID_ARG on a bad config or weight set,
 * TLF_E_UNSUPPORTED on a valid config outside the shapes and sizes listed in
 * tlf_config (head_dim, the multiples of d_model and d_ff, the TLF_MAX_* limits,
 * router_hidden, max_pos and the 32-bit offset limits). */
int tlf_init(const tlf_config* cfg, const tlf_weights* w, void* d_workspace, size_t ws_bytes,
             size_t* ws_needed, void* hip_stream, tlf_ctx** out);

/* Batched prefill (Section 3.3; gather-scatter of Eq. 6-7 with K/V written at
 * the gathered original positions, Eq. 11, and causal attention among the
 * gathered tokens of each loop).  Resets every cache and starts a new batch of
 * `batch` sequences of `seq_len` tokens each.
 * With TLF_PREFILL_APPEND the call is a later chunk of the current batch's
 * prompts (chunked prefill; it may also follow decode steps): its tokens take
 * positions [S, S + seq_len) after the S tokens each sequence holds, loop i
 * appends the chunk's tokens of depth >= i to cache (b, i) after its existing
 * entries, and each of them attends over every entry of that cache up to its
 * own position (Eq. 10).  Prefilling a prompt in chunks gives the results of
 * one call on the whole prompt.  Requires a batch (TLF_E_STATE otherwise),
 * the same `batch`, and S + seq_len <= max_pos.
 *   d_tokens: [batch][seq_len] int32 token ids in [0, V).
 *   d_logits: [batch][V] float32 logits of the call's last position, or
 *             [batch][seq_len][V] with TLF_PREFILL_ALL_LOGITS.
 *   d_depths: [batch][seq_len] int32 routed depths, or NULL.
 * Requires 1 <= batch <= max_batch, 1 <= seq_len <= max_pos.  Pages for an
 * appended chunk are taken on the device; running out sets the sticky
 * TLF_E_OUT_OF_PAGES reported by the next synchronizing call. */
int tlf_prefill(tlf_ctx* ctx, int32_t batch, int32_t seq_len, const int32_t* d_tokens,
                float* d_logits, int32_t* d_depths, uint32_t flags);

/* One decode step for every sequence of the current batch (Section 3.3,
 * Eq. 9-11): token b sits at position seq_len, is routed, runs its m_b loops
 * (appending k, v to each loop's cache and attending over it) and exits.
 *   d_tokens: [batch] int32 token ids (the caller picks them, e.g. d_next of
 *             the previous step for greedy decoding).
 *   d_logits: [batch][V] float32.
 *   d_next:   [batch] int32 greedy token (lowest id among maxima), or NULL.
 *   d_depths: [batch] int32 routed depth, or NULL.
 *   d_margin: [batch] float32 depth-decision margin (argmax: top1 - top2
 *             logit; cumprob: min(p^(m) - threshold, threshold - p^(m+1));
 *             fixed: +inf), or NULL.
 * Returns TLF_E_STATE before a prefill or once seq_len == max_pos. */
int tlf_decode_step(tlf_ctx* ctx, const int32_t* d_tokens, float* d_logits, int32_t* d_next,
                    int32_t* d_depths, float* d_margin);

/* Waits for the stream, then fills *out and, optionally, the logical cache
 * index: which original positions each recursion-wise cache (b, i) holds
 * (Eq. 8; each token of depth m appended to the caches of loops 1..m, Eq. 11).
 *   h_len: [batch][R] int32 host array of cache lengths n_{b,i}, or NULL.
 *   h_pos: host array receiving, for b = 0..batch-1 and i = 1..R in that order,
 *          the ascending original positions held by cache (b, i), or NULL.
 *   pos_cap: capacity of h_pos in int32 elements (TLF_E_INVALID_ARG if short).
 * Physical page ids are implementation-defined and are not reported.
 * Returns the sticky device error, if any, after filling *out. */
int tlf_cache_stats(tlf_ctx* ctx, tlf_cache_stats_t* out, int32_t* h_len, int32_t* h_pos,
                    size_t pos_cap);

/* Measurement switch (decode steps are then launched kernel by kernel, not
 * from the captured graph).
 *   TLF_PROFILE_ATTN:  a pair of HIP events on the context's stream around
 *                      every decode-attention launch (attn_ms) and around each
 *                      step's loop-and-layer region (block_ms);
 *   TLF_PROFILE_BLOCK: events around the loop-and-layer region only, so that
 *                      block_ms carries no event overhead from inside it;
 *   TLF_PROFILE_OFF:   no events.
 * Any mode other than OFF resets the totals reported by tlf_cache_stats
 * (decode_steps, attn_*, block_ms, ...).  It launches one small kernel and
 * does not wait for the stream.  TLF_E_INVALID_ARG for an unknown mode. */
#define TLF_PROFILE_OFF 0
#define TLF_PROFILE_ATTN 1
#define TLF_PROFILE_BLOCK 2
int tlf_set_profiling(tlf_ctx* ctx, int mode);

/* Measurement probe (no context): reads `bytes` of device memory at d_buf
 * once with the 16-byte non-temporal vector loads the decode attention
 * streams its cache with, one workgroup per TLF_PROBE_READ_GRAIN bytes, and
 * writes nothing except, with negligible probability, one word of d_sink.
 * The read rate it reaches is the practical ceiling for the decode
 * attention's streaming.  bytes must be a positive multiple of
 * TLF_PROBE_READ_GRAIN and d_buf 16-byte aligned (else TLF_E_INVALID_ARG);
 * enqueued on `d_stream` without waiting. */
#define TLF_PROBE_READ_GRAIN 32768
int tlf_probe_read(const void* d_buf, size_t bytes, unsigned int* d_sink, void* d_stream);

/* Releases the host context (waits for the stream first).  NULL is ignored. */
void tlf_destroy(tlf_ctx* ctx);

/* Static text for a status code. */
const char* tlf_status_str(int status);

/* ---------------------------------------------------------------------------
 * Training-side gather-scatter (Section 3.2, Eq. 6-7) and the router's
 * straight-through estimator (Appendix B).
 *
 * These calls need no context: they work on caller-owned device buffers and
 * enqueue on `stream` (a hipStream_t; NULL is the null stream) without
 * waiting for it.  The tokens of a batch of B sequences of T tokens are the
 * rows b*T + t of one [B*T, d] float32 tensor (row-major, 16-byte aligned,
 * d a multiple of 4).  Token t takes part in loop i exactly when its depth
 * m_t >= i.  Backward passes reuse the same calls: the gradient of the
 * gather is an in-place tlf_gs_scatter of the compact gradient into the row
 * gradients (tlf_gs_expand where there are none yet), and the gradient of the
 * scatter is the incoming gradient itself for the previous state plus its
 * tlf_gs_gather for the block output.
 * Argument errors return TLF_E_INVALID_ARG before anything is enqueued; a
 * failed launch returns TLF_E_HIP.  Indices and slots are trusted: they must
 * be what tlf_gs_plan wrote for the same depths.
 * ------------------------------------------------------------------------- */

/* Active set of loop `loop` (Section 3.2 and Eq. 6).
 *   d_depth   [batch*seq_len] int32 depths m_t;
 *   d_index   [batch*seq_len] capacity; receives the active rows in
 *             increasing row order (each sequence's run contiguous and in
 *             causal order), *d_count of them;
 *   d_slot    [batch*seq_len] or NULL; receives each row's position in the
 *             compact tensor, -1 for a row not in the loop;
 *   d_offsets [batch+1] or NULL; receives where each sequence's run starts in
 *             the compact tensor, and the total last;
 *   d_count   [1]; the number of active rows.
 * One workgroup; batch*seq_len may be 0. */
int tlf_gs_plan(const int32_t* d_depth, int32_t batch, int32_t seq_len, int32_t loop, int32_t* d_index,
                int32_t* d_slot, int32_t* d_offsets, int32_t* d_count, void* d_stream);

/* The same plan (same outputs) from many workgroups: one launch counts the
 * active rows of each chunk of TLF_GS_PLAN_CHUNK_ROWS rows into the
 * workspace, a second places every chunk's rows after the counts before it
 * (Section 3.2 and Eq. 6).
 *   d_workspace  device scratch of at least tlf_gs_plan_ws_bytes(batch *
 *                seq_len) bytes, 4-byte aligned, borrowed for the call (it may
 *                be reused once the stream has passed this call); NULL when
 *                that size is 0.  Its contents need no initialisation.
 *   ws_bytes     its size.
 * Other arguments as tlf_gs_plan.  TLF_E_INVALID_ARG for a missing or short
 * workspace or batch * seq_len > TLF_GS_PLAN_MAX_ROWS. */
#define TLF_GS_PLAN_CHUNK_ROWS 2048
#define TLF_GS_PLAN_MAX_ROWS 8388608 /* 4096 chunks */
static inline size_t tlf_gs_plan_ws_bytes(int64_t rows) {
  return rows <= 0 ? 0 : (size_t)((rows + TLF_GS_PLAN_CHUNK_ROWS - 1) / TLF_GS_PLAN_CHUNK_ROWS) * 4u;
}
int tlf_gs_plan_ws(const int32_t* d_depth, int32_t batch, int32_t seq_len, int32_t loop, int32_t* d_index,
                   int32_t* d_slot, int32_t* d_offsets, int32_t* d_count, void* d_workspace, size_t ws_bytes,
                   void* d_stream);

/* For callers that cannot allocate device memory (code under HIP graph
 * capture, tight serving or training loops, harnesses that forbid
 * hipMalloc): tlf_gs_plan_ws with its per-chunk counts in a fixed array of
 * the library's own device memory (16 KiB on each GPU that runs it, held
 * until the process ends) instead of a caller workspace.  Nothing is
 * allocated, and the array needs no clearing (every count read is written
 * by the same call first).  All calls on one GPU share the array: calls
 * that overlap on that GPU (other streams, other threads) race and must be
 * serialised by the caller.  The stream must belong to the current device.
 * Same arguments and outputs as tlf_gs_plan; TLF_E_INVALID_ARG when
 * batch * seq_len > TLF_GS_PLAN_NOALLOC_MAX_ROWS (checked before any device
 * work), TLF_E_HIP if the array's address cannot be obtained. */
#define TLF_GS_PLAN_NOALLOC_MAX_ROWS 8388608
int tlf_gs_plan_noalloc(const int32_t* d_depth, int32_t batch, int32_t seq_len, int32_t loop, int32_t* d_index,
                        int32_t* d_slot, int32_t* d_offsets, int32_t* d_count, void* d_stream);

/* Gather (Eq. 6): d_out[r] = d_h[d_index[r]] for r < min(*d_count, max_rows).
 * d_out holds max_rows x d floats; rows past the count are not written.  The
 * count stays on the device (no host synchronisation); max_rows bounds the
 * launch. */
int tlf_gs_gather(const float* d_h, const int32_t* d_index, const int32_t* d_count, int32_t max_rows,
                  int32_t d, float* d_out, void* d_stream);

/* Scatter (Eq. 7): d_h_out[r] = d_y[d_slot[r]] + d_h_prev[r] where
 * d_slot[r] >= 0, else d_h_prev[r]; `rows` rows of d floats.  d_h_out may be
 * d_h_prev (in place: rows not in the loop are then neither read nor written);
 * otherwise the two must not overlap, and d_y must overlap neither. */
int tlf_gs_scatter(const float* d_h_prev, const float* d_y, const int32_t* d_slot, int32_t rows, int32_t d,
                   float* d_h_out, void* d_stream);

/* d_out[r] = d_y[d_slot[r]] where d_slot[r] >= 0, else zeros; `rows` rows of
 * d floats: a scatter into a zeroed tensor, without reading one.  d_out must
 * not overlap d_y. */
int tlf_gs_expand(const float* d_y, const int32_t* d_slot, int32_t rows, int32_t d, float* d_out, void* d_stream);

/* Straight-through estimator of the depth (Appendix B), elementwise over n
 * tokens.  Forward value: d_value[t] = (float)d_depth[t].  Backward: with
 * sigma the logistic function, d_grad_score[t] = d_grad_value[t] *
 * sigma(d_score[t]) * (1 - sigma(d_score[t])).  Either output may be NULL
 * (then its inputs may be NULL too). */
int tlf_ste(const int32_t* d_depth, const float* d_score, const float* d_grad_value, int32_t n, float* d_value,
            float* d_grad_score, void* d_stream);

/* ---------------------------------------------------------------------------
 * Training operators of the block's FFN half: RMSNorm, the gated FFN and their
 * gradients (Appendix A; SwiGLU as in tlf_layer_weights), and AdamW.
 *
 * As above: no context, caller-owned device buffers of the current device,
 * work enqueued on `stream` without waiting, TLF_E_INVALID_ARG or
 * TLF_E_UNSUPPORTED before anything is enqueued, TLF_E_HIP for a failed
 * launch.  No device memory is allocated, so every call may be captured into a
 * graph.  Tensors are row-major and contiguous, 16-byte aligned unless said otherwise;
 * outputs overlap nothing else.  Gradients overwrite their buffers.  Results
 * are the same to the bit from call to call.
 * ------------------------------------------------------------------------- */

/* RMSNorm of rows, with the AdaLN scale of each row's group (Section 3.1):
 *   r = 1 / sqrt(mean(x^2) + eps),  y = x r (1 + gamma[group])
 *   d_x      [rows][d], TLF_DTYPE_F32 or TLF_DTYPE_BF16 (x_dtype);
 *   d_gamma  [groups][d] float32, or NULL with groups = 0: y = x r;
 *   d_group  [rows] int32, the row's gamma (a depth's modulation, say); a row
 *            whose group lies outside [0, groups) takes none.  May be NULL when
 *            groups <= 1: every row takes gamma 0;
 *   d_y      [rows][d] (y_dtype);
 *   d_rstd   [rows] float32, receives r (tlf_rms_norm_grad reads it), or NULL;
 *            4-byte aligned, as d_group.
 * Squares are summed in float32: a row whose sum of squares passes its range
 * gives r = 0.  d a multiple of 4, at most TLF_NORM_MAX_D; groups at most
 * TLF_NORM_MAX_GROUPS, rows at most TLF_NORM_MAX_ROWS. */
#define TLF_NORM_MAX_D 4096
#define TLF_NORM_MAX_ROWS (1 << 30)
#define TLF_NORM_MAX_GROUPS 16
int tlf_rms_norm(const void* d_x, int32_t x_dtype, const float* d_gamma, const int32_t* d_group, int32_t groups,
                 int32_t rows, int32_t d, float eps, void* d_y, int32_t y_dtype, float* d_rstd, void* stream);

/* Gradients of tlf_rms_norm for the same x, gamma and group and the r it wrote:
 *   h = dy (1 + gamma[group]),  dx = r (h - x r^2 mean(h x)),
 *   dgamma[k] = sum over the rows of group k of dy x r
 *   d_dy [rows][d] in y's dtype; d_dx [rows][d] in x's dtype or NULL;
 *   d_dgamma [groups][d] float32 or NULL (zeros for a group without rows).
 *   d_workspace: tlf_rms_norm_grad_ws_bytes bytes, used during the call only;
 *   may be NULL when d_dgamma is. */
int tlf_rms_norm_grad_ws_bytes(int32_t groups, int32_t rows, int32_t d, size_t* ws_bytes);
int tlf_rms_norm_grad(const void* d_dy, int32_t y_dtype, const void* d_x, int32_t x_dtype, const float* d_gamma,
                      const int32_t* d_group, int32_t groups, const float* d_rstd, int32_t rows, int32_t d, void* d_dx,
                      float* d_dgamma, void* d_workspace, size_t ws_bytes, void* stream);

/* Gated FFN (Appendix A with SwiGLU): y = a W_down^T with a = silu(g) u and
 * g | u = x [W_gate | W_up]^T.
 *   dtype         of x, the weights and every output; products are summed in
 *                 float32, and a and the results are rounded to dtype (a is an
 *                 operand of the second product);
 *   d_x           [rows][d];
 *   d_w_gate_up   [2f][d]: rows gate | up (as tlf_layer_weights);
 *   d_w_down      [d][f];
 *   d_kept        tlf_ffn_kept_bytes bytes, receives what tlf_ffn_grad needs of g
 *                 and u (u silu'(g) and silu(g), in an order of its own; bf16: in 18
 *                 bits, float32's range with 9 bits of mantissa), or NULL if no
 *                 gradient follows;
 *   d_a           [rows][f], receives a (read by the second product);
 *   d_y           [rows][d];
 *   d_workspace   tlf_ffn_ws_bytes bytes (may be 0), used during the call only.
 * d and f multiples of 64, at most TLF_FFN_MAX_WIDTH; rows times the larger of
 * them less than 2^35. */
#define TLF_FFN_MAX_WIDTH 16384
static inline size_t tlf_ffn_kept_bytes(int32_t dtype, int32_t rows, int32_t f) {
  return rows <= 0 || f <= 0 ? 0 : ((size_t)rows + 15) / 16 * 8 * (size_t)f * (dtype == TLF_DTYPE_BF16 ? 9u : 16u);
}
int tlf_ffn_ws_bytes(int32_t dtype, int32_t rows, int32_t d, int32_t f, size_t* ws_bytes);
int tlf_ffn(const void* d_x, const void* d_w_gate_up, const void* d_w_down, int32_t dtype, int32_t rows, int32_t d,
            int32_t f, void* d_kept, void* d_a, void* d_y, void* d_workspace, size_t ws_bytes, void* stream);

/* Gradients of tlf_ffn from the `kept` and a that it wrote:
 *   da = dy W_down,  dg = da u silu'(g),  du = da silu(g) (rounded to dtype),
 *   dx = [dg | du] W_gate_up,  dW_gate_up = [dg | du]^T x,  dW_down = dy^T a
 *   d_dy [rows][d]; d_dx [rows][d], d_dw_gate_up [2f][d], d_dw_down [d][f], any
 *   of them NULL (its products are then not computed).  rows = 0: the weights'
 *   gradients are zeros.
 *   d_workspace: tlf_ffn_grad_ws_bytes bytes, used during the call only. */
int tlf_ffn_grad_ws_bytes(int32_t dtype, int32_t rows, int32_t d, int32_t f, size_t* ws_bytes);
int tlf_ffn_grad(const void* d_dy, const void* d_x, const void* d_w_gate_up, const void* d_w_down, const void* d_kept,
                 const void* d_a, int32_t dtype, int32_t rows, int32_t d, int32_t f, void* d_dx, void* d_dw_gate_up,
                 void* d_dw_down, void* d_workspace, size_t ws_bytes, void* stream);

/* One tensor of an AdamW step.  The float arrays need the alignment of their
 * elements only (whole tensors aligned to 16 bytes move in 16-byte vectors). */
#define TLF_ADAMW_BLOCK 256
typedef struct tlf_adamw_tensor {
  float* d_param;       /* [n], updated */
  void* d_copy;         /* [n] bf16, receives the updated parameter rounded, or NULL */
  const void* d_grad;   /* [n] of grad_dtype */
  void* d_m;            /* [n] first moment: float32, or e4m3 (OCP, finite) codes */
  void* d_v;            /* [n] second moment: float32, or e5m2 codes */
  float* d_m_scale;     /* 8 bits: [ceil(n / TLF_ADAMW_BLOCK)]; element e stands for code e times scale e / BLOCK */
  float* d_v_scale;     /* likewise */
  int64_t n;            /* at most 2^35 */
  int64_t step;         /* t >= 1: how many steps this tensor has had, this one included */
  double weight_decay;
  int32_t grad_dtype;   /* TLF_DTYPE_F32 or TLF_DTYPE_BF16 */
  int32_t state_bits;   /* 32 or 8 */
} tlf_adamw_tensor;

/* One AdamW step of `count` tensors (Appendix A's recipe), few launches for all:
 *   m = beta1 m + (1 - beta1) g,  v = beta2 v + (1 - beta2) g^2,
 *   p = p (1 - lr weight_decay) - lr (m / (1 - beta1^t)) / (sqrt(v / (1 - beta2^t)) + eps)
 * with eps at least FLT_MIN.  Moments of zeros (codes and scales too) are a
 * fresh state.  With 8 bits the step uses the new moments before they are
 * rounded; a block's scale is its largest |m| / 448 or v / 57344, and a v > 0
 * keeps at least the smallest code above zero.  A gradient that is not finite,
 * or whose square is none in float32, spoils the moments of its element (8 bits:
 * of its block).
 *   h_tensors: host array, read during the call.  Parameters, copies, moments
 *   and scales overlap nothing else of the call (TLF_E_INVALID_ARG), gradients
 *   may overlap each other.
 * The step counts and rates are values of the call: a captured call replays them. */
int tlf_adamw(const tlf_adamw_tensor* h_tensors, int32_t count, double lr, double beta1, double beta2, double eps,
              void* stream);

/* ---------------------------------------------------------------------------
 * Training operators around the FFN half: the block's attention, the gated
 * residual with the norm that follows, and the clipping of gradients.  As above.
 * ------------------------------------------------------------------------- */

/* Causal attention of ragged rows (Eq. 10 among the gathered tokens of a loop;
 * offsets as tlf_gs_plan writes them), with a sliding window and sinks.
 * Sequence b has nq = q_offsets[b + 1] - q_offsets[b] query rows and n keys from
 * row k_offsets[b]; its last query stands at its last key, query j at position
 * p = n - nq + j.  The key at position x is visible to it when
 *   x <= p and (p - x < window or x < sinks)
 * and o = sum softmax(scale q . k) v over the visible keys.  A query that sees no
 * key, and a row ahead of the first sequence or behind the last, gives zeros (and
 * zero gradients).
 * What a query does not see takes no part, whatever values it has. */
#define TLF_ATTN_MAX_SINKS 64
#define TLF_ATTN_MAX_HEADS 1024
#define TLF_ATTN_MAX_ROWS (1 << 29)
#define TLF_ATTN_MAX_UNITS (1 << 29)     /* rows times heads */
#define TLF_ATTN_MAX_SEQ_HEADS (1 << 22) /* sequences times heads */
#define TLF_ATTN_MAX_STRIDE (1 << 21)
#define TLF_ATTN_MIN_SCALE 1e-12f
#define TLF_ATTN_MAX_SCALE 1e12f
typedef struct tlf_attn_shape {
  int32_t dtype;     /* of q, k, v, o and their gradients: TLF_DTYPE_F32 or TLF_DTYPE_BF16 */
  int32_t batch;     /* sequences */
  int32_t heads;     /* of q and o: a multiple of kv_heads; head h reads key head h / (heads / kv_heads) */
  int32_t kv_heads;
  int32_t head_dim;  /* 64 or 128 (16 for float32 only) */
  int32_t rows_q;    /* rows of q and o */
  int32_t rows_k;    /* rows of k and v */
  int32_t window;    /* 0: every earlier key is visible (sinks is then without effect) */
  int32_t sinks;
  float scale;       /* from TLF_ATTN_MIN_SCALE to TLF_ATTN_MAX_SCALE; 1 / sqrt(head_dim) usually */
  /* Elements between rows, multiples of 16 bytes; a row's heads lie one behind the
   * other.  do lies as o. */
  int64_t q_stride, k_stride, v_stride, o_stride;
  /* Device arrays.  Offsets ascend (where they do not, rows may be left unwritten); they
   * are clamped to the rows there are. */
  const int32_t* d_q_offsets; /* [batch + 1] */
  const int32_t* d_k_offsets; /* [batch + 1]; d_q_offsets itself where the rows are the same */
  const int32_t* d_k_lengths; /* [batch] keys that sequence b holds of the rows up to k_offsets[b + 1], or NULL: all */
} tlf_attn_shape;

/*   d_lse  [heads][rows_q] float32, receives log2 of each softmax sum, base
 *          included (tlf_attn_grad reads it; +inf where nothing is visible), or NULL.
 *   d_o_low [rows_q] rows as o's, bf16 tensors only: receives what o lost where it was
 *          rounded (tlf_attn_grad reads it: without it the gradients of rows that few
 *          keys have most of the weight of are less exact), or NULL.
 *   d_workspace: tlf_attn_ws_bytes bytes (may be 0), used during the call only. */
int tlf_attn_ws_bytes(const tlf_attn_shape* shape, size_t* ws_bytes);
int tlf_attn(const tlf_attn_shape* shape, const void* d_q, const void* d_k, const void* d_v, void* d_o, float* d_lse,
             void* d_o_low, void* d_workspace, size_t ws_bytes, void* stream);

/* Gradients of tlf_attn from its inputs, its o and the lse and o_low (or NULL) that it
 * wrote:
 *   P = exp2(log2(e) scale q . k - lse),  dS = P (do . v - do . o),
 *   dq = scale dS k,  dk = scale dS^T q,  dv = P^T do
 * with sums over the queries and over the heads that share a key head.  P and dS
 * are rounded to dtype as operands, the sums are float32.  All three are written,
 * every row of them; their strides are elements between rows. */
int tlf_attn_grad_ws_bytes(const tlf_attn_shape* shape, size_t* ws_bytes);
int tlf_attn_grad(const tlf_attn_shape* shape, const void* d_do, const void* d_q, const void* d_k, const void* d_v,
                  const void* d_o, const float* d_lse, const void* d_o_low, void* d_dq, int64_t dq_stride, void* d_dk,
                  int64_t dk_stride, void* d_dv, int64_t dv_stride, void* d_workspace, size_t ws_bytes, void* stream);

/* The gated residual of the block with the norm that follows (Section 3.1,
 * Appendix A: x + (1 + alpha) F, then the next operand's norm), in one pass:
 *   t = y, or with post_norm y / sqrt(mean(y^2) + eps)
 *   h = x + (1 + alpha[group]) t,  z = h r (1 + gamma[group]) with r = 1 / sqrt(mean(h^2) + eps)
 *   d_x, d_h   [rows][d] float32: the residual rows before and after (one buffer for
 *              both is allowed);
 *   d_y, d_z   [rows][d] of y_dtype: what is added, and the next operand;
 *   d_alpha, d_gamma  [groups][d] float32; either or, with groups = 0, both NULL (zeros);
 *   d_group    [rows] as for tlf_rms_norm;
 *   d_rstd, d_ystd    [rows] float32, receive r and (post_norm) y's
 *              1 / sqrt(mean(y^2) + eps) for the gradients, or NULL.
 * Sums and limits as tlf_rms_norm. */
int tlf_residual_norm(const float* d_x, const void* d_y, int32_t y_dtype, const float* d_alpha, const float* d_gamma,
                      const int32_t* d_group, int32_t groups, int32_t rows, int32_t d, int32_t post_norm, float eps,
                      float* d_h, void* d_z, float* d_rstd, float* d_ystd, void* stream);

/* Gradients of tlf_residual_norm from the gradients dh of h and dz of z (either may
 * be NULL: zeros), its h, y, scales and the r's that it wrote:
 *   u = dz (1 + gamma[group]),  dx = dh + r (u - h r^2 mean(u h)),  dt = dx (1 + alpha[group]),
 *   dy = dt, or with post_norm ry (dt - y ry^2 mean(dt y)),
 *   dalpha[k] = sum over the rows of group k of dx t,  dgamma[k] = of dz h r
 *   d_dx [rows][d] float32, d_dy [rows][d] of y_dtype; d_dalpha and d_dgamma
 *   [groups][d]: those of the scales that there are, or neither (NULL).
 *   d_workspace: tlf_residual_norm_grad_ws_bytes bytes, used during the call only;
 *   may be NULL without the scales' gradients. */
int tlf_residual_norm_grad_ws_bytes(int32_t groups, int32_t rows, int32_t d, size_t* ws_bytes);
int tlf_residual_norm_grad(const float* d_dh, const void* d_dz, const float* d_h, const void* d_y, int32_t y_dtype,
                           const float* d_alpha, const float* d_gamma, const int32_t* d_group, int32_t groups,
                           const float* d_rstd, const float* d_ystd, int32_t rows, int32_t d, int32_t post_norm, float* d_dx,
                           void* d_dy, float* d_dalpha, float* d_dgamma, void* d_workspace, size_t ws_bytes, void* stream);

/* The norm of all elements of many gradients, and the scale that clips them to
 * max_norm, few launches for all:
 *   *d_norm = sqrt(sum g^2),  *d_scale = 1 where that is at most max_norm, else max_norm / norm
 * Summed in float64.  Gradients that are not finite give a scale of 0 or NaN, whatever
 * max_norm is; where only *d_norm is past float32's range the scale is right.
 * d_scale may be NULL; max_norm > 0 may be infinite.  Gradients need the alignment of their
 * elements only and may overlap.
 *   h_grads: host array, read during the call.
 *   d_workspace: tlf_grad_norm_ws_bytes bytes, 8-byte aligned, used during the call only. */
typedef struct tlf_grad {
  void* d_grad;
  int64_t n;       /* elements, at most 2^35 */
  int32_t dtype;
  int32_t reserved;
} tlf_grad;
int tlf_grad_norm_ws_bytes(const tlf_grad* h_grads, int32_t count, size_t* ws_bytes);
int tlf_grad_norm(const tlf_grad* h_grads, int32_t count, double max_norm, float* d_norm, float* d_scale, void* d_workspace,
                  size_t ws_bytes, void* stream);

/* g = g * *d_scale, rounded to its type; with a scale of 1 nothing is read or written.
 * The gradients overlap neither each other nor the scale. */
int tlf_grad_clip(const tlf_grad* h_grads, int32_t count, const float* d_scale, void* stream);

/* tlf_adamw with gradients times *d_grad_scale, a device value (tlf_grad_norm's): the
 * product is rounded to float32, with 8-bit moments not at all.  The scale overlaps
 * nothing that is updated. */
int tlf_adamw_scaled(const tlf_adamw_tensor* h_tensors, int32_t count, double lr, double beta1, double beta2, double eps,
                     const float* d_grad_scale, void* stream);

#ifdef __cplusplus
}
#endif

#endif /* TLF_H */
