/*
 * moa.h -- C ABI of the MI355X (gfx950) ragged mixture-of-agents generation engine.
 *
 * What it computes. The paper's workload (Section "Problem Setting") is a
 * fixed batch of pre-routed model calls: every (query, expert) pair chosen by
 * the upstream router is an independent generation by that expert, and the
 * aggregator call (Section "MOSAIC: Adaptive Aggregation", Eq. 11) is one more
 * generation on the query followed by the expert outputs. Generation length
 * drives the cost (Section "Workload Characterisation"), and decode is bound
 * by memory bandwidth once a few prompts are in flight (appendix "Pitfalls of
 * Data Concurrency and Over-Sharding"). This engine keeps every model
 * co-resident on one GPU, shares one paged KV pool between them, and runs all
 * models' requests in one ragged continuous batch per step: each call
 * greedily decodes exactly max_new_tokens tokens (no end-of-sequence token).
 *
 * Conventions for every call:
 *   - returns moa_status; MOA_OK == 0, errors are negative; no exception or
 *     signal crosses the ABI;
 *   - pointers named host_* / tokens / res / tok_buf are host memory, copied
 *     before the call returns (the caller keeps ownership);
 *   - dev_arena is device memory owned by the caller; the engine
 *     sub-allocates weights, the KV pool and its workspace inside it and never
 *     calls hipMalloc after moa_create; the arena and the stream must outlive
 *     the engine;
 *   - device work is enqueued on the caller's stream; a bf16 engine with
 *     max_models > 1 also runs part of a step's layers on one internal stream
 *     that waits for the caller's stream when the step starts and that the
 *     caller's stream waits for before the step's final norm and LM head, so
 *     the caller's stream still orders every step (MOA_FLAG_ONE_STREAM keeps
 *     everything on the caller's stream);
 *   - single host thread: an engine is not thread-safe;
 *   - after MOA_EHIP only moa_destroy is valid on that engine.
 */
#ifndef MOA_H
#define MOA_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
  MOA_OK = 0,
  MOA_EINVAL = -1, /* bad argument (shape, id, length, capacity) */
  MOA_ENOMEM = -2, /* arena, token store or block-list store too small */
  MOA_ENOSPC = -3, /* request can never fit the KV pool */
  MOA_ESTATE = -4, /* call not valid in the engine's current state */
  MOA_EHIP = -5    /* HIP runtime error; the engine is unusable */
} moa_status;

enum { MOA_F32 = 0, MOA_BF16 = 1 };

/* flags */
enum {
  /* Scheduler dry run: every call does its host bookkeeping but no device
   * work is enqueued and no tokens are computed (collected tokens read -1).
   * dev_arena and hip_stream may be NULL. */
  MOA_FLAG_PLAN_ONLY = 1,
  /* Run every kernel on the caller's stream. By default a bf16 engine with
   * several models splits each step's model groups in two halves and runs
   * the second half's layers on an internal stream (its own split-K
   * workspace in the arena), so the halves' kernels overlap. Every launch
   * is planned over the whole step either way, so the results are
   * bit-identical; the flag gives launch durations that are not shared with
   * concurrent kernels. */
  MOA_FLAG_ONE_STREAM = 2,
  /* bf16 engines: K and V are cached in 4 bits (the cells of MOA_KV_INT4), 3.6
   * (head_dim 64) to 3.8 (128) times as many positions in a byte. Every row
   * attends to what its own position's and all earlier codes stand for, in
   * prefill too, so chunk lengths change no value. Injected histories are
   * stored in 4 bits from their bf16 values. EINVAL in an f32 engine. */
  MOA_FLAG_KV_INT4 = 4,
  /* Models with norms of queries and keys for each head before the rotation:
   * the weight blob has q_norm[hd], k_norm[hd] after wv of each layer, and
   * rms_eps is their eps too. */
  MOA_FLAG_QK_NORM = 8,
  /* Room in the arena for moa_request_scores. */
  MOA_FLAG_SCORES = 16
};

/* Decoder geometry (Llama-style pre-norm decoder: RMSNorm, GQA attention with
 * rotate-half RoPE, SwiGLU MLP, untied LM head). */
typedef struct {
  int32_t n_layers, d_model, n_heads, n_kv_heads, head_dim, ffn_dim, vocab;
  float rope_theta, rms_eps;
} moa_model_cfg;

typedef struct {
  moa_model_cfg model;        /* geometry shared by every model of the engine */
  int32_t dtype;              /* MOA_F32 or MOA_BF16: weights, activations, KV */
  int32_t kv_block_size;      /* token slots per KV block; must be 16 */
  int32_t num_kv_blocks;      /* blocks in the shared KV pool (all layers) */
  int32_t max_num_seqs;       /* running requests at once */
  int32_t max_prefill_tokens; /* prompt tokens processed per step */
  int32_t max_model_len;      /* max prompt + generated tokens of a request */
  int32_t max_models;         /* models the arena reserves room for */
  int32_t flags;              /* MOA_FLAG_* */
  int64_t token_store;        /* device slots for prompt+output tokens of live requests (0: default) */
  int64_t block_store;        /* device slots for block lists of live requests (0: default) */
} moa_engine_cfg;

typedef struct moa_engine moa_engine;

typedef struct {
  int64_t step;            /* index of the step just enqueued; -1: nothing to run */
  int32_t admitted;        /* requests admitted this step */
  int32_t prefill_tokens;  /* prompt positions processed */
  int32_t decode_rows;     /* decode positions processed */
  int32_t finished;        /* requests retired this step */
  int32_t running;         /* running after the step */
  int32_t pending;         /* waiting for admission after the step */
  int32_t free_blocks;     /* free KV blocks after the step */
  int32_t emitted;         /* tokens the step produces: its decode rows plus the
                              requests whose prompt completes in it */
} moa_step_info;

typedef struct {
  int64_t request_id;
  int32_t model_id;
  int32_t n_tokens;        /* == max_new_tokens of the request */
  int64_t tok_offset;      /* where its tokens start in the caller's tok_buf */
  int64_t finish_step;     /* step at which it retired */
} moa_result;

/* Device bytes moa_create + max_models moa_load_expert calls need in the arena.
 * EINVAL: inconsistent cfg. */
moa_status moa_arena_bytes(const moa_engine_cfg* cfg, size_t* bytes);

/* Create an engine. cfg is copied. Lays out the KV pool and workspace inside
 * dev_arena (arena_bytes >= moa_arena_bytes()). hip_stream is a hipStream_t.
 * EINVAL: bad cfg (kv_block_size != 16, head_dim not 64/128 in bf16 mode,
 * n_heads not a multiple of n_kv_heads, non-positive sizes). ENOMEM: arena too
 * small. EHIP: runtime failure (no engine is returned). */
moa_status moa_create(const moa_engine_cfg* cfg, void* dev_arena, size_t arena_bytes,
                      void* hip_stream, moa_engine** out);

/* Load one model (Section "MOSAIC: Multi-Model Scheduling", subsection
 * "Problem Setting": the deployment draws its experts from a pool of
 * heterogeneous models; here every expert and the aggregator are resident
 * at once, so the per-model load cost l_m of that subsection is paid once,
 * here, instead of per session). host_weights is the packed blob: tensors in the order
 *   embed[V,d], { attn_norm[d], wq[nh*hd,d], wk[nkv*hd,d], wv[nkv*hd,d],
 *   (q_norm[hd], k_norm[hd] with MOA_FLAG_QK_NORM,) wo[d,nh*hd], mlp_norm[d], w_gate[ffn,d], w_up[ffn,d], w_down[d,ffn] } x L,
 *   final_norm[d], lm_head[V,d]
 * each row-major [out, in], elements in the engine dtype (fp32, or bf16 bits),
 * no padding. The engine re-lays the matrices out for its kernels. Model ids
 * are dense, in load order; the aggregator is just another model. Blocks
 * until the weights are resident. EINVAL: cfg differs from the engine's
 * geometry or nbytes is wrong. ENOMEM: more than max_models. ESTATE: called
 * after the first moa_step. */
moa_status moa_load_expert(moa_engine* e, const moa_model_cfg* cfg, const void* host_weights,
                           size_t nbytes, int32_t* model_id);

/* Queue one generation call (subsection "Problem Setting": the fixed prompt
 * set, routed before scheduling, is a batch of (prompt, expert) calls;
 * subsection "MOSAIC: Adaptive Aggregation": the aggregator call is one more
 * such call on the query followed by the expert outputs): prompt
 * tokens[0..n_tokens) for model model_id, emitting exactly max_new_tokens tokens. Request ids are dense and increase
 * in submit order. The request waits in a FIFO until its KV blocks
 * ceil((n_tokens + max_new_tokens - 1) / 16) and a seat are free.
 * EINVAL: n_tokens < 1, max_new_tokens < 1, unknown model, token id outside
 * [0, vocab) (not checked in a MOA_FLAG_PLAN_ONLY dry run), n_tokens +
 * max_new_tokens - 1 > max_model_len, or max_prefill_tokens == 0.
 * ENOSPC: the request needs more blocks than the pool has.
 * ENOMEM: token or block-list store full (collect finished requests first). */
moa_status moa_submit(moa_engine* e, const int32_t* tokens, int32_t n_tokens, int32_t model_id,
                      int32_t max_new_tokens, int64_t* request_id);

/* Queue a call that arrives with a KV history instead of a prompt to prefill
 * (a long generation already in progress): positions 0..ctx_len-1 of every
 * layer hold the given K/V, the call feeds seed_token at position ctx_len and
 * emits exactly max_new_tokens tokens. It needs
 * ceil((ctx_len + max_new_tokens) / 16) blocks and skips the prefill phase.
 * host_kv: [n_layers][2 (K, V)][ctx_len][n_kv_heads][head_dim] elements of the
 * engine dtype (K after RoPE), copied before the call returns and written into
 * the request's blocks when it is admitted (that step drains the stream).
 * host_kv == NULL: the history is filled on the device with values in
 * [-1, 1) from a hash of (request id, layer, K|V, position, head, dim).
 * EINVAL: bad id, ctx_len < 0, max_new_tokens < 1, seed token outside the
 * vocabulary, or ctx_len + max_new_tokens > max_model_len. ENOSPC / ENOMEM as
 * for moa_submit. */
moa_status moa_submit_with_history(moa_engine* e, int32_t model_id, int32_t seed_token, int32_t ctx_len,
                                   const void* host_kv, int32_t max_new_tokens, int64_t* request_id);

/* Plan one step on the host and enqueue its kernels on the stream (the
 * generation phase that subsection "Workload Characterisation" makes the
 * dominant cost, run as continuous batching of every resident model's calls,
 * which appendix "The Pitfalls of Data Concurrency and Over-Sharding" needs
 * to keep decode bound by memory bandwidth):
 *   1 admit FIFO heads while a seat and their blocks are free (head-of-line
 *     blocking); a request gets the smallest free block ids, ascending;
 *   2 prefill: running requests in admission order take prompt positions up
 *     to the per-step budget; completing a prompt emits token 0;
 *   3 decode: every other running request with tokens left feeds its last
 *     token and emits the next one;
 *   4 retire requests that have emitted all tokens; their blocks are freed.
 * Does not wait for the device (the sampled tokens stay on the device and feed
 * the next step). info may be NULL; info->step == -1 when nothing is queued
 * or running. EHIP on a runtime failure. */
moa_status moa_step(moa_engine* e, moa_step_info* info);

/* moa_step for callers that cannot allocate (code under HIP graph capture,
 * tight serving loops, harnesses that forbid allocation): the same step --
 * the same plan and kernels, bit-identical results -- that calls no HIP
 * allocation routine (no hipMalloc / hipHostMalloc / hipFree /
 * hipEventCreate). Its kernels' split-K and split-KV partial sums live in the
 * library's static per-GPU scratch array (64 MiB, one copy on each GPU the
 * library runs on, held until the process ends) instead of the arena; the
 * metadata goes through the pinned staging sized at moa_create; prompts and
 * block lists are uploaded from the engine's own host copies; kernel timing
 * (moa_debug_time_kernels) is skipped for these steps.
 * ENOMEM, with nothing changed: the engine's planned partials (split-K
 * partials of every model stream plus split-KV slots) exceed 64 MiB (then
 * use moa_step). Every moa_step_noalloc on one GPU shares that GPU's array:
 * calls whose steps overlap on the device (engines stepping on different
 * streams at once) race; steps of one engine are ordered by its stream.
 * Other errors as moa_step. */
moa_status moa_step_noalloc(moa_engine* e, moa_step_info* info);

/* Hand back finished calls (subsection "MOSAIC: Adaptive Aggregation": the
 * expert outputs a query's aggregator call, or the confidence gate of Eq. 11,
 * is waiting for). Return requests retired at steps <= upto_step (upto_step < 0: every step
 * enqueued so far) that were not collected yet, in retirement order (step,
 * then admission order), waiting for that step to finish on the device.
 * Tokens are written back to back into tok_buf. If cap or tok_cap is too
 * small nothing is drained, *n_out is set to the number of results that are
 * ready and EINVAL is returned. */
moa_status moa_collect(moa_engine* e, int64_t upto_step, moa_result* res, int32_t cap,
                       int32_t* n_out, int32_t* tok_buf, int64_t tok_cap);

/* Score every token that request_id emits: for output j, logprob[j] = its log
 * probability under the logits that produced it, entropy[j] = their entropy
 * (natural units), top_ids / top_logprobs [j][top_k] = the top_k (0 .. 32)
 * likeliest tokens (moa_score_tokens has the definitions; top_* may be NULL
 * when top_k is 0). The arrays are host memory of max_new_tokens (times top_k)
 * entries that the caller keeps until the request is collected; they are
 * complete when moa_collect returns it (or after moa_sync, for steps enqueued
 * before). EINVAL: bad id, NULL array or top_k. ESTATE: the engine lacks
 * MOA_FLAG_SCORES or is plan-only, or the request's prefill has completed. */
moa_status moa_request_scores(moa_engine* e, int64_t request_id, int32_t top_k, float* logprob, float* entropy,
                              int32_t* top_ids, float* top_logprobs);

/* Wait for every enqueued step. */
moa_status moa_sync(moa_engine* e);

/* Wait for the engine's streams, then free what the engine allocated
 * (host state, pinned staging, streams and events). The device arena stays
 * the caller's: free it after this returns. NULL is a no-op. */
void moa_destroy(moa_engine* e);
/* Static description of a status code ("MOA_OK", "MOA_EINVAL: invalid
 * argument", ...); never NULL. */
const char* moa_status_str(moa_status s);

/* ---- inspection hooks (tests) ---- */

typedef struct {
  int32_t model_id, prompt_len, max_new_tokens, n_blocks;
  int64_t admit_step, finish_step; /* -1 until it happens */
  int32_t n_chunks;                /* prefill chunks so far */
  int32_t state;                   /* 0 pending, 1 running, 2 retired, 3 collected */
} moa_request_info;

moa_status moa_debug_request(moa_engine* e, int64_t request_id, moa_request_info* info);

/* The request's KV block ids (ascending, as admitted). n_out = count. */
moa_status moa_debug_block_table(moa_engine* e, int64_t request_id, int32_t* out, int32_t cap,
                                 int32_t* n_out);

/* What the cache holds of a running request: K and V of positions [0, n) of
 * `layer`, host arrays [n][n_kv_heads][head_dim] in the engine dtype (4-bit
 * values rounded to bf16), for a position that no step has written yet
 * whatever its block held. Waits for the enqueued steps. EINVAL: bad id, layer
 * or n (past the request's blocks). ESTATE: not running, or plan-only. */
moa_status moa_debug_kv(moa_engine* e, int64_t request_id, int32_t layer, int32_t n, void* host_k, void* host_v);

/* The request's prefill chunks as (step, start, length) triples. */
moa_status moa_debug_chunks(moa_engine* e, int64_t request_id, int64_t* out, int32_t cap_triples,
                            int32_t* n_out);

/* Per-step bookkeeping rows (step, admitted, prefill_tokens, decode_rows,
 * finished, free_blocks_after), 6 int64 per step, oldest first, into out
 * (caller-owned, cap_steps rows). *n_out is always set to the number of
 * steps recorded; MOA_EINVAL without writing when cap_steps is smaller (a
 * call with out = NULL and cap_steps = 0 asks for the count) or when e or
 * n_out is NULL. */
moa_status moa_debug_steps(moa_engine* e, int64_t* out, int64_t cap_steps, int64_t* n_out);

/* How the last moa_step split its models over the model streams (a
 * MOA_FLAG_PLAN_ONLY bf16 engine plans the split a GPU engine with two
 * streams would make, so this can be inspected without a GPU).
 *   *n_shares: shares used, 1 .. 4;
 *   *n_models: models with rows in the step;
 *   models[i], i < n_models: those models in the step's row order;
 *   cost[i]: the split's cost of models[i]: its weight bytes times
 *     max(1, rows / 96) plus the K/V bytes its rows' attention reads;
 *   share_models0[u], share_row0[u], share_lm0[u], u <= n_shares: index in
 *     models, row and LM row where share u starts (the last entries are
 *     n_models and the step's row and LM-row counts).
 * share_* hold at least 5 entries, models and cost max_models. */
moa_status moa_debug_step_shares(moa_engine* e, int32_t* n_shares, int32_t* n_models, int32_t* models,
                                 double* cost, int32_t* share_models0, int32_t* share_row0,
                                 int32_t* share_lm0);

/* Capture the fp32 logits row of every token request_id emits: row j (the
 * logits that produced output token j) is copied to host_logits + j * vocab
 * once the step that computes it completes. cap: floats host_logits holds;
 * EINVAL (nothing registered) when it is below max_new_tokens * vocab. The
 * buffer must stay valid until the request is collected. ESTATE when the
 * request's prefill has already completed (register before it). */
moa_status moa_debug_capture_logits(moa_engine* e, int64_t request_id, float* host_logits, int64_t cap);

/* Kernel classes of one step (for moa_debug_time_kernels). */
enum {
  MOA_K_EMBED = 0, MOA_K_NORM, MOA_K_GEMM_QKV, MOA_K_ROPE_KV, MOA_K_ATTN, MOA_K_ATTN_REDUCE,
  MOA_K_GEMM_O, MOA_K_GEMM_GATEUP, MOA_K_GEMM_DOWN, MOA_K_GEMM_LMHEAD, MOA_K_ARGMAX, MOA_K_PREFILL_ATTN,
  /* Two views of the GEMM launches above, by the kernel that runs them: every
   * qkv / o / gate-up / down / LM-head launch is counted once more in exactly
   * one of these (the kernels of small and medium row counts, or the
   * 128-row-tile matrix-core kernel of large row counts). A sum over
   * classes must leave them out. */
  MOA_K_GEMM_SMALL_M, MOA_K_GEMM_LARGE_M,
  MOA_K_COUNT
};

/* Per-class launch statistics of the sampled steps. bytes/flops are the
 * algorithmic figures of those launches: for a GEMM the bf16 weights it
 * streams (N*K*2 per model group) plus its split-bf16 input (M*K*4) and fp32
 * output (M*N*4), flops 2*M*N*K; for attention the K/V it reads
 * (per KV head keys*4*head_dim in bf16, keys*(head_dim + 8) in 4 bits) plus
 * q (fp32) and its output; token scores count under ARGMAX; for causal
 * prefill attention each block's keys once per KV head, and 4*head_dim flops
 * per (query head, query, visible key). */
typedef struct {
  int64_t launches;   /* timed launches (sampled steps) */
  double ms;          /* their summed durations (HIP events around each launch; sampled
                         steps run on one stream, so no other stream's kernels overlap them) */
  double bytes;       /* their algorithmic bytes */
  double flops;       /* their algorithmic flops */
  int64_t launches_all; /* every launch since the reset */
  double bytes_all, flops_all;
  double roof_ms_all; /* sum over every launch of max(bytes / peak_bw, flops / peak_flops) */
} moa_kernel_stats;

/* Reset the statistics; from now on account every launch (bytes, flops,
 * roofline time at the given peaks, bytes/s and flop/s) and time every launch
 * of one step out of `every` (every <= 0: no timing) with an event pair
 * around it on the engine's stream. A timed step runs all of its kernels on
 * the caller's stream (a two-stream engine included; the results are the
 * same bits), so a timed launch carries the whole step and runs beside no
 * other stream's kernels. */
moa_status moa_debug_time_kernels(moa_engine* e, int32_t every, double peak_bw, double peak_flops);

/* Statistics per class, out[MOA_K_COUNT]. Waits for the stream. */
moa_status moa_debug_kernel_stats(moa_engine* e, moa_kernel_stats* out);

/* What this GPU sustains, measured on the engine's stream (the device work
 * runs now; the call returns when it is done): *read_bytes_per_s = streaming
 * HBM read bandwidth over up to 8 GiB of the KV pool (read only; the pool must
 * be at least 1 GiB), *mfma_flops_per_s = bf16 matrix-core throughput of the
 * 32x32x16 MFMA (dense, 2*32*32*16 flops per instruction). Each is the best of
 * five timed runs after a warm-up. Uses the logits workspace as scratch
 * (overwritten; call between steps). EINVAL: null outputs or a pool under
 * 1 GiB; ESTATE: plan-only engine or unusable engine; EHIP: runtime error. */
moa_status moa_debug_measure_peaks(moa_engine* e, double* read_bytes_per_s, double* mfma_flops_per_s);

/* ---- operators on the caller's own tensors ----
 *
 * What a layer does around its paged cache, and what the head says about a
 * token, for callers that keep their own tensors and cache pools; the engine's
 * steps launch the same kernels (MOA_FLAG_KV_INT4, MOA_FLAG_QK_NORM,
 * moa_request_scores).
 *
 * Every pointer but cfg and bytes is device memory of hip_stream's device,
 * which must be the current device; the work is enqueued on hip_stream and
 * nothing is allocated, copied to the host or waited for, so the calls can be
 * captured into a graph. Matrices are row-major; a stride is the elements
 * from one row to the next (at least the row's width, any alignment of the
 * element). No output may overlap an input or another output. Sizes and the
 * values of cfg are checked (MOA_EINVAL): at most 2^20 rows, sequences and
 * chunks, 2^26 entries a table row, 2^30 tokens, and for attention fewer than
 * 2^24 workgroups (KV heads times rows, or blocks of 128 queries, times
 * splits of the keys). Index
 * tensors are read on the device, where an entry that is out of range is
 * skipped as each call states. A call of zero rows does nothing. workspace
 * (256-byte aligned, MOA_ENOMEM if it is smaller than the *_bytes call says)
 * is scratch of one call: calls that may overlap on the device, two graphs
 * that replay at once among them, need one each. MOA_EHIP: the launch failed.
 */

/* How a pool holds K and V. */
enum { MOA_KV_F32 = 0, MOA_KV_BF16 = 1, MOA_KV_INT4 = 2 };

/* A paged pool: [n_layers][num_blocks][n_kv_heads] cells of 16 positions of
 * one head (head_dim D = 64 or 128). n_heads query heads share the KV heads;
 * n_heads / n_kv_heads is 1, 2, 4 or 8. The pool is 16-byte aligned.
 *   F32, BF16: a cell is K [16][D], then V [16][D].
 *   INT4: a cell is 16 D + 128 bytes:
 *     K codes [16][D / 2]: byte i of a position has dims 2 i (low four bits) and 2 i + 1;
 *     V codes [D / 2][16]: byte i of a position has dims i (low four bits) and i + D / 2;
 *     K scales [16], V scales [16]: bf16 pairs (s, m), s in the lower half of the word.
 *   Code c stands for m + s c. A row (a position's K or V of one head, as
 *   float32) is stored with m = bf16(min), s = bf16((max - min) * (1 / 15)),
 *   1 / 15 and the product in float32, and
 *   c = (x - m) / s rounded half to even and clamped to 0 .. 15 (0 where s = 0).
 *   A row with a NaN, an infinity or a range past float32 has s = NaN, so all
 *   of it stands for NaN. Attention sums s c with factors up to 2^24: values
 *   from 2^100 on may become infinite there. */
typedef struct {
  int32_t kind, n_layers, num_blocks, n_heads, n_kv_heads, head_dim;
} moa_kv_cfg;

/* Bytes of a pool. EINVAL: inconsistent cfg. */
moa_status moa_kv_bytes(const moa_kv_cfg* cfg, size_t* bytes);

/* Norms of the queries and keys of each head, the position rotation and the
 * append to the cache in one pass. qkv [n_rows] rows of (n_heads + 2
 * n_kv_heads) * D elements (queries, keys, values) of `type` (MOA_F32 or
 * MOA_BF16). Row r is position p = row_pos[r] of sequence row_seq[r], whose
 * position p lies in block tables[row_seq[r]][p / 16], slot p % 16 (tables:
 * [n_seqs][table_len] block ids).
 *   q_gain, k_gain (both or neither NULL): [D] of gain_type; each query and
 *     key head becomes x / sqrt(mean(x^2) + eps) * gain.
 *   rope (or NULL: no rotation): [rope_len][D / 2] pairs (cos, sin); pairs
 *     (i, i + D / 2) of queries and keys are turned by row p.
 *   q: [n_rows][n_heads][D] of `type`, written; keys and values are written
 *     to `layer` of kv. The keys of a 4-bit pool are computed in 64 bits and
 *     rounded to float32 once, so that no code hangs on the order of a sum.
 * A row with p < 0 (padding) or, with rope, p >= rope_len is left alone; one
 * whose sequence, table entry or block is out of range has its q written and
 * nothing cached. The rows' positions must be distinct: of two rows that name
 * one slot, the bytes of either may stay. */
moa_status moa_kv_append(const moa_kv_cfg* cfg, void* kv, int32_t layer, const void* qkv, int32_t type,
                         int64_t qkv_stride, int32_t n_rows, const int32_t* row_seq, const int32_t* row_pos,
                         const int32_t* tables, int32_t n_seqs, int32_t table_len, const float* rope,
                         int32_t rope_len, const void* q_gain, const void* k_gain, int32_t gain_type, float eps,
                         void* q, void* hip_stream);

/* What the cache holds at given positions: k, v [n_rows][n_kv_heads][D],
 * float32 from an F32 pool, else bf16 (4-bit values rounded to it). Rows
 * that are out of range (position, sequence, table entry, block) read as 0. */
moa_status moa_kv_read(const moa_kv_cfg* cfg, const void* kv, int32_t layer, int32_t n_rows, const int32_t* row_seq,
                       const int32_t* row_pos, const int32_t* tables, int32_t n_seqs, int32_t table_len, void* k,
                       void* v, void* hip_stream);

/* Attention of decode rows over a 4-bit pool: row r's query heads see keys
 * [0, c), c = min(row_ctx[r], max_ctx), of sequence row_seq[r], and out[r]
 * [n_heads][D] = softmax(scale * q . k) . v. q rows (n_heads * D elements) and
 * out are of `type`; sums, the softmax and its statistics are float32. q and
 * the probabilities enter the products with 22 significant bits in float32
 * calls; in bf16 ones q is exact and the probabilities have 11. A
 * row with c <= 0 or a sequence out of range is 0 (rows of one call may share
 * a sequence and may see fewer keys than it has). max_ctx bounds the work
 * (1 <= max_ctx <= 16 table_len): the keys of long rows are split among
 * workgroups and joined in a fixed order, in splits that depend on n_rows,
 * n_kv_heads and max_ctx alone; between those the bits of a row hang on
 * nothing but the row. Block ids out of range are read as the pool's last block.
 * EINVAL too: the pool is not INT4. */
moa_status moa_kv_attend_bytes(const moa_kv_cfg* cfg, int32_t n_rows, int32_t max_ctx, size_t* bytes);
moa_status moa_kv_attend(const moa_kv_cfg* cfg, const void* kv, int32_t layer, const void* q, int32_t type,
                         int64_t q_stride, int32_t n_rows, const int32_t* row_seq, const int32_t* row_ctx,
                         const int32_t* tables, int32_t n_seqs, int32_t table_len, int32_t max_ctx, float scale,
                         void* out, void* workspace, size_t workspace_bytes, void* hip_stream);

/* Causal attention of prompt chunks over a 4-bit pool: chunk i is rows
 * [chunk_start[i], chunk_start[i + 1]) (chunk_start: n_chunks + 1 ascending
 * entries, within [0, n_rows]) and its last row is position chunk_ctx[i] - 1 of
 * the sequence of tables[i]; a row at position p sees keys [0, p], and one at
 * p < 0 is 0. Rows in no chunk are left as they were. Otherwise as
 * moa_kv_attend (the splits depend on n_rows, n_chunks, the heads, type and
 * max_ctx; between those the bits of a row hang on nothing but the row, so
 * not on where its prompt is cut into chunks), with chunk_ctx[i] <= max_ctx (a chunk past it is clamped to end
 * at max_ctx). Chunks of any lengths may stand side by side, empty ones
 * too; single rows are what moa_kv_attend is for. */
moa_status moa_kv_attend_chunks_bytes(const moa_kv_cfg* cfg, int32_t n_rows, int32_t n_chunks, int32_t max_ctx,
                                      size_t* bytes);
moa_status moa_kv_attend_chunks(const moa_kv_cfg* cfg, const void* kv, int32_t layer, const void* q, int32_t type,
                                int64_t q_stride, int32_t n_rows, const int32_t* chunk_start,
                                const int32_t* chunk_ctx, const int32_t* tables, int32_t n_chunks,
                                int32_t table_len, int32_t max_ctx, float scale, void* out, void* workspace,
                                size_t workspace_bytes, void* hip_stream);

/* Log probabilities of given tokens under rows of logits [n_rows][vocab] of
 * `type`, with the entropy of each row and its top_k (0 .. MOA_MAX_TOP, at
 * most vocab) likeliest tokens:
 *   logprob[r] = log softmax(logits[r])[tokens[r]]   (NaN for a token outside [0, vocab));
 *   entropy[r] = -sum p log p, natural units         (an impossible token, logit -inf, adds 0);
 *   top_ids, top_logprobs [n_rows][top_k], by falling logit, ties to the lower id (NULL when top_k is 0).
 * All results are float32 (ids int32), summed in float32. A row that holds a
 * NaN or +inf, or nothing above -inf, has NaN for every probability; its
 * top_ids still name top_k distinct tokens, the order of NaNs being last. */
enum { MOA_MAX_TOP = 32 };
moa_status moa_score_tokens_bytes(int32_t n_rows, int32_t vocab, int32_t top_k, size_t* bytes);
moa_status moa_score_tokens(const void* logits, int32_t type, int64_t stride, int32_t n_rows, int32_t vocab,
                            const int32_t* tokens, float* logprob, float* entropy, int32_t top_k, int32_t* top_ids,
                            float* top_logprobs, void* workspace, size_t workspace_bytes, void* hip_stream);

#ifdef __cplusplus
}
#endif
#endif /* MOA_H */
