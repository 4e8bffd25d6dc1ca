/* cora.h - C ABI of the MI355X (gfx950) CORA-Diff denoising-step library.
 *
 * One executed denoising step of blockwise masked-diffusion decoding (Section 3
 * of the CORA-Diff paper, "Diffusion Decoding Setup" and "Confidence-Oriented
 * Residual Acceptance"): a dense bidirectional Transformer pass over the whole
 * prompt+generation canvas, per-position top-1 token and confidence (Eq. 1),
 * the persistence counter (Eq. 2), the original low-confidence transfer rule,
 * the residual confidence-and-persistence gate (Eq. 3), the commit of both
 * sets (Eq. 4) and block termination once the active block holds no
 * unresolved position (Fig. 2; "From acceptance to runtime").
 *
 * Conventions
 *  - Every function returns cora_status (0 = CORA_OK, < 0 = error) and never
 *    throws (a failed host allocation inside the library is CORA_ERR_OOM, and a
 *    failed create frees whatever it had allocated).  On error, cora_last_error() returns a thread-local message.  A
 *    failed HIP call inside the library is reported through the status alone:
 *    HIP's last-error state is cleared before the function returns.
 *  - "d_" pointers are device pointers, "h_" pointers are host pointers.  All
 *    caller buffers stay owned by the caller.  The library owns the model
 *    weights and a fixed workspace, both allocated in cora_model_create; no
 *    other entry point allocates device memory.
 *  - bf16 values cross the ABI as raw uint16_t bit patterns.
 *  - Work is enqueued on the caller's HIP stream (`hip_stream`, a hipStream_t;
 *    NULL = the default stream) in stream order.  Only cora_block_decode and
 *    cora_model_copy_tensor wait on the host.
 *  - Every call on one model uses that model's single workspace (activations,
 *    logits or score partials, split-K partials, decode state of
 *    cora_block_decode).  Calls on one model must therefore not overlap: issue
 *    them from one host thread at a time and on one stream, or order the
 *    streams.  Different models are independent.
 *  - Shapes are validated up front; unsupported shapes return
 *    CORA_ERR_UNSUPPORTED, malformed arguments CORA_ERR_INVALID_ARG, HIP
 *    failures CORA_ERR_HIP (with hipGetErrorString text in cora_last_error()).
 */
#ifndef CORA_H
#define CORA_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
  CORA_OK = 0,
  CORA_ERR_INVALID_ARG = -1,
  CORA_ERR_UNSUPPORTED = -2,
  CORA_ERR_OOM = -3,
  CORA_ERR_HIP = -4,
  CORA_ERR_STATE = -5
} cora_status;

#define CORA_MAX_BLOCK_LEN 256

/* Backbone shape.  The paper keeps the backbone frozen and runs one dense pass
 * per executed step (Section 3, first paragraph); the pass is a pre-norm
 * bidirectional Transformer: RMSNorm, QKV projection (+ optional bias),
 * rotate-half RoPE on q and k at absolute positions 0..L-1, non-causal
 * softmax attention (grouped kv heads allowed), output projection, RMSNorm,
 * SwiGLU MLP, final RMSNorm and an untied LM head scaled by logit_scale.
 * Limits: head_dim in {64, 128}; n_heads % n_kv_heads == 0; d_model and
 * n_heads*head_dim multiples of 64; d_model <= 8192; vocab >= 2;
 * 0 <= mask_id < vocab. */
typedef struct {
  int32_t n_layers, d_model, n_heads, n_kv_heads, head_dim, ffn_dim, vocab, mask_id;
  int32_t qkv_bias; /* 0/1: bias on the q, k and v projections */
  float rms_eps, rope_theta, logit_scale;
  double init_std;  /* std of the seeded N(0, std) weights, e.g. 0.02 */
} cora_model_cfg;

/* Blockwise schedule: the generation region is split into blocks of
 * block_len positions decoded left to right, each with a fixed horizon of
 * steps_per_block executed steps (Section 3, "Diffusion Decoding Setup").
 * The transfer rule fixes k_s = floor(block_len / S) + [s < block_len mod S]
 * positions at block step s (a linear split of the block's masked positions).
 * 1 <= steps_per_block <= block_len <= CORA_MAX_BLOCK_LEN.
 * eos_enabled != 0 turns on the EOS-aware controller of the deployment runs
 * (Table 2): after a step's commits, the lowest committed eos_id in the
 * generation region cuts the canvas; unresolved positions after it are
 * resolved as eos_id (decision code 3 inside the active block), committed
 * tokens keep their value, the active block finishes its positions before the
 * EOS and the row then stops (block_idx = number of blocks).  eos_enabled = 0
 * (a zero-initialised struct) keeps the fixed horizon. */
typedef struct {
  int32_t block_len, steps_per_block;
  int32_t eos_enabled, eos_id;
} cora_sched_cfg;

/* Residual gate of Eq. (3): accept i iff c_i >= delta_p and m_i >= m_req,
 * both inclusive, on unresolved active-block positions the transfer rule did
 * not fix.  gate_enabled = 0 gives the original dense decoder (no position
 * accepted).  persist_scope (the counter of Eq. (2) in blockwise decoding):
 * 0 = BLOCK: previous top-1 and counters reset when a block becomes active
 * (its first executed step), only the active block is scored;
 * 1 = GLOBAL: every unresolved generation position is scored on every
 * executed pass and its counter runs across blocks without a reset, so a
 * block whose positions already persisted can end after one pass; transfer
 * and gate still act on the active block only.  Other values return
 * CORA_ERR_UNSUPPORTED. */
typedef struct {
  float delta_p;
  int32_t m_req, gate_enabled, persist_scope;
} cora_gate_cfg;

/* Decode state of a batch of independent rows, all device pointers, updated
 * in place.  B rows, canvas length L = prompt_len + gen_len, gen_len a
 * multiple of block_len, n_blocks = gen_len / block_len.
 *   tokens     int32 [B, L]   canvas x; mask_id where masked
 *   unresolved uint8 [B, L]   1 iff the position is in U
 *   prev_top1  int32 [B, L]   top-1 of the previous executed step, -1 = none
 *   persist    int32 [B, L]   persistence counter m (Eq. 2)
 *   block_idx  int32 [B]      active block; n_blocks once the row is finished
 *   step_idx   int32 [B]      executed steps so far in the active block
 *   top1, conf int32/float [B, n_rows]  Eq. (1) outputs of the scored rows
 *   decision   uint8 [B, block_len]     0 none, 1 fixed by the transfer
 *                                       rule, 2 accepted by the gate
 *   done       int32 [B]      1 iff the active block was resolved by this step
 *                             (or the row was already finished)
 *   passes     int32 [B, n_blocks] or NULL: executed passes per block,
 *                             incremented for every row still decoding */
typedef struct {
  int32_t *tokens;
  uint8_t *unresolved;
  int32_t *prev_top1;
  int32_t *persist;
  int32_t *block_idx;
  int32_t *step_idx;
  int32_t *top1;
  float *conf;
  uint8_t *decision;
  int32_t *done;
  int32_t *passes;
  int32_t B, prompt_len, gen_len;
} cora_state;

typedef struct cora_model cora_model;

/* Allocate weights and workspace for batches of up to max_batch rows of up to
 * max_seq positions, and fill every weight with the counter-based generator:
 * element e (row-major [out, in]) of tensor t is
 *   key = mix(seed); ctr = (t << 40) | e;
 *   h1 = mix(key + (2 ctr + 1) G), h2 = mix(key + (2 ctr + 2) G),
 *   u1 = ((h1 >> 11) + 1) 2^-53, u2 = (h2 >> 11) 2^-53,
 *   w  = bf16_rne(float_rne(init_std * sqrt(-2 ln u1) cos(2 pi u2)))
 * with mix the SplitMix64 finaliser and G = 0x9E3779B97F4A7C15.  Tensor ids:
 * 1 embedding [V, d], 2 LM head [V, d], and 100 + 16 l + j for layer l with
 * j = 0 wq, 1 wk, 2 wv, 3 wo, 4 wg, 5 wu, 6 wd, 7 bq, 8 bk, 9 bv.  Norm
 * weights are 1.  The LM head is held once, in the order in which the few-row
 * LM-head kernel streams it (32-row groups of 1 KB MFMA operand blocks, zero
 * rows up to the next multiple of 32).  Synchronous.  *out is set only on success.
 * CORA_ERR_UNSUPPORTED when an activation matrix of max_batch x max_seq rows
 * (fp32 residual rows, bf16 FFN or attention-head rows, max_seq rounded up to
 * 64) would exceed 2 GB: the kernels address one with 32-bit byte offsets.
 * CORA_ERR_OOM when the device allocation fails. */
cora_status cora_model_create(const cora_model_cfg *cfg, uint64_t seed, int32_t max_batch,
                              int32_t max_seq, void *hip_stream, cora_model **out);
cora_status cora_model_destroy(cora_model *model);

/* Dense forward pass over tokens [B, L] (int32, device) and the LM head on
 * canvas rows [row_begin, row_begin + n_rows) of every batch row: writes
 * bf16 logits [B, n_rows, V] (device, caller-allocated).  When
 * max_batch * n_rows <= 64 the few-row LM-head kernel runs, else the tiled
 * GEMM; both round (sum_k a_k w_k) * logit_scale to bf16 and differ only in
 * fp32 summation order.  Every kernel choice that sets a summation order is
 * made for max_batch rows, so a row's logits do not depend on B.  Parity
 * hook. */
cora_status cora_forward_logits(cora_model *model, const int32_t *d_tokens, int32_t B, int32_t L,
                                int32_t row_begin, int32_t n_rows, uint16_t *d_logits,
                                void *hip_stream);

/* One executed denoising step on every row of `state` that is still decoding:
 * dense pass, LM head on the active block rows of each batch row, then the
 * vocab/gate kernels (Eq. 1, Eq. 2, transfer rule, Eq. 3, Eq. 4, termination;
 * see cora_vocab_gate).  top1/conf are [B, block_len] (the active block's
 * rows) under the BLOCK scope and [B, gen_len] (the generation region, LM head
 * and row reduction in chunks of up to 256 rows) under GLOBAL.  Eq. (1) is
 * computed inside the LM-head pass and no logits are written: when max_batch
 * times the rows scored per batch row (per chunk) is at most 64, the pass
 * streams the weights (per-128-entry partial max / first arg max /
 * sum of exp), else each wavefront's logit columns are reduced in the tiled
 * GEMM's epilogue; the partials are merged in vocab order.  The top-1 is then
 * the same as cora_vocab_gate's on the logits cora_forward_logits writes for
 * those rows, at any B (the kernel choices are made for max_batch).
 * Only a vocabulary too small for the partials to fit the logits buffer takes
 * logits + row reduction.  Asynchronous. */
cora_status cora_denoise_step(cora_model *model, cora_state *state, const cora_sched_cfg *sched,
                              const cora_gate_cfg *gate, void *hip_stream);

/* The vocab/gate kernel alone on caller logits.  d_logits: bf16 [B, n_rows, V];
 * row r of batch row b scores canvas position row_begin + r, or, when
 * row_begin < 0, position lo_b + r where lo_b is the first position of b's
 * active block.  For every row: top-1 token (lowest id among equal maxima,
 * mask_id never predicted) and confidence c = 1 / sum_v exp(l_v - l_max)
 * (fp32).  Then, per batch row still decoding, on its active block: counters
 * reset at block step 0, persistence update on unresolved positions, the
 * k highest-confidence unresolved positions (ties: lower position) fixed
 * (k = k_transfer if >= 0, else the schedule's k_s), the gate on the rest,
 * commit of both sets, and the block/step advance once the block is empty.
 * A fixed row_begin must cover the whole generation region; the GLOBAL
 * persistence scope needs fixed rows (it updates every scored unresolved
 * position).  top1/conf receive [B, n_rows].  Two kernel launches on
 * hip_stream (row reduction, then the decision rules); calls on one state must
 * not overlap.  Asynchronous. */
cora_status cora_vocab_gate(const uint16_t *d_logits, int32_t n_rows, int32_t row_begin,
                            int32_t V, int32_t mask_id, cora_state *state, int32_t k_transfer,
                            const cora_sched_cfg *sched, const cora_gate_cfg *gate,
                            void *hip_stream);

/* For callers that cannot allocate device memory (code under HIP graph capture,
 * tight serving loops, harnesses that forbid allocation): cora_vocab_gate with
 * the same arguments, outputs and error behaviour, computed without any
 * allocation.  Each logits row's vocabulary is split into consecutive ranges,
 * one workgroup each (so few rows still fill the GPU); their partial (max,
 * sum of exp, lowest arg max) go to a fixed device array of the library of
 * CORA_VOCAB_GATE_NOALLOC_MAX_PARTIALS entries (12 bytes each, 3 MiB per GPU,
 * held until the process ends) and are merged in vocab order.  top1 equals
 * cora_vocab_gate's bit for bit; conf differs only in fp32 summation order,
 * so decisions agree except where a cut or threshold lies within that
 * rounding.  B * n_rows above CORA_VOCAB_GATE_NOALLOC_MAX_PARTIALS returns
 * CORA_ERR_UNSUPPORTED.  The array's address is looked up on the first call
 * on a device (the current device, which must own the stream and pointers).
 * Every call on one GPU shares that array: calls that overlap on one GPU
 * (other threads, other streams) race and must be ordered by the caller.
 * No hipMalloc, hipFree or other allocating routine is called, also not on
 * error paths.  Asynchronous. */
#define CORA_VOCAB_GATE_NOALLOC_MAX_PARTIALS 262144
cora_status cora_vocab_gate_noalloc(const uint16_t *d_logits, int32_t n_rows, int32_t row_begin,
                                    int32_t V, int32_t mask_id, cora_state *state,
                                    int32_t k_transfer, const cora_sched_cfg *sched,
                                    const cora_gate_cfg *gate, void *hip_stream);

/* Gated block decode of B prompts (d_prompt int32 [B, prompt_len], device):
 * the canvas starts as prompt + gen_len masks, rows decode independently and
 * each block ends once it holds no unresolved position, skipping its
 * remaining passes.  With batch-row compaction on (the default, see
 * cora_model_set_compaction) a row that has finished all its blocks leaves the
 * dense pass: its final tokens and passes are written out and later passes run
 * on the live rows only.  Writes the final canvas to d_out_tokens int32 [B, L]
 * (device) and the executed passes per block to h_passes int32
 * [B, gen_len / block_len] (host).  If h_total_passes is not NULL it receives
 * the number of dense passes launched (the batch runs while any row decodes).
 * Synchronous on return. */
cora_status cora_block_decode(cora_model *model, const int32_t *d_prompt, int32_t B,
                              int32_t prompt_len, int32_t gen_len, const cora_sched_cfg *sched,
                              const cora_gate_cfg *gate, int32_t *d_out_tokens, int32_t *h_passes,
                              int32_t *h_total_passes, void *hip_stream);

/* ---- Sampling ---------------------------------------------------------------------------
 * A token per logits row from a given random number, device arrays of one entry per row.
 * Over the allowed ids of a row (not mask_id, not NaN, not -inf) in the order of falling
 * logits, equal ones by id, with w_j = exp((l_j - l_0) / temperature):
 *   top_k > 0     keeps the first top_k;
 *   top_p < 1     of those, the fewest whose w reach top_p of their sum (at least one);
 *   min_p > 0     those with w >= min_p (at least one);
 * the token is the first whose running sum of w passes u times the kept sum, 0 <= u < 1.
 * temperature <= 0 or NaN: the first of the order (u unused).  top_k, top_p or min_p may be
 * NULL (off for every row).  Sums are 64-bit, so the token does not depend on their order. */
typedef struct {
  const float *temperature;
  const int32_t *top_k;
  const float *top_p, *min_p;
  const float *u;
} cora_sample_rows;

/* Row r of the bf16 logits [R, V] starts at d_logits + r * ld (elements, ld >= V; any
 * alignment of 2 bytes).  mask_id = -1: no id is left out.  d_token int32 [R]; d_conf float
 * [R] is Eq. (1)'s softmax of the token over the allowed ids at temperature 1, so that a
 * greedy row gives cora_vocab_gate's top1 and conf.  A row without an allowed id gives token
 * -1 and confidence 0; a NaN at an allowed id makes the row's confidence NaN.  Rows that hold
 * +inf, NaN, or finite logits of magnitude >= 2^19 or in (0, 2^-44) that can matter take
 * several passes.  R stays below 2^23, V does not exceed 2^30.  Allocates nothing, needs no
 * workspace.  Asynchronous. */
cora_status cora_vocab_sample(const uint16_t *d_logits, int32_t R, int32_t V, int64_t ld,
                              int32_t mask_id, const cora_sample_rows *rows, int32_t *d_token,
                              float *d_conf, void *hip_stream);

/* cora_vocab_gate with sampled tokens: the B * n_rows rows of the logits are drawn as by
 * cora_vocab_sample (`rows` holds one entry per logits row, in their order) into top1 / conf,
 * then the same decision rules run on them; persistence counts equal draws. */
cora_status cora_vocab_gate_sampled(const uint16_t *d_logits, int32_t n_rows, int32_t row_begin,
                                    int32_t V, int32_t mask_id, cora_state *state,
                                    int32_t k_transfer, const cora_sched_cfg *sched,
                                    const cora_gate_cfg *gate, const cora_sample_rows *rows,
                                    void *hip_stream);

/* ---- Beam search --------------------------------------------------------------------------
 * The W best continuations of each of B requests of K beams.  Row r = b K + k of the bf16 logits
 * [B K, V] (row stride ld, any alignment of 2 bytes) and d_score float [B K] are beam k of request b and
 * its running score.  The candidates of a beam are its allowed ids v (not mask_id, not -inf) with
 *   score + l_v - log sum_u exp(l_u)    over the allowed u;
 * a beam with d_done != 0 (uint8 [B K], NULL: none) has the one candidate done_token with its score
 * unchanged.  A beam whose score is -inf, +inf or NaN has none, nor has one without an allowed id or with a NaN or
 * +inf at one.  In the order of falling scores, equal ones by beam, then by falling logit, then by id,
 * the first W of a request go to d_token, d_parent (the row r) and d_next (the score) [B, W]; places
 * left over get token -1, parent -1 and -inf.  16 terms at a time are added in fp32, these sums and the scores in 64 bits:
 * a row's log sum is off by 1e-7 or so (by arithmetic less than 7e-7 for V <= 2^18, 1.5e-6 for any V), the same for equal rows,
 * and the order that of scores further apart than two of these.  mask_id = -1: no id is left out.  1 <= K, W <= CORA_BEAM_MAX,
 * V <= 2^30, B K <= 2^22.  The outputs overlap no input.
 * workspace of cora_vocab_beam_workspace bytes, 16-byte aligned: used from this call's start to its end on the
 * stream, contents not kept; calls that may overlap and captured graphs that may run at once need one
 * each.  Asynchronous. */
#define CORA_BEAM_MAX 64
cora_status cora_vocab_beam_workspace(int32_t B, int32_t K, int32_t V, int32_t W, size_t *bytes);
cora_status cora_vocab_beam(const uint16_t *d_logits, int32_t B, int32_t K, int32_t V, int64_t ld,
                            int32_t mask_id, const float *d_score, const uint8_t *d_done,
                            int32_t done_token, int32_t W, int32_t *d_token, int32_t *d_parent,
                            float *d_next, void *workspace, size_t workspace_bytes, void *hip_stream);

/* ---- Paged K/V cache ----------------------------------------------------------------------
 * Keeps the K and V of resolved positions, so that a step runs on a chunk of positions per
 * request (its active block, a piece of its prompt, one token) instead of the whole canvas.
 * All arrays are device memory owned by the caller.
 *
 * cora_cache: bf16 K and V of n_layers layers, each [n_pages, n_kv_heads, page_size * head_dim].
 * A page of one head holds 32-key groups of 1 KB blocks in MFMA operand order; element (p, d)
 * (position p of the page, dimension d), with k = p % 32, is at
 *   K: (p/32) 32 hd + (k/4 % 2) 16 hd + (d/32) 512 + (d/8 % 4) 128 + (4 (k/8) + k%4) 8 + d%8
 *   V: (p/32) 32 hd + (d/16) 512 + (k/8) 128 + (d%16) 8 + k%8.
 * Limits: head_dim in {64, 128}; page_size 32, 64, 128 or 256; n_pages * page_size < 2^31;
 * k and v aligned to 16 bytes. */
typedef struct {
  uint16_t *k, *v;
  int32_t n_layers, n_pages, n_kv_heads, page_size, head_dim;
} cora_cache;

/* Which pages B requests hold.  table int32 [B, max_pages]: page of positions
 * [j page_size, (j + 1) page_size); len int32 [B]: cached positions; free int32 [n_pages], a
 * stack of the pages nobody holds, n_free int32 [1] of them.  At the start: len 0, free any
 * permutation of 0 .. n_pages - 1, n_free n_pages (or reset, below). */
#define CORA_CACHE_MAX_BATCH 4096
typedef struct {
  int32_t *table, *len, *free, *n_free;
  int32_t B, max_pages, n_pages, page_size;
  int32_t *refs; /* int32 [n_pages]: requests that hold each page, 0 at the start; NULL: no page has two */
} cora_pages;

/* A chunk per request: positions [start, start + count) of each, their rows one request after
 * another.  start, count int32 [B] are the caller's; cora_cache_plan writes cu int32 [B + 1]
 * (request b's rows are [cu[b], cu[b+1])), status int32 [B] and, for `rows` rows, positions and
 * slots int32 [rows] (slot = page * page_size + position in the page; both -1 in rows from
 * cu[B] on, the slot where the table holds no page of the pool).  `rows` is the capacity: fixed
 * for a program, whatever the live count. */
typedef struct {
  const int32_t *start, *count;
  int32_t *cu, *positions, *slots, *status;
  int32_t rows;
} cora_chunk;

/* Block tables and slot maps from the requests' lengths, on the GPU.  First every request with
 * count < 0 gives its pages back and its len becomes 0.  Then each request with count > 0 gets
 * the pages that positions up to start + count need beyond those of its len, taken off the
 * stack in the order of the requests, and len becomes max(len, start + count); a chunk inside
 * len takes none (its positions are stored anew).  count = 0 leaves a request as it is.
 * A request is refused, with its state left as it was, no rows and its status set, when start is
 * negative or beyond len, or start + count beyond max_pages * page_size (CORA_ERR_INVALID_ARG);
 * when the pages needed up to it exceed the free ones (CORA_ERR_OOM); or when the rows up to it
 * exceed chunk->rows (CORA_ERR_UNSUPPORTED).  "Up to it" counts what the valid requests before it
 * asked for, those refused among them, so that no later request overtakes one that waits for pages
 * or rows; one that needs no page never gets CORA_ERR_OOM.  Status 0 otherwise.  With refs (cora_cache_reorder),
 * a page given back is free once nobody holds it, after those of the requests before the lowest one that
 * gave it back, and a chunk that reaches into a cached page which another request holds too is refused with
 * CORA_ERR_STATE.  reset != 0 forgets every
 * request first: len 0, all pages free, page 0 handed out first.  B <= CORA_CACHE_MAX_BATCH.
 * Allocates nothing.  Asynchronous. */
cora_status cora_cache_plan(cora_pages *pages, cora_chunk *chunk, int32_t reset, void *hip_stream);

/* Every request goes on as its parent: request j gets the positions, K and V that request d_parent[j] (int32
 * [B], -1: none, request j becomes empty) had before the call.  Full pages are shared: pages->refs
 * (needed) counts the requests that hold each.  A last page that is not full stays with the parent's lowest
 * child, the others get copies of it in all layers, 32 positions at a time, in pages off the stack in the
 * order of the requests; where none is left, a request becomes empty with status CORA_ERR_OOM, and so do
 * those behind it that need one.  Before that, the pages that nobody holds any more go onto the stack, in the
 * order of the requests that held them, a page of several at its lowest one's.  A parent outside [-1, B) leaves a
 * request as it is, as its own child, with status CORA_ERR_INVALID_ARG.  Status int32 [B] is 0 otherwise.  d_moves int32
 * [1 + 3 B] receives the number of copies and each one's source, destination and 32-position groups.  What the
 * table holds behind a request's pages stays.  A slot map made before the call is not valid after it.  Allocates
 * nothing.  Asynchronous. */
cora_status cora_cache_reorder(const cora_cache *cache, cora_pages *pages, const int32_t *d_parent,
                               int32_t *d_status, int32_t *d_moves, void *hip_stream);

/* Write a chunk's K and V into the pages of one layer, q and k rotated (rotate-half RoPE: pair
 * (j, j + hd/2) of a head by the angle of the row's position).  d_x rows [q | k | v] of
 * (n_heads + 2 n_kv_heads) head_dim elements, row stride ld: bf16 (x_f32 = 0) or fp32, rounded
 * once.  d_rope: (cos, sin) pairs fp32 [n_pos, head_dim / 2], or NULL for rows already rotated.
 * d_q bf16 [rows, n_heads, head_dim] receives the rotated q (NULL: not wanted).  Of the chunk,
 * positions, slots and cu[B] are read.  Rows from cu[B] on are left alone; a row whose slot or
 * position lies outside the cache or the table is not stored and its q is zero.  The slots of a
 * chunk's rows must differ.  d_x, d_q, d_rope 16-byte aligned, rows too.  CORA_ERR_UNSUPPORTED where
 * rows and heads exceed one launch (2^24 workgroups of 32 rows and a head of 128 or two of 64 at the
 * least), as in cora_cache_attention (64 rows and query heads of a kv head).  Asynchronous. */
cora_status cora_cache_store(const cora_cache *cache, int32_t layer, const void *d_x, int32_t x_f32,
                             int64_t ld, int32_t n_heads, const cora_chunk *chunk, int32_t B,
                             const float *d_rope, int32_t n_pos, uint16_t *d_q, void *hip_stream);

/* Attention of the chunk's rows over their requests' pages: query head h reads kv head
 * h / (n_heads / n_kv_heads); keys j < len, and with causal != 0 j <= the row's position.
 * d_q, d_out bf16 [rows, n_heads, head_dim].  A row without a key, or whose scores are all -inf, is
 * zero; rows before cu[0]
 * and from cu[B] on are left alone; what the pages hold behind len is never used.  Read: chunk start, cu; pages
 * table, len.  max_count and max_len are the most rows of a request and the longest len to
 * expect (<= 0: rows and max_pages * page_size); they choose tiles and key ranges, and with
 * them the order of the sums, and longer requests are still computed in full.  workspace of
 * cora_cache_attention_workspace bytes, 16-byte aligned (NULL when that is 0): used from
 * this call's start to its end on the stream, contents not kept; calls that may overlap and
 * captured graphs that may run at once need one each.  Asynchronous. */
cora_status cora_cache_attention_workspace(int32_t n_heads, int32_t n_kv_heads, int32_t head_dim,
                                           int32_t B, int32_t rows, int32_t max_count,
                                           int32_t max_len, size_t *bytes);
cora_status cora_cache_attention(const cora_cache *cache, int32_t layer, const cora_pages *pages,
                                 const cora_chunk *chunk, const uint16_t *d_q, int32_t n_heads,
                                 int32_t max_count, int32_t max_len, int32_t causal, float scale,
                                 uint16_t *d_out, void *workspace, size_t workspace_bytes,
                                 void *hip_stream);

/* The model's pass over a planned chunk against its cache: embedding of d_tokens int32
 * [chunk->rows], every layer with its K and V stored at the chunk's slots and its queries
 * attending to the request's pages (both directions, or causal), LM head on every row: bf16
 * logits [rows, V].  The cache has the model's layers, kv heads and head_dim; its K holds the
 * head's dimensions pair-interleaved (j at 2j, j + hd/2 at 2j + 1).  Rows from cu[B] on compute on
 * whatever d_tokens holds there, their logits are unspecified.  max_seq bounds the rows of a
 * pass, not their positions, which go as far as the table's.  Kernel choices follow chunk->rows, B,
 * max_count and max_len, not the live rows.  CORA_ERR_UNSUPPORTED when rows * (n_heads + 2 n_kv_heads) * head_dim
 * exceeds the model's fp32 workspace (2^25 elements on this GPU) or rows exceed max_batch *
 * max_seq: run a longer prompt in several chunks.  Uses the model's workspace.  Asynchronous. */
cora_status cora_forward_cached(cora_model *model, const cora_cache *cache, const cora_pages *pages,
                                const cora_chunk *chunk, const int32_t *d_tokens,
                                int32_t max_count, int32_t max_len, int32_t causal,
                                uint16_t *d_logits, void *hip_stream);

/* ---- 8-bit rows and their products ---------------------------------------------------------
 * A matrix [rows, cols] in 8-bit floating point (e4m3: OCP's, without infinities), each 128 columns of
 * a row with a power of two as their scale.  Device arrays owned by the caller, of
 * cora_rows_bytes bytes, data aligned to 16 bytes, scale to 4.  With groups of 16 rows, blocks of
 * 128 columns, nb = ceil(cols / 128) and nq = ceil(cols / 512), element (r, c) is at
 *   data:  ((r/16) nb + c/128) 2048 + (c%128 / 64) 1024 + (c/16 % 4) 256 + (r%16) 16 + c%16
 * and its scale, the exponent + 127, at
 *   scale: ((r/16) nq + c/512) 64 + (r%16) 4 + c/128 % 4.
 * Rows and columns up to multiples of 16 and 128 are zero, the scales of blocks past the last one 127.  A scale of 255, which
 * cora_quantize_rows never writes, stands for NaN: what its block's numbers are multiplied into is NaN.
 * Limits: rows <= 2^27, cols <= 2^20. */
typedef struct {
  uint8_t *data, *scale;
  int32_t rows, cols;
} cora_rows8;
cora_status cora_rows_bytes(int32_t rows, int32_t cols, size_t *data_bytes, size_t *scale_bytes);

/* x [rows, cols] to 8 bits, row stride ld (elements, ld >= cols): bf16 (x_f32 = 0, any alignment of 2
 * bytes) or fp32 (any of 4).  The scale of a block is the least power of two, 2^-127 at the least, with
 * which 448 reaches the largest finite magnitude in it (1 for a block of zeros); values are x / scale
 * rounded to e4m3 once, to nearest even.  NaN and infinities become NaN.  Writes the whole arrays, their padding
 * included; they do not overlap x.  ceil(rows / 16) * ceil(cols / 512) stays below 2^23.  Asynchronous. */
cora_status cora_quantize_rows(const void *d_x, int32_t x_f32, int64_t ld, const cora_rows8 *out,
                               void *hip_stream);

/* out[m, n] = sum over k of a[m, k] w[n, k], + d_bias[n] (fp32 [N], NULL: none): M = a->rows, N = w->rows, both
 * of the same cols: bf16 (out_f32 = 0) or fp32 [M, N], row stride ld (elements, ld >= N), no overlap with the
 * inputs.  fp32 results: exact products, sums of 32 bits.  bf16 results: the 8-bit instruction's, which adds a block's
 * products to a sum of 32 bits without the bits below 2^-13 of the largest of them (in the mean 1.6e-5 of the
 * result where they are of a size, 5e-5 where they spread widely; the one rounding to bf16 is off by up to 2^-8).  Sums over cols are split by sizes alone, so that an output's bits do
 * not change with what the other rows hold.  M <= 2^21, N <= 2^25, M N <= 2^40.  workspace of cora_rows_product_workspace bytes, 16-byte
 * aligned (NULL when that is 0): used from this call's start to its end on the stream, contents not
 * kept; calls that may overlap and captured graphs that may run at once need one each.  cols = 0 is
 * refused; M = 0 or N = 0 does nothing.  Asynchronous. */
cora_status cora_rows_product_workspace(int32_t M, int32_t N, int32_t cols, int32_t out_f32,
                                        size_t *bytes);
cora_status cora_rows_product(const cora_rows8 *a, const cora_rows8 *w, const float *d_bias,
                               void *d_out, int32_t out_f32, int64_t ld, void *workspace,
                               size_t workspace_bytes, void *hip_stream);

/* The layers' matrices in 8 bits, in memory of the caller's (256-byte aligned, cora_model_quantized_bytes
 * bytes, their layout the library's): cora_model_quantize rounds them, each row's blocks of 128 columns as
 * cora_quantize_rows does.  Embedding, biases and LM head stay as they are.  cora_forward_quantized is
 * cora_forward_cached on these: the inputs of the four products of a layer (normalised rows, attention output,
 * normalised rows, silu(gate) * up of the bf16 results) are rounded to 8 bits alike, the sums are fp32.  One cache serves
 * both passes.  Splits and tiles follow chunk->rows alone.  workspace of cora_forward_quantized_workspace bytes,
 * 256-byte aligned: used from this call's start to its end on the stream, like the model's workspace, which it uses too.
 * Asynchronous. */
cora_status cora_model_quantized_bytes(cora_model *model, size_t *bytes);
cora_status cora_model_quantize(cora_model *model, void *d_weights, size_t bytes, void *hip_stream);
cora_status cora_forward_quantized_workspace(cora_model *model, int32_t rows, size_t *bytes);
cora_status cora_forward_quantized(cora_model *model, const void *d_weights, size_t weights_bytes,
                                   const cora_cache *cache, const cora_pages *pages,
                                   const cora_chunk *chunk, const int32_t *d_tokens, int32_t max_count,
                                   int32_t max_len, int32_t causal, uint16_t *d_logits, void *workspace,
                                   size_t workspace_bytes, void *hip_stream);

/* Copy weight tensor `tensor_id` (ids as in cora_model_create) to host memory
 * in its logical row-major [out, in] layout as bf16 bits (biases too).
 * `bytes` must equal the tensor's size.  Synchronous. */
cora_status cora_model_copy_tensor(cora_model *model, int32_t tensor_id, void *h_dst, size_t bytes);

/* Kernel timing: while enabled, every launch of the gate/up SwiGLU GEMM is
 * dispatched with a pair of HIP events (hipExtLaunchKernel) that the dispatch
 * stamps with the kernel's start and end on the launching stream.  Enabling
 * and disabling keep what was recorded, so timing can cover a sample of the
 * launches.  Reading waits for the recorded events, returns the summed event
 * time (ms) and the number of timed launches since the previous read, and
 * clears both. */
cora_status cora_model_set_timing(cora_model *model, int32_t enable);
cora_status cora_model_read_timing(cora_model *model, double *total_ms, int64_t *launches);

/* Batch-row compaction in cora_block_decode (rows decode independently, so
 * dropping finished rows from the dense pass changes no live row's inputs).
 * Every kernel choice that sets an output's summation order (split-K count,
 * attention key-range parts, LM-head kernel and vocab partial layout) is made
 * for max_batch rows, never for the live row count, so a row's tokens and
 * passes are bit-identical with compaction on or off and equal to a decode of
 * that row alone on the same model.  enable != 0 turns it on (default), 0 off. */
cora_status cora_model_set_compaction(cora_model *model, int32_t enable);

/* Device bytes the model holds (weights + workspace). */
cora_status cora_model_device_bytes(cora_model *model, size_t *weight_bytes, size_t *workspace_bytes);

const char *cora_last_error(void);

#ifdef __cplusplus
}
#endif

#endif /* CORA_H */
