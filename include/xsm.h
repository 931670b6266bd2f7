/*
 * xsm: multi-head speculative decoding for cross-attention conditioned
 * auto-regressive mesh transformers on one NVIDIA B200 (sm_100a).
 *
 * C ABI.  Every pointer is marked HOST or DEVICE.  The library allocates no
 * device memory: the caller hands it a weight buffer and a workspace and keeps
 * both alive until xsm_destroy.  All work is enqueued on the stream given to
 * xsm_create.  Functions return XSM_OK or an error code; xsm_last_error gives
 * the text.  Argument and capacity errors are found on the host before any
 * launch.  A device-side wait that runs out of patience ends the kernel
 * cleanly and surfaces as XSM_ERR_TIMEOUT at the next synchronising call.
 *
 * Notation follows the paper: s is the number of committed positions whose
 * keys and values are in the cache, x_s the last committed token (not yet in
 * the cache), x_{s+1..s+K} the drafted tokens, K = n_draft the number of
 * decoding heads (the paper's D), V the vocabulary, c the condition latents.
 */
#ifndef XSM_H
#define XSM_H

#include <stddef.h>
#include <stdint.h>

#if defined(__GNUC__)
#define XSM_API __attribute__((visibility("default")))
#else
#define XSM_API
#endif

#ifdef __cplusplus
extern "C" {
#endif

typedef struct xsm_ctx xsm_ctx;

typedef enum {
    XSM_OK = 0,
    XSM_ERR_INVALID_ARG = 1,
    XSM_ERR_STATE = 2,      /* call out of order, e.g. a step before xsm_prefill */
    XSM_ERR_CAPACITY = 3,   /* workspace, page pool or max_seq_len too small */
    XSM_ERR_CUDA = 4,
    XSM_ERR_TIMEOUT = 5     /* a bounded device-side wait expired */
} xsm_status;

#define XSM_MAX_DRAFT 16

/* Model shape.  Weights are one flat DEVICE buffer of `dtype` elements in this
 * order, every matrix row-major [out, in] (y = W x), no biases:
 *   E[V,d]
 *   per layer: g1[d] Wq[d,d] Wk[d,d] Wv[d,d] Wo[d,d]
 *              g2[d] Wqc[d,d] Wkc[d,d_cond] Wvc[d,d_cond] Woc[d,d]
 *              g3[d] Wgate[f,d] Wup[f,d] Wdown[d,f]
 *   gf[d] W0[V,d]
 *   per head i=1..K: W1[head_hidden,d] Wout[V,head_hidden]                        (head_kind 0)
 *                    Wq[d,d] Wk[d,d_cond] Wv[d,d_cond] Wo[d,d] Wout[V,d]          (head_kind 1)
 * Block (Sec. 4.1): pre-norm residual, self-attention (RoPE, causal, cached),
 * cross-attention to c, gated feed-forward network; RMSNorm gains g*.
 * Requirements: n_heads*d_head == d_model, head_hidden == d_model, d_model and d_ff multiples of 128 with rows
 * of at most 16 KB (d_model additionally at most 4 KB per row), d_cond a multiple of 32, d_head 32, 64 or 128,
 * page_size a multiple of 32 with page_size*d_head <= 8192 (bf16) / 16384 (fp32), n_draft <= 15,
 * max_batch*(n_draft+1) <= 128.  fp32 models (the parity configuration): at most 24 token rows per step. */
typedef struct {
    int n_layers, d_model, n_heads, d_head, d_ff, vocab, n_cond, d_cond;
    int n_draft;        /* K; 0 = plain one-token-per-step decoding (Table 3 row A) */
    int head_hidden;
    int head_kind;      /* 0: MLP head, logits = Wout (g + SiLU(W1 g)) (Table 3 rows B, C);
                           1: cross-attention head (Eq. 3), logits = Wout (g + Wo Attn(Wq g, Wk c, Wv c)) */
    int dtype;          /* 0: fp32 weights and cache; 1: bf16 weights, fp16 cache, fp32 arithmetic */
    int page_size;      /* tokens per cache page */
    int max_batch;
    int max_seq_len;    /* largest s; the cache holds max_seq_len + K + 1 positions per sequence */
    float rope_theta, rms_eps;
    int bos_id, eos_id; /* eos_id < 0: no end token */
} xsm_model_config;

/* Verification (Sec. 4.2, Sec. 5.4) and resampling (Appendix, independent sampling). */
typedef struct {
    int verify_mode;    /* 0: strict greedy (top-1); 1: draft within the backbone's top k_accept;
                           2: backbone probability of the draft > delta */
    int k_accept;
    float delta;
    int sample_mode;    /* 0: argmax; 1: every candidate on its own from softmax(top k_sample logits / temperature)
                           (the Appendix's independent sampling); 2: x_{s*} as in mode 1, the K drafts as one path
                           of the Appendix's top-k_sample probability tree over the heads (path weight = product of
                           the tokens' softmax probabilities, paths below 1e-5 pruned) */
    int k_sample;       /* <= 64; mode 2: <= 8 and k_sample ^ n_draft <= 4096 */
    float temperature;
    uint64_t seed;      /* Philox4x32-10 key; sequence b uses (seed_lo ^ b, seed_hi) */
} xsm_decode_config;

typedef struct {
    uint64_t steps;                         /* decoding steps, summed over sequences */
    uint64_t tokens;                        /* committed tokens, summed over sequences */
    uint64_t accept_hist[XSM_MAX_DRAFT + 1];/* steps that accepted a drafts */
    double wall_ms;                         /* device time of the last xsm_generate */
    double scr;                             /* tokens / steps (Sec. 5.1) */
} xsm_stats;

/* Bytes of the flat weight buffer for this shape: the backbone of Sec. 4.1 with its decoder W0 (Eq. 2) and the
 * K decoding heads, in the layout given above. */
XSM_API size_t xsm_weights_bytes(const xsm_model_config *cfg);

/* Bytes of workspace that hold max_batch sequences of max_seq_len positions
 * (page pool, cross-attention cache, activations, decoding state). */
XSM_API size_t xsm_workspace_bytes(const xsm_model_config *cfg);

/* Algorithm 1's inputs other than the condition: the backbone M and the decoding
 * heads {H_i}, as one weight buffer in the layout above.
 * Binds a context to DEVICE weights and DEVICE workspace (both 256-byte
 * aligned, borrowed until xsm_destroy) and a CUDA stream (cudaStream_t passed
 * as void*, may be NULL for the default stream).  A workspace larger than
 * xsm_workspace_bytes adds pages to the shared pool; a smaller one that still
 * holds at least one sequence's pages is accepted and XSM_ERR_CAPACITY is then
 * decided per xsm_prefill.  bf16 models keep cached keys and values as fp16:
 * a key or value element beyond +-65504 is stored as +-65504 without any status
 * (projections of normalised activations by N(0, 0.02) weights stay far below). */
XSM_API xsm_status xsm_create(const xsm_model_config *cfg, const void *d_weights, void *d_workspace,
                      size_t workspace_bytes, void *cuda_stream, xsm_ctx **out);

/* Algorithm 1, line 1, for `batch` independent meshes: computes the cross-
 * attention keys and values of d_cond (DEVICE, [batch, n_cond, d_cond], model
 * dtype), runs prompt tokens 0..prompt_len-2 into the cache, sets x_s to the
 * last prompt token, s = prompt_len-1, draws the K initial drafts uniformly on
 * [0, V) and resets the step counters.  d_prompt: DEVICE int32 [batch,
 * prompt_len].  The prefill kernels and the
 * ingestion of the prompt are then enqueued without waiting. */
XSM_API xsm_status xsm_prefill(xsm_ctx *ctx, int batch, const void *d_cond, const int32_t *d_prompt,
                       int prompt_len, const xsm_decode_config *dc);

/* One iteration of Algorithm 1's loop (lines 3-12) for every unfinished
 * sequence: backbone over x_{s..s+K} against the paged cache, heads, verify,
 * resample, commit, roll back.  d_new_tokens: DEVICE int32 [batch, K+1], the
 * tokens committed by this step, padded with -1; d_n_new: DEVICE int32
 * [batch] (0 for a finished sequence).  Either may be NULL.  Asynchronous. */
XSM_API xsm_status xsm_spec_step(xsm_ctx *ctx, int32_t *d_new_tokens, int32_t *d_n_new);

/* The paper has no counterpart of this call; it serves hosts on a path that must not allocate device memory or
 * synchronise the device.  xsm_spec_step with one difference: the kernels of the step are launched one by one
 * instead of as a recorded graph, whose recording and first launch may make the driver allocate.  The partial
 * results that the key splits of an attention stage hand to one another travel through shared memory and need no
 * scratch.  A batch for which they would exceed 1 MiB (batch * n_heads * splits * (K+1) * (d_head+2) floats, twice)
 * is refused with XSM_ERR_CAPACITY, as it was when they lay in an array of the library.  The two step calls may
 * alternate freely on one context.  Arguments and results as xsm_spec_step.  Asynchronous. */
XSM_API xsm_status xsm_spec_step_static(xsm_ctx *ctx, int32_t *d_new_tokens, int32_t *d_n_new);

/* Algorithm 1's loop (line 2: while s < L_max and no EOS is committed) and its
 * output x_{0:i_EOS} (line 14), for every mesh of the batch.
 * Runs steps until every sequence has committed max_new_tokens tokens since
 * xsm_prefill, met EOS, or reached max_seq_len.  d_tokens: DEVICE int32
 * [batch, max_new_tokens] (x_1, x_2, ...; unused tail -1); d_lengths: DEVICE
 * int32 [batch].  host_stats (HOST, may be NULL) is filled before returning.
 * Synchronises the stream.  XSM_ERR_TIMEOUT where a device-side wait of the
 * request ran out: the tokens are void, and xsm_prefill starts afresh. */
XSM_API xsm_status xsm_generate(xsm_ctx *ctx, int max_new_tokens, int32_t *d_tokens, int32_t *d_lengths,
                        xsm_stats *host_stats);

/* The same job from HOST buffers: copies h_cond ([batch, n_cond, d_cond],
 * model dtype) and h_prompt to the device, prefills, generates, and copies
 * tokens and lengths back to h_tokens / h_lengths.  For callers that hold
 * nothing on the device; staging space comes from the workspace. */
XSM_API xsm_status xsm_generate_host(xsm_ctx *ctx, int batch, const void *h_cond, const int32_t *h_prompt,
                             int prompt_len, const xsm_decode_config *dc, int max_new_tokens,
                             int32_t *h_tokens, int32_t *h_lengths, xsm_stats *host_stats);

/* Ends the context (waits for its stream); weights and workspace go back to the caller. */
XSM_API xsm_status xsm_destroy(xsm_ctx *ctx);

/* Text of the last error of this context (or, when ctx is NULL, of the last failed call of this thread that had no context). */
XSM_API const char *xsm_last_error(const xsm_ctx *ctx);

/* Number of kernels this context has launched so far. */
XSM_API uint64_t xsm_kernel_launches(const xsm_ctx *ctx);

/* ---- inspection, for tests and parity checks; what reads or replaces state synchronises the stream ---- */

/* Logits of the last step: h_logits0 HOST float [batch, K+1, V] (Eq. 2 before the
 * softmax), h_head_logits HOST float [K, batch, K+1, V].  Either may be NULL. */
XSM_API xsm_status xsm_debug_get_logits(xsm_ctx *ctx, float *h_logits0, float *h_head_logits);

/* Cached keys and values of positions pos0..pos0+n-1 of one sequence and layer,
 * widened to float: h_k, h_v HOST float [n, d_model]. */
XSM_API xsm_status xsm_debug_get_kv(xsm_ctx *ctx, int layer, int seq, int pos0, int n, float *h_k, float *h_v);

/* Replaces the drafted tokens x_{s+1..s+K} of every sequence: h_drafts HOST int32 [batch, K]. */
XSM_API xsm_status xsm_debug_set_drafts(xsm_ctx *ctx, const int32_t *h_drafts);

/* Decoding state: h_len [batch] (s), h_window [batch, K+1] (x_s and drafts), h_finished
 * [batch], h_pages [batch] (pages held), h_free_pages [1].  Any may be NULL. */
XSM_API xsm_status xsm_debug_get_state(xsm_ctx *ctx, int32_t *h_len, int32_t *h_window, int32_t *h_finished,
                               int32_t *h_pages, int32_t *h_free_pages);

/* Runs one decoding step (as xsm_spec_step does, without returning its tokens) and records its timeline:
 * h_times HOST uint64 [n_rows][n_ctas] nanoseconds of the GPU's global timer; row 0 = the step starts, row
 * 1 + 2p = stage p of the step is past its wait for the stage before, row 2 + 2p = stage p is done; one column
 * for each of a stage's first n_ctas CTAs; 0 = the stage has no such CTA, or it had nothing to do.
 * capacity = number of uint64 words h_times can hold.  Synchronises the stream. */
XSM_API xsm_status xsm_debug_trace_step(xsm_ctx *ctx, uint64_t *h_times, size_t capacity, int *n_rows, int *n_ctas);

/* Load generator for Sec. 5.1's speedup = SCR x latency(K = 0) / latency(K): from the next step on, the drafts of
 * every sequence are taken from h_tokens (HOST int32 [batch, n], token of every absolute position 0..n-1) instead
 * of from the decoding heads; at step t the first floor((t+1) a) - floor(t a) drafts are left intact and the others
 * are made wrong (a = mean_accept in [0, K]); the token resampled at the first rejected position is replaced by the
 * script's too.  With a script that the backbone reproduces (its own greedy continuation under strict-greedy
 * verification) the accept length of every step is forced, and SCR = 1 + a; where the backbone's two best logits
 * nearly tie and it disagrees with the script, that one step accepts less and the run stays on the script.
 * h_tokens == NULL or n == 0 turns it off (without waiting); xsm_prefill turns it off too. */
XSM_API xsm_status xsm_debug_set_script(xsm_ctx *ctx, const int32_t *h_tokens, int n, float mean_accept);

/* Bounds of the device-side waits: polls of one word in memory and tries of one shared-memory barrier before a
 * CTA gives up and raises XSM_ERR_TIMEOUT.  0 restores the default (2^21, 2^22). */
XSM_API xsm_status xsm_debug_set_wait_limits(xsm_ctx *ctx, uint32_t polls, uint32_t barrier_tries);

/* Launches stage `stage` (0-based: eight per layer, seven where the cross-attention projects its
 * own queries, then the tail) of the current step alone, without advancing the
 * step counter.  A stage that does not follow the one launched last waits for its turn until the limit above
 * runs out; the status then shows at the next synchronising call, and xsm_prefill starts afresh. */
XSM_API xsm_status xsm_debug_launch_stage(xsm_ctx *ctx, int stage);

/* How one decoding step of `batch` sequences (prompt_positions 0), or a chunk of so many positions of each of their prompts, is cut over
 * a chip of `sms` SMs on which clusters[s] clusters of s = 2..8 CTAs run at a time (HOST int32 [9]; NULL: the current device).  Nothing
 * is launched, and with `clusters` no device is needed.  h_stages HOST int32 [capacity][8], a row for every kernel: its kind (0: tensor
 * cores of the 5th generation; 1: mma.sync; 2: fp32; 3: attention; 4: tail; 5: embedding) and, for kind 0, what it does (0: q, k, v; 1:
 * residual; 2: cross q; 3: gate/up; 4: logits; 6: head out-projection), threads, CTAs of a cluster, token rows of a tile, token rows that
 * a CTA finishes, columns of tensor memory, bytes of shared memory that a CTA takes at least.  Returns the number of kernels, 0 where
 * there is no such step. */
XSM_API int xsm_debug_plan(const xsm_model_config *cfg, int batch, int prompt_positions, int sms, const int32_t *clusters,
                           int32_t *h_stages, int capacity);

/* Launches the stages of a step one after the other, without overlap, instead of as a recorded graph (1) or back (0). */
XSM_API xsm_status xsm_debug_set_phase_launch(xsm_ctx *ctx, int on);

/* ---- operators on a caller's own paged cache and on a caller's own logits ----
 *
 * What a decoder with another block than this library's needs next to it: keys and values appended to pages with the
 * rotation of the positions, attention of the newest tokens over the pages, log probabilities of given tokens with
 * their gradient.  No xsm_ctx is involved; the library allocates no device memory and keeps none of the arrays of a call.  Every call
 * is enqueued on the CUDA stream that is handed to it (cudaStream_t as void*, NULL: the default stream) of the current device, waits for
 * nothing and may be captured.  Errors are found on the host before the launch; their text is xsm_last_error(NULL) of the same thread.
 * What only the device knows (page numbers, lengths, tokens) is bounded there: see each call.  Element types: */
typedef enum { XSM_F32 = 0, XSM_BF16 = 1, XSM_F16 = 2 } xsm_dtype;

/* Pools of keys and of values, DEVICE [n_pages][n_kv_heads][page_size][d_head] with strides in elements (the elements of a row are
 * neighbours; [n_pages][page_size][n_kv_heads][d_head] is the same with other strides).  Position p of a sequence is row p mod page_size
 * of page block_table[sequence][p / page_size].  d_head 32, 64, 96, 128 or 256, page_size a multiple of 16, pools 16-byte aligned, strides
 * multiples of 16 bytes. */
typedef struct {
    int64_t page_stride, head_stride, row_stride;
    int32_t n_pages, n_kv_heads, page_size, d_head, dtype;
} xsm_kv_config;

typedef struct xsm_kv xsm_kv;      /* HOST description of two pools; borrows them until xsm_kv_destroy */
XSM_API xsm_status xsm_kv_create(const xsm_kv_config *cfg, void *d_k, void *d_v, xsm_kv **out);
XSM_API xsm_status xsm_kv_destroy(xsm_kv *kv);

/* Appends m new tokens to each of `batch` sequences: token j of sequence b goes to position starts[b] + j, if j < counts[b].  Keys, and
 * queries where there are any, are rotated by their position before: pair i of the first rope_dims elements of a head, (i, i + rope_dims/2)
 * or with `interleaved` (2i, 2i + 1), by the angle whose cosine and sine are rope[position][i]; the other elements pass.  Values
 * pass.  Arithmetic in fp32, rounded once to the pool's type (fp16: beyond +-65504 stored as +-65504) and to in_dtype for q_out.
 * A token without a place (a position below 0 or beyond the table's or, where there is one, the rope's last; a page number outside the pool) is not
 * written; the row of q_out of a token that is not to be appended (j >= counts[b]), or whose position the rope does not have, is zero.
 * q, k, v, q_out: DEVICE, strides in elements of sequence, token, head; neighbouring elements of a head.  q_out may be q. */
typedef struct {
    const void *q, *k, *v;                /* in_dtype [batch][m][n_heads or n_kv_heads][d_head]; q may be NULL */
    void *q_out;                          /* in_dtype [batch][m][n_heads][d_head] */
    const int32_t *block_table;           /* DEVICE [batch][max_pages]; may be NULL where max_pages is 0 */
    const int32_t *starts, *counts;       /* DEVICE [batch]; counts may be NULL: m each */
    const float *rope;                    /* DEVICE [rope_positions][rope_dims/2][2] cosine, sine; NULL: no rotation */
    int64_t q_stride[3], k_stride[3], v_stride[3], q_out_stride[3], table_stride;
    int32_t batch, m, n_heads, in_dtype, max_pages, rope_positions, rope_dims, interleaved;
} xsm_kv_append_args;
XSM_API xsm_status xsm_kv_append(const xsm_kv *kv, const xsm_kv_append_args *a, void *cuda_stream);

/* Attention of the m newest tokens of each sequence (1 to 16) over its pages.  Query j of sequence b, of n_b = counts[b] (NULL: m), sees the
 * positions t < lengths[b] and, with `causal`, t <= p = lengths[b] - n_b + j, with `window` > 0 also t > p - window.  For every query head,
 * which reads key head (head / (n_heads / n_kv_heads)):  out = sum_t softmax_t(scale q.k_t) v_t,  lse = log sum_t exp(scale q.k_t).
 * Where nothing is visible, and for j >= n_b, out is zero and lse -infinity.  What unseen positions hold does not matter, infinities and
 * NaN included; in what a row does see they may make that row's results NaN or infinite, never another row's.  Lengths beyond the table's
 * end there; pages whose number lies outside the pool are not seen.
 * Sums and softmax in fp32; the weights of 16-bit values enter as two parts of the pools' type, with an error of 2^-16 (bf16), 2^-22 and 2^-40 of the
 * row's largest weight (fp16).  q_dtype is the pool's type, or, over an fp16 pool, any: queries then enter as fp16 (fp32 ones as two parts of it):
 * beyond +-65504 they are infinite, and their smallest step is 2^-24 (bf16 ones below 2^-17 lose bits).
 * workspace: DEVICE, xsm_kv_attend_workspace bytes, 16-byte aligned, zeroed by the caller before its first use; calls that share
 * one follow each other on one stream.  Its first 32-bit word is XSM_ERR_TIMEOUT once a bounded wait of the device has run out, and the
 * results of that call are then void. */
typedef struct {
    const void *q;                        /* q_dtype [batch][m][n_heads][d_head], strides as above, 16-byte aligned */
    void *out;                            /* likewise */
    float *lse;                           /* [batch][m][n_heads], may be NULL */
    const int32_t *block_table;           /* DEVICE [batch][max_pages]; may be NULL where max_pages is 0 */
    const int32_t *lengths, *counts;      /* DEVICE [batch]: positions in the cache, the new ones included */
    void *workspace;
    int64_t q_stride[3], out_stride[3], table_stride, workspace_bytes;
    int32_t batch, m, n_heads, q_dtype, max_pages, causal, window;
    float scale;
} xsm_kv_attend_args;
XSM_API size_t xsm_kv_attend_workspace(const xsm_kv *kv, int batch, int m, int n_heads);
XSM_API xsm_status xsm_kv_attend(const xsm_kv *kv, const xsm_kv_attend_args *a, void *cuda_stream);
/* Tries of a shared-memory barrier before a wait of the following xsm_kv_attend calls gives up (0: the default, 2^22).  starve: these calls fetch no
 * keys, so that their waits run out. */
XSM_API xsm_status xsm_debug_kv_waits(xsm_kv *kv, uint32_t tries, int starve);

/* For a caller that keeps a workspace for each graph that it records.  xsm_capture_id: the number of the capture that the stream takes part in, 0: none.
 * xsm_capture_watch: *out belongs to the graph that is being recorded on the stream; xsm_capture_gone says 1, once, when that graph and all that was
 * instantiated of it are destroyed, and frees it.  xsm_capture_mode: what the calling thread may do while streams are recorded (cudaStreamCaptureMode);
 * returns the mode before, or -1. */
typedef struct xsm_capture xsm_capture;
XSM_API uint64_t xsm_capture_id(void *cuda_stream);
XSM_API xsm_status xsm_capture_watch(void *cuda_stream, xsm_capture **out);
XSM_API int xsm_capture_gone(xsm_capture *c);
XSM_API int xsm_capture_mode(int mode);

/* Log probabilities under softmax(logits / temperature), of `rows` rows of `vocab` logits:
 *   lse = log sum_j exp(z_j),  logprob = z_token - lse,  entropy = -sum_j p_j log p_j,  z = logits / temperature, p = exp(z - lse),
 * and the `top` (0 to 32) largest logits, equal ones by the lower index first: top_ids, top_logprobs = z - lse.
 * A token outside [0, vocab) is no token: its logprob is 0.  Logits of -infinity have no part (p log p = 0); a row that has
 * nothing else has lse and logprobs of -infinity and entropy 0.  A row with NaN or +infinity has NaN results; NaN ranks below everything. */
typedef struct {
    const void *logits;                   /* DEVICE dtype [rows][vocab], row stride in elements */
    const void *tokens;                   /* DEVICE int32 or int64 [rows], stride in elements */
    float *logprob, *entropy, *lse;       /* DEVICE [rows] */
    int32_t *top_ids;                     /* DEVICE [rows][top] */
    float *top_logprobs;                  /* DEVICE [rows][top] */
    int64_t row_stride, token_stride;
    int32_t rows, vocab, dtype, token_bytes, top;
    float temperature;
} xsm_logprob_args;
XSM_API xsm_status xsm_token_logprobs(const xsm_logprob_args *a, void *cuda_stream);

/* The gradient of sum_rows (g logprob + g_entropy entropy + g_lse lse + sum_i g_top_i top_logprob_i) by the logits, in their type:
 *   d_j = ([j = token] g + sum_i [j = top_ids_i] g_top_i - p_j (g + sum_i g_top_i - g_lse) - g_entropy p_j (log p_j + entropy)) / temperature,
 * from lse, entropy and top_ids of the call above.  g counts only where there is a token.  Rows with an lse of -infinity have gradient 0.
 * d_logits may be logits. */
typedef struct {
    const void *logits, *tokens;          /* as above */
    const float *lse, *entropy;           /* DEVICE [rows]; entropy may be NULL without g_entropy */
    const int32_t *top_ids;               /* DEVICE [rows][top]; NULL with top 0 */
    const float *g_logprob, *g_entropy, *g_lse;      /* DEVICE [rows], strides in elements; each may be NULL */
    const float *g_top;                   /* DEVICE [rows][top], may be NULL */
    void *d_logits;                       /* DEVICE dtype [rows][vocab] */
    int64_t row_stride, token_stride, g_logprob_stride, g_entropy_stride, g_lse_stride, d_row_stride;
    int32_t rows, vocab, dtype, token_bytes, top;
    float temperature;
} xsm_logprob_grad_args;
XSM_API xsm_status xsm_token_logprobs_grad(const xsm_logprob_grad_args *a, void *cuda_stream);
/* The same with the log probabilities of the call above (DEVICE [rows], may be NULL): rows with a token take their probabilities from the differences to the
 * token's logit, and what all logits of a row have in common does not matter.  Without them, in rows without a token, and where the gradient takes the place of
 * rows of more than 8192 bytes, p is exp(z - lse) from an lse that is rounded to fp32: off by 2^-24 |lse| of itself. */
XSM_API xsm_status xsm_token_logprobs_grad_near(const xsm_logprob_grad_args *a, const float *logprob, void *cuda_stream);

/* ---- operators on a caller's own activations and weights ----
 *
 * Products on the tensor cores with what follows them in the same kernel: 16-bit elements (XSM_BF16, XSM_F16; rows 16-byte aligned, strides in elements), sums in
 * fp32.  `d`, the summed axis of the forward products, is a multiple of 8; other sizes are any, up to 2^30.  As above: the caller's stream of the current device, nothing is waited
 * for, calls may be captured.  status: DEVICE, a 32-bit word, zeroed by the caller before its first use, which calls may share: XSM_ERR_TIMEOUT once a bounded wait of the
 * device has run out, and the results of that call are then void.  counters: DEVICE, XSM_COUNTERS words, zero before their first use and again after every call, but for one whose
 * wait ran out; calls that share them follow each other on one stream.  workspace: DEVICE, 16-byte aligned, as many bytes as the function of that name says, of any
 * content; calls that share one follow each other on one stream. */

enum { XSM_COUNTERS = 2048 };

/* Log probabilities of given tokens under softmax(logits / temperature), logits = hidden . weight^T, which are never in memory:
 *   z_rj = sum_i hidden[r][i] weight[j][i] / temperature,  lse_r = log sum_j exp(z_rj),  logprob_r = z_r,token - lse_r.
 * Tokens outside [0, vocab), logits of -infinity and NaN as for xsm_token_logprobs. */
typedef struct {
    const void *hidden, *weight;          /* DEVICE dtype [rows][d], [vocab][d] */
    const void *tokens;                   /* DEVICE int32 or int64 [rows], stride in elements */
    float *logprob, *lse;                 /* DEVICE [rows] */
    void *workspace;
    int32_t *status;
    uint32_t *counters;                   /* may be NULL; with them up to 16 rows take one kernel instead of two */
    int64_t hidden_stride, weight_stride, token_stride, workspace_bytes;
    int32_t rows, vocab, d, dtype, token_bytes;
    float temperature;
} xsm_linear_logprobs_args;
XSM_API size_t xsm_linear_logprobs_workspace(int rows, int vocab, int d);
XSM_API xsm_status xsm_linear_logprobs(const xsm_linear_logprobs_args *a, void *cuda_stream);
/* The same, and logprob once more (DEVICE [rows], may be NULL), for a gradient that is to find it whatever becomes of the first. */
XSM_API xsm_status xsm_linear_logprobs_keep(const xsm_linear_logprobs_args *a, float *kept, void *cuda_stream);

/* The gradient of sum_rows (g_logprob logprob + g_lse lse) by hidden and weight, in their type, from lse of the call above:
 *   dz_rj = ([j = token_r] g_logprob_r - exp(z_rj - lse_r) (g_logprob_r - g_lse_r)) / temperature,  d_hidden = dz . weight,  d_weight = dz^T . hidden.
 * g_logprob counts only where there is a token; rows with an lse of -infinity have none.  The logits are computed again, piece by piece of the vocabulary; dz is
 * rounded to dtype once (up to 128 rows or 64 tokens: held in two parts of it; fp16: scaled by
 * a power of two that takes its largest possible element to 2^13, rows whose elements are below 2^-12 of that by up to 2^14 more, and back in the sums; g_logprob of rows without a token
 * does not count, nor what rows with an lse of -infinity have).  The workspace holds a
 * piece of dz of at most 256 MiB (1024 tokens at least), fp16's scaled rows of hidden and partial sums.  d_hidden or d_weight may be NULL. */
typedef struct {
    const void *hidden, *weight, *tokens; /* as above */
    const float *lse;                     /* DEVICE [rows] */
    const float *g_logprob, *g_lse;       /* DEVICE [rows], strides in elements; each may be NULL */
    void *d_hidden, *d_weight;            /* DEVICE dtype [rows][d], [vocab][d] */
    void *workspace;
    int32_t *status;
    uint32_t *counters;
    int64_t hidden_stride, weight_stride, token_stride, g_logprob_stride, g_lse_stride, d_hidden_stride, d_weight_stride, workspace_bytes;
    int32_t rows, vocab, d, dtype, token_bytes;
    float temperature;
} xsm_linear_logprobs_grad_args;
XSM_API size_t xsm_linear_logprobs_grad_workspace(int rows, int vocab, int d);
XSM_API xsm_status xsm_linear_logprobs_grad(const xsm_linear_logprobs_grad_args *a, void *cuda_stream);
/* The same with the log probabilities of the call above (DEVICE [rows], may be NULL): the token's own element is g_logprob (1 - p) + g_lse p with p = exp(logprob), which next to p = 1 an lse that
 * is rounded to fp32 does not tell: otherwise p is exp(z - lse), off by 2^-24 |lse| of itself. */
XSM_API xsm_status xsm_linear_logprobs_grad_near(const xsm_linear_logprobs_grad_args *a, const float *logprob, void *cuda_stream);

/* The gated feed-forward part of a block: out[r][f] = act(gate) up, gate = sum_i x[r][i] w_gate[f][i], up = sum_i x[r][i] w_up[f][i], gate and up in fp32;
 * act(g) = g / (1 + exp(-g)) (activation 0, silu) or g (1 + erf(g / sqrt 2)) / 2 (1, gelu). */
typedef struct {
    const void *x, *w_gate, *w_up;        /* DEVICE dtype [rows][d], [ff][d], [ff][d] */
    void *out;                            /* DEVICE dtype [rows][ff]; aligned to its elements */
    int32_t *status;
    int64_t x_stride, w_gate_stride, w_up_stride, out_stride;
    int32_t rows, ff, d, dtype, activation;
} xsm_gated_ff_args;
XSM_API xsm_status xsm_gated_ff(const xsm_gated_ff_args *a, void *cuda_stream);

/* The gradient of sum(g_out * out) by x, w_gate and w_up, in their type.  gate and up are computed again; their gradients g_out up act'(gate) and g_out act(gate) are
 * rounded to dtype once (up to 128 rows or 32 columns: held in two parts of it; fp16: scaled by
 * powers of two, which take a row's bound |g_out| |x| max(1.13 |w_up|, |w_gate|), over the largest finite elements and rows, to 2^13 for the largest row and to 2 at least for rows down to
 * 2^-26 of it, and back in the sums: nothing finite becomes infinite on the way).  d_x, or d_w_gate and d_w_up, may be NULL. */
typedef struct {
    const void *x, *w_gate, *w_up;        /* as above */
    const void *g_out;                    /* DEVICE dtype [rows][ff]; aligned to its elements */
    void *d_x, *d_w_gate, *d_w_up;        /* DEVICE dtype [rows][d], [ff][d], [ff][d], the latter of one stride */
    void *workspace;
    int32_t *status;
    uint32_t *counters;
    int64_t x_stride, w_gate_stride, w_up_stride, g_out_stride, d_x_stride, d_w_stride, workspace_bytes;
    int32_t rows, ff, d, dtype, activation;
} xsm_gated_ff_grad_args;
XSM_API size_t xsm_gated_ff_grad_workspace(int rows, int ff, int d);
XSM_API xsm_status xsm_gated_ff_grad(const xsm_gated_ff_grad_args *a, void *cuda_stream);
/* Tries of a shared-memory barrier before a wait of the following calls of the four above, in this process, gives up (0: the default, 2^22).  starve: these
 * calls fetch no operands, so that their waits run out. */
XSM_API xsm_status xsm_debug_product_waits(uint32_t tries, int starve);

/* Norms of queries and keys for each head with the rotation of the positions:  y = R (gain x / sqrt(mean(x^2) + eps)), mean over the head, R as in xsm_kv_append.  fp32 within,
 * rounded once.  The position of token j of a sequence is positions[sequence][j] (NULL: j); rows of a token whose position the rope does not have are zero, and
 * so are their gradients.  d_head 32, 64, 96, 128 or 256; strides in elements of sequence, token, head, neighbouring elements of a head; q_out may be q, k_out k.
 * n_heads or n_kv_heads may be 0. */
typedef struct {
    const void *q, *k;                    /* DEVICE dtype [batch][m][n_heads or n_kv_heads][d_head] */
    void *q_out, *k_out;                  /* likewise */
    const void *q_gain, *k_gain;          /* DEVICE gain_dtype [d_head] */
    const int32_t *positions;             /* DEVICE [batch][m] */
    const float *rope;                    /* as in xsm_kv_append_args */
    int64_t q_stride[3], k_stride[3], q_out_stride[3], k_out_stride[3];
    int32_t batch, m, n_heads, n_kv_heads, d_head, dtype, gain_dtype, rope_positions, rope_dims, interleaved;
    float eps;
} xsm_norm_rotate_args;
XSM_API xsm_status xsm_norm_rotate(const xsm_norm_rotate_args *a, void *cuda_stream);

/* The gradient of sum(g_q * q_out) + sum(g_k * k_out) by q, k and the gains (the latter in gain_dtype, added up in fp32 in an order of its own sizes' making; without heads they are not
 * written). */
typedef struct {
    const void *q, *k, *q_gain, *k_gain;  /* as above */
    const int32_t *positions;
    const float *rope;
    const void *g_q, *g_k;                /* DEVICE dtype, like q and k */
    void *d_q, *d_k, *d_q_gain, *d_k_gain;
    void *workspace;                      /* DEVICE, xsm_norm_rotate_grad_workspace bytes, of any content; calls that share one follow each other on one stream */
    uint32_t *counters;                   /* as for the products above */
    int64_t q_stride[3], k_stride[3], g_q_stride[3], g_k_stride[3], d_q_stride[3], d_k_stride[3], workspace_bytes;
    int32_t batch, m, n_heads, n_kv_heads, d_head, dtype, gain_dtype, rope_positions, rope_dims, interleaved;
    float eps;
} xsm_norm_rotate_grad_args;
XSM_API size_t xsm_norm_rotate_grad_workspace(int d_head);
XSM_API xsm_status xsm_norm_rotate_grad(const xsm_norm_rotate_grad_args *a, void *cuda_stream);

/* xsm_kv_append with the norms of keys, and of queries where there are any, before the rotation. */
typedef struct {
    const void *q_gain, *k_gain;          /* DEVICE gain_dtype [d_head] */
    int32_t gain_dtype;
    float eps;
} xsm_head_norm;
XSM_API xsm_status xsm_kv_append_norm(const xsm_kv *kv, const xsm_kv_append_args *a, const xsm_head_norm *n, void *cuda_stream);

#ifdef __cplusplus
}
#endif
#endif /* XSM_H */
