/*
 * sps.h -- C ABI of the B200 speculative-sampling library (libsps_b200.so).
 *
 * The library implements the hot path of speculative sampling (Chen et al.,
 * "Accelerating Large Language Model Decoding with Speculative Sampling"):
 * K single-row draft-model steps, one (K+1)-row target-model scoring pass and
 * the modified rejection sampler, as CUDA kernels for sm_100a.  Notation is
 * the paper's: q = TARGET model, p = DRAFT model, K = lookahead.
 *
 * Conventions
 *   - every function returns an int status: SPS_OK (0) or a negative error.
 *     Nothing throws, aborts or prints.  sps_last_error() describes the last
 *     failure on a handle (or, with a NULL handle, of the handle-less calls).
 *   - "host" / "device" in a comment says where the pointer must point.
 *   - weight and logit buffers passed in are caller-owned and never written
 *     unless stated; the handle owns its KV caches, work buffers and graphs.
 *   - one handle = one CUDA stream; calls on a handle are not re-entrant.
 *
 * Random numbers.  Algorithm 2 draws r ~ U[0,1] and samples tokens; this
 * library fixes the generator so results can be reproduced elsewhere:
 * Philox4x32-10, key = (seed low 32, seed high 32), counter =
 * (t, s, b, 0) with t the position inside the loop (0..K-1 drafts, K the extra
 * token), s the loop index, b the sequence index.  Word 0 -> u_draft (draw of
 * draft token t), word 1 -> u_acc (accept test), word 2 -> u_res (resample at
 * t, or extra-token draw at t = K).  u = (word >> 8) * 2^-24.
 * Every draw is an inverse-CDF draw in index order on unnormalised weights.
 */
#ifndef SPS_B200_H
#define SPS_B200_H

#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

#define SPS_OK 0
#define SPS_EINVAL (-1)   /* bad argument or unsupported shape                     */
#define SPS_ENOMEM (-2)   /* device or host allocation failed                      */
#define SPS_ECUDA (-3)    /* a CUDA call failed; sps_last_error has its message    */
#define SPS_ERANGE (-4)   /* token id >= vocab, or sequence would exceed max_seq   */
#define SPS_ESTATE (-5)   /* call order (e.g. step before prefill)                 */
#define SPS_ETIMEOUT (-6) /* a bounded device-side wait ran out                    */

#define SPS_MAX_K 15      /* K + 1 rows <= 16 per sequence                         */

/* sps_accept / sps_step flag bits (per sequence) */
#define SPS_FLAG_RESAMPLED 1u /* a draft was rejected; token drawn from norm(max(0, q - p)) */
#define SPS_FLAG_BONUS 2u     /* all K drafts accepted; extra token drawn from q_{K+1}       */
#define SPS_FLAG_FALLBACK 4u  /* rejected with sum max(0, q - p) == 0: token drawn from q_t  */
#define SPS_FLAG_TIMEOUT 8u   /* sps_accept only: a bounded wait inside the kernel ran out; this
                                 sequence's outputs are meaningless (handle calls return SPS_ETIMEOUT) */

/* sps_cfg.flags */
#define SPS_CFG_NO_GRAPH 1u   /* launch kernels one by one instead of replaying CUDA graphs  */
#define SPS_CFG_TENSOR_PARALLEL 2u /* the weights are one rank's shard of both models (see sps_tp_attach) */

typedef struct sps_handle sps_handle;

/* One decoder-only transformer: pre-RMSNorm, multi-head attention with
 * n_heads * d_head == d_model, rotary positions on adjacent pairs over the
 * whole head, non-gated FFN with tanh-GeLU, no biases, untied (un)embedding.
 * (The paper's Hyperparams table fixes d_model / heads / layers only.)
 * n_kv_heads: key / value heads; 0 or n_heads = one per query head.  A divisor
 * of n_heads below it gives grouped-query attention, 1 multi-query attention
 * (Related Work: multi-query attention shrinks the key / value cache;
 * Conclusion: it combines with this method, which leaves the transformer
 * body alone): query head h attends
 * over key / value head h / (n_heads / n_kv_heads), wk and wv have
 * n_kv_heads * d_head rows, and the cache holds that many numbers per position.
 * dtype: 0 = fp32, 1 = bf16; it is the storage type of the weight matrices,
 * the embeddings and the KV cache.  Norm gains are always fp32.
 * dtype 2 = weight-only int8: the linear layers' matrices (wq .. w_down and the
 * unembedding) are signed bytes with one fp32 scale per output row,
 * w[n][k] = scale[n] * byte[n][k] (sps_weights' *_scale members); the token
 * embedding and the KV cache stay bf16.  (The paper notes that quantisation
 * composes with speculative sampling, since the method does not touch the
 * transformer body; half the bytes per weight halve the floor of every pass.)
 * bf16 / int8 models need d_model and d_ff to be multiples of 128; d_head is 64 or 128. */
typedef struct {
  int32_t n_layers, d_model, n_heads, d_head, d_ff, vocab;
  int32_t dtype;
  float rms_eps, rope_base;
  int32_t n_kv_heads;
} sps_model_cfg;

typedef struct {
  sps_model_cfg target, draft;
  int32_t max_seq;   /* longest sequence (prompt + generated + K) a cache row exists for */
  int32_t max_batch; /* sequences decoded together, <= 8; max_batch * (max_K + 1) <= 16,
                        or <= 128 when the target is bf16 (passes above 16 rows run
                        their linear layers as tensor-core GEMMs)                        */
  int32_t max_K;     /* largest lookahead that will be asked for, <= SPS_MAX_K           */
  int32_t device;    /* CUDA device ordinal                                              */
  void* stream;      /* cudaStream_t to run on; NULL = the library creates its own       */
  uint32_t flags;    /* SPS_CFG_*                                                        */
} sps_cfg;

/* Weights of one model.  All pointers are DEVICE pointers, borrowed for the
 * life of the handle and never written.  Matrices are row-major [out, in]
 * (y = W x), in the model's dtype.  The per-layer members are HOST arrays of
 * n_layers device pointers. */
typedef struct {
  const void* tok_embed;  /* [vocab, d_model]            */
  const void* unembed;    /* [vocab, d_model]            */
  const void* final_norm; /* [d_model] fp32              */
  const void* const* attn_norm; /* each [d_model] fp32   */
  const void* const* ffn_norm;  /* each [d_model] fp32   */
  const void* const* wq;        /* each [d_model, d_model] */
  const void* const* wk;        /* each [n_kv_heads * d_head, d_model] */
  const void* const* wv;
  const void* const* wo;
  const void* const* w_up;      /* each [d_ff, d_model]  */
  const void* const* w_down;    /* each [d_model, d_ff]  */
  /* dtype 2 only (NULL otherwise): fp32 row scales, 16-byte aligned, one per output row of the matrix */
  const float* unembed_scale;        /* [vocab]               */
  const float* const* wq_scale;      /* each [d_model]        */
  const float* const* wk_scale;      /* each [n_kv_heads * d_head] */
  const float* const* wv_scale;
  const float* const* wo_scale;
  const float* const* w_up_scale;    /* each [d_ff]           */
  const float* const* w_down_scale;  /* each [d_model]        */
} sps_weights;

/* What a generation did (the Results section counts the tokens each
 * speculative loop produced; so does this). */
typedef struct {
  int32_t loops;         /* target calls                                             */
  int32_t draft_calls;   /* draft forward passes                                     */
  int32_t emitted;       /* tokens produced before truncation to n_new               */
  int32_t accepted;      /* draft tokens accepted                                    */
  int32_t resampled;     /* loops that ended in a residual resample                  */
  int32_t bonus;         /* loops that accepted all K drafts and drew the extra token */
  int32_t fallback;      /* loops that took the sum max(0, q-p) == 0 fallback         */
  int32_t overshoot;     /* tokens of the last loop dropped to return exactly n_new  */
  int32_t hist_emitted[SPS_MAX_K + 2]; /* hist_emitted[j] = loops that emitted j tokens */
  float ms_prefill;      /* device time of the prompt pass                           */
  float ms_decode;       /* device time from the first loop's start to the last loop's end,
                            host turnaround between loops included                   */
  float ms_draft, ms_verify, ms_accept; /* device time inside the three phases       */
  int32_t kernel_launches; /* kernels the loops launched (graph nodes counted per replay) */
} sps_stats;

/* Build a handle for a (target, draft) pair: the target model q and the draft
 * model p of Algorithm 2's preamble.  draft_w may be NULL, then
 * only K = 0 (Algorithm 1) is available.  Allocates the KV caches
 * [layer][sequence][head][position][d_head] in the model dtype, work buffers
 * and rotary tables on cfg->device.  *out receives the handle. */
int sps_create(const sps_weights* target_w, const sps_weights* draft_w, const sps_cfg* cfg, sps_handle** out);
int sps_destroy(sps_handle* h);
/* NUL-terminated text owned by the handle (or by the library when h is NULL: what the calling thread was told last). */
const char* sps_last_error(sps_handle* h);

/* Algorithm 2 (K >= 1) or Algorithm 1 (K == 0) for one sequence: ingest the
 * prompt, then loop { draft K tokens; score K+1 positions; accept / resample /
 * extra token } until n_new tokens exist.  "T" of the algorithms is a minimum
 * length: the last loop may overshoot and is truncated to exactly n_new.
 *   prompt      host  [prompt_len], prompt_len >= 1, ids < vocab
 *   out_tokens  host  [n_new]
 *   out_stats   host, may be NULL
 * temperature > 0 scales both models' logits before the rejection scheme
 * (section Modified Rejection Sampling: a temperature changes the
 * probabilities the scheme is applied to);
 * temperature == 0 is greedy decoding (top-k with k = 1 on both models, see
 * sps_set_sampling).  SPS_ERANGE if prompt_len + n_new + K > max_seq. */
int sps_generate(sps_handle* h, const int32_t* prompt, int32_t prompt_len, int32_t n_new, int32_t K,
                 float temperature, uint64_t seed, int32_t* out_tokens, sps_stats* out_stats);

/* Top-k and nucleus filtering of BOTH models' distributions ahead of the
 * rejection scheme.  The section Modified Rejection Sampling says these
 * methods are handled by changing the probabilities before the scheme is
 * applied and gives no formula; this library's:
 * after softmax(l / temperature), top_k >= 1 keeps every token whose logit is
 * at least the k-th largest (tokens tied with it stay; 0 = off); then
 * 0 < top_p < 1 keeps, of those, the tokens whose logit is at least v, v the
 * largest logit value such that the tokens with logit >= v hold at least top_p
 * of the mass top-k kept (1 = off); the rest weigh nothing and what is left is
 * renormalised.  The setting stays on the handle for every later sps_generate*,
 * sps_step; no device work.  SPS_EINVAL for top_k < 0 or top_p outside (0, 1]. */
int sps_set_sampling(sps_handle* h, int32_t top_k, float top_p);

/* sps_generate with the lookahead adapted from loop to loop.  The paper fixes K
 * per experiment and finds that the best value depends on the domain (the K
 * trade-off figure); the rule here is this library's: K starts at
 * (K_min + K_max) / 2, grows by one after a loop that accepted every draft,
 * shrinks by one after a loop that rejected its first draft, within
 * [K_min, K_max], 1 <= K_min <= K_max <= max_K.  K depends on the past only, so
 * every loop is an exact iteration of Algorithm 2 and the output law is the
 * target's.  With K_min == K_max it is sps_generate.  out_stats->draft_calls /
 * loops is the mean lookahead used. */
int sps_generate_adaptive(sps_handle* h, const int32_t* prompt, int32_t prompt_len, int32_t n_new, int32_t K_min,
                          int32_t K_max, float temperature, uint64_t seed, int32_t* out_tokens, sps_stats* out_stats);

/* Same for B sequences with equal prompt lengths, advanced in lock-step with
 * ragged progress; sequence b uses Philox sequence index index0 + b, index0
 * being 0 unless sps_set_sequence_index0 changed it.  A sequence that has its
 * n_new tokens keeps its rows in the later passes (their shape is fixed) but
 * is no longer advanced, and its overshoot never counts against max_seq:
 * prompt_len + n_new + K <= max_seq is all that is required.
 *   prompts host [B, prompt_len]; out_tokens host [B, n_new]; out_stats host [B] or NULL. */
int sps_generate_batch(sps_handle* h, const int32_t* prompts, int32_t B, int32_t prompt_len, int32_t n_new,
                       int32_t K, float temperature, uint64_t seed, int32_t* out_tokens, sps_stats* out_stats);

/* Sequence b of the following sps_generate*, sps_step calls draws its random
 * numbers as Philox sequence index0 + b (counter word c2; the paper runs one
 * sequence and names no generator -- this is how independent sequences get
 * independent uniforms here).  With it a batch, or a replica on another GPU,
 * can carry global sequence numbers and reproduce exactly what each sequence
 * would have produced alone.  Stays on the handle until changed; default 0. */
int sps_set_sequence_index0(sps_handle* h, uint32_t index0);

/* Measurement mode (not part of the method): every draft is accepted with the
 * fixed probability alpha instead of min(1, q/p), so that tokens per loop --
 * (1 - alpha^(K+1)) / (1 - alpha) in expectation -- can be swept independently
 * of how well a draft model happens to agree with its target (the Results
 * section's speed-ups depend on that agreement; random-init models have
 * little).  The emitted tokens then follow no particular law; every kernel
 * runs exactly as otherwise.  alpha in (0, 1]; 0 switches the mode off (the
 * default).  Applies to the generate / step calls of this handle. */
int sps_set_forced_acceptance(sps_handle* h, float alpha);

/* Per-loop record of the last sps_generate / sps_generate_adaptive /
 * sps_generate_batch call, for latency percentiles (the Results section
 * reports mean per-token latency; a loop delivers its tokens together, so the
 * distribution of per-loop times is what a serving system sees).
 *   loop_ms      host [cap], device time of loop i (draft + scoring + accept), may be NULL
 *   loop_emitted host [cap], tokens loop i emitted for sequence 0 (before truncation to n_new), may be NULL
 *   loop_K       host [cap], lookahead loop i ran with, may be NULL
 *   *out_loops   loops the call ran (may exceed cap: only the first cap are copied)
 * SPS_ESTATE before the first generation. */
int sps_last_loop_trace(sps_handle* h, float* loop_ms, int32_t* loop_emitted, int32_t* loop_K, int32_t cap, int32_t* out_loops);

/* Pieces of sps_generate, for tests that drive the loop themselves. */
/* forget every sequence and both caches' lengths */
int sps_reset(sps_handle* h);
/* make toks[0..n-1] (host) the sequence so far of a batch-1 run; both caches take positions 0..n-2 */
int sps_prefill(sps_handle* h, const int32_t* toks, int32_t n);
/* the same for B sequences of their own lengths: sequence b is toks[b * ld .. b * ld + lens[b]) (host, lens[b] >= 1,
 * lens[b] <= ld); both caches take positions 0 .. lens[b] - 2 of each.  What follows a sequence's length in its
 * row of toks is ignored.  B <= max_batch. */
int sps_prefill_batch(sps_handle* h, const int32_t* toks, const int32_t* lens, int32_t B, int32_t ld);
/* one loop iteration (Algorithm 2's while-body) with loop index `step`, for every sequence the last prefill set:
 * out_tokens host [B, K+1] (emitted first, -1 after), out_n_emitted host [B] = n_accepted + 1,
 * out_flags host [B] SPS_FLAG_* (may be NULL); B = 1 after sps_prefill */
int sps_step(sps_handle* h, int32_t K, float temperature, uint64_t seed, uint32_t step, int32_t* out_tokens,
             int32_t* out_n_emitted, uint32_t* out_flags);
/* copy what the last sps_step saw to HOST buffers (any may be NULL):
 * q_logits [B, K+1, V], p_logits [B, K, V], drafts [B, K] */
int sps_last_logits(sps_handle* h, int32_t K, float* q_logits, float* p_logits, int32_t* drafts);

/* The scoring step of Algorithm 2 alone (section Conditional Scoring): one
 * target pass that yields the K+1 conditional logit rows for the K drafts and
 * the position after them.  Feeds rows[0..K] (host) to the TARGET at positions
 * len..len+K where len is the target cache's valid length, appends their
 * keys/values, and writes logits.  Does not move the valid length (calling it
 * again overwrites the same positions), so it can be timed repeatedly.
 *   out_logits DEVICE fp32 [K+1, vocab], caller-owned; out_ms host, device time, may be NULL. */
int sps_verify(sps_handle* h, const int32_t* rows, int32_t K, float* out_logits, float* out_ms);
/* The same pass over n_rows rows (1..16) of either model; which: 0 = target, 1 = draft. */
int sps_score(sps_handle* h, int32_t which, const int32_t* rows, int32_t n_rows, float* out_logits, float* out_ms);

/* The modified rejection sampler alone (Algorithm 2's second for-loop and its
 * extra-token line; section "Modified Rejection Sampling"), one fused kernel:
 * softmax statistics of q_0..q_K and p_0..p_{K-1} at `temperature`; for
 * t = 0..K-1 accept draft t iff u_acc < min(1, q_t(d_t) / p_t(d_t)); at the
 * first rejection draw from max(0, q_t - p_t) / sum max(0, q_t - p_t) and stop;
 * if none, draw from q_K.
 *   q_logits      device fp32 [B, K+1, V]
 *   p_logits      device fp32 [B, K, V]   (the logits the drafts were drawn from)
 *   draft_tokens  device int32 [B, K]
 *   stream        cudaStream_t (NULL = default stream); the call only enqueues
 *   out_n_accepted device int32 [B]
 *   out_tokens    device int32 [B, K+1]: accepted drafts, then the resampled / extra token, then -1
 *   out_flags     device uint32 [B], SPS_FLAG_*
 * Sequence b uses Philox counter (t, step, b, 0).  0 <= K <= SPS_MAX_K, V >= 1. */
int sps_accept(const float* q_logits, const float* p_logits, const int32_t* draft_tokens, int32_t B, int32_t K,
               int32_t V, float temperature, uint64_t seed, uint32_t step, void* stream, int32_t* out_n_accepted,
               int32_t* out_tokens, uint32_t* out_flags);

/* sps_accept with both distributions filtered as sps_set_sampling describes
 * (top_k 0 and top_p 1 = plain sps_accept; temperature 0 = greedy). */
int sps_accept_filtered(const float* q_logits, const float* p_logits, const int32_t* draft_tokens, int32_t B, int32_t K,
                        int32_t V, float temperature, int32_t top_k, float top_p, uint64_t seed, uint32_t step,
                        void* stream, int32_t* out_n_accepted, int32_t* out_tokens, uint32_t* out_flags);

/* One inverse-CDF draw per row from softmax(logits / temperature) with
 * u_draft of counter (t, step, b, 0): the draft draw of Algorithm 2's first
 * for-loop, for given logits.  logits device fp32 [B, V];
 * out_tokens device int32 [B]. */
int sps_sample(const float* logits, int32_t B, int32_t V, float temperature, uint64_t seed, uint32_t step, uint32_t t,
               void* stream, int32_t* out_tokens);

/* sps_sample from the filtered distribution (see sps_set_sampling). */
int sps_sample_filtered(const float* logits, int32_t B, int32_t V, float temperature, int32_t top_k, float top_p,
                        uint64_t seed, uint32_t step, uint32_t t, void* stream, int32_t* out_tokens);

/* The memory-bound linear layer alone (section Conditional Scoring: at small
 * batch the linear layers are bound by memory): Y[M, N] = X[M, D] W[N, D]^T with fp32
 * accumulation.  W device, row-major [N, D], dtype 0 fp32 / 1 bf16; X device
 * fp32 [M, D]; Y device fp32 [M, N]; 1 <= M <= 16.  bf16 needs D % 128 == 0 and
 * 16-byte aligned W.  workspace: device scratch of sps_linear_workspace_bytes()
 * bytes for the same (dtype, M, N, D), zero-filled once before its first use
 * (the kernel leaves it ready for the next call).
 * out_ms: host, device time of the kernel, may be NULL; when given the call
 * waits for the kernel and returns SPS_ETIMEOUT if a bounded wait inside it ran out
 * (Y is then meaningless; the workspace stays usable for the next call).
 * sps_linear_scaled also takes dtype 2: W device int8 [N, D] (signed bytes) with
 * row_scale device fp32 [N], Y[m, n] = row_scale[n] * sum_k X[m, k] W[n, k] -- the
 * weight-only quantisation the paper's closing remark on quantisation refers to
 * (it composes with speculative sampling because the transformer body is not
 * touched): half the bytes per weight.  row_scale must be NULL for dtypes 0, 1.
 * The same workspace size function serves all three. */
int sps_linear_scaled(const void* W, int32_t dtype, const float* row_scale, const float* X, int32_t M, int32_t N, int32_t D,
                      float* Y, void* workspace, void* stream, float* out_ms);
int sps_linear(const void* W, int32_t dtype, const float* X, int32_t M, int32_t N, int32_t D, float* Y,
               void* workspace, void* stream, float* out_ms);
int64_t sps_linear_workspace_bytes(int32_t dtype, int32_t M, int32_t N, int32_t D);

/* The linear layer of the prompt pass (Algorithm 2 starts from a prompt of t
 * tokens whose keys and values both models must hold before the first loop):
 * the same product Y[M, N] = X[M, D] W[N, D]^T for up to 128 rows at once, so
 * that the weights are read once for the whole prompt chunk.  bf16 weights
 * only; W device row-major [N, D], 16-byte aligned; X device fp32 [M, D]; Y
 * device fp32 [M, N]; 1 <= M <= 128; D a multiple of 64.  The activations enter
 * the tensor cores as two bf16 halves (about 16 significant bits), products
 * accumulate in fp32.  workspace: device scratch of
 * sps_linear_wide_workspace_bytes(N, D) bytes, contents irrelevant.  The call
 * waits for the result; out_ms (host, may be NULL) receives the device time.
 * Returns SPS_ETIMEOUT if a bounded wait inside the kernel ran out. */
int sps_linear_wide(const void* W, const float* X, int32_t M, int32_t N, int32_t D, float* Y, void* workspace, void* stream,
                    float* out_ms);
int64_t sps_linear_wide_workspace_bytes(int32_t N, int32_t D);

/* The same linear layer for callers that cannot allocate device memory (the
 * paper has no counterpart: this is a service of the library, not a step of
 * the method).  A host that runs inside a stream capture, or serves under a
 * frozen memory budget, or is a plugin that only ever receives buffers, has no
 * workspace to hand to sps_linear; here the split-K scratch is a fixed array
 * inside the library's device image (about 16 MiB on every GPU that loads the
 * library, held until the process exits).  The call makes no cudaMalloc /
 * cudaFree and uses no allocating library routine.
 *   W, X, Y, dtype, M, N, D: as for sps_linear (all device pointers).
 *   stream: cudaStream_t, NULL = default stream; the call only enqueues.
 * Limit: sps_linear_static_floats_needed(dtype, M, N, D) <=
 * sps_linear_static_max_floats() (4 Mi floats).  The need is N * 16 * splits,
 * where splits is how many ranges the kernel cuts D into on the current device
 * (1 for fp32; for bf16 D over the largest multiple of 128 that divides D and
 * is at most 2048 -- 1024 for M > 8 or for layers with few rows); ask the
 * helper rather than redoing that rule.  Larger shapes return SPS_EINVAL with
 * a message.  The first call on a device looks up the array's device address
 * (cudaGetSymbolAddress) with that device current; make that first call
 * before any stream capture begins.
 * All calls share the one array: two calls whose kernels overlap on the GPU
 * (different streams) race on it -- keep them on one stream or order them.
 * Each call clears the array's counters before its kernel, so a call that
 * follows an aborted one starts clean.  The call only enqueues and cannot
 * report a bounded wait that ran out inside the kernel (sps_linear with
 * out_ms can); Y is then meaningless. */
int sps_linear_static(const void* W, int32_t dtype, const float* X, int32_t M, int32_t N, int32_t D, float* Y,
                      void* stream);
int64_t sps_linear_static_max_floats(void);
/* floats of split-K scratch the shape needs on the current device; -1 for arguments sps_linear_static rejects */
int64_t sps_linear_static_floats_needed(int32_t dtype, int32_t M, int32_t N, int32_t D);

/* ---------------------------------------------------------------------------------------------------------------
 * A paged key / value cache, for a serving program that runs many sequences of unlike lengths through the pieces of
 * this library (sps_linear, sps_accept, sps_sample, ...) and keeps its own sequences: rotary positions, the append of
 * new keys and values, and the attention of every sequence's new rows over its pages.  The paper serves one sequence
 * from one dense cache; these calls change where keys and values live, not the method: a scoring pass of K + 1 rows
 * is a batch whose sequences bring K + 1 new rows each, and the rollback after a rejection is a smaller kv_len.
 *
 * These three calls only enqueue (one kernel; attention of many bf16 rows two) on `stream`, read lengths and page tables on
 * the device -- so that a captured call can be replayed after these have moved -- and allocate nothing.  Pointers belong to the current
 * device.  dtype here: 0 = fp32, 1 = bf16.
 * ------------------------------------------------------------------------------------------------------------- */

/* Activations by row and head: element e of head h of row r is p[r * row_stride + h * head_stride + e] (strides in
 * elements; a head's elements are contiguous).  q, k and v may be slices of one q | k | v buffer. */
typedef struct {
  void* p;                         /* device */
  int64_t row_stride, head_stride; /* elements */
  int32_t dtype, heads;
} sps_rows;

#define SPS_ROTARY_PAIRS 0   /* rotated pairs are elements (2 i, 2 i + 1): what this library's models use */
#define SPS_ROTARY_HALVES 1  /* rotated pairs are elements (i, i + rot_dim / 2)                            */
typedef struct {
  const double* freq; /* device [rot_dim / 2]: radians per position of each pair                            */
  int32_t rot_dim;    /* the first rot_dim elements of a head are rotated (even, <= d_head), the rest kept   */
  int32_t layout;     /* SPS_ROTARY_PAIRS or SPS_ROTARY_HALVES                                               */
  float gain;         /* multiplies the rotated elements (1 = a pure rotation)                               */
} sps_rotary_plan;

/* Frequencies of the pairs, in 64 bits, into the HOST array out [rot_dim / 2]; no device work.  With
 * f_i = base^(-2 i / rot_dim):
 *   SPS_ROTARY_PLAIN   f_i
 *   SPS_ROTARY_LINEAR  f_i / factor                       (positions squeezed into the trained length)
 *   SPS_ROTARY_BASE    f_i with base * factor^(rot_dim / (rot_dim - 2)) in base's place (the fastest pair keeps its
 *                      frequency, the slowest is divided by factor)
 *   SPS_ROTARY_BANDS   a pair makes r_i = trained_len f_i / 2 pi turns within the trained length; with
 *                      w_i = clamp((r_i - low_turns) / (high_turns - low_turns), 0, 1):  w_i f_i + (1 - w_i) f_i / factor
 * factor >= 1 (ignored by PLAIN); trained_len >= 1 and 0 <= low_turns < high_turns for BANDS only. */
#define SPS_ROTARY_PLAIN 0
#define SPS_ROTARY_LINEAR 1
#define SPS_ROTARY_BASE 2
#define SPS_ROTARY_BANDS 3
int sps_rotary_frequencies(int32_t rot_dim, double base, int32_t scaling, double factor, int32_t trained_len, double low_turns,
                           double high_turns, double* out);

/* y[r, h] = gain * R(positions[r]) x[r, h] over the first rot_dim elements, the others copied: the pair (a, b) at
 * frequency f becomes gain * (a cos - b sin, a sin + b cos) of the angle position * f (worked out in 64 bits, so that
 * far positions keep their phase).  transposed != 0 turns the other way -- gain * R^T: the operator's gradient, and
 * for gain 1 its inverse.  positions device int32 [rows], any value.  x, y: [rows][heads] of d_head elements (even,
 * 2 .. 1024) of one dtype; y may be x itself, other overlaps are not supported.  Rows, heads and strides of any
 * alignment; 16-byte aligned ones are read and written 16 bytes at a time. */
int sps_rotary(const sps_rotary_plan* plan, const sps_rows* x, const sps_rows* y, int32_t rows, int32_t d_head,
               const int32_t* positions, int32_t transposed, void* stream);

/* The cache of one layer: slot s of page p of key head h is k[p * page_stride + h * head_stride + s * pos_stride]
 * and the d_head elements after it, v likewise.  k and v 16-byte aligned, strides multiples of 16 bytes, d_head 64 or
 * 128, page_size a power of two, 8 .. 512. */
typedef struct {
  void *k, *v;                                  /* device, caller-owned */
  int64_t page_stride, head_stride, pos_stride; /* elements             */
  int32_t dtype, n_pages, page_size, n_kv_heads, d_head;
} sps_paged_cache;

/* The sequences of one call.  Sequence b owns rows q_start[b] .. q_start[b + 1] - 1 of the call's row buffers (none:
 * q_start[b + 1] == q_start[b]) and has kv_len[b] tokens, these new ones included: its last row is at position
 * kv_len[b] - 1.  Token j is in slot j % page_size of page pages[b * pages_ld + j / page_size]; table entries behind
 * the last token's are never read; slots behind it are never used, though a page that holds any of the sequence's tokens
 * may be read whole.  Rows behind the last sequence's are left as they were.  Sequences may share pages that none of
 * them appends to.
 * The host sees none of these numbers.  What does not fit is skipped, never followed: row numbers outside the call's
 * buffers (the other rows of their sequence keep their positions), tokens behind pages_ld * page_size (not appended;
 * attention takes a kv_len above it as if it were that), a page number outside 0 .. n_pages - 1 (its tokens are not
 * appended, and read as zeros); the last two also set a bit of *status, which the calls never clear. */
#define SPS_PAGED_BAD_PAGE 1    /* bits of *status */
#define SPS_PAGED_BAD_LENGTH 2
#define SPS_PAGED_TIMEOUT 4     /* a bounded wait inside the attention kernel ran out: rows the call did not finish are NaN
                                   (log-sum-exp too), others may be; until its workspace is zero-filled again every
                                   call on it sets this bit and makes its rows NaN */
typedef struct {
  const int32_t* q_start; /* device [B + 1], not decreasing      */
  const int32_t* kv_len;  /* device [B]                          */
  const int32_t* pages;   /* device [B][pages_ld]                */
  int32_t* status;        /* device [1], may be NULL             */
  int32_t B, pages_ld;    /* B: up to 2^27                       */
  int32_t max_q;          /* the most rows a sequence brings, as far as the host knows (>= 1): picks the kernel for the whole
                             call, results hold for any q_start; for bf16 queries it decides the probabilities' bits,
                             see sps_paged_attention             */
} sps_paged_batch;

/* Append: for every row of every sequence, its keys -- rotated by the row's position under `plan`, unless plan is
 * NULL -- and its values go to the row's slot, rounded to the cache's dtype.  With q (needs a plan; q_out too) the
 * row's rotated queries go to q_out in the same kernel: q may be NULL, q_out may be q itself.  q, k, v share a dtype;
 * q_out is fp32 or bf16 for fp32 q, bf16 for bf16 q; an fp32 cache takes fp32 rows only.  A row whose position is
 * negative (more rows than kv_len) is skipped, its q_out too.  k, v, q: [rows] rows. */
int sps_paged_append(const sps_paged_cache* cache, const sps_paged_batch* batch, const sps_rotary_plan* plan, int32_t rows,
                     const sps_rows* k, const sps_rows* v, const sps_rows* q, const sps_rows* q_out, void* stream);

/* Attention: row i of sequence b, at position p = kv_len[b] - (rows of b) + i, over the tokens 0 .. p of its sequence:
 *   out[row, h] = sum_j softmax_j(scale q[row, h] . k[j, h / G]) v[j, h / G],   G = heads of q / n_kv_heads,
 * scale 0 meaning 1 / sqrt(d_head).  A row at a negative position sees nothing: its output is 0.
 * q and out: [rows] rows of the same heads, rows x heads below 2^31; out has q's dtype, or is fp32; a bf16 cache takes fp32 or
 * bf16 queries, an fp32 cache fp32 ones.  Sums and scores are fp32, whatever the scores' size.  Over a bf16 cache fp32 queries
 * and their probabilities enter the tensor cores as three bf16 parts each, which keep their 24 bits.  With bf16 queries
 * the probabilities are two bf16 parts (16 bits) where max_q * G is at most 64, and one (8 bits) where it is more, in all
 * rows of the call, an fp32 out's too: a max_q below the truth keeps 16 bits, at the cost of a prompt's speed.
 * out may be q itself (same dtype and strides), other overlaps are not supported.  lse: device fp32 [rows][heads], may be
 * NULL: log sum_j exp(scale q . k_j), -inf for a row that sees nothing or whose scores are all -inf (its output is 0 too).
 * What lies in slots behind a sequence's tokens never matters, whatever it is, nor do tokens behind a row's own.  An infinite
 * or NaN value (v) makes its element of the rows that see it infinite or NaN (which of the two is left open; where its weight is 0
 * it may be left out); over a bf16 cache, where its token is among the sequence's new ones, it may make every element of
 * those rows NaN, and values beyond 2^80 may overflow to infinite ones.  An infinite or NaN key makes the rows that see it NaN,
 * or is left out where its score is -inf.
 * workspace: device scratch of sps_paged_attention_workspace_bytes bytes, 16-byte aligned, zero-filled once before its
 * first use (every call leaves it ready for the next; calls that share one must not run at the same time, captured
 * ones included).  The size holds for every batch on this cache shape. */
int sps_paged_attention(const sps_paged_cache* cache, const sps_paged_batch* batch, int32_t rows, const sps_rows* q,
                        const sps_rows* out, float scale, float* lse, void* workspace, void* stream);
int64_t sps_paged_attention_workspace_bytes(const sps_paged_cache* cache, int32_t n_heads, int32_t q_dtype);

/* ---------------------------------------------------------------------------------------------------------------
 * Which pages a sequence has.  A pool counts, page by page, the table rows that hold it; a table has a row per sequence
 * (or per beam of one).  Rows may share pages: a prompt's pages are held once by all that continue it, and a row gets a page of
 * its own only where it is about to write (sps_paged_append) into one that others hold too.  The paper decodes one
 * sequence; these calls serve programs that decode several continuations of a prompt, admit and drop sequences, and roll
 * rejected drafts back.  One table serves all layers: page p is page p of every layer's cache.
 *
 * All calls only enqueue on `stream` (one kernel each; sps_paged_compact of a large pool or table two, sps_paged_copy one per 64
 * layers, sps_beam_select of much work two), read and write their state on the device -- so that a captured call can be replayed -- and allocate nothing.  A pool's, a table's or a
 * workspace's calls must not run at the same time.  Results do not depend on timing: of free pages the lowest are taken, rows are
 * served in their order.  What does not fit is skipped, never followed, and sets a bit of the pool's status: page numbers
 * outside the pool (SPS_PAGED_BAD_PAGE; a fork and a compaction keep such an entry), counts outside their row -- held, and in
 * sps_paged_reserve len and want; a fork and a compaction hand len on as it is -- (SPS_PAGED_BAD_LENGTH; they are clipped),
 * parents outside their table, -1 apart (SPS_PAGED_BAD_ROW; none).  Entries that a call does not read are not looked at.
 * ------------------------------------------------------------------------------------------------------------- */
#define SPS_PAGED_NO_PAGE 8    /* more bits of *status: a row was left without the pages that it wanted */
#define SPS_PAGED_BAD_ROW 16
typedef struct {
  int32_t* refs;     /* device [n_pages]: table rows that hold the page, 0 = free (all zeros: an empty pool) */
  int32_t* status;   /* device [1], SPS_PAGED_* bits, never cleared by the calls; may be NULL */
  int32_t n_pages, page_size;   /* n_pages: up to 2^20; page_size: tokens, a power of two, 8 .. 512 */
} sps_page_pool;

/* Row r holds the pages in entries 0 .. held[r] - 1 of pages[r * ld ...], for len[r] tokens (len[r] <= held[r] * page_size).
 * Entries behind held[r] are never read, and stay as they are unless pages are taken.  pages, with len as kv_len, is what
 * sps_paged_batch takes; its append and attention need held to cover kv_len. */
typedef struct {
  int32_t* pages;    /* device [B][ld] */
  int32_t *held, *len;   /* device [B]  */
  int32_t B, ld;     /* B: up to 8192, ld: up to 2^20, B x ld below 2^31 */
} sps_page_table;

/* Pages to be copied, as a call leaves them: list[i] = (from, to, slots), the first `slots` of page `from`, *count of them. */
typedef struct {
  int32_t* list;     /* device [capacity][3] */
  int32_t* count;    /* device [1]           */
  int32_t capacity;
} sps_page_moves;

/* Fork / reorder: row i of dst becomes row parents[i] of src (its entries, held and len); parents[i] = -1 makes an empty row.
 * Several children share their parent's pages.  dst takes src's place: src's rows give up their references, pages without a child
 * become free, and src is not to be used as a table again before it has been a dst (a beam search takes two in turn).  parents:
 * device [dst->B].  src and dst share no array; dst->ld >= src->ld. */
int sps_paged_fork(const sps_page_pool* pool, const sps_page_table* src, const sps_page_table* dst, const int32_t* parents, void* stream);

/* Roll back, free and make room, for every row of the table; want: device [B].  With n = min(len, want) tokens kept, first of all rows:
 *   the entries behind ceil(n / page_size) are given up (want = 0: the whole row);
 * then, where want > n, row after row:
 *   the page of token n, if n is inside it and other rows hold it too, is exchanged for a fresh one, and (old, fresh, n % page_size)
 *   is added to `moves` -- unless all who hold it go on in this call: then the first of them keeps it, or, if the pool has too few
 *   pages for all rows of the call, the one that has the most tokens in it, the first of those;
 *   fresh pages are appended up to ceil(want / page_size) entries.
 * Fresh pages are the free ones in ascending order.  A row whose pages are no longer to be had gets none of them, nor does any
 * row behind it that needs some: it keeps its n tokens and the pages that they are in -- no other row's room reaches into them --,
 * and SPS_PAGED_NO_PAGE is set.  held and len (= n) are written.  room: device [B], may be NULL (and may be want): the tokens that
 * the row may be written up to -- want, or n where it went without (its last page may then be shared still: nothing is to be
 * appended to it).  Before new tokens are appended, the moves are to be carried out (sps_paged_copy).  moves->capacity >= B.
 * workspace: device scratch of sps_paged_pool_workspace_bytes(n_pages) bytes, 16-byte aligned, zero-filled once before its first
 * use (every call leaves it ready for the next). */
int sps_paged_reserve(const sps_page_pool* pool, const sps_page_table* table, const int32_t* want, int32_t* room, const sps_page_moves* moves,
                      void* workspace, void* stream);
int64_t sps_paged_pool_workspace_bytes(int32_t n_pages);

/* Compact: with U pages in use, those numbered U and above move to the free ones below U, the i-th such page to the i-th such
 * hole, at most moves->capacity of them, lowest first; afterwards (without that limit) pages 0 .. U - 1 are in use and the rest
 * of the pool can be given back.  src must be the only table that holds pages of the pool.  dst receives the table, refs_out
 * (device [n_pages]) the references, `moves` the copies to carry out, whole pages.  In place: dst may share src's
 * arrays (the same ld), refs_out may be pool->refs; else src and pool->refs stay as they are.  workspace: as for sps_paged_reserve (the same one will do). */
int sps_paged_compact(const sps_page_pool* pool, const sps_page_table* src, const sps_page_table* dst, int32_t* refs_out, const sps_page_moves* moves,
                      void* workspace, void* stream);

/* Copy: the listed pages' first slots, in the keys and values of every layer; slots behind them are left as they were.  layers: HOST
 * array of n_layers caches of one shape, dtype and strides.  Items of the list outside the caches are skipped, slots clipped to page_size.  No page may be
 * the destination of two items, or a source and a destination (what the calls above list is of that kind). */
int sps_paged_copy(const sps_paged_cache* layers, int32_t n_layers, const sps_page_moves* moves, void* stream);

/* The selection of a beam step: for each of B sequences the N best continuations of its W beams, best first,
 *   c[w, v] = scores[w] + logits[w, v] / T - log sum_u exp(logits[w, u] / T),
 * equal ones in the order of w V + v: so are a beam's equal logits, and the candidates of alike beams, which have one score and the
 * same logits, wherever their rows lie.  (The paper samples; beam search is another way to decode from the same logits, and with
 * sps_paged_fork over the same cache.)
 *   logits        device, dtype 0 fp32 / 1 bf16: row b W + w at logits + (b W + w) row_stride (elements), V of them; any alignment
 *                 of the rows
 *   scores        device fp32 [B][W]: log-probability of each beam so far; -inf: there is no such beam (the first step after
 *                 a prompt has one beam, or one score that is not -inf)
 *   done          device int32 [B][W], may be NULL: a beam that has ended (not 0) is not continued; it offers itself as one candidate,
 *                 (end_token, its score), whatever its logits are
 *   end_token     -1: none; else candidates with it are done
 *   out_scores    device fp32 [B][N]: c, rounded to fp32 (candidates are compared before)
 *   out_parents   device int32 [B][N]: row b W + w of the continued beam -- the parents of sps_paged_fork when N = W
 *   out_tokens    device int32 [B][N]
 *   out_done      device int32 [B][N], may be NULL: 1 where the token is end_token, else 0
 * c is worked out and compared in 64 bits, but the sum under its logarithm is of fp32 exponentials added up in fp32: by its
 * relative error, about 2^-22 (2^-21 was the largest found, over vocabularies of 1000 .. 2^24), c is off.  Within a beam that
 * changes no order; candidates of unlike beams that are closer than this may change places.  The order of the additions follows from
 * the shape of the call and the rows' alignment: the same beams in another batch may get scores that differ by as much.
 * A logit of -inf is no candidate.  A beam whose score is not finite, or whose logits hold a NaN or +inf or nothing above -inf, offers
 * none; a sequence that has fewer than N candidates gets (-inf, -1, -1, 0) for the rest.
 * With N = W, out_scores may be scores and out_done may be done.  B up to 8192, W and N up to 128, V up to 2^24, W V below 2^31.
 * workspace: device scratch of sps_beam_select_workspace_bytes bytes, 16-byte aligned, whatever is in it (calls that share one must
 * not run at the same time, captured ones included). */
int sps_beam_select(const void* logits, int32_t dtype, int64_t row_stride, int32_t B, int32_t W, int32_t V, double temperature,
                    const float* scores, const int32_t* done, int32_t end_token, int32_t N, float* out_scores, int32_t* out_parents,
                    int32_t* out_tokens, int32_t* out_done, void* workspace, void* stream);
int64_t sps_beam_select_workspace_bytes(int32_t B, int32_t W, int32_t V);

/* Tensor-parallel passes (section Conditional Scoring: the models are served Megatron-style over several chips, the
 * attention and feed-forward blocks sharded and each followed by an all-reduce of (K + 1) x d_model numbers, which
 * is latency-bound and about as costly for K + 1 rows as for one; section Choice of Draft Models: the draft is shaped
 * to be served on the same chips).  One process per GPU; rank r of `world` (<= 8) creates its handle with
 * SPS_CFG_TENSOR_PARALLEL and ITS SHARD of both models:
 *   wq, wk, wv, w_up : the shard's output rows -- n_heads / world query heads, n_kv_heads / world key / value heads,
 *                      d_ff / world feed-forward features (contiguous blocks, rank r the r-th);
 *   wo, w_down       : the matching input COLUMNS, stored densely: [d_model, n_heads * d_head / world],
 *                      [d_model, d_ff / world];
 *   embeddings, unembedding, norm gains: whole, on every rank.
 * sps_model_cfg then describes the shard: d_model as in the whole model, n_heads / n_kv_heads / d_ff the shard's
 * (n_heads * d_head < d_model is allowed under this flag).  After every output projection the ranks exchange their
 * partial updates of the residual stream: each rank stores its partial into a slot of every rank's inbox (plain
 * stores into peer memory) and raises a flag there; each rank then sums the slots of its OWN inbox in rank order, so
 * every rank holds the same bits and runs the same loop.  No library collective, no multicast.
 *
 * sps_tp_buffers returns this rank's inbox and flag array (device pointers, with their sizes) for export to the
 * peers (e.g. as CUDA IPC handles, which the caller exchanges however it talks to its peers).
 * sps_tp_attach gives the handle every rank's inbox and flag array as THIS device addresses them (entry `rank`: its
 * own); attach every rank before any of them runs a pass.  Afterwards the handle's calls (sps_prefill, sps_step,
 * sps_generate, ...) are collective: every rank makes the same calls with the same arguments.  Waits on peers are
 * bounded like every other wait (SPS_ETIMEOUT). */
int sps_tp_buffers(sps_handle* h, void** inbox, void** flags, int64_t* inbox_bytes, int64_t* flags_bytes);
int sps_tp_attach(sps_handle* h, int32_t rank, int32_t world, void* const* peer_inbox, void* const* peer_flags);
/* A whole group emulated on ONE GPU, for checking the sharded arithmetic and the exchange kernels without `world`
 * GPUs: ranks[r] is rank r's handle, all created on one device with the same cfg.stream and attached to one another
 * with plain device pointers.  The calls enqueue what the `world` processes would, phase by phase (every rank's
 * store phase of an exchange before any rank's sum), so nothing ever waits for a kernel that is launched later.
 * sps_tp_group_prefill: as sps_prefill on every rank.  sps_tp_group_score: as sps_score on every rank; out_logits
 * host array of `world` DEVICE buffers [n_rows, vocab], which come out identical.  sps_tp_group_generate: below. */
int sps_tp_group_prefill(sps_handle* const* ranks, int32_t world, const int32_t* toks, int32_t n);
/* sps_generate for the emulated group (one sequence): every rank drafts, scores and runs the accept kernel on its own
 * copy of the logits; the ranks' decisions are compared after every loop (SPS_ESTATE if they ever differ) and rank 0's
 * tokens are returned.  out_stats: counts and the decode time only. */
int sps_tp_group_generate(sps_handle* const* ranks, int32_t world, const int32_t* prompt, int32_t prompt_len, int32_t n_new,
                          int32_t K, float temperature, uint64_t seed, int32_t* out_tokens, sps_stats* out_stats);
int sps_tp_group_score(sps_handle* const* ranks, int32_t world, int32_t which, const int32_t* rows, int32_t n_rows,
                       float* const* out_logits, float* out_ms);

/* Test hook for the give-up path of the kernels' waits.  Every wait inside a
 * kernel (on a copy, on another CTA, on a tile queue) is bounded by the global
 * timer: when the bound runs out the kernel records an error, lets the copies
 * it has in flight land, frees what it holds and returns, and the host call
 * reports SPS_ETIMEOUT.  limit_us shortens that bound (0 = the default of 2 s;
 * at most 2 s), and drop_stage >= 0 makes the copy producer of the first CTA
 * of sps_linear / sps_linear_wide / sps_paged_attention (bf16 cache) leave out
 * that stage of its ring, so that a wait runs out on purpose with nothing left in flight (-1 = leave nothing
 * out).  Process-wide; not thread-safe; meant for tests only. */
int sps_debug_set_wait(int64_t limit_us, int32_t drop_stage);

/* Philox4x32-10 on the device, for known-answer tests: ctr device uint32 [n,4],
 * key device uint32 [n,2], out device uint32 [n,4]. */
int sps_philox(const uint32_t* ctr, const uint32_t* key, int32_t n, void* stream, uint32_t* out);

#ifdef __cplusplus
}
#endif
#endif
