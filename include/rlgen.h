/*
 * rlgen -- generation hot path of asynchronous online-DPO RLHF on one MI355X (gfx950).
 *
 * The method (paper, Section 3 and Appendix D, Algorithm 1, procedure Generate) spends most of
 * its run time drawing K completions per prompt from the current policy pi_theta at a sampling
 * temperature (0.7 in Appendix A.1-A.3) and needs, for every drawn token, log pi(y_t | x, y_<t):
 * the per-token terms of log pi_theta(y|x) in the Online DPO objective (Section 2.1) and of
 * pi_old in the importance ratio of Appendix B, Eq. 1.  This library is that computation for a
 * GPT-NeoX-shaped (Pythia) or Llama-shaped decoder, written as hand-made HIP kernels.
 *
 * Conventions
 *  - Plain C ABI.  Every pointer is a DEVICE pointer unless its comment says HOST.
 *  - The caller owns all memory, including the workspace.  The library allocates no device
 *    memory (host side it allocates its context, small pinned staging buffers, two internal streams
 *    and a few events); rlgen_destroy frees only that host-side state.
 *  - rlgen_generate / rlgen_score enqueue work on the stream given to the call and return; outputs
 *    are valid once the caller has synchronised that stream.  HOST arrays are read before return.
 *  - One context serves one call at a time (calls on one context must not overlap).
 *  - Every function returns RLGEN_OK (0) or a negative RLGEN_ERR_* code.  A call rejected by host
 *    validation launches nothing and writes nothing.  Conditions only the device can see (a token
 *    id outside [0, vocab), a uniform outside [0, 1)) clamp the value, never read out of bounds,
 *    and set a sticky flag reported by rlgen_status.
 *  - Arithmetic: weights are bf16 values (held in fp16, which represents them exactly in its normal
 *    range); GEMM and attention inputs are fp16; the KV cache is bf16; accumulation, the residual
 *    stream, normalisation statistics, softmax and log-sum-exp are fp32 (fp64 for the CDF scan).
 *    cfg.precise = 1 widens every 16-bit activation and cache entry to a pair of bf16 numbers.
 */
#ifndef RLGEN_H
#define RLGEN_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

#define RLGEN_OK                  0
#define RLGEN_ERR_NULL           -1   /* a required pointer is null                         */
#define RLGEN_ERR_BAD_CFG        -2   /* inconsistent or unsupported model configuration    */
#define RLGEN_ERR_BAD_ARG        -3   /* a per-call argument is out of its domain           */
#define RLGEN_ERR_CAPACITY       -4   /* the call exceeds max_seqs / max_kv_tokens / max_seq_len / max_batch_tokens */
#define RLGEN_ERR_WORKSPACE      -5   /* workspace too small or misaligned                  */
#define RLGEN_ERR_UNIMPLEMENTED  -6
#define RLGEN_ERR_DEVICE         -7   /* a HIP call failed, or a device-detected input fault */

#define RLGEN_ARCH_NEOX   0  /* LayerNorm+bias, parallel residual, GELU (erf), biased linears   */
#define RLGEN_ARCH_LLAMA  1  /* RMSNorm, sequential residual, SwiGLU, no biases, grouped KV heads */

#define RLGEN_DTYPE_F32   0  /* tensors supplied as fp32; rounded to bf16 (nearest even) on load */
#define RLGEN_DTYPE_BF16  1  /* tensors supplied as bf16                                          */
#define RLGEN_DTYPE_F16   2  /* tensors supplied as fp16 (the operators over pages and packed rows, and the learner's, only) */
#define RLGEN_DTYPE_E4M3  3  /* rlgen_add_rms_norm's output in 8 bits only: 4 exponent and 3 mantissa bits, largest value 448 */

/* Threads: calls on one context must not overlap; different contexts may be used from different
 * threads.  The library reads no environment variables. */
typedef struct rlgen_ctx rlgen_ctx; /* opaque */

typedef struct {
  int32_t arch;            /* RLGEN_ARCH_*                                                     */
  int32_t n_layers;
  int32_t d_model;         /* = n_q_heads * head_dim; multiple of 32                            */
  int32_t n_q_heads;
  int32_t n_kv_heads;      /* divides n_q_heads; = n_q_heads for NeoX                            */
  int32_t head_dim;        /* multiple of 16, at most 256                                        */
  int32_t d_ffn;           /* multiple of 32                                                     */
  int32_t vocab;
  int32_t rotary_dim;      /* even, <= head_dim: first rotary_dim dims of each head are rotated  */
  float   rope_theta;      /* 10000 for the Pythia shapes, 500000 for the Llama-3.1 shape        */
  float   norm_eps;
  int32_t weight_dtype;    /* RLGEN_DTYPE_*: element type of every tensor in rlgen_weights       */
  int32_t max_seqs;        /* capacity: sequences alive in one call (prompts * k)                */
  int32_t max_seq_len;     /* capacity: longest prompt_len + max_new, or scored sequence         */
  int64_t max_kv_tokens;   /* capacity: sum over sequences of (prompt_len + max_new) rounded up
                              to a multiple of 32                                                */
  int32_t max_batch_tokens;/* rows processed at once by prefill / score; >= max_seq_len;
                              0 selects a default (32768, or max_seqs * max_seq_len if smaller)      */
  int32_t share_prompt_kv; /* 0: every sequence owns a contiguous cache holding prompt and new tokens.
                              1: rlgen_generate stores a prompt's keys/values once and its k samples
                              read them together (the k samples of a prompt condition on the same
                              prefix: Section 2.1, Section 4.2); results are the same up to rounding
                              order.  Then k * (n_q_heads / n_kv_heads) <= 16 is required and the
                              max_kv_tokens need is sum over prompts of round32(prompt_len) +
                              prompts * k * round32(max_new).  rlgen_score is unaffected.        */
  int32_t precise;         /* 0: the formats of the Conventions above (fp16 matrix-product inputs, bf16 cache).
                              1: every 16-bit activation and every cached key and value is held as the sum of
                              two bf16 numbers (16 significant bits, fp32's exponent range), the queries stay
                              fp32, the weights stay the caller's bf16 values, and each matrix product runs once
                              per half on the bf16 matrix instructions.  For checking a policy against an fp32
                              reference where the 16-bit formats themselves exceed the tolerance (random
                              Llama-shaped weights amplify every rounding: Appendix A.2's model shape); it
                              doubles the cache, the activation buffers and the matrix work.  Requires
                              rotary_dim % 4 == 0 and head_dim <= 128.                              */
} rlgen_model_cfg;

/* Per-layer tensors, row-major, linear layers stored [out, in] and applied as y = W x + b.
 * Pointers marked (NeoX) are null for Llama and vice versa. */
typedef struct {
  const void *norm1_g, *norm1_b;  /* [d]; _b (NeoX)                                     */
  const void *norm2_g, *norm2_b;  /* [d]; _b (NeoX)                                     */
  const void *wq, *wk, *wv;       /* [Hq*h, d], [Hkv*h, d], [Hkv*h, d]                  */
  const void *bq, *bk, *bv;       /* (NeoX)                                             */
  const void *wo, *bo;            /* [d, Hq*h]; bo (NeoX)                               */
  const void *w_up, *b_up;        /* [F, d]; b_up (NeoX)                                */
  const void *w_gate;             /* [F, d] (Llama)                                     */
  const void *w_down, *b_down;    /* [d, F]; b_down (NeoX)                              */
} rlgen_layer_weights;

typedef struct {
  const void *embed_in;                      /* [V, d]                                    */
  const void *final_norm_g, *final_norm_b;   /* [d]; _b (NeoX)                            */
  const void *lm_head;                       /* [V, d], no bias, not tied to embed_in     */
  const rlgen_layer_weights *layers;         /* HOST array of n_layers entries            */
} rlgen_weights;

/* Bytes of workspace rlgen_create needs for this configuration (its private 16-bit copy of the
 * weights, the KV cache, activations and sampler partials), or 0 if cfg is null or invalid. */
size_t rlgen_workspace_bytes(const rlgen_model_cfg *cfg);

/* Builds a context for one policy (Algorithm 1: procedure Generate starts by loading the current
 * parameters theta_i into the generation model).
 * cfg, weights: HOST structs holding DEVICE tensor pointers.  workspace: DEVICE, 256-byte aligned,
 * at least rlgen_workspace_bytes(cfg); it must stay alive, and must not be written by the caller,
 * until rlgen_destroy.  The weight tensors are converted/copied on `hip_stream` (a hipStream_t, or
 * null for the default stream); once that stream has been synchronised the library no longer reads
 * them.  *out receives the context.  Errors: NULL, BAD_CFG, WORKSPACE, DEVICE.
 * Creation also times the tile shapes of every linear layer at this configuration's row counts (on
 * `hip_stream` and two internal streams, a few hundred launches, 1-3 s at the 2.8B shape) and
 * synchronises with them, so it must not be called under stream capture.  Timing chooses tile shapes
 * only: how a linear layer's sum over its inner dimension is cut and ordered is a fixed function of
 * the configuration, so two contexts of one configuration return the same bits whatever they picked. */
int rlgen_create(const rlgen_model_cfg *cfg, const rlgen_weights *weights, void *workspace,
                 size_t workspace_bytes, void *hip_stream, rlgen_ctx **out);

/* Replaces the policy's weights in place with a new theta_i of the same shape (Algorithm 1,
 * procedure Generate, first step; Appendix A.2 notes that this hand-off blocks the learner). */
int rlgen_update_weights(rlgen_ctx *ctx, const rlgen_weights *weights, void *hip_stream);

/* y ~ pi_theta(. | x): k completions of exactly max_new tokens per prompt by inverse-CDF sampling
 * from softmax(z / temperature), plus the log-probability of each emitted token under that same
 * distribution (Section 2.1; Algorithm 1, procedure Generate; temperature: Appendix A.1).
 *
 *  prompts        [B, prompt_stride] int32, right-padded; cells at or beyond prompt_lens[b] are never read
 *  prompt_lens    HOST [B] int32, each >= 1
 *  uniforms       [B, k, max_new] fp32 in [0, 1): the random numbers of the draw.  Token t of sample
 *                 (b, j) is the first vocabulary index whose cumulative probability, accumulated in
 *                 ascending index order, exceeds uniforms[b, j, t] (if rounding leaves none, the last
 *                 index with positive probability)
 *  forced         nullable [B, k, max_new] int32: an entry >= 0 replaces the drawn token (used by
 *                 parity tests to keep two implementations on one trajectory); its log-prob is reported
 *  tokens         out [B, k, max_new] int32
 *  token_logprobs out [B, k, max_new] fp32 = log softmax(z / temperature)[token]
 *
 * The k samples of one prompt share one prompt pass.  Errors: NULL, BAD_ARG (B, k, max_new < 1,
 * prompt_len < 1, prompt_stride < max prompt_len, temperature not finite or < 0, or with
 * share_prompt_kv k * (n_q_heads / n_kv_heads) > 16), CAPACITY, DEVICE.
 *
 * temperature == 0 decodes greedily (the evaluation protocol of Section 5.2): every token is the
 * first index of the largest logit, uniforms are not read (but must be non-null), and
 * token_logprobs = log softmax(z)[token].
 * With an EOS token set (rlgen_set_eos) a completion ends at its first EOS: the entries after it
 * hold the EOS id at log-prob 0 (forced entries after it are ignored); rlgen_set_eos says what then
 * happens to the ended sequence's place in the batch. */
int rlgen_generate(rlgen_ctx *ctx, const int32_t *prompts, const int32_t *prompt_lens, int32_t B,
                   int32_t prompt_stride, int32_t k, int32_t max_new, float temperature,
                   const float *uniforms, const int32_t *forced, int32_t *tokens,
                   float *token_logprobs, void *hip_stream);

/* Teacher-forced log-probabilities, the terms of log pi(y | x) in the DPO objective (Section 2.1)
 * and of the ratio in Appendix B, Eq. 1:
 *   out[n, t] = log softmax(z_{t-1} / temperature)[seqs[n, t]]   for max(1, score_from[n]) <= t < seq_lens[n]
 *   out[n, t] = 0                                                 elsewhere in [0, stride)
 *  seqs [N, stride] int32 right-padded; seq_lens HOST [N]; score_from HOST [N] or null (= 1).
 * Errors: NULL, BAD_ARG, CAPACITY, DEVICE. */
int rlgen_score(rlgen_ctx *ctx, const int32_t *seqs, const int32_t *seq_lens,
                const int32_t *score_from, int32_t N, int32_t stride, float temperature,
                float *token_logprobs, void *hip_stream);

/* Raw (temperature 1) logits at the last position of each sequence, [N, vocab] fp32.  The product
 * path never writes logits to memory; this entry point exists so that tests can bound them. */
int rlgen_debug_logits(rlgen_ctx *ctx, const int32_t *seqs, const int32_t *seq_lens, int32_t N,
                       int32_t stride, float *logits, void *hip_stream);

/* The final-norm + LM-head + sampling stage alone (the last line of procedure Generate applied to
 * given residual rows): hidden [R, d] fp32, uniforms [R], forced nullable [R] -> tokens [R],
 * token_logprobs [R].  R <= max_batch_tokens. */
int rlgen_debug_sample(rlgen_ctx *ctx, const float *hidden, int32_t R, float temperature,
                       const float *uniforms, const int32_t *forced, int32_t *tokens,
                       float *token_logprobs, void *hip_stream);

/* rlgen_debug_sample for callers that cannot allocate or hand over scratch memory at the time of the call: code under
 * HIP graph capture, tight serving loops, harnesses that forbid hipMalloc.  Same arguments, same kernels, same results;
 * the stage's intermediate buffers (the normalised rows, the per-row per-64-column softmax partials) live in a static
 * device array of the library (about 4.3 MB per GPU, held until the process ends) instead of the context's workspace,
 * so the call does not touch the workspace's activation buffers.  It allocates nothing, on the host or the device.
 * Limits: R <= 64 rows, d_model <= 8192, vocab <= 262144; beyond them RLGEN_ERR_CAPACITY.  The device the context was
 * created on must be current.  All calls on one GPU, from any context, share the one array: calls that overlap in time
 * on that GPU (different streams or contexts) race; calls on one stream are ordered.  Nothing in the array needs to
 * start at zero: every element a call reads it has written itself.
 * Errors: NULL, BAD_ARG, CAPACITY, DEVICE. */
int rlgen_sample_static(rlgen_ctx *ctx, const float *hidden, int32_t R, float temperature,
                        const float *uniforms, const int32_t *forced, int32_t *tokens,
                        float *token_logprobs, void *hip_stream);

/* Consumers of the log-probs (Section 2.1, DPO objective).  seq_logprob[n] = sum of
 * token_logprobs[n, t] over from[n] <= t < lens[n] (from, lens: DEVICE [N] int32). */
int rlgen_sequence_logprob(const float *token_logprobs, const int32_t *from, const int32_t *lens,
                           int32_t N, int32_t stride, float *seq_logprob, void *hip_stream);
/* loss[p] = -log sigmoid(beta * ((pol_pos[p] - ref_pos[p]) - (pol_neg[p] - ref_neg[p]))), all [P] fp32. */
int rlgen_dpo_loss(const float *pol_pos, const float *ref_pos, const float *pol_neg,
                   const float *ref_neg, int32_t P, float beta, float *loss, void *hip_stream);

/* Proximal RLOO, the off-policy baseline the paper compares Online DPO with (Appendix B, Eq. 1): for each of
 * a prompt's k >= 2 completions, objective = min(r A, clip(r, 1 - epsilon, 1 + epsilon) A) with
 * r = exp(pol_logprob - old_logprob) (pi_theta over the generating policy pi_old, both sequence log-probs as
 * rlgen_sequence_logprob returns them) and A = the completion's reward minus the mean reward of the prompt's
 * other k - 1 completions (at k = 2, the other completion's reward, as the appendix writes it).
 * pol_logprob, old_logprob, rewards, objective: DEVICE [B, k] fp32.
 * Errors: NULL, BAD_ARG (B < 1, k < 2, epsilon negative or not finite), DEVICE. */
int rlgen_proximal_rloo(const float *pol_logprob, const float *old_logprob, const float *rewards, int32_t B,
                        int32_t k, float epsilon, float *objective, void *hip_stream);

/* Which two of a prompt's k completions are trained on (Section 2.1: the two samples ranked by reward;
 * Section 4.2: of K = 4 samples the highest and the lowest rewarded).  rewards [B, k] fp32 (the caller's
 * reward model; no NaN), idx_pos / idx_neg [B] int32 out, all DEVICE: idx_pos[b] = first index of the
 * maximum, idx_neg[b] = last index of the minimum (so they differ whenever k >= 2).
 * Errors: NULL, BAD_ARG (B or k < 1), DEVICE. */
int rlgen_select_pairs(const float *rewards, int32_t B, int32_t k, int32_t *idx_pos, int32_t *idx_neg,
                       void *hip_stream);

/* Per-phase device times of the last rlgen_generate / rlgen_score on this context, in ms (any
 * pointer may be null).  Synchronises the events it reads.  decode_attn_ms / decode_attn_launches
 * cover the decode-attention kernel alone and are filled only while profiling is on:
 * rlgen_set_profiling(ctx, n) with n >= 1 brackets every n-th decode-attention launch (rotating
 * over the layers from step to step) with events on the call's stream; decode_attn_ms is the sum
 * over the decode_attn_launches bracketed launches.  Each bracketed launch costs about 10 us. */
int rlgen_get_timings(rlgen_ctx *ctx, float *prefill_ms, float *decode_ms, float *decode_attn_ms,
                      int32_t *decode_attn_launches);
int rlgen_set_profiling(rlgen_ctx *ctx, int32_t on);

/* The token id that ends a completion in later rlgen_generate calls on this context (the paper's
 * completions end in an EOS token or are penalised for lacking one: hyper-parameter tables of
 * Appendix A.1 and A.2); -1 (the default) = none.  With an EOS id set and one cache per sequence
 * (share_prompt_kv = 0), rlgen_generate drops ended sequences from the batch: every 8 decode steps
 * it WAITS for the stream, reads which sequences have ended, fills the rest of their outputs and
 * continues with the others (and returns early once none is left), so the call is no longer purely
 * asynchronous.  With share_prompt_kv = 1 ended sequences stay in the batch and only stop reading
 * their cache.  The outputs are the same either way.
 * Errors: NULL, BAD_ARG (id outside [-1, vocab)). */
int rlgen_set_eos(rlgen_ctx *ctx, int32_t eos_token);

/* The sequences a learner scores come in groups: a prompt x and its k completions (the pair y+, y-
 * of the DPO objective, Section 2.1; K = 4 in Section 4.2).  After rlgen_set_score_groups(ctx, k),
 * k > 1, rlgen_score requires N to be a multiple of k, score_from non-null and equal within every
 * group of k consecutive sequences (1 <= score_from <= seq_len), and takes the caller's word that
 * the group's sequences agree in their first score_from tokens: that shared part then goes through
 * the model once per group instead of once per sequence.  Outputs are the same as without grouping
 * up to rounding order.  The agreement is checked on the device; a group that breaks it sets the
 * sticky status (rlgen_status returns DEVICE) and its log-probs are meaningless.  k = 1 (the
 * default) scores every sequence on its own.  A call falls back to scoring every sequence on its
 * own when a group does not fit one chunk of max_batch_tokens rows, or when rotary_dim is not a
 * multiple of 4.  Errors: NULL, BAD_ARG (k < 1). */
int rlgen_set_score_groups(rlgen_ctx *ctx, int32_t k);

/* rlgen_generate decodes a batch of 256 or more sequences as two halves on two internal streams
 * (forked from and joined to the call's stream), so that one half's cache-streaming attention runs
 * beside the other half's linear layers.  on = 0 turns that off for later calls on this context
 * (every kernel then runs alone on the call's stream, which is what a per-kernel measurement
 * needs); on != 0 turns it back on.  Results do not depend on it. */
int rlgen_set_decode_split(rlgen_ctx *ctx, int32_t on);

/* ended sequences leave the batch every `every` decode steps (default 8; 0: never, they stay in the batch and
 * only stop reading their cache).  Outputs do not depend on it.  Errors: NULL, BAD_ARG (every < 0). */
int rlgen_set_eos_compaction(rlgen_ctx *ctx, int32_t every);

/* min_seqs >= 2 replaces the 256-sequence threshold of the two-stream decode together with its criterion that a
 * step's cache traffic must outweigh the weights four times (tests use it to send small batches down that path);
 * 0 restores the default.  Results do not depend on it.  Errors: NULL, BAD_ARG. */
int rlgen_set_decode_split_min(rlgen_ctx *ctx, int32_t min_seqs);

/* The tile shape (`variant`, an index into the library's list of GEMM tilings) and the K split the context uses for
 * linear layer `which` (0 QKV, 1 attention output, 2 FFN up, 3 FFN down, 4 LM head) in `mode` (0: decode of the whole
 * batch, 1: prompt pass and scoring, 2: decode of half a batch).  variant -1 = chosen per call from the problem size; -2
 * (FFN up of a GPT-NeoX block only) = computed in QKV's launch, with QKV's tile shape.
 * rlgen_debug_set_gemm replaces the tile shape (testing and measurement); the K split cannot be set: it is a function
 * of the configuration.  A shape set for an FFN up in QKV's launch gives it a launch of its own, and -2 takes it back where
 * the context had it there.  With the GPT-NeoX block (n_q_heads * head_dim a multiple of 64) the attention output is part of
 * FFN down's product and `which` 1 has no launch of its own: replacing its tile shape changes nothing.  Errors: NULL, BAD_ARG
 * (mode, which or variant out of range, -2 where the context has no such launch, or a tile shape this layer's epilogue
 * does not support). */
int rlgen_debug_get_gemm(rlgen_ctx *ctx, int32_t mode, int32_t which, int32_t *variant, int32_t *splits);
int rlgen_debug_set_gemm(rlgen_ctx *ctx, int32_t mode, int32_t which, int32_t variant);

/* Synchronises `hip_stream` and returns RLGEN_ERR_DEVICE if a kernel has flagged a device-detected fault since the
 * context was created (sticky), else RLGEN_OK: a token id outside [0, vocab), a uniform outside [0, 1), a score group
 * whose members disagree on their shared part, or an activation beyond the largest finite fp16 value (65504), which
 * the library's fp16 matrix-product inputs cannot hold: such a value is clamped to +-65504, never turned into
 * infinity.  *faults (nullable, HOST) receives the bit set: 1 token id, 2 uniform, 4 score group, 8 fp16 range. */
int rlgen_status(rlgen_ctx *ctx, void *hip_stream);
int rlgen_status_bits(rlgen_ctx *ctx, void *hip_stream, uint32_t *faults);

/* ------------------------------------------------------------------ operators over a cache in pages and packed rows
 *
 * The blocks around attention for a policy whose layers normalise queries and keys per head and attend to a window, and for
 * requests that come and go: a cache in pages, the plan of a pass over it, norms and rotation with the cache write, attention over
 * packed rows and over the cache, and the gradients of the last two.  They need no context.  Element type `dtype` is RLGEN_DTYPE_BF16
 * or RLGEN_DTYPE_F16 for queries, keys, values, outputs and their gradients; statistics, sums and gains are fp32.
 *
 * Layouts
 *  - Packed rows: the tokens of S sequences one behind the other; row_starts [S + 1] int32 holds the first row of each and the number
 *    of rows.  A tensor [rows, heads, head_dim] has head_dim and heads contiguous and any row stride (in elements) up to 2^23 that is a
 *    multiple of 8, so a column range of a fused projection's output can be passed as it is.  All bases 16-byte aligned.
 *  - Cache: pages [n_pages, 2, n_kv_heads, page_size, head_dim]: of a page's tokens first the keys, then the values.  page_size is a power
 *    of two from 8 to 1024.  Sequence s has its token t in page page_table[s * table_stride + t / page_size].  A slot is
 *    page * page_size + t % page_size.
 *  - head_dim is a multiple of 16, at most 256; n_kv_heads divides n_q_heads.
 *  - Visibility: a query at position p sees key j if j <= p and (j > p - window, or j < sinks, or window == 0: no window).  A query that
 *    sees nothing has output 0 and log-sum-exp -infinity.
 *  - Without rows (0) an operator returns at once, gradients of gains are zeroed, and pointers to tensors of rows may be null.
 *  - Sizes: rows * heads, S * heads and n_pages * page_size below 2^31.  Offsets are 64-bit.  A launch has fewer than 2^24 blocks: of the attention
 *    over rows S * n_kv_heads (rounded up to 8) times the tiles, of 128 pairs of a row and a query head of the group, that max_len (at most rows)
 *    or max_new makes, and in the backward pass the tiles of 128 keys, two blocks each beyond 96 dims; of single tokens S * n_kv_heads / 4
 *    times the query heads of a group over 16 (over 8 beyond 128 dims), rounded up.
 * Entries of row_starts, page_table and slots that lie outside their arrays are clamped or skipped, never followed: a token whose page lies
 * outside the cache is seen by no query. */
#define RLGEN_PLAN_ROWS    1   /* counts[3]: more rows than max_rows or 2^31 - 2 (those beyond are not written) */
#define RLGEN_PLAN_PAGES   2   /* the free list ran out (pages and slots that lack one are -1)                 */
#define RLGEN_PLAN_TABLE   4   /* a sequence needs more pages than a table row has (its slots beyond are -1)   */
#define RLGEN_PLAN_LENGTH  8   /* a negative length (taken as 0), or one that passes 2^31 - 1 (cut there)      */

/* The plan of one pass over the cache, from the requests' lengths alone: sequence s holds ctx_lens[s] tokens and gets new_lens[s] more.
 * Pages that it needs for them are taken from free_pages [n_free] in the order of the sequences, from entry *free_head on (DEVICE, null:
 * 0), and entered into page_table, whose earlier entries are read for tokens that go into a page already begun.
 *  total_lens [S], row_starts [S + 1]   out: lengths after the pass; first row of each sequence
 *  slots, positions [max_rows]          out: where row i's key and value go, and its position; rows that no sequence has: -1 and 0
 *  counts [4]                           out: rows; the free list's next head (min(head + pages taken, n_free)); longest length after the
 *                                       pass; RLGEN_PLAN_* bits
 * Sums stop at 2^31 - 1 (row_starts and counts[0] with RLGEN_PLAN_ROWS), so no length or head leads outside the arrays.
 * free_head must not be counts + 1 itself; two counts arrays in turn chain passes without the host.
 * Errors: NULL, BAD_ARG (S < 1, max_rows < 0, n_free < 0, table_stride < 1, page_size), DEVICE. */
int rlgen_plan_pages(const int32_t *ctx_lens, const int32_t *new_lens, int32_t S, int32_t page_size, const int32_t *free_pages,
                     int32_t n_free, const int32_t *free_head, int32_t *page_table, int32_t table_stride, int32_t max_rows,
                     int32_t *total_lens, int32_t *row_starts, int32_t *slots, int32_t *positions, int32_t *counts,
                     void *hip_stream);

/* cos and sin of position * theta^(-2 i / rotary_dim), evaluated in fp64: table [max_pos, rotary_dim / 2, 2] fp32.
 * Errors: NULL, BAD_ARG, DEVICE. */
int rlgen_rope_table(float *table, int32_t max_pos, int32_t rotary_dim, float theta, void *hip_stream);

/* RMS norm of every query and key head over its head_dim, gains, then rotation of the first rotary_dim dims (pairs i, i + rotary_dim / 2,
 * as in rlgen_generate), in one pass over the fused projection's output:
 *  qkv [rows, (n_q_heads + 2 n_kv_heads) head_dim] of type src_dtype (any RLGEN_DTYPE_*), row stride qkv_stride
 *  q_gain, k_gain [head_dim] fp32; rope: rlgen_rope_table's, positions [rows] int32 (clamped to [0, max_pos))
 *  q out [rows, n_q_heads, head_dim]; k, v nullable out [rows, n_kv_heads, head_dim]; pages nullable: keys and values go to slots[row]
 *  (a slot outside the cache is skipped).  Values are neither normalised nor rotated.
 * At least one of pages (with slots) and k must be given; rope may be null if rotary_dim is 0.  Errors: NULL, BAD_ARG, DEVICE. */
int rlgen_qk_norm_rope(const void *qkv, int64_t qkv_stride, int32_t src_dtype, int32_t rows, int32_t n_q_heads, int32_t n_kv_heads,
                       int32_t head_dim, const float *q_gain, const float *k_gain, float eps, const float *rope, int32_t max_pos,
                       int32_t rotary_dim, const int32_t *positions, int32_t dtype, void *q, int64_t q_stride, void *k,
                       int64_t k_stride, void *v, int64_t v_stride, void *pages, int32_t n_pages, int32_t page_size,
                       const int32_t *slots, void *hip_stream);

/* Its gradients: dq, dk, dv (type dtype, of q, k and v as rlgen_qk_norm_rope returns them) to dqkv (type src_dtype, all of it written)
 * and dq_gain, dk_gain [head_dim] fp32 (sums over all rows and heads in a fixed order, padding rows among them).  workspace: 16-byte aligned,
 * rlgen_qk_norm_rope_backward_workspace(rows, head_dim) bytes.  Errors: NULL, BAD_ARG, WORKSPACE, DEVICE. */
size_t rlgen_qk_norm_rope_backward_workspace(int32_t rows, int32_t head_dim);
int rlgen_qk_norm_rope_backward(const void *qkv, int64_t qkv_stride, int32_t src_dtype, int32_t rows, int32_t n_q_heads,
                                int32_t n_kv_heads, int32_t head_dim, const float *q_gain, const float *k_gain, float eps,
                                const float *rope, int32_t max_pos, int32_t rotary_dim, const int32_t *positions, int32_t dtype,
                                const void *dq, int64_t dq_stride, const void *dk, int64_t dk_stride, const void *dv,
                                int64_t dv_stride, void *dqkv, int64_t dqkv_stride, float *dq_gain, float *dk_gain, void *workspace,
                                size_t workspace_bytes, void *hip_stream);

/* Causal attention within each packed sequence: out [rows, n_q_heads, head_dim], lse nullable [rows, n_q_heads] fp32 = log of the sum of
 * exp(scale q k) over the visible keys.  max_len (HOST) bounds every sequence's rows; rows of a sequence beyond it are not computed.
 * A key or value that a query does not see never reaches its output, be it infinite or NaN.
 * Errors: NULL, BAD_ARG, DEVICE. */
int rlgen_window_attention(const void *q, int64_t q_stride, const void *k, int64_t k_stride, const void *v, int64_t v_stride,
                           int32_t dtype, int32_t rows, int32_t n_q_heads, int32_t n_kv_heads, int32_t head_dim,
                           const int32_t *row_starts, int32_t S, int32_t max_len, int32_t window, int32_t sinks, float scale, void *out,
                           int64_t out_stride, float *lse, void *hip_stream);

/* Its gradients, from its own inputs and outputs and dout.  Written are the rows of dq, dk and dv that a sequence has within max_len (zeros for a
 * query that sees nothing and a key that nobody sees); the others, and lse and out of the forward pass there, are left as they are: zero
 * them where a later sum goes over all rows.  Within a sequence infinities and NaN go where the products carry them; no other sequence's
 * values change a bit of its gradients.
 * workspace: 16-byte aligned, rlgen_window_attention_backward_workspace(...) bytes.  Errors: NULL, BAD_ARG, WORKSPACE, DEVICE. */
size_t rlgen_window_attention_backward_workspace(int32_t rows, int32_t n_q_heads, int32_t n_kv_heads, int32_t head_dim, int32_t S,
                                                 int32_t max_len, int32_t window, int32_t sinks);
int rlgen_window_attention_backward(const void *q, int64_t q_stride, const void *k, int64_t k_stride, const void *v, int64_t v_stride,
                                    const void *out, int64_t out_stride, const float *lse, const void *dout, int64_t dout_stride,
                                    int32_t dtype, int32_t rows, int32_t n_q_heads, int32_t n_kv_heads, int32_t head_dim,
                                    const int32_t *row_starts, int32_t S, int32_t max_len, int32_t window, int32_t sinks, float scale,
                                    void *dq, int64_t dq_stride, void *dk, int64_t dk_stride, void *dv, int64_t dv_stride,
                                    void *workspace, size_t workspace_bytes, void *hip_stream);

/* Attention of new tokens over the cache that already holds them: the rows of sequence s are its last row_starts[s + 1] - row_starts[s]
 * tokens of total_lens[s] (as rlgen_plan_pages gives them).  max_new, max_total (HOST) bound rows and total_lens of every sequence;
 * max_new == 1 is a decode step: a sequence's keys are then parted over many waves where there are few sequences.  workspace: 16-byte
 * aligned, rlgen_window_attention_paged_workspace(...) bytes (may be 0, and workspace null then).  max_new > 1 needs none; with
 * rlgen_window_attention_chunk_workspace(...) bytes (0: parting would not pay) the keys of a few new rows behind a long context are parted
 * over many blocks too.
 * Errors: NULL, BAD_ARG, WORKSPACE, DEVICE. */
size_t rlgen_window_attention_paged_workspace(int32_t n_q_heads, int32_t n_kv_heads, int32_t head_dim, int32_t S, int32_t max_new,
                                              int32_t max_total, int32_t window, int32_t sinks);
size_t rlgen_window_attention_chunk_workspace(int32_t n_q_heads, int32_t n_kv_heads, int32_t head_dim, int32_t S, int32_t max_new,
                                              int32_t max_total, int32_t window, int32_t sinks);
int rlgen_window_attention_paged(const void *q, int64_t q_stride, int32_t dtype, int32_t rows, int32_t n_q_heads, int32_t n_kv_heads,
                                 int32_t head_dim, const void *pages, int32_t n_pages, int32_t page_size, const int32_t *page_table,
                                 int32_t table_stride, const int32_t *row_starts, const int32_t *total_lens, int32_t S,
                                 int32_t max_new, int32_t max_total, int32_t window, int32_t sinks, float scale, void *out,
                                 int64_t out_stride, float *lse, void *workspace, size_t workspace_bytes, void *hip_stream);

/* ------------------------------------------------------------------ the learner's rows: norm, log-probs, loss
 *
 * What a policy's learner runs between its matrix products, from the branch of a block to the gradient of the loss; the norm and the log-probs
 * serve single tokens as well.  They need no context, keep nothing between calls, and have no sums whose order changes: the same call
 * returns the same bits (log-probs of another number of rows may be added up in another order).  Statistics, sums, log-probs, losses and gains are fp32 or wider.
 *
 * Layouts
 *  - Rows of the norm: width elements, a multiple of 8 up to 16384, any row stride (in elements) that is a multiple of 8 (fp32: 4), bases and gains
 *    16-byte aligned, fewer than 2^23 rows.
 *  - Rows of logits: vocab elements, at most 2^24, any row stride from vocab on and any base that suits the element type, fewer than 2^24 rows.
 *  - A workspace serves one call at a time: calls that may overlap (on two streams, in two captured graphs) need their own.
 *  - Without rows (0) an operator returns at once, the gain's gradient is zeroed, and pointers to tensors of rows may be null. */

/* h = residual + dropout(x) and y = RMS norm of h times the gain, in one pass.
 *  x [rows, width] of type dtype (RLGEN_DTYPE_F32, _BF16 or _F16); residual nullable (h is then dropout(x)) and h nullable out, both of type
 *  residual_dtype, F32 or dtype: the residual stream.
 *  y nullable out (gain is then not read): of type dtype, or any of the three where dtype is F32, or RLGEN_DTYPE_E4M3 with scales [rows, groups] fp32: y's value is
 *  scales[row, c / scale_group] times the element; scale_group 32, 64 or 128 columns to a scale (the last group may be shorter), or 0: one
 *  for the row.  A scale is the group's largest magnitude / 448; a group below 2^-100 has scale 0 and zeros; NaN is kept and counts for no scale.
 *  The norm is that of h before it is rounded to residual_dtype; squares are summed in fp32.  Values beyond a 16-bit type become infinite, as a
 *  cast makes them.
 * Dropout: an element is dropped with probability drop_p in [0, 1], rounded to a multiple of 2^-16, else multiplied by the inverse of the rest.
 *  The mask is a function of rng, row and column alone and never stored: rng [2] int64 DEVICE holds a seed and an offset (read when the
 *  launch runs, so that a captured call draws anew when the caller advances the offset); Philox4x32 of ten rounds with key = the seed's
 *  words and counter = (column / 8, row, the offset's words) gives 16 bits for each of eight columns, the low half of a word first,
 *  and an element is dropped if its bits are below 65536 drop_p.  Calls that are to draw apart need offsets (or seeds) of their own.  rng
 *  may be null if drop_p is 0.
 * h may be residual or x itself, y may be x itself (same type and stride); other overlaps are not allowed.
 * Errors: NULL, BAD_ARG, DEVICE. */
int rlgen_add_rms_norm(const void *x, int64_t x_stride, int32_t dtype, const void *residual, int64_t residual_stride,
                       int32_t residual_dtype, int32_t rows, int32_t width, double drop_p, const int64_t *rng, const float *gain, float eps,
                       void *h, int64_t h_stride, void *y, int64_t y_stride, int32_t y_dtype, float *scales, int32_t scale_group,
                       void *hip_stream);

/* Its gradients, from h as rlgen_add_rms_norm returned it, dy (type dtype) and dh (nullable, type residual_dtype: the gradient that reaches h past
 * the norm): dresidual (nullable, residual_dtype) = the gradient of h, dx (nullable, dtype) = the same through the dropout (drop_p and rng as
 * they were), dgain [width] fp32 (the sum over all rows, padding rows among them).  gain null: no norm was taken, dy and dgain are null too and h is
 * not read.  dresidual may be dh itself, dx may be dy itself.  workspace: 16-byte aligned, rlgen_add_rms_norm_backward_workspace(rows, width)
 * bytes (0, and it may be null, for few rows; null without a gain).
 * Errors: NULL, BAD_ARG, WORKSPACE, DEVICE. */
size_t rlgen_add_rms_norm_backward_workspace(int32_t rows, int32_t width);
int rlgen_add_rms_norm_backward(const void *h, int64_t h_stride, int32_t residual_dtype, const void *dy, int64_t dy_stride, int32_t dtype,
                                const void *dh, int64_t dh_stride, int32_t rows, int32_t width, double drop_p, const int64_t *rng,
                                const float *gain, float eps, void *dresidual, int64_t dresidual_stride, void *dx, int64_t dx_stride,
                                float *dgain, void *workspace, size_t workspace_bytes, void *hip_stream);

/* Of each row of logits [rows, vocab] (type dtype: RLGEN_DTYPE_F32, _BF16 or _F16), under softmax(z / temperature):
 *  logprobs [rows]       log-prob of tokens[row]; tokens and logprobs are given both or neither
 *  entropy [rows]        nullable: -sum p log p
 *  stats [rows, 2]       the largest logit m, and log sum exp((z - m) / temperature): what the backward pass needs
 *  top_tokens, top_logprobs [rows, n_top]   the n_top (0 to 64, at most vocab) likeliest tokens in descending order, of equal ones the lowest index first
 * A row whose token lies outside [0, vocab) (padding, a prompt's rows) is not read: its log-prob, entropy and stats are 0, its alternatives -1 and
 * -infinity.  A logit of -infinity is masked: it counts 0.  The type's lowest value is a value like any other: beside an allowed logit m its term is 0 once
 * (m - z) / temperature passes 104 (fp16's -65504: at temperatures up to 600), and a row of lowest values alone is uniform.  A row of -infinity alone has
 * log-prob -infinity, entropy 0, stats (-infinity, -infinity), and alternatives at -infinity.  A NaN or +infinity makes the row's log-prob, entropy and
 * log sum NaN (m passes over NaN); among the alternatives NaN counts as the largest.  temperature is finite and at least 1e-6.
 * workspace: 16-byte aligned, rlgen_token_logprobs_workspace(...) bytes (0, and workspace may be null, unless few rows are parted over many
 * blocks).  Errors: NULL, BAD_ARG, WORKSPACE, DEVICE. */
size_t rlgen_token_logprobs_workspace(int32_t dtype, int32_t rows, int32_t vocab, int32_t n_top);
int rlgen_token_logprobs(const void *logits, int64_t stride, int32_t dtype, int32_t rows, int32_t vocab, const int32_t *tokens,
                         float temperature, float *logprobs, float *stats, float *entropy, int32_t n_top, int32_t *top_tokens,
                         float *top_logprobs, void *workspace, size_t workspace_bytes, void *hip_stream);

/* The gradient of logprobs and entropy to the logits: dlogits [rows, vocab] of type dtype, every element written, zeros in rows that were not read
 * or hold -infinity alone.  dlogprobs, dentropy [rows]: at least one of them; with dlogprobs tokens, with dentropy the forward pass's entropy.
 * tokens null: no row is left out.  dlogits may be logits itself (same stride); other overlaps are not allowed.
 * A launch has fewer than 2^24 blocks: rows times vocab / 8192 (fp32: 4096), rounded up.  Errors: NULL, BAD_ARG, DEVICE. */
int rlgen_token_logprobs_backward(const void *logits, int64_t stride, int32_t dtype, int32_t rows, int32_t vocab, const int32_t *tokens,
                                  float temperature, const float *stats, const float *entropy, const float *dlogprobs, const float *dentropy,
                                  void *dlogits, int64_t dlogits_stride, void *hip_stream);

/* The DPO loss of packed sequences, and its gradient, in one launch: prompt b has the k sequences b k to b k + k - 1 of row_starts [B k + 1], and
 * idx_pos, idx_neg [B] (rlgen_select_pairs's) say which of them are y+ and y-.  token_logprobs, ref_logprobs [rows] fp32: per row, 0 where it does not
 * count (as rlgen_token_logprobs leaves rows without a token).
 *  loss [B]          -log sigmoid(beta ((sum pol - sum ref over y+) - (sum pol - sum ref over y-)))
 *  dlogprobs [rows]  the gradient of weight * sum of the losses to token_logprobs: one value on y+'s rows, its negative on y-'s, 0 on the other
 *                    sequences'; rows that no sequence has are left as they are
 * idx_pos[b] == idx_neg[b] is a pair without a difference, whatever its log-probs: log 2 and zeros.  A sum that is infinite or NaN (a masked token's log-prob
 * is -infinity) gives its own pair's loss and rows their limits, or NaN where there is none (-infinity in both models), and no other rows anything.
 * Indices and row starts outside their ranges are clamped.  Sums and the loss are formed in fp64, of beta and weight as fp32 holds them.  All DEVICE.
 * Errors: NULL, BAD_ARG (B or k < 1, B >= 2^22, beta or weight not finite), DEVICE. */
int rlgen_dpo_pairs(const float *token_logprobs, const float *ref_logprobs, int32_t rows, const int32_t *row_starts, int32_t B, int32_t k,
                    const int32_t *idx_pos, const int32_t *idx_neg, float beta, float weight, float *loss, float *dlogprobs,
                    void *hip_stream);

const char *rlgen_strerror(int code);
void rlgen_destroy(rlgen_ctx *ctx);

#ifdef __cplusplus
}
#endif
#endif /* RLGEN_H */
