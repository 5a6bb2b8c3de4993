/*
 * hbsjd.h -- C ABI of the batched speculative-Jacobi rollout library for NVIDIA B200 (sm_100a).
 *
 * The library replaces the token-by-token student rollout of visual on-policy
 * distillation: given a real prefix x_1..x_k per image and its class, it samples
 * x_{k+1}..x_T from the student (Eq. 2), using independent per-image Jacobi
 * windows verified in batched forwards (Sec. 4.2) with Full / Compact execution
 * switching as images finish (Sec. 4.3, Eq. 6).
 *
 * General conventions
 *   - Every function returns 0 (HBSJD_OK) or a negative error code; nothing
 *     aborts or throws across this boundary.  hbsjd_strerror() names a code and
 *     hbsjd_last_error(ctx) gives a one-line detail of the last failure.
 *   - "device" pointers are CUDA global-memory addresses of the context's GPU;
 *     "host" pointers are ordinary process memory.  The caller owns every
 *     argument buffer; the context owns weights, KV pages, rollout state and
 *     all scratch, allocated in hbsjd_create and freed in hbsjd_destroy.
 *   - All GPU work is enqueued on the stream given to hbsjd_create (a
 *     cudaStream_t passed as void*, NULL = the legacy default stream).  Calls
 *     that report a live count synchronise that stream before returning.  A
 *     rollout waits for its rounds as the process has set the device's schedule
 *     flag (cudaSetDeviceFlags): by default it polls.
 *   - A context is not thread-safe; use one context per host thread / stream.
 *   - There is no CPU path: if no CUDA device is usable the calls fail with
 *     HBSJD_ECUDA.
 */
#ifndef HBSJD_H_
#define HBSJD_H_

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

enum {
    HBSJD_OK = 0,
    HBSJD_EINVAL = -1,   /* bad argument; no kernel was launched */
    HBSJD_ENOMEM = -2,   /* device or host allocation failed */
    HBSJD_ECUDA = -3,    /* a CUDA call failed (detail in hbsjd_last_error) */
    HBSJD_ESTATE = -4,   /* call not valid in the context's current state */
    HBSJD_ETIMEOUT = -5  /* a bounded device-side wait gave up; the context stays usable */
};

enum { HBSJD_DTYPE_FP32 = 0, HBSJD_DTYPE_BF16 = 1 };
enum { HBSJD_VERIFY_PROB = 0, HBSJD_VERIFY_GREEDY = 1 };              /* Eq. 5 / Eq. 4 */
enum { HBSJD_EXEC_FULL = 0, HBSJD_EXEC_COMPACT = 1, HBSJD_EXEC_HYBRID = 2,  /* Sec. 4.3 */
       /* Full execution with batch-synchronous progress: every live image advances by the smallest commit of
        * the batch (an image that verified more keeps only that many of its accepted drafts).  The baseline of
        * the ablation "Is independent progress necessary for batched SJD?" (Sec. 5.3, Table 2); not a mode to
        * use for speed. */
       HBSJD_EXEC_SYNC = 3 };

typedef struct hbsjd_ctx hbsjd_ctx;

/* Decoder description.  Pre-norm blocks: h += Wo Attn(rope(Wq a), rope(Wk a), Wv a), a = rmsnorm(h) g_attn;
 * h += W2 (silu(W1 m) * (W3 m)), m = rmsnorm(h) g_ffn; logits = W_head rmsnorm(h) g_out.
 * Sequence index 0 is the class token, index s >= 1 is image token x_s on a grid_h x grid_w raster;
 * T = grid_h * grid_w tokens per image.  The paper names the model family only (Sec. 5.1). */
typedef struct {
    int32_t n_layers, dim, n_heads, ffn_hidden, vocab, grid_h, grid_w, n_classes;
    int32_t dtype;      /* HBSJD_DTYPE_*: element type of the weight image and of activations */
    float rms_eps;
    float rope_base;
} hbsjd_model_desc;

/* Rollout parameters. */
typedef struct {
    int32_t window;          /* W: inputs per image per round = last committed token + W-1 drafts (Sec. 4.2) */
    int32_t history_offset;  /* H: new draft slots copy the token H positions back (Sec. 4.2) */
    float cfg_scale;         /* 1 = no guidance; otherwise logits = l_u + s (l_c - l_u) (Sec. 4.2) */
    float temperature;       /* > 0 */
    int32_t top_k;           /* 0 or >= vocab: off; ties at the k-th value are kept */
    int32_t verify_mode;     /* HBSJD_VERIFY_* */
    int32_t exec_mode;       /* HBSJD_EXEC_* */
    int32_t gamma;           /* HYBRID: Full iff live images > gamma, else Compact (Eq. 6) */
    uint64_t seed;           /* key of the counter-based generator; counter = (image, position, round) */
    int32_t max_rounds;      /* < 0: run to completion; 0: init + prefill only; > 0: at most that many rounds */
    int32_t reserved;
} hbsjd_params;

typedef struct {
    int64_t rounds;            /* verification rounds run with at least one live image */
    int64_t image_forwards;    /* sum over rounds of live images */
    int64_t committed;         /* tokens committed (accepted drafts + replacement / bonus tokens) */
    int64_t rejects;           /* image-rounds that ended in a rejection */
    int64_t full_rounds;       /* rounds executed in Full form */
    int64_t compact_rounds;    /* rounds executed in Compact form */
    int64_t prefill_forwards;  /* longest prefix / window, rounded up: the forwards of a pre-filling window by window.  NOT the
                                * forwards that ran, which take many windows at a time: hbsjd_prefill_passes */
    int64_t kernel_launches;   /* kernels of this library launched by the call */
    float ms_total;            /* GPU time of the call (CUDA events on the context's stream) */
    float ms_prefill;          /* of which state init + prefix pre-filling */
} hbsjd_stats;

/* Creates a context on the current CUDA device.
 *   m            model description
 *   weights      HOST pointer to the flat weight image: tok_emb[V,D], cls_emb[C+1,D] (row C = null
 *                class), per layer g_attn[D], w_qkv[3D,D], w_o[D,D], g_ffn[D], w_13[2F,D], w_2[D,F],
 *                then g_out[D], w_head[V,D]; matrices row-major [out,in]; each tensor starts on a
 *                256-byte boundary.  The image is copied; the caller keeps ownership.
 *   weight_bytes size of the image; must match the description exactly
 *   max_batch    largest batch of hbsjd_rollout; max_window largest params.window (<= 64)
 *   cuda_stream  cudaStream_t as void*
 * Constraints: dim % n_heads == 0; head size 16/32/64/128 for fp32 models, 32 or 64 for bf16 models (64 runs
 * the tensor-core attention kernel, 32 a plain one); dim, ffn_hidden, vocab multiples of 64 for bf16;
 * vocab <= 32768 (a position's probabilities stay in one CTA's shared memory).
 * Device memory, but for some KB per image: the weights; keys and values of 2 max_batch sequences of T tokens, T rounded up to
 * 64; 16 max_batch max_window vocab bytes of logits and probabilities; and activations of R = max(2 max_batch max_window,
 * min(4096, 2 max_batch T)) rows, so that pre-filling and scoring take few forwards: 10.125 dim + 2 ffn_hidden bytes
 * a row for bf16 models, 28 dim + 12 ffn_hidden for fp32.  Where that does not fit, R is 2 max_batch max_window, what a
 * round needs: the results are the same.
 * Errors: HBSJD_EINVAL, HBSJD_ENOMEM, HBSJD_ECUDA. */
int hbsjd_create(hbsjd_ctx **out, const hbsjd_model_desc *m, const void *weights, size_t weight_bytes,
                 int max_batch, int max_window, void *cuda_stream);

/* Student rollout of Eq. 2 for `batch` images (Sec. 4.2-4.3).
 *   prefix_tokens DEVICE int32 [batch, T]; only the first prefix_len[b] entries of row b are read
 *   prefix_len    DEVICE int32 [batch], 0..T
 *   class_labels  DEVICE int32 [batch], 0..n_classes-1 (n_classes selects the null class)
 *   p             HOST parameters
 *   out_tokens    DEVICE int32 [batch, T]; row b receives x_1..x_T, the prefix copied through.
 *                 With max_rounds >= 0 positions not yet committed hold drafts / zeros.
 *   stats         HOST, may be NULL
 * Runs state init, prefix pre-filling, the initial history windows, then rounds until every image
 * is complete or max_rounds is reached; returns after the stream has finished that work.
 * Errors: HBSJD_EINVAL for batch/window beyond the context's limits, prefix_len > T, label or
 * prefix token out of range, non-positive temperature; HBSJD_ECUDA; HBSJD_ETIMEOUT. */
int hbsjd_rollout(hbsjd_ctx *c, int batch, const int32_t *prefix_tokens, const int32_t *prefix_len,
                  const int32_t *class_labels, const hbsjd_params *p, int32_t *out_tokens, hbsjd_stats *stats);

/* *passes (HOST) = the batched forwards that pre-filled the prefixes of the last hbsjd_rollout of the context (0 before the
 * first; of one that failed, those that were enqueued). */
int hbsjd_prefill_passes(hbsjd_ctx *c, int64_t *passes);

/* hbsjd_rollout for callers whose buffers live in HOST memory (pinned memory makes the copies
 * asynchronous): copies the three inputs to staging buffers of the context, runs the rollout, and copies
 * the tokens back, all on the context's stream; returns after the result has arrived.
 *   prefix_tokens HOST int32 [batch, T];  prefix_len, class_labels HOST int32 [batch];  out_tokens HOST int32 [batch, T] */
int hbsjd_rollout_host(hbsjd_ctx *c, int batch, const int32_t *prefix_tokens, const int32_t *prefix_len,
                       const int32_t *class_labels, const hbsjd_params *p, int32_t *out_tokens, hbsjd_stats *stats);

/* Threshold calibration of Sec. 4.3 ("a lightweight, data-independent latency test with a few verifier
 * forwards"): times the verifier forward of a `batch`-image rollout (window, guidance on/off) with A live
 * images, once in Full form (all `batch` slots) and once in Compact form (A slots), for
 * A = batch, 3/4, 1/2, 1/4 and 1/8 of the batch, on a synthetic state (cursors at T/2).  *gamma_out (HOST) =
 * the largest tested A at which Compact is not slower than Full beyond 1 % timing noise (Eq. 6 keeps Full for
 * A > gamma); 0 if Compact
 * is slower everywhere.  ms_full / ms_compact: HOST float[5] or NULL, the measured milliseconds in that order.
 * Discards the context's rollout state.  Errors: HBSJD_EINVAL, HBSJD_ECUDA, HBSJD_ETIMEOUT. */
int hbsjd_calibrate_gamma(hbsjd_ctx *c, int batch, int window, int guidance, int *gamma_out, float *ms_full,
                          float *ms_compact);

/* One verification round (Sec. 4.2 "Batched verification" .. "Independent progress") on the state left
 * by hbsjd_rollout or a previous hbsjd_round.  *live_out (HOST) = images still incomplete afterwards.
 * A sequence of hbsjd_rollout(max_rounds = 0) and hbsjd_round calls yields the same tokens as one
 * monolithic hbsjd_rollout.  Errors: HBSJD_ESTATE without a preceding hbsjd_rollout.
 * A round that ends in an error (here or inside hbsjd_rollout) is not counted: nothing runs any more when the call
 * returns, and the round index, statistics and proposals stand as before it. */
int hbsjd_round(hbsjd_ctx *c, int *live_out);

/* Copies the current token rows (committed tokens, then drafts) to DEVICE int32 [batch, T]. */
int hbsjd_tokens(hbsjd_ctx *c, int32_t *out_tokens);

/* Frees every resource of the context.  NULL is allowed. */
void hbsjd_destroy(hbsjd_ctx *c);

/* ---- state export / import (debugging, parity tests, resuming a rollout); HOST buffers ----
 * cursor int32[batch]: committed tokens per image (Sec. 4.2 "committed cursor")
 * seq    int32[batch, T+1]: seq[b][t] = token at position t (1-based; entry 0 unused); t <= cursor committed,
 *        cursor < t < cursor+window: drafts
 * delta  uint8[batch, T+1]: 1 where the draft is a history / fallback draft (point-mass proposal)
 * qbase  int32[batch]: cursor at the start of the previous round (row t-qbase-1 of the previous
 *        round's probabilities is the proposal of draft t)
 * round  next round index.
 * hbsjd_set_state leaves the KV pages and the stored probabilities untouched. */
int hbsjd_get_state(hbsjd_ctx *c, int32_t *cursor, int32_t *seq, uint8_t *delta, int32_t *qbase, int32_t *round);
int hbsjd_set_state(hbsjd_ctx *c, const int32_t *cursor, const int32_t *seq, const uint8_t *delta,
                    const int32_t *qbase, int32_t round);

/* Reads intermediate results of the last round into a HOST buffer.
 *   HBSJD_DBG_PROBS   index = image: fp32 [window, V] probabilities of the last round
 *   HBSJD_DBG_LOGITS  index = 2*image + branch (0 conditional, 1 unconditional): fp32 [window, V]
 *   HBSJD_DBG_SLOTS   index ignored: int32 [3, n_slots] = image, cursor, n of each physical slot; returns n_slots
 *   After hbsjd_debug_forward (index = 2*image + branch; elements of the context's type unless stated):
 *   HBSJD_DBG_ACT_A   [n, dim]  operand of the next projection: fp32 models, the normed rows of the last norm that ran;
 *                     bf16 models (RMSNorm folded into the GEMMs), the bf16 copy of the residual stream
 *   HBSJD_DBG_ACT_Q   [n, dim]  rotated queries        HBSJD_DBG_ACT_O  [n, dim]  attention output
 *   HBSJD_DBG_ACT_FFN [n, ffn_hidden]  silu(gate) * up  HBSJD_DBG_ACT_H  fp32 [n, dim]  residual stream
 *   HBSJD_DBG_KV_K / HBSJD_DBG_KV_V  [cursor + n, dim]  cache rows of sequence indices 0..cursor+n-1 of that layer;
 *                     returns cursor + n
 * Returns the number of leading rows that are valid (or n_slots), or a negative error. */
enum { HBSJD_DBG_PROBS = 0, HBSJD_DBG_LOGITS = 1, HBSJD_DBG_SLOTS = 2, HBSJD_DBG_ACT_A = 3, HBSJD_DBG_ACT_Q = 4,
       HBSJD_DBG_ACT_O = 5, HBSJD_DBG_ACT_FFN = 6, HBSJD_DBG_ACT_H = 7, HBSJD_DBG_KV_K = 8, HBSJD_DBG_KV_V = 9 };
int hbsjd_debug_read(hbsjd_ctx *c, int what, int index, void *host_dst, size_t max_bytes);

/* Component-parity aid: runs the verifier forward of the current rollout state (Full layout, Sec. 4.2 "Batched
 * verification") up to and including layer `layer` -- stage 0: through the attention sub-block (norm, QKV + RoPE +
 * KV write, attention, output projection into the residual stream); stage 1: the whole block -- and stops, so
 * that hbsjd_debug_read can fetch that layer's intermediates.  No logits, no verification; the rollout state
 * is untouched (the KV rows written are the ones the next round rewrites with the same values).
 * Errors: HBSJD_ESTATE without a preceding hbsjd_rollout; HBSJD_EINVAL for layer / stage out of range. */
int hbsjd_debug_forward(hbsjd_ctx *c, int layer, int stage);

/* Decoder GEMM as used by the round (Sec. 4.2 verifier forward): C[M,N] (+)= A[M,K] . W[N,K]^T on the
 * context's stream.  A, W: DEVICE, element type of the context (bf16: tcgen05 tensor cores, fp32
 * accumulation; fp32: CUDA cores).  C: DEVICE fp32 [M,N]; accumulate != 0 adds into C.
 * M may be any size; bf16 needs N % 64 == 0, K % 64 == 0 and A, W, C 16-byte aligned (HBSJD_EINVAL).  A, W and C are ordered
 * like any other kernel argument behind earlier work of the stream. */
int hbsjd_gemm(hbsjd_ctx *c, const void *A, const void *W, float *C, int M, int N, int K, int accumulate);

/* accumulate = 2 (bf16 contexts, N = dim, M <= 2 max_batch max_window): the residual-update form the
 * forward itself uses, C += A W^T together with the bf16 copy and the per-row partial sums of squares of the new C
 * (written to buffers of the context), so that it can be timed and checked alone.
 * hbsjd_gemm `reps` times back to back before the one synchronisation (micro-benchmarks time the decoder's GEMM
 * shapes the way a forward issues them), and -- acc_wait_ns > 0, bf16 contexts -- with a bounded wait shortened to that
 * many nanoseconds (Sec. 4.2 verifier forward; the paper has no counterpart of the failure path): of the epilogue
 * warps on their accumulator, or, with a tile of the kernel for few rows, of its warps on their operands (tile 0
 * then means the former).  A limit shorter than the main loop makes a healthy pipeline take the
 * time-out path: every role leaves its loop, copies and MMAs in flight are drained, TMEM is freed, the call
 * returns HBSJD_ETIMEOUT with C partly written, and the context stays usable.  Tests use it to exercise that path.
 * tile (bf16 contexts): 0 = the library's own choice for the shape; 32, 64, 96, 128, 160, 192, 256 = one
 * CTA per 128 x tile block of C; 512 / 640 = 256 x 256 / 256 x 128 blocks on CTA pairs (N a multiple of 256 / 128);
 * 16032, 16064, 32032, 32064 = the kernel for few rows, 16 x 32 .. 32 x 64 blocks of C.  Every choice gives the
 * same bits (each element's products are summed in the same order); HBSJD_EINVAL for any other value. */
int hbsjd_debug_gemm(hbsjd_ctx *c, const void *A, const void *W, float *C, int M, int N, int K, int accumulate,
                     int reps, unsigned int acc_wait_ns, int tile);

/* Chooses the form of RMSNorm of a bf16 context (Sec. 4.2 verifier forward; the paper does not go below the model):
 * on = 1 folds it into the GEMM epilogues (bf16 copy of the unnormalised residual stream as the operand, gain in the
 * weights, row factor in the next epilogue), on = 0 runs it as a kernel of its own in front of the projections.
 * hbsjd_create picks the folded form for contexts whose largest round has at most 2048 rows (2 x max_batch x max_window) and the
 * separate one above; this call lets tests run either form at any size.  The two forms round the GEMM operand at
 * different points (x r g against x), so their results differ at bf16-noise level; one context always uses one form,
 * so Full and Compact execution stay bit-identical.  Only before the first rollout, and only for models whose norm
 * gains are all 1 (nothing to re-fold): HBSJD_ESTATE otherwise. */
int hbsjd_debug_fold_norm(hbsjd_ctx *c, int on);

/* Scatters the context's KV pages over the page pool (a seeded permutation of the page table) so that tests can
 * check that results do not depend on where a row's pages lie (Sec. 4.2: per-image KV-cache locations).  Only
 * before the first rollout of the context; HBSJD_ESTATE afterwards. */
int hbsjd_debug_shuffle_pages(hbsjd_ctx *c, uint64_t seed);

/* The tile (see hbsjd_debug_gemm: 0, 64, 96, 160, 192, 512 or one of the kernel for few rows) of every decoder GEMM of a bf16 context's
 * forwards, so that tests can compare the two kernels in each fused epilogue (Sec. 4.2 verifier forward).  Every choice
 * gives the same bits. */
int hbsjd_debug_force_tile(hbsjd_ctx *c, int tile);

/* Plants the error that a bounded device wait leaves when it gives up in the next round with this index (host memory only
 * until then; -1 takes it back), so that tests can check what a failed round leaves (Sec. 4.2 rounds; the paper has no
 * counterpart). */
int hbsjd_debug_fail_round(hbsjd_ctx *c, int round);

/* Probability pipeline of the verification step on caller-supplied logits (Sec. 4.2: "verification uses the
 * fused guided logits"): p = softmax(top_k((l_u + s (l_c - l_u)) / temperature)), ties at the k-th value kept.
 * logits_c, logits_u: DEVICE fp32 [rows, V] (logits_u may be NULL: no guidance); probs: DEVICE fp32 [rows, V].
 * V is the context's vocabulary.  Runs on the context's stream and waits for completion. */
int hbsjd_probs(hbsjd_ctx *c, const float *logits_c, const float *logits_u, int rows, float cfg_scale,
                float temperature, int top_k, float *probs);

/* Verification step of one round on caller-supplied logits (Sec. 4.2, Eq. 5 / Eq. 4): probability pipeline,
 * accept test of every draft left to right, residual resampling at the first reject (or the bonus token),
 * commit, cursor advance and draft refresh, for `batch` images in Full layout.  All pointers DEVICE.
 *   logits  fp32 [branches, batch, window, V]  branch 0 conditional, branch 1 unconditional (branches = 1 or 2)
 *   q_prev  fp32 [batch, window, V]  previous round's probabilities (row t - qbase - 1 = proposal of draft t)
 *   p_out   fp32 [batch, window, V]  this round's probabilities (rows 0..n-1 of each live image written)
 *   cursor int32 [batch], seq int32 [batch, T+1], delta uint8 [batch, T+1], qbase int32 [batch]: rollout
 *           state as in hbsjd_get_state, updated in place;  m_out int32 [batch]: tokens committed (images
 *           with cursor == T are skipped and keep their m_out entry)
 * The random words are Philox(seed; image, position, round).  Uses scratch buffers of the context; runs on
 * the context's stream and waits for completion.  Limits: batch <= max_batch and window <= max_window of the
 * context, V % 4 == 0, V <= 32768. */
typedef struct {
    int32_t batch, window, T, V, branches, history_offset, greedy, top_k;
    float cfg_scale, temperature;
    uint64_t seed;
    uint32_t round;
    uint32_t reserved;
} hbsjd_verify_desc;
int hbsjd_verify(hbsjd_ctx *c, const hbsjd_verify_desc *d, const float *logits, const float *q_prev, float *p_out,
                 int32_t *cursor, int32_t *seq, uint8_t *delta, int32_t *qbase, int32_t *m_out);

/* hbsjd_verify for callers that must not allocate device memory.  (The paper has no counterpart of this
 * entry point; it exists for deployment reasons only.)
 *
 * Who needs it: code that runs where cudaMalloc is off limits -- a training process whose framework has
 * handed the whole device to its own caching allocator (a raw allocation there can fail or fragment the
 * pool), a latency-critical loop in which an allocation would synchronise the device, or a plug-in called
 * from inside another runtime that owns all device memory.  Such a caller cannot create an hbsjd_ctx either,
 * so this function takes no context: it needs only the stream, the descriptor and the same input / output
 * buffers as hbsjd_verify.
 *
 * How: the scratch of the verification kernels (slot tables, accept flags, candidate tokens, counters) lives
 * in a fixed array of 192 KiB that is part of the library image; every GPU that loads the library holds it
 * until the process exits.  The function calls no cudaMalloc / cudaFree and no allocating library routine.
 *   - Limits: batch <= 1024, batch * window <= 16384, window <= 64, V % 4 == 0, V <= 32768; larger requests
 *     are refused with HBSJD_EINVAL and nothing is launched.
 *   - The first call on each device looks up the array's device address and raises the kernels' shared-
 *     memory limit; make that first call before any stream capture begins.
 *   - Every call uses the same array and finds the previous call's contents in it; the function clears
 *     what has to start at zero.  Calls that overlap on the GPU (other streams, other host threads) race on
 *     the array: serialise them.
 *   - cuda_stream is a cudaStream_t passed as void*; the call returns after the stream has finished the work.
 * Results are identical to hbsjd_verify on the same inputs. */
int hbsjd_verify_static(void *cuda_stream, const hbsjd_verify_desc *d, const float *logits, const float *q_prev,
                        float *p_out, int32_t *cursor, int32_t *seq, uint8_t *delta, int32_t *qbase,
                        int32_t *m_out);

/* Bidirectional KL of Eq. 3 per row: out[r] = 1/2 KL(p || q) + 1/2 KL(q || p) with p = softmax(logits_s[r]),
 * q = softmax(logits_t[r]).  logits_s, logits_t: DEVICE fp32 [rows, V], V the context's vocabulary; out: DEVICE
 * fp32 [rows].  fp32 arithmetic with running maxima (no overflow for any finite logits).  Runs on the context's
 * stream and waits for completion. */
int hbsjd_bikl(hbsjd_ctx *c, const float *logits_s, const float *logits_t, int rows, float *out);

/* Distillation score of completed trajectories (Eq. 3): for image b with real prefix k_b, the mean over the
 * generated positions t = k_b+1..T of D_biKL(p_S(. | x_<t), p_T(. | x_<t)), where both models read the same
 * tokens and class label (no guidance, temperature 1, no top-k), then the mean over the images of the batch that
 * generated anything (k_b < T).  This is the step that follows the rollout in the on-policy distillation loop.
 *   student, teacher  two contexts with the same grid (T) and vocabulary; batch <= max_batch of both.  Both
 *                     models run full-sequence causal forwards, of as many tokens as their activation rows allow,
 *                     through the same kernels as the rollout; their rollout state and KV caches are
 *                     overwritten (a stepped rollout cannot be continued afterwards).
 *   tokens        DEVICE int32 [batch, T]   completed trajectories (e.g. hbsjd_rollout's out_tokens)
 *   prefix_len    DEVICE int32 [batch]      k_b in 0..T
 *   class_labels  DEVICE int32 [batch]
 *   bikl_pos      DEVICE fp32 [batch, T] or NULL: entry t-1 = the term of position t (0 for t <= k_b)
 *   per_image     DEVICE fp32 [batch] or NULL: the per-image means (0 where k_b = T)
 *   loss          HOST float: the batch mean
 * Work is enqueued on each context's own stream with event dependencies between them; contexts that share a stream run
 * side by side all the same (the student on a stream of its own of the same priority, ordered between the shared
 * stream's earlier and later work).  The call returns after all of it finished.  Errors as hbsjd_rollout (arguments are validated on the host before
 * any launch). */
int hbsjd_score(hbsjd_ctx *student, hbsjd_ctx *teacher, int batch, const int32_t *tokens, const int32_t *prefix_len,
                const int32_t *class_labels, float *bikl_pos, float *per_image, float *loss);

/* ---- operators on rows of logits ------------------------------------------------------------------------------------
 * What the distillation loop does with logits next to the rollout: rules in front of the sampler, the teacher's distribution
 * as a list of its largest logits, and divergences with their gradients (the score above is a value only).
 *   - They take no context: a stream (cudaStream_t as void*) of the current device, a descriptor and DEVICE pointers.
 *   - They launch one kernel and return; results are there when the stream has got that far.  They keep nothing of a call's
 *     arrays (of a device, that a kernel's limits are set and how many clusters it holds) and allocate nothing: any number of
 *     calls may run at once, and a call may be captured into a CUDA graph.
 *   - Rows lie ld elements apart, any ld >= V (for what is only read: any ld >= 0; 0 is one row for all).  Pointers are
 *     aligned to their elements; rows that start on 16 bytes and arrays alike in that are fastest.
 *   - An array that is written may be one that is read (same pointer, stride and type); else they do not overlap.
 *   - Temperatures are those for which log2(e) / temperature is a number: 4.3e-39 and above.
 *   - 1 <= V <= 131072, 0 <= rows < 2^27; rows = 0 does nothing.  Element types are HBSJD_DTYPE_*; arithmetic is fp32,
 *     bf16 results are rounded once.
 *   - A call gives the same bits every time.  The order of a row's sums depends on how the row is aligned and on how many rows
 *     there are, not on what else is asked for.
 *   - Errors: HBSJD_EINVAL (nothing was launched), HBSJD_ECUDA.  hbsjd_last_error(NULL) tells the calling thread the
 *     details of its last failed one. */

/* Rules on logits in front of hbsjd_probs / hbsjd_verify (Sec. 4.2 "verification uses the fused guided logits").  Entry v of row r:
 *   x = logits, or guided: logits_u + cfg_scale (logits - logits_u);
 *   n = occurrences of v among the first history_len[r] tokens of the row's history; n > 0:
 *       x = x > 0 ? x / repetition : x * repetition;  x -= n frequency + presence;
 *   x += bias[v];  x = -inf where the row's mask has bit v = 0, and where x is NaN (guidance of two masked branches).
 *   logits, out [rows, V];  logits_u [rows, V] or NULL
 *   bias         fp32 [V] or NULL
 *   mask         uint32 [masks, ld_mask] or NULL: bit v & 31 of word v >> 5 allows v; ld_mask >= (V + 31) / 32 words
 *   mask_row     int32 [rows] or NULL (all 0): the row's mask; a number outside 0..masks-1: none
 *   history      int32 [sequences, ld_history] or NULL: tokens; those outside 0..V-1 are passed over
 *   history_row  int32 [rows] or NULL (row r: sequence r, sequences >= rows); a number outside 0..sequences-1: none.  The
 *                windows of an image share its sequence, with a longer history_len from position to position.
 *   history_len  int32 [rows] or NULL (all history_cap): taken as 0..history_cap */
typedef struct {
    int32_t rows, V, dtype, masks, sequences, history_cap;
    int64_t ld, ld_u, ld_out, ld_mask, ld_history;
    float cfg_scale, repetition, frequency, presence;   /* repetition > 0; 1, 0, 0: no penalty */
} hbsjd_adjust_desc;
int hbsjd_adjust_logits(void *cuda_stream, const hbsjd_adjust_desc *d, const void *logits, const void *logits_u,
                        const float *bias, const uint32_t *mask, const int32_t *mask_row, const int32_t *history,
                        const int32_t *history_row, const int32_t *history_len, void *out);

/* The k largest logits of every row and the mass of all others.
 *   values  fp32 [rows, k]  the logits, largest first;  indices int32 [rows, k]  their tokens; equal logits: the lowest
 *           token first.  -inf and NaN are no entries: where a row has fewer than k others, it ends in (-inf, -1).
 *   rest    fp32 [rows] or NULL: log of the sum of e^{logit / temperature} over the entries that are not listed (-inf: none)
 * 1 <= k <= min(V, 1024). */
typedef struct {
    int32_t rows, V, dtype, k;
    int64_t ld;
    float temperature;
    uint32_t reserved;
} hbsjd_topk_desc;
int hbsjd_topk_logits(void *cuda_stream, const hbsjd_topk_desc *d, const void *logits, float *values, int32_t *indices,
                      float *rest);

/* The lists of a model's distributions over completed trajectories: what hbsjd_distill_topk needs of a teacher, at 8 k + 4 bytes
 * a position in place of 4 V (Sec. 4.1, Eq. 3: teacher and student read the same tokens).  The model of context c runs
 * the forwards of hbsjd_score; entry [b, t - 1] of the outputs is the distribution of position t given x_<t, for the positions
 * t > prefix_len[b] (the others get empty lists: hbsjd_distill_topk leaves them out).
 *   tokens DEVICE int32 [batch, T], prefix_len, class_labels DEVICE int32 [batch]: as hbsjd_score
 *   values DEVICE fp32 [batch, T, k], indices DEVICE int32 [batch, T, k], rest DEVICE fp32 [batch, T] or NULL: as hbsjd_topk_logits
 * Runs on the context's stream and waits; its rollout state and KV caches are overwritten.  Errors as hbsjd_score. */
int hbsjd_score_topk(hbsjd_ctx *c, int batch, const int32_t *tokens, const int32_t *prefix_len, const int32_t *class_labels, int k,
                     float temperature, float *values, int32_t *indices, float *rest);

/* Divergence of the student's distribution q = softmax(logits_s / temperature) from the teacher's p and its gradient:
 *   loss[r] = forward KL(p || q) + reverse KL(q || p);   grad[r] = weight[r] d loss[r] / d logits_s[r]
 * forward = reverse = 1/2 at temperature 1 is Eq. 3, as hbsjd_bikl computes it.
 *   logits_s [rows, V] of type dtype_s;  grad [rows, V] of the same type, or NULL (loss only)
 *   weight   fp32 [rows] or NULL (all 1): a row's weight in the total, e.g. 1 / positions.  0 leaves the row out: it is not
 *            read, its loss is 0 and its gradient zeros
 *   loss     fp32 [rows] or NULL
 * An entry of -inf has no mass, neither has one of 88 temperatures and more below the row's largest (the type's lowest value
 * beside any other); between a share of 2^-126 and that it may count or not.
 * Where the divergence is infinite (the student has no mass where the teacher has: forward; the other way: reverse) so is the
 * loss, or as large as a finite masking value makes it; the gradient of KL(p || q) is q - p all the same, that of KL(q || p)
 * is then not defined.  A row without mass on one side has loss 0 and gradient 0.  NaN and +inf make the row's loss and
 * gradient NaN.  A small loss has digits of its own: rows near one another are summed as terms none of which is negative.
 *
 * hbsjd_distill: p = softmax(logits_t / temperature), logits_t [rows, V] of type dtype_t.
 *
 * hbsjd_distill_topk: the teacher as hbsjd_topk_logits lists it, values and indices [rows, k], 1 <= k <= 1024.  Entries
 * with a value of -inf, a token outside 0..V-1, or a token that an earlier entry of the row has, count for nothing.
 *   rest fp32 [rows]: all tokens that are not listed are one outcome, of mass e^rest beside the e^{value / temperature} of
 *                     those listed (same temperature); both divergences are over these k + 1 outcomes
 *   rest NULL:        the teacher is what is listed, renormalised; reverse has to be 0 */
typedef struct {
    int32_t rows, V, dtype_s, dtype_t, k, reserved;
    int64_t ld_s, ld_t, ld_grad;
    float temperature, forward, reverse;   /* forward, reverse >= 0 */
    uint32_t reserved2;
} hbsjd_distill_desc;
int hbsjd_distill(void *cuda_stream, const hbsjd_distill_desc *d, const void *logits_s, const void *logits_t,
                  const float *weight, float *loss, void *grad);
int hbsjd_distill_topk(void *cuda_stream, const hbsjd_distill_desc *d, const void *logits_s, const float *values,
                       const int32_t *indices, const float *rest, const float *weight, float *loss, void *grad);

/* ---- training by rewards and preferences -----------------------------------------------------------------------------------
 * The on-policy step without a teacher: log-probabilities of the sampled tokens, losses on them with their gradients, and the
 * clipping of the gradients that they end in.  The conventions are those of the operators on rows of logits (but where more
 * kernels or a workspace are named), with x = logits / temperature and q = softmax(x); tokens are int32 [rows], and one
 * outside 0..V-1 leaves its row out: it is not read, its outputs are 0 and its gradient zeros.  An entry of -inf has no mass; NaN and +inf make what their row gives NaN.
 *
 * hbsjd_token_logprobs: logp[r] = log q_token (-inf: no mass), entropy[r] = -sum q log q;  fp32 [rows], either may be NULL.  A row
 *   without mass: -inf and 0.
 * hbsjd_token_logprobs_grad: grad[r] = d (d_logp[r] logp[r] + d_entropy[r] entropy[r]) / d logits[r], what a loss of the caller's
 *   own gives back; d_logp, d_entropy fp32 [rows], d_entropy may be NULL.  Rows where both are 0 are left out. */
typedef struct {
    int32_t rows, V, dtype, reserved;
    int64_t ld, ld_grad;
    float temperature;
    uint32_t reserved2;
} hbsjd_token_desc;
int hbsjd_token_logprobs(void *cuda_stream, const hbsjd_token_desc *d, const void *logits, const int32_t *tokens, float *logp,
                         float *entropy);
int hbsjd_token_logprobs_grad(void *cuda_stream, const hbsjd_token_desc *d, const void *logits, const int32_t *tokens,
                              const float *d_logp, const float *d_entropy, void *grad);

/* hbsjd_token_logprobs of a model's own distributions over completed trajectories, at 8 bytes a position in place of 4 V: the old
 * policy's and the reference's sides of the losses below.  The model of context c runs the forwards of hbsjd_score; entry
 * [b, t - 1] of the outputs is of token x_t given x_<t, 0 for the positions t <= prefix_len[b].
 *   tokens DEVICE int32 [batch, T], prefix_len, class_labels DEVICE int32 [batch]: as hbsjd_score
 *   logp, entropy DEVICE fp32 [batch, T], entropy may be NULL
 * Runs on the context's stream and waits; its rollout state and KV caches are overwritten.  Errors as hbsjd_score. */
int hbsjd_score_logprobs(hbsjd_ctx *c, int batch, const int32_t *tokens, const int32_t *prefix_len, const int32_t *class_labels,
                         float temperature, float *logp, float *entropy);

/* The clipped policy loss of every row and its gradient.  With l = log q_token, r = e^{l - old_logp}, A = advantage, d = ref_logp - l:
 *   loss[r] = -min(r A, clip(r, 1 - clip_low, 1 + clip_high) A)      (A < 0 and dual_clip > 0: at most -dual_clip A)
 *             + kl (e^d - 1 - d) - entropy H;                         grad[r] = weight[r] d loss[r] / d logits[r]
 *   advantage fp32 [rows];  old_logp fp32 [rows] or NULL: l itself, the ratio is 1;  ref_logp fp32 [rows], NULL where kl = 0
 *   weight    fp32 [rows] or NULL (all 1): as hbsjd_distill; 0 leaves the row out
 *   loss, logp, entropy_out  fp32 [rows] or NULL;  grad [rows, V] of type dtype, or NULL
 * Where the ratio is clipped, its slope is 0.  A row without mass has loss 0 and gradient 0.  Of a token without mass the ratio is 0 (1
 * where old_logp is -inf, too); with a KL term against a finite ref_logp its loss is +inf, and its gradient not defined.
 * 0 <= clip_low <= 1, clip_high >= 0, dual_clip = 0 (none) or > 1, kl >= 0, entropy any finite number. */
typedef struct {
    int32_t rows, V, dtype, reserved;
    int64_t ld, ld_grad;
    float temperature, clip_low, clip_high, dual_clip, kl, entropy;
} hbsjd_policy_desc;
int hbsjd_policy_loss(void *cuda_stream, const hbsjd_policy_desc *d, const void *logits, const int32_t *tokens,
                      const float *advantage, const float *old_logp, const float *ref_logp, const float *weight, float *loss,
                      float *logp, float *entropy_out, void *grad);

/* A loss of pairs of sequences, one preferred to the other, and its gradient.  Sequence s is rows offsets[s] .. offsets[s + 1] - 1;
 *   S_s = sum over its rows of weight[r] (log q_token - ref_logp[r]),   h = S_chosen - S_rejected:
 *   HBSJD_PREFERENCE_SIGMOID  z = beta h - margin,  loss = -(1 - smoothing) log sigmoid(z) - smoothing log sigmoid(-z)
 *   HBSJD_PREFERENCE_HINGE    the same z,           loss = max(0, 1 - z)
 *   HBSJD_PREFERENCE_SQUARE   loss = (h - 1 / (2 beta))^2
 *   grad[r] = d (sum over pairs of pair_weight loss) / d logits[r]
 * Pair p is sequences 2 p (chosen) and 2 p + 1 where `interleaved`, else p (chosen) and pairs + p.
 *   offsets   int32 [2 pairs + 1], not decreasing, within 0..rows; else all losses, sums and gradients are NaN (but
 *             of rows whose token is none)
 *   ref_logp  fp32 [rows] or NULL (0);  weight fp32 [rows] or NULL (all 1): 0 leaves a row out;  pair_weight fp32 [pairs] or NULL
 *   loss fp32 [pairs] or NULL;  sums fp32 [2 pairs] or NULL: S_s;  logp fp32 [rows] or NULL: log q_token (0: left out)
 *   grad [rows, V] or NULL: zeros for rows of no sequence
 *   workspace hbsjd_preference_workspace(d) bytes, aligned to 16, which no other call uses at the same time; whatever it holds
 * smoothing in 0..1 and margin are 0 where the loss has none; beta > 0.  Launches three kernels. */
enum { HBSJD_PREFERENCE_SIGMOID = 0, HBSJD_PREFERENCE_HINGE = 1, HBSJD_PREFERENCE_SQUARE = 2 };
typedef struct {
    int32_t rows, V, dtype, pairs, kind, interleaved;
    int64_t ld, ld_grad;
    float temperature, beta, smoothing, margin;
} hbsjd_preference_desc;
size_t hbsjd_preference_workspace(const hbsjd_preference_desc *d);
int hbsjd_preference_loss(void *cuda_stream, const hbsjd_preference_desc *d, const void *logits, const int32_t *tokens,
                          const int32_t *offsets, const float *ref_logp, const float *weight, const float *pair_weight,
                          void *workspace, float *loss, float *sums, float *logp, void *grad);

/* The norm of all gradients as one vector, and their scaling by min(1, max_norm / (norm + 1e-6)).
 *   gradients, out, sizes, dtypes  HOST arrays [count]: DEVICE pointers to dense arrays of sizes[i] elements of type dtypes[i], which
 *             may be dropped when the call returns.  out NULL or out[i] = gradients[i]: in place, else out[i] gets the scaled ones, or
 *             copies where nothing is scaled; all of them or none.  No two arrays may overlap.
 *   norm      DEVICE fp32: before scaling.  HBSJD_NORM_2: root of the sum of squares, summed so that neither large nor small
 *             gradients leave the type's range on the way; HBSJD_NORM_MAX: the largest magnitude
 *   max_norm  >= 0; +inf: the norm alone.  Where the norm is infinite or NaN nothing is scaled, and the norm says so
 *   workspace hbsjd_clip_workspace(count) bytes, aligned to 16, which no other call uses at the same time; whatever it holds
 * 0 <= count <= 2^20.  The parameters of its kernels hold the pointers, so a captured call keeps them.  Launches two kernels (two
 * for each 1024 arrays beyond 128). */
enum { HBSJD_NORM_2 = 0, HBSJD_NORM_MAX = 1 };
typedef struct {
    int32_t count, norm;
    float max_norm;
    uint32_t reserved;
} hbsjd_clip_desc;
size_t hbsjd_clip_workspace(int count);
int hbsjd_clip_gradients(void *cuda_stream, const hbsjd_clip_desc *d, const void *const *gradients, void *const *out,
                         const int64_t *sizes, const int32_t *dtypes, void *workspace, float *norm);

/* Per-kernel-class timing with CUDA events on the context's stream (off by default).  While enabled,
 * every launch of a timed class is bracketed by an event pair; totals accumulate until the next
 * hbsjd_profile(c, 1), which also resets them.  work = algorithmic FLOPs (GEMM: 2 M N K per launch) or
 * algorithmic bytes (attention: K,V rows read + q read + output written; accept: logits read + probabilities
 * written) of the launches that were timed. */
enum { HBSJD_PROF_GEMM = 0, HBSJD_PROF_ATTENTION = 1, HBSJD_PROF_ACCEPT = 2, HBSJD_PROF_OTHER = 3 };
typedef struct {
    double ms[4];
    double work[4];
    int64_t launches[4];
    int64_t dropped;   /* launches not timed because the event pool was exhausted */
    /* the GEMM class again, split by the number of activation rows M of the launch:
     * M <= 512, 512 < M <= 2048, 2048 < M <= 6144, M > 6144 */
    double gemm_ms_by_rows[4];
    double gemm_work_by_rows[4];
    int64_t gemm_launches_by_rows[4];
    double gemm_bytes_by_rows[4];   /* algorithmic bytes: operands read once, outputs written (residual: read + written) */
} hbsjd_kernel_profile;
int hbsjd_profile(hbsjd_ctx *c, int enable);
int hbsjd_profile_read(hbsjd_ctx *c, hbsjd_kernel_profile *out);
/* What an event pair adds to a timed launch: an event between two kernels makes the second one start only after
 * the first has completed, so its launch latency lies inside the bracket (in normal operation the library's
 * kernels are launched programmatically dependent and that latency overlaps the previous kernel).  This call
 * brackets `reps` launches of an empty kernel in the same way and returns the median bracket in microseconds;
 * benchmarks report it beside the per-class times so that a reader can net it out. */
int hbsjd_profile_launch_floor(hbsjd_ctx *c, int reps, float *us_out);

const char *hbsjd_strerror(int code);
const char *hbsjd_last_error(const hbsjd_ctx *c);   /* NULL: of the calling thread's last failed call without a context */

#ifdef __cplusplus
}
#endif
#endif /* HBSJD_H_ */
