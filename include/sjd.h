/* sjd.h -- C ABI of the MI355X (gfx950) hot path of Speculative Jacobi Decoding (SJD).
 *
 * The problem (paper Sec. 4.1, first paragraph): after the prompt has been pre-filled, decode the
 * image tokens W at a time.  Each iteration runs ONE causal forward of the auto-regressive
 * transformer over the W draft tokens (Step 2), accepts a prefix of them with the probabilistic
 * criterion of Eq. 1, resamples the first rejected position from the calibrated distribution of
 * Eq. 2, re-draws every later position from this iteration's distributions (Eq. 3), and slides the
 * window (Step 4).  By Theorem 1 every produced token is distributed exactly as under ordinary
 * auto-regressive sampling.  W is called L here.
 *
 * Conventions
 *  - Every function returns SJD_OK (0) or a negative SJD_E* code; nothing aborts or throws.
 *  - "dev" pointers are device (HBM) addresses on the current HIP device, "host" pointers are
 *    ordinary host memory.  The caller owns every buffer it passes; the library owns only its
 *    opaque handles.  Buffers must not overlap unless stated.
 *  - `stream` is a hipStream_t passed as void* (NULL = the default stream).  Device work is
 *    enqueued on it and is asynchronous; outputs are valid once the caller has synchronised.
 *  - Probabilities and logits are fp32 rows over the SAMPLING vocabulary: column t stands for
 *    token id samp_lo + t, V_s = samp_hi - samp_lo columns per row.
 *  - All decisions are deterministic functions of the inputs: identical calls give identical bits.
 *  - Threads: a model is read-only once built; a cache handle (sjd_kv) is used by one host thread at a
 *    time.  Different handles of one model may be driven from different host threads on different streams
 *    at the same time (the handles of one batched call belong to that call).
 */
#ifndef SJD_H
#define SJD_H
#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

#define SJD_OK 0
#define SJD_EINVAL (-1) /* bad argument (null pointer, size out of range, unsupported shape)   */
#define SJD_ENOMEM (-2) /* device or host allocation failed                                    */
#define SJD_ESEQ (-3)   /* the call would run past max_seq                                     */
#define SJD_EHIP (-4)   /* a HIP runtime call failed; sjd_strerror() reports the last message  */
#define SJD_ELIMIT (-5) /* a size exceeds a fixed limit of the entry point; sjd_strerror() says which */

#define SJD_MAX_WINDOW 64     /* largest L accepted by sjd_step / sjd_generate                 */
#define SJD_MAX_ROWS 128      /* rows one window forward computes: L x contexts (2 under guidance) x
                                 images of a batch, each image's rows rounded up to a power of two  */
#define SJD_MAX_SAMP_VOCAB 32768 /* largest V_s the verification kernels hold in LDS          */

typedef struct sjd_model sjd_model; /* repacked device weights + tables; immutable after init  */
typedef struct sjd_kv sjd_kv;       /* KV cache, its length n, ids of the cached tokens, scratch */

/* Llama-style decoder (the paper fixes no architecture; Sec. 3.1 only requires an
 * auto-regressive transformer with a softmax classifier over the token vocabulary).          */
typedef struct {
    int32_t n_layers, d_model, n_heads, d_ffn;
    int32_t vocab_total, samp_lo, samp_hi; /* sampling ids = [samp_lo, samp_hi)                */
    int32_t max_seq;                       /* KV rows; needs prompt + N + L                    */
    int32_t dtype;                         /* 0 = fp32 throughout; 1 = bf16 weights, activations
                                              and cache as bf16 operand pairs hi + lo (about 16
                                              significant bits), fp32 accumulation             */
    float rope_theta, rms_eps;
} sjd_config;

/* top-K sampling (Sec. 3.1).  temperature == 0 or top_k == 1 selects greedy decoding, which
 * turns SJD into the deterministic Jacobi iteration of Sec. 3.2.                              */
typedef struct {
    int32_t top_k;
    float temperature;
} sjd_sampler;

/* Initialisation of new window slots (Sec. 4.2).  mode 0: uniform over the sampling ids;
 * mode 1: strategy (b), repeat the token one grid row above (uniform in the first grid row);
 * mode 2: strategy (a), repeat the token at the previous raster position;
 * mode 3: strategy (c), a fresh draw from the distribution on record for the nearest slot to the left
 *         that is not a forced row end (a run of new slots all draw from the last model row);
 * mode 4: strategy (d), a fresh draw from the distribution on record for the position one grid row
 *         up (the cache handle keeps the distributions of the last row_stride accepted positions;
 *         uniform in the first grid row).  The row drawn from is the slot's row in Eq. 1.
 * eol_id >= 0 forces that id at the last position of every grid row.
 * flags bit 0 (SJD_INIT_NO_REFINE): the ablation without refinement (App. "acceleration originates
 * from the refinement"): only the resampled position survives an iteration, every later slot of the
 * next window is newly initialised instead of re-drawn by Eq. 3.                                */
#define SJD_INIT_NO_REFINE 1
typedef struct {
    int32_t mode;
    int32_t row_stride; /* image tokens per grid row, a row-end token included                 */
    int32_t eol_id;
    int32_t flags;
} sjd_init;

typedef struct {
    int32_t steps;           /* window forwards (the paper's "decoding steps", Sec. 5.1)        */
    int32_t accept_hist[65]; /* accept_hist[a] = number of steps that accepted a tokens         */
    float ms_prefill;        /* host wall-clock of the prefill, milliseconds                    */
    float ms_decode;         /* host wall-clock of the decoding loop (all steps), milliseconds  */
} sjd_stats;

/* ---- model and cache ---------------------------------------------------------------------- */
/* host_weights: flat blob, element type per cfg->dtype (fp32, or bf16 bit patterns), tensors in
 * the order E[vocab,d]; per layer g1[d] Wq Wk Wv Wo [d,d] g2[d] Wg Wu [F,d] Wd [d,F]; gf[d];
 * Wlm[vocab,d]; every matrix row-major [out][in].  The blob is copied and repacked; the pointer
 * is not retained.  nbytes must match the configuration exactly (else SJD_EINVAL).            */
int sjd_init_model(const sjd_config *cfg, const void *host_weights, size_t nbytes, sjd_model **out);
void sjd_free_model(sjd_model *m);

/* A handle holds its cache and scratch for forwards of up to SJD_MAX_ROWS rows: at 7B about 47 MB besides the
 * cache and the rows of logits (17 of them partial sums of the projections), used by its own prompts and
 * iterations and, in a batch, by those of the batch's first handle for all.                     */
int sjd_kv_create(const sjd_model *m, sjd_kv **out);
void sjd_kv_free(sjd_kv *kv);
int sjd_kv_reset(sjd_kv *kv);                     /* n = 0                                       */
int sjd_kv_len(const sjd_kv *kv, int32_t *n);     /* synchronises the device, then reads n       */
int sjd_kv_set_len(sjd_kv *kv, int32_t n);        /* roll the cache back/forward to n rows (resume) */

/* ---- the path ----------------------------------------------------------------------------- */
/* Pre-fill the prompt (Sec. 4.1 "after pre-filling the tokens of text prompts"): n_ids token ids
 * (host) followed by n_embeds raw embedding rows (host fp32 [n_embeds x d_model]); either may be
 * empty, not both.  Resets the cache, leaves n = n_ids + n_embeds, and writes
 * q_last (dev [V_s]) = the sampling distribution of the first image token.                     */
int sjd_prefill(sjd_model *m, sjd_kv *kv, const int32_t *ids, int32_t n_ids, const float *embeds,
                int32_t n_embeds, const sjd_sampler *smp, const sjd_init *init, float *q_last, void *stream);

/* Classifier-free guidance (Sec. 5.1 runs its text-to-image models with guidance weight 3; the
 * mechanism is the usual one in logit space): right after sjd_prefill, pre-fill a second,
 * unconditional prompt into a second cache of the same handle.  From then on every window forward
 * runs both contexts on the same draft tokens (one pass over the weights, 2 x L rows) and Step 3
 * works on z = z_uncond + guidance * (z_cond - z_uncond); both caches advance by the accepted
 * count.  q_last is overwritten with the guided distribution of the first image token.  Windows go
 * up to SJD_MAX_WINDOW tokens with guidance on as well (two contexts x 64 rows = SJD_MAX_ROWS; fp32
 * models: 32); the next sjd_prefill switches it off.                                             */
int sjd_prefill_uncond(sjd_model *m, sjd_kv *kv, const int32_t *ids, int32_t n_ids, const float *embeds,
                       int32_t n_embeds, float guidance, const sjd_sampler *smp, const sjd_init *init, float *q_last,
                       void *stream);

/* First Jacobi window (Sec. 4.1 "starts with a sequence of initialized candidate tokens"):
 * slot 0 is sampled from q_first (dev [V_s]) and carries it as its distribution; slots 1..L-1
 * follow `init`.  Uses step counter 0.  draft dev [L], p_old dev [L x V_s].                   */
int sjd_first_window(const sjd_model *m, const float *q_first, int32_t L, const sjd_init *init,
                     uint64_t philox_seed, int32_t *draft, float *p_old, void *stream);

/* One SJD iteration (Sec. 4.1 Steps 1-4) on the window that starts at cache length n:
 *   draft   dev [L]        token ids of the window (Step 1)
 *   p_old   dev [L x V_s]  the distribution each draft was drawn from; row 0 must be the exact
 *                          conditional of draft[0] (it is never re-verified)
 *   img_pos0               image index of draft[0] (decides row ends and the row above)
 *   philox_seed, counter   random stream: Philox4x32-10 keyed by the seed, counter = (counter,
 *                          window index); counter 0 belongs to sjd_first_window
 * Outputs (dev): n_accepted[1] in [1, L]; new_draft[L] and p_new[L x V_s] already in the layout
 * of the next window (unaccepted positions first, then newly initialised slots).  new_draft may
 * alias draft and p_new may alias p_old.  The cache length advances by n_accepted and the ids of
 * the accepted tokens are recorded in the cache.  SJD_ESEQ if n + L > max_seq.                 */
int sjd_step(sjd_model *m, sjd_kv *kv, const int32_t *draft, const float *p_old, int32_t L,
             const sjd_sampler *smp, const sjd_init *init, int32_t img_pos0, uint64_t philox_seed,
             uint64_t counter, int32_t *n_accepted, int32_t *new_draft, float *p_new, void *stream);

/* Whole generation: prefill, first window, then iterations until N image tokens are fixed.
 * out_tokens host [N]; stats may be NULL.  Runs on the default stream and synchronises.        */
int sjd_generate(sjd_model *m, sjd_kv *kv, const int32_t *ids, int32_t n_ids, const float *embeds,
                 int32_t n_embeds, int32_t N, int32_t L, const sjd_sampler *smp, const sjd_init *init,
                 uint64_t philox_seed, int32_t *out_tokens, sjd_stats *stats);

/* sjd_generate with classifier-free guidance: both prompts, then the guided loop.                */
int sjd_generate_cfg(sjd_model *m, sjd_kv *kv, const int32_t *ids, int32_t n_ids, const float *embeds,
                     int32_t n_embeds, const int32_t *uncond_ids, int32_t n_uncond_ids, const float *uncond_embeds,
                     int32_t n_uncond_embeds, float guidance, int32_t N, int32_t L, const sjd_sampler *smp,
                     const sjd_init *init, uint64_t philox_seed, int32_t *out_tokens, sjd_stats *stats);

/* The same loop in pieces, with the loop state (cache length, image position, Philox counter,
 * window, its distributions) resident on the device so that iterations can be enqueued without
 * waiting for the outcome of the previous one (Sec. 4.1: the accepted count of Step 3 decides
 * where the next window starts, which is a data dependence, not a host decision).
 *   sjd_decode_begin   after sjd_prefill: first window from q_first (dev [V_s]), counters reset.
 *   sjd_decode_steps   enqueue n_steps iterations on `stream` (one HIP-graph replay each);
 *                      an iteration that starts after the N-th token is fixed changes nothing
 *                      (its forward still runs, on rows nobody reads: do not enqueue far past
 *                      the end; an iteration fixes at most L tokens).
 *   sjd_decode_status  synchronise; image tokens fixed so far, iterations run, finished flag.
 *   sjd_decode_result  after `done`: the N tokens (host) and the step statistics.
 *   sjd_kv_use_graph   0: launch kernels one by one instead of replaying a captured graph.     */
int sjd_decode_begin(sjd_model *m, sjd_kv *kv, const float *q_first, int32_t N, int32_t L,
                     const sjd_sampler *smp, const sjd_init *init, uint64_t philox_seed, void *stream);
int sjd_decode_steps(sjd_model *m, sjd_kv *kv, int32_t n_steps, void *stream);
int sjd_decode_status(sjd_kv *kv, int32_t *n_fixed, int32_t *steps, int32_t *done);
int sjd_decode_result(sjd_kv *kv, int32_t *out_tokens, sjd_stats *stats);
int sjd_kv_use_graph(sjd_kv *kv, int32_t on);

/* Per-kernel-class timing: runs n_steps iterations of the loop above kernel by kernel, every launch
 * carrying a start/stop HIP event pair that the runtime stamps with the kernel's own begin and end
 * (on `stream`), and adds up milliseconds, launch counts and HBM bytes (weights for the
 * projections; for attention the K/V records, as stored -- hi and lo halves, twice the bf16 size --
 * of the positions each profiled step really attended over; logits + both probability windows for
 * the verification) per class.  The per-launch intervals include a few microseconds of dispatch latency each, so the
 * projections (the dominant class) are timed a second time: the projection launches of n_steps
 * iterations alone, back to back in one event interval (ms_gemm_back_to_back; the same number of
 * launches and bytes as in the per-launch pass).  Synchronises.                                */
#define SJD_PROF_GEMM 0        /* QKV / O / gate-up / down projections and the LM head           */
#define SJD_PROF_ATTENTION 1   /* window attention incl. the merge of its key chunks             */
#define SJD_PROF_ELEMENTWISE 2 /* embedding, RMSNorm, RoPE + cache write, SiLU*up, reductions    */
#define SJD_PROF_VERIFY 3      /* Sec. 4.1 Step 3 + Step 4 kernels                               */
typedef struct {
    double ms[4];
    double bytes[4];
    int64_t launches[4];
    int32_t steps;
    double ms_gemm_back_to_back;
} sjd_profile;
int sjd_profile_steps(sjd_model *m, sjd_kv *kv, int32_t n_steps, sjd_profile *out, void *stream);
/* the same for iterations of sjd_decode_steps_batch */
int sjd_profile_steps_batch(sjd_model *m, sjd_kv *const *kvs, int32_t B, int32_t n_steps, sjd_profile *out,
                            void *stream);

/* ---- batched decoding --------------------------------------------------------------------------
 * B independent images share every window forward (Sec. 4.1 Step 2 for B windows at once): one pass
 * over the weights serves B x L rows, so an iteration costs little more than for one image and the
 * throughput grows almost B-fold.  Each image keeps its own handle (cache, loop state, random
 * stream); Steps 3 and 4 run per image exactly as in sjd_decode_steps.  bf16 models.  Guidance: all
 * handles guided (each after its own sjd_prefill_uncond, each with its own weight) or none; a guided
 * image brings two contexts.  The contexts' windows (each rounded up to a power of two of rows) must
 * fit the SJD_MAX_ROWS rows of one forward, at most 8 contexts: L <= 64 for 2 contexts, L <= 32 for
 * up to 4, L <= 16 for up to 8.  The first handle lends its activation buffers and, with graphs on,
 * holds the captured iteration (re-captured when the set of handles or their settings change).
 *
 * sjd_decode_steps_batch: every handle has been through sjd_prefill (+ sjd_prefill_uncond) +
 * sjd_decode_begin with the same L, sampler and initialiser (seeds may differ); poll and collect per handle with
 * sjd_decode_status / sjd_decode_result.  A handle whose image is complete sits out further
 * iterations.  kvs: host array of B distinct handles.                                          */
int sjd_decode_steps_batch(sjd_model *m, sjd_kv *const *kvs, int32_t B, int32_t n_steps, void *stream);

/* Prompts to images for B handles, without guidance (it pre-fills every handle anew; guided batches go
 * through the pieces above).  ids / embeds: host arrays of B host pointers (embeds and
 * n_embeds may be NULL), out_tokens host [B x N], stats host [B] or NULL (times are the batch's). */
int sjd_generate_batch(sjd_model *m, sjd_kv *const *kvs, int32_t B, const int32_t *const *ids, const int32_t *n_ids,
                       const float *const *embeds, const int32_t *n_embeds, int32_t N, int32_t L,
                       const sjd_sampler *smp, const sjd_init *init, const uint64_t *philox_seeds, int32_t *out_tokens,
                       sjd_stats *stats);

/* ---- pieces of the step, exported for parity tests and profiling --------------------------- */
/* Step 2 alone: forward `L` tokens (dev ids) at positions n..n+L-1, write their K/V rows, return
 * logits dev [L x V_s] fp32 (the guided logits while guidance is on).  Does not advance n.     */
int sjd_forward_logits(sjd_model *m, sjd_kv *kv, const int32_t *tokens, int32_t L, float *logits, void *stream);

/* The same for B handles in one forward: tokens dev [B x L], logits dev [B x L x V_s] (of guided handles:
 * the guided logits).  A handle
 * inside a generation (sjd_decode_begin) whose image is complete takes no part: what its rows of
 * `logits` hold afterwards means nothing.                                                        */
int sjd_forward_logits_batch(sjd_model *m, sjd_kv *const *kvs, int32_t B, const int32_t *tokens, int32_t L,
                             float *logits, void *stream);

/* Step 3 + Step 4 alone, from logits (row s belongs to window index s+1).  hist: dev ids of the
 * image tokens fixed so far [img_pos0] (may be NULL when init->mode is 0 or 3, or img_pos0 == 0).
 * ring: dev [row_stride x V_s], in/out, init->mode == 4 only (else may be NULL): entry p % row_stride
 * holds the distribution on record for accepted image position p; the call adds the positions it
 * accepts.  V_s <= SJD_MAX_SAMP_VOCAB.                                                          */
int sjd_verify(const float *logits, const float *p_old, const int32_t *draft, int32_t L, int32_t V_s,
               int32_t samp_lo, const sjd_sampler *smp, const sjd_init *init, int32_t img_pos0,
               const int32_t *hist, float *ring, uint64_t philox_seed, uint64_t counter, int32_t *n_accepted,
               int32_t *new_draft, float *p_new, void *stream);

/* Same from precomputed distributions q dev [(L+1) x V_s] (row 0 ignored, row L = the bonus
 * distribution of the position just past the window).                                          */
int sjd_verify_probs(const float *q, const float *p_old, const int32_t *draft, int32_t L, int32_t V_s,
                     int32_t samp_lo, const sjd_init *init, int32_t img_pos0, const int32_t *hist, float *ring,
                     uint64_t philox_seed, uint64_t counter, int32_t *n_accepted, int32_t *new_draft,
                     float *p_new, void *stream);

/* sjd_verify for callers that cannot allocate device memory (code under HIP graph capture, tight
 * serving loops, harnesses that forbid hipMalloc): same arguments, same outputs, but the scratch that
 * sjd_verify allocates per call (the distributions of the L + 1 window indices, candidates, flags)
 * lives in a static device array of the library, SJD_STATIC_VERIFY_FLOATS floats (1.06 MiB, held on
 * every GPU the library runs on until the process ends).  The call allocates nothing, frees nothing
 * and does not synchronise: outputs are valid once `stream` has been synchronised.  SJD_ELIMIT when
 * (L + 1) * V_s exceeds SJD_STATIC_VERIFY_FLOATS (the 7B and 775M workloads fit: 33 x 8192 and
 * 17 x 16384).  Every call on a GPU shares that GPU's array: calls that overlap on one GPU (two
 * streams, two threads) race; run them one after the other.                                      */
#define SJD_STATIC_VERIFY_FLOATS (17 * 16384)
int sjd_verify_static(const float *logits, const float *p_old, const int32_t *draft, int32_t L, int32_t V_s,
                      int32_t samp_lo, const sjd_sampler *smp, const sjd_init *init, int32_t img_pos0,
                      const int32_t *hist, float *ring, uint64_t philox_seed, uint64_t counter, int32_t *n_accepted,
                      int32_t *new_draft, float *p_new, void *stream);

/* The sampling distribution of Sec. 3.1 for `rows` logits rows: top-K, temperature, softmax.
 * forced: dev [rows] column index to make one-hot, or -1; may be NULL.  q dev [rows x V_s].     */
int sjd_dist(const float *logits, int32_t rows, int32_t V_s, const sjd_sampler *smp, const int32_t *forced,
             float *q, void *stream);

/* C[M x N] (fp32, dev) = A[M x K] * W[N x K]^T with the kernel the model uses for its projections.
 * dtype as in sjd_config; A and W are dev, row-major, element type per dtype; W is repacked into
 * the library's streaming layout first (not timed separately).  dtype 2: W bf16 and A fp32, A taken
 * through the 3-byte form (16 significant bits) in which bf16 models hand the attention output and
 * the FFN hidden to their projections.  For kernel-level parity tests.                            */
int sjd_gemm_test(int32_t dtype, const void *A, const void *W, int32_t M, int32_t N, int32_t K, float *C,
                  void *stream);

/* Which kernel a projection of a bf16 model (M rows, N x K weights) runs on, without running it (no GPU needed).  resid: its
 * output is added to the residual stream (O, down).  *kernel: SJD_GEMM_*; *tn: 16-feature tiles per packed weight group; *g: weight
 * groups per workgroup (span, sliced) or per wave (wide), else 1; *ks: K-slices.                 */
#define SJD_GEMM_SKINNY 0    /* up to 32 rows: a group per workgroup, its waves split K                        */
#define SJD_GEMM_SPAN 1      /* a workgroup owns its groups for the whole reduction, at any row count           */
#define SJD_GEMM_SLICED 2    /* the same with K cut into slices whose sums meet in one launch                    */
#define SJD_GEMM_WIDE 3      /* waves split N, K cut into slices, a second kernel adds them                      */
int sjd_gemm_plan(int32_t M, int32_t N, int32_t K, int32_t resid, int32_t *kernel, int32_t *tn, int32_t *g, int32_t *ks);

/* Tuning aid: average microseconds per launch of the bf16 projection kernel (plain-store epilogue) at
 * shape M x N x K over `iters` back-to-back launches on zero-filled operands (activations in the
 * 3-byte form the model's projections read).  `tn` = output tiles
 * per workgroup (1..3), wk = waves splitting K (8 or 4; 0 = the choice the model makes), u = k-steps per
 * prefetch stage (2; 4 for wk = 4, M <= 16; 0 = the choice the model makes).
 * wk >= 200: the span kernel with K cut into wk - 200 slices whose sums meet in one launch, u one-tile groups per workgroup
 * (u = 2 with up to 8 slices, 8 with up to 8 slices and 32 rows, 4 with up to 4 at 33 .. 64 rows; tn = 1).
 * wk = u = 0 runs the kernel that the model would for QKV, gate/up and the LM head (sjd_gemm_plan with resid = 0), wk = -1 and
 * u = 0 the one for O and down (resid = 1), provided that tn is the packing the plan gives.
 * More than 32 rows otherwise run the wide kernel (waves split N and share the activations through LDS, K split
 * across workgroups, a second kernel adds the slices): then wk = K-slices and u = weight groups per wave
 * (0 = automatic); wk >= 100 asks for the wide kernel at any row count, with wk - 100 K-slices.  M above
 * SJD_MAX_ROWS is an off-path measurement of the wide kernel's matrix-core rate: the rows are cut into
 * chunks of SJD_MAX_ROWS, one launch pair each over the same weights.
 * A negative `iters` times |iters| launches that rotate through more than 1 GiB of weight copies,
 * so that no launch finds its weights in the last-level cache (the situation inside a step).
 * tn = 0 measures the floor instead of the projection: a kernel that only reads the same N x K x 2 bytes
 * (wk workgroups of 256 threads, 0 = 256, four 16-byte loads per lane in flight; u = 0: every workgroup a
 * contiguous share, as the projection kernels read their packed weights; u = 1: all workgroups sweep the bytes
 * together, 4 KiB per wave and round).
 * SJD_EINVAL for an unsupported combination.                                                     */
int sjd_gemm_bench(int32_t M, int32_t N, int32_t K, int32_t tn, int32_t wk, int32_t u, int32_t iters,
                   float *us_per_launch);

/* ---- microscaled operators ----------------------------------------------------------------------
 * The operators of a decoder layer whose weights have 4 bits, whose activations have 8 (or 4) and whose
 * cache has 8.  A 7B layer's weights are 0.27 of their bf16 bytes, a cached token a quarter of what bf16
 * models store.  Rounded like this a layer is an approximation (E2M1 keeps one mantissa bit): these calls
 * stand beside sjd_gemm_test and sjd_dist for programs that build such a layer; sjd_step does not use them.
 *
 * Numbers.  E4M3: sign, 4 exponent bits (bias 7), 3 mantissa bits, largest 448, 0x7F is NaN, no infinity.
 * E2M1: 0, 0.5, 1, 1.5, 2, 3, 4, 6 and their negatives, code bit 3 the sign.  Every 32 values along a row
 * (the cache: the 32 positions of a block x head_dim, keys and values apart) share the scale
 * 2^(byte - 127), the smallest power of two (byte >= 0) with which the largest finite magnitude does not
 * exceed 448 (E4M3) or 6 (E2M1) times it: nothing saturates, and rounding to the format (nearest, ties to
 * even) is the only loss.  The scale byte of a block of zeros is 0.  An infinity or NaN becomes the code
 * 0x7F (E4M3) and does not count for the scale; E2M1 has no such code: a block that holds one gets the
 * scale byte 255, which is NaN, and codes 0.
 * A row of K values is held as Kp = K rounded up to a multiple of 128: codes [rows][Kp] bytes (E4M3) or
 * [rows][Kp / 2] (E2M1, the first of two values in the low half), scales [rows][Kp / 32]; what lies behind
 * K is zero.
 *
 * dtype: 0 = fp32, 1 = bf16.  ld*: elements from one row to the next (at least the row's length; rows of
 * a wider matrix may be given).  codes, scales, packed weights, caches and workspaces: 16-byte aligned.
 * These calls allocate nothing and do not synchronise, so they can be captured into a graph.  A
 * workspace holds nothing between calls; calls (and captured graphs) that may run at the same time need
 * one each.  SJD_EINVAL: a size, type, alignment or workspace that does not fit, or a launch of 2^32 threads
 * (hundreds of millions of rows).                                                                   */
#define SJD_MX8 8                  /* E4M3 */
#define SJD_MX4 4                  /* E2M1 */
#define SJD_MX_MAX_K (1 << 20)     /* longest row */

/* x dev [rows x K] -> codes, scales in `format`.  up != NULL (dev, like x): of SiLU(x) * up instead.   */
int sjd_mx_quantize(int32_t format, int32_t dtype, const void *x, const void *up, int64_t ld, int32_t rows, int32_t K,
                    uint8_t *codes, uint8_t *scales, void *stream);

/* h = resid + x, kept in resid (dev fp32 [rows x d], in and out); h / sqrt(mean(h^2) + eps) * gain -> codes,
 * scales in `format`.  gain dev fp32 [d].  x NULL: h = resid (dtype and ldx are ignored); resid NULL: h = x, and nothing is kept.
 * Not both.  Sums of squares are fp32: a row of zeros with eps = 0 gives NaN, as the formula does, and so may rows whose squares underflow
 * (below 1e-19) with eps = 0; rows whose squares overflow (above 1e19) give zeros.                   */
int sjd_mx_rmsnorm(int32_t format, int32_t dtype, const void *x, int64_t ldx, float *resid, int64_t ldr, const float *gain,
                   float eps, int32_t rows, int32_t d, uint8_t *codes, uint8_t *scales, void *stream);

/* Weights W dev [N x K] -> E2M1, in the order in which the product streams them.  Tile t (16 features) and group
 * g (512 values) are one record of 4352 bytes at (t * ceil(K / 512) + g) * 4352.  Byte 1024 s + 16 (16 q + f) + j holds
 * W[16 t + f][512 g + 128 s + 32 q + 2 j] (low half) and the next value; byte 4096 + 4 (16 q + f) + s their
 * scale.  What lies behind N or K is zero.  sjd_mx_weights_bytes: the size.                            */
int sjd_mx_weights_bytes(int32_t N, int32_t K, size_t *bytes);
int sjd_mx_weights(int32_t dtype, const void *W, int64_t ld, int32_t N, int32_t K, uint8_t *packed, void *stream);

/* C[M x N] (dev, dtype, row length ldc) = A W^T: A codes and scales in `format` as above (K values a row), W packed.  fp32 results:
 * products of codes are exact, sums are fp32.  bf16 results from E4M3 rows: among eight neighbouring products (columns 8 i .. 8 i + 7)
 * each is cut towards zero by less than 2^-13 of the largest one; that is 5e-6 of a result in the 2-norm of random rows, and may be all of a
 * result whose large products cancel.  Sums are fp32 and rounded once.  workspace: sjd_mx_product_workspace bytes (may be 0).   */
int sjd_mx_product_workspace(int32_t M, int32_t N, int32_t K, size_t *bytes);
int sjd_mx_product(int32_t format, const uint8_t *codes, const uint8_t *scales, const uint8_t *packed, int32_t M, int32_t N,
                   int32_t K, int32_t dtype, void *C, int64_t ldc, void *workspace, size_t workspace_bytes, void *stream);

/* Which kernel sjd_mx_product runs on (no GPU needed): *rows x *cols of C to a workgroup, K in *slices.  16 or 32 rows: the kernel for
 * few rows, whose waves split K; else one of 64 x 64, 64 x 128, 64 x 192, 128 x 128, 128 x 192, 128 x 256 and 256 x 256, for more than
 * 32 rows, in 1, 2 or 4 slices (of whole groups of 512 values, so perhaps fewer).                     */
int sjd_mx_product_plan(int32_t M, int32_t N, int32_t K, int32_t *rows, int32_t *cols, int32_t *slices);

/* sjd_mx_product on the kernel that is named as above, whatever the plan says; workspace: slices * M * (N up to a multiple of 4) floats
 * where slices > 1.  For kernel-level parity tests.  SJD_EINVAL for a kernel that no plan has for M.     */
int sjd_mx_product_test(int32_t rows, int32_t cols, int32_t slices, int32_t format, const uint8_t *codes, const uint8_t *scales,
                        const uint8_t *packed, int32_t M, int32_t N, int32_t K, int32_t dtype, void *C, int64_t ldc, void *workspace,
                        size_t workspace_bytes, void *stream);

/* A cache in 8 bits of n_seqs sequences, `cap` positions each: cache dev [n_seqs][n_kv_heads][ceil(cap / 32)][64 * head_dim],
 * scales dev [n_seqs][n_kv_heads][ceil(cap / 32)][2] (keys, values).  head_dim: 32, 64, 96, 128 or 256.  A block's record
 * holds its keys, then its values, as the lanes of the attention read them:
 *   K[p][d] at 1024 (o / 2) + 16 l + 8 (o % 2) + d % 8, o = (p / 16)(head_dim / 32) + d / 32, l = 16 (d % 32 / 8) + p % 16
 *   V[p][d] at 32 head_dim + 1024 (o / 2) + 16 l + 8 (o % 2) + 4 (p / 16) + p % 4, o = d / 16, l = 16 (p % 16 / 4) + d % 16
 * len dev [n_seqs]: cached positions per sequence before the window; the window's L tokens are positions len .. len + L - 1.
 * A sequence with len < 0 or len + L > cap sits out: neither its cache nor its rows of `out` are touched.
 *
 * sjd_kv8_append: k, v dev [n_seqs * L][n_kv_heads * head_dim] (rows of length ld) into the cache.  The scale of a block that holds
 * positions already is made anew from those and the new ones; their codes move to it (exact but for codes that become
 * subnormal).  Positions of a touched block behind the window are zero afterwards; other blocks are not touched.  A window may be
 * appended again at the same or a smaller len (after a rejection).  len itself is the caller's to advance.
 * So the cache is not strictly causal inside a block: keys and values that are more than 2^13 times smaller than the largest of their
 * block, of a later position or of a draft too, are rounded to that one's grid, by up to 2^-16 of it, for the queries of the same forward
 * already, and stay rounded when that position is rejected.  Where a decoder compares probabilities of two forwards, they differ by what
 * that gives; values within 2^13 of each other keep their codes, and a block of 32 positions is not touched by any other.       */
int sjd_kv8_append(int32_t dtype, const void *k, const void *v, int64_t ld, const int32_t *len, int32_t n_seqs, int32_t L,
                   int32_t n_kv_heads, int32_t head_dim, int32_t cap, uint8_t *cache, uint8_t *scales, void *stream);

/* Attention of the window's queries q dev [n_seqs * L][n_heads * head_dim] (rows of length ldq) over the cache, the appended window
 * included: softmax(q k / sqrt(head_dim)) v.  The query at position p sees the positions j <= p with, if window > 0, also
 * j > p - window or j < sinks.  Query head h reads cache head h / (n_heads / n_kv_heads).  out dev, like q, rows of length ldo,
 * of the same dtype (which also says how finely probabilities are held: 22 bits for fp32, 11 for bf16).  workspace:
 * sjd_kv8_attention_workspace bytes (may be 0).  n_seqs is at most 32767, n_seqs * ceil(L * n_heads / n_kv_heads / 16) at most 65535.
 * Scores are fp32: one that overflows there gives NaN.  What masked positions hold, NaN included, does not reach `out`.               */
int sjd_kv8_attention_workspace(int32_t n_seqs, int32_t L, int32_t n_heads, int32_t n_kv_heads, int32_t head_dim, int32_t cap,
                                size_t *bytes);
int sjd_kv8_attention(int32_t dtype, const void *q, int64_t ldq, const uint8_t *cache, const uint8_t *scales, const int32_t *len,
                      int32_t n_seqs, int32_t L, int32_t n_heads, int32_t n_kv_heads, int32_t head_dim, int32_t cap, int32_t window,
                      int32_t sinks, void *out, int64_t ldo, void *workspace, size_t workspace_bytes, void *stream);

/* ---- operators around a layer's products, over a paged cache ---------------------------------------
 * What a decoder layer does besides its products when its keys and values lie in pages: rotary positions, the append of new keys and
 * values, the attention over them, and the norms, gate and residual scale between two blocks.  They stand beside the microscaled operators, for
 * programs that build their own layers (sjd_step uses neither), keep everything in the type it comes in (dtype: 0 = fp32, 1 = bf16) and
 * hold sums, statistics and angles in 32 bits or more.  They allocate nothing, do not synchronise and can be captured into a graph; workspaces hold
 * nothing between calls, calls that may run at the same time need one each.  ld*: elements from one row to the next.  SJD_EINVAL: a size, type,
 * alignment or workspace that does not fit, or a launch of 2^32 threads.
 *
 * Rotary positions.  A frequency is a whole number of 2^-64 turns a position, turns dev uint64 [rot_dim / 2]; a position's angle is their product
 * modulo whole turns, exact however far the position is (any int32, negative ones too).  Pair i of a head, values (i, i + rot_dim / 2) or, interleaved = 1,
 * (2 i, 2 i + 1), becomes magnitude * (a cos - b sin, b cos + a sin); values from rot_dim on stay.  rot_dim is even and at most head_dim.
 * sjd_rope_turns fills a host table (no GPU needed), 2 <= rot_dim <= 256, 1 < theta <= 1e30, with f_i = theta^(-2 i / rot_dim) radians a position, scaled:
 *   LINEAR  f_i / factor
 *   BASE    theta * factor^(rot_dim / (rot_dim - 2)) in theta's place (rot_dim > 2)
 *   PARTS   with n_i = original f_i / 2 pi turns in the trained context and w = (n_i - slow) / (fast - slow) cut to 0 .. 1: w f_i + (1 - w) f_i / factor
 * (1 <= factor <= 1e6; a magnitude of 0.1 ln(factor) + 1 goes with PARTS where scores are to keep their spread.)  Other frequencies may be written into the
 * table by hand.
 *
 * sjd_rope: x dev [rows x n_heads * head_dim] -> out, alike, rows turned by pos dev int32 [rows] (inverse = 1: by minus the angle, which is also the gradient).
 * out may be x.  Any even head_dim up to 256.  Rows of 16-byte units with rot_dim % 16 = 0 and head_dim % 16 = 0 take the faster kernel.   */
#define SJD_ROPE_PLAIN 0
#define SJD_ROPE_LINEAR 1
#define SJD_ROPE_BASE 2
#define SJD_ROPE_PARTS 3
int sjd_rope_turns(double theta, int32_t rot_dim, int32_t scaling, double factor, double original, double slow, double fast, uint64_t *turns);
int sjd_rope(int32_t dtype, const void *x, int64_t ldx, void *out, int64_t ldo, const int32_t *pos, int32_t rows, int32_t n_heads, int32_t head_dim,
             const uint64_t *turns, int32_t rot_dim, int32_t interleaved, float magnitude, int32_t inverse, void *stream);

/* A pool of pages for one layer: cache dev [n_pages][n_kv_heads][page / 32] records of 64 * head_dim values of dtype, 16-byte aligned.  page: a power of two
 * of positions, 32 .. 65536; head_dim: 32, 64, 96, 128 or 256.  Position p of sequence b is in page table[b][p / page] (table dev int32 [n_seqs x width]), there in
 * record p % page / 32 of each head.  A record holds the keys, then the values of 32 positions in units of 16 bytes, E = 8 (bf16) or 4 (fp32) values:
 *   K[p][d] at E (32 (d / E) + p) + d % E                                      (a unit: E dimensions of a position)
 *   V[p][d] at 32 head_dim + E ((1024 / E) (d / 32) + 32 u + d % 32) + e       (a unit: a dimension of E positions)
 *     bf16: p = 16 t + 8 j + 4 h + i, u = 2 t + h, e = 4 j + i                 fp32: u = p / 4, e = p % 4
 * A call is about `rows` rows of n_seqs sequences: start dev int32 [n_seqs + 1], ascending, rows start[b] .. start[b + 1] - 1 are the new tokens of sequence b, any
 * number from zero on, and stand at positions len[b] .. (len dev int32 [n_seqs], positions before them).  Rows outside all sequences are not touched.  A sequence with
 * len < 0, or whose tokens do not fit its table row, sits out: neither its pages nor its rows of the outputs are touched.  Where a table names a
 * page outside the pool nothing is stored, and nothing is seen.  len is the caller's to advance; tokens may be appended again at the same or a smaller len.  */
typedef struct { int32_t dtype, n_kv_heads, head_dim, page, n_pages; } sjd_pages;

/* k, v dev [rows x n_kv_heads * head_dim] (rows of length ld) into the pages, keys turned by their positions (turns NULL and rot_dim 0: as they are, without queries).  Other positions of the
 * records keep what they hold; a page that is written belongs to one sequence of the call.  q dev [rows x n_heads * head_dim], turned likewise, goes to q_out (which may
 * be q); both NULL: keys and values only.                                                        */
int sjd_page_append(const sjd_pages *pages, const void *q, int64_t ldq, int32_t n_heads, void *q_out, int64_t ldqo, const void *k, const void *v, int64_t ld,
                    int32_t rows, const int32_t *start, const int32_t *len, int32_t n_seqs, const int32_t *table, int32_t width, const uint64_t *turns,
                    int32_t rot_dim, int32_t interleaved, float magnitude, void *cache, void *stream);

/* Attention of the new tokens' queries q dev [rows x n_heads * head_dim] (as they are: turned already) over the pages, the tokens' own keys included:
 * softmax(scale q k) v -> out, like q, rows of length ldo.  The query at position p sees the positions j <= p with, if window > 0, also j > p - window or j < sinks; one
 * that sees nothing gives zeros.  (A prompt takes no less time for a window: all its tiles walk from the first block that its first token sees.)  Query head h reads cache head h / (n_heads / n_kv_heads).
 * Groups: the sequences groups[g] .. groups[g + 1] - 1 (groups dev int32 [n_groups + 1], ascending) begin with the same prefix[g] positions (dev int32 [n_groups]), say
 * images of one prompt, and their table rows name the same pages for the whole pages of it, prefix[g] / page of them: those are read and weighed once for all.
 * (What is left of the prefix lies in pages that each sequence goes on in, so in copies.)  The result does not depend on it but for the order of sums.  n_groups 0:
 * none.  With window > 0 groups are not used.
 * scale is above zero and below 1e30.  Scores and sums are fp32, bf16 probabilities have at least 8 bits.  A visible score that overflows upwards gives NaN; those that overflow
 * downwards weigh nothing, and a query that sees no others gives NaN.  A visible infinity or NaN among the values
 * gives an infinity or NaN in that dimension, and so may a finite one above 2^80: sums are up to 2^16 times what the softmax weighs, times the positions.
 * What masked positions hold, NaN included, does not reach `out`.  workspace: sjd_page_attention_workspace bytes (may be 0), 16-byte aligned.
 * rows <= 2^24, n_seqs <= 65535, heads <= 4096.                                                  */
int sjd_page_attention_workspace(const sjd_pages *pages, int32_t rows, int32_t n_seqs, int32_t n_groups, int32_t n_heads, int32_t width, size_t *bytes);
int sjd_page_attention(const sjd_pages *pages, const void *q, int64_t ldq, int32_t n_heads, int32_t rows, const int32_t *start, const int32_t *len, int32_t n_seqs,
                       const int32_t *table, int32_t width, const int32_t *groups, const int32_t *prefix, int32_t n_groups, const void *cache, float scale,
                       int32_t window, int32_t sinks, void *out, int64_t ldo, void *workspace, size_t workspace_bytes, void *stream);

/* Between two blocks of a decoder: h = resid + scale * gate * x / sqrt(mean(x^2) + eps) * post, kept in resid (dev fp32 [rows x d], in and out); h / sqrt(mean(h^2) + eps) * pre -> out.
 * x, out dev [rows x d] of dtype; post, pre dev fp32 [d]; gate dev of dtype, rows of length ldg (0: one row for all).  post NULL: x as it is; gate NULL: ones; pre and out
 * NULL: h only.  out may be x.  d <= SJD_NORM_MAX_D.  Sums of squares are fp32: rows whose squares overflow give zeros.                       */
#define SJD_NORM_MAX_D 16384
int sjd_block_norm(int32_t dtype, const void *x, int64_t ldx, const float *post, const void *gate, int64_t ldg, float scale, float *resid, int64_t ldr,
                   const float *pre, float eps, int32_t rows, int32_t d, void *out, int64_t ldo, void *stream);

const char *sjd_strerror(int code);

#ifdef __cplusplus
}
#endif
#endif
