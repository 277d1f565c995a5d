/*
 * keyformer.h -- C ABI of the B200 (sm_100a) Keyformer score-and-evict library.
 *
 * The library keeps, per (layer, batch row, head), a KV cache of at most k
 * entries together with each entry's original token position and accumulated
 * Keyformer score f_theta, and implements the two phases of Algorithm 1 of the
 * Keyformer paper:
 *
 *   prompt phase      kf_prefill_score_prune   (Algorithm 1 with m <- n; section 3.4)
 *   generation phase  kf_decode_step           (Algorithm 1 with m <- k; section 3.4)
 *
 * Conventions
 *   - Every pointer whose name starts with d_ is a DEVICE pointer, h_ a HOST pointer.
 *   - All device buffers, the workspace included, are owned by the caller; the
 *     context owns host metadata only and kf_destroy frees no device memory.
 *   - Q/K/V tensors are IEEE binary16 ("fp16"), contiguous, row-major in the
 *     shapes stated per call.  Scores are binary32.
 *   - Work is enqueued on the CUDA stream passed as `stream` (a cudaStream_t cast
 *     to void*; NULL = the default stream).  No call synchronises except
 *     kf_poll_error and the *_host variants' final wait when asked to.
 *   - Return value 0 = success, negative = one of the KF_E* codes; on an error
 *     detected on the host nothing has been enqueued.
 *   - There is no CPU fallback: without a CUDA device every compute call
 *     returns KF_ECUDA.
 */
#ifndef KEYFORMER_B200_H
#define KEYFORMER_B200_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

#define KF_OK        0
#define KF_EINVAL   -1   /* bad argument or configuration                         */
#define KF_ENOSPC   -2   /* workspace too small                                   */
#define KF_ESTATE   -3   /* call out of order (decode before prefill, ...)        */
#define KF_ECUDA    -4   /* a CUDA runtime call failed / no device                */
#define KF_ETIMEOUT -5   /* a bounded device-side wait ran out (error word)       */
#define KF_EBOUNDS  -6   /* a device-side bounds check failed (error word)        */

/* Logit adjustment zeta of Eq. 4 (section 4.4.3 lists the alternatives). */
#define KF_NOISE_GUMBEL 0   /* zeta = -ln(-ln u), standard Gumbel, Eq. 7 (the method) */
#define KF_NOISE_NONE   1   /* zeta = 0 (accumulated-attention score, H2O-like)      */
#define KF_NOISE_CONST  2   /* zeta = noise_const                                     */
#define KF_NOISE_GAUSS  3   /* zeta = noise_mu + noise_sigma * N(0,1) (the Gaussian alternative of section 4.4.3;
                               Box-Muller on two Philox words)                        */

/* How kf_prefill_score_prune computes the prompt logits Q K^T. */
#define KF_PREFILL_TENSOR 0 /* tcgen05 tensor cores, accumulators in tensor memory (default) */
#define KF_PREFILL_SIMT   1 /* CUDA cores; scores are summed with floating-point atomics     */

/* Which streaming kernel kf_decode_step uses. */
#define KF_DECODE_AUTO       0 /* tensor cores where several query heads share a cache and head_dim is 128, else CUDA cores */
#define KF_DECODE_CUDA_CORES 1 /* lane-per-row mixed-precision fma (every shape)                                          */
#define KF_DECODE_TENSOR     2 /* tcgen05 logits and value sums, accumulators in tensor memory (head_dim 128 only)        */

#define KF_BIAS_NONE  0
#define KF_BIAS_ALIBI 1     /* x_ij += -slope_h * (i - j); which i and j is chosen by pos_mode */

/* Positional information seen by the bias once the cache has been reduced (section 4.4.2). */
#define KF_POS_ORIGINAL 0   /* i, j = positions of the tokens in the text ("Org Pos", the method's default) */
#define KF_POS_NEW      1   /* i, j = places within the reduced cache, counted in position order ("New Pos"):
                               the oldest kept entry is 0, the current token is the last.  Only the generation
                               phase differs (nothing has been dropped while the prompt is scored); the noise
                               is keyed by the original positions in both modes.                              */

typedef struct kf_ctx kf_ctx;

/* Inputs of Algorithm 1 (cache size k, recent window w, generation length T,
 * tau_init, tau_end) plus the tensor geometry. */
typedef struct kf_config {
  int32_t n_layers;        /* L >= 1                                              */
  int32_t batch;           /* B >= 1 (beams are batch rows)                       */
  int32_t n_heads;         /* H >= 1                                              */
  int32_t head_dim;        /* d in {64, 128, 256}                                 */
  int32_t budget_k;        /* k >= 1 : KV cache entries kept per (layer, b, head) */
  int32_t recent_w;        /* 0 <= w <= k : most recent tokens always kept        */
  int32_t max_prompt_len;  /* largest n accepted by kf_prefill_score_prune        */
  int32_t gen_len_T;       /* T >= 0 : delta_tau = (tau_end - tau_init) / T (Eq. 12); 0 = constant tau_init */
  float   tau_init;        /* > 0, paper default 1                                */
  float   tau_end;         /* > 0, paper default 2                                */
  uint64_t noise_seed;     /* Philox key                                          */
  int32_t noise_mode;      /* KF_NOISE_*                                          */
  int32_t bias_mode;       /* KF_BIAS_*                                           */
  const float* h_alibi_slopes; /* HOST [H], read during kf_create when bias_mode == KF_BIAS_ALIBI */
  float   logit_scale;     /* 0 => 1/sqrt(d) (Eq. 1 / Eq. 4)                      */
  float   noise_const;     /* c of KF_NOISE_CONST                                 */
  int32_t decode_splits;   /* 0 = choose automatically; else CTAs per unit in the decode kernel (at most 64) */
  int32_t prefill_impl;    /* KF_PREFILL_*                                        */
  float   noise_mu;        /* mean of KF_NOISE_GAUSS (the paper matches Gumbel's 0.5772)          */
  float   noise_sigma;     /* standard deviation of KF_NOISE_GAUSS (1.2825 in the paper)         */
  int32_t pos_mode;        /* KF_POS_*; KF_POS_NEW keeps one more int32 per cache slot            */
  int32_t n_kv_heads;      /* key/value heads Hkv (section 6: multi-query / grouped-query attention).  0 or H: every head
                              has its own cache, the method as printed.  Otherwise H / Hkv must be 2, 4 or 8: that many
                              consecutive query heads share one cache and one f_theta; each of them has its own logits,
                              noise (drawn with its own head index), bias slope and softmax of Eq. 11, and f_theta
                              accumulates the mean of their scores.  Caches are then per (layer, batch row, key/value
                              head): wherever a shape below says [B][H] for K, V, k_new, v_new, scores, positions or entry
                              counts read [B][Hkv]; q and out stay [B][H].                                         */
  int32_t rotary_dims;     /* R.  0: Q and K carry whatever positional rotation the model applies (the library never looks).
                              R > 0 (a power of two, 8 <= R <= d): Q and K are passed WITHOUT rotary embedding and the cache
                              keeps keys unrotated; the library applies the embedding to the first R features (interleaved
                              pairs (2i, 2i+1), angle position * rotary_base^(-2i/R)) when a logit is formed -- in the prompt
                              phase at each token's own position, in the generation phase according to pos_mode: KF_POS_ORIGINAL
                              rotates at the positions in the text, KF_POS_NEW at the places within the reduced cache (section
                              4.4.2 on rotary models).  Generation then accepts positions below max_prompt_len + max(T, 1)
                              (KF_EINVAL beyond: the table of angles ends there); not available with KF_DECODE_TENSOR.   */
  float   rotary_base;     /* > 1 when rotary_dims > 0; 10000 in the published embedding                               */
  int32_t decode_impl;     /* KF_DECODE_*                                                                              */
  int32_t debug_canaries;  /* 1: a 256-byte guard of a known pattern follows every sub-buffer of the workspace
                              (kf_workspace_bytes grows accordingly); kf_check_canaries verifies them.  0: none */
  int32_t debug_fail_first_wait; /* self-test of the error path: 1 makes every warp of the generation kernel give up
                              its first wait for a cache tile at once, as if the bounded wait had run out: the step
                              reports KF_ETIMEOUT through kf_poll_error (after waiting, with the full limit, for the
                              copies in flight) and leaves the layer's state undefined.  0 in normal use.          */
} kf_config;

/* Bytes of device workspace kf_create needs for this configuration
 * (KV cache, positions, scores, kernel scratch).  Returns 0 if the
 * configuration is invalid. */
size_t kf_workspace_bytes(const kf_config* cfg);

/* Build a context over a caller-owned device workspace of at least
 * kf_workspace_bytes(cfg) bytes, 256-byte aligned.  Clears the cache state
 * (asynchronously, on `stream`).  *out receives the context. */
int kf_create(const kf_config* cfg, void* d_workspace, size_t workspace_bytes, void* stream, kf_ctx** out);

/* Prompt phase of Algorithm 1 (t = 0, temperature tau_init; section 3.4).
 * For every (batch row, head) of `layer`: causal logits x_ij = scale * Q_i.K_j
 * (+ bias), y_ij = (x_ij + zeta_ij) / tau_init, row-wise softmax (Eq. 11), sum
 * over query rows into f_theta(j); keep the w most recent positions plus the
 * top-(k-w) of the others by f_theta (ties: lower position), and store the
 * kept K/V rows, positions and scores in ascending position order.  If
 * n_prompt <= k everything is kept.
 *   d_q, d_k, d_v : DEVICE fp16 [B][H][n_prompt][d], read only, each 16-byte aligned (KF_EINVAL otherwise,
 *                   with either scoring implementation).
 *   d_score_opt   : DEVICE fp32 [B][H][n_prompt] or NULL; receives f_theta
 *                   before pruning.
 * Must be called once per layer before that layer's first kf_decode_step. */
int kf_prefill_score_prune(kf_ctx* ctx, int32_t layer, int32_t n_prompt,
                           const void* d_q, const void* d_k, const void* d_v,
                           float* d_score_opt, void* stream);

/* Attention output of the prompt phase (Eq. 1 under the causal mask): for every (batch row, head) and query
 * position i, out_i = sum_{j <= i} softmax_j(x_ij) V_j with the plain softmax of x_ij = scale * Q_i.K_j
 * (+ bias) -- no logit adjustment and temperature 1, i.e. what the model's attention layer produces, which
 * section 3.4 leaves untouched.  Runs on the tensor cores; does not read or change the cache state.
 *   d_q, d_k, d_v : DEVICE fp16 [B][H][n_prompt][d], read only, 16-byte aligned.
 *   d_out         : DEVICE fp16 [B][H][n_prompt][d], 16-byte aligned.
 * kf_prefill_attend_score_prune is the two calls in one: attention output, then kf_prefill_score_prune. */
int kf_prefill_attend(kf_ctx* ctx, int32_t n_prompt, const void* d_q, const void* d_k, const void* d_v,
                      void* d_out, void* stream);
int kf_prefill_attend_score_prune(kf_ctx* ctx, int32_t layer, int32_t n_prompt,
                                  const void* d_q, const void* d_k, const void* d_v,
                                  void* d_out, float* d_score_opt, void* stream);

/* One generation step of Algorithm 1 (t = step >= 1; section 3.4) for every
 * (batch row, head) of `layer`.  The new token (original position
 * p = n_prompt + step - 1) joins the cached entries, so m = len + 1 logits:
 *   out   = sum_j softmax(x)_j V_j                       (Eq. 1; no noise, temperature 1)
 *   z_j   = softmax_j((x_j + zeta_j) / tau_step)          (Eq. 4, 11; tau of Eq. 12, clamped at T)
 *   f_theta(j) += z_j                                     (the new token starts from 0)
 *   if m > k: evict the entry with the smallest f_theta among those not in
 *   the w most recent (ties: the higher position leaves); the new token's
 *   row takes the freed slot.  Slot order is therefore arbitrary; the
 *   position array identifies the entries.
 *   d_q, d_knew, d_vnew : DEVICE fp16 [B][H][d], each 16-byte aligned (KF_EINVAL otherwise).
 *   d_out               : DEVICE fp16 [B][H][d], 16-byte aligned.
 *   d_score_opt         : DEVICE fp32 [B][H][k+1] or NULL; receives z for the
 *                         slots [0, len) followed by the new token at index len.
 * The steps of a layer must be consecutive: the first call after the prompt phase (or after kf_import_state with
 * last_step = s) has step 1 (s + 1), every later call the previous step plus one; anything else is KF_ESTATE and
 * enqueues nothing.  (The position of the token, hence its noise and temperature, follows from the step.)
 * A unit whose entry count in the workspace is outside 0..k (a damaged or foreign state image) is left untouched
 * and reported as KF_EBOUNDS by kf_poll_error. */
int kf_decode_step(kf_ctx* ctx, int32_t layer, int32_t step,
                   const void* d_q, const void* d_knew, const void* d_vnew,
                   void* d_out, float* d_score_opt, void* stream);

/* Same step with HOST buffers (pinned memory recommended).  The three inputs are copied to the device on an
 * internal copy stream, so that they overlap the kernel of the previous call; the step runs on `stream`; `out`
 * is copied back on a second internal stream, overlapping the next call's kernel.
 *   - h_q, h_knew, h_vnew must hold their values when the call is made (they are read without waiting for
 *     work queued earlier on `stream`) and stay unchanged until the step has run.
 *   - h_out is valid after a call with `wait` != 0 has returned (that call drains `stream` and the result
 *     copies of all earlier calls), or after kf_poll_error.  With `wait` == 0 nothing is waited for.
 * The first call creates two streams and six events (host resources; no device memory). */
int kf_decode_step_host(kf_ctx* ctx, int32_t layer, int32_t step,
                        const void* h_q, const void* h_knew, const void* h_vnew,
                        void* h_out, int32_t wait, void* stream);

/* Size in bytes of the scratch block built into the library (see kf_decode_step_static). */
#define KF_STATIC_SCRATCH_BYTES (16u << 20)

/* Arguments of kf_decode_step_static: the quantities kf_decode_step takes from its context. */
typedef struct kf_static_step {
  int32_t batch, n_heads, head_dim;   /* B, H, d in {64, 128, 256}                          */
  int32_t budget_k, recent_w;         /* k, w                                               */
  int32_t layer;                      /* layer index (part of the noise coordinates)        */
  int32_t position;                   /* p: original position of the token being generated  */
  int32_t noise_mode, bias_mode;      /* KF_NOISE_GUMBEL, KF_NOISE_NONE or KF_NOISE_CONST (the Gaussian alternative needs
                                         its mean and deviation: use a context); KF_BIAS_*  */
  int32_t reserved;                   /* must be 0 (KF_EINVAL otherwise)                    */
  double  tau;                        /* temperature of this step (Eq. 12, computed by the caller) */
  uint64_t noise_seed;
  float   logit_scale;                /* 0 => 1/sqrt(d)                                     */
  float   noise_const;
  const float* d_alibi_slopes;        /* DEVICE [H] when bias_mode == KF_BIAS_ALIBI, else NULL */
} kf_static_step;

/* (The paper has no counterpart for this call: it is a packaging variant of kf_decode_step.)
 *
 * The same generation step, for callers that have no way to obtain device memory for the
 * library's scratch: code that runs where cudaMalloc is off limits -- inside a region that is
 * being captured or replayed and must not allocate, under a framework that owns every byte of
 * the GPU through its own pool, or in a process whose memory budget is fixed up front.  Such a
 * caller keeps the cache tensors itself and passes them in; the per-launch scratch (adjusted
 * logits, split partials) lives in a block of KF_STATIC_SCRATCH_BYTES of device
 * memory that is part of the library image.  Every GPU that loads the library holds that block
 * until the process exits.  The call itself calls no cudaMalloc, cudaFree or other allocating
 * routine.
 *
 *   d_K, d_V  : DEVICE fp16 [B][H][k][d]   cache rows, updated in place (one row replaced or appended)
 *   d_pos     : DEVICE int32 [B][H][k]     original positions, updated in place
 *   d_acc     : DEVICE fp32 [B][H][k]      accumulated scores f_theta, updated in place
 *   d_len     : DEVICE int32 [B][H]        entries in use, updated in place
 *   d_q, d_knew, d_vnew, d_out, d_score_opt : as in kf_decode_step
 *   d_K, d_V, d_q, d_knew, d_vnew, d_out must be 16-byte aligned, d_pos, d_acc, d_len 4-byte aligned (KF_EINVAL
 *   otherwise).  A unit whose d_len entry is outside 0..k is skipped: nothing of it is read or written.
 *
 * Limits and rules
 *   - The step needs about 4*B*H*(k+1) + 4*B*H*splits*(d+4) bytes of scratch; if that exceeds the
 *     block the call returns KF_ENOSPC and enqueues nothing.
 *   - The first call on a device looks up the block's device address (with that device current);
 *     make that first call outside any stream capture.
 *   - All calls on a device share the one block, which keeps the previous call's contents; no
 *     part of it has to start at zero (the step's first kernel writes every word its second
 *     kernel reads), so nothing is cleared.  Two calls whose kernels overlap on the GPU (different
 *     streams, no ordering between them) would race on it: keep them on one stream or order them.
 *   - Device-side self-checks have nowhere to report to in this variant (there is no context to
 *     poll); arguments are validated on the host as far as possible. */
int kf_decode_step_static(const kf_static_step* args,
                          void* d_K, void* d_V, int32_t* d_pos, float* d_acc, int32_t* d_len,
                          const void* d_q, const void* d_knew, const void* d_vnew,
                          void* d_out, float* d_score_opt, void* stream);

/* Borrowed DEVICE pointers into the workspace for one layer:
 *   K, V fp16 [B][H][k][d]; pos int32 [B][H][k] (original positions; -1 marks a slot left empty by the prompt phase);
 *   acc fp32 [B][H][k] (f_theta); len int32 [B][H] (entries in use).  Any may be NULL. */
int kf_view_state(kf_ctx* ctx, int32_t layer, const void** d_K, const void** d_V,
                  const int32_t** d_pos, const float** d_acc, const int32_t** d_len);

/* In-place compaction of one layer's cache into position order (Algorithm 1 describes the reduced cache as a
 * subsequence of the token sequence, S_key and the recent window S_w; section 3.4).  kf_decode_step keeps each
 * unit's entries as an unordered set -- the token that leaves is overwritten by the one that arrives -- and
 * identifies them by their positions, so no call needs this one.  It exists for callers that want the layout the
 * prompt phase produces back: slot s of every (batch row, head) holds the entry with the s-th smallest position
 * (K row, V row, position, f_theta), e.g. to compare or store state images independent of the eviction history.
 * The permutation is applied in place, cycle by cycle, with no staging buffer; asynchronous on `stream`.
 * KF_ESTATE before the layer's prompt phase; KF_EINVAL when budget_k exceeds 16384 (the ranks of a unit's
 * entries are computed in shared memory). */
int kf_compact_layer(kf_ctx* ctx, int32_t layer, void* stream);

/* KF_POS_NEW only: borrowed DEVICE pointer to the places, int32 [B][H][k]; entry j of a unit holds the
 * number of entries of that unit with a smaller position.  KF_EINVAL in the other mode. */
int kf_view_place(kf_ctx* ctx, int32_t layer, const int32_t** d_place);

/* Checkpoint of one layer's cache (section 3.3: the reduced KV cache and f_theta are the whole state the
 * method carries from step to step).  kf_state_bytes gives the size of one layer's image: K, V, f_theta,
 * positions and entry counts, each block padded to 256 bytes, in that order.  kf_export_state copies the
 * image to a caller-owned DEVICE buffer and reports how far the layer has come (prompt length, last decode
 * step); kf_import_state loads an image into a context created with the same configuration and sets that
 * progress, after which kf_decode_step continues with step last_step + 1 and reproduces the original run
 * bit for bit (noise and temperature are functions of the coordinates, not of hidden state).  Both are
 * enqueued on `stream`.  KF_ESTATE if the layer has no prompt yet; KF_ENOSPC if `bytes` is too small. */
size_t kf_state_bytes(const kf_ctx* ctx);
int kf_export_state(kf_ctx* ctx, int32_t layer, void* d_dst, size_t bytes,
                    int32_t* n_prompt, int32_t* last_step, void* stream);
int kf_import_state(kf_ctx* ctx, int32_t layer, const void* d_src, size_t bytes,
                    int32_t n_prompt, int32_t last_step, void* stream);

/* Waits for `stream`, then returns and clears the device error word:
 * 0, KF_ETIMEOUT or KF_EBOUNDS. */
int kf_poll_error(kf_ctx* ctx, void* stream);

/* Debug layout only (kf_config.debug_canaries = 1): waits for `stream`, then compares the guard behind every
 * sub-buffer of the workspace with its pattern.  KF_OK if all are intact; KF_EBOUNDS if one was overwritten, with
 * *first_bad (may be NULL) = index of the sub-buffer in front of it, in layout order: K, V, scores, positions,
 * entry counts, adjusted-logit scratch, split partials, error word, slopes, prompt scores, kept indices, host
 * staging, the two row-statistics arrays, places.  KF_EINVAL for a context without guards. */
int kf_check_canaries(kf_ctx* ctx, void* stream, int32_t* first_bad);

/* Writes into buf (n bytes, always terminated) which kernels a kf_decode_step of this context launches, with their
 * template arguments, and how a layer call is cut into CTAs, e.g.
 * "decode_kernel<128,5,2,0> + decode_close_kernel<128>; units=1024 k=2048 splits=3 tiles_per_split=24 group=1".
 * Profiles are keyed by this string.  Returns the length the full text needs (as snprintf does) or KF_EINVAL. */
int kf_describe_decode(const kf_ctx* ctx, char* buf, size_t n);

/* Number of kernel launches this context has enqueued so far. */
int64_t kf_launch_count(const kf_ctx* ctx);

/* ------------------------------------------------------------------------------------------------------------------
 * Operators around the generation step that need no context.  As above: device buffers and scratch belong to the
 * caller, work is enqueued on `stream` of the current device, arguments are checked on the host before anything is
 * enqueued, and nothing is allocated.  Scratch holds nothing between calls and need not be cleared; two calls that may run at
 * the same time (other streams, other captured graphs) need scratch of their own.  Nothing that a call
 * writes, its scratch included, may share memory with another of its tensors (KF_EINVAL; a tensor with strides counts from its first
 * element to its last, so that two written tensors whose rows alternate within one buffer are refused as well; kf_prefill_attend_ragged and
 * kf_pages_read take rows that alternate within one buffer, where they come at the same strides).
 * ------------------------------------------------------------------------------------------------------------------ */

#define KF_TYPE_FP16 0
#define KF_TYPE_BF16 1
#define KF_TYPE_FP32 2

/* ---- 4-bit caches.  A slot holds the K and the V row of one entry in kf_packed_slot_bytes(d) = 5d/4 bytes:
 *   [0, d/2)      K codes, two features per byte, the even feature in the low nibble
 *   [d/2, d)      V codes
 *   [d, 9d/8)     K groups: for every 32 features two binary16 numbers, scale s and minimum m
 *   [9d/8, 5d/4)  V groups
 * A code c stands for the binary16 number s c + m (rounded once).  For a group with extremes lo and hi:
 * s = (hi - lo) / 15 rounded down to binary16, m = lo, c = rint((x - lo) * (1 / s)) in binary32, at most 15 (0 if s is 0).
 * A group that holds a NaN or an infinity reads back as NaN throughout. */
int32_t kf_packed_slot_bytes(int32_t head_dim);   /* 0 if head_dim is not 64, 128 or 256 */

/* Rows of a binary16 cache to slots, e.g. of a layer's kf_view_state after the prompt phase, and back.
 *   d_K, d_V : DEVICE fp16 [units][n][d], 16-byte aligned;  d_cache : DEVICE [units][budget_k][5d/4], 16-byte aligned, budget_k >= n,
 *              units * n * d <= 2^37
 *   d_len    : DEVICE int32 [units] or NULL.  Row j of a unit is converted if j < d_len[unit]; the other slots (rows) and
 *              those from n on are left as they were. */
int kf_pack_cache(int64_t units, int32_t n, int32_t budget_k, int32_t head_dim, const void* d_K, const void* d_V,
                  const int32_t* d_len, void* d_cache, void* stream);
int kf_unpack_cache(int64_t units, int32_t n, int32_t budget_k, int32_t head_dim, const void* d_cache, const int32_t* d_len,
                    void* d_K, void* d_V, void* stream);

/* Arguments of kf_decode_step_packed: the quantities kf_decode_step takes from its context. */
typedef struct kf_packed_step {
  int32_t batch, n_heads;             /* B, H (B H <= 65535)                                                      */
  int32_t n_kv_heads;                 /* Hkv: 0 or H, or H / Hkv in {2, 4, 8} query heads share a cache (see kf_config)   */
  int32_t head_dim;                   /* d in {64, 128, 256}                                                      */
  int32_t budget_k, recent_w;         /* k, w                                                                     */
  int32_t layer;                      /* layer index (part of the noise coordinates)                              */
  int32_t position;                   /* p: original position of the token being generated                        */
  int32_t noise_mode, bias_mode;      /* KF_NOISE_*, KF_BIAS_*                                                    */
  double  tau;                        /* temperature of this step (Eq. 12, computed by the caller)                */
  uint64_t noise_seed;
  float   logit_scale;                /* 0 => 1/sqrt(d)                                                           */
  float   noise_const;                /* c of KF_NOISE_CONST                                                      */
  float   noise_mu, noise_sigma;      /* KF_NOISE_GAUSS                                                           */
  const float* d_alibi_slopes;        /* DEVICE [H] when bias_mode == KF_BIAS_ALIBI, else ignored                 */
  int32_t debug_fail_first_wait;      /* self-test of the error path, see kf_config: 1 makes every warp give up its first wait
                                         for cache rows at once.  0 in normal use                                  */
} kf_packed_step;

/* One generation step of Algorithm 1 (as kf_decode_step, original positions, keys stored as they are to be multiplied)
 * over a caller-held cache in 4 bits.  Cached rows take part as the values their codes stand for, the new token's own row
 * as it was passed; it is quantised when it enters the cache.
 *   d_cache  : DEVICE [B][Hkv][k][5d/4]       slots, updated in place (one replaced or appended per unit)
 *   d_pos, d_acc, d_len : DEVICE int32 [B][Hkv][k], fp32 [B][Hkv][k], int32 [B][Hkv], updated in place
 *   d_q, d_out : DEVICE fp16 [B][H][d];  d_knew, d_vnew : DEVICE fp16 [B][Hkv][d]
 *   d_score_opt : DEVICE fp32 [B][Hkv][k+1] or NULL; z of the slots [0, len), the new token's at index len
 *   d_slot_opt  : DEVICE int32 [B][Hkv] or NULL; the slot the new row went to, -1 if it was not stored (w = 0 and its own
 *                 score was the smallest), KF_EBOUNDS or KF_ETIMEOUT where the step could not be taken (below)
 *   d_row_opt   : DEVICE fp16 [B][Hkv][2][d] or NULL; the new K and V row as the values their codes stand for
 *   d_scratch   : DEVICE, kf_packed_scratch_bytes(args) bytes, 256-byte aligned (KF_ENOSPC if `scratch_bytes` is less)
 * d_cache, d_q, d_knew, d_vnew, d_out must be 16-byte aligned.  A unit whose d_len entry is outside 0..k is skipped:
 * nothing of it is read or written.  The positions of a unit's entries are distinct and lie before args->position; where they are not
 * and every entry of a full unit is inside the recent window, outputs and scores are as ever, but the new row is not stored and
 * the unit's d_slot_opt entry is KF_EBOUNDS.  A unit whose rows did not arrive within the kernel's bounded wait keeps its state
 * (cache, positions, scores, count): its rows of d_out and its z are NaN, and its d_slot_opt entry is KF_ETIMEOUT.  Scores in d_acc
 * are not negative (sums of softmax values).  A group of a cached K row that is not finite makes the unit's rows of d_out NaN, and what
 * becomes of its scores is not specified; a group of a V row makes its own 32 features of them NaN and nothing else. */
size_t kf_packed_scratch_bytes(const kf_packed_step* args);   /* 0 if the arguments are invalid */
int kf_decode_step_packed(const kf_packed_step* args, void* d_cache, int32_t* d_pos, float* d_acc, int32_t* d_len,
                          const void* d_q, const void* d_knew, const void* d_vnew, void* d_out, float* d_score_opt,
                          int32_t* d_slot_opt, void* d_row_opt, void* d_scratch, size_t scratch_bytes, void* stream);

/* ---- From projection rows to what the prompt phase and the generation step take.  Per head of queries and keys:
 *   norm     (KF_NORM_RMS)  x <- x * w / sqrt(mean(x^2) + eps), w = 1 where no weight is passed
 *   rotation (R > 0)        pair i < R/2 of the first R features turned by position * base^(-2i/R); the pair is (2i, 2i+1)
 *                           with KF_ROTARY_PAIRS (the embedding of kf_config.rotary_dims) or (i, i + R/2) with KF_ROTARY_HALVES
 * and head-major rows; the values are only laid out.  Results are rounded once, to binary16 (beyond 65504: infinity). */
#define KF_NORM_NONE 0
#define KF_NORM_RMS  1
#define KF_ROTARY_PAIRS  0
#define KF_ROTARY_HALVES 1
typedef struct kf_qk_norm_args {
  int32_t batch, n_tokens;            /* B n < 2^31                                                               */
  int32_t n_heads, n_kv_heads;        /* H, Hkv >= 1                                                              */
  int32_t head_dim;                   /* d in {64, 128, 256}                                                      */
  int32_t input_type;                 /* of the rows and the weights: KF_TYPE_FP16 or KF_TYPE_BF16                */
  int64_t batch_stride, token_stride; /* of the rows, in elements, multiples of 8; token_stride >= (H + 2 Hkv) d  */
  int32_t norm_mode;                  /* KF_NORM_*                                                                */
  float   eps;                        /* >= 0                                                                     */
  int32_t rotary_dims, rotary_style;  /* R: 0 or a power of two, 8 <= R <= d; KF_ROTARY_*                         */
  float   rotary_base;                /* > 1 when R > 0                                                           */
  int32_t position0;                  /* without d_positions token t of every row stands at position0 + t         */
} kf_qk_norm_args;
/*   d_qkv : DEVICE [B][n] rows of H query, Hkv key and Hkv value heads of d features
 *   d_q_weight, d_k_weight : DEVICE [d] or NULL (only with KF_NORM_RMS);  d_positions : DEVICE int32 [B][n] or NULL
 *   d_q : DEVICE fp16 [B][H][n][d];  d_k, d_v_opt : DEVICE fp16 [B][Hkv][n][d], d_v_opt may be NULL
 * All but d_positions 16-byte aligned. */
int kf_qk_norm_rotate(const kf_qk_norm_args* args, const void* d_qkv, const void* d_q_weight, const void* d_k_weight,
                      const int32_t* d_positions, void* d_q, void* d_k, void* d_v_opt, void* stream);

/* ---- Beam search (beams are batch rows).  Of the beams x vocabulary continuations of every request the `take` best by
 *   value(b, t) = score_b + log softmax(logits_b)_t
 * best first; equal values: the lower beam, then the lower token.  Values are formed in binary64, rounded to binary32.
 *   - A logit that is NaN or +infinity counts as -infinity (a forbidden token).
 *   - A beam that d_finished_opt marks (non-zero) goes on with pad_token alone, at value score_b; its logits are not read.
 *   - A beam whose score is not finite, or whose logits are all forbidden, has value -infinity throughout.
 *   Continuations at -infinity are returned only when there are no others left, in the order above. */
typedef struct kf_beam_args {
  int32_t batch, beams;               /* beams <= 32, batch * beams <= 65535                                      */
  int32_t vocab, take;                /* take <= 64, take <= beams * vocab                                        */
  int32_t logits_type;                /* KF_TYPE_*                                                                */
  int32_t pad_token;                  /* 0 <= pad_token < vocab                                                   */
  int64_t row_stride;                 /* elements between the rows of two beams, >= vocab                         */
} kf_beam_args;
/*   d_logits : DEVICE [B * beams] rows;  d_scores : DEVICE fp32 [B][beams];  d_finished_opt : DEVICE uint8 [B][beams] or NULL
 *   d_out_scores fp32, d_out_parent, d_out_token int32 : DEVICE [B][take]
 *   d_scratch : DEVICE, kf_beam_scratch_bytes(args) bytes, 256-byte aligned */
size_t kf_beam_scratch_bytes(const kf_beam_args* args);
int kf_beam_select(const kf_beam_args* args, const void* d_logits, const float* d_scores, const uint8_t* d_finished_opt,
                   float* d_out_scores, int32_t* d_out_parent, int32_t* d_out_token, void* d_scratch, size_t scratch_bytes, void* stream);

/* State rows that follow their beam: in every buffer [outer][batch * beams][row_bytes], row (b, i) becomes what row
 * (b, d_parent[b][i]) was before the call, in place.  A parent outside 0..beams-1 leaves its row as it is.
 *   d_parent : DEVICE int32 [batch][beams].  At most 8 buffers, which may not overlap (nor interleave);
 *   any row_bytes (multiples of 16 move fastest). */
typedef struct kf_row_buffer {
  void*   d_base;
  int64_t row_bytes;
  int64_t outer_stride;               /* bytes between two outer indices (layers), >= batch * beams * row_bytes; unused when outer is 1 */
  int32_t outer;                      /* >= 1                                                                     */
} kf_row_buffer;
int kf_reorder_rows(const kf_row_buffer* buffers, int32_t n_buffers, int32_t batch, int32_t beams, const int32_t* d_parent, void* stream);

/* The same for the caches of a context (K, V, positions, scores, entry counts, places): its batch rows are
 * batch / beams requests of `beams` beams each (KF_EINVAL if beams does not divide the batch).  layer >= 0: that layer
 * (KF_ESTATE before its prompt phase); layer = -1: all layers, one launch.  d_parent lies outside the workspace (KF_EINVAL). */
int kf_reorder_beams(kf_ctx* ctx, int32_t layer, int32_t beams, const int32_t* d_parent, void* stream);

/* ---- Prompts of different lengths, one after the other without padding.  Sequence s owns the rows d_begin[s] .. d_begin[s + 1] - 1
 * of q, k, v and out; within it, in every head, as kf_prefill_attend:
 *   out_i = sum_{j <= i} softmax_j(x_ij) v_j,   x_ij = logit_scale q_i k_j (- slope_h (i - j) with KF_BIAS_ALIBI)
 * Query head h reads key/value head h / (H / Hkv).  Rows of no sequence are left as they were, and what they hold reaches no
 * output: a sequence ends where its range ends, whatever stands behind it.  Within a sequence a value row that is not finite may make any
 * earlier row of the same 128 NaN.  A prompt sees the rows of its own range only: behind tokens that are in pages already (a prefix) it does not
 * attend to those.  A sequence whose range is empty or not within 0 .. tokens has no output; ranges do not descend. */
typedef struct kf_ragged_args {
  int32_t tokens, sequences;          /* rows of q, k, v and out (<= 2^28); S (<= 2^20); (tokens / 128 + S) H < 2^31 */
  int32_t n_heads, n_kv_heads;        /* H, Hkv: Hkv divides H                                                    */
  int32_t head_dim, type;             /* d in {64, 128, 256}; KF_TYPE_FP16 or KF_TYPE_BF16, of all four           */
  int32_t bias_mode;                  /* KF_BIAS_*                                                                */
  float   logit_scale;                /* 0 => 1/sqrt(d)                                                           */
  const float* d_alibi_slopes;        /* DEVICE [H] when bias_mode == KF_BIAS_ALIBI, else ignored                 */
  int64_t q_token_stride, q_head_stride;      /* in elements, multiples of 8, at least d, below 2^38: any order of */
  int64_t k_token_stride, k_head_stride;      /* heads and tokens, e.g. the rows of a projection that holds q, k   */
  int64_t v_token_stride, v_head_stride;      /* and v, or head-major rows.  The features of a head are contiguous */
  int64_t out_token_stride, out_head_stride;  /* rows of two (token, head) pairs may not share memory             */
  int32_t debug_fail_first_wait;      /* self-test of the error path, see kf_config                                */
  int32_t debug_fail_after;           /* with it: n >= 0: n pieces of work of every CTA go right before a wait fails; -1 - n: n, then the wait */
                                      /* for the next piece fails                                                 */
} kf_ragged_args;
/*   d_q, d_out : DEVICE [tokens][H] rows of d;  d_k, d_v : DEVICE [tokens][Hkv] rows of d (strides above, 16-byte aligned)
 *   d_begin    : DEVICE int32 [S + 1]
 * Output weights are rounded to the type of v (11 or 8 bits), the output once more; sums and references are binary32.  In binary16 a weight below 2^-21
 * of its row's largest keeps fewer bits: it may be off by 2^-32 of that.  Logits are binary32 too: up to 10^6 in magnitude (with the bias) rows
 * are as exact as that allows, beyond 4 * 10^6 they may be NaN or off by more.  Rows that
 * did not arrive within the kernel's bounded wait make the output rows that need them NaN. */
int kf_prefill_attend_ragged(const kf_ragged_args* args, const void* d_q, const void* d_k, const void* d_v, const int32_t* d_begin,
                             void* d_out, void* stream);

/* ---- Caches in pages of 8 bits.  A page holds page_tokens consecutive tokens of a sequence for every key/value head:
 *   d_cache : int8 [n_pages][Hkv][2][page_tokens][d]   K codes, then V codes, 16-byte aligned
 *   d_scale : fp32 [n_pages][Hkv][2]                   a code c stands for c * scale
 *   d_table : int32 [S][table_width]                   the pages of a sequence in order, -1 where it has none
 *   d_length: int32 [S]                                tokens in use
 * kf_pages_write makes scales powers of two: the smallest 2^e with max |x| <= 127 * 2^e over the rows of a page, head and side
 * (e >= -120), c = rint(x / 2^e) (ties to even).  While a page fills its scale never shrinks; when it grows, the rows that are there already are
 * brought to it, c <- rint(c * old / new).  As a scale at least doubles then, a row written long before is off by
 * less than one step of the final scale.  A NaN or an infinity among the rows makes the scale NaN: everything of that page, head and side reads as NaN.
 * Scales of another origin may be any positive normal numbers.  The calls below have at least one row or sequence: a step without any makes none. */
typedef struct kf_page_cache {
  int32_t n_pages, page_tokens;       /* page_tokens in {16, 32, 64, 128}; n_pages * Hkv * 2 * page_tokens < 2^31 */
  int32_t n_kv_heads, head_dim;       /* Hkv; d in {64, 128, 256}                                                  */
  int32_t sequences, table_width;     /* S (<= 2^20), pages a sequence may have (table_width * page_tokens < 2^30)      */
} kf_page_cache;

/* Rows of tokens for kf_pages_write and kf_pages_read. */
typedef struct kf_page_rows {
  int32_t tokens, type;               /* rows (<= 2^28); KF_TYPE_FP16 or KF_TYPE_BF16                              */
  int64_t k_token_stride, k_head_stride;      /* in elements, multiples of 8, at least d                          */
  int64_t v_token_stride, v_head_stride;
} kf_page_rows;
/* Rows d_begin[s] .. d_begin[s + 1] - 1 of d_k and d_v become tokens d_length[s], d_length[s] + 1, ... of sequence s.
 *   d_begin : DEVICE int32 [S + 1], not descending, or NULL: one row per sequence, row s (tokens == S)
 * d_length is not changed (every layer of a model writes at the same place): the caller adds to it when all layers have written.
 * The pages that are written belong to one sequence alone.  A row whose page is missing (table entry outside 0 .. n_pages - 1, or
 * behind the table) is not written; a sequence whose d_length entry is negative is skipped. */
int kf_pages_write(const kf_page_cache* cache, const kf_page_rows* rows, const void* d_k, const void* d_v, const int32_t* d_begin,
                   const int32_t* d_length, const int32_t* d_table, void* d_cache, float* d_scale, void* stream);
/* The way back: rows d_begin[s] .. of d_k and d_v are tokens d_first[s] (NULL: 0), ... of sequence s as the numbers their codes
 * stand for, rounded once (beyond the type's
 * largest: infinity; with scales of another origin the product of code and scale is rounded to binary32 before).  Rows whose page is missing are NaN; rows of no sequence are left as they were. */
int kf_pages_read(const kf_page_cache* cache, const kf_page_rows* rows, const void* d_cache, const float* d_scale, const int32_t* d_table,
                  const int32_t* d_begin, const int32_t* d_first, void* d_k, void* d_v, void* stream);

/* One query token per sequence, the newest, over the d_length[s] tokens of its pages (its own row among them):
 *   out = sum_j softmax_j(x_j) v_j,   x_j = logit_scale q k_j (- slope_h (length - 1 - j) with KF_BIAS_ALIBI)
 * A weight times the scale of its V rows may be off by 2^-32 of the largest of them, beside binary32 roundings.
 * Logits may be of any size that binary32 holds in units of log 2 (a row of which all are -infinity, or one is NaN or +infinity, is NaN).
 * A sequence without tokens gets zeros; one whose length is negative or behind its table, or that needs a missing page, gets NaN. */
typedef struct kf_pages_attend_args {
  kf_page_cache cache;                /* S * table_width * page_tokens * H < 2^35 is always accepted              */
  int32_t n_heads, type;              /* H: Hkv divides H; of q and out: KF_TYPE_FP16 or KF_TYPE_BF16              */
  int32_t bias_mode;                  /* KF_BIAS_*                                                                */
  float   logit_scale;                /* 0 => 1/sqrt(d)                                                           */
  const float* d_alibi_slopes;        /* DEVICE [H] when bias_mode == KF_BIAS_ALIBI, else ignored                 */
  int64_t q_sequence_stride, q_head_stride;       /* in elements, multiples of 8, at least d                       */
  int64_t out_sequence_stride, out_head_stride;   /* rows of two (sequence, head) pairs may not share memory       */
  int32_t debug_fail_first_wait;      /* self-test of the error path, see kf_config                                */
  int32_t debug_fail_after;           /* with it, >= 0: every warp's waits fail once it has looked up 16 times as many tiles */
} kf_pages_attend_args;
/*   d_q, d_out : DEVICE [S][H] rows of d, 16-byte aligned
 *   d_scratch  : DEVICE, kf_pages_attend_scratch_bytes(args) bytes, 256-byte aligned (KF_ENOSPC if `scratch_bytes` is less)
 * Rows that did not arrive within the kernel's bounded wait make the outputs that need them NaN. */
size_t kf_pages_attend_scratch_bytes(const kf_pages_attend_args* args);   /* 0 if the arguments are invalid */
int kf_pages_attend(const kf_pages_attend_args* args, const void* d_q, const void* d_cache, const float* d_scale, const int32_t* d_table,
                    const int32_t* d_length, void* d_out, void* d_scratch, size_t scratch_bytes, void* stream);

/* Sequences forked, ended and grown, in place.  Sequence s goes on as a copy of what sequence p = d_parent[s] was before the call
 * (NULL: p = s): full pages are shared; of the sequences that go on from p the first keeps its page that is filled in part, the others get a
 * page of their own with a copy of its rows, in all layers.  p outside 0 .. S - 1 (-1): s has ended and is empty.  Then
 * pages are added until s has room for d_grow[s] more tokens (NULL: grow); pages behind those are given back.
 *   d_refs    : DEVICE int32 [n_pages], how many table entries name a page (plus what the caller counts: a page with
 *               references is never handed out).  Updated; a page is free when its count is 0.
 *   d_missing : DEVICE int32 [1], pages that could not be added because none was free or the table too narrow (at most 2^31 - 1)
 * Free pages are handed out lowest first, in the order of sequences and of the pages of each; where there is none the table
 * entry is -1; a copy of a page that was missing itself reads as NaN.  d_length[s] becomes the parent's length (0 for an ended one),
 * without the room added.  A length outside 0 .. table_width * page_tokens counts as 0; negative growth counts as none.  Pages filled in part belong to one sequence alone before and after. */
typedef struct kf_pages_update_args {
  kf_page_cache cache;                /* S <= 8192, S * table_width <= 2^28                                       */
  int32_t n_layers;                   /* d_cache, d_scale: [n_layers] caches one after the other; one table serves all */
  int32_t grow;                       /* without d_grow                                                           */
} kf_pages_update_args;
size_t kf_pages_update_scratch_bytes(const kf_pages_update_args* args);   /* 0 if the arguments are invalid */
int kf_pages_update(const kf_pages_update_args* args, int32_t* d_table, int32_t* d_length, int32_t* d_refs, const int32_t* d_parent,
                    const int32_t* d_grow, void* d_cache, float* d_scale, int32_t* d_missing, void* d_scratch, size_t scratch_bytes, void* stream);

/* The rows that a selection kept into new pages: row j of (s, head) in the pages of d_new_table is token d_keep[s][head][j] in those of
 * d_table, j < d_n_keep[s] (e.g. the positions that a layer's prompt phase kept).  The scale of a new page is the largest of those that
 * its rows come from, c <- rint(c * old / new).  What lies behind the last row of a page is left as it was.  The new pages are none of those
 * that the call reads.  From then on a row's place in the pages is no longer its token's place in the text: KF_BIAS_ALIBI of kf_pages_attend counts places
 * (as KF_POS_NEW does, not KF_POS_ORIGINAL), keys that were rotated keep the positions at which they were, and rows that follow are rotated by the caller at positions
 * of the text, not at d_length.  A token outside 0 .. d_length[s] - 1, or whose page is missing, makes the scales of its new page and head NaN; a new page that is
 * missing is not written. */
int kf_pages_compact(const kf_page_cache* cache, int32_t keep_width, int32_t new_table_width, const int32_t* d_table, const int32_t* d_length,
                     const int32_t* d_keep, const int32_t* d_n_keep, const int32_t* d_new_table, void* d_cache, float* d_scale, void* stream);

/* Frees host metadata.  The workspace stays with the caller. */
int kf_destroy(kf_ctx* ctx);

const char* kf_strerror(int code);

#ifdef __cplusplus
}
#endif
#endif /* KEYFORMER_B200_H */
