/*
 * libshadowkv -- ShadowKV decode hot path on one MI355X (gfx950), C ABI.
 *
 * Two main operations, both enqueue-only on caller-owned HIP streams (further down: the decode step
 * with a chunk cache of an offloaded value store, the append of generated tokens to the context, the
 * SVD line of the pre-filling algorithm, and the ArgTopK primitive on its own; rotary positions, a paged
 * cache and attention over it; the choice of a beam search, and the state that follows it):
 *
 *   shadowkv_build_landmarks  pre-filling algorithm (Alg. 1) after its SVD
 *                             line: chunk means of the post-RoPE keys,
 *                             per-chunk minimum cosine between mean and keys,
 *                             the o lowest chunks become resident outliers,
 *                             the other chunk means become landmarks.
 *   shadowkv_decode_step      decoding algorithm (Alg. 2) plus the attention
 *                             over the selected set ("Theoretical Equivalent
 *                             Bandwidth" section): landmark scores, per-head
 *                             softmax, max over the GQA group, top-k chunks;
 *                             values of those chunks gathered, their keys
 *                             rebuilt from the rank-r factors and rotated at
 *                             their true positions; softmax attention over
 *                             [outliers ; selected chunks ; recent tokens].
 *
 * Notation (paper): b batch, h_q / h_kv query / KV heads, G = h_q / h_kv,
 * d head dim, s chunked context length, c chunk size, n_ch = s / c, o outlier
 * chunks, n_c = n_ch - o landmarks, k selected chunks, w recent tokens, r rank.
 *
 * Conventions for every pointer argument:
 *   - "dev"  = device (HBM) memory, "dev|pinned" = HBM or device-readable
 *     pinned host memory.  All tensors are dense, row-major in the layout
 *     written next to them, 16-byte aligned.  bf16 = raw 16-bit patterns;
 *     where a tensor is marked bf16 below and belongs to the KV cache it is
 *     E5M2 bytes instead when params->kv_dtype says so (see shadowkv_kv).
 *   - The caller owns every buffer (workspace included) and both streams.
 *     The library allocates no device memory; it keeps two HIP events per
 *     device for the side-stream fork/join, released by shadowkv_shutdown().
 *   - Calls return after enqueuing; outputs are valid once `stream` has been
 *     synchronised.  Work put on `side_stream` is joined back into `stream`
 *     before the call returns.
 *   - Return value: SHADOWKV_OK or a negative code.  Arguments are validated
 *     on the host before anything is enqueued, so a rejected call has no
 *     effect on the GPU (and can be exercised on a machine without one).
 */
#ifndef SHADOWKV_H
#define SHADOWKV_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

#define SHADOWKV_OK 0
#define SHADOWKV_EINVAL (-1)     /* bad shape, null pointer, unsupported size */
#define SHADOWKV_EWORKSPACE (-2) /* workspace missing, misaligned or too small */
#define SHADOWKV_EHIP (-3)       /* HIP runtime / launch error (see last_error) */

#define SHADOWKV_VALUES_DEVICE 0 /* value store in HBM: attention reads it in place */
#define SHADOWKV_VALUES_HOST 1   /* pinned host store: staged by a gather kernel   */

/* flags */
#define SHADOWKV_FLAG_STAGE_VALUES 1u      /* run the chunk gather even for an HBM store            */
#define SHADOWKV_FLAG_KEEP_REBUILT_KEYS 2u /* also write RoPE(Gather(A,I) B) to the workspace (tests) */

typedef uint16_t shadowkv_bf16;
/* Element of a KV-cache tensor (A, B, landmarks, outlier / recent K,V, value store, value cache, and the keys
 * and values handed to build_landmarks / append_chunk): bf16 (2 bytes) or FP8 E5M2 (1 byte), chosen for all of
 * them at once by params->kv_dtype.  Written "kv" next to the arguments below.  The query and the attention
 * output are activations and are always bf16. */
typedef void shadowkv_kv;

#define SHADOWKV_KV_BF16 0
#define SHADOWKV_KV_FP8_E5M2 1   /* section "Precision Sensitivity": sign, 5 exponent bits (bias 15), 2 fraction bits,
                                    subnormals / infinities / NaNs as in IEEE 754 (the upper byte of a half).  Stored
                                    elements are widened exactly; the arithmetic is the bf16 mode's; what the library
                                    stores itself (landmarks, low-rank states of appended tokens) is rounded once, to
                                    nearest-even, from the fp64 value, overflow to infinity. */

typedef struct shadowkv_params {
  int32_t batch;            /* b  >= 1 */
  int32_t n_q_heads;        /* h_q, multiple of n_kv_heads, G <= 64 */
  int32_t n_kv_heads;       /* h_kv >= 1 */
  int32_t head_dim;         /* d in {64, 96, 128} */
  int32_t ctx_len;          /* s: tokens covered by A / landmarks / value store; multiple of chunk_size */
  int32_t chunk_size;       /* c in [1, 64] */
  int32_t rank;             /* r: multiple of 8, 8 <= r <= 256 */
  int32_t n_outlier_chunks; /* o >= 0, o <= 1024 */
  int32_t topk_chunks;      /* k: 1 <= k <= n_c = s/c - o */
  int32_t local_len;        /* w >= 0 resident recent tokens (the current token included) */
  int32_t value_location;   /* SHADOWKV_VALUES_DEVICE | SHADOWKV_VALUES_HOST */
  uint32_t flags;           /* SHADOWKV_FLAG_* */
  double rope_theta;        /* RoPE base; frequency i is theta^(-2i/d), i < d/2, pairs (i, i + d/2) */
  double softmax_scale;     /* 0 => 1/sqrt(d); used for landmark scores and for attention */
  const float *inv_freq;    /* optional dev [d/2]: replaces theta^(-2i/d) (scaled-RoPE models) */
  int32_t ctx_capacity;     /* cap: tokens the context arrays are laid out for; 0 => ctx_len.  Multiple of
                               chunk_size, >= ctx_len.  Room for shadowkv_append_chunk to grow the context. */
  int32_t kv_dtype;         /* SHADOWKV_KV_BF16 | SHADOWKV_KV_FP8_E5M2: storage type of every "kv" tensor */
} shadowkv_params;

/*
 * Layout with room to grow.  The arrays that have a token or a landmark axis are laid out for
 * cap = ctx_capacity tokens (nc_cap = cap/c - o landmark rows), and only the first s = ctx_len tokens
 * (n_c landmark rows) of each unit are valid:
 *   A [b, cap, r]   value_store [b, h_kv, cap, d]   landmarks [b, h_kv, nc_cap, d]
 *   landmark_chunk_ids [b, h_kv, nc_cap]
 * With ctx_capacity == 0 these are the dense shapes written next to each argument below (s for cap,
 * n_c for nc_cap).  Everything else (k_rope of the prefill, outliers, recent tokens, outputs) is dense.
 */

/*
 * Alg. 1, every line after the SVD.  Per (batch, KV head):
 *   C_j   = mean of the c post-RoPE keys of chunk j            (fp64 accumulate)
 *   m_j   = min over the chunk's tokens of cos(C_j, key), each norm clamped at 1e-8
 *   outliers = the o chunks with the smallest m_j (ties: lower chunk id)
 *   landmarks = bf16(C_j) of the other chunks in ascending chunk order.
 *
 *   k_rope              dev        [b, h_kv, s, d] bf16   post-RoPE keys
 *   v                   dev|pinned [b, h_kv, s, d] bf16   the value store (laid out for cap tokens, see above);
 *                                                          may be NULL (then v_outlier is untouched)
 *   landmarks           dev  out   [b, h_kv, n_c, d] bf16
 *   landmark_chunk_ids  dev  out   [b, h_kv, n_c] int32   true chunk id of each landmark slot, ascending
 *   outlier_chunk_ids   dev  out   [b, h_kv, o] int32     ascending chunk id
 *   k_outlier,v_outlier dev  out   [b, h_kv, o*c, d] bf16 exact copies, chunk order as outlier_chunk_ids
 *   workspace           dev        >= shadowkv_build_workspace_bytes(), 256-byte aligned
 * The fields rank, topk_chunks, local_len of params are ignored here.
 */
int shadowkv_build_landmarks(const shadowkv_params *params, const shadowkv_kv *k_rope,
                             const shadowkv_kv *v, shadowkv_kv *landmarks,
                             int32_t *landmark_chunk_ids, int32_t *outlier_chunk_ids,
                             shadowkv_kv *k_outlier, shadowkv_kv *v_outlier, void *workspace,
                             size_t workspace_bytes, void *stream);

/*
 * Alg. 2 followed by softmax attention over the selected set, for one new token per sequence.
 *
 *   q                   dev        [b, h_q, d] bf16       post-RoPE query; head g uses KV head g / G
 *   A                   dev        [b, s, r] bf16         left low-rank factor of the pre-RoPE keys (no head axis)
 *   B                   dev        [b, h_kv, r, d] bf16   right factor, per KV head
 *   landmarks, landmark_chunk_ids  as produced by shadowkv_build_landmarks
 *   k_outlier,v_outlier dev        [b, h_kv, o*c, d] bf16 (may be NULL when o == 0)
 *   k_local, v_local    dev        [b, h_kv, w, d] bf16   post-RoPE keys / values of the w most recent tokens
 *                                                          (may be NULL when w == 0)
 *   value_store         dev|pinned [b, h_kv, s, d] bf16   per params->value_location
 *   pos_offset          dev        [b] int32 or NULL      position of context token 0 (NULL => 0)
 *   out                 dev  out   [b, h_q, d] bf16
 *   out_chunk_ids       dev  out   [b, h_kv, k] int32 or NULL: the selected true chunk ids, ascending
 *   workspace           dev        >= shadowkv_decode_workspace_bytes(), 256-byte aligned
 *   stream              HIP stream all work is ordered on
 *   side_stream         NULL (recommended): a value gather, where one is needed, is done by the first
 *                       workgroups of the launch that rebuilds the keys, so the two overlap inside one
 *                       launch and the whole step is ordered on `stream` alone (it can be captured into a
 *                       HIP graph as it is).  Non-NULL and different from `stream`: the gather is a launch
 *                       of its own on that stream, forked from and joined back into `stream` with events
 *                       (the two-stream arrangement the paper describes; slower here by the cost of the
 *                       events).  Ignored when no gather is needed.
 *
 * Scores are ranked in the log domain: score(slot) = max over the group's heads of
 * (logit_g(slot) - logsumexp_g), which orders slots exactly like softmax-then-max.  The logit is
 * scale * <q_g, L_slot> in fp64 (exact bf16 products, fp64 sum); the normaliser is formed from the fp64
 * logits; the ranking is the one of the fp64 scores (the search runs on fp32 copies of the logits and
 * settles its boundary on fp64 scores formed again from q and the landmarks); ties go to the lower slot.
 */
int shadowkv_decode_step(const shadowkv_params *params, const shadowkv_bf16 *q,
                         const shadowkv_kv *A, const shadowkv_kv *B,
                         const shadowkv_kv *landmarks, const int32_t *landmark_chunk_ids,
                         const shadowkv_kv *k_outlier, const shadowkv_kv *v_outlier,
                         const shadowkv_kv *k_local, const shadowkv_kv *v_local,
                         const shadowkv_kv *value_store, const int32_t *pos_offset,
                         shadowkv_bf16 *out, int32_t *out_chunk_ids, void *workspace,
                         size_t workspace_bytes, void *stream, void *side_stream);

/*
 * shadowkv_decode_step for callers that cannot allocate device memory or hand over a workspace: code
 * under HIP graph capture, tight serving loops, harnesses that forbid hipMalloc.  Same arguments and
 * same results (bit for bit) as shadowkv_decode_step without `workspace`, `workspace_bytes` and
 * `side_stream`: the intermediates live in a scratch array inside the library's device image,
 * shadowkv_static_scratch_bytes() bytes (96 MiB) per GPU the library is loaded on, held until the process
 * ends.  A shape whose shadowkv_decode_workspace_bytes() exceeds that is rejected with SHADOWKV_EWORKSPACE
 * before anything is enqueued (all five benchmark shapes fit).  The call allocates nothing (no hipMalloc,
 * no events); its first use on a device looks up the array's address there.  Nothing in the scratch has to
 * start at zero and nothing is cleared; it keeps the last call's intermediates.  All calls on one GPU share
 * the one array: calls whose work overlaps on that GPU (different streams, or another thread) race -- order
 * them on one stream.  A value gather, where the shape needs one, runs inside the key-phase launch.
 */
int shadowkv_decode_step_static(const shadowkv_params *params, const shadowkv_bf16 *q,
                                const shadowkv_kv *A, const shadowkv_kv *B,
                                const shadowkv_kv *landmarks, const int32_t *landmark_chunk_ids,
                                const shadowkv_kv *k_outlier, const shadowkv_kv *v_outlier,
                                const shadowkv_kv *k_local, const shadowkv_kv *v_local,
                                const shadowkv_kv *value_store, const int32_t *pos_offset,
                                shadowkv_bf16 *out, int32_t *out_chunk_ids, void *stream);
size_t shadowkv_static_scratch_bytes(void);

/*
 * The same decode step with a chunk cache of the value store (section "High-throughput Decoding":
 * the chunks selected by adjacent steps repeat to a large part; an index scan finds the missing ones
 * and only those are fetched -- the (1 - alpha) term of the equivalent-bandwidth formula in section
 * "Theoretical Equivalent Bandwidth").  Meant for a store in pinned host memory; legal for HBM too.
 *
 * Arguments as shadowkv_decode_step, plus
 *   cache_slots      S: slots of one chunk each per (batch, KV head); topk_chunks <= S <= 8192
 *   value_cache      dev in/out [b, h_kv, S*c, d] bf16  shadowkv_value_cache_bytes() bytes, 16-byte aligned
 *   cache_chunk_ids  dev in/out [b, h_kv, S] int32      true chunk id held by each slot, -1 = empty
 *   cache_stamps     dev in/out [b, h_kv, S+1] int32    clock value of each slot's last use, then the
 *                                                       unit's clock (one tick per step)
 *   out_miss_count   dev out    [b, h_kv] int32 or NULL number of chunks fetched for this step
 * The three cache arrays must be what the previous cached step (same params, same store) left there,
 * or freshly reset.
 *
 * Policy (the paper names "a cache policy" without fixing one): least recently used.  A selected
 * chunk found in a slot stays there.  The selected chunks found nowhere take the slots that were not
 * hit in this step and have the oldest stamps (empty slots first; equal stamps: lower slot first);
 * among those slots, missing chunks in ascending chunk id go to slots in ascending index.  With
 * S == topk_chunks the slots hold exactly the last step's selection.  Attention reads each selected
 * chunk's values from its slot in the usual (ascending chunk id) order, so `out` and out_chunk_ids
 * are bit-identical to shadowkv_decode_step with SHADOWKV_FLAG_STAGE_VALUES.  Ownership: the caller
 * owns the buffers and keeps them between steps; the library keeps no pointer to them.
 */
int shadowkv_decode_step_cached(const shadowkv_params *params, const shadowkv_bf16 *q,
                                const shadowkv_kv *A, const shadowkv_kv *B,
                                const shadowkv_kv *landmarks, const int32_t *landmark_chunk_ids,
                                const shadowkv_kv *k_outlier, const shadowkv_kv *v_outlier,
                                const shadowkv_kv *k_local, const shadowkv_kv *v_local,
                                const shadowkv_kv *value_store, const int32_t *pos_offset,
                                int32_t cache_slots, shadowkv_kv *value_cache,
                                int32_t *cache_chunk_ids, int32_t *cache_stamps,
                                int32_t *out_miss_count, shadowkv_bf16 *out, int32_t *out_chunk_ids,
                                void *workspace, size_t workspace_bytes, void *stream,
                                void *side_stream);

/*
 * One more chunk of context from generated tokens (last paragraph of section "High-throughput
 * Decoding" and its footnote): the pre-RoPE keys K' of c tokens that have left the recent-token window
 * are stored as the low-rank states K' Psi, Psi = right singular matrix of the context keys, which here
 * is B transposed over the full key width: Psi[(h, x), rho] = B[b, h, rho, x].  The tokens become chunk
 * number s/c exactly as if the pre-filling algorithm had seen them (never an outlier: the outlier set
 * is fixed at pre-filling).
 *
 *   k_pre   dev [b, c, h_kv*d] bf16   pre-RoPE keys of the c tokens, heads side by side
 *   k_rope  dev [b, h_kv, c, d] bf16  the same keys after RoPE at their positions
 *   v       dev [b, h_kv, c, d] bf16  their values
 *   B       dev [b, h_kv, r, d] bf16
 *   in/out, laid out for ctx_capacity tokens: A (rows s .. s+c-1 written, fp64 accumulate, rounded once),
 *   landmarks (row n_c: mean of the chunk's post-RoPE keys), landmark_chunk_ids (entry n_c = s/c),
 *   value_store (dev|pinned; tokens s .. s+c-1).
 * Needs ctx_len + chunk_size <= ctx_capacity (else SHADOWKV_EINVAL).  params->ctx_len is the length
 * BEFORE the call; the caller continues with ctx_len + chunk_size.  The fields topk_chunks and local_len
 * are ignored.  A value cache (shadowkv_decode_step_cached) stays valid: existing chunks do not change.
 */
int shadowkv_append_chunk(const shadowkv_params *params, const shadowkv_kv *k_pre,
                          const shadowkv_kv *k_rope, const shadowkv_kv *v, const shadowkv_kv *B,
                          shadowkv_kv *A, shadowkv_kv *landmarks, int32_t *landmark_chunk_ids,
                          shadowkv_kv *value_store, void *stream);

/*
 * Alg. 1, first line: A, B <- SVD(K), the rank-r factors of the pre-RoPE keys of every sequence.  With
 * K = Phi Sigma Psi^T the thin SVD of the [s, D = h_kv*d] key matrix of one sequence, truncated to the r largest
 * singular values: B = Psi^T (reshaped [h_kv, r, d]: B[h, rho, x] = Psi[h*d + x, rho]) and A = K Psi = Phi Sigma
 * (the low-rank states of section "High-throughput Decoding": keys are kept as K Psi and projected back with Psi^T).
 * Singular vectors are defined up to sign; the convention here makes the component of largest magnitude of every
 * right singular vector positive (ties: lowest index).  Computed from the Gram matrix K^T K (stored as fp64; its
 * products are exact, its sums exact or fp64) by subspace iteration with `n_iter` steps on r + 32 vectors and a
 * Rayleigh-Ritz step; accurate when sigma_r and sigma_(r+33) are apart (the convergence factor per step is
 * (sigma_(r+33) / sigma_r)^2).  n_iter = 0, the default, stands for sixteen steps.  Where r + 32 < h_kv*d and the r-th
 * eigenvalue of K^T K as the fourth step sees it is at least four times the (r+32)-th, it takes thirteen, the last nine of
 * them shifted, which come as close to within D rounding units of the largest eigenvalue.
 *
 *   k_pre      dev      [b, s, h_kv*d] kv   pre-RoPE keys, heads side by side
 *   A          dev out  [b, cap, r] kv      rows 0 .. s-1 written: sums good to 2^-24 of each entry, or fp64 sums where an
 *                                           entry is too small beside its row for that; rounded once to storage
 *   B          dev out  [b, h_kv, r, d] kv
 *   psi_out    dev out  [b, r, h_kv*d] fp64 optional (NULL): the right singular vectors before rounding, as rows
 *   sigma_out  dev out  [b, r] fp64         optional (NULL): singular values, largest first
 *   workspace  dev      >= shadowkv_factorize_workspace_bytes(), 256-byte aligned
 * Needs rank <= h_kv*d.  topk_chunks, local_len, n_outlier_chunks are ignored.  Enqueues some 190 launches at rank
 * 160, most of them small (one per dependent step of the orthogonalisation and of the Jacobi sweeps).
 */
int shadowkv_factorize_keys(const shadowkv_params *params, const shadowkv_kv *k_pre, shadowkv_kv *A,
                            shadowkv_kv *B, double *psi_out, double *sigma_out, int32_t n_iter,
                            void *workspace, size_t workspace_bytes, void *stream);
size_t shadowkv_factorize_workspace_bytes(const shadowkv_params *params);

/*
 * How shadowkv_factorize_keys of this shape is laid out on the GPU, and where it leaves which way each sequence went (for
 * tests and profiling).  Writes 5 values to `plan` (host):
 *   [0] token parts of the Gram matrix; [1] tokens per part; [2] entries that a list of a part has room for (lists hold what
 *       the keys' digits leave out: one per 128 columns and quarter of a part's tokens);
 *   [3] byte offset in the workspace of an int32 per sequence, valid after the call: 0 Gram matrix and A from digits,
 *       1 both from fp64 sums, 2 the Gram matrix from digits and A from fp64 sums (A always is where h_kv*d is beyond 32768);
 *   [4] waves that share a 64 x 64 block of a part's fp64 sums (1, 2, 4 or 8).
 * Returns SHADOWKV_OK or SHADOWKV_EINVAL (bad params / plan NULL).
 */
int shadowkv_factorize_plan(const shadowkv_params *params, int64_t *plan);

/* Bytes of `value_cache` for the given shape and slot count (0 if either is invalid). */
size_t shadowkv_value_cache_bytes(const shadowkv_params *params, int32_t cache_slots);

/* Empties the cache: every slot of cache_chunk_ids -1, every stamp and the clocks 0; enqueued on `stream`. */
int shadowkv_value_cache_reset(const shadowkv_params *params, int32_t cache_slots,
                               int32_t *cache_chunk_ids, int32_t *cache_stamps, void *stream);

/*
 * ArgTopK as both algorithms of the paper use it (outlier chunks in Alg. 1, selected chunks in Alg. 2),
 * on its own: for each of `units` rows of `n` fp64 scores, the indices of the k largest values
 * (largest = sign * score, sign = +1 or -1), ties to the lower index, written in ascending index order.
 * NaN scores are not allowed.  Exact for any fp64 input (the internal search runs on a coarser monotone
 * key first and settles coarse ties on the exact values).
 *   scores    dev [units, n] fp64     out_ids  dev out [units, k] int32
 *   workspace dev, >= shadowkv_argtopk_workspace_bytes(units, n, k), 256-byte aligned
 * 1 <= k <= n, units <= 65535; SHADOWKV_EINVAL if the sizes exceed what the selection kernels hold.
 */
int shadowkv_argtopk(const double *scores, int32_t units, int32_t n, int32_t k, double sign,
                     int32_t *out_ids, void *workspace, size_t workspace_bytes, void *stream);
size_t shadowkv_argtopk_workspace_bytes(int32_t units, int32_t n, int32_t k);

/*
 * ---- The prompt's way into the cache: rotary positions, a paged KV cache, attention of new tokens over it ----
 *
 * Arrays of heads, [n_seqs, n_tokens, n_heads, d], are handed over with their strides (in elements); the d elements of
 * a head are contiguous.  Pointers, and strides of dimensions longer than one, are multiples of 16 bytes, and no stride
 * is negative.  An array that is written may not overlap itself or, unless a call says so, any other argument (it is refused where its
 * first or last head lies in the array that it is made of, or the other way round; arrays that only interleave do not overlap).
 * Ragged runs of tokens are one sequence of n_tokens = T tokens, cut by seq_starts.
 */
typedef struct shadowkv_heads {
  void *data;                                    /* dev */
  int64_t seq_stride, token_stride, head_stride; /* elements */
  int32_t n_seqs, n_tokens, n_heads;             /* n_seqs and n_tokens may be 0 */
  int32_t dtype;                                 /* SHADOWKV_KV_BF16 | SHADOWKV_KV_FP8_E5M2 */
} shadowkv_heads;

#define SHADOWKV_ROPE_HALF 0        /* pairs (i, i + rot_dim/2), as shadowkv_decode_step rotates */
#define SHADOWKV_ROPE_INTERLEAVED 1 /* pairs (2i, 2i + 1) */

/* Scaling of the frequencies w_i = theta^(-2i/rot_dim) for contexts longer than a model was trained on (f = factor): */
#define SHADOWKV_ROPE_PLAIN 0       /* w_i */
#define SHADOWKV_ROPE_LINEAR 1      /* w_i / f: positions interpolated */
#define SHADOWKV_ROPE_NTK 2         /* theta replaced by theta * f^(rot_dim / (rot_dim - 2)); needs rot_dim > 2 */
#define SHADOWKV_ROPE_BANDS 3       /* by the turns t_i = original_len w_i / 2 pi: w_i where t_i >= high, w_i / f where
                                       t_i <= low, mixed linearly in t_i between; needs low < high */
#define SHADOWKV_ROPE_YARN 4        /* by the index i: w_i up to the pair that makes `high` turns in original_len, w_i / f from
                                       the one that makes `low` (> 0), mixed linearly between (their indices rounded outwards and
                                       kept in [0, rot_dim - 1]) */

typedef struct shadowkv_rope {
  int32_t head_dim;     /* d in {64, 96, 128} */
  int32_t rot_dim;      /* leading elements of a head that are rotated, a multiple of 8; 0 => head_dim */
  int32_t layout;       /* SHADOWKV_ROPE_HALF | SHADOWKV_ROPE_INTERLEAVED */
  int32_t scaling;      /* SHADOWKV_ROPE_PLAIN ... SHADOWKV_ROPE_YARN */
  double theta;         /* > 0 (> 1 for YARN) */
  double factor;        /* f > 0; ignored for PLAIN */
  double low, high;     /* BANDS, YARN */
  int32_t original_len; /* BANDS, YARN: > 0 */
  int32_t reserved;     /* 0 */
  double magnitude;     /* cosine and sine are multiplied by it; 0 => 1, and 0.1 ln f + 1 for YARN with f > 1 */
  const float *inv_freq; /* optional dev [rot_dim/2]: replaces the frequencies; scaling must be PLAIN */
} shadowkv_rope;

/* The rot_dim/2 frequencies in radians per position, to host memory (fp64).  Rounded to fp32 on the device they are the
 * inv_freq of shadowkv_params; that rounding turns a pair by up to 2^-25 of its position in radians (0.03 at 1M tokens), so
 * what a decode step with them is to read is rotated with the same fp32 numbers as inv_freq here.  Returns SHADOWKV_OK or
 * SHADOWKV_EINVAL (also where rope->inv_freq is set). */
int shadowkv_rope_frequencies(const shadowkv_rope *rope, double *out);

/*
 * Turns every head of x to its token's position:  for a pair (x_i, x_j) with frequency w,
 *   out_i = m (x_i cos(pos w) - x_j sin(pos w)),   out_j = m (x_j cos(pos w) + x_i sin(pos w));
 * elements from rot_dim on are copied.  transposed != 0: with -pos in place of pos, which is the gradient with respect to
 * x of a gradient with respect to out, and undoes the rotation where m = 1.  Angles are formed in fp64 and reduced to one
 * turn, the rest is fp32, rounded once.
 *
 *   x          [n_seqs, n_tokens, n_heads, d]   bf16 or E5M2
 *   out        same sizes, bf16 or E5M2, any strides; may be x itself (same pointer, type and strides)
 *   positions  dev [n_seqs, n_tokens] int32 or NULL: position of every token
 *   pos_offset dev [n_seqs] int32 or NULL (only with positions == NULL): token t of sequence i is at pos_offset[i] + t
 * pre-RoPE keys [b, s, h_kv*d] turned into [b, h_kv, s, d] is one call with those strides.  At most 2^27 tokens a call.
 */
int shadowkv_rotate(const shadowkv_rope *rope, const shadowkv_heads *x, const shadowkv_heads *out,
                    const int32_t *positions, const int32_t *pos_offset, int32_t transposed, void *stream);

/*
 * A cache of keys and values in pages of page_size tokens.  Row (page, head, row) of the keys is at
 * k + page * k_page_stride + head * k_head_stride + row * k_token_stride elements, and likewise the values.  Token l of
 * sequence i lies in page page_table[i * table_stride + l / page_size], row l % page_size.  The rows of one head span
 * less than 64 GiB, and a sequence has room for 2^30 tokens at most.  An entry outside [0, n_pages)
 * holds no tokens: what is appended there is dropped, and attention leaves its tokens out.
 * A dense array [b, h_kv, cap, d] is such a cache with page_stride = page_size * d, head_stride = cap * d, pages
 * (i * h_kv * cap) / page_size + j and n_pages = ((b - 1) * h_kv + 1) * cap / page_size.
 */
typedef struct shadowkv_paged_cache {
  void *k, *v;                                          /* dev kv */
  int64_t k_page_stride, k_head_stride, k_token_stride; /* elements */
  int64_t v_page_stride, v_head_stride, v_token_stride;
  const int32_t *page_table;                            /* dev [batch, table_stride], the first pages_per_seq used */
  int64_t table_stride;
  int32_t batch, pages_per_seq, n_pages;
  int32_t n_kv_heads, head_dim;                         /* d in {64, 96, 128} */
  int32_t page_size;                                    /* a power of two, up to 65536 */
  int32_t kv_dtype;                                     /* SHADOWKV_KV_* */
  int32_t reserved;                                     /* 0 */
} shadowkv_paged_cache;

/*
 * Appends the keys and values of new tokens, rotating the keys (and the tokens' queries) on the way.  The new tokens of
 * sequence i are rows seq_starts[i] .. seq_starts[i+1] - 1 of k, v and q; the j-th of its n_i goes to place
 * l = kv_lens[i] - n_i + j of the sequence, and is rotated to position pos_offset[i] + l.  kv_lens therefore counts the new tokens,
 * as shadowkv_paged_attention wants it.  Places below 0 or beyond pages_per_seq pages are dropped, as those on entries without a
 * page; queries are turned all the same.  Rows outside every run are left as they were.
 *
 *   rope       NULL: keys are stored as they come; q and q_out must be NULL then
 *   k, v       [1, T, h_kv, d]  bf16, or the cache's type; both the same
 *   q, q_out   [1, T, h_q, d]   bf16 both, or both NULL; q_out may be q itself
 *   seq_starts dev [batch + 1] int32, ascending, held to [0, T]; NULL: T / batch tokens of every sequence (batch must divide T)
 *   kv_lens    dev [batch] int32
 *   pos_offset dev [batch] int32 or NULL (0)
 * No place may be written twice in a call.  T <= 2^27.
 */
int shadowkv_paged_append(const shadowkv_paged_cache *cache, const shadowkv_rope *rope, const shadowkv_heads *k,
                          const shadowkv_heads *v, const shadowkv_heads *q, const shadowkv_heads *q_out,
                          const int32_t *seq_starts, const int32_t *kv_lens, const int32_t *pos_offset, void *stream);

/*
 * Attention of new tokens over the paged cache, which holds them already: for token j of the n_i of sequence i and query head g,
 *   out = sum over the places l it sees of softmax_l(scale <q, k_l>) v_l   (KV head g / (h_q / h_kv)),
 * where it sees l <= kv_lens[i] - n_i + j with causal != 0, else every l < kv_lens[i]; places below 0 or beyond
 * pages_per_seq pages, which shadowkv_paged_append drops, hold nothing.  A negative kv_lens counts as 0.
 * What a token does not see (later tokens, entries without a page, rows behind the length) has no influence on it, whatever is stored there, NaN and infinities among it.  A token that sees nothing, or whose logits
 * are all minus infinity, gets out = 0 and lse = -inf.  An infinite value that a token does see makes its element infinite; NaN where
 * infinities of both signs meet, and possibly where its weight is less than 2^-90 of the largest.
 *
 *   q, out     [1, T, h_q, d] bf16, T <= 2^30; h_q / h_kv <= 64; rows outside every run are left as they were
 *   lse        dev out [T, h_q] fp32 or NULL: natural logarithm of the sum of exp(scale <q, k_l>)
 *   seq_starts, kv_lens  as shadowkv_paged_append
 *   softmax_scale  0 => 1/sqrt(d); else times log2(e) a normal positive fp32 number, 8.15e-39 ... 2.35e38
 *   workspace  dev >= shadowkv_paged_attention_workspace_bytes(), 256-byte aligned; its contents do not matter.  Two
 *              calls whose work may overlap need a workspace each.
 * Products and sums are fp32; the softmax weights are rounded to bf16 for the product with the values where a call has more than
 * 32 rows (T x h_q / h_kv, divided by batch) a sequence on average, and enter as two bf16 terms otherwise.  So a token's weights may
 * enter with 8 bits or with 16 according to what else is in its call, rows outside every run included: off by up to 2^-8 of
 * sum |weight value|, or 2^-16.
 * The same call gives the same bits, whatever else the GPU does.
 */
int shadowkv_paged_attention(const shadowkv_paged_cache *cache, const shadowkv_heads *q, const shadowkv_heads *out,
                             float *lse, const int32_t *seq_starts, const int32_t *kv_lens, int32_t causal,
                             double softmax_scale, void *workspace, size_t workspace_bytes, void *stream);
/* For n_tokens = T rows and h_q = n_q_heads (0 if the arguments are invalid; pointers are not looked at). */
size_t shadowkv_paged_attention_workspace_bytes(const shadowkv_paged_cache *cache, int32_t n_q_heads, int32_t n_tokens);

/*
 * ---- A search over several continuations: the choice over beams and vocabulary, and the state that follows it ----
 *
 * Rows are beams: group g (one prompt) has rows g * n_beams .. g * n_beams + n_beams - 1.  A step of a search chooses
 * (shadowkv_beam_select), which names for every new row the row that it continues, its parent; then the state of the rows follows
 * their parents: dense arrays in place (shadowkv_reorder_rows), sequences in pages (shadowkv_pages_update, shadowkv_pages_copy).
 */
#define SHADOWKV_LOGITS_BF16 0
#define SHADOWKV_LOGITS_FP16 1
#define SHADOWKV_LOGITS_FP32 2

typedef struct shadowkv_logits {
  const void *data;                      /* dev [n_groups, n_beams, vocab], aligned to its element */
  int64_t group_stride, beam_stride;     /* elements, >= 0; the logits of a row are contiguous */
  int32_t n_groups, n_beams, vocab;      /* n_groups >= 0, n_beams in [1, 64], vocab in [1, 2^30]; at most 2^20 rows */
  int32_t dtype;                         /* SHADOWKV_LOGITS_* */
} shadowkv_logits;

/*
 * The n_out best continuations of every group.  Row r offers every token v with a logit x_v above minus infinity:
 *   score = scores[r] + c x_v - log sum_w exp(c x_w)   (c = logit_scale, the inverse of a temperature),
 *   rank  = score / (lengths[r] + 1)^length_penalty,
 * a finished row only itself: score = scores[r], rank = score / lengths[r]^length_penalty.  What a group chooses comes in descending
 * order of rank; where ranks are equal the lower row goes first, and in a row the higher logit, then the lower token.
 * A row offers nothing where its score is not finite, or (unless it is finished) where a logit is NaN or plus infinity or all are
 * minus infinity.  Places that are left over get score -inf, parent -1, token -1, finished 0, length 0.
 *
 *   scores       dev [n_groups, n_beams] fp32: summed log-probabilities of the rows; -inf for rows that do not exist (all but one of a
 *                group in the first step)
 *   finished     dev [n_groups, n_beams] bytes, not 0: the row has ended; or NULL
 *   lengths      dev [n_groups, n_beams] int32, tokens of a row (a rank divides by a length of at least 1); may be NULL with
 *                length_penalty == 0
 *   length_penalty in [-16, 16]; logit_scale 0 => 1, else positive and a normal number in fp32
 *   end_token    in [-1, vocab): a row that takes it is finished; also the token that a finished row reports
 *   n_out        in [1, 64]
 *   out_scores   dev [n_groups, n_out] fp32, out_parents (rows 0 .. n_groups * n_beams - 1) and out_tokens int32;
 *   out_finished (bytes, 0 or 1) and out_lengths (int32; those of the parent, + 1 unless it had finished; needs lengths) may be NULL.  With
 *                n_out == n_beams they may be scores, finished and lengths themselves; no other arguments may share memory.
 *   workspace    dev >= shadowkv_beam_select_workspace_bytes(), 256-byte aligned; its contents do not matter.  Two calls whose work
 *                may overlap need a workspace each.
 * Sums, logarithms and ranks are fp64, the sum of exponentials right to 2^-39 (so that scores of different rows nearer than 2^-37 are
 * not told apart, unless the rows have the same logits); scores are rounded once.  The same call gives the same bits, and rows of equal
 * logits equal sums, whatever their addresses are; a row's sum may differ in its last bits with how many rows a call has.
 */
int shadowkv_beam_select(const shadowkv_logits *logits, const float *scores, const uint8_t *finished, const int32_t *lengths,
                         double length_penalty, double logit_scale, int32_t end_token, int32_t n_out, float *out_scores,
                         int32_t *out_parents, int32_t *out_tokens, uint8_t *out_finished, int32_t *out_lengths,
                         void *workspace, size_t workspace_bytes, void *stream);
/* (0 if the sizes are invalid; pointers are not looked at) */
size_t shadowkv_beam_select_workspace_bytes(const shadowkv_logits *logits, int32_t n_out);

/* Rows of a dense state array: row i is n_outer pieces of `inner` bytes, at data + i * row_stride + j * outer_stride. */
typedef struct shadowkv_rows {
  void *data;                        /* dev */
  int64_t row_stride, outer_stride;  /* bytes, >= 0 */
  int64_t inner;                     /* bytes, >= 0 */
  int32_t n_outer;                   /* >= 0 */
  int32_t reserved;                  /* 0 */
} shadowkv_rows;

/*
 * Replaces row i of every array by what row parents[i] was before the call, in place, in one launch for up to 64 arrays.  Rows with
 * a parent outside [0, n_rows), and those that are their own parent, are left as they are (and not read).
 *   arrays  host [n_arrays], n_arrays in [0, 4096]; an array may not overlap itself, another one of the call, or parents (it is refused
 *           where its first or last piece lies in the other; arrays that only interleave do not overlap)
 *   parents dev [n_rows] int32, n_rows in [0, 2048]
 * Pieces are moved 16 bytes at a time where the address, the strides and `inner` of an array are multiples of 16, else 4 or 1.
 */
int shadowkv_reorder_rows(const shadowkv_rows *arrays, int32_t n_arrays, const int32_t *parents, int32_t n_rows, void *stream);

/*
 * Who holds which page.  Sequence i of `batch` holds the first ceil(kv_lens[i] / page_size) entries of its row of the page table;
 * page_refs[p] is the number of entries that hold page p, plus whatever the caller adds for holders of its own (a prefix kept
 * for later); a page is free where it is 0.  Entries outside [0, n_pages) are no pages, and those behind a row's pages are written
 * as -1.  The table is shared by the caches of all layers (shadowkv_paged_cache.page_table); an empty pool has kv_lens 0, page_refs 0.
 */
typedef struct shadowkv_page_pool {
  int32_t *page_table;                             /* dev [batch, table_stride], the first pages_per_seq used */
  int64_t table_stride;
  int32_t *kv_lens;                                /* dev [batch], in [0, pages_per_seq * page_size] */
  int32_t *page_refs;                              /* dev [n_pages] */
  int32_t batch, pages_per_seq, n_pages;           /* batch in [1, 4096]; n_pages <= 2^28 */
  int32_t page_size;                               /* a power of two, up to 65536 */
} shadowkv_page_pool;

/* Pages to be copied: move i takes the first rows[i] tokens (all with rows == NULL) of every head of page src[i] to page dst[i]. */
typedef struct shadowkv_page_moves {
  int32_t *src, *dst, *rows;                       /* dev [capacity] */
  int32_t *count;                                  /* dev, moves that there are; NULL: capacity */
  int32_t capacity;
  int32_t reserved;                                /* 0 */
} shadowkv_page_moves;

/*
 * Makes every sequence a continuation of another one, and room for its new tokens: row i becomes the first
 *   kept_i = min(kv_lens[parents[i]], keep_lens[i])  tokens of what row parents[i] was before the call,
 * and then, where that is granted, n_i further tokens that shadowkv_paged_append may write (kv_lens[i] = kept_i + n_i counts them,
 * as it wants it).  Forking is two rows with one parent; a row whose parent lies outside [0, batch) is emptied (kept_i = 0);
 * drafted tokens are taken back with keep_lens.
 * Pages are shared and page_refs follow.  Where n_i > 0 and kept_i is no multiple of page_size the row's last page will be written:
 * rows in ascending order, a row takes a copy of it unless it is the only holder left, so that the last of them keeps the page.  New
 * pages and copies are the lowest free pages (after the pages that this call frees), in order of row and place.
 * Granted are rows in ascending order until one needs more pages than are left: from there on, rows that need a page, or whose
 * last page another one held, keep kept_i tokens and nothing more.  Rows with kept_i + n_i > pages_per_seq * page_size too, wherever they are.  A last page
 * that is outside [0, n_pages) is not copied or replaced.
 *
 *   parents    dev [batch] int32 or NULL (every row itself);  keep_lens dev [batch] int32 or NULL (all; below 0 counts as 0)
 *   n_new      dev [batch] int32 (below 0 counts as 0) or NULL: n_new_all (>= 0) of every row
 *   moves      out: the copies to be made (rows: tokens that the page holds), before anything is appended; capacity >= batch, no
 *              member NULL
 *   workspace  dev >= shadowkv_pages_workspace_bytes(), 256-byte aligned, contents do not matter, one for each call that may overlap
 * parents, keep_lens and n_new may not share memory with what is written, nor the pool, moves and the workspace with each other.
 */
int shadowkv_pages_update(const shadowkv_page_pool *pool, const int32_t *parents, const int32_t *keep_lens, const int32_t *n_new,
                          int32_t n_new_all, const shadowkv_page_moves *moves, void *workspace, size_t workspace_bytes, void *stream);

/*
 * Moves pages in use down into free ones: the i-th free page from below takes what the i-th used page from above holds, as long
 * as that lies above it and i < min(max_moves, moves->capacity).  page_refs follow, and the entries of the page table; other places where
 * the caller holds page numbers are the caller's (moves->src, moves->dst).  Afterwards every page from *n_used on is free.
 *   moves      out: the pages to be copied, in every layer; rows may be NULL (else page_size is written), the other members may not
 *   n_used     dev out int32, or NULL
 */
int shadowkv_pages_compact(const shadowkv_page_pool *pool, int32_t max_moves, const shadowkv_page_moves *moves, int32_t *n_used,
                           void *workspace, size_t workspace_bytes, void *stream);
/* For shadowkv_pages_update and shadowkv_pages_compact (0 if the sizes are invalid; pointers are not looked at). */
size_t shadowkv_pages_workspace_bytes(const shadowkv_page_pool *pool);

/*
 * Copies pages, keys and values, from cache to cache: from[l] to to[l] for every l < n_layers (to may be from: copies
 * inside a cache).  from[l] and to[l] agree in n_kv_heads, head_dim, page_size and kv_dtype, and may differ in n_pages and strides; their page
 * tables are not looked at and may be NULL.  Moves whose pages lie outside them are left out; rows[i] is held to [0, page_size].
 * In a call no page may be written twice, or be read and written, and the pages of the layers may not overlap; a device cannot
 * refuse that: such pages hold either contents, or parts of both.
 *   from, to   host arrays of n_layers pointers;  n_layers in [0, 4096]
 */
int shadowkv_pages_copy(const shadowkv_paged_cache *const *from, const shadowkv_paged_cache *const *to, int32_t n_layers,
                        const shadowkv_page_moves *moves, void *stream);

/* Workspace sizes in bytes for the given shape (0 if params are invalid). */
size_t shadowkv_build_workspace_bytes(const shadowkv_params *params);
size_t shadowkv_decode_workspace_bytes(const shadowkv_params *params);

/* Host-only check of a parameter block: SHADOWKV_OK or SHADOWKV_EINVAL (reason via last_error). */
int shadowkv_validate_params(const shadowkv_params *params, int for_decode);

/*
 * Intermediates of the last decode step inside `workspace` (for tests and profiling).
 * which: 0 = rebuilt rotated keys RoPE(Gather(A, I) B), fp32 [b, h_kv, k*c, d], rows in out_chunk_ids order
 *            (only with SHADOWKV_FLAG_KEEP_REBUILT_KEYS; the keys normally live in registers only);
 *        1 = staged values Gather(V_store, I), bf16 [b, h_kv, k*c, d] (NULL when the gather did not run);
 *        2 = selected true chunk ids, int32 [b, h_kv, k];
 *        3 = scaled landmark logits P / sqrt(d) as stored for the search, fp32 [b, h_q, ld], ld = n_c rounded up
 *            to a multiple of 4 (the first n_c of a row are valid);
 *        4 = slots filled by the last cached step, int32 [b, h_kv, k] (first out_miss_count entries per unit);
 *        5 = slot of every selected chunk after the last cached step, int32 [b, h_kv, k].
 * Returns a pointer into `workspace`, or NULL.
 */
void *shadowkv_decode_workspace_view(const shadowkv_params *params, void *workspace, int which);

/*
 * How a plain shadowkv_decode_step (no value cache) of this shape is laid out on the GPU (measurement aid: lets
 * a benchmark say which launch the bytes of a stage belong to).  Writes 8 values to `plan` (host):
 *   [0] splits of the selected rows per (sequence, KV head); [1] rows per split;
 *   [2] 1 if the rows resident in HBM (outliers, recent tokens) are attended over by extra workgroups of the
 *       selection launch, 0 if by the attention launch;
 *   [3] 1 if the attention launch is the kernel with key waves and value waves, 0 the single-role kernel;
 *   [4] threads and [5] candidates per thread of the selection's first launch; [6] its launches (1 or 2, 3 with
 *       a middle level); [7] floats per row of the stored logits.
 * Returns SHADOWKV_OK or SHADOWKV_EINVAL (bad params / plan NULL).
 */
int shadowkv_decode_plan(const shadowkv_params *params, int32_t *plan);

/* Landmark rows per scoring workgroup of a decode step of this shape: 64, 128 or 256 (0 if params are invalid). */
int shadowkv_decode_score_rows(const shadowkv_params *params);

/*
 * Per-stage timing of decode steps with HIP events recorded on the caller's stream at the
 * stage boundaries (measurement aid, not part of the method).  Between begin and end every
 * decode step (up to max_steps) records 5 events; end synchronises, writes the summed
 * milliseconds of the 4 stages -- landmark scoring | selection | staged value gather (zero when
 * values are read in place) | attention with key rebuild -- to stage_ms[4] and the number of recorded steps to n_steps.
 */
int shadowkv_profile_begin(int max_steps);
int shadowkv_profile_end(double *stage_ms, int *n_steps);

const char *shadowkv_status_string(int status); /* static string for a return code            */
const char *shadowkv_last_error(void);          /* thread-local detail of the last failure     */
int shadowkv_version(void);                     /* major*10000 + minor*100 + patch             */
void shadowkv_shutdown(void);                   /* destroy cached events; safe to call twice   */

#ifdef __cplusplus
}
#endif
#endif /* SHADOWKV_H */
