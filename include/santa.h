/*
 * santa.h -- C ABI of libsanta: one decode step of SANTA / S2ANTA attention on
 * an AMD Instinct MI355X (gfx950).
 *
 * Method: "Stochastic Sparse Attention for Memory-Bound Inference" (arXiv
 * 2605.01910).  A decode step computes, for every query row (batch b, query
 * head h) with context length L = ctx_len[b] and KV head k = h / (Hq / Hkv):
 *
 *   scores   s_j = scale * <q_h, K_{b,j,k}>,  j < L             (Sec. 2, SDPA equation)
 *   softmax  p = softmax(s)                                      (Sec. 2, SDPA equation)
 *   dense    out = sum_j p_j V_{b,j,k}                           (Sec. 2, SDPA equation)
 *   sampled  out = (1/S) sum_m V_{b,J_m,k},  J_m = F^{-1}(T_m)   (Sec. 2, Eq. "stochastic-add-only-attn";
 *            F = CDF of p; T_m systematic or stratified          Sec. 2.1, "Construction")
 *
 * Conventions shared by every entry point
 * ---------------------------------------
 * - Every pointer argument except `stream` and the structs (`shape`, `kv`, `kt`,
 *   `chunk`, `window`, `rows`, `rope`, `params`) is a DEVICE pointer owned by the
 *   caller, and so are the pointers inside the structs.  The library never allocates, frees
 *   or synchronises; all kernels are enqueued on `stream` (a hipStream_t,
 *   NULL = the null stream) and the call returns before they finish.
 * - Element type: `shape->dtype` (SANTA_BF16 or SANTA_F32) is the type of q, K,
 *   V and out.  Accumulation is float32.
 * - q is [batch, num_q_heads, head_dim] contiguous; out is the same shape and
 *   type; idx_out (optional, NULL to skip) is int32 [batch, num_q_heads, S].
 * - head_dim must be 128; num_q_heads / num_kv_heads must be 1, 2, 4 or 8.
 * - Errors: arguments are validated on the host before any launch; on error
 *   nothing is enqueued and a status code is returned (santa_last_error() gives
 *   a message).  A launch failure returns SANTA_ERR_HIP.  No C++ exception
 *   crosses this interface.
 * - Not checked on the device (preconditions): u values in [0, 1),
 *   0 <= ctx_len[b] <= n_k, block-table entries naming valid pages.  A row with
 *   ctx_len 0 yields a zero output and idx -1.
 * - Workspace: `ws` must be at least santa_workspace_size(...) bytes, 256-byte
 *   aligned, and initialised once by santa_workspace_init() (or zero-filled)
 *   before its first use.  Every call leaves it ready for the next call, of
 *   any kind and shape, provided the workspace is large enough for that call.
 *   Calls that share one workspace must be ordered (same stream or
 *   synchronised).
 * - Bounded waits: the single-launch paths wait on other workgroups of the
 *   same launch with a spin limit.  A wait that gives up sets the int32 at
 *   byte 0 of the workspace to nonzero; that call's outputs are then not
 *   valid and the workspace needs santa_workspace_init() again.  The library
 *   never reads the flag back (it does not synchronise); callers may.
 * - Per-thread state: the last error message, a pending call timer
 *   (santa_time_next_call) and the launch options (santa_set_options).
 *   Nothing else persists between calls outside the caller's workspace.
 */
#ifndef SANTA_H
#define SANTA_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
  SANTA_OK = 0,
  SANTA_ERR_INVALID_ARG = 1, /* null pointer, bad size, inconsistent shape   */
  SANTA_ERR_UNSUPPORTED = 2, /* valid but not implemented (head_dim, G, ...) */
  SANTA_ERR_WORKSPACE = 3,   /* workspace missing, too small or misaligned   */
  SANTA_ERR_HIP = 4          /* a HIP runtime call or kernel launch failed    */
} santa_status_t;

typedef enum { SANTA_BF16 = 0, SANTA_F32 = 1 } santa_dtype_t;

typedef enum {
  SANTA_KIND_DENSE = 0,
  SANTA_KIND_SYSTEMATIC = 1,
  SANTA_KIND_STRATIFIED = 2,
  SANTA_KIND_BERNOULLI = 3,
  SANTA_KIND_FLASH = 4,
  SANTA_KIND_IID = 5
} santa_kind_t;

/* Problem shape.  dtype is a santa_dtype_t. */
typedef struct {
  int32_t batch;
  int32_t num_q_heads;
  int32_t num_kv_heads;
  int32_t head_dim;
  int32_t dtype;
} santa_shape_t;

/* KV cache descriptor (device pointers, caller-owned).  The feature dimension
 * is always contiguous (stride 1); strides are in ELEMENTS and must keep every
 * 128-feature row 16-byte aligned.
 *
 * Contiguous cache (block_table == NULL): element (b, j, k, i) of K or V is at
 *   base + b*stride_b + j*stride_n + k*stride_h + i,
 * so the sequence-major layout [B, n, Hkv, d] of the paper's microbenchmark and
 * the head-major layout [B, Hkv, n, d] are both expressible.
 *
 * Paged cache (block_table != NULL, int32 [batch, max_pages]): token j of
 * sequence b lives in page P = block_table[b*max_pages + j/page_size]; its
 * element (k, i) is at
 *   base + P*stride_b + (j % page_size)*stride_n + k*stride_h + i,
 * e.g. stride_b = Hkv*page_size*d, stride_h = page_size*d, stride_n = d for a
 * [pages, Hkv, page_size, d] pool.  page_size must be a power of two.
 *
 * ctx_len: int32 [batch] per-sequence lengths, or NULL for "every sequence has
 * n_k keys".  n_k (host value) is the maximum length; it sizes the launch. */
typedef struct {
  const void *k;
  const void *v;
  int64_t stride_b, stride_n, stride_h;
  const int32_t *ctx_len;
  const int32_t *block_table;
  int32_t page_size;
  int32_t max_pages;
  int32_t n_k;
  /* Fused current-token append (nullable, both or neither; 16-byte aligned,
   * [batch, num_kv_heads, head_dim] in the cache's dtype).  A decode step
   * first stores the new token's key and value in the cache, then attends
   * over it; FlashAttention-2's decode call fuses that store, the paper's
   * kernels take a cache that already holds the token (App. Decode-Step
   * Kernel Microbenchmark Details, note on KV-cache appends).  When set, the
   * call writes k_new / v_new into row ctx_len[b] - 1 (n_k - 1 without
   * ctx_len) of every (b, kv head), through the block table for paged
   * caches, inside the attention launch, and attends over the cache with
   * those rows: the cache memory must be writable and ctx_len[b] >= 1.
   * Supported by the dense, flash and sampled calls on their fused paths;
   * the Bernoulli call and the multi-kernel path return
   * SANTA_ERR_UNSUPPORTED. */
  const void *k_new;
  const void *v_new;
  /* Element type of K and V (a santa_kv_dtype_t).  SANTA_KV_AS_Q (0, the
   * default): shape->dtype.  SANTA_KV_FP8_E4M3 (1): one byte per element, an
   * OCP FP8 E4M3 code (1 sign bit, 4 exponent bits with bias 7, 3 mantissa
   * bits; exponent field 0 encodes the subnormals m/8 * 2^-6; S.1111.111 is
   * NaN; no infinities), scaled per (batch, KV head): element (b, j, k, i) of
   * K is k_scale[b*num_kv_heads + k] * e4m3(code), and likewise for V with
   * v_scale (device float32 arrays [batch, num_kv_heads]).  Quantising the
   * cache is complementary to SANTA (Sec. 1; Related Work on KV-cache
   * compression): keys and values are read at one byte each.  Needs
   * shape->dtype == SANTA_BF16 (q and out stay bfloat16); strides are in
   * elements (= bytes) and must keep rows 16-byte aligned.  Supported by the
   * dense, flash, systematic, stratified and i.i.d. calls on their fused
   * paths; the Bernoulli call, the multi-kernel path and the fused append
   * return SANTA_ERR_UNSUPPORTED. */
  int32_t kv_dtype;
  const float *k_scale;
  const float *v_scale;
} santa_kv_t;

typedef enum { SANTA_KV_AS_Q = 0, SANTA_KV_FP8_E4M3 = 1 } santa_kv_dtype_t;

/* Feature-major key cache for the Bernoulli score stage: element (b, k, i, j)
 * (feature i of key j) at k_t + b*stride_b + k*stride_h + i*stride_d + j; keys
 * are contiguous so that skipping a feature skips a contiguous row of K^T
 * (Sec. 5: features whose query sample is zero need not be read). */
typedef struct {
  const void *k_t;
  int64_t stride_b, stride_h, stride_d;
} santa_kt_t;

/* Bytes of workspace the given call needs (kind: santa_kind_t; S ignored for
 * SANTA_KIND_DENSE and SANTA_KIND_FLASH).  Returns 0 if the arguments are invalid. */
size_t santa_workspace_size(const santa_shape_t *shape, const santa_kv_t *kv, int32_t S,
                            int32_t kind);

/* Prepare a workspace for first use (zero-fills it on `stream`). */
santa_status_t santa_workspace_init(void *ws, size_t ws_bytes, void *stream);

/* Exact decode attention (Sec. 2, SDPA equation): out = softmax(scale q K^T) V,
 * computed split-K with a max/sum-exp merge.  The like-for-like dense baseline
 * of the sampled entry points below. */
santa_status_t santa_decode_dense(const void *q, const santa_kv_t *kv, const santa_shape_t *shape,
                                  float scale, void *out, void *ws, size_t ws_bytes,
                                  void *stream);

/* S2ANTA-sys (Sec. 2.1, "Construction", systematic): one uniform u per row
 * (u: float32 [batch, num_q_heads], in [0,1)); thresholds T_m = (m + u)/S for
 * m = 0..S-1; J_m = F^{-1}(T_m) is the key whose CDF interval [F(j-1), F(j))
 * contains T_m (App. A, "Unbiasedness of S2ANTA"); out = (1/S) sum_m V_{J_m}.
 * Samples are assigned to KV splits by the exact global CDF, so the estimator
 * is the paper's systematic one for any split size.  1 <= S <= 2^24. */
santa_status_t santa_decode_systematic(const void *q, const santa_kv_t *kv,
                                       const santa_shape_t *shape, float scale, int32_t S,
                                       const float *u, int32_t *idx_out, void *out, void *ws,
                                       size_t ws_bytes, void *stream);

/* S2ANTA-strat (Sec. 2.1, "Construction", independent stratified): S uniforms
 * per row (u: float32 [batch, num_q_heads, S]); T_m = (m + u_m)/S lies in
 * stratum [m/S, (m+1)/S); otherwise as santa_decode_systematic. */
santa_status_t santa_decode_stratified(const void *q, const santa_kv_t *kv,
                                       const santa_shape_t *shape, float scale, int32_t S,
                                       const float *u, int32_t *idx_out, void *out, void *ws,
                                       size_t ws_bytes, void *stream);

/* SANTA with i.i.d. draws (Sec. 2, Eq. "stochastic-add-only-attn": S indices
 * drawn independently from the attention distribution, with replacement).
 * The draws are the inverse CDF (as above) of S sorted independent uniforms,
 * built without a sort from S + 1 uniforms per row (u: float32 [batch,
 * num_q_heads, S + 1], in [0,1)): E_i = -ln(1 - u_i), T_m = C_m / C_S with
 * C_m = sum_{i<=m} E_i (the normalised partial sums of S + 1 unit
 * exponentials are the order statistics of S uniforms); out = (1/S)
 * sum_m V_{J_m}.  Requires G*(2S + 1) <= 4096 (G = num_q_heads /
 * num_kv_heads; S <= 511 at G = 4); workspace as SANTA_KIND_IID.  Needs the
 * fused launch layout: returns SANTA_ERR_UNSUPPORTED under SANTA_PATH_MULTI
 * and when batch * num_kv_heads exceeds 4096. */
santa_status_t santa_decode_iid(const void *q, const santa_kv_t *kv, const santa_shape_t *shape,
                                float scale, int32_t S, const float *u, int32_t *idx_out,
                                void *out, void *ws, size_t ws_bytes, void *stream);

/* No-allocation form of santa_decode_stratified, for callers that cannot
 * allocate device memory at call time: code under HIP graph capture, serving
 * loops and harnesses that forbid it.  Same arguments, computation and
 * outputs as santa_decode_stratified, without the workspace: the call uses a
 * scratch array of SANTA_STATIC_SCRATCH_BYTES (64 MiB) in the library's own
 * device memory, one per GPU, placed when the library's code is loaded on that
 * GPU and held until the process ends.  The first call on a device looks up
 * the array's address there.  Every call first clears the part of the array
 * that must start at zero (a fill kernel on `stream`), so it does not depend
 * on what earlier calls left; calls on one GPU share the array, so calls that
 * overlap in time on one GPU (on different streams, or from different
 * threads without ordering) race and give invalid outputs.  `stream` must
 * belong to the calling thread's current device.  Errors: as
 * santa_decode_stratified; SANTA_ERR_WORKSPACE when the call needs more than
 * SANTA_STATIC_SCRATCH_BYTES of workspace (santa_workspace_size with
 * SANTA_KIND_STRATIFIED gives the need); SANTA_ERR_UNSUPPORTED under
 * SANTA_PATH_MULTI.  It never calls hipMalloc or hipFree. */
#define SANTA_STATIC_SCRATCH_BYTES (64u << 20)
santa_status_t santa_decode_stratified_noalloc(const void *q, const santa_kv_t *kv,
                                               const santa_shape_t *shape, float scale, int32_t S,
                                               const float *u, int32_t *idx_out, void *out,
                                               void *stream);

/* Bernoulli qK^T score sampling (Sec. 5, Eq. "qk_estimator"; App. C) followed
 * by the systematic value stage.
 *   mode 0, per-head ternary query: norm = max_i |q_i|, pi_i = |q_i|/norm,
 *           w_i = (norm/B) * sign(q_i) * c_i;
 *   mode 1, mean group query (Sec. 5, Eq. "mean_group_query"; App. C, GQA):
 *           m_i = mean over the group of |q_{g,i}|, norm = max_i m_i,
 *           pi_i = m_i/norm, w_{g,i} = (norm/B) c_i q_{g,i} / m_i (0 if m_i = 0);
 *   with B = B_draws and the stratified count c_i = #{n < B : (n + u_i)/B < pi_i}
 *   (for B = 1 this is one Bernoulli(pi_i) draw).  The decision is taken in
 *   float32.  Scores s_j = scale * <w, k_j> read only the features in the
 *   union over the GQA group of nonzero weights, from the feature-major cache kt.
 * u_q: float32 [batch, num_q_heads, head_dim] (mode 0) or
 *      [batch, num_kv_heads, head_dim] (mode 1).
 * kv:  supplies V (kv->k is ignored), ctx_len and n_k; contiguous only.
 * u:   systematic uniforms [batch, num_q_heads].
 * feat_mask_out: optional uint8 [batch, num_kv_heads, head_dim], 1 where the
 *      feature row of K^T was read.  1 <= B_draws <= 64. */
santa_status_t santa_decode_bernoulli_qk(const void *q, const santa_kt_t *kt,
                                         const santa_kv_t *kv, const santa_shape_t *shape,
                                         float scale, int32_t B_draws, int32_t mode,
                                         const float *u_q, int32_t S, const float *u,
                                         int32_t *idx_out, uint8_t *feat_mask_out, void *out,
                                         void *ws, size_t ws_bytes, void *stream);

/* S2ANTA-flash (Sec. 3.3, "Speculative Sampling with Deferred Normalization";
 * App. "S2ANTA-Flash Pseudocode", Kernels 1 and 2).  Each row's keys are cut
 * into tiles of `tile` keys (tile t = [t*tile, min((t+1)*tile, L))); every
 * tile draws S_tile samples by systematic sampling on its own distribution
 * e_j / l_t, e_j = exp(s_j - m_t), m_t = max_t s, l_t = sum e_j (thresholds
 * (i + a)/S_tile with the tile's uniform a, inverse CDF as above, clamped to
 * the tile), giving the tile estimate O_t = (1/S_tile) sum_i V_{J_{t,i}}; the
 * tiles are merged by their softmax mass: out = sum_t W_t O_t / sum_t W_t,
 * W_t = exp(m_t - max_t m_t) l_t.  The paper's budget is S_tile ~ S/T for a
 * total of S draws over T tiles; the caller passes S_tile.
 * tile:    keys per tile, a power of two in [16, 1024].
 * S_tile:  draws per tile and query head, 1 <= S_tile <= 4096.
 * u:       float32 [batch, num_q_heads, T_max], T_max = ceil(n_k / tile): the
 *          uniform in [0,1) of each (row, tile).
 * idx_out: optional int32 [batch, num_q_heads, T_max, S_tile]: the drawn keys
 *          (logical positions) tile by tile, -1 for tiles at or past the row's
 *          length.
 * The workspace is sized by santa_workspace_size(..., SANTA_KIND_FLASH) (the
 * dense step's workspace).  Contiguous and paged caches.  Needs the fused
 * launch layout: returns SANTA_ERR_UNSUPPORTED under SANTA_PATH_MULTI and
 * when batch * num_kv_heads exceeds 4096. */
santa_status_t santa_decode_flash(const void *q, const santa_kv_t *kv, const santa_shape_t *shape,
                                  float scale, int32_t tile, int32_t S_tile, const float *u,
                                  int32_t *idx_out, void *out, void *ws, size_t ws_bytes,
                                  void *stream);

/* ---------------------------------------------------------------------------
 * New tokens: rotary positions, cache store, attention of a chunk
 * ---------------------------------------------------------------------------
 * The decode calls attend over a cache that holds the current token.  The calls
 * below bring tokens into that cache and attend with them: any number of new
 * tokens per sequence, of a prompt or of a part of it as well as one at a time.
 *
 * santa_chunk_t: the new tokens of a batch.  Sequence b's are rows q_start[b] ..
 * q_start[b + 1] - 1 of the row buffers (q, k, v, out: one row per token) and
 * take the LAST positions of its ctx_len[b] keys (n_k without ctx_len): with c
 * tokens, token i stands at position ctx_len[b] - c + i, so one token stands
 * where the decode calls have the current one.  A sequence may have none.  Rows
 * before q_start[0] and from q_start[batch] to num_tokens - 1 hold no token: they
 * are not read or stored and their output rows are left as they were (a view into
 * longer prefix sums; a batch padded to a captured graph's size).
 *   q_start:    device int32 [batch + 1], non-decreasing, q_start[0] >= 0
 *               (entries past num_tokens count as num_tokens, a sequence whose
 *               end lies below its start has no tokens); or NULL: one token per
 *               sequence, num_tokens == batch.
 *   num_tokens: rows of the buffers, >= q_start[batch], at most 2^25.
 *   max_tokens: the most tokens that a sequence is expected to have (host
 *               value; 0 = unknown).  It chooses the kernel and the splits:
 *               any value gives the same results within rounding. */
typedef struct {
  const int32_t *q_start;
  int32_t num_tokens;
  int32_t max_tokens;
} santa_chunk_t;

/* Sliding window with sinks: the token at position p sees position j <= p if
 * j > p - window or j < sinks.  window >= 1 (it counts the token itself),
 * sinks >= 0.  Cache rows that no token of the call sees are not read, so pages
 * wholly between sinks and window may be freed. */
typedef struct {
  int32_t window;
  int32_t sinks;
} santa_window_t;

/* Rotary frequencies.  Pair i < rotary_dim / 2 turns by f_i radians per
 * position, f_i = theta^(-2 i / rotary_dim), changed for long contexts by
 *   SANTA_ROPE_LINEAR  f_i / factor;
 *   SANTA_ROPE_BASE    theta replaced by theta * factor^(R / (R - 2)), R = rotary_dim;
 *   SANTA_ROPE_BANDS   by the turns n_i = original_len * f_i / (2 pi) that the
 *                      pair makes over the original context: f_i for n_i >= high,
 *                      f_i / factor for n_i <= low, linear in n_i between;
 *   SANTA_ROPE_RAMP    f_i for pairs below d(high), f_i / factor above d(low),
 *                      linear in i between, d(n) = R ln(original_len / (2 pi n)) /
 *                      (2 ln theta), rounded down (high) and up (low).
 * gain multiplies the rotated features; 0 takes the usual one (RAMP with
 * factor > 1: 0.1 ln factor + 1; else 1). */
typedef enum {
  SANTA_ROPE_PLAIN = 0,
  SANTA_ROPE_LINEAR = 1,
  SANTA_ROPE_BASE = 2,
  SANTA_ROPE_BANDS = 3,
  SANTA_ROPE_RAMP = 4
} santa_rope_scaling_t;

typedef struct {
  int32_t rotary_dim;  /* a multiple of 16 in [16, 128]; later features pass through */
  int32_t interleaved; /* 0: pair i is features (i, i + rotary_dim / 2); 1: (2 i, 2 i + 1) */
  double theta;        /* > 1 */
  int32_t scaling;     /* santa_rope_scaling_t */
  double factor;       /* > 0 (PLAIN: ignored) */
  double original_len; /* BANDS, RAMP: > 0 */
  double low, high;    /* BANDS, RAMP: 0 < low < high */
  double gain;
} santa_rope_params_t;

/* The plan that the call takes: made once on the host, kept by the caller. */
typedef struct {
  int32_t rotary_dim;
  int32_t interleaved;
  float gain;
  int32_t reserved;
  uint64_t step[64]; /* turns per position of each pair, the fraction in units of 2^-64 */
} santa_rope_t;

/* Fill *rope from *params (host only; no stream, no device memory). */
santa_status_t santa_rope_init(const santa_rope_params_t *params, santa_rope_t *rope);

/* The new tokens' rows, in shape->dtype: element (t, h, i) of q at q + t*q_stride
 * + h*head_dim + i, of k and v likewise (strides in elements; parts of one
 * projection's rows are three pointers and one stride).  16-byte aligned, as
 * every row must be.  q may be NULL (no queries).  positions (nullable, int32
 * [num_tokens]): the positions to rotate by, where they are not the cache
 * positions. */
typedef struct {
  const void *q, *k, *v;
  int64_t q_stride, k_stride, v_stride;
  const int32_t *positions;
} santa_rows_t;

/* Rotary positions and the store into the cache, in one pass: every pair (a, b)
 * of a query or key at position p becomes gain * (a cos - b sin, b cos + a sin)
 * at the angle p * f_i, with whole turns left out exactly (off by at most |p| * 2^-60
 * of a turn, for any p, and by the float32 sine and cosine); rotated queries go to q_out
 * ([num_tokens, num_q_heads, head_dim] contiguous; may be q itself if q is
 * contiguous), rotated keys and the values as they are to the tokens' rows of
 * the cache.  rope = NULL rotates nothing (q and q_out must then be NULL): a
 * store alone.  An FP8 cache gets the E4M3 code nearest to x / scale, ties to
 * even, saturated at +-448; NaN stays NaN.  No two tokens may name the same
 * cache row (sequences that share pages must not store into shared ones).  A
 * token at a position outside [0, n_k), or whose page is negative, is rotated
 * but not stored.  kv->k_new and kv->v_new must be NULL. */
santa_status_t santa_rope_append(const santa_rows_t *rows, const santa_kv_t *kv,
                                 const santa_shape_t *shape, const santa_chunk_t *chunk,
                                 const santa_rope_t *rope, void *q_out, void *stream);

/* Bytes of workspace of santa_attend_chunk and (chunk = NULL: one token per
 * sequence) santa_decode_window; window = NULL: none.  Returns 0 if the
 * arguments are invalid.  The workspace is one of santa_workspace_init and may
 * be shared with the other calls. */
size_t santa_attend_workspace_size(const santa_shape_t *shape, const santa_kv_t *kv,
                                   const santa_chunk_t *chunk, const santa_window_t *window);

/* Exact attention of a chunk of new tokens over the cache, which already holds
 * their keys and values (santa_rope_append stores them): the token at position p
 * of sequence b sees keys 0 .. p, or with `window` (nullable) those of
 * santa_window_t:  out = softmax(scale q K^T) V over the visible keys.
 * q, out: [num_tokens, num_q_heads, head_dim] contiguous, 16-byte aligned,
 * rotated as the keys are.  A row that sees no key (a token before position 0)
 * is zero; what hidden keys and values hold, infinities and NaN too, reaches no
 * row.  A NaN in a row's query or in a key or value that it sees makes its
 * outputs NaN (a value's: those of its feature), an infinite value makes them
 * infinite or, where its weight rounds to zero, NaN.  Scores, sums and outputs are
 * kept in float32; over bfloat16 and FP8 caches a weight is rounded before it
 * multiplies its value, by up to 2^-14 of itself where max_tokens (num_tokens, if
 * unknown) times the group is at most 32, by up to 2^-8 (bfloat16) beyond.
 * Contiguous and paged caches of up to 2^30 keys, every kv_dtype; kv->k_new and
 * kv->v_new must be NULL.  santa_set_options: `splits` sets the key splits per tile, the path is
 * ignored. */
santa_status_t santa_attend_chunk(const void *q, const santa_kv_t *kv, const santa_shape_t *shape,
                                  const santa_chunk_t *chunk, const santa_window_t *window,
                                  float scale, void *out, void *ws, size_t ws_bytes, void *stream);

/* Exact decode attention with a sliding window and sinks: santa_attend_chunk
 * with one token per sequence.  q and out as in santa_decode_dense. */
santa_status_t santa_decode_window(const void *q, const santa_kv_t *kv, const santa_shape_t *shape,
                                   const santa_window_t *window, float scale, void *out, void *ws,
                                   size_t ws_bytes, void *stream);

/* Profiling hook (not part of the method).  start_event and stop_event are
 * hipEvent_t handles created by the caller with timing enabled.  The next
 * santa_decode_*, santa_rope_append or santa_attend_chunk (or santa_stream_read)
 * call made on the calling thread attaches them to its own kernels: the GPU
 * records start_event when the call's first kernel is dispatched and stop_event when its last kernel completes, so
 * hipEventElapsedTime(start, stop) is the call's execution time on the device
 * without host launch latency.  One-shot: that call consumes the request even
 * if it fails validation.  (NULL, NULL) cancels a pending request; exactly one
 * NULL is SANTA_ERR_INVALID_ARG.  The events stay owned by the caller and must
 * outlive the call's kernels. */
santa_status_t santa_time_next_call(void *start_event, void *stop_event);

/* Measurement helper (not part of the method): the attainable HBM read rate.
 * Streams `bytes` from the device buffer buf with the load the decode kernels
 * use for keys (16 bytes per lane, non-temporal, up to 16 loads in flight per
 * lane) over at most SANTA_STREAM_READ_GROUPS workgroups, each reading one
 * contiguous share, and writes to sink[w] (device,
 * caller-owned, SANTA_STREAM_READ_GROUPS uint32) the XOR of all 32-bit words
 * workgroup w read; words past the grid keep their contents, so with sink
 * zeroed first the XOR over sink is the XOR over the buffer.  buf must be
 * 16-byte aligned and bytes a positive multiple of 16 below
 * 2^34 * SANTA_STREAM_READ_GROUPS (else SANTA_ERR_INVALID_ARG).  Asynchronous
 * on `stream`; santa_time_next_call applies to it as to a decode call.  Timed
 * on a buffer the size of a step's algorithmic bytes, it is the ceiling those
 * bytes can be read at. */
#define SANTA_STREAM_READ_GROUPS 4096
santa_status_t santa_stream_read(const void *buf, size_t bytes, uint32_t *sink, void *stream);

/* Launch options (not part of the method): which kernels a call runs.  They
 * exist for tuning sweeps and for tests that cover every path; the defaults
 * choose by problem size.
 *   SANTA_PATH_AUTO        by measured speed: systematic and stratified steps
 *                          with at most 64 splits per row take the scheduled
 *                          path for S <= 1024 (paged caches up to 8192
 *                          workgroups, KV rows x splits, FP8 caches up to
 *                          2048), i.i.d. steps too at num_q_heads /
 *                          num_kv_heads <= 4 for S <= 256, or larger S on
 *                          grids of at most 256 workgroups; other sampled
 *                          steps whose rows fit one
 *                          resident round of about 1024 workgroups take one
 *                          persistent launch, larger ones the two-launch path;
 *   SANTA_PATH_ONE_LAUNCH  sampled steps: one persistent launch (k_fused_sampled);
 *   SANTA_PATH_TWO_LAUNCH  sampled steps: key stream with a CDF stash, then one
 *                          workgroup per query head (k_stream_cdf, k_value_heads);
 *   SANTA_PATH_MULTI       every step: the multi-kernel variant (score/CDF,
 *                          offsets, sampling and merge kernels);
 *   SANTA_PATH_SCHEDULED   systematic and stratified steps with at most 64
 *                          splits per row, and i.i.d. steps among them at
 *                          num_q_heads / num_kv_heads <= 4 (S <= 256, or
 *                          larger S on grids of at most 256 workgroups): one
 *                          hardware-scheduled launch, a
 *                          workgroup per split that keeps its CDF in LDS across
 *                          a row barrier (k_row_sampled); other sampled steps
 *                          as under AUTO.
 * splits: KV splits per row of the fused paths (0 = by size; at least
 * ceil(n_k / 1024)).  The options apply to every later call made on the
 * calling thread (santa_workspace_size and santa_plan_info included) until
 * they are set again; opts = NULL restores the defaults {AUTO, 0}.  A
 * workspace must be sized under the options of the calls that use it.
 * Returns SANTA_ERR_INVALID_ARG for an unknown path or splits outside
 * [0, 256]. */
typedef enum {
  SANTA_PATH_AUTO = 0,
  SANTA_PATH_ONE_LAUNCH = 1,
  SANTA_PATH_TWO_LAUNCH = 2,
  SANTA_PATH_MULTI = 3,
  SANTA_PATH_SCHEDULED = 4
} santa_path_t;

typedef struct {
  int32_t path;   /* santa_path_t */
  int32_t splits; /* 0 = by size */
} santa_options_t;

santa_status_t santa_set_options(const santa_options_t *opts);

/* The calling thread's current options (written to *opts). */
santa_status_t santa_get_options(santa_options_t *opts);

/* What a call with these arguments would launch under the calling thread's
 * options, without launching anything: the path taken (a santa_path_t other
 * than AUTO), the KV splits per row, the longest split in keys, the
 * workspace bytes (as santa_workspace_size) and the names of the kernels.
 * kernels points to a static string.  Same argument rules as
 * santa_workspace_size (S is ignored for dense and flash). */
typedef struct {
  int32_t path;
  int32_t splits;
  int32_t split_len;
  size_t workspace;
  const char *kernels;
} santa_plan_info_t;

santa_status_t santa_plan_info(const santa_shape_t *shape, const santa_kv_t *kv, int32_t S,
                               int32_t kind, santa_plan_info_t *info);

/* Human-readable name of a status code. */
const char *santa_status_string(santa_status_t status);

/* Message describing the last error returned on the calling thread ("" if none). */
const char *santa_last_error(void);

#ifdef __cplusplus
}
#endif

#endif /* SANTA_H */
