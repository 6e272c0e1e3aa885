// santa_api.hip -- C ABI of libsanta (declared in include/santa.h): argument
// validation, launch plan, workspace carve-up and kernel dispatch.  Nothing
// here allocates device memory or synchronises.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstdlib>
#include <mutex>
#include <string>

#include "santa.h"
#include "santa_chunk.h"
#include "santa_kernels.h"
#include "santa_plan.h"

namespace {

thread_local std::string g_last_error;
thread_local santa::CallTimer g_timer;

// Consumes the pending call timer when an entry point that launches kernels returns.
struct TimerScope {
  ~TimerScope() { g_timer = santa::CallTimer{}; }
};

santa_status_t fail(santa_status_t s, const std::string &msg) {
  g_last_error = msg;
  return s;
}

size_t align256(size_t x) { return (x + 255) & ~size_t(255); }

bool is_pow2(int64_t x) { return x > 0 && (x & (x - 1)) == 0; }

int ilog2(int64_t x) {
  int r = 0;
  while ((int64_t(1) << (r + 1)) <= x) ++r;
  return r;
}

// Split length: enough workgroups to cover the chip several times over (256 CUs),
// at most kSplitMax keys (the LDS tile), at least 256.
int choose_split(int64_t rows, int64_t n_k) {
  const int64_t target_wg = 2048;
  int64_t ls = (n_k * rows) / target_wg;
  int p = 256;
  while (p < santa::kSplitMax && p * 2 <= ls) p *= 2;
  return p;
}

// The calling thread's launch options (santa_set_options).  They select a
// launch path for tuning and for tests of every path; a workspace must be
// sized under the options of the calls that use it.
thread_local santa_options_t g_opts{SANTA_PATH_AUTO, 0};

// Splits per row of the fused path: enough that the whole batch of rows fills
// about `target` workgroups, at least ceil(n_k / kSplitMax).  Sampled steps
// with budgets up to S = 1024 take 256 (one per CU): at batch 1 and 32k keys
// the stratified S = 256 step runs in 27.5 us against 28.3 us with 512,
// systematic S = 512 in 27.7 against 29.1 us, S = 1024 in 29.4 against
// 29.7 us, the i.i.d. S = 256 step in 29.4 against 29.8 us.  Larger budgets
// put more claims in each split and take 512 (systematic S = 2048: 32.7 us
// against 34.2 us), and so do the dense and flash steps (level either way).
int fused_splits(int64_t rows_kv, int64_t n_k, int64_t target) {
  const int tmin = (int)((n_k + santa::kSplitMax - 1) / santa::kSplitMax);
  int fill = 128;
  while (fill > 1 && (int64_t)fill * rows_kv > target) fill >>= 1;
  int T = std::max(tmin, fill);
  if (g_opts.splits > 0) T = std::max(tmin, (int)g_opts.splits);
  return T;
}

santa_status_t check_shape(const santa_shape_t *sh) {
  if (!sh) return fail(SANTA_ERR_INVALID_ARG, "shape is NULL");
  if (sh->batch < 1 || sh->num_q_heads < 1 || sh->num_kv_heads < 1)
    return fail(SANTA_ERR_INVALID_ARG, "batch and head counts must be >= 1");
  if (sh->num_q_heads % sh->num_kv_heads)
    return fail(SANTA_ERR_INVALID_ARG, "num_q_heads must be a multiple of num_kv_heads");
  const int G = sh->num_q_heads / sh->num_kv_heads;
  if (G != 1 && G != 2 && G != 4 && G != 8)
    return fail(SANTA_ERR_UNSUPPORTED, "GQA group size must be 1, 2, 4 or 8");
  if (sh->head_dim != santa::kHeadDim) return fail(SANTA_ERR_UNSUPPORTED, "head_dim must be 128");
  if (sh->dtype != SANTA_BF16 && sh->dtype != SANTA_F32)
    return fail(SANTA_ERR_INVALID_ARG, "dtype must be SANTA_BF16 or SANTA_F32");
  return SANTA_OK;
}

// What a plan takes from the cache: its length and element type.
santa_status_t check_kv_kind(const santa_kv_t *kv, const santa_shape_t *sh) {
  if (kv->n_k < 1) return fail(SANTA_ERR_INVALID_ARG, "n_k must be >= 1");
  if (kv->kv_dtype != SANTA_KV_AS_Q && kv->kv_dtype != SANTA_KV_FP8_E4M3)
    return fail(SANTA_ERR_INVALID_ARG, "kv_dtype must be SANTA_KV_AS_Q or SANTA_KV_FP8_E4M3");
  if (kv->kv_dtype == SANTA_KV_FP8_E4M3 && sh->dtype != SANTA_BF16)
    return fail(SANTA_ERR_UNSUPPORTED, "an FP8 cache needs bfloat16 queries (shape->dtype)");
  return SANTA_OK;
}

// decode: the call is a decode step, which reads an FP8 cache on its fused paths only
santa_status_t check_kv(const santa_kv_t *kv, const santa_shape_t *sh, bool need_k, bool decode = true) {
  if (!kv) return fail(SANTA_ERR_INVALID_ARG, "kv is NULL");
  if ((need_k && !kv->k) || !kv->v) return fail(SANTA_ERR_INVALID_ARG, "kv->k or kv->v is NULL");
  const santa_status_t s = check_kv_kind(kv, sh);
  if (s != SANTA_OK) return s;
  const bool fp8 = kv->kv_dtype == SANTA_KV_FP8_E4M3;
  if (fp8) {
    if (!kv->k_scale || !kv->v_scale)
      return fail(SANTA_ERR_INVALID_ARG, "an FP8 cache needs k_scale and v_scale");
    if (kv->k_new || kv->v_new)
      return fail(SANTA_ERR_UNSUPPORTED, "the fused append is not available with an FP8 cache");
    if (decode && g_opts.path == SANTA_PATH_MULTI)
      return fail(SANTA_ERR_UNSUPPORTED, "an FP8 cache needs the fused launch layout");
  }
  const int64_t esz = fp8 ? 1 : sh->dtype == SANTA_BF16 ? 2 : 4;
  const int64_t a = 16 / esz;  // elements per 16 bytes
  if (kv->stride_b < 0 || kv->stride_n < 0 || kv->stride_h < 0)
    return fail(SANTA_ERR_INVALID_ARG, "strides must be non-negative");
  if (kv->stride_b % a || kv->stride_n % a || kv->stride_h % a)
    return fail(SANTA_ERR_UNSUPPORTED, "strides must keep every row 16-byte aligned");
  // a lane's byte offset inside a 16-row batch of keys is 32 bits
  if ((15 * kv->stride_n + santa::kHeadDim) * esz >= (int64_t(1) << 31))
    return fail(SANTA_ERR_UNSUPPORTED, "stride_n too large");
  if ((need_k && (reinterpret_cast<uintptr_t>(kv->k) & 15)) ||
      (reinterpret_cast<uintptr_t>(kv->v) & 15))
    return fail(SANTA_ERR_UNSUPPORTED, "k and v must be 16-byte aligned");
  if (!kv->k_new != !kv->v_new) return fail(SANTA_ERR_INVALID_ARG, "k_new and v_new go together");
  if ((reinterpret_cast<uintptr_t>(kv->k_new) & 15) || (reinterpret_cast<uintptr_t>(kv->v_new) & 15))
    return fail(SANTA_ERR_UNSUPPORTED, "k_new and v_new must be 16-byte aligned");
  if (kv->block_table) {
    if (!is_pow2(kv->page_size)) return fail(SANTA_ERR_UNSUPPORTED, "page_size must be a power of two");
    if (kv->max_pages < 1) return fail(SANTA_ERR_INVALID_ARG, "max_pages must be >= 1");
    if ((int64_t)kv->max_pages * kv->page_size < kv->n_k)
      return fail(SANTA_ERR_INVALID_ARG, "max_pages * page_size < n_k");
  }
  return SANTA_OK;
}

// The flash step takes the scheduled kernel (k_row_flash: no barrier before
// the value stage, one arrival per split) under the automatic and scheduled
// paths for G <= 4 and at most kRowTMax splits per row; k_fused_dense's flash
// mode otherwise.
static bool flash_rows(const santa::Plan &p) {
  return p.fused && (g_opts.path == SANTA_PATH_AUTO || g_opts.path == SANTA_PATH_SCHEDULED) &&
         p.G <= 4 && p.T <= santa::kRowTMax;
}

santa::Plan make_plan(const santa_shape_t *sh, const santa_kv_t *kv, int S, int kind) {
  santa::Plan p{};
  p.B = sh->batch;
  p.Hq = sh->num_q_heads;
  p.Hkv = sh->num_kv_heads;
  p.G = p.Hq / p.Hkv;
  p.dtype = sh->dtype;
  p.elem = kv->kv_dtype == SANTA_KV_FP8_E4M3 ? 2 : sh->dtype == SANTA_BF16 ? 0 : 1;
  p.n_k = kv->n_k;
  p.Ls = choose_split((int64_t)p.B * p.Hkv, p.n_k);
  p.T = (int)((p.n_k + p.Ls - 1) / p.Ls);
  p.S = kind == SANTA_KIND_DENSE ? 0 : S;
  p.kind = kind;
  const size_t rows = (size_t)p.B * p.Hq;
  const size_t D = santa::kHeadDim;
  size_t off = 0;
  auto take = [&](size_t bytes) {
    const size_t o = off;
    off = align256(off + bytes);
    return o;
  };
  // Every layout, fused or not, starts with the error flag and the fused
  // paths' counter area, at the same offsets
  // and of the same size, so that calls of any kind and shape can share one
  // workspace in any order: no layout puts data where another keeps counters.
  // The counters must start at zero (santa_workspace_init).
  p.off_err = take(santa::kErrBytes);
  p.off_sync = take((size_t)santa::kSyncRowsMax * santa::kSyncStride * 4);
  const bool fused = g_opts.path != SANTA_PATH_MULTI;
  // (kind FLASH: the scheduled flash kernel's plan, the dense layout with the
  // small budget's split count, which is never more than the dense step's)
  const bool small_budget = ((kind == SANTA_KIND_SYSTEMATIC || kind == SANTA_KIND_STRATIFIED ||
                              kind == SANTA_KIND_IID) && S <= 1024) || kind == SANTA_KIND_FLASH;
  const int Tf = fused_splits((int64_t)p.B * p.Hkv, p.n_k, small_budget ? 256 : 512);
  if (kind != SANTA_KIND_BERNOULLI && fused && Tf <= santa::kMaxSplits &&
      (int64_t)p.B * p.Hkv <= santa::kSyncRowsMax) {
    p.fused = 1;
    p.T = Tf;
    // rows use ceil(L_b / T) keys per split rounded up to 64; Ls is the longest
    p.Ls = (int)(((p.n_k + p.T - 1) / p.T + 63) & ~63);
    // only splits that hold keys (short caches: fewer than T splits of 64 keys)
    p.T = (int)((p.n_k + p.Ls - 1) / p.Ls);
    const bool sampled = kind != SANTA_KIND_DENSE && kind != SANTA_KIND_FLASH;
    const bool big = (int64_t)p.B * p.Hkv * p.T > 1024;  // workgroups beyond one resident round
    // systematic and stratified steps, and i.i.d. steps at G <= 4 whose sorted
    // thresholds fit registers or LDS (iid_rows), take the scheduled path
    // (its row offsets live in LDS, so at most kRowTMax splits per row) when
    // asked for, and by default where it measured faster than both other
    // paths: budgets up to 1024; paged caches up to 8192 workgroups and FP8
    // caches up to 2048 (beyond those the two-launch path was faster)
    const int64_t grid = (int64_t)p.B * p.Hkv * p.T;
    // i.i.d. thresholds: in registers up to 256 per head, in LDS up to 2048
    // on grids of at most kDirectPollMax workgroups
    const bool iid_rows = p.G <= 4 && (S <= 256 || (S <= 2048 && grid <= santa::kDirectPollMax));
    const bool rows_ok = (kind == SANTA_KIND_SYSTEMATIC || kind == SANTA_KIND_STRATIFIED ||
                          (kind == SANTA_KIND_IID && iid_rows)) &&
                         p.T <= santa::kRowTMax;
    const bool rows_auto = rows_ok && S <= 1024 && (!kv->block_table || grid <= 8192) &&
                           (p.elem != 2 || grid <= 2048);
    p.rows = g_opts.path == SANTA_PATH_SCHEDULED ? rows_ok
                                                 : (g_opts.path == SANTA_PATH_AUTO && rows_auto);
    // other sampled steps whose rows do not fit in one resident round of about
    // 1024 workgroups take the two-launch path
    p.split2 = sampled && !p.rows &&
               (g_opts.path == SANTA_PATH_TWO_LAUNCH ||
                ((g_opts.path == SANTA_PATH_AUTO || g_opts.path == SANTA_PATH_SCHEDULED) && big));
    if (p.split2) {
      p.npitch = ((int64_t)p.n_k + 63) & ~int64_t(63);
      p.off_stats = take(rows * p.T * 8);
      p.off_stash = take(rows * (size_t)p.npitch * 2);   // 16-bit in-block CDF
      p.off_coarse = take(rows * (size_t)(p.npitch / 32) * 4);
    } else {
      p.off_stats = take(rows * p.T * 8);
      p.off_part = take((size_t)p.B * p.Hkv * p.T * p.G * D * 4);
    }
    p.total = off;
    return p;
  }
  if (kind == SANTA_KIND_BERNOULLI && fused && Tf <= santa::kMaxSplits) {
    // Bernoulli scores from the feature-major cache, then the value stage of
    // the two-launch path (one workgroup per query head)
    p.fused = 1;
    p.split2 = 1;
    // splits of at most 512 keys by default: the feature-row stream of a
    // split is short, so more workgroups keep more of it in flight; a split
    // count set in the options applies as given (at least n_k / 1024)
    p.T = g_opts.splits > 0 ? Tf
                            : std::min(santa::kMaxSplits, std::max(Tf, (int)((p.n_k + 511) / 512)));
    p.Ls = (int)(((p.n_k + p.T - 1) / p.T + 63) & ~63);
    p.npitch = ((int64_t)p.n_k + 63) & ~int64_t(63);
    p.off_stats = take(rows * p.T * 8);
    p.off_stash = take(rows * (size_t)p.npitch * 2);
    p.off_coarse = take(rows * (size_t)(p.npitch / 32) * 4);
    p.total = off;
    return p;
  }
  p.off_stats = take(rows * p.T * 8);
  p.off_part = take((size_t)p.B * p.Hkv * p.T * p.G * D * 4);
  if (kind != SANTA_KIND_DENSE) {
    p.off_stash = take(rows * (size_t)p.T * p.Ls * 4);
    p.off_offs = take(rows * (size_t)(p.T + 1) * 4);
    p.off_alpha = take(rows * (size_t)p.T * 4);
    p.off_rowst = take(rows * 8);
    p.off_flag = take((size_t)p.B * p.Hkv * p.T * 4);
  }
  if (kind == SANTA_KIND_BERNOULLI) {
    p.off_bw = take(rows * D * 4);
    p.off_blist = take((size_t)p.B * p.Hkv * D * 4);
    p.off_bn = take((size_t)p.B * p.Hkv * 4);
  }
  p.total = off;
  return p;
}

santa_status_t check_ws(size_t need, void *ws, size_t ws_bytes) {
  if (!ws) return fail(SANTA_ERR_WORKSPACE, "workspace is NULL");
  if (reinterpret_cast<uintptr_t>(ws) & 255) return fail(SANTA_ERR_WORKSPACE, "workspace must be 256-byte aligned");
  if (ws_bytes < need)
    return fail(SANTA_ERR_WORKSPACE, "workspace too small: need " + std::to_string(need) +
                                         " bytes, got " + std::to_string(ws_bytes));
  return SANTA_OK;
}

santa_status_t check_ws(const santa::Plan &p, void *ws, size_t ws_bytes) { return check_ws(p.total, ws, ws_bytes); }

bool misaligned(const void *p) { return reinterpret_cast<uintptr_t>(p) & 15; }

// The attention numbers keys in 32 bits and steps past the last of a split by a tile.
santa_status_t check_attend_keys(const santa_kv_t *kv) {
  if (kv->n_k > (1 << 30)) return fail(SANTA_ERR_UNSUPPORTED, "n_k must be at most 2^30");
  return SANTA_OK;
}

constexpr int64_t kMaxWorkgroups = UINT32_MAX / santa::kThreads;

// Whether both launches of the plan count their threads in 32 bits (a wave per row that is joined).
bool attend_fits(const santa::AttendPlan &p) {
  const int64_t groups = p.grid_tiles * p.Hkv;
  return groups * p.T <= kMaxWorkgroups &&
         (p.T == 1 || p.join || groups * p.rows / (santa::kThreads / 64) <= kMaxWorkgroups);
}

// Chunk of new tokens (NULL: one per sequence).
santa_status_t check_chunk(const santa_chunk_t *ch, const santa_shape_t *sh, santa_chunk_t *out) {
  *out = ch ? *ch : santa_chunk_t{nullptr, sh->batch, 1};
  if (out->num_tokens < 1) return fail(SANTA_ERR_INVALID_ARG, "num_tokens must be >= 1");
  if (out->num_tokens > (1 << 25)) return fail(SANTA_ERR_UNSUPPORTED, "num_tokens must be at most 2^25");
  if (out->max_tokens < 0) return fail(SANTA_ERR_INVALID_ARG, "max_tokens must be >= 0");
  if (!out->q_start) {
    if (out->num_tokens != sh->batch)
      return fail(SANTA_ERR_INVALID_ARG, "without q_start, num_tokens must equal batch");
    out->max_tokens = 1;
  }
  return SANTA_OK;
}

santa_status_t check_window(const santa_window_t *win) {
  if (win && (win->window < 1 || win->sinks < 0))
    return fail(SANTA_ERR_INVALID_ARG, "window must be >= 1 and sinks >= 0");
  return SANTA_OK;
}

santa::AttendPlan make_attend_plan(const santa_shape_t *sh, const santa_kv_t *kv, const santa_chunk_t &ch,
                                   const santa_window_t *win) {
  santa::AttendPlan p{};
  p.B = sh->batch;
  p.Hq = sh->num_q_heads;
  p.Hkv = sh->num_kv_heads;
  p.G = p.Hq / p.Hkv;
  p.dtype = sh->dtype;
  p.elem = kv->kv_dtype == SANTA_KV_FP8_E4M3 ? 2 : sh->dtype == SANTA_BF16 ? 0 : 1;
  const int64_t longest = ch.max_tokens ? std::min(ch.max_tokens, ch.num_tokens) : ch.num_tokens;
  // Few rows, up to one matrix tile's columns (us, this kernel / full tiles, groups of
  // four.  bf16: one sequence over 8k keys, 32 rows 17.5 / 22.3, 128 rows 25.7 / 25.4;
  // 8 over 4k, 32 rows 31.9 / 32.7, 48 rows in two tiles 44.3 / 33.7; 32 over 8k 172 /
  // 209, 275 / 210.  FP8 and float32 tiles cost more per key and would gain up to 64
  // rows: FP8, 32 over 8k, 113 / 175, 160 / 184, 128 rows 278 / 205; float32, 8 over 4k,
  // 72.9 / 136, 108 / 140, 182 / 148, but one over 1k keys 20.7 / 16.6, 20.6 / 19.6).
  p.few = longest * p.G <= santa::kFewRows;
  p.rows = p.few ? santa::kFewRows : santa::kManyRows;
  p.tile_tokens = p.rows / p.G;
  // whatever the lengths: n sequences with tokens have at most this many tiles
  const int64_t n = std::min(p.B, ch.num_tokens);
  p.tiles = (ch.num_tokens - n) / p.tile_tokens + n;
  const int64_t keys = win ? std::min<int64_t>(kv->n_k, (int64_t)win->sinks + win->window + p.tile_tokens - 1) : kv->n_k;
  p.step = p.few || p.elem == 1 ? 32 : 64;
  // Splits.  A longer split costs its stream, another split its share of the
  // joining: the length that balances them grows with the root of the keys (one
  // token, us at T splits: 1k keys 16.6 at 1, 12.9 at 8, 14.5 at 24; 4k 39 / 15.1
  // at 12 / 18.5 at 32; 16k 21.8 at 24 / 28.4 at 64).  32-bit full tiles spend
  // eight times as long on a key and take the root itself (77 tokens over 1k
  // keys: 147 at 1, 19.5 at 32).  Grids past one workgroup per CU take a whole
  // second one or none (32k keys: 256 workgroups 32.0, 384 37.6, 512 37.2; two
  // tiles of them 57.6, 44.4, 40.1).
  // (the tiles to expect, where the caller says how long a sequence's chunk may be; only
  // these are split and have partial results, however many rows the buffers hold)
  p.grid_tiles = std::min(p.tiles, n * ((longest + p.tile_tokens - 1) / p.tile_tokens));
  // (a launch counts its threads in 32 bits: the grid's workgroups take what is past that too)
  p.grid_tiles = std::max<int64_t>(1, std::min(p.grid_tiles, kMaxWorkgroups / p.Hkv));
  const int64_t busy = p.grid_tiles * p.Hkv;
  const double root = std::sqrt((double)keys);
  const bool heavy = p.elem == 1 && !p.few;
  const int64_t len = std::max<int64_t>(heavy ? 32 : 128, (int64_t)(heavy ? root : 5 * root));
  int64_t T = keys / len;
  if (busy * T > 256) T = T >= 512 / busy ? 512 / busy : 256 / busy;
  if (g_opts.splits > 0) T = g_opts.splits;
  p.T = (int)std::max<int64_t>(1, std::min<int64_t>(T, santa::kMaxSplits));
  size_t off = 0;
  auto take = [&](size_t bytes) {
    const size_t o = off;
    off = align256(off + bytes);
    return o;
  };
  take(santa::kErrBytes);  // the head that every layout shares (make_plan)
  p.off_sync = take((size_t)santa::kSyncRowsMax * santa::kSyncStride * 4);
  // With a row per wave to join, the tile's last split does it in passing; more
  // rows queue up in that one workgroup and are faster in a launch of their own
  // (us, last split / launch, window of 1024: one sequence of G = 4 11.2 / 12.0, of
  // G = 8 12.0 / 11.9, 16 of G = 4 17.7 / 18.9, of G = 8 19.8 / 18.9; 32k keys,
  // G = 4 27.3 / 27.9, G = 8 31.0 / 27.8; two tokens of G = 4 29.2 / 28.2).
  p.join = p.few && p.T > 1 && p.T <= 64 && longest * p.G <= 4 && busy <= santa::kSyncRowsMax;
  if (p.T > 1) {
    const size_t rows = (size_t)busy * p.T * p.rows;
    p.off_stat = take(rows * 8);
    p.off_part = take(rows * santa::kHeadDim * 4);
  }
  p.total = off;
  return p;
}

santa::KvView make_view(const santa_kv_t *kv) {
  santa::KvView v{};
  v.k = kv->k;
  v.v = kv->v;
  v.sb = kv->stride_b;
  v.sn = kv->stride_n;
  v.sh = kv->stride_h;
  v.ctx = kv->ctx_len;
  v.bt = kv->block_table;
  v.ps_log2 = kv->block_table ? ilog2(kv->page_size) : 0;
  v.max_pages = kv->max_pages;
  v.n_k = kv->n_k;
  v.k_new = kv->k_new;
  v.v_new = kv->v_new;
  v.ks = kv->kv_dtype == SANTA_KV_FP8_E4M3 ? kv->k_scale : nullptr;
  v.vs = kv->kv_dtype == SANTA_KV_FP8_E4M3 ? kv->v_scale : nullptr;
  return v;
}

santa_status_t hip_status(hipError_t e) {
  if (e != hipSuccess) return fail(SANTA_ERR_HIP, std::string("HIP: ") + hipGetErrorString(e));
  return SANTA_OK;
}

float log2_scale(float scale) { return scale * 1.44269504088896340736f; }

santa_status_t common_checks(const void *q, const santa_kv_t *kv, const santa_shape_t *sh,
                             float scale, void *out, bool need_k) {
  g_last_error.clear();
  santa_status_t s = check_shape(sh);
  if (s != SANTA_OK) return s;
  s = check_kv(kv, sh, need_k);
  if (s != SANTA_OK) return s;
  if (!q || !out) return fail(SANTA_ERR_INVALID_ARG, "q or out is NULL");
  if ((reinterpret_cast<uintptr_t>(q) & 15)) return fail(SANTA_ERR_UNSUPPORTED, "q must be 16-byte aligned");
  if (!std::isfinite(scale)) return fail(SANTA_ERR_INVALID_ARG, "scale must be finite");
  return SANTA_OK;
}

// santa_attend_chunk and santa_decode_window
santa_status_t attend(const void *q, const santa_kv_t *kv, const santa_shape_t *sh, const santa_chunk_t *chunk,
                      const santa_window_t *win, float scale, void *out, void *ws, size_t ws_bytes, void *stream) {
  TimerScope timer_scope;
  g_last_error.clear();
  santa_chunk_t ch;
  santa_status_t s = check_shape(sh);
  if (s == SANTA_OK) s = check_kv(kv, sh, true, false);
  if (s == SANTA_OK) s = check_attend_keys(kv);
  if (s == SANTA_OK) s = check_chunk(chunk, sh, &ch);
  if (s == SANTA_OK) s = check_window(win);
  if (s != SANTA_OK) return s;
  if (kv->k_new) return fail(SANTA_ERR_UNSUPPORTED, "k_new and v_new must be NULL: santa_rope_append stores new rows");
  if (!q || !out) return fail(SANTA_ERR_INVALID_ARG, "q or out is NULL");
  if (misaligned(q) || misaligned(out)) return fail(SANTA_ERR_UNSUPPORTED, "q and out must be 16-byte aligned");
  if (!std::isfinite(scale)) return fail(SANTA_ERR_INVALID_ARG, "scale must be finite");
  const santa::AttendPlan p = make_attend_plan(sh, kv, ch, win);
  if (!attend_fits(p)) return fail(SANTA_ERR_UNSUPPORTED, "too many KV heads or splits for one launch");
  s = check_ws(p.total, ws, ws_bytes);
  if (s != SANTA_OK) return s;
  santa::AttendArgs a{};
  a.kv = make_view(kv);
  a.ch = santa::ChunkView{ch.q_start, sh->batch, ch.num_tokens};
  a.q = q;
  a.out = out;
  a.stat = reinterpret_cast<float2 *>(static_cast<char *>(ws) + p.off_stat);
  a.part = reinterpret_cast<float *>(static_cast<char *>(ws) + p.off_part);
  a.sync = p.join ? reinterpret_cast<unsigned long long *>(static_cast<char *>(ws) + p.off_sync) : nullptr;
  a.Hq = p.Hq;
  a.Hkv = p.Hkv;
  a.g_log2 = ilog2(p.G);
  a.tile_tokens = p.tile_tokens;
  a.T = p.T;
  a.step = p.step;
  a.tiles = p.tiles;
  a.grid_tiles = p.grid_tiles;
  a.window = win ? win->window : 0;
  a.sinks = win ? win->sinks : 0;
  a.scale_log2 = log2_scale(scale);
  return hip_status(santa::launch_attend(p, a, static_cast<hipStream_t>(stream)));
}

// Turns per position of pair i, before any whole turns are left out.  In 64 bits of
// mantissa: an error of a frequency grows with the position (a double's 2^-53 would
// be 1e-7 of a turn at 2^30, and more than the sine's 32 bits from 2^24 on).
long double rope_turns(const santa_rope_params_t &r, int i) {
  const long double pi2 = 6.283185307179586476925286766559L, R = r.rotary_dim;
  const long double theta =
      r.scaling == SANTA_ROPE_BASE ? r.theta * std::pow((long double)r.factor, R / (R - 2)) : (long double)r.theta;
  const long double f = std::pow(theta, -2 * i / R);
  long double keep = 1;  // share of the unscaled frequency
  if (r.scaling == SANTA_ROPE_LINEAR) keep = 0;
  if (r.scaling == SANTA_ROPE_BANDS) keep = (r.original_len * f / pi2 - r.low) / ((long double)r.high - r.low);
  if (r.scaling == SANTA_ROPE_RAMP) {
    const long double ln = std::log((long double)r.theta);
    auto pair = [&](double turns) { return R * std::log(r.original_len / (pi2 * turns)) / (2 * ln); };
    const long double lo = std::max(0.0L, std::floor(pair(r.high))), hi = std::min(R - 1, std::ceil(pair(r.low)));
    keep = 1 - (i - lo) / std::max(hi - lo, 0.001L);
  }
  keep = std::min(1.0L, std::max(0.0L, keep));
  const bool scaled = r.scaling != SANTA_ROPE_PLAIN && r.scaling != SANTA_ROPE_BASE;
  return (scaled ? f * keep + f / r.factor * (1 - keep) : f) / pi2;
}

santa_status_t sampled(const void *q, const santa_kv_t *kv, const santa_shape_t *sh, float scale,
                       int32_t S, const float *u, int32_t *idx_out, void *out, void *ws,
                       size_t ws_bytes, void *stream, bool strat) {
  TimerScope timer_scope;
  santa_status_t s = common_checks(q, kv, sh, scale, out, true);
  if (s != SANTA_OK) return s;
  if (S < 1 || S > (1 << 24)) return fail(SANTA_ERR_INVALID_ARG, "S must be in [1, 2^24]");
  if (!u) return fail(SANTA_ERR_INVALID_ARG, "u is NULL");
  const santa::Plan p = make_plan(sh, kv, S, strat ? SANTA_KIND_STRATIFIED : SANTA_KIND_SYSTEMATIC);
  s = check_ws(p, ws, ws_bytes);
  if (s == SANTA_OK && kv->k_new && !p.fused)
    s = fail(SANTA_ERR_UNSUPPORTED, "the fused append (k_new, v_new) needs the fused path");
  if (s == SANTA_OK && kv->kv_dtype != SANTA_KV_AS_Q && !p.fused)
    s = fail(SANTA_ERR_UNSUPPORTED, "an FP8 cache needs the fused launch layout");
  if (s != SANTA_OK) return s;
  if (p.fused)
    return hip_status(santa::launch_fused_sampled(p, make_view(kv), q, log2_scale(scale),
                                                  strat ? 1 : 0, u, idx_out, out,
                                                  static_cast<char *>(ws),
                                                  static_cast<hipStream_t>(stream)));
  return hip_status(santa::launch_sampled(p, make_view(kv), q, log2_scale(scale), strat, u, idx_out,
                                          out, static_cast<char *>(ws),
                                          static_cast<hipStream_t>(stream)));
}

// Scratch of the no-allocation entry point: the workspace of its calls, one
// array per GPU in the library's own device memory (a code-object global, so
// the loader places it and nothing is allocated at call time).  In host code
// `scratch` names a host-side stand-in, never a device address: its device
// address on each GPU comes from hipGetSymbolAddress, taken once per device
// with that device current, and only that address is passed to kernels.
static __device__ __align__(256) unsigned char scratch[SANTA_STATIC_SCRATCH_BYTES];

constexpr int kMaxDevices = 64;
std::mutex g_scratch_mu;
void *g_scratch_ptr[kMaxDevices];  // device address of `scratch` on each GPU (null: not yet)

// The calling thread's current device, which must also own `stream`, and the
// device address of its scratch array (set up on the device's first call).
santa_status_t scratch_for(hipStream_t stream, void **ptr) {
  int dev = -1, sdev = -1;
  if (hipGetDevice(&dev) != hipSuccess || dev < 0 || dev >= kMaxDevices)
    return fail(SANTA_ERR_HIP, "no usable current device");
  if (stream && (hipStreamGetDevice(stream, &sdev) != hipSuccess || sdev != dev))
    return fail(SANTA_ERR_INVALID_ARG, "stream must belong to the current device");
  std::lock_guard<std::mutex> lock(g_scratch_mu);
  if (!g_scratch_ptr[dev]) {
    void *p = nullptr;
    const hipError_t e = hipGetSymbolAddress(&p, HIP_SYMBOL(scratch));
    if (e != hipSuccess || !p) return fail(SANTA_ERR_HIP, "hipGetSymbolAddress(scratch) failed");
    g_scratch_ptr[dev] = p;
  }
  *ptr = g_scratch_ptr[dev];
  return SANTA_OK;
}

}  // namespace

santa::CallTimer &santa::call_timer() { return g_timer; }

extern "C" {

size_t santa_workspace_size(const santa_shape_t *shape, const santa_kv_t *kv, int32_t S,
                            int32_t kind) {
  if (check_shape(shape) != SANTA_OK || !kv || kv->n_k < 1) return 0;
  if (kind < SANTA_KIND_DENSE || kind > SANTA_KIND_IID) return 0;
  if (kind == SANTA_KIND_FLASH) kind = SANTA_KIND_DENSE;  // the same launch layout
  if (kind != SANTA_KIND_DENSE && (S < 1 || S > (1 << 24))) return 0;
  return make_plan(shape, kv, S, kind).total;
}

santa_status_t santa_workspace_init(void *ws, size_t ws_bytes, void *stream) {
  g_last_error.clear();
  if (!ws) return fail(SANTA_ERR_WORKSPACE, "workspace is NULL");
  if (reinterpret_cast<uintptr_t>(ws) & 255) return fail(SANTA_ERR_WORKSPACE, "workspace must be 256-byte aligned");
  return hip_status(santa::launch_zero(ws, ws_bytes & ~size_t(15), static_cast<hipStream_t>(stream)));
}

santa_status_t santa_decode_dense(const void *q, const santa_kv_t *kv, const santa_shape_t *shape,
                                  float scale, void *out, void *ws, size_t ws_bytes,
                                  void *stream) {
  TimerScope timer_scope;
  santa_status_t s = common_checks(q, kv, shape, scale, out, true);
  if (s != SANTA_OK) return s;
  const santa::Plan p = make_plan(shape, kv, 0, SANTA_KIND_DENSE);
  s = check_ws(p, ws, ws_bytes);
  if (s == SANTA_OK && kv->k_new && !p.fused)
    s = fail(SANTA_ERR_UNSUPPORTED, "the fused append (k_new, v_new) needs the fused path");
  if (s == SANTA_OK && kv->kv_dtype != SANTA_KV_AS_Q && !p.fused)
    s = fail(SANTA_ERR_UNSUPPORTED, "an FP8 cache needs the fused launch layout");
  if (s != SANTA_OK) return s;
  if (p.fused)
    return hip_status(santa::launch_fused_dense(p, make_view(kv), q, log2_scale(scale), out,
                                                static_cast<char *>(ws),
                                                static_cast<hipStream_t>(stream)));
  return hip_status(santa::launch_dense(p, make_view(kv), q, log2_scale(scale), out,
                                        static_cast<char *>(ws), static_cast<hipStream_t>(stream)));
}

santa_status_t santa_decode_systematic(const void *q, const santa_kv_t *kv,
                                       const santa_shape_t *shape, float scale, int32_t S,
                                       const float *u, int32_t *idx_out, void *out, void *ws,
                                       size_t ws_bytes, void *stream) {
  return sampled(q, kv, shape, scale, S, u, idx_out, out, ws, ws_bytes, stream, false);
}

santa_status_t santa_decode_stratified(const void *q, const santa_kv_t *kv,
                                       const santa_shape_t *shape, float scale, int32_t S,
                                       const float *u, int32_t *idx_out, void *out, void *ws,
                                       size_t ws_bytes, void *stream) {
  return sampled(q, kv, shape, scale, S, u, idx_out, out, ws, ws_bytes, stream, true);
}

santa_status_t santa_decode_stratified_noalloc(const void *q, const santa_kv_t *kv,
                                               const santa_shape_t *shape, float scale, int32_t S,
                                               const float *u, int32_t *idx_out, void *out,
                                               void *stream) {
  TimerScope timer_scope;
  santa_status_t s = common_checks(q, kv, shape, scale, out, true);
  if (s != SANTA_OK) return s;
  if (S < 1 || S > (1 << 24)) return fail(SANTA_ERR_INVALID_ARG, "S must be in [1, 2^24]");
  if (!u) return fail(SANTA_ERR_INVALID_ARG, "u is NULL");
  const santa::Plan p = make_plan(shape, kv, S, SANTA_KIND_STRATIFIED);
  if (p.total > SANTA_STATIC_SCRATCH_BYTES)
    return fail(SANTA_ERR_WORKSPACE, "the call needs more workspace than the static scratch array "
                                     "holds (SANTA_STATIC_SCRATCH_BYTES)");
  if (!p.fused) return fail(SANTA_ERR_UNSUPPORTED, "the no-allocation call needs the fused launch layout");
  const hipStream_t st = static_cast<hipStream_t>(stream);
  void *ws = nullptr;
  s = scratch_for(st, &ws);
  if (s != SANTA_OK) return s;
  // The array keeps the previous call's contents.  Clear what must start at
  // zero: the wait flag and the row counters this call uses (a fill kernel,
  // not a memset, so that the call can be captured in a graph).  Everything
  // else the call reads it writes first.
  const size_t head = p.off_sync + (size_t)p.B * p.Hkv * santa::kSyncStride * 4;
  hipError_t e = santa::launch_zero(ws, head, st);
  if (e != hipSuccess) return hip_status(e);
  return hip_status(santa::launch_fused_sampled(p, make_view(kv), q, log2_scale(scale), 1, u,
                                                idx_out, out, static_cast<char *>(ws), st));
}

santa_status_t santa_decode_bernoulli_qk(const void *q, const santa_kt_t *kt,
                                         const santa_kv_t *kv, const santa_shape_t *shape,
                                         float scale, int32_t B_draws, int32_t mode,
                                         const float *u_q, int32_t S, const float *u,
                                         int32_t *idx_out, uint8_t *feat_mask_out, void *out,
                                         void *ws, size_t ws_bytes, void *stream) {
  TimerScope timer_scope;
  santa_status_t s = common_checks(q, kv, shape, scale, out, false);
  if (s != SANTA_OK) return s;
  if (kv->block_table) return fail(SANTA_ERR_UNSUPPORTED, "Bernoulli scores need a contiguous cache");
  if (kv->kv_dtype != SANTA_KV_AS_Q)
    return fail(SANTA_ERR_UNSUPPORTED, "Bernoulli scores need a cache in the query's dtype");
  if (!kt || !kt->k_t) return fail(SANTA_ERR_INVALID_ARG, "kt or kt->k_t is NULL");
  const int64_t a = shape->dtype == SANTA_BF16 ? 8 : 4;
  if (kt->stride_b < 0 || kt->stride_h < 0 || kt->stride_d < kv->n_k)
    return fail(SANTA_ERR_INVALID_ARG, "kt strides must be >= 0 and stride_d >= n_k");
  if (kt->stride_b % a || kt->stride_h % a || kt->stride_d % a ||
      (reinterpret_cast<uintptr_t>(kt->k_t) & 15))
    return fail(SANTA_ERR_UNSUPPORTED, "kt rows must be 16-byte aligned");
  if (mode != 0 && mode != 1) return fail(SANTA_ERR_INVALID_ARG, "mode must be 0 or 1");
  if (B_draws < 1 || B_draws > 64) return fail(SANTA_ERR_INVALID_ARG, "B_draws must be in [1, 64]");
  if (!u_q || !u) return fail(SANTA_ERR_INVALID_ARG, "u_q or u is NULL");
  if (S < 1 || S > (1 << 24)) return fail(SANTA_ERR_INVALID_ARG, "S must be in [1, 2^24]");
  const santa::Plan p = make_plan(shape, kv, S, SANTA_KIND_BERNOULLI);
  s = check_ws(p, ws, ws_bytes);
  if (s == SANTA_OK && kv->k_new)
    s = fail(SANTA_ERR_UNSUPPORTED, "the fused append (k_new, v_new) is not available with Bernoulli scores");
  if (s != SANTA_OK) return s;
  santa::KtView ktv{kt->k_t, kt->stride_b, kt->stride_h, kt->stride_d};
  if (p.fused)
    return hip_status(santa::launch_fused_bernoulli(
        p, make_view(kv), ktv, q, log2_scale(scale), B_draws, mode, u_q, u, idx_out,
        feat_mask_out, out, static_cast<char *>(ws), static_cast<hipStream_t>(stream)));
  return hip_status(santa::launch_bernoulli(p, make_view(kv), ktv, q, log2_scale(scale), B_draws,
                                            mode, u_q, u, idx_out, feat_mask_out, out,
                                            static_cast<char *>(ws),
                                            static_cast<hipStream_t>(stream)));
}

santa_status_t santa_decode_iid(const void *q, const santa_kv_t *kv, const santa_shape_t *shape,
                                float scale, int32_t S, const float *u, int32_t *idx_out,
                                void *out, void *ws, size_t ws_bytes, void *stream) {
  TimerScope timer_scope;
  santa_status_t s = common_checks(q, kv, shape, scale, out, true);
  if (s != SANTA_OK) return s;
  const int G = shape->num_q_heads / shape->num_kv_heads;
  if (S < 1 || (int64_t)G * (2 * S + 1) > 4096)
    return fail(SANTA_ERR_INVALID_ARG, "S must satisfy 1 <= S and G*(2S+1) <= 4096 for the i.i.d. step");
  if (!u) return fail(SANTA_ERR_INVALID_ARG, "u is NULL");
  const santa::Plan p = make_plan(shape, kv, S, SANTA_KIND_IID);
  s = check_ws(p, ws, ws_bytes);
  if (s == SANTA_OK && kv->k_new && !p.fused)
    s = fail(SANTA_ERR_UNSUPPORTED, "the fused append (k_new, v_new) needs the fused path");
  if (s == SANTA_OK && kv->kv_dtype != SANTA_KV_AS_Q && !p.fused)
    s = fail(SANTA_ERR_UNSUPPORTED, "an FP8 cache needs the fused launch layout");
  if (s != SANTA_OK) return s;
  if (!p.fused) return fail(SANTA_ERR_UNSUPPORTED, "the i.i.d. step needs the fused launch layout");
  return hip_status(santa::launch_fused_sampled(p, make_view(kv), q, log2_scale(scale), 2, u,
                                                idx_out, out, static_cast<char *>(ws),
                                                static_cast<hipStream_t>(stream)));
}

santa_status_t santa_decode_flash(const void *q, const santa_kv_t *kv, const santa_shape_t *shape,
                                  float scale, int32_t tile, int32_t S_tile, const float *u,
                                  int32_t *idx_out, void *out, void *ws, size_t ws_bytes,
                                  void *stream) {
  TimerScope timer_scope;
  santa_status_t s = common_checks(q, kv, shape, scale, out, true);
  if (s != SANTA_OK) return s;
  if (!is_pow2(tile) || tile < 16 || tile > santa::kSplitMax)
    return fail(SANTA_ERR_INVALID_ARG, "tile must be a power of two in [16, 1024]");
  if (S_tile < 1 || S_tile > 4096) return fail(SANTA_ERR_INVALID_ARG, "S_tile must be in [1, 4096]");
  if (!u) return fail(SANTA_ERR_INVALID_ARG, "u is NULL");
  santa::Plan p = make_plan(shape, kv, 0, SANTA_KIND_DENSE);
  const bool rows = flash_rows(p);
  if (rows) p = make_plan(shape, kv, 0, SANTA_KIND_FLASH);
  s = check_ws(p, ws, ws_bytes);
  if (s == SANTA_OK && kv->k_new && !p.fused)
    s = fail(SANTA_ERR_UNSUPPORTED, "the fused append (k_new, v_new) needs the fused path");
  if (s == SANTA_OK && kv->kv_dtype != SANTA_KV_AS_Q && !p.fused)
    s = fail(SANTA_ERR_UNSUPPORTED, "an FP8 cache needs the fused launch layout");
  if (s != SANTA_OK) return s;
  if (!p.fused) return fail(SANTA_ERR_UNSUPPORTED, "the flash step needs the fused launch layout");
  return hip_status(santa::launch_fused_flash(p, make_view(kv), q, log2_scale(scale), ilog2(tile),
                                              S_tile, u, idx_out, out, static_cast<char *>(ws),
                                              static_cast<hipStream_t>(stream), rows));
}

santa_status_t santa_rope_init(const santa_rope_params_t *params, santa_rope_t *rope) {
  g_last_error.clear();
  if (!params || !rope) return fail(SANTA_ERR_INVALID_ARG, "params or rope is NULL");
  const santa_rope_params_t &r = *params;
  if (r.rotary_dim < 16 || r.rotary_dim > santa::kHeadDim || r.rotary_dim % 16)
    return fail(SANTA_ERR_UNSUPPORTED, "rotary_dim must be a multiple of 16 in [16, 128]");
  if (r.interleaved != 0 && r.interleaved != 1) return fail(SANTA_ERR_INVALID_ARG, "interleaved must be 0 or 1");
  if (!(r.theta > 1.0) || !std::isfinite(r.theta)) return fail(SANTA_ERR_INVALID_ARG, "theta must be > 1");
  if (r.scaling < SANTA_ROPE_PLAIN || r.scaling > SANTA_ROPE_RAMP)
    return fail(SANTA_ERR_INVALID_ARG, "scaling must be a santa_rope_scaling_t");
  if (r.scaling != SANTA_ROPE_PLAIN && (!(r.factor > 0.0) || !std::isfinite(r.factor)))
    return fail(SANTA_ERR_INVALID_ARG, "factor must be > 0");
  if (r.scaling == SANTA_ROPE_BANDS || r.scaling == SANTA_ROPE_RAMP) {
    if (!(r.original_len > 0.0) || !std::isfinite(r.original_len))
      return fail(SANTA_ERR_INVALID_ARG, "original_len must be > 0");
    if (!(r.low > 0.0) || !(r.high > r.low) || !std::isfinite(r.high))
      return fail(SANTA_ERR_INVALID_ARG, "low and high must satisfy 0 < low < high");
  }
  if (!std::isfinite(r.gain)) return fail(SANTA_ERR_INVALID_ARG, "gain must be finite");
  *rope = santa_rope_t{};
  rope->rotary_dim = r.rotary_dim;
  rope->interleaved = r.interleaved;
  rope->gain = (float)(r.gain != 0.0 ? r.gain
                       : r.scaling == SANTA_ROPE_RAMP && r.factor > 1.0 ? 0.1 * std::log(r.factor) + 1.0 : 1.0);
  for (int i = 0; i < r.rotary_dim / 2; ++i) {
    const long double turns = rope_turns(r, i), x = std::ldexp(turns - std::floor(turns), 64);
    rope->step[i] = x < 18446744073709551616.0L ? (uint64_t)x : 0;
  }
  return SANTA_OK;
}

santa_status_t santa_rope_append(const santa_rows_t *rows, const santa_kv_t *kv, const santa_shape_t *shape,
                                 const santa_chunk_t *chunk, const santa_rope_t *rope, void *q_out, void *stream) {
  TimerScope timer_scope;
  g_last_error.clear();
  santa_chunk_t ch;
  santa_status_t s = check_shape(shape);
  if (s == SANTA_OK) s = check_kv(kv, shape, true, false);
  if (s == SANTA_OK) s = check_chunk(chunk, shape, &ch);
  if (s != SANTA_OK) return s;
  if (!rows || !rows->k || !rows->v) return fail(SANTA_ERR_INVALID_ARG, "rows, rows->k or rows->v is NULL");
  if (!rows->q != !q_out) return fail(SANTA_ERR_INVALID_ARG, "rows->q and q_out go together");
  if (!rope && rows->q) return fail(SANTA_ERR_INVALID_ARG, "without rope there is nothing to do for q: pass NULL");
  if (kv->k_new) return fail(SANTA_ERR_INVALID_ARG, "kv->k_new and kv->v_new must be NULL (rows holds the new rows)");
  if (rope && (rope->rotary_dim < 16 || rope->rotary_dim > santa::kHeadDim || rope->rotary_dim % 16))
    return fail(SANTA_ERR_INVALID_ARG, "rope was not filled by santa_rope_init");
  const int64_t a = shape->dtype == SANTA_BF16 ? 8 : 4;  // elements per 16 bytes
  const int64_t qw = (int64_t)shape->num_q_heads * santa::kHeadDim, kw = (int64_t)shape->num_kv_heads * santa::kHeadDim;
  if ((rows->q && rows->q_stride < qw) || rows->k_stride < kw || rows->v_stride < kw)
    return fail(SANTA_ERR_INVALID_ARG, "row strides must hold all heads");
  if (rows->q_stride % a || rows->k_stride % a || rows->v_stride % a || misaligned(rows->q) || misaligned(rows->k) ||
      misaligned(rows->v) || misaligned(q_out))
    return fail(SANTA_ERR_UNSUPPORTED, "rows and q_out must be 16-byte aligned");
  if (q_out == rows->q && rows->q && rows->q_stride != qw)
    return fail(SANTA_ERR_INVALID_ARG, "q_out may be q only if q is contiguous");
  santa::RopeArgs r{};
  r.kv = make_view(kv);
  r.ch = santa::ChunkView{ch.q_start, shape->batch, ch.num_tokens};
  r.q = rows->q;
  r.k = rows->k;
  r.v = rows->v;
  r.q_st = rows->q_stride;
  r.k_st = rows->k_stride;
  r.v_st = rows->v_stride;
  r.q_out = q_out;
  r.positions = rows->positions;
  r.Hq = rows->q ? shape->num_q_heads : 0;
  r.Hkv = shape->num_kv_heads;
  if (rope) {
    r.rotary = rope->rotary_dim;
    r.interleaved = rope->interleaved;
    r.gain = rope->gain;
    std::copy(rope->step, rope->step + santa::kHeadDim / 2, r.step);
  }
  return hip_status(santa::launch_rope(r, shape->dtype, kv->kv_dtype == SANTA_KV_FP8_E4M3 ? 2 : shape->dtype == SANTA_BF16 ? 0 : 1,
                                       static_cast<hipStream_t>(stream)));
}

size_t santa_attend_workspace_size(const santa_shape_t *shape, const santa_kv_t *kv, const santa_chunk_t *chunk,
                                   const santa_window_t *window) {
  santa_chunk_t ch;
  if (check_shape(shape) != SANTA_OK || !kv || check_kv_kind(kv, shape) != SANTA_OK ||
      check_attend_keys(kv) != SANTA_OK || check_chunk(chunk, shape, &ch) != SANTA_OK ||
      check_window(window) != SANTA_OK)
    return 0;
  const santa::AttendPlan p = make_attend_plan(shape, kv, ch, window);
  return attend_fits(p) ? p.total : 0;
}

santa_status_t santa_attend_chunk(const void *q, const santa_kv_t *kv, const santa_shape_t *shape,
                                  const santa_chunk_t *chunk, const santa_window_t *window, float scale, void *out,
                                  void *ws, size_t ws_bytes, void *stream) {
  return attend(q, kv, shape, chunk, window, scale, out, ws, ws_bytes, stream);
}

santa_status_t santa_decode_window(const void *q, const santa_kv_t *kv, const santa_shape_t *shape,
                                   const santa_window_t *window, float scale, void *out, void *ws, size_t ws_bytes,
                                   void *stream) {
  if (!window) {
    TimerScope timer_scope;
    return fail(SANTA_ERR_INVALID_ARG, "window is NULL");
  }
  return attend(q, kv, shape, nullptr, window, scale, out, ws, ws_bytes, stream);
}

santa_status_t santa_stream_read(const void *buf, size_t bytes, uint32_t *sink, void *stream) {
  TimerScope timer_scope;
  g_last_error.clear();
  if (!buf || !sink) return fail(SANTA_ERR_INVALID_ARG, "buf or sink is NULL");
  if (bytes == 0 || bytes % 16) return fail(SANTA_ERR_INVALID_ARG, "bytes must be a positive multiple of 16");
  if (bytes / 16 / SANTA_STREAM_READ_GROUPS >= (size_t(1) << 30))
    return fail(SANTA_ERR_INVALID_ARG, "bytes too large");
  if (reinterpret_cast<uintptr_t>(buf) & 15) return fail(SANTA_ERR_INVALID_ARG, "buf must be 16-byte aligned");
  return hip_status(santa::launch_stream_read(buf, bytes, sink, SANTA_STREAM_READ_GROUPS,
                                              static_cast<hipStream_t>(stream)));
}

santa_status_t santa_set_options(const santa_options_t *opts) {
  g_last_error.clear();
  if (!opts) {
    g_opts = santa_options_t{SANTA_PATH_AUTO, 0};
    return SANTA_OK;
  }
  if (opts->path < SANTA_PATH_AUTO || opts->path > SANTA_PATH_SCHEDULED)
    return fail(SANTA_ERR_INVALID_ARG, "path must be a santa_path_t");
  if (opts->splits < 0 || opts->splits > santa::kMaxSplits)
    return fail(SANTA_ERR_INVALID_ARG, "splits must be in [0, 256]");
  g_opts = *opts;
  return SANTA_OK;
}

santa_status_t santa_get_options(santa_options_t *opts) {
  g_last_error.clear();
  if (!opts) return fail(SANTA_ERR_INVALID_ARG, "opts is NULL");
  *opts = g_opts;
  return SANTA_OK;
}

santa_status_t santa_plan_info(const santa_shape_t *shape, const santa_kv_t *kv, int32_t S,
                               int32_t kind, santa_plan_info_t *info) {
  g_last_error.clear();
  if (!info) return fail(SANTA_ERR_INVALID_ARG, "info is NULL");
  santa_status_t s = check_shape(shape);
  if (s != SANTA_OK) return s;
  if (!kv || kv->n_k < 1) return fail(SANTA_ERR_INVALID_ARG, "kv is NULL or n_k < 1");
  if (kind < SANTA_KIND_DENSE || kind > SANTA_KIND_IID) return fail(SANTA_ERR_INVALID_ARG, "bad kind");
  const int32_t plan_kind = kind == SANTA_KIND_FLASH ? SANTA_KIND_DENSE : kind;
  if (plan_kind != SANTA_KIND_DENSE && (S < 1 || S > (1 << 24)))
    return fail(SANTA_ERR_INVALID_ARG, "S must be in [1, 2^24]");
  santa::Plan p = make_plan(shape, kv, S, plan_kind);
  const bool frows = kind == SANTA_KIND_FLASH && flash_rows(p);
  if (frows) p = make_plan(shape, kv, S, SANTA_KIND_FLASH);
  info->splits = p.T;
  info->split_len = p.Ls;
  info->workspace = p.total;
  if (!p.fused) {
    info->path = SANTA_PATH_MULTI;
    info->kernels = "multi-kernel variant (k_score_cdf / k_dense_split / k_bern_score, k_offsets, "
                    "k_sample, k_merge_*)";
  } else if (kind == SANTA_KIND_BERNOULLI) {
    info->path = SANTA_PATH_TWO_LAUNCH;
    info->kernels = "k_bern_stream + k_value_heads";
  } else if (frows) {
    info->path = SANTA_PATH_SCHEDULED;
    info->kernels = "k_row_flash";
  } else if (kind == SANTA_KIND_DENSE || kind == SANTA_KIND_FLASH) {
    info->path = SANTA_PATH_ONE_LAUNCH;
    info->kernels = kind != SANTA_KIND_DENSE                            ? "k_fused_dense (flash mode)"
                    : santa::dense_streams(p, kv->block_table != nullptr) ? "k_dense_stream"
                                                                            : "k_fused_dense";
  } else if (p.rows) {
    info->path = SANTA_PATH_SCHEDULED;
    info->kernels = "k_row_sampled";
  } else if (p.split2) {
    info->path = SANTA_PATH_TWO_LAUNCH;
    info->kernels = "k_stream_cdf + k_value_heads";
  } else {
    info->path = SANTA_PATH_ONE_LAUNCH;
    info->kernels = "k_fused_sampled";
  }
  return SANTA_OK;
}

santa_status_t santa_time_next_call(void *start_event, void *stop_event) {
  g_last_error.clear();
  if ((start_event == nullptr) != (stop_event == nullptr))
    return fail(SANTA_ERR_INVALID_ARG, "start_event and stop_event must both be set or both NULL");
  g_timer.start = static_cast<hipEvent_t>(start_event);
  g_timer.stop = static_cast<hipEvent_t>(stop_event);
  return SANTA_OK;
}

const char *santa_status_string(santa_status_t status) {
  switch (status) {
    case SANTA_OK: return "SANTA_OK";
    case SANTA_ERR_INVALID_ARG: return "SANTA_ERR_INVALID_ARG";
    case SANTA_ERR_UNSUPPORTED: return "SANTA_ERR_UNSUPPORTED";
    case SANTA_ERR_WORKSPACE: return "SANTA_ERR_WORKSPACE";
    case SANTA_ERR_HIP: return "SANTA_ERR_HIP";
  }
  return "SANTA_ERR_UNKNOWN";
}

const char *santa_last_error(void) { return g_last_error.c_str(); }

}  // extern "C"
