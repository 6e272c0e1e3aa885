// santa_chunk.h -- ragged batches of new tokens (santa_chunk_t) as the kernels
// of santa_rope_append and santa_attend_chunk see them, and their launchers.
#pragma once

#include <hip/hip_ext.h>
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "santa.h"
#include "santa_plan.h"

namespace santa {

// New tokens of a batch: sequence b's are rows [q_start[b], q_start[b + 1]) of
// the row buffers and take the last positions of its ctx_len[b] keys.
struct ChunkView {
  const int32_t *q_start;  // [B + 1]; null: one token per sequence, row b
  int32_t B, tokens;       // sequences; rows of the buffers
};

struct RopeArgs {
  KvView kv;
  ChunkView ch;
  const void *q, *k, *v;
  int64_t q_st, k_st, v_st;  // elements from one token's row to the next
  void *q_out;
  const int32_t *positions;  // nullable: the positions to rotate by, per token
  int32_t Hq, Hkv;           // Hq = 0: no queries
  int32_t rotary, interleaved;
  float gain;
  uint64_t step[kHeadDim / 2];  // 2^64 * fraction of a turn per position, by pair
};

// dtype: 0 bfloat16, 1 float32 rows; elem: as Plan::elem
hipError_t launch_rope(const RopeArgs &a, int dtype, int elem, hipStream_t st);

// Launch plan of the chunk's attention: a pure function of (shape, n_k, chunk,
// window, options), so santa_attend_workspace_size and the calls agree.
struct AttendPlan {
  int B, Hq, Hkv, G, dtype, elem;
  int few;            // 1: tiles of up to kFewRows rows whose waves share out the keys
  int rows;           // query rows (tokens x group) per tile
  int tile_tokens;    // tokens per tile: rows / G
  int64_t tiles;      // upper bound of the batch's tiles per KV head
  int64_t grid_tiles; // tiles to expect: the grid's; its workgroups take any others too, unsplit
  int T;              // key splits per tile of the grid; 1: no partial results
  int step;           // split lengths are multiples of this
  int join;           // a tile's last split joins its splits (few rows); 0: a launch of its own
  size_t off_sync;    // the shared head's counters (Plan::off_sync)
  size_t off_stat;    // float2 [grid_tiles * Hkv * T * rows] (reference in log2 units, sum)
  size_t off_part;    // float [grid_tiles * Hkv * T * rows * 128]
  size_t total;
};

struct AttendArgs {
  KvView kv;
  ChunkView ch;
  const void *q;
  void *out;
  float2 *stat;
  float *part;
  unsigned long long *sync;  // the row counters, if the last split joins; else null
  int32_t Hq, Hkv, g_log2, tile_tokens, T, step;
  int64_t tiles, grid_tiles;
  int32_t window, sinks;  // window 0: every earlier key
  float scale_log2;
};

constexpr int kFewRows = 32;    // rows of a "few" tile: one matrix instruction's columns
constexpr int kAttendCounter = 2;  // u64 of a row's sync block that counts a tile's splits: zero between calls
constexpr int kManyRows = 128;  // rows of a full tile: 32 per wave

hipError_t launch_attend(const AttendPlan &p, const AttendArgs &a, hipStream_t st);
template <typename E>
hipError_t launch_attend_e(const AttendPlan &p, const AttendArgs &a, hipStream_t st);

#ifdef __HIPCC__
// Sequence i's range of rows.  Ends outside [0, tokens] are clamped and falling
// ones hold nothing, so no row outside the buffers is ever named.
struct RowRange {
  int first, end;
};
__device__ __forceinline__ RowRange row_range(const ChunkView &c, int i) {
  const int s = min(max(c.q_start[i], 0), c.tokens);
  return RowRange{s, min(max(c.q_start[i + 1], s), c.tokens)};
}

// The sequence that row t belongs to and the range of its rows, by the whole
// wave: 64 sequences per load, no search chain.  b = B where none holds it (rows
// before the first sequence's and behind the last one's).
struct TokenAt {
  int b, first, count;
};
__device__ __forceinline__ TokenAt find_token(const ChunkView &c, int t) {
  if (!c.q_start) return t < c.B ? TokenAt{t, t, 1} : TokenAt{c.B, 0, 0};
  const int lane = threadIdx.x & 63;
  for (int base = 0; base < c.B; base += 64) {
    const int i = base + lane;
    const RowRange r = i < c.B ? row_range(c, i) : RowRange{0, 0};
    const unsigned long long hit = __ballot(r.first <= t && t < r.end);
    if (hit) {
      const int l = __builtin_ctzll(hit);
      const int first = __shfl(r.first, l), end = __shfl(r.end, l);
      return TokenAt{base + l, first, end - first};
    }
  }
  return TokenAt{c.B, 0, 0};
}

// Tile x of the batch (every sequence's tokens in tiles of `tt`, sequence by
// sequence): its sequence, its first token in the chunk and the chunk's range.
// b = B past the last tile.
struct TileAt {
  int b, first, count, i0;
};
__device__ __forceinline__ TileAt find_tile(const ChunkView &c, int64_t x, int tt) {
  if (!c.q_start) return x < c.B ? TileAt{(int)x, (int)x, 1, 0} : TileAt{c.B, 0, 0, 0};
  const int lane = threadIdx.x & 63;
  int64_t before = 0;
  for (int base = 0; base < c.B; base += 64) {
    const int i = base + lane;
    const RowRange r = i < c.B ? row_range(c, i) : RowRange{0, 0};
    const int n = (r.end - r.first + tt - 1) / tt;
    int incl = n;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
      const int o = __shfl_up(incl, d);
      if (lane >= d) incl += o;
    }
    const unsigned long long hit = __ballot(before + incl > x);
    if (hit) {
      const int l = __builtin_ctzll(hit);
      const int fs = __shfl(r.first, l), fe = __shfl(r.end, l), fi = __shfl(incl - n, l);
      return TileAt{base + l, fs, fe - fs, (int)(x - before - fi) * tt};
    }
    before += __shfl(incl, 63);
  }
  return TileAt{c.B, 0, 0, 0};
}
#endif

}  // namespace santa
