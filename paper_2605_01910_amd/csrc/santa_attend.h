// santa_attend.h -- attention of a chunk of new tokens over the KV cache, causal
// or with a sliding window and sinks (santa_attend_chunk, santa_decode_window).
//
// Rows.  The G query heads of a KV head attend over the same keys, so a tile's
// rows are (token, head) pairs, row r = token r / G, head r % G: a key row read
// once serves the whole group, and eight single-token rows fill a matrix tile
// as well as a long chunk does.
//
// Scores are computed transposed, S^T = K Q^T, with 32 keys as the matrix
// instruction's rows and 32 query rows as its columns: lane l then holds 16
// keys of query row l % 32 (keys 8 a + 4 (l / 32) + j in accumulator 4 a + j),
// so the running maximum and sum of a row need one exchange between two lanes.
// The output is transposed too, O^T += V^T P^T, and the weights are its right
// operand as they stand: an instruction sums over 16 keys, and which of them a
// lane holds is free as long as both operands agree, so lane l takes the keys
// it scored and V's operand is read from LDS to match (a transposing read for
// 16-bit elements).  Rescaling a row of O^T is one multiplication per register.
//
// Keys.  The keys that a tile's tokens can see are the sinks and a run that
// ends at its last token; they are numbered v = 0 .. nv - 1 with the hidden gap
// between left out, so no tile is spent on it.  The numbering keeps positions
// modulo 16, so that 16 rows from a multiple of 16 on are a run of one page (of
// 16 keys or more) and need one address; a row of such a group that no token
// sees is replaced by one that some token does, so hidden rows are never read
// (their pages may have been freed) and are masked like every other.
#pragma once

#include "santa_chunk.h"
#include "santa_device.h"
#include "santa_kernels.h"
#include "santa_tiles.h"

namespace santa {

typedef __bf16 abf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 abf16x2 __attribute__((ext_vector_type(2)));
typedef short as16x4 __attribute__((ext_vector_type(4)));
typedef float af32x16 __attribute__((ext_vector_type(16)));

// Element type in LDS: FP8 codes are widened (exactly) on the way in.
template <typename E>
using LE = QE<E>;

// Keys of a tile by number: v < n0 is position v, v >= n0 position v + shift;
// positions in [sinks, lo) are hidden from all of the tile's tokens.
struct KeyMap {
  int n0, shift, nv, sinks, lo;
  __device__ __forceinline__ int pos(int v) const { return v < n0 ? v : v + shift; }
  // the position whose row stands in for v's: a visible one
  __device__ __forceinline__ int row(int v) const {
    const int p = pos(v);
    return p >= sinks ? max(p, lo) : p;
  }
};

// Tokens at positions p_lo .. p_hi together see [0, sinks) and (p_lo - window, p_hi].
__device__ __forceinline__ KeyMap key_map(int p_lo, int p_hi, int window, int sinks) {
  const int lo = window ? max(0, p_lo - window + 1) : 0;
  const int n0 = (int)min((int64_t)sinks + 15, (int64_t)p_hi + 16) & ~15;
  if ((lo & ~15) <= n0) return KeyMap{0, 0, p_hi + 1, sinks, lo};
  const int shift = (lo & ~15) - n0;
  return KeyMap{n0, shift, p_hi + 1 - shift, sinks, lo};
}

// What a token sees, in v: v < hi and (v >= lo or v < sv).
struct RowSight {
  int lo, hi, sv;
};
__device__ __forceinline__ RowSight row_sight(const KeyMap &km, int p, int window) {
  const int first = window ? max(0, p - window + 1) : 0;  // the window's first position, past any gap
  return RowSight{first - km.shift, p + 1 - km.shift, min(km.sinks, km.nv)};
}

// Rows in LDS.  L: bfloat16, float32, or FP8 codes as they are in the cache
// (the operands are widened as they are read).  16-byte chunk c of row `row`
// stands at chunk c ^ swizzle: the lanes of a key read take one chunk of 32
// rows, those of a value read the same chunks of four rows (codes: of 16, 32-bit
// values: of two); either way they spread over all banks.
template <typename L>
__device__ __forceinline__ int k_swz(int row) {
  return sizeof(L) == 1 ? (row >> 1) & 7 : row & 15;
}
template <typename L>
__device__ __forceinline__ int v_swz(int row) {
  return sizeof(L) == 1 ? (row >> 1) & 7 : sizeof(L) == 2 ? (row & 3) << 2 : ((row >> 2) & 1) << 3;
}
template <typename L>
constexpr int lds_row() {
  return kHeadDim * (int)sizeof(L);
}

// Query rows as the right operand of S^T = K Q^T: lane l holds row l % 32,
// features 16 s + 8 (l / 32) .. + 7 of step s.
template <typename L>
struct AQ;
template <>
struct AQ<uint16_t> {
  abf16x8 f[8];
};
template <>
struct AQ<float> {
  float4 f[16];  // features 8 s + 4 (l / 32) .. + 3
};

// `neg`: the negated row (a negative scale becomes a positive one).
__device__ __forceinline__ void load_rows(AQ<uint16_t> &q, const uint16_t *p, bool valid, bool neg) {
  const int h = (threadIdx.x >> 5) & 1;
  const uint32_t flip = neg ? 0x80008000u : 0u;
#pragma unroll
  for (int s = 0; s < 8; ++s) {
    uint4 w = make_uint4(0, 0, 0, 0);
    if (valid) w = *reinterpret_cast<const uint4 *>(p + 16 * s + 8 * h);
    q.f[s] = __builtin_bit_cast(abf16x8, make_uint4(w.x ^ flip, w.y ^ flip, w.z ^ flip, w.w ^ flip));
  }
}
__device__ __forceinline__ void load_rows(AQ<float> &q, const float *p, bool valid, bool neg) {
  const int h = (threadIdx.x >> 5) & 1;
#pragma unroll
  for (int s = 0; s < 16; ++s) {
    float4 w = make_float4(0, 0, 0, 0);
    if (valid) w = *reinterpret_cast<const float4 *>(p + 8 * s + 4 * h);
    q.f[s] = neg ? make_float4(-w.x, -w.y, -w.z, -w.w) : w;
  }
}

// Scores of keys [32 t, 32 t + 32) of the tile at K, raw (before the scale).
__device__ __forceinline__ af32x16 score_block(const AQ<uint16_t> &q, const char *K, int t, uint8_t) {
  const int lane = threadIdx.x & 63, r = lane & 31, h = lane >> 5;
  const char *row = K + (32 * t + r) * lds_row<uint8_t>() + 8 * h;
  const int x = (r >> 1) & 7;
  af32x16 s = {};
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const Chunk<uint8_t> k{*reinterpret_cast<const uint2 *>(row + ((i ^ x) << 4))};
    s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(abf16x8, k.to_bf16()), q.f[i], s, 0, 0, 0);
  }
  return s;
}
__device__ __forceinline__ af32x16 score_block(const AQ<uint16_t> &q, const char *K, int t, uint16_t) {
  const int lane = threadIdx.x & 63, r = lane & 31, h = lane >> 5;
  const char *row = K + (32 * t + r) * lds_row<uint16_t>();
  const int x = h ^ (r & 15);
  af32x16 s = {};
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const abf16x8 k = *reinterpret_cast<const abf16x8 *>(row + (((2 * i) ^ x) << 4));
    s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(k, q.f[i], s, 0, 0, 0);
  }
  return s;
}
__device__ __forceinline__ af32x16 score_block(const AQ<float> &q, const char *K, int t, float) {
  const int lane = threadIdx.x & 63, r = lane & 31, h = lane >> 5;
  const char *row = K + (32 * t + r) * lds_row<float>();
  const int x = h ^ (r & 15);
  af32x16 s = {};
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    const float4 k = *reinterpret_cast<const float4 *>(row + (((2 * i) ^ x) << 4));
    s = __builtin_amdgcn_mfma_f32_32x32x2f32(k.x, q.f[i].x, s, 0, 0, 0);
    s = __builtin_amdgcn_mfma_f32_32x32x2f32(k.y, q.f[i].y, s, 0, 0, 0);
    s = __builtin_amdgcn_mfma_f32_32x32x2f32(k.z, q.f[i].z, s, 0, 0, 0);
    s = __builtin_amdgcn_mfma_f32_32x32x2f32(k.w, q.f[i].w, s, 0, 0, 0);
  }
  return s;
}

// The running state of 32 rows in a wave: maximum (raw score units, the same
// on both lanes of a row), the lane's share of the sum, and O^T: feature
// 32 n + 8 a + 4 (l / 32) + j of row l % 32 in o[n][4 a + j].
struct RowState {
  float m, l;
  af32x16 o[4];
};

// Values as the left operand of O^T += V^T P^T: features 32 n + l % 32 of the
// keys row .. row + 3 and row + 8 .. row + 11 (row: 16 b + 4 (l / 32)), the
// ones whose weights the lane holds.
__device__ __forceinline__ as16x4 value_quad(const char *V, int row, int n) {
  const int l = threadIdx.x & 15, g = (threadIdx.x >> 4) & 1, k = l >> 2;
  const char *p = V + (row + k) * lds_row<uint16_t>() + (((4 * n + 2 * g + ((l & 3) >> 1)) ^ (k << 2)) << 4) +
                  (l & 1) * 8;
  return __builtin_amdgcn_ds_read_tr16_b64_v4i16(
      (__attribute__((address_space(3))) as16x4 *)(reinterpret_cast<const as16x4 *>(p)));
}
__device__ __forceinline__ uint4 value_operand(const char *V, int row, int n, uint16_t) {
  const uint2 u = __builtin_bit_cast(uint2, value_quad(V, row, n));
  const uint2 v = __builtin_bit_cast(uint2, value_quad(V, row + 8, n));
  return make_uint4(u.x, u.y, v.x, v.y);
}
__device__ __forceinline__ uint4 value_operand(const char *V, int row, int n, uint8_t) {
  typedef int i32x2 __attribute__((ext_vector_type(2)));
  const int l = threadIdx.x & 15, g = (threadIdx.x >> 4) & 1, k = l >> 1;  // the lane's eighth of 8 rows x 16 codes
  const int rr = row + (k & 3) + 2 * (k & 4);
  const char *p = V + rr * lds_row<uint8_t>() + (((2 * n + g) ^ v_swz<uint8_t>(rr)) << 4) + (l & 1) * 8;
  const i32x2 w = __builtin_amdgcn_ds_read_tr8_b64_v2i32(
      (__attribute__((address_space(3))) i32x2 *)(reinterpret_cast<const i32x2 *>(p)));
  return Chunk<uint8_t>{make_uint2((unsigned)w[0], (unsigned)w[1])}.to_bf16();
}

// Non-finite values stand apart: a key that some rows of the tile do not see
// must not reach them as 0 * inf.  clean: the operand with those elements 0;
// mark: 1 where the element is of the kind (0: +inf, 1: -inf, 2: NaN).
__device__ __forceinline__ uint32_t nonfinite2(uint32_t w) {  // 0xffff halves where exponent is all ones
  const uint32_t e = w & 0x7f807f80u;
  return ((e & 0xffffu) == 0x7f80u ? 0xffffu : 0u) | ((e >> 16) == 0x7f80u ? 0xffff0000u : 0u);
}
__device__ __forceinline__ uint32_t mark2(uint32_t w, int kind) {
  auto one = [&](uint32_t x) {
    const bool inf = (x & 0x7fffu) == 0x7f80u, nan = (x & 0x7fffu) > 0x7f80u;
    return (kind == 2 ? nan : inf && ((x >> 15) != 0) == (kind == 1)) ? 0x3f80u : 0u;
  };
  return one(w & 0xffffu) | one(w >> 16) << 16;
}
__device__ __forceinline__ float mark1(float x, int kind) {
  const bool nan = x != x;
  return (kind == 2 ? nan : x == (kind ? -kInf : kInf)) ? 1.0f : 0.0f;
}
__device__ __forceinline__ float mark_value(int kind) {
  return kind == 0 ? kInf : kind == 1 ? -kInf : __builtin_nanf("");
}

// O^T += V^T P^T over keys [32 t, 32 t + 32) of the tile at V (rows of type L).
// EDGE: some row may not see some of the keys (their weights are 0).
template <bool EDGE, typename L, std::enable_if_t<sizeof(L) <= 2, int> = 0>
__device__ __forceinline__ void add_values(RowState &st, const af32x16 &p, const char *V, int t, L) {
  const int h = (threadIdx.x >> 5) & 1;
  abf16x8 pf[2];
#pragma unroll
  for (int b = 0; b < 2; ++b)
#pragma unroll
    for (int i = 0; i < 8; ++i) pf[b][i] = (__bf16)p[8 * b + i];  // nearest even: 2^-9 of a weight, the sum keeps 32 bits
  uint32_t bad = 0;
#pragma unroll
  for (int n = 0; n < 4; ++n)
#pragma unroll
    for (int b = 0; b < 2; ++b) {
      uint4 w = value_operand(V, 32 * t + 16 * b + 4 * h, n, L{});
      if constexpr (EDGE) {
        const uint4 f = make_uint4(nonfinite2(w.x), nonfinite2(w.y), nonfinite2(w.z), nonfinite2(w.w));
        bad |= f.x | f.y | f.z | f.w;
        w = make_uint4(w.x & ~f.x, w.y & ~f.y, w.z & ~f.z, w.w & ~f.w);
      }
      st.o[n] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(abf16x8, w), pf[b], st.o[n], 0, 0, 0);
    }
  if (EDGE && __any(bad != 0)) {
#pragma unroll 1
    for (int kind = 0; kind < 3; ++kind) {
      const float add = mark_value(kind);
#pragma unroll
      for (int n = 0; n < 4; ++n) {
        af32x16 c = {};
#pragma unroll
        for (int b = 0; b < 2; ++b) {
          const uint4 w = value_operand(V, 32 * t + 16 * b + 4 * h, n, L{});
          const uint4 mk = make_uint4(mark2(w.x, kind), mark2(w.y, kind), mark2(w.z, kind), mark2(w.w, kind));
          c = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(abf16x8, mk), pf[b], c, 0, 0, 0);
        }
#pragma unroll
        for (int i = 0; i < 16; ++i) st.o[n][i] += c[i] > 0.0f ? add : 0.0f;
      }
    }
  }
}
template <bool EDGE, typename L, std::enable_if_t<sizeof(L) == 4, int> = 0>
__device__ __forceinline__ void add_values(RowState &st, const af32x16 &p, const char *V, int t, L) {
  const int lane = threadIdx.x & 63, d = lane & 31, h = lane >> 5;
  auto value = [&](int n, int i) {
    const char *col = V + (32 * t + 4 * h) * lds_row<float>() + (((8 * n + (d >> 2)) ^ (h << 3)) << 4) + (d & 3) * 4;
    return *reinterpret_cast<const float *>(col + (8 * (i >> 2) + (i & 3)) * lds_row<float>());
  };
  bool bad = false;
#pragma unroll
  for (int n = 0; n < 4; ++n)
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      float w = value(n, i);
      if constexpr (EDGE) {
        const bool finite = fabsf(w) < kInf;
        bad |= !finite;
        w = finite ? w : 0.0f;
      }
      st.o[n] = __builtin_amdgcn_mfma_f32_32x32x2f32(w, p[i], st.o[n], 0, 0, 0);
    }
  if (EDGE && __any(bad)) {
#pragma unroll 1
    for (int kind = 0; kind < 3; ++kind) {
      const float add = mark_value(kind);
#pragma unroll
      for (int n = 0; n < 4; ++n) {
        af32x16 c = {};
#pragma unroll
        for (int i = 0; i < 16; ++i) c = __builtin_amdgcn_mfma_f32_32x32x2f32(mark1(value(n, i), kind), p[i], c, 0, 0, 0);
#pragma unroll
        for (int i = 0; i < 16; ++i) st.o[n][i] += c[i] > 0.0f ? add : 0.0f;
      }
    }
  }
}

// One step of the online softmax: raw scores of NB blocks of 32 keys from
// number v0 on become weights, and the running state follows.  The reference m
// of a row moves only when a score passes it by more than 8 in log2 units: a
// weight is at most 2^8, which costs 32-bit sums and the weights' rounding
// nothing, and the output is rescaled in the first tiles only instead of
// whenever one of 32 rows finds a new maximum.
template <int NB, bool EDGE>
__device__ __forceinline__ void softmax_step(RowState &st, af32x16 (&s)[NB], int v0, const RowSight &rs, float c) {
  const int h = (threadIdx.x >> 5) & 1;
  float tm = -kInf;
#pragma unroll
  for (int t = 0; t < NB; ++t)
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      if constexpr (EDGE) {
        const int v = v0 + 32 * t + 8 * (i >> 2) + 4 * h + (i & 3);
        if (!(v < rs.hi && (v >= rs.lo || v < rs.sv))) s[t][i] = -kInf;
      }
      tm = fmaxf(tm, s[t][i]);
    }
  tm = xor32_max(tm);
  if (__any(tm * c > fmaf(st.m, c, 8.0f))) {  // (no score yet: -inf, passed by any score but -inf)
    const float mn = fmaxf(st.m, tm);
    const float f = mn == -kInf ? 1.0f : fast_exp2((st.m - mn) * c);
    st.l *= f;
#pragma unroll
    for (int n = 0; n < 4; ++n)
#pragma unroll
      for (int i = 0; i < 16; ++i) st.o[n][i] *= f;
    st.m = mn;
  }
  const float mc = st.m == -kInf ? 0.0f : st.m * c;  // nothing visible yet: every weight is 0
  float l[2] = {0.0f, 0.0f};
#pragma unroll
  for (int t = 0; t < NB; ++t)
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      s[t][i] = fast_exp2(fmaf(s[t][i], c, -mc));
      l[i & 1] += s[t][i];
    }
  st.l += l[0] + l[1];
}

// ---------------------------------------------------------------------------
// Cache rows into LDS
// ---------------------------------------------------------------------------
// A wave's share of a tile: R rows, copied straight into LDS (no registers in
// between), RPL rows per copy of 1 KiB.  Copy n's lane takes chunk `lane % CPR`,
// as the swizzle moves it, of row n * RPL + lane / CPR.  Rows of a multiple of
// 16 on are one run in memory (see KeyMap), so a copy's address is a uniform
// base and a lane's constant offset; groups at the ends of what is visible, and
// pages of fewer than 16 keys, take an address per row.
template <typename E, bool PAGED, int R>
struct RowCopies {
  static constexpr int CPR = kHeadDim * (int)sizeof(E) / 16, RPL = 64 / CPR, NL = R / RPL;
  static constexpr int GR = R < 16 ? R : 16, GN = GR / RPL, NG = R / GR;  // rows and copies of a group, groups
  static_assert(R % RPL == 0 && R % GR == 0 && GR % RPL == 0, "whole copies, whole groups");
  const KvView &kv;
  const KeyMap km;
  int64_t base;         // elements to the sequence's (contiguous) or the pool's (paged) KV head
  int b, end, row0;     // rows at or past `end` repeat the last one before it; row0: the share's row in the tile
  int win, nxt, first;  // paged: lane i holds the sequence's table entries first + i and first + 64 + i
  int last_entry;       // (table entries past the last key's are not read)
  uint32_t lane_off;    // the lane's row within a copy, in bytes
  int v0;
  bool runs;            // every group of them is a run; otherwise they take an address per row
  uint64_t at[NG];      // byte offset of each group's first row

  __device__ __forceinline__ RowCopies(const KvView &kv_, const KeyMap &km_, int b_, int kvh, int end_, int row0_)
      : kv(kv_), km(km_), b(b_), end(end_), row0(row0_), win(0), nxt(0), first(-256) {
    base = (int64_t)kvh * kv.sh + (PAGED ? 0 : (int64_t)b * kv.sb);
    lane_off = (uint32_t)((int64_t)((threadIdx.x & 63) / CPR) * kv.sn * (int64_t)sizeof(E));
    last_entry = PAGED && end > 0 ? km.row(end - 1) >> kv.ps_log2 : 0;
  }
  __device__ __forceinline__ int entry(int i) const {
    return kv.bt[(int64_t)b * kv.max_pages + min(i + (int)(threadIdx.x & 63), last_entry)];
  }

  // The rows from key v on are next (some of the tile's keys lie before `end`).
  __device__ __forceinline__ void seek(int v) {
    v0 = v;
    runs = v + R <= end && (!PAGED || kv.ps_log2 >= 4);
#pragma unroll
    for (int g = 0; g < NG; ++g) {
      const int p = km.pos(v + g * GR);
      runs = runs && (p >= km.lo || p + GR <= km.sinks);
    }
    if (!runs) return;
#pragma unroll
    for (int g = 0; g < NG; ++g) {
      const int p = km.pos(v + g * GR);
      if constexpr (PAGED) {
        const int e = p >> kv.ps_log2;
        if (e < first || e >= first + 64) {  // the next 64 entries are fetched 64 entries ahead of their use
          const bool ahead = e >= first + 64 && e < first + 128;
          first = ahead ? first + 64 : e;
          win = ahead ? nxt : entry(first);
          nxt = entry(first + 64);
        }
        const int page = __builtin_amdgcn_readlane(win, e - first);
        at[g] = (uint64_t)((base + (int64_t)page * kv.sb + (int64_t)(p & ((1 << kv.ps_log2) - 1)) * kv.sn) *
                           (int64_t)sizeof(E));
      } else {
        at[g] = (uint64_t)((base + (int64_t)p * kv.sn) * (int64_t)sizeof(E));
      }
    }
  }

  // Start copying the rows of `src` (kv.k or kv.v) into the LDS tile at `dst`.
  // NT: read once by the whole call, so that they do not displace other lines.
  template <bool VALUES, bool NT>
  __device__ __forceinline__ void copy(const void *src, char *dst) const {
    const unsigned m = (unsigned)__builtin_amdgcn_readfirstlane((int)lds_addr(dst + row0 * lds_row<E>()));
    const int lane = threadIdx.x & 63;
    auto chunk = [&](int row) {
      return (lane % CPR) ^ (VALUES ? v_swz<E>(row0 + row) : k_swz<E>(row0 + row));
    };
    if (runs) {
#pragma unroll
      for (int n = 0; n < NL; ++n) {
        const char *s = static_cast<const char *>(src) + at[n / GN] + (uint64_t)(n % GN * RPL) * (uint64_t)kv.sn * sizeof(E);
        const uint32_t o = lane_off + chunk(n * RPL + lane / CPR) * 16;
        if constexpr (NT)
          asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2 nt"
                       ::"s"(m + n * 1024u), "v"(o), "s"(s) : "memory", "m0");
        else
          asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2"
                       ::"s"(m + n * 1024u), "v"(o), "s"(s) : "memory", "m0");
      }
    } else {
#pragma unroll 1
      for (int n = 0; n < NL; ++n) {
        const int row = n * RPL + lane / CPR, p = km.row(min(v0 + row, end - 1));
        int64_t off = base;
        if constexpr (PAGED)
          off += (int64_t)kv.bt[(int64_t)b * kv.max_pages + (p >> kv.ps_log2)] * kv.sb +
                 (int64_t)(p & ((1 << kv.ps_log2) - 1)) * kv.sn;
        else
          off += (int64_t)p * kv.sn;
        const char *s = static_cast<const char *>(src) + off * (int64_t)sizeof(E) + chunk(row) * 16;
        asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off"
                     ::"s"(m + n * 1024u), "v"(s) : "memory", "m0");
      }
    }
  }
};

// At most N of the wave's copies (and loads) outstanding.
template <int N>
__device__ __forceinline__ void wait_copies() {
  asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory");
}
// Every LDS read of the wave has returned: what it read may be overwritten.
__device__ __forceinline__ void wait_reads() { asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory"); }

// FP8 rows of a full tile: codes through registers, widened on the way into LDS,
// once for the four waves.  NC: 16-byte chunks of K and of V per lane.
template <bool PAGED, int KEYS>
struct WidenedRows {
  static constexpr int NC = KEYS * 8 / kThreads;
  uint4 k[NC], v[NC];
  __device__ __forceinline__ void load(const KvView &kv, const KeyMap &km, int b, int kvh, int v0, int end) {
#pragma unroll
    for (int n = 0; n < NC; ++n) {
      const int i = n * kThreads + threadIdx.x;
      const int64_t off = row_offset<PAGED>(kv, b, kvh, km.row(min(v0 + i / 8, end - 1))) + (i % 8) * 16;
      k[n] = *reinterpret_cast<const uint4 *>(static_cast<const char *>(kv.k) + off);
      v[n] = *reinterpret_cast<const uint4 *>(static_cast<const char *>(kv.v) + off);
    }
  }
  __device__ __forceinline__ void store(char *K, char *V) const {
#pragma unroll
    for (int n = 0; n < NC; ++n) {
      const int i = n * kThreads + threadIdx.x, row = i / 8, c = 2 * (i % 8);
      char *kd = K + row * lds_row<uint16_t>(), *vd = V + row * lds_row<uint16_t>();
      const int kx = k_swz<uint16_t>(row), vx = v_swz<uint16_t>(row);
      *reinterpret_cast<uint4 *>(kd + ((c ^ kx) << 4)) = Chunk<uint8_t>{make_uint2(k[n].x, k[n].y)}.to_bf16();
      *reinterpret_cast<uint4 *>(kd + (((c + 1) ^ kx) << 4)) = Chunk<uint8_t>{make_uint2(k[n].z, k[n].w)}.to_bf16();
      *reinterpret_cast<uint4 *>(vd + ((c ^ vx) << 4)) = Chunk<uint8_t>{make_uint2(v[n].x, v[n].y)}.to_bf16();
      *reinterpret_cast<uint4 *>(vd + (((c + 1) ^ vx) << 4)) = Chunk<uint8_t>{make_uint2(v[n].z, v[n].w)}.to_bf16();
    }
  }
};

// ---------------------------------------------------------------------------
// Tiles
// ---------------------------------------------------------------------------
// A workgroup's tile and key range.  Blocks are numbered KV head fastest (with
// 8 KV heads each XCD works on one head's keys), then split, then tile from
// the batch's last to its first: in a chunk the later tiles see more keys.
struct Work {
  TileAt at;
  int kvh, t, rows, p_lo;  // rows: valid ones; p_lo: position of the tile's first token
  int v_begin, v_end;
  KeyMap km;
  int64_t out_row;         // first row of the tile's partial results
  bool any;                // the tile exists
};
__device__ __forceinline__ Work find_work(const AttendArgs &a, int rows_per_tile) {
  Work w;
  const int64_t id = blockIdx.x;
  w.kvh = (int)(id % a.Hkv);
  w.t = (int)(id / a.Hkv % a.T);
  const int64_t x = a.tiles - 1 - id / a.Hkv / a.T;
  const TileAt at = find_tile(a.ch, x, a.tile_tokens);
  auto uniform = [](int i) { return __builtin_amdgcn_readfirstlane(i); };
  w.at = TileAt{uniform(at.b), uniform(at.first), uniform(at.count), uniform(at.i0)};
  w.any = w.at.b < a.ch.B;
  w.out_row = ((x * a.Hkv + w.kvh) * a.T + w.t) * rows_per_tile;
  if (!w.any) return w;
  const int L = uniform(seq_len(a.kv, w.at.b)), n = min(a.tile_tokens, w.at.count - w.at.i0);
  w.rows = n * a.G;
  w.p_lo = L - w.at.count + w.at.i0;
  // (a chunk longer than its context: tokens before position 0 see nothing)
  w.km = w.p_lo + n - 1 < 0 ? KeyMap{0, 0, 0, 0, 0} : key_map(max(w.p_lo, 0), w.p_lo + n - 1, a.window, a.sinks);
  const int len = ((w.km.nv + a.T - 1) / a.T + a.step - 1) / a.step * a.step;
  w.v_begin = min(w.t * len, w.km.nv);
  w.v_end = min(w.v_begin + len, w.km.nv);
  return w;
}

__device__ __forceinline__ RowSight tile_sight(const AttendArgs &a, const Work &w, int r) {
  const int p = w.p_lo + r / a.G;
  return p < 0 ? RowSight{0, 0, 0} : row_sight(w.km, p, a.window);
}

// Row r of the tile: its query row, and what it sees.  Rows past the last see
// what the last one sees (their results are dropped).
struct Row {
  bool valid;
  int64_t at;  // elements into q and out
  RowSight see;
};
__device__ __forceinline__ Row tile_row(const AttendArgs &a, const Work &w, int r) {
  Row x;
  x.valid = r < w.rows;
  const int rr = min(r, w.rows - 1), i = rr / a.G;
  x.at = ((int64_t)(w.at.first + w.at.i0 + i) * a.Hq + w.kvh * a.G + rr % a.G) * kHeadDim;
  x.see = tile_sight(a, w, rr);
  return x;
}

__device__ __forceinline__ uint32_t pack2(float a, float b) {
  const abf16x2 v = {(__bf16)a, (__bf16)b};  // the one rounding of an output
  return __builtin_bit_cast(uint32_t, v);
}
__device__ __forceinline__ void store4(uint16_t *p, float4 v) {
  *reinterpret_cast<uint2 *>(p) = make_uint2(pack2(v.x, v.y), pack2(v.z, v.w));
}
__device__ __forceinline__ void store4(float *p, float4 v) { *reinterpret_cast<float4 *>(p) = v; }

// Scale of the scores as a non-negative factor and the sign that goes into the
// queries; with a factor of 0 the queries are zeroed instead.
struct Scale {
  float c;
  bool neg, zero;
};
template <typename E>
__device__ __forceinline__ Scale score_scale(const AttendArgs &a, float2 sc) {
  const float c = a.scale_log2 * sc.x;
  return c == 0.0f ? Scale{1.0f, false, true} : Scale{fabsf(c), c < 0.0f, false};
}

// Many rows: 128 rows, 32 per wave; K and V tiles of KEYS keys shared by the
// four waves, two of each in LDS: the next keys are copied while this tile's
// scores are taken, the next values while its weights are used.
template <typename E>
constexpr int many_keys() {
  return sizeof(E) == 4 ? 32 : 64;
}
template <typename E, bool PAGED>
__global__ __launch_bounds__(kThreads) __attribute__((amdgpu_waves_per_eu(2))) void k_attend_many(AttendArgs a) {
  using L = LE<E>;
  constexpr int KEYS = many_keys<E>(), NB = KEYS / 32, TB = KEYS * lds_row<L>();
  constexpr bool WIDEN = sizeof(E) == 1;
  extern __shared__ __attribute__((aligned(16))) char lds[];  // K0, K1, V0, V1 (FP8: K0, V0)
  const Work w = find_work(a, kManyRows);
  if (!w.any) return;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int r = 32 * wave + (lane & 31), h = lane >> 5;
  const Row row = tile_row(a, w, r);
  const float2 sc = kv_scales<E>(a.kv, w.at.b, w.kvh, a.Hkv);
  const Scale scale = score_scale<E>(a, sc);
  AQ<L> q;
  load_rows(q, static_cast<const L *>(a.q) + row.at, row.valid && !scale.zero, scale.neg);
  // a tile is whole if every row sees all of its keys
  const RowSight first = tile_sight(a, w, 0), last = tile_sight(a, w, w.rows - 1);
  const int all_hi = min(first.hi, w.v_end);
  RowSight see = row.see;
  see.hi = min(see.hi, w.v_end);

  RowState st;
  st.m = -kInf;
  st.l = 0.0f;
#pragma unroll
  for (int n = 0; n < 4; ++n) st.o[n] = af32x16{};
  auto step = [&](int v0, const char *K, const char *V, auto between) {
    auto body = [&](auto edge) {
      constexpr bool EDGE = decltype(edge)::value;
      af32x16 s[NB];
#pragma unroll
      for (int t = 0; t < NB; ++t) s[t] = score_block(q, K, t, L{});
      softmax_step<NB, EDGE>(st, s, v0, see, scale.c);
      between();
#pragma unroll
      for (int t = 0; t < NB; ++t) add_values<EDGE>(st, s[t], V, t, L{});
    };
    if (v0 + KEYS <= all_hi && (v0 >= last.lo || v0 + KEYS <= last.sv)) body(std::false_type{});
    else body(std::true_type{});
  };
  if constexpr (WIDEN) {
    WidenedRows<PAGED, KEYS> next;
    char *K = lds, *V = lds + TB;
    if (w.v_begin < w.v_end) next.load(a.kv, w.km, w.at.b, w.kvh, w.v_begin, w.v_end);
    for (int v0 = w.v_begin; v0 < w.v_end; v0 += KEYS) {
      __syncthreads();
      next.store(K, V);
      __syncthreads();
      if (v0 + KEYS < w.v_end) next.load(a.kv, w.km, w.at.b, w.kvh, v0 + KEYS, w.v_end);
      step(v0, K, V, [] {});
    }
  } else {
    constexpr int R = KEYS / 4;
    RowCopies<E, PAGED, R> rc(a.kv, w.km, w.at.b, w.kvh, w.v_end, R * wave);
    if (w.v_begin < w.v_end) {
      rc.seek(w.v_begin + R * wave);
      rc.template copy<false, false>(a.kv.k, lds);
      rc.template copy<true, false>(a.kv.v, lds + 2 * TB);
    }
    int turn = 0;
    for (int v0 = w.v_begin; v0 < w.v_end; v0 += KEYS) {
      const bool more = v0 + KEYS < w.v_end;
      char *K = lds + turn * TB, *V = lds + (2 + turn) * TB;
      // this tile's keys are here when every wave's copies are; all waves are
      // done with the other key tile since the barrier before their values
      wait_copies<decltype(rc)::NL>();
      __syncthreads();
      if (more) {
        rc.seek(v0 + KEYS + R * wave);
        rc.template copy<false, false>(a.kv.k, lds + (turn ^ 1) * TB);
      }
      step(v0, K, V, [&] {
        if (more) wait_copies<decltype(rc)::NL>();
        else wait_copies<0>();
        __syncthreads();
        if (more) rc.template copy<true, false>(a.kv.v, lds + (2 + (turn ^ 1)) * TB);
      });
      turn ^= 1;
    }
  }

  const float l = xor32_sum(st.l);
  if (!row.valid) return;
  if (a.T == 1) {
    const float f = l > 0.0f || l != l ? sc.y / l : 0.0f;  // a row that sees nothing is zero
    L *out = static_cast<L *>(a.out) + row.at;
#pragma unroll
    for (int n = 0; n < 4; ++n)
#pragma unroll
      for (int g = 0; g < 4; ++g)
        store4(out + 32 * n + 8 * g + 4 * h, make_float4(st.o[n][4 * g] * f, st.o[n][4 * g + 1] * f,
                                                         st.o[n][4 * g + 2] * f, st.o[n][4 * g + 3] * f));
  } else {
    const int64_t at = w.out_row + r;
    if (h == 0) a.stat[at] = make_float2(st.m == -kInf ? -kInf : st.m * scale.c, l);
    if (st.m == -kInf) return;  // (nothing seen here: the sum 0 says so)
#pragma unroll
    for (int n = 0; n < 4; ++n)
#pragma unroll
      for (int g = 0; g < 4; ++g)
        *reinterpret_cast<float4 *>(a.part + at * kHeadDim + 32 * n + 8 * g + 4 * h) =
            make_float4(st.o[n][4 * g], st.o[n][4 * g + 1], st.o[n][4 * g + 2], st.o[n][4 * g + 3]);
  }
}

// Few rows: up to 32, the same for all four waves, which share out the keys:
// each wave streams its own run of them through its own two slots of LDS, the
// keys' and the values' in turn, with no barrier inside the stream, and keeps
// its own softmax; they join their results through LDS at the end.
template <typename E>
constexpr int few_wgs() {  // workgroups per CU that the slots leave room for
  return sizeof(E) == 4 ? 1 : 2;
}
template <typename E, bool PAGED>
__global__ __launch_bounds__(kThreads) __attribute__((amdgpu_waves_per_eu(few_wgs<E>()))) void k_attend_few(AttendArgs a) {
  using L = LE<E>;
  extern __shared__ __attribute__((aligned(16))) char lds[];
  __shared__ float wm[4][kFewRows], wl[4][kFewRows];
  const Work w = find_work(a, kFewRows);
  if (!w.any) return;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int r = lane & 31, h = lane >> 5;
  char *K = lds + wave * 64 * lds_row<E>(), *V = K + 32 * lds_row<E>();
  // the wave's keys: a quarter of the split's, in whole tiles
  const int quarter = ((w.v_end - w.v_begin + 3) / 4 + 31) & ~31;
  const int begin = min(w.v_begin + wave * quarter, w.v_end), end = min(begin + quarter, w.v_end);
  RowCopies<E, PAGED, 32> rc(a.kv, w.km, w.at.b, w.kvh, end, 0);
  constexpr int NL = decltype(rc)::NL;
  if (begin < end) {
    rc.seek(begin);
    rc.template copy<false, true>(a.kv.k, K);
    rc.template copy<true, true>(a.kv.v, V);
  }
  const Row row = tile_row(a, w, r);
  const float2 sc = kv_scales<E>(a.kv, w.at.b, w.kvh, a.Hkv);
  const Scale scale = score_scale<E>(a, sc);
  AQ<L> q;
  load_rows(q, static_cast<const L *>(a.q) + row.at, row.valid && !scale.zero, scale.neg);
  const RowSight first = tile_sight(a, w, 0), last = tile_sight(a, w, w.rows - 1);
  RowSight see = row.see;
  see.hi = min(see.hi, end);
  const int all_hi = min(first.hi, end);

  RowState st;
  st.m = -kInf;
  st.l = 0.0f;
#pragma unroll
  for (int n = 0; n < 4; ++n) st.o[n] = af32x16{};
  for (int v0 = begin; v0 < end; v0 += 32) {
    const bool more = v0 + 32 < end;
    wait_copies<NL>();
    af32x16 s[1] = {score_block(q, K, 0, E{})};
    wait_reads();
    if (more) {
      rc.seek(v0 + 32);
      rc.template copy<false, true>(a.kv.k, K);
    }
    auto rest = [&](auto edge) {
      constexpr bool EDGE = decltype(edge)::value;
      softmax_step<1, EDGE>(st, s, v0, see, scale.c);
      if (more) wait_copies<NL>();
      else wait_copies<0>();
      add_values<EDGE>(st, s[0], V, 0, E{});
    };
    if (v0 + 32 <= all_hi && (v0 >= last.lo || v0 + 32 <= last.sv)) rest(std::false_type{});
    else rest(std::true_type{});
    wait_reads();
    if (more) rc.template copy<true, true>(a.kv.v, V);
  }

  // join the waves: out = sum_w 2^(m_w - m) O_w / sum_w 2^(m_w - m) l_w
  const float l = xor32_sum(st.l);
  if (h == 0) {
    wm[wave][r] = st.m == -kInf ? -kInf : st.m * scale.c;
    wl[wave][r] = l;
  }
  __syncthreads();  // (also: every wave is done with its tile's memory)
  float m = -kInf;
#pragma unroll
  for (int i = 0; i < 4; ++i) m = fmaxf(m, wm[i][r]);
  const float f = st.m == -kInf ? 0.0f : fast_exp2(st.m * scale.c - m);
  float4 *part = reinterpret_cast<float4 *>(lds);  // [wave][32 quads of features][32 rows]
#pragma unroll
  for (int n = 0; n < 4; ++n)
#pragma unroll
    for (int g = 0; g < 4; ++g)
      part[(wave * 32 + 8 * n + 2 * g + h) * 32 + r] = make_float4(st.o[n][4 * g] * f, st.o[n][4 * g + 1] * f,
                                                                   st.o[n][4 * g + 2] * f, st.o[n][4 * g + 3] * f);
  __syncthreads();
  const int r2 = tid & 31, d0 = tid >> 5;  // row, and its features 16 d0 .. + 15
  if (r2 >= w.rows) return;
  float mm = -kInf, ll = 0.0f;
#pragma unroll
  for (int i = 0; i < 4; ++i) mm = fmaxf(mm, wm[i][r2]);
#pragma unroll
  for (int i = 0; i < 4; ++i) ll += wm[i][r2] == -kInf ? 0.0f : fast_exp2(wm[i][r2] - mm) * wl[i][r2];
  const int64_t at = w.out_row + r2;
  const float g = a.T > 1 ? 1.0f : ll > 0.0f || ll != ll ? sc.y / ll : 0.0f;
  const Row row2 = tile_row(a, w, r2);
  if (a.T > 1 && d0 == 0) a.stat[at] = make_float2(mm, ll);
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    float4 x = make_float4(0, 0, 0, 0);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float4 y = part[(i * 32 + 4 * d0 + k) * 32 + r2];
      x = make_float4(x.x + y.x, x.y + y.y, x.z + y.z, x.w + y.w);
    }
    x = make_float4(x.x * g, x.y * g, x.z * g, x.w * g);
    if (a.T > 1) *reinterpret_cast<float4 *>(a.part + at * kHeadDim + 16 * d0 + 4 * k) = x;
    else store4(static_cast<L *>(a.out) + row2.at + 16 * d0 + 4 * k, x);
  }
}

// Joins the splits' partial results, a wave per (KV head, row of a tile).
template <typename E, int ROWS>
__global__ __launch_bounds__(kThreads) void k_attend_merge(AttendArgs a) {
  using L = LE<E>;
  const int lane = threadIdx.x & 63;
  const int64_t id = (int64_t)blockIdx.x * (kThreads / 64) + (threadIdx.x >> 6);
  const int r = (int)(id % ROWS), kvh = (int)(id / ROWS % a.Hkv);
  const int64_t x = id / ROWS / a.Hkv;
  if (x >= a.tiles) return;
  const TileAt at = find_tile(a.ch, x, a.tile_tokens);
  if (at.b >= a.ch.B) return;
  const int i = r / a.G;
  if (i >= min(a.tile_tokens, at.count - at.i0) || i >= a.tile_tokens) return;
  const int64_t base = (x * a.Hkv + kvh) * a.T * ROWS + r;
  float m = -kInf;
  for (int t = 0; t < a.T; ++t) m = fmaxf(m, a.stat[base + (int64_t)t * ROWS].x);
  float2 o = make_float2(0, 0);
  float l = 0.0f;
  for (int t = 0; t < a.T; ++t) {
    const float2 s = a.stat[base + (int64_t)t * ROWS];
    if (s.x == -kInf) continue;  // the split holds no key that the row sees
    const float f = fast_exp2(s.x - m);
    const float2 y = reinterpret_cast<const float2 *>(a.part + (base + (int64_t)t * ROWS) * kHeadDim)[lane];
    l = fmaf(f, s.y, l);
    o = make_float2(fmaf(f, y.x, o.x), fmaf(f, y.y, o.y));
  }
  const float g = l > 0.0f || l != l ? kv_scales<E>(a.kv, at.b, kvh, a.Hkv).y / l : 0.0f;
  L *out = static_cast<L *>(a.out) + ((int64_t)(at.first + at.i0 + i) * a.Hq + kvh * a.G + r % a.G) * kHeadDim;
  if constexpr (sizeof(L) == 2) reinterpret_cast<uint32_t *>(out)[lane] = pack2(o.x * g, o.y * g);
  else reinterpret_cast<float2 *>(out)[lane] = make_float2(o.x * g, o.y * g);
}

// Few rows: a K and a V slot of 32 rows per wave, and at the end the waves'
// outputs.  Many: two tiles of K and of V (FP8: one, the next is in registers).
template <typename E>
constexpr size_t attend_lds(bool few) {
  const size_t slots = (size_t)4 * 64 * lds_row<E>(), join = (size_t)4 * kFewRows * kHeadDim * 4;
  return few ? (slots > join ? slots : join) : (size_t)(sizeof(E) == 1 ? 2 : 4) * many_keys<E>() * lds_row<LE<E>>();
}

template <typename E>
hipError_t launch_attend_e(const AttendPlan &p, const AttendArgs &a, hipStream_t st) {
  const CallTimer tm = call_timer();
  void *params[] = {const_cast<AttendArgs *>(&a)};
  const bool paged = a.kv.bt != nullptr;
  const void *fn = p.few ? (paged ? (const void *)k_attend_few<E, true> : (const void *)k_attend_few<E, false>)
                         : (paged ? (const void *)k_attend_many<E, true> : (const void *)k_attend_many<E, false>);
  hipError_t e = hipExtLaunchKernel(fn, dim3((unsigned)(p.tiles * p.Hkv * p.T)), dim3(kThreads), params,
                                    attend_lds<E>(p.few), st, tm.start, p.T > 1 ? nullptr : tm.stop, 0);
  if (e != hipSuccess || p.T == 1) return e;
  const void *mf = p.few ? (const void *)k_attend_merge<E, kFewRows> : (const void *)k_attend_merge<E, kManyRows>;
  return hipExtLaunchKernel(mf, dim3((unsigned)(p.tiles * p.Hkv * p.rows / (kThreads / 64))), dim3(kThreads), params,
                            0, st, nullptr, tm.stop, 0);
}

}  // namespace santa
