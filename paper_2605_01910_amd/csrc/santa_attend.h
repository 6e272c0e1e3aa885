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

// Element type of q and out.
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

// Bits of the non-finite elements of two bfloat16.
__device__ __forceinline__ uint32_t nonfinite2(uint32_t w) {
  const uint32_t e = w & 0x7f807f80u;
  return ((e & 0xffffu) == 0x7f80u ? 0xffffu : 0u) | ((e >> 16) == 0x7f80u ? 0xffff0000u : 0u);
}

// Scale of the scores as a positive factor and what goes into the queries instead:
// a sign, and a scale of zero as zero times the query (NaN where that is not finite).
struct Scale {
  float c;
  bool neg, zero;
};
__device__ __forceinline__ Scale score_scale(float scale_log2, float2 sc) {
  const float c = scale_log2 * sc.x;
  return c == 0.0f ? Scale{1.0f, false, true} : Scale{fabsf(c), c < 0.0f, false};
}

__device__ __forceinline__ void load_rows(AQ<uint16_t> &q, const uint16_t *p, bool valid, const Scale &sc) {
  const int h = (threadIdx.x >> 5) & 1;
  const uint32_t flip = sc.neg ? 0x80008000u : 0u;
#pragma unroll
  for (int s = 0; s < 8; ++s) {
    uint4 w = make_uint4(0, 0, 0, 0);
    if (valid) w = *reinterpret_cast<const uint4 *>(p + 16 * s + 8 * h);
    if (sc.zero) w = make_uint4(nonfinite2(w.x), nonfinite2(w.y), nonfinite2(w.z), nonfinite2(w.w));  // all bits: NaN
    q.f[s] = __builtin_bit_cast(abf16x8, make_uint4(w.x ^ flip, w.y ^ flip, w.z ^ flip, w.w ^ flip));
  }
}
__device__ __forceinline__ void load_rows(AQ<float> &q, const float *p, bool valid, const Scale &sc) {
  const int h = (threadIdx.x >> 5) & 1;
  const float f = sc.zero ? 0.0f : sc.neg ? -1.0f : 1.0f;
#pragma unroll
  for (int s = 0; s < 16; ++s) {
    float4 w = make_float4(0, 0, 0, 0);
    if (valid) w = *reinterpret_cast<const float4 *>(p + 8 * s + 4 * h);
    q.f[s] = make_float4(w.x * f, w.y * f, w.z * f, w.w * f);
  }
}

// Raw scores (before the scale) of the tile's NB blocks of 32 keys.
template <int NB>
__device__ __forceinline__ void score_tile(af32x16 (&s)[NB], const AQ<uint16_t> &q, const char *K, uint8_t) {
  const int lane = threadIdx.x & 63, r = lane & 31, h = lane >> 5;
  const char *row = K + r * lds_row<uint8_t>() + 8 * h;
  const int x = (r >> 1) & 7;
#pragma unroll
  for (int t = 0; t < NB; ++t)
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const Chunk<uint8_t> k{*reinterpret_cast<const uint2 *>(row + 32 * t * lds_row<uint8_t>() + ((i ^ x) << 4))};
      s[t] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(abf16x8, k.to_bf16()), q.f[i],
                                                     i ? s[t] : af32x16{}, 0, 0, 0);
    }
}
template <int NB>
__device__ __forceinline__ void score_tile(af32x16 (&s)[NB], const AQ<uint16_t> &q, const char *K, uint16_t) {
  const int lane = threadIdx.x & 63, r = lane & 31, h = lane >> 5;
  const char *row = K + r * lds_row<uint16_t>();
  const int x = h ^ (r & 15);
#pragma unroll
  for (int t = 0; t < NB; ++t)
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const abf16x8 k = *reinterpret_cast<const abf16x8 *>(row + 32 * t * lds_row<uint16_t>() + (((2 * i) ^ x) << 4));
      s[t] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(k, q.f[i], i ? s[t] : af32x16{}, 0, 0, 0);
    }
}
template <int NB>
__device__ __forceinline__ void score_tile(af32x16 (&s)[NB], const AQ<float> &q, const char *K, float) {
  const int lane = threadIdx.x & 63, r = lane & 31, h = lane >> 5;
  const char *row = K + r * lds_row<float>();
  const int x = h ^ (r & 15);
#pragma unroll
  for (int t = 0; t < NB; ++t)
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      const float4 k = *reinterpret_cast<const float4 *>(row + 32 * t * lds_row<float>() + (((2 * i) ^ x) << 4));
      af32x16 y = i ? s[t] : af32x16{};
      y = __builtin_amdgcn_mfma_f32_32x32x2f32(k.x, q.f[i].x, y, 0, 0, 0);
      y = __builtin_amdgcn_mfma_f32_32x32x2f32(k.y, q.f[i].y, y, 0, 0, 0);
      y = __builtin_amdgcn_mfma_f32_32x32x2f32(k.z, q.f[i].z, y, 0, 0, 0);
      s[t] = __builtin_amdgcn_mfma_f32_32x32x2f32(k.w, q.f[i].w, y, 0, 0, 0);
    }
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

// 32-bit values as an operand: feature 32 n + l % 32 of the key of accumulator i.
__device__ __forceinline__ float value32(const char *V, int t, int n, int i) {
  const int lane = threadIdx.x & 63, d = lane & 31, h = lane >> 5;
  const char *col = V + (32 * t + 4 * h) * lds_row<float>() + (((8 * n + (d >> 2)) ^ (h << 3)) << 4) + (d & 3) * 4;
  return *reinterpret_cast<const float *>(col + (8 * (i >> 2) + (i & 3)) * lds_row<float>());
}

// The weights over NB blocks of keys, as operands.  The matrix instruction that
// takes bfloat16 values takes bfloat16 weights, rounded by at most 2^-8 of a weight
// (nearest even; their sum keeps 32 bits).  FINE: in two parts, off by 2^-14: what
// the first leaves is a second operand.  The first lies half a step to one and a
// half below the weight, so that both are positive: an infinite value is infinite
// times either.  Few rows wait for memory and take it (us, one part / two: one window
// of 1024 keys 11.2 / 11.6, 64 of 4096 169.0 / 169.1, 16 in FP8 21.5 / 22.2, drafted
// tokens 71.3 / 70.3), full tiles wait for the products and do not (512 tokens at 32k
// 317 / 424, an 8k prompt 597 / 797, a window of 1024 over 2k tokens 53.9 / 67.1).
template <typename L, int NB, bool FINE>
struct Weights {
  abf16x8 f[2 * NB], rest[FINE ? 2 * NB : 1];
};
template <int NB, bool FINE>
struct Weights<float, NB, FINE> {
  af32x16 f[NB];
};

// O^T += V^T P^T over the tile at V (rows of type L).
template <typename L, int NB, bool FINE>
__device__ __forceinline__ void add_values(RowState &st, const Weights<QE<L>, NB, FINE> &p, const char *V, L) {
  const int h = (threadIdx.x >> 5) & 1;
  if constexpr (sizeof(L) <= 2) {
#pragma unroll
    for (int b = 0; b < 2 * NB; ++b) {
      abf16x8 w[4];
#pragma unroll
      for (int n = 0; n < 4; ++n) {
        w[n] = __builtin_bit_cast(abf16x8, value_operand(V, 16 * b + 4 * h, n, L{}));
        st.o[n] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(w[n], p.f[b], st.o[n], 0, 0, 0);
      }
      if constexpr (FINE)
#pragma unroll
        for (int n = 0; n < 4; ++n)
          st.o[n] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(w[n], p.rest[b], st.o[n], 0, 0, 0);
    }
  } else {
#pragma unroll
    for (int t = 0; t < NB; ++t)
#pragma unroll
      for (int n = 0; n < 4; ++n)
#pragma unroll
        for (int i = 0; i < 16; ++i)
          st.o[n] = __builtin_amdgcn_mfma_f32_32x32x2f32(value32(V, t, n, i), p.f[t][i], st.o[n], 0, 0, 0);
  }
}

// Non-finite values stand apart: a key that some rows of a tile do not see must
// not reach them as 0 * inf.  In a tile that not all rows see whole, zeros take
// their place in LDS (clean_values), and add_nonfinite gives them at the end to
// the rows that do see them.
//
// Whether words w hold a non-finite element, and the words with those zeroed.
__device__ __forceinline__ bool clean_words(uint4 &w, uint16_t) {
  const uint4 f = make_uint4(nonfinite2(w.x), nonfinite2(w.y), nonfinite2(w.z), nonfinite2(w.w));
  w = make_uint4(w.x & ~f.x, w.y & ~f.y, w.z & ~f.z, w.w & ~f.w);
  return (f.x | f.y | f.z | f.w) != 0;
}
__device__ __forceinline__ bool clean_words(uint4 &w, float) {
  bool bad = false;
  auto one = [&](uint32_t &x) {
    const bool b = (x & 0x7f800000u) == 0x7f800000u;
    bad |= b;
    x = b ? 0u : x;
  };
  one(w.x), one(w.y), one(w.z), one(w.w);
  return bad;
}
__device__ __forceinline__ bool clean_words(uint4 &w, uint8_t) {  // E4M3: NaN is the only one
  bool bad = false;
  auto one = [&](uint32_t &x) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const uint32_t m = 0x7fu << (8 * i);
      if ((x & m) == m) {
        bad = true;
        x &= ~(0xffu << (8 * i));
      }
    }
  };
  one(w.x), one(w.y), one(w.z), one(w.w);
  return bad;
}
// Over BYTES of V by a team of TEAM lanes; whether there were any.
template <typename L, int BYTES, int TEAM>
__device__ __forceinline__ bool clean_values(char *V, int tl) {
  uint4 w[BYTES / 16 / TEAM];
  bool bad = false;
#pragma unroll
  for (int i = 0; i < BYTES / 16 / TEAM; ++i) w[i] = *reinterpret_cast<const uint4 *>(V + (i * TEAM + tl) * 16);
#pragma unroll
  for (int i = 0; i < BYTES / 16 / TEAM; ++i)
    if (clean_words(w[i], L{})) {
      *reinterpret_cast<uint4 *>(V + (i * TEAM + tl) * 16) = w[i];
      bad = true;
    }
  return bad;
}

// The online softmax, in three parts.  The reference m of a row moves only when
// a score passes it by more than kLag in log2 units, so that the output is
// rescaled in the first tiles only instead of whenever one of 32 rows finds a
// new maximum.  Weights are taken under m + kLag: none is above 1 (2^8 times a
// large value would overflow) and the largest is at least 2^-8, which costs 32-bit
// sums and the weights' rounding nothing.
constexpr float kLag = 8.0f;
__device__ __forceinline__ float reference(const RowState &st, float c) { return fmaf(st.m, c, kLag); }
template <int NB>
__device__ __forceinline__ void hide(af32x16 (&s)[NB], int v0, const RowSight &rs) {
  const int h = (threadIdx.x >> 5) & 1;
#pragma unroll
  for (int t = 0; t < NB; ++t)
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      const int v = v0 + 32 * t + 8 * (i >> 2) + 4 * h + (i & 3);
      if (!(v < rs.hi && (v >= rs.lo || v < rs.sv))) s[t][i] = -kInf;
    }
}
template <int NB>
__device__ __forceinline__ float row_max(const af32x16 (&s)[NB]) {
  float tm = -kInf;
#pragma unroll
  for (int t = 0; t < NB; ++t)
#pragma unroll
    for (int i = 0; i < 16; ++i) tm = fmaxf(tm, s[t][i]);
  return xor32_max(tm);
}
// The factor that the output and the sum so far take (1 if the reference stays;
// no score yet: m is -inf, passed by any score but -inf).
__device__ __forceinline__ float move_reference(RowState &st, float tm, float c) {
  const bool move = tm * c > reference(st, c);
  const float f = move ? fast_exp2((st.m - tm) * c) : 1.0f;
  st.m = move ? tm : st.m;
  st.l *= f;
  return f;
}
__device__ __forceinline__ void rescale(RowState &st, float f) {
#pragma unroll
  for (int n = 0; n < 4; ++n)
#pragma unroll
    for (int i = 0; i < 16; ++i) st.o[n][i] *= f;
}
// Scores become weights, and their sum the row's.
template <int NB>
__device__ __forceinline__ void weigh(RowState &st, af32x16 (&s)[NB], float c) {
  const float mc = st.m == -kInf ? 0.0f : reference(st, c);  // nothing visible yet: every weight is 0
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
template <int NB, bool FINE>
__device__ __forceinline__ void pack(Weights<uint16_t, NB, FINE> &w, const af32x16 (&s)[NB]) {
#pragma unroll
  for (int b = 0; b < 2 * NB; ++b)
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const float x = s[b / 2][8 * (b & 1) + i];
      if constexpr (FINE) {
        const uint32_t part = __builtin_elementwise_sub_sat(__float_as_uint(x), 0x8000u) & 0xffff0000u;
        w.f[b][i] = __builtin_bit_cast(__bf16, (uint16_t)(part >> 16));
        w.rest[b][i] = (__bf16)(x - __uint_as_float(part));
      } else {
        w.f[b][i] = (__bf16)x;
      }
    }
}
template <int NB, bool FINE>
__device__ __forceinline__ void pack(Weights<float, NB, FINE> &w, const af32x16 (&s)[NB]) {
#pragma unroll
  for (int t = 0; t < NB; ++t) w.f[t] = s[t];
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

// ---------------------------------------------------------------------------
// Tiles
// ---------------------------------------------------------------------------
// A workgroup's tile and key range.  Blocks are numbered KV head fastest (with
// 8 KV heads each XCD works on one head's keys), then split, then tile from
// the last to the first: in a chunk the later tiles see more keys.  The grid has
// the tiles to expect; where a batch may have more (MORE: rows enough for chunks
// longer than max_tokens says), each workgroup goes on with the others in turn, a
// tile at a time and unsplit, so that only the tiles to expect need room for
// partial results: the (split, tile) workgroups of a KV head share out the rest.
// A grid for all that there may be would spend its time on empty workgroups: one
// token with 2000 padding rows over 2k keys 13.7 us, 91.7 with a workgroup for every
// tile that the rows could make.  (Without the loop 11.1 us for 12.0 in one user's
// window.)
struct Work {
  TileAt at;
  int kvh, rows, p_lo;     // rows: valid ones; p_lo: position of the tile's first token
  int t, T;                // split, of how many
  int v_begin, v_end;
  KeyMap km;
  int64_t group;           // number of the tile and KV head
  int64_t out_row;         // first row of the split's partial results
  bool any;                // the tile exists
};
__device__ __forceinline__ Work find_work(const AttendArgs &a, int rows_per_tile, int turn) {
  Work w;
  const uint32_t id = blockIdx.x, y = id / (uint32_t)a.Hkv, z = y / (uint32_t)a.T;
  w.kvh = (int)(id - y * a.Hkv);
  w.t = (int)(y - z * a.T);
  w.T = a.T;
  int64_t x = a.grid_tiles - 1 - (int64_t)z;
  if (turn) {
    x += ((int64_t)(turn - 1) * a.T + w.t + 1) * a.grid_tiles;
    w.t = 0;
    w.T = 1;
  }
  w.any = x < a.tiles;
  if (!w.any) return w;
  const TileAt at = find_tile(a.ch, x, a.tile_tokens);
  auto uniform = [](int i) { return __builtin_amdgcn_readfirstlane(i); };
  w.at = TileAt{uniform(at.b), uniform(at.first), uniform(at.count), uniform(at.i0)};
  w.any = w.at.b < a.ch.B;
  w.group = x * a.Hkv + w.kvh;
  w.out_row = (w.group * w.T + w.t) * rows_per_tile;  // (unused where a tile is not split)
  if (!w.any) return w;
  const int L = uniform(seq_len(a.kv, w.at.b)), n = min(a.tile_tokens, w.at.count - w.at.i0);
  w.rows = n << a.g_log2;
  w.p_lo = L - w.at.count + w.at.i0;
  // (a chunk longer than its context: tokens before position 0 see nothing)
  w.km = w.p_lo + n - 1 < 0 ? KeyMap{0, 0, 0, 0, 0} : key_map(max(w.p_lo, 0), w.p_lo + n - 1, a.window, a.sinks);
  const int len = ((w.km.nv + w.T - 1) / w.T + a.step - 1) / a.step * a.step;
  w.v_begin = min(w.t * len, w.km.nv);
  w.v_end = min(w.v_begin + len, w.km.nv);
  return w;
}

__device__ __forceinline__ RowSight tile_sight(const AttendArgs &a, const Work &w, int r) {
  const int p = w.p_lo + (r >> a.g_log2);
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
  const int rr = min(r, w.rows - 1), i = rr >> a.g_log2;
  x.at = ((int64_t)(w.at.first + w.at.i0 + i) * a.Hq + (w.kvh << a.g_log2) + rr - (i << a.g_log2)) * kHeadDim;
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

// A row's reference as waves and splits give it to the join beside their sum l, in
// log2 units.  -inf: no score here, neither the sum nor the outputs count.  A NaN
// score shows in no maximum; the sum that it makes NaN stands above every other,
// or the join would leave it out beside larger scores, or as a split without any.
__device__ __forceinline__ float join_reference(const RowState &st, float l, float c) {
  return l != l ? kInf : st.m == -kInf ? -kInf : reference(st, c);
}
// A split's weight under the maximum of all; negative: it has none and is left out.
// (One that rounds to zero is not left out: zero times its outputs is NaN where
// they are not finite.)
__device__ __forceinline__ float join_weight(float split_max, float top) {
  return split_max == -kInf ? -1.0f : fast_exp2(split_max - top);
}

// Adds the non-finite values of keys [lo, hi) that a row sees to N of its
// features from d on: add(i, value).  (Adding one that the sum has already changes
// nothing: they absorb.)  A slow loop for a cache that holds such values.
__device__ __forceinline__ void add_to(uint16_t *p, float x) { *p = (uint16_t)pack2(to_f32(*p) + x, 0.0f); }
__device__ __forceinline__ void add_to(float *p, float x) { *p += x; }
__device__ __forceinline__ float cache_value(uint16_t x) { return to_f32(x); }
__device__ __forceinline__ float cache_value(float x) { return x; }
__device__ __forceinline__ float cache_value(uint8_t x) { return (x & 0x7f) == 0x7f ? __builtin_nanf("") : 0.0f; }
template <typename E, bool PAGED, int N, typename F>
__device__ __forceinline__ void add_nonfinite(const AttendArgs &a, const Work &w, const RowSight &see, int lo, int hi,
                                              int d, F &&add) {
#pragma unroll 1
  for (int v = lo; v < min(hi, w.v_end); ++v) {
    if (!(v < see.hi && (v >= see.lo || v < see.sv))) continue;
    const E *p = static_cast<const E *>(a.kv.v) + row_offset<PAGED>(a.kv, w.at.b, w.kvh, w.km.pos(v)) + d;
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const float x = cache_value(p[i]);
      if (!(fabsf(x) < kInf)) add(i, x);
    }
  }
}

// Many rows: 128, 32 per wave; K and V tiles of KEYS keys shared by the four
// waves, two of each in LDS.
//
// What bounds it: a wave's 64 keys x 32 rows take the matrix cores 1024 cycles, the
// vector unit about 900 (an exponential is 16 of them) and 48 operand reads from
// LDS; two waves per SIMD overlap these in part.  An 8k prompt runs at 0.92 to 0.98
// PFLOP/s, 558 to 597 us from card to card, at the 2.0 GHz that this load holds (left
// out, the operand reads give 30 % of the time, the softmax 20, the copies 17).
//
// Measured at a time of 600 us and not taken: 64 rows per wave at one wave per SIMD, the
// values of a tile added while the next one's scores become weights (1049 us: the
// outputs travel between the register files); 64 rows and half of the keys
// per wave (837 us, registers spill); 32 keys per tile at three waves per SIMD
// (630); eight waves on 256 rows (621); wave priorities and instruction orders
// (590 to 640).
template <typename E>
constexpr int many_keys() {
  return sizeof(E) == 4 ? 32 : 64;
}
template <typename E, bool PAGED>
__device__ __forceinline__ void many_tile(const AttendArgs &a, const Work &w, char *lds) {  // lds: K0, K1, V0, V1
  using L = LE<E>;
  constexpr int KEYS = many_keys<E>(), NB = KEYS / 32, TB = KEYS * lds_row<E>();
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), h = lane >> 5;
  const int r = 32 * wave + (lane & 31);
  const Row row = tile_row(a, w, r);
  const float2 sc = kv_scales<E>(a.kv, w.at.b, w.kvh, a.Hkv);
  const Scale scale = score_scale(a.scale_log2, sc);
  AQ<L> q;
  load_rows(q, static_cast<const L *>(a.q) + row.at, row.valid, scale);
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

  // Two tiles of K and V in turn and one barrier per tile: past it, every wave's
  // copies of this tile are here and every wave is done with the other one,
  // which the next tile's copies then fill.
  constexpr int R = KEYS / 4;
  RowCopies<E, PAGED, R> rc(a.kv, w.km, w.at.b, w.kvh, w.v_end, R * wave);
  auto copy = [&](int v, int turn) {
    rc.seek(v + R * wave);
    rc.template copy<false, false>(a.kv.k, lds + turn * TB);
    rc.template copy<true, false>(a.kv.v, lds + (2 + turn) * TB);
  };
  if (w.v_begin < w.v_end) copy(w.v_begin, 0);
  int turn = 0, bad_lo = INT32_MAX, bad_hi = 0;  // (bad: the keys that clean_values found something in)
#pragma unroll 1
  for (int v0 = w.v_begin; v0 < w.v_end; v0 += KEYS) {
    wait_copies<0>();
    __syncthreads();
    if (v0 + KEYS < w.v_end) copy(v0 + KEYS, turn ^ 1);
    const char *K = lds + turn * TB;
    char *V = lds + (2 + turn) * TB;
    const bool whole = v0 + KEYS <= all_hi && (v0 >= last.lo || v0 + KEYS <= last.sv);
    if (!whole && __syncthreads_or(clean_values<E, TB, kThreads>(V, tid))) {
      bad_lo = min(bad_lo, v0);
      bad_hi = v0 + KEYS;
    }
    af32x16 s[NB];
    score_tile(s, q, K, E{});
    if (!whole) hide(s, v0, see);
    const float f = move_reference(st, row_max(s), scale.c);
    if (__any(f != 1.0f)) rescale(st, f);
    weigh(st, s, scale.c);
    Weights<L, NB, false> p;
    pack(p, s);
    add_values(st, p, V, E{});
    turn ^= 1;
  }

  const float l = xor32_sum(st.l);
  if (!row.valid) return;
  const int64_t at = w.out_row + r;
  float f = 1.0f;
  if (w.T == 1) {
    f = l > 0.0f || l != l ? sc.y / l : 0.0f;  // a row that sees nothing is zero
  } else {
    const float m = join_reference(st, l, scale.c);
    if (h == 0) a.stat[at] = make_float2(m, l);
    if (m == -kInf) return;  // (nothing seen here: the statistics say so)
  }
#pragma unroll
  for (int n = 0; n < 4; ++n)
#pragma unroll
    for (int g = 0; g < 4; ++g) {
      const float4 x = make_float4(st.o[n][4 * g] * f, st.o[n][4 * g + 1] * f, st.o[n][4 * g + 2] * f, st.o[n][4 * g + 3] * f);
      const int d = 32 * n + 8 * g + 4 * h;
      if (w.T == 1) store4(static_cast<L *>(a.out) + row.at + d, x);
      else *reinterpret_cast<float4 *>(a.part + at * kHeadDim + d) = x;
    }
  if (bad_lo < bad_hi) {
#pragma unroll 1
    for (int d = 4 * h; d < kHeadDim; d += 8) {
      L *out = static_cast<L *>(a.out) + row.at + d;
      float *part = a.part + at * kHeadDim + d;
      add_nonfinite<E, PAGED, 4>(a, w, see, bad_lo, bad_hi, d, [&](int i, float x) {
        if (w.T == 1) add_to(out + i, x);
        else add_to(part + i, x);
      });
    }
  }
}

template <typename E, bool PAGED, bool MORE>
__global__ __launch_bounds__(kThreads) __attribute__((amdgpu_waves_per_eu(2))) void k_attend_many(AttendArgs a) {
  extern __shared__ __attribute__((aligned(16))) char lds[];
  for (int turn = 0; MORE || turn == 0; ++turn) {
    const Work w = find_work(a, kManyRows, turn);
    if (!w.any) return;
    if (turn) __syncthreads();  // every wave is done with the last tile's memory
    many_tile<E, PAGED>(a, w, lds);
  }
}

// Few rows: up to 32, the same for all four waves, which share out the keys:
// each wave streams its own run of them through its own two slots of LDS, the
// keys' and the values' in turn, with no barrier inside the stream, and keeps
// its own softmax; they join their results through LDS at the end.
constexpr int kFewKeys = 32;  // keys per slot (FP8, 64 instead: 22.7 us for 20.7 in 16 windows of 2048 keys, level at 32k)
template <typename E>
constexpr int few_wgs() {  // workgroups per CU that the slots leave room for
  return sizeof(E) == 4 ? 1 : 2;
}
template <typename E, bool PAGED>
__device__ __forceinline__ void few_tile(const AttendArgs &a, const Work &w, char *lds) {
  using L = LE<E>;
  constexpr int KEYS = kFewKeys, NB = KEYS / 32, TB = KEYS * lds_row<E>();
  __shared__ float wm[4][kFewRows], wl[4][kFewRows];
  __shared__ int bad[4][2];  // the keys that clean_values found something in
  __shared__ int rank;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int r = lane & 31, h = lane >> 5;
  char *K = lds + wave * 2 * TB, *V = K + TB;
  // the wave's keys: a quarter of the split's, in whole tiles
  const int quarter = ((w.v_end - w.v_begin + 3) / 4 + KEYS - 1) & ~(KEYS - 1);
  const int begin = min(w.v_begin + wave * quarter, w.v_end), end = min(begin + quarter, w.v_end);
  RowCopies<E, PAGED, KEYS> rc(a.kv, w.km, w.at.b, w.kvh, end, 0);
  constexpr int NL = decltype(rc)::NL;
  if (begin < end) {
    rc.seek(begin);
    rc.template copy<false, true>(a.kv.k, K);
    rc.template copy<true, true>(a.kv.v, V);
  }
  const Row row = tile_row(a, w, r);
  const float2 sc = kv_scales<E>(a.kv, w.at.b, w.kvh, a.Hkv);
  const Scale scale = score_scale(a.scale_log2, sc);
  AQ<L> q;
  load_rows(q, static_cast<const L *>(a.q) + row.at, row.valid, scale);
  const RowSight first = tile_sight(a, w, 0), last = tile_sight(a, w, w.rows - 1);
  RowSight see = row.see;
  see.hi = min(see.hi, end);
  const int all_hi = min(first.hi, end);

  RowState st;
  st.m = -kInf;
  st.l = 0.0f;
#pragma unroll
  for (int n = 0; n < 4; ++n) st.o[n] = af32x16{};
  int bad_lo = INT32_MAX, bad_hi = 0;
  for (int v0 = begin; v0 < end; v0 += KEYS) {
    const bool more = v0 + KEYS < end;
    wait_copies<NL>();
    af32x16 s[NB];
    score_tile(s, q, K, E{});
    wait_reads();
    if (more) {
      rc.seek(v0 + KEYS);
      rc.template copy<false, true>(a.kv.k, K);
    }
    const bool whole = v0 + KEYS <= all_hi && (v0 >= last.lo || v0 + KEYS <= last.sv);
    if (!whole) hide(s, v0, see);
    const float f = move_reference(st, row_max(s), scale.c);
    if (__any(f != 1.0f)) rescale(st, f);
    weigh(st, s, scale.c);
    Weights<L, NB, true> p;
    pack(p, s);
    if (more) wait_copies<NL>();
    else wait_copies<0>();
    if (!whole && __any(clean_values<E, TB, 64>(V, lane))) {
      bad_lo = min(bad_lo, v0);
      bad_hi = v0 + KEYS;
    }
    add_values(st, p, V, E{});
    wait_reads();
    if (more) rc.template copy<true, true>(a.kv.v, V);
  }

  // join the waves: out = sum_w 2^(m_w - m) O_w / sum_w 2^(m_w - m) l_w
  const float l = xor32_sum(st.l);
  if (h == 0) {
    wm[wave][r] = join_reference(st, l, scale.c);
    wl[wave][r] = l;
  }
  if (lane == 0) {
    bad[wave][0] = bad_lo;
    bad[wave][1] = bad_hi;
  }
  __syncthreads();  // (also: every wave is done with its tile's memory)
  float m = -kInf;
#pragma unroll
  for (int i = 0; i < 4; ++i) m = fmaxf(m, wm[i][r]);
  const float f = st.m == -kInf ? 0.0f : fast_exp2(reference(st, scale.c) - m);
  float4 *part = reinterpret_cast<float4 *>(lds);  // [wave][32 quads of features][32 rows]
  if (r < w.rows)
#pragma unroll
    for (int n = 0; n < 4; ++n)
#pragma unroll
      for (int g = 0; g < 4; ++g)
        part[(wave * 32 + 8 * n + 2 * g + h) * 32 + r] = make_float4(st.o[n][4 * g] * f, st.o[n][4 * g + 1] * f,
                                                                     st.o[n][4 * g + 2] * f, st.o[n][4 * g + 3] * f);
  __syncthreads();
  const int r2 = tid & 31, d0 = tid >> 5;  // row, and its features 16 d0 .. + 15
  if (r2 < w.rows) {
    float mm = -kInf, ll = 0.0f;
#pragma unroll
    for (int i = 0; i < 4; ++i) mm = fmaxf(mm, wm[i][r2]);
#pragma unroll
    for (int i = 0; i < 4; ++i) ll += wm[i][r2] == -kInf ? 0.0f : fast_exp2(wm[i][r2] - mm) * wl[i][r2];
    const float g = w.T > 1 ? 1.0f : ll > 0.0f || ll != ll ? sc.y / ll : 0.0f;
    float x[16];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      float4 s = make_float4(0, 0, 0, 0);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float4 y = part[(i * 32 + 4 * d0 + k) * 32 + r2];
        s = make_float4(s.x + y.x, s.y + y.y, s.z + y.z, s.w + y.w);
      }
      x[4 * k] = s.x * g, x[4 * k + 1] = s.y * g, x[4 * k + 2] = s.z * g, x[4 * k + 3] = s.w * g;
    }
    const Row row2 = tile_row(a, w, r2);
#pragma unroll 1
    for (int i = 0; i < 4; ++i)
      if (bad[i][0] < bad[i][1])
        add_nonfinite<E, PAGED, 16>(a, w, row2.see, bad[i][0], bad[i][1], 16 * d0, [&](int j, float y) { x[j] += y; });
    const int64_t at = w.out_row + r2;
    if (w.T == 1) {
#pragma unroll
      for (int k = 0; k < 4; ++k)
        store4(static_cast<L *>(a.out) + row2.at + 16 * d0 + 4 * k,
               make_float4(x[4 * k], x[4 * k + 1], x[4 * k + 2], x[4 * k + 3]));
    } else if (!a.sync) {
      if (d0 == 0) a.stat[at] = make_float2(mm, ll);
#pragma unroll
      for (int k = 0; k < 4; ++k)
        *reinterpret_cast<float4 *>(a.part + at * kHeadDim + 16 * d0 + 4 * k) =
            make_float4(x[4 * k], x[4 * k + 1], x[4 * k + 2], x[4 * k + 3]);
    } else {
      if (d0 == 0) st_coherent(a.stat + at, make_float2(mm, ll));
      float2 *to = reinterpret_cast<float2 *>(a.part + at * kHeadDim + 16 * d0);
#pragma unroll
      for (int k = 0; k < 8; ++k) st_coherent(to + k, make_float2(x[2 * k], x[2 * k + 1]));
    }
  }
  if (w.T == 1 || !a.sync) return;

  // The tile's last split joins them all, a wave per row: every split has stored
  // its part, coherently, before it counts itself; the last one sees T - 1 before
  // it and leaves the counter at zero.  Nobody waits.
  unsigned long long *count = a.sync + w.group * (kSyncStride / 2) + kAttendCounter;
  wait_stores();
  __syncthreads();
  if (tid == 0) {
    rank = (int)__hip_atomic_fetch_add(count, 1ull, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    if (rank == w.T - 1) __hip_atomic_store(count, 0ull, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  }
  __syncthreads();
  if (rank != w.T - 1) return;
  for (int r3 = wave; r3 < w.rows; r3 += 4) {
    const int64_t base = w.out_row - (int64_t)w.t * kFewRows + r3;  // split 0's
    const float2 s = lane < w.T ? ld_coherent(a.stat + base + (int64_t)lane * kFewRows) : make_float2(-kInf, 0.0f);
    const float u = join_weight(s.x, wave_max(s.x));
    const float total = wave_sum(u < 0.0f ? 0.0f : u * s.y);
    float2 o = make_float2(0, 0);
#pragma unroll 1
    for (int t = 0; t < w.T; t += 8) {
      float2 y[8];
#pragma unroll
      for (int j = 0; j < 8; ++j)
        y[j] = ld_coherent(reinterpret_cast<const float2 *>(a.part + (base + (int64_t)min(t + j, w.T - 1) * kFewRows) * kHeadDim) + lane);
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const float uj = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(u), min(t + j, 63)));
        if (t + j < w.T && !(uj < 0.0f)) o = make_float2(fmaf(uj, y[j].x, o.x), fmaf(uj, y[j].y, o.y));
      }
    }
    const float g = total > 0.0f || total != total ? sc.y / total : 0.0f;
    L *out = static_cast<L *>(a.out) + tile_row(a, w, r3).at;
    if constexpr (sizeof(L) == 2) reinterpret_cast<uint32_t *>(out)[lane] = pack2(o.x * g, o.y * g);
    else reinterpret_cast<float2 *>(out)[lane] = make_float2(o.x * g, o.y * g);
  }
}

template <typename E, bool PAGED, bool MORE>
__global__ __launch_bounds__(kThreads) __attribute__((amdgpu_waves_per_eu(few_wgs<E>()))) void k_attend_few(AttendArgs a) {
  extern __shared__ __attribute__((aligned(16))) char lds[];
  for (int turn = 0; MORE || turn == 0; ++turn) {
    const Work w = find_work(a, kFewRows, turn);
    if (!w.any) return;
    if (turn) __syncthreads();  // every wave is done with the last tile's memory
    few_tile<E, PAGED>(a, w, lds);
  }
}

// Joins the splits' partial results, a wave per (KV head, row of a grid tile): lane i
// takes split i's statistics (and i + 64's, ..), then the half-waves take the even
// and the odd splits' rows, four features per lane, several rows in flight.
template <typename E, int ROWS>
__global__ __launch_bounds__(kThreads) void k_attend_merge(AttendArgs a) {
  using L = LE<E>;
  constexpr int MS = kMaxSplits / 64;
  const int lane = threadIdx.x & 63, odd = lane >> 5;
  const uint32_t id = blockIdx.x * (kThreads / 64) + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int r = (int)(id % ROWS);
  const uint32_t y = id / ROWS, z = y / (uint32_t)a.Hkv;
  const int kvh = (int)(y - z * a.Hkv);
  const TileAt at = find_tile(a.ch, z, a.tile_tokens);
  if (at.b >= a.ch.B) return;
  const int i = r >> a.g_log2;
  if (i >= min(a.tile_tokens, at.count - at.i0)) return;
  const int64_t base = ((int64_t)z * a.Hkv + kvh) * a.T * ROWS + r;
  float2 s[MS];
  float m = -kInf, l = 0.0f;
#pragma unroll
  for (int k = 0; k < MS; ++k) {
    const int t = 64 * k + lane;
    s[k] = t < a.T ? a.stat[base + (int64_t)t * ROWS] : make_float2(-kInf, 0.0f);
    m = fmaxf(m, s[k].x);
  }
  m = wave_max(m);
#pragma unroll
  for (int k = 0; k < MS; ++k) {
    s[k].x = join_weight(s[k].x, m);
    l += s[k].x < 0.0f ? 0.0f : s[k].x * s[k].y;
  }
  l = wave_sum(l);
  float4 o = make_float4(0, 0, 0, 0);
#pragma unroll
  for (int k = 0; k < MS; ++k) {
#pragma unroll 1
    for (int t = 0; t < min(64, a.T - 64 * k); t += 8) {
      float f[4];
      float4 y[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int tt = t + 2 * j + odd;
        f[j] = __shfl(s[k].x, tt);  // (negative past the last split)
        const int64_t at_row = base + (int64_t)min(64 * k + tt, a.T - 1) * ROWS;
        y[j] = reinterpret_cast<const float4 *>(a.part + at_row * kHeadDim)[lane & 31];
      }
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        if (f[j] < 0.0f) continue;  // (a split without scores may not have written its rows)
        o = make_float4(fmaf(f[j], y[j].x, o.x), fmaf(f[j], y[j].y, o.y), fmaf(f[j], y[j].z, o.z), fmaf(f[j], y[j].w, o.w));
      }
    }
  }
  const float g = l > 0.0f || l != l ? kv_scales<E>(a.kv, at.b, kvh, a.Hkv).y / l : 0.0f;
  o = make_float4(xor32_sum(o.x) * g, xor32_sum(o.y) * g, xor32_sum(o.z) * g, xor32_sum(o.w) * g);
  const int64_t row = (int64_t)(at.first + at.i0 + i) * a.Hq + (kvh << a.g_log2) + r - (i << a.g_log2);
  if (!odd) store4(static_cast<L *>(a.out) + row * kHeadDim + 4 * lane, o);
}

// Few rows: a K and a V slot per wave, and at the end the waves' outputs.  Many: two tiles of K and of V.
template <typename E>
constexpr size_t attend_lds(bool few) {
  const size_t slots = (size_t)4 * 2 * kFewKeys * lds_row<E>(), join = (size_t)4 * kFewRows * kHeadDim * 4;
  return few ? (slots > join ? slots : join) : (size_t)4 * many_keys<E>() * lds_row<E>();
}

template <typename E>
hipError_t launch_attend_e(const AttendPlan &p, const AttendArgs &a, hipStream_t st) {
  const CallTimer tm = call_timer();
  void *params[] = {const_cast<AttendArgs *>(&a)};
  const void *fn = nullptr;
  auto pick = [&](auto paged, auto more) {
    constexpr bool P = decltype(paged)::value, M = decltype(more)::value;
    fn = p.few ? (const void *)k_attend_few<E, P, M> : (const void *)k_attend_many<E, P, M>;
  };
  const bool more = p.grid_tiles < p.tiles;
  if (a.kv.bt) more ? pick(std::true_type{}, std::true_type{}) : pick(std::true_type{}, std::false_type{});
  else more ? pick(std::false_type{}, std::true_type{}) : pick(std::false_type{}, std::false_type{});
  hipError_t e = hipExtLaunchKernel(fn, dim3((unsigned)(p.grid_tiles * p.Hkv * p.T)),
                                    dim3(kThreads), params,
                                    attend_lds<E>(p.few), st, tm.start, p.T > 1 && !p.join ? nullptr : tm.stop, 0);
  if (e != hipSuccess || p.T == 1 || p.join) return e;
  const void *mf = p.few ? (const void *)k_attend_merge<E, kFewRows> : (const void *)k_attend_merge<E, kManyRows>;
  return hipExtLaunchKernel(mf, dim3((unsigned)(p.grid_tiles * p.Hkv * p.rows / (kThreads / 64))), dim3(kThreads), params,
                            0, st, nullptr, tm.stop, 0);
}

}  // namespace santa
