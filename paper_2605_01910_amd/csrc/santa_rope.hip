// santa_rope.hip -- rotary positions of a batch of new tokens, fused with the
// store of their keys and values into the KV cache (santa_rope_append), and
// the host side of the rotary plan (santa_rope_init).
#include "santa_chunk.h"
#include "santa_device.h"
#include "santa_kernels.h"

namespace santa {

namespace {

// 8 consecutive features as float32, from and to rows of type E.
__device__ __forceinline__ void load8(const uint16_t *p, float (&f)[8]) {
  Chunk<uint16_t>::load(p).to_float(f);
}
__device__ __forceinline__ void load8(const float *p, float (&f)[8]) { Chunk<float>::load(p).to_float(f); }

__device__ __forceinline__ uint32_t pack_bf16(float a, float b) {
  typedef __bf16 bf2 __attribute__((ext_vector_type(2)));
  const bf2 v = {(__bf16)a, (__bf16)b};  // round to nearest even
  return __builtin_bit_cast(uint32_t, v);
}
__device__ __forceinline__ void store8(uint16_t *p, const float (&f)[8]) {
  *reinterpret_cast<uint4 *>(p) = make_uint4(pack_bf16(f[0], f[1]), pack_bf16(f[2], f[3]),
                                             pack_bf16(f[4], f[5]), pack_bf16(f[6], f[7]));
}
__device__ __forceinline__ void store8(float *p, const float (&f)[8]) {
  reinterpret_cast<float4 *>(p)[0] = make_float4(f[0], f[1], f[2], f[3]);
  reinterpret_cast<float4 *>(p)[1] = make_float4(f[4], f[5], f[6], f[7]);
}
// E4M3 codes, nearest even, saturated at the largest finite value; NaN stays NaN.
__device__ __forceinline__ float sat8(float x) { return x < -448.0f ? -448.0f : (x > 448.0f ? 448.0f : x); }
__device__ __forceinline__ void store8(uint8_t *p, const float (&f)[8]) {
  int lo = 0, hi = 0;
  lo = __builtin_amdgcn_cvt_pk_fp8_f32(sat8(f[0]), sat8(f[1]), lo, false);
  lo = __builtin_amdgcn_cvt_pk_fp8_f32(sat8(f[2]), sat8(f[3]), lo, true);
  hi = __builtin_amdgcn_cvt_pk_fp8_f32(sat8(f[4]), sat8(f[5]), hi, false);
  hi = __builtin_amdgcn_cvt_pk_fp8_f32(sat8(f[6]), sat8(f[7]), hi, true);
  *reinterpret_cast<uint2 *>(p) = make_uint2((unsigned)lo, (unsigned)hi);
}

// cos and sin of position * frequency, times the gain.  The product is taken
// in whole 2^-64ths of a turn, where leaving out whole turns is the wrap of
// the multiplication: what grows with the position is only the plan's error of a
// few 2^-64ths.
__device__ __forceinline__ float2 turn(int64_t pos, uint64_t step, float gain) {
  const uint64_t phase = (uint64_t)pos * step;
  const float half_turns = (float)(int32_t)(phase >> 32) * 0x1p-31f;  // in [-1, 1]
  float s, c;
  sincospif(half_turns, &s, &c);
  return make_float2(c * gain, s * gain);
}

}  // namespace

// Bound by HBM on prompts (q, k and v read once, their results written once: 16k
// tokens of 48 heads in 77 us, 5.2 TB/s, a copy's rate), by the launch and the
// chain of table, length and row loads on single tokens (3.7 us).
//
// One workgroup rotates and stores TT tokens.  Wave w finds token w's sequence
// and cache row and takes the token's 64 angles, one per lane, for all its
// heads; then all threads pass over the (token, head, unit) items, a unit being
// 16 features that hold whole pairs: 8 u .. + 7 of both halves of the rotary
// part (or 16 u .. + 15 of it, interleaved pairs).
// E: cache element, Q: row element.
template <typename Q, typename E, int TT>
__global__ __launch_bounds__(kThreads) void k_rope_append(RopeArgs a) {
  __shared__ float2 cs[TT][kHeadDim / 2];
  __shared__ int64_t row_off[TT];
  __shared__ int seq[TT], stored[TT];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int t0 = blockIdx.x * TT;
  if (wave < TT) {
    const int t = t0 + wave;
    const TokenAt at = t < a.ch.tokens ? find_token(a.ch, t) : TokenAt{a.ch.B, 0, 0};
    int pos = 0, ok = 0;
    int64_t off = 0;
    if (at.b < a.ch.B) {
      int L = a.kv.ctx ? a.kv.ctx[at.b] : a.kv.n_k;
      L = L < 0 ? 0 : (L > a.kv.n_k ? a.kv.n_k : L);
      pos = L - at.count + (t - at.first);
      ok = pos >= 0 && pos < a.kv.n_k;
      if (ok) {
        if (a.kv.bt) {
          const int page = a.kv.bt[(int64_t)at.b * a.kv.max_pages + (pos >> a.kv.ps_log2)];
          ok = page >= 0;
          off = (int64_t)page * a.kv.sb + (int64_t)(pos & ((1 << a.kv.ps_log2) - 1)) * a.kv.sn;
        } else {
          off = (int64_t)at.b * a.kv.sb + (int64_t)pos * a.kv.sn;
        }
      }
      if (lane < a.rotary / 2)
        cs[wave][lane] = turn(a.positions ? (int64_t)a.positions[t] : (int64_t)pos, a.step[lane], a.gain);
    }
    if (lane == 0) {
      seq[wave] = at.b;
      stored[wave] = ok;
      row_off[wave] = off;
    }
  }
  __syncthreads();

  const int H = a.Hq + 2 * a.Hkv, units = kHeadDim / 16, rot_units = a.rotary / 16;
  for (int it = tid; it < TT * H * units; it += kThreads) {
    const int u = it % units, rest = it / units, w = rest / H, h = rest - w * H;
    const int t = t0 + w, b = seq[w];
    if (b >= a.ch.B) continue;  // rows of no sequence stay as they are
    const bool is_q = h < a.Hq, is_k = !is_q && h < a.Hq + a.Hkv;
    if (!is_q && !stored[w]) continue;
    const int hk = is_q ? 0 : is_k ? h - a.Hq : h - a.Hq - a.Hkv;
    const Q *src = is_q   ? static_cast<const Q *>(a.q) + (int64_t)t * a.q_st + h * kHeadDim
                   : is_k ? static_cast<const Q *>(a.k) + (int64_t)t * a.k_st + hk * kHeadDim
                          : static_cast<const Q *>(a.v) + (int64_t)t * a.v_st + hk * kHeadDim;
    const bool rot = u < rot_units && (is_q || is_k);
    // the unit's two runs of 8 features
    const bool split = u < rot_units && !a.interleaved;
    const int f0 = split ? 8 * u : 16 * u, f1 = split ? a.rotary / 2 + 8 * u : 16 * u + 8;
    float x[8], y[8];
    load8(src + f0, x);
    load8(src + f1, y);
    if (rot) {
      const float2 *c = cs[w] + 8 * u;
      if (a.interleaved) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float2 p = c[i], r = c[4 + i];
          const float x0 = x[2 * i], x1 = x[2 * i + 1], y0 = y[2 * i], y1 = y[2 * i + 1];
          x[2 * i] = x0 * p.x - x1 * p.y;
          x[2 * i + 1] = x1 * p.x + x0 * p.y;
          y[2 * i] = y0 * r.x - y1 * r.y;
          y[2 * i + 1] = y1 * r.x + y0 * r.y;
        }
      } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const float2 p = c[i];
          const float x0 = x[i], y0 = y[i];
          x[i] = x0 * p.x - y0 * p.y;
          y[i] = y0 * p.x + x0 * p.y;
        }
      }
    }
    if (is_q) {
      Q *dst = static_cast<Q *>(a.q_out) + ((int64_t)t * a.Hq + h) * kHeadDim;
      store8(dst + f0, x);
      store8(dst + f1, y);
    } else {
      E *dst = const_cast<E *>(static_cast<const E *>(is_k ? a.kv.k : a.kv.v)) + row_off[w] + (int64_t)hk * a.kv.sh;
      if constexpr (sizeof(E) == 1) {
        // the quotient rounds once to 32 bits, its code once more from there
        const float s = (is_k ? a.kv.ks : a.kv.vs)[(int64_t)b * a.Hkv + hk];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          x[i] = x[i] / s;
          y[i] = y[i] / s;
        }
      }
      store8(dst + f0, x);
      store8(dst + f1, y);
    }
  }
}

template <typename Q, typename E>
static hipError_t launch_rope_e(const RopeArgs &a, hipStream_t st) {
  const CallTimer tm = call_timer();
  void *params[] = {const_cast<RopeArgs *>(&a)};
  // Four tokens per workgroup pay where one has too few items to fill it, on long
  // chunks (us, one / four: 10 heads 2048 tokens 4.6 / 5.2, 4096 7.5 / 6.2, 16384
  // 24.1 / 16.9; 48 heads 1024 6.4 / 8.0, 4096 19.3 / 18.7, 16384 77 / 81).  A launch
  // counts its threads in 32 bits (and wraps without an error): 2^24 workgroups are
  // too many.
  const bool one = a.ch.tokens < 4096 ||
                   ((a.Hq + 2 * a.Hkv) * (kHeadDim / 16) >= kThreads && a.ch.tokens < (1 << 24));
  const void *fn = one ? (const void *)k_rope_append<Q, E, 1> : (const void *)k_rope_append<Q, E, 4>;
  return hipExtLaunchKernel(fn, dim3(one ? a.ch.tokens : (a.ch.tokens + 3) / 4), dim3(kThreads), params, 0, st,
                            tm.start, tm.stop, 0);
}

hipError_t launch_rope(const RopeArgs &a, int dtype, int elem, hipStream_t st) {
  if (elem == 2) return launch_rope_e<uint16_t, uint8_t>(a, st);
  return dtype == 0 ? launch_rope_e<uint16_t, uint16_t>(a, st) : launch_rope_e<float, float>(a, st);
}

}  // namespace santa
