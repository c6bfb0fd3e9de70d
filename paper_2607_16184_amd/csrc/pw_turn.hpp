// Norms of query and key heads with the position rotation, as the kernels that write
// them into rows and into the paged cache share them (gfx950).
#pragma once

#include "pw_kv.hpp"

namespace pw {
namespace {

// G lanes hold a head, eight channels each; a wave takes one token and 64 / G of
// its heads at a time. The norm is a sum over the G lanes. A pair's other half
// lies in the same lane (neighbouring pairs) or in the lane R / 16 further on or
// back, which hands over its 16-bit values as they were read. The angles of a
// token are the same for all its heads: they are reduced in 64 bits to a part of
// a turn (positions may be large), and their sines and cosines stay in registers
// while the wave goes through the heads, three steps of loads ahead.
// Bound by memory where there are many tokens: 4001 tokens, 36 heads of 128 in fp16
// (74 MB) 19 us in a graph, 3.9 TB/s (a large copy: 4.85); one token of 40 heads 4.1, a
// chain of positions, frequencies and heads.

// Cosine and sine of an angle, times the amplitude: quarters (a position, in quarters
// of a turn a radian) times a frequency. Whole quarters are taken off in 64 bits (added
// to 3 x 2^51, the sum is rounded to one and its lowest bits say which); an angle of at
// most pi / 4 is left, for which the series up to z^9 and z^8 are within 2^-25. (With
// the library's sine and cosine and two 64-bit products more the 4001-token rotated
// append took 34.6 us, with this 29.1.)
__device__ __forceinline__ void angle_of(const Rotate& r, double quarters, double freq, float* co, float* si) {
  const double t = fma(quarters, freq, 6755399441055744.0), n = t - 6755399441055744.0;
  // (past 2^51 quarters, where 64 bits no longer tell them, the rest is kept within its range)
  const float part = __builtin_amdgcn_fmed3f(static_cast<float>(fma(quarters, freq, -n)), -0.5f, 0.5f);
  const float z = part * 1.57079632679489662f, y = z * z;
  float s = fmaf(y, 2.7557319224e-6f, -1.98412698413e-4f);
  s = fmaf(fmaf(fmaf(y, s, 8.33333333333e-3f), y, -0.166666666667f), y * z, z);
  float c = fmaf(y, 2.48015873016e-5f, -1.38888888889e-3f);
  c = fmaf(fmaf(fmaf(y, c, 4.16666666667e-2f), y, -0.5f), y, 1.0f);
  const uint32_t k = static_cast<uint32_t>(__double_as_longlong(t));
  const float a = k & 1 ? s : c, b = k & 1 ? c : s;              // of the cosine, of the sine
  *co = (k + 1) & 2 ? -a * r.amplitude : a * r.amplitude;
  *si = k & 2 ? -b * r.amplitude : b * r.amplitude;
}
__device__ __forceinline__ double quarters_of(const Rotate& r, int64_t tok) {
  return (static_cast<double>(r.positions[tok]) + static_cast<double>(r.offset)) * 0.63661977236758134;
}

// cos and sin of the eight channels' angles, sin with the sign that the partner's
// value takes; 1 and 0 past the rotated channels. By all lanes of a wave for one token:
// each has one pair's angle, or two, and hands it to those that need it (one token 4.1
// us, with eight angles in every lane 4.2; 64 tokens into the cache 5.5 and 5.7).
struct Turn {
  float cs[8], sn[8];
};
__device__ __forceinline__ void turn_of(const Rotate& r, int64_t tok, int c, Turn* t) {
  const int half = r.R / 2, lane = lane_id();
  const bool on = 8 * c < r.R, hi = 8 * c >= half;
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    t->cs[j] = 1.0f;
    t->sn[j] = 0.0f;
  }
  if (r.R == 0) return;                                          // (uniform)
  const double quarters = quarters_of(r, tok);
  float co[2] = {1.0f, 1.0f}, si[2] = {0.0f, 0.0f};
#pragma unroll
  for (int i = 0; i < 2; ++i)
    if (64 * i + lane < half) angle_of(r, quarters, r.inv_freq[64 * i + lane], &co[i], &si[i]);
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    if (r.interleaved && (j & 1)) continue;
    const int i = r.interleaved ? 4 * c + j / 2 : 8 * c + j - (hi ? half : 0);
    float cj = __shfl(co[0], i & 63), sj = __shfl(si[0], i & 63);
    if (half > 64) {                                             // (uniform)
      const float c1 = __shfl(co[1], i & 63), s1 = __shfl(si[1], i & 63);
      cj = i >= 64 ? c1 : cj;
      sj = i >= 64 ? s1 : sj;
    }
    if (!on) continue;
    if (r.interleaved) {
      t->cs[j] = t->cs[j ^ 1] = cj;
      t->sn[j] = -sj;
      t->sn[j ^ 1] = sj;
    } else {
      t->cs[j] = cj;
      t->sn[j] = hi ? sj : -sj;
    }
  }
}

// f: the normed and turned values of a head's channels 8 c ..; x its values as
// read, w and wp the weights of these channels and of their partners'.
template <int ACT>
__device__ __forceinline__ void head_values(const HeadsArgs& a, u32x4 x, u32x4 w, u32x4 wp, const Turn& t, int c, int G,
                                            float* f) {
  unpack8<ACT>(x, f);
  float inv = 1.0f;
  if (a.norm) {
    float sq = 0.0f;
#pragma unroll
    for (int j = 0; j < 8; ++j) sq = fmaf(f[j], f[j], sq);
    for (int o = G / 2; o; o >>= 1) sq += __shfl_xor(sq, o);
    inv = 1.0f / sqrtf(sq / static_cast<float>(a.D) + a.eps);
  }
  float g[8], m[8];
  if (a.rot.interleaved) {
    unpack8<ACT>(w, m);
#pragma unroll
    for (int j = 0; j < 8; ++j) f[j] *= inv * m[j];
#pragma unroll
    for (int j = 0; j < 8; ++j) g[j] = f[j ^ 1];
  } else {
    const int by = a.rot.R / 16, p = static_cast<int>(lane_id()) + (c < by ? by : c < 2 * by ? -by : 0);
    u32x4 y;
#pragma unroll
    for (int i = 0; i < 4; ++i) y[i] = static_cast<uint32_t>(__shfl(static_cast<int>(x[i]), p));
    unpack8<ACT>(y, g);
    unpack8<ACT>(w, m);
#pragma unroll
    for (int j = 0; j < 8; ++j) f[j] *= inv * m[j];
    unpack8<ACT>(wp, m);
#pragma unroll
    for (int j = 0; j < 8; ++j) g[j] *= inv * m[j];
  }
  if (8 * c < a.rot.R) {
#pragma unroll
    for (int j = 0; j < 8; ++j) f[j] = fmaf(f[j], t.cs[j], g[j] * t.sn[j]);
  }
}

constexpr int kHeadsAhead = 3;        // heads of a lane group in flight

// Wave: token unit / parts, of its heads (queries, keys, then, with a cache, values)
// the `steps` x 64 / G from steps (64 / G) (unit mod parts) on.
template <int ACT, int BITS>                                     // BITS 0: keys into rows
__device__ __forceinline__ void heads_wave(const HeadsArgs& a, int64_t unit, int G, int steps, int parts) {
  const int lane = lane_id(), c = lane % G, per = 64 / G;
  const int64_t tok = unit / parts;
  if (tok >= a.T) return;
  const int first = static_cast<int>(unit % parts) * steps * per + lane / G;
  const int n = a.n_q + (BITS ? 2 : 1) * a.n_k;
  const int by = a.rot.R / 16, cp = c < by ? c + by : c < 2 * by ? c - by : c;
  const bool in = 8 * c < a.D;
  const u32x4 one = ACT == PW_BF16 ? u32x4{0x3F803F80u, 0x3F803F80u, 0x3F803F80u, 0x3F803F80u}
                                   : u32x4{0x3C003C00u, 0x3C003C00u, 0x3C003C00u, 0x3C003C00u};
  u32x4 w[2] = {one, one}, wp[2] = {one, one};
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const uint16_t* src = i ? a.k_weight : a.q_weight;
    if (src && in) {
      w[i] = ld16(reinterpret_cast<const uint8_t*>(src + 8 * c));
      wp[i] = ld16(reinterpret_cast<const uint8_t*>(src + 8 * cp));
    }
  }
  int64_t slot = -1;
  if constexpr (BITS > 0) slot = a.slots[tok];
  Turn t;
  turn_of(a.rot, tok, c, &t);
  const auto load = [&](int hh) {
    const uint16_t* src = a.q + tok * a.ldq + hh * a.ldqh;
    if (hh >= a.n_q) src = a.k + tok * a.ldk + (hh - a.n_q) * a.ldkh;
    if (BITS && hh >= a.n_q + a.n_k) src = a.v + tok * a.ldk + (hh - a.n_q - a.n_k) * a.ldkh;
    return hh < n && in ? ld16(reinterpret_cast<const uint8_t*>(src + 8 * c)) : u32x4{0u, 0u, 0u, 0u};
  };
  // the next heads are on their way while these are worked on
  u32x4 now[kHeadsAhead];
#pragma unroll
  for (int i = 0; i < kHeadsAhead; ++i) now[i] = i < steps ? load(first + i * per) : u32x4{0u, 0u, 0u, 0u};
  for (int i0 = 0; i0 < steps; i0 += kHeadsAhead) {
    u32x4 next[kHeadsAhead];
#pragma unroll
    for (int i = 0; i < kHeadsAhead; ++i)
      next[i] = i0 + kHeadsAhead + i < steps ? load(first + (i0 + kHeadsAhead + i) * per) : u32x4{0u, 0u, 0u, 0u};
#pragma unroll
    for (int i = 0; i < kHeadsAhead; ++i) {
      if (i0 + i >= steps) break;
      const int hh = first + (i0 + i) * per;
      const u32x4 x = now[i];
      const bool key = hh >= a.n_q, value = BITS && hh >= a.n_q + a.n_k;
      float f[8];
      head_values<ACT>(a, x, key ? w[1] : w[0], key ? wp[1] : wp[0], t, c, G, f);   // (exchanges: by all lanes)
      u32x4 y;
#pragma unroll
      for (int j = 0; j < 4; ++j) y[j] = pack16<ACT>(f[2 * j], f[2 * j + 1]);
      if (!key) {
        if (in && hh < n) *reinterpret_cast<u32x4*>(a.q_out + tok * a.ldqo + hh * a.ldqoh + 8 * c) = y;
      } else if constexpr (BITS == 0) {
        if (in && hh < n) *reinterpret_cast<u32x4*>(a.k_out + tok * a.ldko + (hh - a.n_q) * a.ldkoh + 8 * c) = y;
      }
      if constexpr (BITS > 0) {
        if (!slot_ok(a.kv, slot)) continue;                      // (wave-uniform)
        const int h = value ? hh - a.n_q - a.n_k : hh - a.n_q;
        if constexpr (BITS == 16) {
          if (key && hh < n) put16(a.kv, value ? x : y, slot, h, value, c);
        } else {
          if (value) unpack8<ACT>(x, f);
          if (key && hh < n) put8(a.kv, f, slot, h, value, c, G);   // (the same for all G lanes)
        }
      }
    }
#pragma unroll
    for (int i = 0; i < kHeadsAhead; ++i) now[i] = next[i];
  }
}

// How waves share the heads of T tokens: lanes of a head, steps of a wave, waves of a
// token.
struct HeadsCut {
  int G, steps, parts;
  int64_t blocks;          // of four waves
};
inline HeadsCut heads_cut(int T, int D, int n_heads) {
  HeadsCut k{8, 1, 1, 0};
  while (8 * k.G < D) k.G *= 2;
  const int per = 64 / k.G, groups = (n_heads + per - 1) / per;
  while (k.steps < groups && static_cast<int64_t>(T) * ((groups + k.steps - 1) / k.steps) > 4096) ++k.steps;
  k.parts = (groups + k.steps - 1) / k.steps;
  k.blocks = (static_cast<int64_t>(T) * k.parts + 3) / 4;
  return k;
}

}  // namespace
}  // namespace pw
