// Between a projection's rows and the attention, gfx950: norms of query and key
// heads with the position rotation, into rows or (keys, with the values) into the
// paged cache (k_heads), and drafted tokens moved together in it (k_kv_keep).
#include "pw_kv.hpp"

namespace pw {
namespace {

// ---------------------------------------------------------------------------
// Norm and rotation
// ---------------------------------------------------------------------------
//
// G lanes hold a head, eight channels each; a wave takes one token and 64 / G of
// its heads at a time. The norm is a sum over the G lanes. A pair's other half
// lies in the same lane (neighbouring pairs) or in the lane R / 16 further on or
// back, which hands over its 16-bit values as they were read. The angles of a
// token are the same for all its heads: they are reduced in 64 bits to a part of
// a turn (positions may be large), and their sines and cosines stay in registers
// while the wave goes through the heads.

// cos and sin of the eight channels' angles, sin with the sign that the partner's
// value takes; 1 and 0 past the rotated channels.
struct Turn {
  float cs[8], sn[8];
};
__device__ __forceinline__ void turn_of(const Rotate& r, int64_t tok, int c, Turn* t) {
  const bool on = 8 * c < r.R;
  const int half = r.R / 2;
  const bool hi = 8 * c >= half;
  const double pos = on ? static_cast<double>(r.positions[tok]) + static_cast<double>(r.offset) : 0.0;
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    t->cs[j] = 1.0f;
    t->sn[j] = 0.0f;
  }
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    if (!on || (r.interleaved && (j & 1))) continue;
    const int i = r.interleaved ? 4 * c + j / 2 : 8 * c + j - (hi ? half : 0);
    double x = pos * r.inv_freq[i] * 0.15915494309189535;        // turns
    x -= __builtin_rint(x);
    float s, co;
    sincospif(static_cast<float>(2.0 * x), &s, &co);
    s *= r.amplitude;
    co *= r.amplitude;
    if (r.interleaved) {
      t->cs[j] = t->cs[j ^ 1] = co;
      t->sn[j] = -s;
      t->sn[j ^ 1] = s;
    } else {
      t->cs[j] = co;
      t->sn[j] = hi ? s : -s;
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

// Wave: token unit / parts, of its heads (queries, keys, then, with a cache, values)
// the `steps` x 64 / G from steps (64 / G) (unit mod parts) on.
template <int ACT, int BITS>                                     // BITS 0: keys into rows
__global__ __launch_bounds__(256) void k_heads(HeadsArgs a, int G, int steps, int parts) {
  const int lane = lane_id(), c = lane % G, per = 64 / G;
  const int64_t unit = static_cast<int64_t>(blockIdx.x) * 4 + __builtin_amdgcn_readfirstlane(static_cast<int>(threadIdx.x) >> 6);
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
  u32x4 next = load(first);
  for (int i = 0; i < steps; ++i) {
    const int hh = first + i * per;
    const u32x4 x = next;
    if (i + 1 < steps) next = load(hh + per);
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
      if (!slot_ok(a.kv, slot)) continue;                        // (wave-uniform)
      const int h = value ? hh - a.n_q - a.n_k : hh - a.n_q;
      if constexpr (BITS == 16) {
        if (key && hh < n) put16(a.kv, value ? x : y, slot, h, value, c);
      } else {
        if (value) unpack8<ACT>(x, f);
        if (key && hh < n) put8(a.kv, f, slot, h, value, c, G);  // (the same for all G lanes)
      }
    }
  }
}

template <int ACT>
hipError_t heads(const HeadsArgs& a, hipStream_t st) {
  const int bits = a.slots ? a.kv.bits : 0;
  int G = 8;
  while (8 * G < a.D) G *= 2;
  const int per = 64 / G, groups = (a.n_q + (bits ? 2 : 1) * a.n_k + per - 1) / per;
  int steps = 1;
  while (steps < groups && static_cast<int64_t>(a.T) * ((groups + steps - 1) / steps) > 4096) ++steps;
  const int parts = (groups + steps - 1) / steps;
  const int64_t grid = (static_cast<int64_t>(a.T) * parts + 3) / 4;
  if (grid > INT32_MAX) return hipErrorInvalidConfiguration;
  const dim3 g(static_cast<uint32_t>(grid));
  if (bits == 0) k_heads<ACT, 0><<<g, 256, 0, st>>>(a, G, steps, parts);
  else if (bits == 16) k_heads<ACT, 16><<<g, 256, 0, st>>>(a, G, steps, parts);
  else k_heads<ACT, 8><<<g, 256, 0, st>>>(a, G, steps, parts);
  return hipGetLastError();
}

// ---------------------------------------------------------------------------
// Keeping drafted tokens
// ---------------------------------------------------------------------------
//
// A workgroup takes one sequence and key head. Each thread moves one piece of
// the entries (16 or 8 bytes of a key, one element of a value, a scale), token
// after token in their order: a token moves to its own position or a lower one,
// above every earlier token's, so no write meets a read that is still to come and
// no thread another's. What bounds it is the chain of starts, table, reads and
// writes.
constexpr int kKeepAtOnce = 8;        // tokens read before the first of them is written
template <int BITS>
__global__ __launch_bounds__(256) void k_kv_keep(KeepArgs a) {
  constexpr int kE = BITS / 8;
  __shared__ int64_t src[64], dst[64];                           // (block * block_tokens + position)
  __shared__ int n_list;
  const int h = blockIdx.x, b = blockIdx.y, tid = static_cast<int>(threadIdx.x);
  const int D = a.kv.head_dim, P = a.kv.block_tokens, H = a.kv.n_kv_heads;
  // (starts and lengths are the device's: sums in 64 bits, whatever they hold)
  const int64_t n64 = static_cast<int64_t>(a.starts[b + 1]) - a.starts[b];
  const int n = static_cast<int>(n64 < 0 ? 0 : n64 > (1 << 30) ? 1 << 30 : n64);
  const int64_t c64 = static_cast<int64_t>(a.lens[b]) - n;
  const int ctx = static_cast<int>(c64 < -(1 << 30) ? -(1 << 30) : c64), base = max(ctx, 0);
  const auto slot_at = [&](int64_t p) -> int64_t {
    if (p < 0 || p >= a.max_len) return -1;
    const int blk = a.table[b * a.ld_table + p / P];
    return blk >= 0 && blk < a.kv.n_blocks ? static_cast<int64_t>(blk) * P + p % P : -1;
  };
  int count = 0;                                                 // chosen so far
  for (int w = 0; w < a.words && 64 * w < n; ++w) {
    uint64_t bits = static_cast<uint64_t>(a.chosen[static_cast<int64_t>(b) * a.words + w]);
    if (n - 64 * w < 64) bits &= (1ull << (n - 64 * w)) - 1ull;
    const int below = -ctx - 64 * w;                             // drafted tokens before position 0 do not exist
    if (ctx < 0 && below > 0) bits &= below >= 64 ? 0ull : ~0ull << below;
    if (tid < 64) {
      const bool on = (bits >> tid) & 1ull;
      const int64_t from = static_cast<int64_t>(ctx) + 64 * w + tid;
      const int64_t to = static_cast<int64_t>(base) + count + __popcll(bits & ((1ull << tid) - 1ull));
      int64_t s = -1, d = -1;
      if (on && from != to) {
        s = slot_at(from);
        d = slot_at(to);
      }
      const uint64_t move = __ballot(s >= 0 && d >= 0);
      const int at = __popcll(move & ((1ull << tid) - 1ull));
      if (s >= 0 && d >= 0) {
        src[at] = s;
        dst[at] = d;
      }
      if (tid == 0) n_list = __popcll(move);
    }
    count += __popcll(bits);
    __syncthreads();
    const int m = n_list;
    const int units = D / 8 + D + (BITS == 8 ? 2 : 0);
    for (int u = tid; u < units; u += 256) {
      const auto at = [&](int64_t slot) -> uint8_t* {            // the unit's place in a slot
        const int t = static_cast<int>(slot % P);
        uint8_t* blk = a.kv.pool + slot / P * a.kv.block_stride;
        uint8_t* head = blk + static_cast<size_t>(2 * h) * P * D * kE;
        if (u < D / 8) {
          if constexpr (BITS == 16) return head + ((t / 16) * (D / 32) + u / 4) * 1024 + 16 * (16 * (u & 3) + t % 16);
          return head + ((t / 16) * (D / 64) + u / 8) * 1024 + 16 * (16 * (u & 3) + t % 16) + 8 * (u / 4 % 2);
        }
        if (u < D / 8 + D) {
          const int d = u - D / 8;
          uint8_t* v = head + static_cast<size_t>(P) * D * kE;
          if constexpr (BITS == 16)
            return v + ((t / 32) * (D / 16) + d / 16) * 1024 + 16 * (16 * (t / 4 % 4) + d % 16) + 2 * (4 * (t / 16 % 2) + t % 4);
          return v + ((t / 32) * (D / 32) + d / 32) * 1024 + 16 * (16 * (t / 4 % 4) + d % 16) + 8 * (d / 16 % 2) +
                 4 * (t / 16 % 2) + t % 4;
        }
        return blk + static_cast<size_t>(2) * H * P * D + 4 * static_cast<size_t>(((u - D / 8 - D) * H + h) * P + t);
      };
      for (int i0 = 0; i0 < m; i0 += kKeepAtOnce) {
        const int k = min(kKeepAtOnce, m - i0);
        if (u < D / 8) {
          u32x4 x[kKeepAtOnce];
#pragma unroll
          for (int i = 0; i < kKeepAtOnce; ++i)
            if (i < k) {
              if constexpr (BITS == 16) {
                x[i] = ld16(at(src[i0 + i]));
              } else {
                const u32x2 y = *reinterpret_cast<const u32x2*>(at(src[i0 + i]));
                x[i] = u32x4{y[0], y[1], 0u, 0u};
              }
            }
#pragma unroll
          for (int i = 0; i < kKeepAtOnce; ++i)
            if (i < k) {
              if constexpr (BITS == 16) *reinterpret_cast<u32x4*>(at(dst[i0 + i])) = x[i];
              else *reinterpret_cast<u32x2*>(at(dst[i0 + i])) = u32x2{x[i][0], x[i][1]};
            }
        } else if (u < D / 8 + D) {
          uint32_t x[kKeepAtOnce];
#pragma unroll
          for (int i = 0; i < kKeepAtOnce; ++i)
            if (i < k) x[i] = BITS == 16 ? *reinterpret_cast<const uint16_t*>(at(src[i0 + i])) : *at(src[i0 + i]);
#pragma unroll
          for (int i = 0; i < kKeepAtOnce; ++i)
            if (i < k) {
              if constexpr (BITS == 16) *reinterpret_cast<uint16_t*>(at(dst[i0 + i])) = static_cast<uint16_t>(x[i]);
              else *at(dst[i0 + i]) = static_cast<uint8_t>(x[i]);
            }
        } else {
          float x[kKeepAtOnce];
#pragma unroll
          for (int i = 0; i < kKeepAtOnce; ++i)
            if (i < k) x[i] = *reinterpret_cast<const float*>(at(src[i0 + i]));
#pragma unroll
          for (int i = 0; i < kKeepAtOnce; ++i)
            if (i < k) *reinterpret_cast<float*>(at(dst[i0 + i])) = x[i];
        }
      }
    }
    __syncthreads();                                             // the list is read
  }
  if (h == 0 && tid == 0) a.new_lens[b] = base + count;
}

}  // namespace

hipError_t launch_heads(const HeadsArgs& a, hipStream_t st) {
  return a.act == PW_BF16 ? heads<PW_BF16>(a, st) : heads<PW_F16>(a, st);
}

hipError_t launch_kv_keep(const KeepArgs& a, hipStream_t st) {
  const dim3 g(a.kv.n_kv_heads, a.B);
  if (a.kv.bits == 16) k_kv_keep<16><<<g, 256, 0, st>>>(a);
  else k_kv_keep<8><<<g, 256, 0, st>>>(a);
  return hipGetLastError();
}

}  // namespace pw
