// Paged KV cache, gfx950: writing new tokens into it (k_kv_append) and the
// attention of one new token per sequence over it (k_attn, k_attn_join).
#include "pw_turn.hpp"

namespace pw {
namespace {

// ---------------------------------------------------------------------------
// Append
// ---------------------------------------------------------------------------

// One token's key (is_v 0) or value (1) of head h by G neighbouring lanes (a
// power of two, at least D / 8), lane c of them with channels 8 c .. 8 c + 7: its
// load, and what is done with it.
__device__ __forceinline__ u32x4 load_one(const AppendArgs& a, int64_t tok, int h, int is_v, int c) {
  return ld16(reinterpret_cast<const uint8_t*>((is_v ? a.v : a.k) + tok * a.ld + h * a.ldh + 8 * c));
}
template <int ACT, int BITS>
__device__ __forceinline__ void append_one(const AppendArgs& a, u32x4 raw, int64_t slot, int h, int is_v, int c, int G) {
  if constexpr (BITS == 16) {
    put16(a.kv, raw, slot, h, is_v, c);
  } else {
    float f[8];
    unpack8<ACT>(raw, f);
    put8(a.kv, f, slot, h, is_v, c, G);
  }
}
__device__ __forceinline__ bool slot_ok(const AppendArgs& a, int64_t slot) { return slot_ok(a.kv, slot); }

// Few tokens, or none next to each other (a decode step), or few heads: G lanes
// per token, head and side.
template <int ACT, int BITS>
__global__ __launch_bounds__(256) void k_kv_append(AppendArgs a, int G) {
  const int H = a.kv.n_kv_heads;
  const int64_t items = static_cast<int64_t>(a.T) * H * 2;
  const int per = 256 / G, c = static_cast<int>(threadIdx.x) % G;
  for (int64_t item = static_cast<int64_t>(blockIdx.x) * per + static_cast<int>(threadIdx.x) / G; item < items;
       item += static_cast<int64_t>(gridDim.x) * per) {
    const int64_t tok = (item >> 1) / H, slot = a.slots[tok];
    const int h = static_cast<int>((item >> 1) % H), is_v = static_cast<int>(item & 1);
    const u32x4 raw = 8 * c < a.kv.head_dim ? load_one(a, tok, h, is_v, c) : u32x4{0u, 0u, 0u, 0u};
    if (slot_ok(a, slot)) append_one<ACT, BITS>(a, raw, slot, h, is_v, c, G);   // (the same for all G lanes)
  }
}

// Many tokens (a prefill chunk): a wave per window of 32 tokens, head and side.
// Tokens that follow each other inside a 32-token tile of the cache are a run;
// the wave of the window that holds its first token writes it as a piece of the
// tile: keys in the order in which they are loaded, 16 bytes a lane, values
// turned in LDS. Tokens of runs shorter than kMinRun go one by one.
// (A value's elements lie 16 bytes apart, so tokens written one by one take long
// where there are many: 4001 of 8 heads x 128 channels 26.7 us in 16 bits and 18.1
// in 8, as runs 10.9 and 12.5. A run is a longer chain of loads, turns and stores,
// so few tokens or heads are done sooner one by one, whatever the channels. Runs /
// one by one in us, consecutive tokens x heads x channels: 16 bits, 512 x 8 x 128
// 8.0 / 6.7, 768 x 8 x 128 8.1 / 8.8, 3073 x 2 x 128 7.9 / 8.1, 4096 x 1 x 128 7.5
// / 5.4, 768 x 8 x 64 5.7 / 5.5, 768 x 8 x 256 13.8 / 13.5; 8 bits, 1536 x 8 x 128
// 11.6 / 10.0, 2048 12.1 / 11.7, 3073 12.6 / 15.6, 2048 x 8 x 64 7.6 / 7.7, 1024 x
// 16 x 64 7.7 / 8.0, 2048 x 8 x 256 19.9 / 18.2. Tokens in no order lose by runs,
// 512 x 8 x 128 in 16 bits 12.1 / 6.7: from kAppendMany on a step's tokens are
// hardly those of a decode batch.)
constexpr int kAppendWaves = 4;
constexpr int kAppendMany = 512;          // tokens
constexpr int kRunItems16 = 6144, kRunItems8 = 16384;   // tokens x heads
constexpr int kMinRun = 8;

// The values of place c's token (at row `tok`, channels 32 i + 8 lg .. of its key x) as
// heads_wave has them; a pair's other half lies in the same lane.
template <int ACT, int D>
__device__ __forceinline__ void turned_key(const HeadsArgs& t, const u32x4 (&x)[D / 32], int64_t tok, int lg, float (&f)[D / 32][8]) {
  float sq = 0.0f;
#pragma unroll
  for (int i = 0; i < D / 32; ++i) {
    unpack8<ACT>(x[i], f[i]);
#pragma unroll
    for (int j = 0; j < 8; ++j) sq = fmaf(f[i][j], f[i][j], sq);
  }
  if (t.norm) {
    sq += __shfl_xor(sq, 16);
    sq += __shfl_xor(sq, 32);
    const float inv = 1.0f / sqrtf(sq / static_cast<float>(D) + t.eps);
#pragma unroll
    for (int i = 0; i < D / 32; ++i) {
      float w[8];
      if (t.k_weight) unpack8<ACT>(ld16(reinterpret_cast<const uint8_t*>(t.k_weight + 32 * i + 8 * lg)), w);
#pragma unroll
      for (int j = 0; j < 8; ++j) f[i][j] *= t.k_weight ? inv * w[j] : inv;
    }
  }
  const double quarters = t.rot.R > 0 ? quarters_of(t.rot, tok) : 0.0;
  if (t.rot.interleaved) {
#pragma unroll
    for (int i = 0; i < D / 32; ++i) {
      if (32 * i + 8 * lg >= t.rot.R) continue;
      double freq[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) freq[j] = t.rot.inv_freq[16 * i + 4 * lg + j];
#pragma unroll
      for (int j = 0; j < 8; j += 2) {
        float co, si;
        angle_of(t.rot, quarters, freq[j / 2], &co, &si);
        const float y = f[i][j], z = f[i][j + 1];
        f[i][j] = fmaf(y, co, z * -si);
        f[i][j + 1] = fmaf(z, co, y * si);
      }
    }
  } else {
#pragma unroll
    for (int by = 1; by <= D / 64; ++by) {                       // R = 64 by
      if (t.rot.R != 64 * by) continue;
#pragma unroll
      for (int i = 0; i < by; ++i) {
        double freq[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) freq[j] = t.rot.inv_freq[32 * i + 8 * lg + j];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          float co, si;
          angle_of(t.rot, quarters, freq[j], &co, &si);
          const float y = f[i][j], z = f[i + by][j];
          f[i][j] = fmaf(y, co, z * -si);
          f[i + by][j] = fmaf(z, co, y * si);
        }
      }
    }
  }
}

// turn_of for a token per lane group.
__device__ __forceinline__ void own_turn(const Rotate& r, int64_t tok, int c, Turn* t) {
  const int half = r.R / 2;
  const bool hi = 8 * c >= half;
  const double quarters = r.R > 0 ? quarters_of(r, tok) : 0.0;
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    t->cs[j] = 1.0f;
    t->sn[j] = 0.0f;
    if (8 * c >= r.R) continue;
    float co, si;
    angle_of(r, quarters, r.inv_freq[r.interleaved ? 4 * c + j / 2 : 8 * c + j - (hi ? half : 0)], &co, &si);
    t->cs[j] = co;
    t->sn[j] = (r.interleaved ? j & 1 : hi) ? si : -si;
  }
}

// Window, head and side `unit` of a.T tokens, by one wave with `mine` of LDS. TURN: keys
// normed and turned (t).
template <int ACT, int BITS, int D, bool TURN>
__device__ __forceinline__ void append_window(const AppendArgs& a, const HeadsArgs& t_args, int64_t unit, uint8_t* mine) {
  constexpr int kE = BITS / 8, kPitch = D * kE + 4;
  const int lane = lane_id();
  const int H = a.kv.n_kv_heads, P = a.kv.block_tokens;
  const int is_v = static_cast<int>(unit & 1), h = static_cast<int>((unit >> 1) % H);
  const int64_t first = (unit >> 1) / H * 32;                    // first token of the window
  if (first >= a.T) return;                                      // (wave-uniform; no barrier follows)

  // slots of the tokens first - 32 + lane and first + 32 + lane
  const auto slot_of = [&](int64_t n) { return n >= 0 && n < a.T ? a.slots[n] : int64_t(-1); };
  const int64_t sa = slot_of(first - 32 + lane), sb = slot_of(first + 32 + lane);
  const auto shfl64 = [&](int64_t v, int l) {
    return static_cast<int64_t>((static_cast<uint64_t>(static_cast<uint32_t>(__shfl(static_cast<int>(v >> 32), l))) << 32) |
                                static_cast<uint32_t>(__shfl(static_cast<int>(v), l)));
  };
  const int64_t end = shfl64(sa, 63);
  int64_t pa = shfl64(sa, (lane + 63) & 63), pb = shfl64(sb, (lane + 63) & 63);
  if (lane == 0) {
    pa = -1;
    pb = end;
  }
  // bit i of (mb : ma): token i of these 128 goes on with its predecessor's run
  const uint64_t ma = __ballot(slot_ok(a, sa) && (sa & 31) != 0 && pa == sa - 1);
  const uint64_t mb = __ballot(slot_ok(a, sb) && (sb & 31) != 0 && pb == sb - 1);
  // the window's own tokens are those of lanes 32 and up: the start of a token's
  // run (no more than 31 before it) and its length
  const bool own = lane >= 32 && slot_ok(a, sa);
  const uint64_t starts = ~ma & (lane == 63 ? ~0ull : (2ull << lane) - 1ull);
  const int s0 = starts ? 63 - __clzll(static_cast<long long>(starts)) : 0;
  const uint64_t after = s0 == 63 ? mb : (ma >> (s0 + 1)) | (mb << (63 - s0));
  const int len = __ffsll(static_cast<long long>(~after));        // one more than the ones that follow
  uint64_t lead = __ballot(own && s0 == lane && len >= kMinRun);
  const uint64_t single = __ballot(own && len < kMinRun) >> 32;

  while (lead) {
    const int ll = __ffsll(static_cast<long long>(lead)) - 1;
    lead &= lead - 1;
    const int64_t slot = shfl64(sa, ll);
    const int n_run = __builtin_amdgcn_readlane(len, ll);
    const int t = static_cast<int>(slot % P) & ~31, t0 = static_cast<int>(slot & 31);   // the tile, the run's place in it
    const int64_t n0 = first - 32 + ll - t0;                     // token of the tile's first place
    const auto in = [&](int place) { return place >= t0 && place < t0 + n_run; };
    uint8_t* blk = a.kv.pool + slot / P * a.kv.block_stride;
    uint8_t* dst = blk + static_cast<size_t>(2 * h + is_v) * P * D * kE + static_cast<size_t>(t) * D * kE;
    const int c = lane & 15, lg = lane >> 4;
    u32x4 x[2][D / 32];                                          // place c of either half, channels 32 i + 8 lg ..
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      const uint16_t* src = (is_v ? a.v : a.k) + (n0 + 16 * u + c) * a.ld + h * a.ldh + 8 * lg;
#pragma unroll
      for (int i = 0; i < D / 32; ++i)
        x[u][i] = in(16 * u + c) ? ld16(reinterpret_cast<const uint8_t*>(src + 32 * i)) : u32x4{0u, 0u, 0u, 0u};
    }
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      float kf[D / 32][8];                                       // TURN: the keys
      if constexpr (TURN) {
        if (!is_v) {
          turned_key<ACT, D>(t_args, x[u], in(16 * u + c) ? n0 + 16 * u + c : n0 + t0, lg, kf);
#pragma unroll
          for (int i = 0; i < D / 32; ++i)
#pragma unroll
            for (int w = 0; w < 4; ++w) x[u][i][w] = pack16<ACT>(kf[i][2 * w], kf[i][2 * w + 1]);
        }
      }
      uint8_t* row = mine + (16 * u + c) * kPitch + 8 * lg * kE;
      const bool here = in(16 * u + c);
      if constexpr (BITS == 16) {
#pragma unroll
        for (int i = 0; i < D / 32; ++i) {
          if (!is_v) {
            if (here) *reinterpret_cast<u32x4*>(dst + (u * (D / 32) + i) * 1024 + 16 * lane) = x[u][i];
          } else {
#pragma unroll
            for (int w = 0; w < 4; ++w) *reinterpret_cast<any_u32*>(row + 64 * i + 4 * w) = x[u][i][w];
          }
        }
      } else {
        float m = 0.0f;
#pragma unroll
        for (int i = 0; i < D / 32; ++i)
#pragma unroll
          for (int j = 0; j < 8; ++j)
            m = fmaxf(m, fabsf(TURN && !is_v ? kf[i][j] : val16(x[u][i][j / 2] >> (16 * (j & 1)), ACT)));
        m = fmaxf(m, __shfl_xor(m, 16));
        m = fmaxf(m, __shfl_xor(m, 32));
        const float s = f8_scale(m);
        u32x2 q[D / 32];
#pragma unroll
        for (int i = 0; i < D / 32; ++i) {
          float f[8];
#pragma unroll
          for (int j = 0; j < 8; ++j) f[j] = TURN && !is_v ? kf[i][j] : val16(x[u][i][j / 2] >> (16 * (j & 1)), ACT);
          q[i] = f8_codes8(f, s);
        }
        if (lg == 0 && here) {
          float* sc = reinterpret_cast<float*>(blk + static_cast<size_t>(2) * H * P * D);
          sc[(is_v * H + h) * P + t + 16 * u + c] = s;
        }
#pragma unroll
        for (int i = 0; i < D / 32; i += 2) {
          if (!is_v) {
            if (here)
              *reinterpret_cast<u32x4*>(dst + (u * (D / 64) + i / 2) * 1024 + 16 * lane) =
                  u32x4{q[i][0], q[i][1], q[i + 1][0], q[i + 1][1]};
          } else {
#pragma unroll
            for (int w = 0; w < 4; ++w) *reinterpret_cast<any_u32*>(row + 32 * (i + w / 2) + 4 * (w & 1)) = q[i + w / 2][w & 1];
          }
        }
      }
    }
    if (is_v) {
      wave_exchange();
      // lane: channel c of a tile, places 4 lg .. + 3 of either half
      bool all[2], some[2];
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        const int p0 = 16 * u + 4 * lg;
        all[u] = in(p0) && in(p0 + 3);
        some[u] = p0 + 3 >= t0 && p0 < t0 + n_run;
      }
#pragma unroll
      for (int j = 0; j < D * kE / 32; ++j) {
        u32x4 v;
#pragma unroll
        for (int w = 0; w < 4; ++w) {
          uint32_t o = 0;
          if constexpr (BITS == 16) {
#pragma unroll
            for (int e = 0; e < 2; ++e) {
              const int tok = 16 * (w / 2) + 4 * lg + 2 * (w & 1) + e;
              o |= static_cast<uint32_t>(*reinterpret_cast<const any_u16*>(mine + tok * kPitch + 2 * (16 * j + c))) << (16 * e);
            }
          } else {
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const int tok = 16 * (w & 1) + 4 * lg + e;
              o |= static_cast<uint32_t>(mine[tok * kPitch + 32 * j + 16 * (w / 2) + c]) << (8 * e);
            }
          }
          v[w] = o;
        }
        uint8_t* at = dst + j * 1024 + 16 * lane;
        if (n_run == 32) {
          *reinterpret_cast<u32x4*>(at) = v;
          continue;
        }
        // four places of one channel: whole, or element by element
#pragma unroll
        for (int u = 0; u < 2; ++u) {
          if constexpr (BITS == 16) {
            if (all[u]) {
              *reinterpret_cast<u32x2*>(at + 8 * u) = u32x2{v[2 * u], v[2 * u + 1]};
            } else if (some[u]) {
#pragma unroll
              for (int e = 0; e < 4; ++e)
                if (in(16 * u + 4 * lg + e))
                  *reinterpret_cast<uint16_t*>(at + 8 * u + 2 * e) = static_cast<uint16_t>(v[2 * u + e / 2] >> (16 * (e & 1)));
            }
          } else {
#pragma unroll
            for (int jh = 0; jh < 2; ++jh) {
              const uint32_t o = v[2 * jh + u];
              if (all[u]) {
                *reinterpret_cast<uint32_t*>(at + 8 * jh + 4 * u) = o;
              } else if (some[u]) {
#pragma unroll
                for (int e = 0; e < 4; ++e)
                  if (in(16 * u + 4 * lg + e)) at[8 * jh + 4 * u + e] = static_cast<uint8_t>(o >> (8 * e));
              }
            }
          }
        }
      }
      wave_exchange();
    }
  }
  if (single) {
    constexpr int G = D <= 64 ? 8 : D <= 128 ? 16 : 32, kAtOnce = 64 / G, kTurns = 32 / kAtOnce;
    const int c = lane % G;
    u32x4 raw[kTurns];                                           // (all loads before the first use)
#pragma unroll
    for (int j = 0; j < kTurns; ++j) {
      const int n = j * kAtOnce + lane / G;
      raw[j] = u32x4{0u, 0u, 0u, 0u};
      if (8 * c < D && ((single >> n) & 1ull)) raw[j] = load_one(a, first + n, h, is_v, c);
    }
#pragma unroll
    for (int j = 0; j < kTurns; ++j) {
      const int n = j * kAtOnce + lane / G;
      const int64_t slot = shfl64(sa, 32 + n);
      if constexpr (TURN) {
        if (!is_v) {
          const int by = t_args.rot.R / 16, cp = c < by ? c + by : c < 2 * by ? c - by : c;
          const uint32_t one2 = ACT == PW_BF16 ? 0x3F803F80u : 0x3C003C00u;
          u32x4 w{one2, one2, one2, one2}, wp = w;
          if (t_args.k_weight && 8 * c < D) {
            w = ld16(reinterpret_cast<const uint8_t*>(t_args.k_weight + 8 * c));
            wp = ld16(reinterpret_cast<const uint8_t*>(t_args.k_weight + 8 * cp));
          }
          Turn tn;
          own_turn(t_args.rot, min(first + n, static_cast<int64_t>(a.T) - 1), c, &tn);
          float f[8];
          head_values<ACT>(t_args, raw[j], w, wp, tn, c, G, f);
          if ((single >> n) & 1ull) {
            if constexpr (BITS == 16) {
              u32x4 y;
#pragma unroll
              for (int i = 0; i < 4; ++i) y[i] = pack16<ACT>(f[2 * i], f[2 * i + 1]);
              put16(a.kv, y, slot, h, 0, c);
            } else {
              put8(a.kv, f, slot, h, 0, c, G);
            }
          }
          continue;
        }
      }
      if ((single >> n) & 1ull) append_one<ACT, BITS>(a, raw[j], slot, h, is_v, c, G);
    }
  }
}

template <int ACT, int BITS, int D>
__global__ __launch_bounds__(64 * kAppendWaves) void k_kv_append_tiles(AppendArgs a) {
  __shared__ __attribute__((aligned(16))) uint8_t lds[kAppendWaves][32 * (D * (BITS / 8) + 4)];
  const int wave = __builtin_amdgcn_readfirstlane(static_cast<int>(threadIdx.x) >> 6);
  append_window<ACT, BITS, D, false>(a, HeadsArgs{}, static_cast<int64_t>(blockIdx.x) * kAppendWaves + wave, lds[wave]);
}

// The rotated append of many tokens: keys and values by windows, first (they take
// longest), the queries by tokens (k, without keys). 4001 tokens, 32 query and 8 key
// heads of 128 in bf16 (90 MB into 8 bits, 107 into 16): 29 and 27 us, without a
// rotation 20.5; token by token, and with the library's sine, 34 in 8 bits. What the rotation adds is the chain of a
// key wave: its 64 angles, 32 a lane, one wave per SIMD.
template <int ACT, int BITS, int D>
__global__ __launch_bounds__(64 * kAppendWaves) void k_append_runs(AppendArgs a, HeadsArgs t, HeadsCut k, int64_t window_blocks) {
  __shared__ __attribute__((aligned(16))) uint8_t lds[kAppendWaves][32 * (D * (BITS / 8) + 4)];
  const int wave = __builtin_amdgcn_readfirstlane(static_cast<int>(threadIdx.x) >> 6);
  const int64_t block = blockIdx.x;
  if (block < window_blocks) append_window<ACT, BITS, D, true>(a, t, block * kAppendWaves + wave, lds[wave]);
  else heads_wave<ACT, 0>(t, (block - window_blocks) * kAppendWaves + wave, k.G, k.steps, k.parts);
}

// ---------------------------------------------------------------------------
// Attention
// ---------------------------------------------------------------------------
//
// One workgroup of four or eight waves takes a split of a sequence for one key
// head and up to 16 of its query heads; the waves take its tiles of 32 tokens in
// turn. In matrix instructions of 16 x 16 x 32:
//   scores S[token, head] = K q^T: two row tiles of 16 tokens, keys as the row
//     operand straight from memory, queries (in registers all along) as the
//     column operand; a lane then holds tokens 4 g .. 4 g + 3 of either tile
//     (g = lane / 16) for head lane mod 16;
//   outputs O[channel, head] += V^T P^T: the same lane feeds its eight
//     probabilities as the column operand without moving one, because a
//     32-token tile of values is stored in that order of tokens.
// The running maximum is raised only when a score passes it by more than 2^8:
// until then exponentials stay below 2^8 and neither a maximum across lanes nor
// a rescaling of O is needed (fp16 caches: below); sums are per lane, joined at
// the end.
// Probabilities enter the second product as two 16-bit terms, the rounded value
// and what rounding left. The matrix units have room for it: the kernel is bound
// by the cache's bytes. Two bf16 terms leave at most 2^-16 of a probability,
// whatever its size (bf16 caches, and 8-bit ones, whose values widen to bf16). fp16 has no
// numbers below 2^-24, so there (fp16 caches) the exponentials are taken against
// the tile's own maximum, times 2^15, the second term times 2^12, and the tile's
// products enter O with one multiply-add by the tile's share: that leaves 2^-22
// of a probability and 2^-52 of the tile's largest, which for values of up to
// 65504 is below fp16's last step. Without it a key that is 17 nats ahead of 32767
// equal ones and has no value leaves an output that is 44 % off, at 18 nats zeros.
// It costs 0.2 us in the shortest call (300 tokens 6.3 -> 6.5) and less than 1 % in
// long ones (16 ragged sequences to 8192, 8 key heads of 128: 49.7 -> 49.9).
// 8-bit codes are widened to 16 bits exactly; the keys' scales multiply the
// scores, the values' scales the probabilities.
// Measured: 16 ragged sequences up to 32768 tokens, 8 key heads of 128 in 8 bits
// (519 MB) 81 us in shares (6.4 TB/s) and 4.2 for their join; 64 up to 4096, 16
// heads of 64, window 1500 (301 MB) 49.8 (6.0); one of 300 tokens 5.1, a chain of
// table, keys and values.

constexpr int kAttnWaves = 4, kManyWaves = 8;
constexpr int kFewBytes = 256;        // of a token's key, for the second

// Attended positions [lo, hi) of a sequence of n cached tokens, and their tiles.
struct Span {
  int lo, hi, t0, tiles;
};
__device__ __forceinline__ Span span_of(const AttnArgs& a, int n) {
  Span s;
  s.hi = n < 0 ? 0 : (n > a.max_len ? a.max_len : n);
  s.lo = a.window > 0 && s.hi > a.window ? s.hi - a.window : 0;
  s.t0 = s.lo / kTile;
  s.tiles = (s.hi + kTile - 1) / kTile - s.t0;
  return s;
}

// How the work is cut. An item is one sequence, key head and tile of 16 query
// heads; its tiles go to one or more workgroups, whose partial results lie in
// consecutive slots.
//   split (a.n_splits > 0): workgroup (split, item) takes split_tiles tiles.
//   shares (a.n_splits = 0): all items' tiles form one line, cut into equal
//     shares, one per workgroup, wherever the items end: sequences of unlike
//     lengths leave no workgroup with more than another. Workgroup w's part of
//     item i lies in slot w + i (one of the two grows from part to part).
// Sequence lengths are read on the device in both, and nothing else decides.
constexpr int kShareBatch = 1024;     // sequences that the shares' sums take

// Tiles of the sequences before b and of all of them, in every lane (B <=
// kShareBatch).
__device__ __forceinline__ void tiles_before(const AttnArgs& a, int b, int lane, int* before, int* all) {
  int x = 0, y = 0;
  for (int i = lane; i < a.B; i += 64) {
    const int n = span_of(a, a.lens[i]).tiles;
    y += n;
    x += i < b ? n : 0;
  }
#pragma unroll
  for (int o = 32; o; o >>= 1) {
    x += __shfl_xor(x, o);
    y += __shfl_xor(y, o);
  }
  *before = x;
  *all = y;
}
// Tiles of a share: a multiple of the waves, all of them equally loaded.
__device__ __forceinline__ int share_of(const AttnArgs& a, int tiles, int items_per_seq) {
  const int total = tiles * items_per_seq, r = (total + a.n_shares - 1) / a.n_shares;
  return (r + kAttnWaves - 1) / kAttnWaves * kAttnWaves;
}

// Block number of a tile of sequence b (counted from position 0); -1 past max_len.
__device__ __forceinline__ int block_at(const AttnArgs& a, int b, int tile) {
  const int most = (a.max_len + kTile - 1) / kTile;
  if (tile >= most) return -1;
  return a.table[b * a.ld_table + (static_cast<int64_t>(tile) * kTile >> __builtin_ctz(a.kv.block_tokens))];   // (a power of two)
}

template <int D, int W>
struct AttnLds {
  float o[W][16][D + 4];
  float m[W][16], l[W][16];
};

// Tiles [begin, end) of a sequence's span for one key head h and its query
// heads 16 qt and up, by the workgroup's W waves. ids: block numbers of the wave's first
// 64 tiles, one per lane. whole: no other workgroup has tiles of the item, the
// result goes to the output; else to slot `slot`.
template <int ACT, int BITS, int D, int W>
__device__ __forceinline__ void attend(const AttnArgs& a, AttnLds<D, W>& lds, int b, int h, int qt, const Span& sp, int begin,
                                       int end, int ids, bool whole, int64_t slot) {
  constexpr int kPv = BITS == 8 ? PW_BF16 : ACT;      // 16-bit type of the second product
  constexpr bool kByTile = kPv == PW_F16;             // exponentials against the tile's maximum
  constexpr int kLoads = D * BITS / 8 * 16 / 1024;    // 1 KB loads of 16 tokens' keys
  const int wave = __builtin_amdgcn_readfirstlane(static_cast<int>(threadIdx.x) >> 6), lane = lane_id();
  const int col = lane & 15, lg = lane >> 4;
  const int P = a.kv.block_tokens;
  const int first = begin + wave;                                // the wave's tiles: first, first + W, ...
  const int n_my = first < end ? (end - first + W - 1) / W : 0;

  const int g = a.n_q_heads / a.kv.n_kv_heads;
  const int n_col = g - 16 * qt < 16 ? g - 16 * qt : 16;
  const int hq0 = h * g + 16 * qt;
  u32x4 q[D / 32];
#pragma unroll
  for (int i = 0; i < D / 32; ++i) {
    q[i] = u32x4{0u, 0u, 0u, 0u};
    if (col < n_col)
      q[i] = ld16(reinterpret_cast<const uint8_t*>(a.q + b * a.ldq + (hq0 + col) * a.ldqh + 32 * i + 8 * lg));
  }

  // The tiles in blocks of the pool, one after the other (tiles in other blocks
  // are left out): bits of the 64 numbers at hand, then the next 64.
  int chunk = 0;
  uint64_t todo = __ballot(lane < n_my && ids >= 0 && ids < a.kv.n_blocks);
  int next_t = -1, next_id = 0;                                  // first token of the next tile (-1: none), its block
  const auto advance = [&] {
    while (todo == 0 && chunk + 64 < n_my) {
      chunk += 64;
      ids = chunk + lane < n_my ? block_at(a, b, sp.t0 + first + W * (chunk + lane)) : -1;
      todo = __ballot(ids >= 0 && ids < a.kv.n_blocks);
    }
    next_t = -1;
    if (todo) {
      const int l = __ffsll(static_cast<long long>(todo)) - 1;
      todo &= todo - 1;
      next_id = __builtin_amdgcn_readlane(ids, l);
      next_t = (sp.t0 + first + W * (chunk + l)) * kTile;
    }
  };
  const size_t head_off = static_cast<size_t>(2 * h) * P * D * (BITS / 8);
  const size_t v_off = static_cast<size_t>(P) * D * (BITS / 8);
  const size_t sc_off = static_cast<size_t>(2) * a.kv.n_kv_heads * P * D + static_cast<size_t>(h) * P * 4;
  const size_t vs_off = static_cast<size_t>(a.kv.n_kv_heads) * P * 4;
  const float scale2 = a.scale * kLog2e;

  u32x4 k[2][kLoads], v[2 * kLoads];
  f32x4 ks[2], vs[2];
  const auto load_k = [&] {
    const int t = next_t & (P - 1);                              // in the block
    const uint8_t* blk = a.kv.pool + static_cast<int64_t>(next_id) * a.kv.block_stride;
    const uint8_t* p = blk + head_off + static_cast<size_t>(t) * D * (BITS / 8) + 16 * lane;
#pragma unroll
    for (int r = 0; r < 2; ++r)
#pragma unroll
      for (int j = 0; j < kLoads; ++j) k[r][j] = ld16_nt(p + (r * kLoads + j) * 1024);
    if constexpr (BITS == 8) {
#pragma unroll
      for (int r = 0; r < 2; ++r) ks[r] = *reinterpret_cast<const f32x4*>(blk + sc_off + 4 * t + 16 * lg + 64 * r);
    }
  };
  const auto load_v = [&] {
    const int t = next_t & (P - 1);
    const uint8_t* blk = a.kv.pool + static_cast<int64_t>(next_id) * a.kv.block_stride;
    const uint8_t* p = blk + head_off + v_off + static_cast<size_t>(t) * D * (BITS / 8) + 16 * lane;
#pragma unroll
    for (int j = 0; j < 2 * kLoads; ++j) v[j] = ld16_nt(p + j * 1024);
    if constexpr (BITS == 8) {
#pragma unroll
      for (int r = 0; r < 2; ++r) vs[r] = *reinterpret_cast<const f32x4*>(blk + sc_off + vs_off + 4 * t + 16 * lg + 64 * r);
    }
  };

  f32x4 o[D / 16];
#pragma unroll
  for (int j = 0; j < D / 16; ++j) o[j] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
  float m = kNoMax, l = 0.0f;

  advance();
  if (next_t >= 0) {
    load_k();
    load_v();
  }
  while (next_t >= 0) {
    const int t = next_t;
    f32x4 s[2];
#pragma unroll
    for (int r = 0; r < 2; ++r) {
      s[r] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
      for (int j = 0; j < D / 32; ++j) {
        if constexpr (BITS == 16)
          s[r] = mma<ACT>(k[r][j], q[j], s[r]);
        else
          s[r] = mma<ACT>(widen8<ACT>(k[r][j / 2][2 * (j & 1)], k[r][j / 2][2 * (j & 1) + 1]), q[j], s[r]);
      }
    }
#pragma unroll
    for (int r = 0; r < 2; ++r)
#pragma unroll
      for (int e = 0; e < 4; ++e) s[r][e] *= BITS == 8 ? scale2 * ks[r][e] : scale2;
    // the tile at either end of the span: what lies outside is left out,
    // whatever its bits
    if (t < sp.lo || t + kTile > sp.hi) {
      uint32_t keep[2][2];                                       // of four tokens' 8 or 16 bits
#pragma unroll
      for (int r = 0; r < 2; ++r) {
        keep[r][0] = keep[r][1] = 0u;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int tok = t + 16 * r + 4 * lg + e;
          const bool in = tok >= sp.lo && tok < sp.hi;
          s[r][e] = in ? s[r][e] : -INFINITY;
          if constexpr (BITS == 8) {
            vs[r][e] = in ? vs[r][e] : 0.0f;
            keep[r][0] |= in ? 0xFFu << (8 * e) : 0u;
          } else {
            keep[r][e / 2] |= in ? 0xFFFFu << (16 * (e & 1)) : 0u;
          }
        }
      }
#pragma unroll
      for (int j = 0; j < 2 * kLoads; ++j)
#pragma unroll
        for (int w = 0; w < 4; ++w) v[j][w] &= BITS == 8 ? keep[w & 1][0] : keep[w / 2][w & 1];
    }
    advance();
    if (next_t >= 0) load_k();
    float top = s[0][0];
#pragma unroll
    for (int e = 1; e < 8; ++e) top = fmaxf(top, s[e / 4][e & 3]);
    float base = m;                                              // probabilities are exp2(s - base)
    float f = 1.0f, share = 1.0f;                                // factors of what is there and of this tile
    bool raise;
    if constexpr (kByTile) {
      top = fmaxf(column_max(top), kNoMax);                      // (a number, whatever the scores)
      raise = __any(top > m);
      const float m_new = fmaxf(m, top);
      f = __builtin_amdgcn_exp2f(m - m_new);
      share = __builtin_amdgcn_exp2f(top - m_new);
      base = top;
      m = m_new;
    } else {
      raise = __any(top > m + kSlack);
      if (raise) {
        const float m_new = fmaxf(m, column_max(top));
        f = __builtin_amdgcn_exp2f(m - m_new);
        base = m = m_new;
      }
    }
    if (raise) {
      l *= f;
#pragma unroll
      for (int j = 0; j < D / 16; ++j)
#pragma unroll
        for (int e = 0; e < 4; ++e) o[j][e] *= f;
    }
    float sum = 0.0f;
    u32x4 p_hi, p_lo;
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      float p[2];
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const int r = w / 2, x = 2 * (w & 1) + e;
        p[e] = __builtin_amdgcn_exp2f(s[r][x] - base);
        sum += p[e];
        if constexpr (BITS == 8) p[e] *= vs[r][x];
        if constexpr (kByTile) p[e] *= kLift;
      }
      p_hi[w] = pack16<kPv>(p[0], p[1]);
      p[0] -= val16(p_hi[w] & 0xFFFFu, kPv);
      p[1] -= val16(p_hi[w] >> 16, kPv);
      p_lo[w] = kByTile ? pack16<kPv>(p[0] * kLow, p[1] * kLow) : pack16<kPv>(p[0], p[1]);
    }
    l = fmaf(share, sum, l);
    if constexpr (kByTile) share *= 1.0f / kLift;
#pragma unroll
    for (int j = 0; j < D / 16; ++j) {
      u32x4 x;
      if constexpr (BITS == 16)
        x = v[j];
      else
        x = widen8<kPv>(v[j / 2][2 * (j & 1)], v[j / 2][2 * (j & 1) + 1]);
      if constexpr (kByTile) {
        const f32x4 zero{0.0f, 0.0f, 0.0f, 0.0f}, hi = mma<kPv>(x, p_hi, zero), lo = mma<kPv>(x, p_lo, zero);
#pragma unroll
        for (int e = 0; e < 4; ++e) o[j][e] = fmaf(share, fmaf(lo[e], 1.0f / kLow, hi[e]), o[j][e]);
        asm volatile("" : "+v"(o[j]));                           // (not all products before all sums: registers)
      } else {
        o[j] = mma<kPv>(x, p_hi, o[j]);
        o[j] = mma<kPv>(x, p_lo, o[j]);
      }
    }
    if (next_t >= 0) load_v();
  }

  // join the waves
  l += __shfl_xor(l, 16);
  l += __shfl_xor(l, 32);
  if (col < n_col) {
    if (lg == 0) {
      lds.m[wave][col] = m;
      lds.l[wave][col] = l;
    }
#pragma unroll
    for (int j = 0; j < D / 16; ++j) *reinterpret_cast<f32x4*>(&lds.o[wave][col][16 * j + 4 * lg]) = o[j];
  }
  __syncthreads();
  const int n_part = g < 16 ? g : 16;                            // rows of a slot
  for (int e = threadIdx.x; e < n_col * (D / 4); e += 64 * W) {
    const int c = e / (D / 4), d = 4 * (e % (D / 4));
    float mx = lds.m[0][c];
#pragma unroll
    for (int w = 1; w < W; ++w) mx = fmaxf(mx, lds.m[w][c]);
    f32x4 acc = {0.0f, 0.0f, 0.0f, 0.0f};
    float sum = 0.0f;
#pragma unroll
    for (int w = 0; w < W; ++w) {
      const float f = __builtin_amdgcn_exp2f(lds.m[w][c] - mx);
      sum = fmaf(f, lds.l[w][c], sum);
      const f32x4 x = *reinterpret_cast<const f32x4*>(&lds.o[w][c][d]);
#pragma unroll
      for (int j = 0; j < 4; ++j) acc[j] = fmaf(f, x[j], acc[j]);
    }
    if (whole) {
      const size_t row = static_cast<size_t>(b) * a.n_q_heads + hq0 + c;
      const float inv = sum == 0.0f ? 0.0f : 1.0f / sum;
      *reinterpret_cast<u32x2*>(a.out + row * D + d) =
          u32x2{pack16<ACT>(acc[0] * inv, acc[1] * inv), pack16<ACT>(acc[2] * inv, acc[3] * inv)};
      if (a.lse && d == 0) a.lse[row] = sum == 0.0f ? -INFINITY : (mx + log2f(sum)) * kLn2;
    } else {
      const size_t at = static_cast<size_t>(slot) * n_part + c;
      *reinterpret_cast<f32x4*>(a.part_o + at * D + d) = acc;
      if (d == 0) {
        a.part_ml[2 * at] = mx;
        a.part_ml[2 * at + 1] = sum;
      }
    }
  }
}

template <int ACT, int BITS, int D, int W>
__global__ __launch_bounds__(64 * W, D <= 128 || W > kAttnWaves ? 2 : 1) void k_attn(AttnArgs a, int q_tiles) {
  __shared__ AttnLds<D, W> lds;
  const int split = blockIdx.x, b = blockIdx.z;
  const int h = q_tiles == 1 ? blockIdx.y : blockIdx.y / q_tiles, qt = q_tiles == 1 ? 0 : blockIdx.y % q_tiles;
  const int wave = static_cast<int>(threadIdx.x) >> 6, lane = lane_id();
  const int begin = split * a.split_tiles;
  // Without a window the block numbers do not hang on the sequence's length, so
  // they come along with it (what lies past the length is dropped later).
  int ids = a.window == 0 ? block_at(a, b, begin + wave + W * lane) : -1;
  const Span sp = span_of(a, a.lens[b]);
  const int n_act = (sp.tiles + a.split_tiles - 1) / a.split_tiles;
  if (split > 0 && split >= n_act) return;
  if (a.window > 0) ids = block_at(a, b, sp.t0 + begin + wave + W * lane);
  const int end = begin + a.split_tiles < sp.tiles ? begin + a.split_tiles : sp.tiles;
  const int64_t item = static_cast<int64_t>(b) * gridDim.y + blockIdx.y;
  attend<ACT, BITS, D, W>(a, lds, b, h, qt, sp, begin, end, ids, n_act <= 1, item * a.n_splits + split);
}

// The workgroup's share, an item's part after the other.
template <int ACT, int BITS, int D>
__global__ __launch_bounds__(64 * kAttnWaves, D <= 128 ? 2 : 1) void k_attn_shares(AttnArgs a, int q_tiles) {
  __shared__ AttnLds<D, kAttnWaves> lds;
  const int w = blockIdx.x, wave = static_cast<int>(threadIdx.x) >> 6, lane = lane_id();
  const int per_seq = a.kv.n_kv_heads * q_tiles;                 // items of a sequence
  // lane l sums sequences l per .. (l + 1) per - 1, then the lanes' sums
  const int per = (a.B + 63) / 64;
  int sum = 0;
  for (int i = lane * per; i < (lane + 1) * per && i < a.B; ++i) sum += span_of(a, a.lens[i]).tiles;
  int upto = sum;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const int x = __shfl_up(upto, o);
    if (lane >= o) upto += x;
  }
  const int r = share_of(a, __builtin_amdgcn_readlane(upto, 63), per_seq);
  const int total = __builtin_amdgcn_readlane(upto, 63) * per_seq;
  // (the products below stay below 2^31: checked on the host for max_len)
  int pos = w * r < total && r > 0 ? w * r : total;
  const int stop = total - pos < r ? total : pos + r;
  if (pos >= stop) return;
  // the sequence at `pos`: the first lane whose sums reach past it, then its sequences
  const int l = __ffsll(static_cast<long long>(__ballot(upto * per_seq > pos))) - 1;
  int b = l * per;
  int start = (__builtin_amdgcn_readlane(upto, l) - __builtin_amdgcn_readlane(sum, l)) * per_seq;   // of sequence b
  Span sp = span_of(a, a.lens[b]);
  while (start + sp.tiles * per_seq <= pos) {
    start += sp.tiles * per_seq;
    sp = span_of(a, a.lens[++b]);
  }
  while (true) {
    const int item = (pos - start) / sp.tiles, begin = pos - start - item * sp.tiles;
    const int n = min(sp.tiles - begin, stop - pos);
    const int h = item / q_tiles, qt = item % q_tiles;
    const int ids = block_at(a, b, sp.t0 + begin + wave + kAttnWaves * lane);
    attend<ACT, BITS, D, kAttnWaves>(a, lds, b, h, qt, sp, begin, begin + n, ids, n == sp.tiles,
                         w + static_cast<int64_t>(b) * per_seq + item);
    pos += n;
    if (pos >= stop) return;
    __syncthreads();                                             // the joins above read LDS
    while (start + sp.tiles * per_seq <= pos) {
      start += sp.tiles * per_seq;
      sp = span_of(a, a.lens[++b]);
    }
  }
}

// Joins the parts of one row (sequence and query head), and writes the rows of
// empty sequences where no workgroup has them. Four waves take every fourth part
// and join in a fixed order.
template <int ACT, int D>
__global__ __launch_bounds__(256) void k_attn_join(AttnArgs a) {
  constexpr int kC = D / 64;
  __shared__ float lds_o[4][D], lds_l[4];
  const int wave = static_cast<int>(threadIdx.x) >> 6, lane = lane_id();
  const int b = blockIdx.y, hq = blockIdx.x, g = a.n_q_heads / a.kv.n_kv_heads;
  const int q_tiles = (g + 15) / 16, n_part = g < 16 ? g : 16, per_seq = a.kv.n_kv_heads * q_tiles;
  const int item = hq / g * q_tiles + hq % g / 16;               // of the sequence
  const Span sp = span_of(a, a.lens[b]);
  int64_t slot;
  int n;
  if (a.n_splits > 0) {
    slot = (static_cast<int64_t>(b) * per_seq + item) * a.n_splits;
    n = (sp.tiles + a.split_tiles - 1) / a.split_tiles;
    if (n <= 1) return;
  } else {
    int before, all;
    tiles_before(a, b, lane, &before, &all);
    const int r = share_of(a, all, per_seq), start = before * per_seq + item * sp.tiles;
    if (sp.tiles > 0) {
      n = (start + sp.tiles - 1) / r - start / r + 1;
      slot = start / r + static_cast<int64_t>(b) * per_seq + item;
      if (n == 1) return;
    } else {
      n = 0;
      slot = 0;
    }
  }
  const size_t row = static_cast<size_t>(b) * a.n_q_heads + hq;
  const size_t at = static_cast<size_t>(slot) * n_part + hq % g % 16;
  float mx = kNoMax;
  for (int s = lane; s < n; s += 64) mx = fmaxf(mx, a.part_ml[2 * (at + static_cast<size_t>(s) * n_part)]);
#pragma unroll
  for (int o = 32; o; o >>= 1) mx = fmaxf(mx, __shfl_xor(mx, o));
  float acc[kC] = {}, sum = 0.0f;
#pragma unroll 4
  for (int s = wave; s < n; s += 4) {
    const size_t x = at + static_cast<size_t>(s) * n_part;
    const float f = __builtin_amdgcn_exp2f(a.part_ml[2 * x] - mx);
    sum = fmaf(f, a.part_ml[2 * x + 1], sum);
#pragma unroll
    for (int j = 0; j < kC; ++j) acc[j] = fmaf(f, a.part_o[x * D + 64 * j + lane], acc[j]);
  }
#pragma unroll
  for (int j = 0; j < kC; ++j) lds_o[wave][64 * j + lane] = acc[j];
  if (lane == 0) lds_l[wave] = sum;
  __syncthreads();
  sum = (lds_l[0] + lds_l[1]) + (lds_l[2] + lds_l[3]);
  const float inv = sum == 0.0f ? 0.0f : 1.0f / sum;
  for (int d = threadIdx.x; d < D; d += 256)
    a.out[row * D + d] =
        static_cast<uint16_t>(pack16<ACT>(((lds_o[0][d] + lds_o[1][d]) + (lds_o[2][d] + lds_o[3][d])) * inv, 0.0f));
  if (a.lse && threadIdx.x == 0) a.lse[row] = sum == 0.0f ? -INFINITY : (mx + log2f(sum)) * kLn2;
}

template <int ACT, int BITS, int D>
hipError_t launch_attn_d(const AttnArgs& a, hipStream_t st) {
  const int g = a.n_q_heads / a.kv.n_kv_heads, q_tiles = (g + 15) / 16;
  const dim3 items(a.n_splits, a.kv.n_kv_heads * q_tiles, a.B);
  constexpr int kMost = D * BITS / 8 <= kFewBytes ? kManyWaves : kAttnWaves;
  if (a.n_splits > 0 && a.many_waves)
    k_attn<ACT, BITS, D, kMost><<<items, 64 * kMost, 0, st>>>(a, q_tiles);
  else if (a.n_splits > 0)
    k_attn<ACT, BITS, D, kAttnWaves><<<items, 64 * kAttnWaves, 0, st>>>(a, q_tiles);
  else
    k_attn_shares<ACT, BITS, D><<<a.n_shares, 64 * kAttnWaves, 0, st>>>(a, q_tiles);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || a.n_splits == 1) return e;
  k_attn_join<ACT, D><<<dim3(a.n_q_heads, a.B), 256, 0, st>>>(a);
  return hipGetLastError();
}

template <int ACT, int BITS>
hipError_t launch_attn_bits(const AttnArgs& a, hipStream_t st) {
  switch (a.kv.head_dim) {
    case 64: return launch_attn_d<ACT, BITS, 64>(a, st);
    case 128: return launch_attn_d<ACT, BITS, 128>(a, st);
    case 192: return launch_attn_d<ACT, BITS, 192>(a, st);
    case 256: return launch_attn_d<ACT, BITS, 256>(a, st);
  }
  return hipErrorInvalidValue;
}

}  // namespace

// How the work is cut (see above).
AttnPlan attn_plan(int B, int n_q_heads, int n_kv_heads, int head_dim, int bits, int max_len, int window) {
  AttnPlan p{1, kManyWaves, 0, 0, 0};
  int64_t tiles = (static_cast<int64_t>(max_len) + kTile - 1) / kTile;
  if (window > 0) {
    const int64_t w = (static_cast<int64_t>(window) + 2 * kTile - 2) / kTile;   // a window that starts inside a tile
    tiles = w < tiles ? w : tiles;
  }
  const int64_t g = n_q_heads / n_kv_heads, q_tiles = (g + 15) / 16, rows = g < 16 ? g : 16;
  const int64_t items = static_cast<int64_t>(B) * n_kv_heads * q_tiles;
  if (items == 0 || tiles == 0) return p;
  const size_t slot = static_cast<size_t>(rows) * (head_dim + 2) * sizeof(float);
  // as many workgroups as the chip holds at once, by the kernels' registers
  const int64_t resident = 256 * (head_dim <= 64 ? 4 : head_dim <= 128 ? 3 : head_dim <= 192 ? 2 : 1);
  // Equal shares cost each workgroup the sums over the lengths and, where an item
  // ends inside its share, a second start, and they need the join; splits leave
  // unlike lengths unbalanced. 16 bits, 8 key heads of 128 channels, ragged (us,
  // shares / splits): 64 sequences up to 8192 tokens 166 / 206, up to 4096 92.6 /
  // 108, up to 2048 56 / 58 (in 8 bits 42 / 36); 16 up to 8192 51 / 61, up to 4096
  // 31 / 35; 256 up to 2048, more items than workgroups, 207 / 171.
  if (B > 1 && B <= kShareBatch && items <= resident && tiles >= 96 && items * tiles >= 16 * resident &&
      items * tiles < (int64_t(1) << 31) - (1 << 20)) {
    p.n_splits = 0;
    p.n_shares = static_cast<int>(resident);
    p.ws_bytes = static_cast<size_t>(resident + items) * slot;
    return p;
  }
  // A CU reads 57 KB/us at most, which four waves reach with more than 16 KB each
  // in flight; smaller tiles take eight where there are no more workgroups than
  // CUs. Eight / four waves (us): 8 bits, 4 sequences of 1000 tokens with 8 key
  // heads of 128 9.6 / 12.3, 16 of them 11.5 / 13.3, 32 of 1300 16.4 / 18.3; heads
  // of 64 in 16 bits, 4 of 1500 10.3 / 13.0; of 256 in 8 bits, 16 of 600 13.3 /
  // 14.6; of 128 in 16 bits 12.9 / 13.0.
  // A second workgroup per item costs the join, 5 to 6 us with its launch: it is
  // left out where one workgroup takes no longer than that over the tiles, and
  // where there is an item for every CU. 16 bits, 8 key heads, one workgroup /
  // split (us): 128 channels, 4 sequences of 1000 tokens 13.0 / 15.3, of 1300
  // 14.6 / 16.8, of 1600 18.1 / 16.4; 256 channels, of 400 12.4 / 16.2, of 800
  // 18.8 / 18.2 (16.6 in finer splits); 2 key heads of 128, 64 sequences of 516
  // 10.4 / 17.5. From 256 items on: 32 sequences of 2000 42.6 / 48.7, of 2900 61.0
  // / 67.2, ragged 37.7 / 42.9, in 8 bits 34.5 / 38.6, ragged 30.7 / 26.7; 40 of
  // 2000 61.5 / 58.5.
  const int row = head_dim * bits / 8;
  int64_t n = 1;
  if (tiles * (row < 128 ? 128 : row) > 40 * 256 && items < 256) {
    const int64_t most = (tiles + 15) / 16;
    n = (resident + items - 1) / items;
    n = n < most ? n : most;
  }
  const int64_t per = ((tiles + n - 1) / n + kManyWaves - 1) / kManyWaves * kManyWaves;
  n = (tiles + per - 1) / per;
  p.split_tiles = static_cast<int>(per);
  p.n_splits = static_cast<int>(n);
  p.many_waves = row <= kFewBytes && items * n <= 256;
  if (n > 1) p.ws_bytes = static_cast<size_t>(items * n) * slot;
  return p;
}

namespace {

template <int ACT, int BITS>
hipError_t append_tiles(const AppendArgs& a, hipStream_t st) {
  const int64_t units = (static_cast<int64_t>(a.T) + 31) / 32 * a.kv.n_kv_heads * 2;
  const int64_t grid = (units + kAppendWaves - 1) / kAppendWaves;
  if (grid >= (1 << 23)) return hipErrorInvalidConfiguration;
  const dim3 g(static_cast<uint32_t>(grid)), b(64 * kAppendWaves);
  switch (a.kv.head_dim) {
    case 64: k_kv_append_tiles<ACT, BITS, 64><<<g, b, 0, st>>>(a); break;
    case 128: k_kv_append_tiles<ACT, BITS, 128><<<g, b, 0, st>>>(a); break;
    case 192: k_kv_append_tiles<ACT, BITS, 192><<<g, b, 0, st>>>(a); break;
    case 256: k_kv_append_tiles<ACT, BITS, 256><<<g, b, 0, st>>>(a); break;
    default: return hipErrorInvalidValue;
  }
  return hipGetLastError();
}

template <int ACT, int BITS>
hipError_t append(const AppendArgs& a, hipStream_t st) {
  const int64_t all = static_cast<int64_t>(a.T) * a.kv.n_kv_heads;
  if (a.T >= kAppendMany && all >= (BITS == 16 ? kRunItems16 : kRunItems8)) return append_tiles<ACT, BITS>(a, st);
  int G = 8;
  while (8 * G < a.kv.head_dim) G *= 2;
  const int64_t per = 256 / G, items = static_cast<int64_t>(a.T) * a.kv.n_kv_heads * 2;
  const int64_t blocks = (items + per - 1) / per;
  k_kv_append<ACT, BITS><<<static_cast<uint32_t>(blocks), 256, 0, st>>>(a, G);
  return hipGetLastError();
}

template <int ACT, int BITS>
hipError_t append_runs(const HeadsArgs& t, hipStream_t st) {
  const AppendArgs a{t.kv, t.k, t.v, t.ldk, t.ldkh, t.slots, t.T};
  HeadsArgs q = t;                                               // the queries alone
  q.n_k = 0;
  const HeadsCut k = heads_cut(t.T, t.D, t.n_q);
  const int64_t windows = ((static_cast<int64_t>(t.T) + 31) / 32 * t.n_k * 2 + kAppendWaves - 1) / kAppendWaves;
  const int64_t grid = windows + (t.n_q ? k.blocks : 0);
  if (grid >= (1 << 24)) return hipErrorInvalidConfiguration;
  const dim3 g(static_cast<uint32_t>(grid)), b(64 * kAppendWaves);
  switch (t.D) {
    case 64: k_append_runs<ACT, BITS, 64><<<g, b, 0, st>>>(a, q, k, windows); break;
    case 128: k_append_runs<ACT, BITS, 128><<<g, b, 0, st>>>(a, q, k, windows); break;
    case 192: k_append_runs<ACT, BITS, 192><<<g, b, 0, st>>>(a, q, k, windows); break;
    case 256: k_append_runs<ACT, BITS, 256><<<g, b, 0, st>>>(a, q, k, windows); break;
    default: return hipErrorInvalidValue;
  }
  return hipGetLastError();
}

}  // namespace

// By runs, where a pair lies in one lane there: from 16384 tokens x heads on. By runs each
// key head has the angles of its tokens for itself, so in 16 bits that is later than in
// pw_kv_append. 32 query and 8 key heads of 128 in bf16, consecutive positions, by runs
// and by tokens (us): 16 bits 768 tokens 18.9 and 13.4, 1536 tokens 22.5
// and 19.8; 2304 tokens 25.3 and 31.3, 4001 29.8 and 40.4; 8 bits 2304 tokens 26.9 and 27.5,
// 4001 31.0 and 33.2. Slots in no order: 16 bits 768 tokens 25.7 and 13.5.
bool append_by_runs(const HeadsArgs& a) {
  return a.T >= kAppendMany && static_cast<int64_t>(a.T) * a.n_k >= kRunItems8 && (a.rot.interleaved || a.rot.R % 64 == 0);
}

hipError_t launch_append_runs(const HeadsArgs& a, hipStream_t st) {
  if (a.act == PW_BF16) return a.kv.bits == 16 ? append_runs<PW_BF16, 16>(a, st) : append_runs<PW_BF16, 8>(a, st);
  return a.kv.bits == 16 ? append_runs<PW_F16, 16>(a, st) : append_runs<PW_F16, 8>(a, st);
}

hipError_t launch_kv_append(const AppendArgs& a, hipStream_t st) {
  if (a.kv.act == PW_BF16) return a.kv.bits == 16 ? append<PW_BF16, 16>(a, st) : append<PW_BF16, 8>(a, st);
  return a.kv.bits == 16 ? append<PW_F16, 16>(a, st) : append<PW_F16, 8>(a, st);
}

hipError_t launch_attn(const AttnArgs& a, hipStream_t st) {
  if (a.kv.act == PW_BF16)
    return a.kv.bits == 16 ? launch_attn_bits<PW_BF16, 16>(a, st) : launch_attn_bits<PW_BF16, 8>(a, st);
  return a.kv.bits == 16 ? launch_attn_bits<PW_F16, 16>(a, st) : launch_attn_bits<PW_F16, 8>(a, st);
}

}  // namespace pw
