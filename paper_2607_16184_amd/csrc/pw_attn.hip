// Paged KV cache, gfx950: writing new tokens into it (k_kv_append) and the
// attention of one new token per sequence over it (k_attn, k_attn_join).
#include "pw_device.hpp"
#include "pw_ops.hpp"

namespace pw {
namespace {

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

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
  const int D = a.kv.head_dim, P = a.kv.block_tokens, H = a.kv.n_kv_heads;
  const int t = static_cast<int>(slot % P);
  uint8_t* blk = a.kv.pool + slot / P * a.kv.block_stride;
  uint8_t* dst = blk + static_cast<size_t>(2 * h + is_v) * P * D * (BITS / 8);
  if constexpr (BITS == 16) {
    if (8 * c >= D) return;
    if (!is_v) {
      *reinterpret_cast<u32x4*>(dst + ((t / 16) * (D / 32) + c / 4) * 1024 + 16 * (16 * (c & 3) + t % 16)) = raw;
    } else {
      uint16_t* p = reinterpret_cast<uint16_t*>(dst + ((t / 32) * (D / 16) + c / 2) * 1024) +
                    8 * (16 * (t / 4 % 4) + 8 * (c & 1)) + 4 * (t / 16 % 2) + t % 4;
#pragma unroll
      for (int j = 0; j < 8; ++j) p[8 * j] = static_cast<uint16_t>(raw[j / 2] >> (16 * (j & 1)));
    }
  } else {
    float f[8], m = 0.0f;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      f[j] = val16(raw[j / 2] >> (16 * (j & 1)), ACT);
      m = fmaxf(m, fabsf(f[j]));
    }
    for (int o = G / 2; o; o >>= 1) m = fmaxf(m, __shfl_xor(m, o));
    const float s = f8_scale(m);
    if (8 * c >= D) return;
    const u32x2 q = f8_codes8(f, s);
    if (!is_v) {
      *reinterpret_cast<u32x2*>(dst + ((t / 16) * (D / 64) + c / 8) * 1024 + 16 * (16 * (c & 3) + t % 16) +
                                8 * (c / 4 % 2)) = q;
    } else {
      uint8_t* p = dst + ((t / 32) * (D / 32) + c / 4) * 1024 + 16 * (16 * (t / 4 % 4) + 8 * (c & 1)) +
                   8 * (c / 2 % 2) + 4 * (t / 16 % 2) + t % 4;
#pragma unroll
      for (int j = 0; j < 8; ++j) p[16 * j] = static_cast<uint8_t>(q[j / 4] >> (8 * (j & 3)));
    }
    if (c == 0) {
      float* sc = reinterpret_cast<float*>(blk + static_cast<size_t>(2) * H * P * D);
      sc[(is_v * H + h) * P + t] = s;
    }
  }
}
__device__ __forceinline__ bool slot_ok(const AppendArgs& a, int64_t slot) {
  return slot >= 0 && slot / a.kv.block_tokens < a.kv.n_blocks;
}

// Few tokens, or none next to each other (a decode step): G lanes per token,
// head and side.
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
// turned in LDS. Tokens of runs shorter than kMinRun go one by one. (A value's
// elements lie 16 bytes apart: written token by token, 4001 tokens of 8 heads
// x 128 channels take 25.8 us in 16 bits and 18.2 in 8, as runs 8.3 and 10.4.
// Tokens in no order lose by it, 512 of them 7.0 -> 13.6 us, and from 256 in a row
// on runs win: the kernel is taken from kAppendMany on, where a step's tokens
// are hardly those of a decode batch.)
constexpr int kAppendWaves = 4;
constexpr int kAppendMany = 512;          // tokens
constexpr int kMinRun = 8;
template <int ACT, int BITS, int D>
__global__ __launch_bounds__(64 * kAppendWaves) void k_kv_append_tiles(AppendArgs a) {
  constexpr int kE = BITS / 8, kPitch = D * kE + 4;
  __shared__ __attribute__((aligned(16))) uint8_t lds[kAppendWaves][32 * kPitch];
  const int wave = __builtin_amdgcn_readfirstlane(static_cast<int>(threadIdx.x) >> 6), lane = lane_id();
  const int H = a.kv.n_kv_heads, P = a.kv.block_tokens;
  const int64_t unit = static_cast<int64_t>(blockIdx.x) * kAppendWaves + wave;
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
    uint8_t* mine = lds[wave];
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      uint8_t* row = mine + (16 * u + c) * kPitch + 8 * lg * kE;
      const bool here = in(16 * u + c);
      if constexpr (BITS == 16) {
#pragma unroll
        for (int i = 0; i < D / 32; ++i) {
          if (!is_v) {
            if (here) *reinterpret_cast<u32x4*>(dst + (u * (D / 32) + i) * 1024 + 16 * lane) = x[u][i];
          } else {
#pragma unroll
            for (int w = 0; w < 4; ++w) *reinterpret_cast<uint32_t*>(row + 64 * i + 4 * w) = x[u][i][w];
          }
        }
      } else {
        float m = 0.0f;
#pragma unroll
        for (int i = 0; i < D / 32; ++i)
#pragma unroll
          for (int j = 0; j < 8; ++j) m = fmaxf(m, fabsf(val16(x[u][i][j / 2] >> (16 * (j & 1)), ACT)));
        m = fmaxf(m, __shfl_xor(m, 16));
        m = fmaxf(m, __shfl_xor(m, 32));
        const float s = f8_scale(m);
        u32x2 q[D / 32];
#pragma unroll
        for (int i = 0; i < D / 32; ++i) {
          float f[8];
#pragma unroll
          for (int j = 0; j < 8; ++j) f[j] = val16(x[u][i][j / 2] >> (16 * (j & 1)), ACT);
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
            for (int w = 0; w < 4; ++w) *reinterpret_cast<uint32_t*>(row + 32 * (i + w / 2) + 4 * (w & 1)) = q[i + w / 2][w & 1];
          }
        }
      }
    }
    if (is_v) {
      __builtin_amdgcn_wave_barrier();                           // the wave's own LDS: in order
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
              o |= static_cast<uint32_t>(*reinterpret_cast<const uint16_t*>(mine + tok * kPitch + 2 * (16 * j + c))) << (16 * e);
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
      __builtin_amdgcn_wave_barrier();
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
      if ((single >> n) & 1ull) append_one<ACT, BITS>(a, raw[j], slot, h, is_v, c, G);
    }
  }
}

// ---------------------------------------------------------------------------
// Attention
// ---------------------------------------------------------------------------
//
// One workgroup of four waves takes a split of a sequence for one key head and
// up to 16 of its query heads; a wave takes every fourth tile of 32 tokens. In
// matrix instructions of 16 x 16 x 32:
//   scores S[token, head] = K q^T: two row tiles of 16 tokens, keys as the row
//     operand straight from memory, queries (in registers all along) as the
//     column operand; a lane then holds tokens 4 g .. 4 g + 3 of either tile
//     (g = lane / 16) for head lane mod 16;
//   outputs O[channel, head] += V^T P^T: the same lane feeds its eight
//     probabilities as the column operand without moving one, because a
//     32-token tile of values is stored in that order of tokens.
// The running maximum is raised only when a score passes it by more than 2^8:
// until then exponentials stay below 2^8 and neither a maximum across lanes nor
// a rescaling of O is needed; sums are per lane, joined at the end.
// Probabilities enter the second product as two 16-bit terms (the rounded
// value and what rounding left), so O carries fp32's error, not 16 bits'. The
// matrix units have room for it: the kernel is bound by the cache's bytes.
// 8-bit codes are widened to 16 bits exactly; the keys' scales multiply the
// scores, the values' scales the probabilities.

constexpr int kTile = 32;
constexpr int kAttnWaves = 4;
constexpr float kNoMax = -1e30f;      // below every score, and exp2(-inf - it) = 0
constexpr float kSlack = 8.0f;

// Attended positions [lo, hi) of sequence b, and their tiles.
struct Span {
  int lo, hi, t0, tiles;
};
__device__ __forceinline__ Span span_of(const AttnArgs& a, int b) {
  Span s;
  const int n = a.lens[b];
  s.hi = n < 0 ? 0 : (n > a.max_len ? a.max_len : n);
  s.lo = a.window > 0 && s.hi > a.window ? s.hi - a.window : 0;
  s.t0 = s.lo / kTile;
  s.tiles = (s.hi + kTile - 1) / kTile - s.t0;
  return s;
}

// Two e4m3 codes (the low or high half of a word) as two 16-bit values.
template <int ACT, bool HI>
__device__ __forceinline__ uint32_t widen2(uint32_t c) {
  if constexpr (ACT == PW_BF16)
    return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(c, 1.0f, HI));
  else
    return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(c, 1.0f, HI));
}
template <int ACT>
__device__ __forceinline__ u32x4 widen8(uint32_t lo, uint32_t hi) {
  return u32x4{widen2<ACT, false>(lo), widen2<ACT, true>(lo), widen2<ACT, false>(hi), widen2<ACT, true>(hi)};
}

template <int ACT, int BITS, int D>
__global__ __launch_bounds__(64 * kAttnWaves, D <= 128 ? 2 : 1) void k_attn(AttnArgs a, int q_tiles) {
  constexpr int kPv = BITS == 8 ? PW_BF16 : ACT;      // 16-bit type of the second product
  constexpr int kLoads = D * BITS / 8 * 16 / 1024;    // 1 KB loads of 16 tokens' keys
  constexpr int kPad = D + 4;
  __shared__ float lds_o[kAttnWaves][16][kPad];
  __shared__ float lds_m[kAttnWaves][16], lds_l[kAttnWaves][16];

  const int split = static_cast<int>(blockIdx.x) % a.n_splits, item = static_cast<int>(blockIdx.x) / a.n_splits;
  const int qt = item % q_tiles, h = item / q_tiles % a.kv.n_kv_heads;
  const int b = item / q_tiles / a.kv.n_kv_heads;
  const Span sp = span_of(a, b);
  const int n_act = (sp.tiles + a.split_tiles - 1) / a.split_tiles;
  if (split > 0 && split >= n_act) return;

  const int wave = __builtin_amdgcn_readfirstlane(static_cast<int>(threadIdx.x) >> 6), lane = lane_id();
  const int col = lane & 15, lg = lane >> 4;
  const int g = a.n_q_heads / a.kv.n_kv_heads;
  const int n_col = g - 16 * qt < 16 ? g - 16 * qt : 16;
  const int hq0 = h * g + 16 * qt;
  const int P = a.kv.block_tokens, p_shift = __builtin_ctz(P);   // a power of two

  u32x4 q[D / 32];
#pragma unroll
  for (int i = 0; i < D / 32; ++i) {
    q[i] = u32x4{0u, 0u, 0u, 0u};
    if (col < n_col)
      q[i] = ld16(reinterpret_cast<const uint8_t*>(a.q + b * a.ldq + (hq0 + col) * a.ldqh + 32 * i + 8 * lg));
  }

  const int first = split * a.split_tiles + wave;                 // the wave's tiles: first, first + 4, ...
  int end = (split + 1) * a.split_tiles;
  end = end < sp.tiles ? end : sp.tiles;
  const int n_my = first < end ? (end - first + kAttnWaves - 1) / kAttnWaves : 0;
  const int32_t* table = a.table + b * a.ld_table;
  const size_t head_off = static_cast<size_t>(2 * h) * P * D * (BITS / 8);
  const size_t v_off = static_cast<size_t>(P) * D * (BITS / 8);
  const size_t sc_off = static_cast<size_t>(2) * a.kv.n_kv_heads * P * D + (static_cast<size_t>(h) * P + 4 * lg) * 4;
  const float scale2 = a.scale * kLog2e;

  u32x4 k[2][kLoads], v[2 * kLoads];
  f32x4 ks[2], vs[2];
  const auto tile_of = [&](int i) { return sp.t0 + first + kAttnWaves * i; };
  // block numbers of the wave's next 64 tiles, one per lane
  int ids = 0;
  const auto fetch_ids = [&](int i) {
    const int j = i + lane;
    ids = j < n_my ? table[tile_of(j) * kTile >> p_shift] : -1;
  };
  const auto block_of = [&](int i) { return __builtin_amdgcn_readlane(ids, i & 63); };
  const auto ok = [&](int id) { return id >= 0 && id < a.kv.n_blocks; };
  const auto load_k = [&](int i, int id) {
    if (!ok(id)) return;
    const int t = tile_of(i) * kTile & (P - 1);                         // first token in the block
    const uint8_t* blk = a.kv.pool + static_cast<int64_t>(id) * a.kv.block_stride;
    const uint8_t* p = blk + head_off + static_cast<size_t>(t) * D * (BITS / 8) + 16 * lane;
#pragma unroll
    for (int r = 0; r < 2; ++r)
#pragma unroll
      for (int j = 0; j < kLoads; ++j) k[r][j] = ld16_nt(p + (r * kLoads + j) * 1024);
    if constexpr (BITS == 8) {
#pragma unroll
      for (int r = 0; r < 2; ++r)
        ks[r] = *reinterpret_cast<const f32x4*>(blk + sc_off + 4 * t + 64 * r);
    }
  };
  const auto load_v = [&](int i, int id) {
    if (!ok(id)) return;
    const int t = tile_of(i) * kTile & (P - 1);
    const uint8_t* blk = a.kv.pool + static_cast<int64_t>(id) * a.kv.block_stride;
    const uint8_t* p = blk + head_off + v_off + static_cast<size_t>(t) * D * (BITS / 8) + 16 * lane;
#pragma unroll
    for (int j = 0; j < 2 * kLoads; ++j) v[j] = ld16_nt(p + j * 1024);
    if constexpr (BITS == 8) {
#pragma unroll
      for (int r = 0; r < 2; ++r)
        vs[r] = *reinterpret_cast<const f32x4*>(blk + sc_off + static_cast<size_t>(a.kv.n_kv_heads) * P * 4 + 4 * t + 64 * r);
    }
  };

  f32x4 o[D / 16];
#pragma unroll
  for (int j = 0; j < D / 16; ++j) o[j] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
  float m = kNoMax, l = 0.0f;

  int id = -1;
  if (n_my > 0) {
    fetch_ids(0);
    id = block_of(0);
    load_k(0, id);
    load_v(0, id);
  }
  for (int i = 0; i < n_my; ++i) {
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
    f32x4 vsc[2];
    if constexpr (BITS == 8) {
      vsc[0] = vs[0];
      vsc[1] = vs[1];
    }
    // a tile at either end of the span, or in a missing block: what lies
    // outside is left out, whatever its bits
    const int t = tile_of(i) * kTile;
    const bool edge = t < sp.lo || t + kTile > sp.hi || !ok(id);
    if (edge) {
#pragma unroll
      for (int r = 0; r < 2; ++r) {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int tok = t + 16 * r + 4 * lg + e;
          const bool in = tok >= sp.lo && tok < sp.hi && ok(id);
          s[r][e] = in ? s[r][e] : -INFINITY;
          if constexpr (BITS == 8) vsc[r][e] = in ? vsc[r][e] : 0.0f;
        }
      }
    }
    int next = -1;
    if (i + 1 < n_my) {
      if (((i + 1) & 63) == 0) fetch_ids(i + 1);
      next = block_of(i + 1);
      load_k(i + 1, next);
    }
    float top = s[0][0];
#pragma unroll
    for (int e = 1; e < 8; ++e) top = fmaxf(top, s[e / 4][e & 3]);
    if (__any(top > m + kSlack)) {
      top = fmaxf(top, __shfl_xor(top, 16));
      top = fmaxf(top, __shfl_xor(top, 32));
      const float m_new = fmaxf(m, top);
      const float f = exp2f(m - m_new);
      m = m_new;
      l *= f;
#pragma unroll
      for (int j = 0; j < D / 16; ++j)
#pragma unroll
        for (int e = 0; e < 4; ++e) o[j][e] *= f;
    }
    u32x4 p_hi, p_lo;
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      float p[2];
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const int r = w / 2, x = 2 * (w & 1) + e;
        p[e] = exp2f(s[r][x] - m);
        l += p[e];
        if constexpr (BITS == 8) p[e] *= vsc[r][x];
      }
      p_hi[w] = pack16<kPv>(p[0], p[1]);
      p_lo[w] = pack16<kPv>(p[0] - val16(p_hi[w] & 0xFFFFu, kPv), p[1] - val16(p_hi[w] >> 16, kPv));
    }
#pragma unroll
    for (int j = 0; j < D / 16; ++j) {
      u32x4 x;
      if constexpr (BITS == 16)
        x = v[j];
      else
        x = widen8<kPv>(v[j / 2][2 * (j & 1)], v[j / 2][2 * (j & 1) + 1]);
      if (edge) {
#pragma unroll
        for (int w = 0; w < 4; ++w) {
          uint32_t keep = 0u;
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            const int tok = t + 16 * (w / 2) + 4 * lg + 2 * (w & 1) + e;
            if (tok >= sp.lo && tok < sp.hi && ok(id)) keep |= 0xFFFFu << (16 * e);
          }
          x[w] &= keep;
        }
      }
      o[j] = mma<kPv>(x, p_hi, o[j]);
      o[j] = mma<kPv>(x, p_lo, o[j]);
    }
    if (i + 1 < n_my) load_v(i + 1, next);
    id = next;
  }

  // join the four waves
  l += __shfl_xor(l, 16);
  l += __shfl_xor(l, 32);
  if (col < n_col) {
    if (lg == 0) {
      lds_m[wave][col] = m;
      lds_l[wave][col] = l;
    }
#pragma unroll
    for (int j = 0; j < D / 16; ++j) *reinterpret_cast<f32x4*>(&lds_o[wave][col][16 * j + 4 * lg]) = o[j];
  }
  __syncthreads();
  for (int e = threadIdx.x; e < n_col * (D / 4); e += 64 * kAttnWaves) {
    const int c = e / (D / 4), d = 4 * (e % (D / 4));
    float mx = lds_m[0][c];
#pragma unroll
    for (int w = 1; w < kAttnWaves; ++w) mx = fmaxf(mx, lds_m[w][c]);
    f32x4 acc = {0.0f, 0.0f, 0.0f, 0.0f};
    float sum = 0.0f;
#pragma unroll
    for (int w = 0; w < kAttnWaves; ++w) {
      const float f = exp2f(lds_m[w][c] - mx);
      sum = fmaf(f, lds_l[w][c], sum);
      const f32x4 x = *reinterpret_cast<const f32x4*>(&lds_o[w][c][d]);
#pragma unroll
      for (int j = 0; j < 4; ++j) acc[j] = fmaf(f, x[j], acc[j]);
    }
    const size_t row = static_cast<size_t>(b) * a.n_q_heads + hq0 + c;
    if (n_act <= 1) {
      const float inv = sum == 0.0f ? 0.0f : 1.0f / sum;
      *reinterpret_cast<u32x2*>(a.out + row * D + d) =
          u32x2{pack16<ACT>(acc[0] * inv, acc[1] * inv), pack16<ACT>(acc[2] * inv, acc[3] * inv)};
      if (a.lse && d == 0) a.lse[row] = sum == 0.0f ? -INFINITY : (mx + log2f(sum)) * kLn2;
    } else {
      const size_t at = row * a.n_splits + split;
      *reinterpret_cast<f32x4*>(a.part_o + at * D + d) = acc;
      if (d == 0) {
        a.part_ml[2 * at] = mx;
        a.part_ml[2 * at + 1] = sum;
      }
    }
  }
}

// Joins the splits of one row (sequence and query head) per wave, in the
// order of the splits.
template <int ACT, int D>
__global__ __launch_bounds__(256) void k_attn_join(AttnArgs a) {
  const int lane = lane_id();
  const int row = static_cast<int>(blockIdx.x) * 4 + (static_cast<int>(threadIdx.x) >> 6);
  if (row >= a.B * a.n_q_heads) return;
  const Span sp = span_of(a, row / a.n_q_heads);
  const int n = (sp.tiles + a.split_tiles - 1) / a.split_tiles;
  if (n <= 1) return;
  const size_t at = static_cast<size_t>(row) * a.n_splits;
  float mx = kNoMax;
  for (int s = lane; s < n; s += 64) mx = fmaxf(mx, a.part_ml[2 * (at + s)]);
#pragma unroll
  for (int o = 32; o; o >>= 1) mx = fmaxf(mx, __shfl_xor(mx, o));
  float acc[D / 64] = {}, sum = 0.0f;
#pragma unroll 4
  for (int s = 0; s < n; ++s) {
    const float f = exp2f(a.part_ml[2 * (at + s)] - mx);
    sum = fmaf(f, a.part_ml[2 * (at + s) + 1], sum);
#pragma unroll
    for (int j = 0; j < D / 64; ++j) acc[j] = fmaf(f, a.part_o[(at + s) * D + 64 * j + lane], acc[j]);
  }
  const float inv = sum == 0.0f ? 0.0f : 1.0f / sum;
#pragma unroll
  for (int j = 0; j < D / 64; ++j)
    a.out[static_cast<size_t>(row) * D + 64 * j + lane] = static_cast<uint16_t>(pack16<ACT>(acc[j] * inv, 0.0f));
  if (a.lse && lane == 0) a.lse[row] = sum == 0.0f ? -INFINITY : (mx + log2f(sum)) * kLn2;
}

template <int ACT, int BITS, int D>
hipError_t launch_attn_d(const AttnArgs& a, hipStream_t st) {
  const int g = a.n_q_heads / a.kv.n_kv_heads, q_tiles = (g + 15) / 16;
  k_attn<ACT, BITS, D><<<a.B * a.kv.n_kv_heads * q_tiles * a.n_splits, 64 * kAttnWaves, 0, st>>>(a, q_tiles);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || a.n_splits == 1) return e;
  k_attn_join<ACT, D><<<(a.B * a.n_q_heads + 3) / 4, 256, 0, st>>>(a);
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

// How far a sequence is split: enough workgroups for every CU to hold a few,
// and at least eight tiles (two per wave) to a split.
AttnPlan attn_plan(int B, int n_q_heads, int n_kv_heads, int head_dim, int, int max_len, int window) {
  AttnPlan p{1, 4, 0};
  int64_t tiles = (static_cast<int64_t>(max_len) + kTile - 1) / kTile;
  if (window > 0) {
    const int64_t w = (static_cast<int64_t>(window) + 2 * kTile - 2) / kTile;   // a window that starts inside a tile
    tiles = w < tiles ? w : tiles;
  }
  const int64_t q_tiles = (n_q_heads / n_kv_heads + 15) / 16;
  const int64_t items = static_cast<int64_t>(B) * n_kv_heads * q_tiles;
  if (items == 0 || tiles == 0) return p;
  int64_t n = (1024 + items - 1) / items;
  const int64_t most = (tiles + 7) / 8;
  n = n < most ? n : most;
  const int64_t per = ((tiles + n - 1) / n + kAttnWaves - 1) / kAttnWaves * kAttnWaves;
  n = (tiles + per - 1) / per;
  p.split_tiles = static_cast<int>(per);
  p.n_splits = static_cast<int>(n);
  if (n > 1) p.ws_bytes = static_cast<size_t>(B) * n_q_heads * n * (head_dim + 2) * sizeof(float);
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
  if (a.T >= kAppendMany) return append_tiles<ACT, BITS>(a, st);
  int G = 8;
  while (8 * G < a.kv.head_dim) G *= 2;
  const int64_t per = 256 / G, items = static_cast<int64_t>(a.T) * a.kv.n_kv_heads * 2;
  const int64_t blocks = (items + per - 1) / per;
  k_kv_append<ACT, BITS><<<static_cast<uint32_t>(blocks), 256, 0, st>>>(a, G);
  return hipGetLastError();
}

}  // namespace

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
