// Attention of several new tokens per sequence over the paged KV cache, gfx950:
// trees of drafted tokens and prompt chunks (k_attn_rows, k_rows_join).
#include "pw_kv.hpp"
#include "pw_lds.hpp"

namespace pw {
namespace {

// Rows and query heads of a key head are the columns of the products that one
// token's attention (pw_attn.hip) has its query heads for: scores S[token, column]
// = K q^T, outputs O[channel, column] += V^T P^T, a lane holding tokens 4 g .. 4 g
// + 3 of either half of a 32-token tile for column lane mod 16. What a column sees
// of a tile is 32 bits: a range of positions, and for trees the row's mask shifted
// to the tile. Tiles that all columns see whole are taken without them.
//
// Two kernels, by the columns that a sequence and key head have on average:
//   up to 64, k_attn_rows: the waves of a workgroup have the same 16 or 32 columns and
//     take tiles in turn, keys and values straight to registers, as pw_attn.hip does.
//     Bound by the cache's bytes and, with 32 columns or fp16, by vector instructions:
//     64 ragged trees of up to 16 tokens, contexts to 4096, 8 key heads x 4, heads of
//     128 in 16 bits (509 MB) 135 us, in 8 bits (267 MB) 115; heads of 64 in fp16,
//     window 1500 (156 MB), 45; 8 tokens after 300 (one sequence) 9.1, a chain of
//     starts, table, tiles and the join of the waves. 64 columns a wave were slower
//     everywhere (the first 176 us, the second 186): their registers leave one wave
//     per SIMD, and groups are rarely full.
//   above, k_attn_tiles: see there.
// At 68 columns on average (500 rows beside 31 single ones) the second takes 79 us and
// the first 96; at 64 (the first case above) 142 and 135.

constexpr int kRowsWaves = 4;

struct Item {
  int b, h;
  int row0, n;             // first row of the sequence, its rows
  int col0, n_col;         // first column of the group, columns
  int ctx;                 // positions before the rows' own
  int lo, hi;              // positions that some column sees lie in [lo, hi)
  int t0, tiles;
};

__device__ __forceinline__ int clamp64(int64_t v, int lo, int hi) {
  return static_cast<int>(v < lo ? lo : v > hi ? hi : v);
}

// How the work is cut.
//   splits (a.n_shares 0): the first a.whole items go to a workgroup each, the others to
//     a.n_splits, each of which takes a.split_tiles tiles of the item. Workgroups that
//     run together then read the same tiles for other columns, from the L2.
//   shares: each head's items form a line of tiles, cut into equal shares, one per
//     workgroup, wherever the items end: sequences of unlike lengths leave no workgroup
//     with more than another. Workgroups that run together read other tiles, so this
//     is for few groups of columns (with k_attn_tiles 24 sequences of 1152 rows took
//     1632 us, by splits 1206).
// A part of an item that is not all of it goes to a slot of the workspace: split s of
// item i to slot (i - whole) n_splits + s, share s's part of item i to slot s + i (one
// of the two grows from part to part); k_rows_join adds them up. Lengths are read on
// the device, and nothing else decides.

// Sequence b's rows; none outside 0 .. T - 1, whatever the starts are.
__device__ __forceinline__ void rows_of(const RowsArgs& a, int b, int* row0, int* n) {
  *row0 = clampi(a.starts[b], 0, a.T);
  *n = clampi(a.starts[b + 1], *row0, a.T) - *row0;
}
// x / g for 0 <= x < 2^31 by the reciprocal m = floor(2^32 / g), which gives it or one
// less.
__device__ __forceinline__ int over(int x, int g, uint32_t m) {
  const int q = static_cast<int>(__umulhi(static_cast<uint32_t>(x), m));
  return x - q * g >= g ? q + 1 : q;
}
// Group gi of a sequence's columns.
__device__ __forceinline__ Item item_of(const RowsArgs& a, int b, int h, int row0, int n, int64_t len, int gi, int cols, int g) {
  Item it;
  it.b = b;
  it.h = h;
  it.row0 = row0;
  it.n = n;
  it.col0 = gi * cols;
  it.n_col = min(cols, n * g - it.col0);
  it.ctx = clamp64(len - n, -(1 << 30), INT32_MAX);
  if (a.masks) {
    it.hi = clamp64(len, 0, a.max_len);
    it.lo = a.window ? clamp64(static_cast<int64_t>(it.ctx) - a.window, 0, it.hi) : 0;
  } else {
    const int first = over(it.col0, g, a.over_g), last = over(it.col0 + it.n_col - 1, g, a.over_g);
    it.hi = clamp64(static_cast<int64_t>(it.ctx) + last + 1, 0, a.max_len);
    it.lo = a.window ? clamp64(static_cast<int64_t>(it.ctx) + first + 1 - a.window, 0, it.hi) : 0;
  }
  it.t0 = it.lo / kTile;
  it.tiles = it.hi > it.lo ? (it.hi + kTile - 1) / kTile - it.t0 : 0;
  return it;
}
__device__ __forceinline__ int scan64(int x, int lane) {         // sums of the lanes up to this one
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const int y = __shfl_up(x, o);
    if (lane >= o) x += y;
  }
  return x;
}
// Item `item` in the order of sequences and groups; false past the last one.
__device__ __forceinline__ bool item_at(const RowsArgs& a, int64_t item, int h, int cols, int lane, Item* it) {
  const int g = a.n_q_heads / a.kv.n_kv_heads;
  int64_t before = 0;
  for (int base = 0; base < a.B; base += 64) {
    int row0 = 0, n = 0, len = 0;
    if (base + lane < a.B) {
      rows_of(a, base + lane, &row0, &n);
      len = a.lens[base + lane];
    }
    const int groups = (n * g + cols - 1) / cols, upto = a.B > 1 ? scan64(groups, lane) : __builtin_amdgcn_readlane(groups, 0);
    const int all = __builtin_amdgcn_readlane(upto, 63);
    if (item < before + all) {
      const int l = __ffsll(static_cast<long long>(__ballot(before + upto > item))) - 1;
      if (l < 0) return false;
      n = __builtin_amdgcn_readlane(n, l);
      const int64_t gi = item - before - (__builtin_amdgcn_readlane(upto, l) - __builtin_amdgcn_readlane(groups, l));
      if (gi < 0 || gi * cols >= static_cast<int64_t>(n) * g) return false;
      *it = item_of(a, base + l, h, __builtin_amdgcn_readlane(row0, l), n, __builtin_amdgcn_readlane(len, l),
                    static_cast<int>(gi), cols, g);
      return true;
    }
    before += all;
  }
  return false;
}
// Tiles of a sequence's items.
__device__ __forceinline__ int tiles_of(const RowsArgs& a, int row0, int n, int64_t len, int cols, int g) {
  const int groups = (n * g + cols - 1) / cols;
  int sum = 0;
  if (a.masks && groups > 0) return groups * item_of(a, 0, 0, row0, n, len, 0, cols, g).tiles;   // one span for all
  for (int gi = 0; gi < groups; ++gi) sum += item_of(a, 0, 0, row0, n, len, gi, cols, g).tiles;
  return sum;
}

// The workgroup's items, or parts of them, one after the other.
struct Walk {
  int pos, stop;           // its tiles of the line, from the next part on
  int start, index;        // of the item that `pos` lies in: first tile, number
  int b, gi, r;            // its sequence and group; tiles of a share
};
struct Part {
  int begin, end;          // tiles of the item's span
  bool whole;
  int64_t slot;
};
// The workgroup's split of an item; false where there is none.
__device__ __forceinline__ bool split_of(const RowsArgs& a, int cols, int lane, Item* it, Part* p) {
  const int H = a.kv.n_kv_heads, h = blockIdx.x % H, w = blockIdx.x / H;
  const bool all = w < a.whole;
  const int rest = static_cast<int>(a.items - a.whole), y = w - static_cast<int>(a.whole);
  const int split = all ? 0 : y / rest, item = all ? w : static_cast<int>(a.whole) + y % rest;
  // (the last rows first: of a prompt's chunk they have the longest spans)
  if (!item_at(a, a.items - 1 - item, h, cols, lane, it)) return false;
  const int per = all ? max(it->tiles, 1) : a.split_tiles, n_act = (it->tiles + per - 1) / per;
  if (split > 0 && split >= n_act) return false;
  *p = Part{split * per, min(split * per + per, it->tiles), n_act <= 1,
            (h * static_cast<int64_t>(rest) + item - a.whole) * a.n_splits + split};
  return true;
}
// The first of its parts of the line; false where there is none.
__device__ __forceinline__ bool walk_begin(const RowsArgs& a, int cols, int lane, Walk* k) {
  const int H = a.kv.n_kv_heads, w = blockIdx.x / H, g = a.n_q_heads / H;
  // tiles of all sequences (the sums stay below 2^31: checked on the host for max_len)
  int total = 0;
  for (int base = 0; base < a.B; base += 64) {
    int row0 = 0, n = 0, x = 0;
    if (base + lane < a.B) {
      rows_of(a, base + lane, &row0, &n);
      x = tiles_of(a, row0, n, a.lens[base + lane], cols, g);
    }
    total += __builtin_amdgcn_readlane(scan64(x, lane), 63);
  }
  const int r = (total + a.n_shares - 1) / a.n_shares;
  k->r = max((r + kRowsWaves - 1) / kRowsWaves * kRowsWaves, a.least);
  const int64_t pos = static_cast<int64_t>(w) * k->r;
  if (pos >= total) return false;
  k->pos = static_cast<int>(pos);
  k->stop = min(total - k->pos, k->r) + k->pos;
  k->start = k->index = k->b = k->gi = 0;
  for (int base = 0; base < a.B; base += 64) {
    int row0 = 0, n = 0, x = 0;
    if (base + lane < a.B) {
      rows_of(a, base + lane, &row0, &n);
      x = tiles_of(a, row0, n, a.lens[base + lane], cols, g);
    }
    const int groups = (n * g + cols - 1) / cols, x_upto = scan64(x, lane), g_upto = scan64(groups, lane);
    const int l = __ffsll(static_cast<long long>(__ballot(k->start + x_upto > k->pos))) - 1;
    if (l >= 0) {
      k->b = base + l;
      k->start += __builtin_amdgcn_readlane(x_upto, l) - __builtin_amdgcn_readlane(x, l);
      k->index += __builtin_amdgcn_readlane(g_upto, l) - __builtin_amdgcn_readlane(groups, l);
      return true;
    }
    k->start += __builtin_amdgcn_readlane(x_upto, 63);
    k->index += __builtin_amdgcn_readlane(g_upto, 63);
  }
  return false;                                                  // (only if a length changes meanwhile)
}
// The part at `pos`, which is moved past it.
__device__ __forceinline__ bool walk_on(const RowsArgs& a, int cols, Walk* k, Item* it, Part* p) {
  const int H = a.kv.n_kv_heads, h = blockIdx.x % H, w = blockIdx.x / H;
  const int g = a.n_q_heads / H;
  if (k->pos >= k->stop) return false;
  while (true) {
    int row0, n;
    rows_of(a, k->b, &row0, &n);
    const int64_t len = a.lens[k->b];
    while (k->gi * static_cast<int64_t>(cols) < static_cast<int64_t>(n) * g) {
      *it = item_of(a, k->b, h, row0, n, len, k->gi, cols, g);
      if (k->start + it->tiles > k->pos) {
        const int begin = k->pos - k->start, end = min(it->tiles, begin + k->stop - k->pos);
        const int first = k->start / k->r, parts = (k->start + it->tiles - 1) / k->r - first + 1;
        if (k->index >= a.items) return false;                   // (only if a length changes meanwhile)
        if (begin == 0 && threadIdx.x == 0) {
          int32_t* meta = a.meta + 2 * (h * a.items + k->index);
          meta[0] = first + k->index;
          meta[1] = parts;
        }
        *p = Part{begin, end, parts == 1, h * (a.n_shares + a.items) + w + k->index};
        k->pos += end - begin;
        return true;
      }
      k->start += it->tiles;
      ++k->index;
      ++k->gi;
    }
    k->gi = 0;
    if (++k->b >= a.B) return false;                             // (the same)
  }
}

// What column c (row i, one of the lane's) sees: positions [lo, hi), and of a tree
// the drafted tokens in its mask.
struct Column {
  int lo, hi;
  int row;                 // of q and the masks; -1: no column
};
__device__ __forceinline__ Column column_at(const RowsArgs& a, const Item& it, int c, int g) {
  Column x{0, 0, -1};
  if (c >= it.n_col) return x;
  const int i = (it.col0 + c) / g;
  x.row = it.row0 + i;
  if (a.masks) {
    x.hi = clampi(it.ctx, 0, a.max_len);
    if (a.window) {
      int64_t seen = 0;
      for (int w = 0; w < a.words && 64 * w < it.n; ++w) {
        uint64_t m = static_cast<uint64_t>(a.masks[static_cast<int64_t>(x.row) * a.words + w]);
        if (it.n - 64 * w < 64) m &= (1ull << (it.n - 64 * w)) - 1ull;
        seen += __popcll(m);
      }
      x.lo = clamp64(it.ctx + seen - a.window, 0, x.hi);
    }
  } else {
    x.hi = clamp64(static_cast<int64_t>(it.ctx) + i + 1, 0, a.max_len);
    x.lo = a.window ? clamp64(static_cast<int64_t>(it.ctx) + i + 1 - a.window, 0, x.hi) : 0;
  }
  return x;
}
__device__ __forceinline__ uint32_t first_bits(int n) { return n >= 32 ? ~0u : (1u << n) - 1u; }
__device__ __forceinline__ uint64_t first_word(const RowsArgs& a, const Column& x) {
  return a.masks && x.row >= 0 ? static_cast<uint64_t>(a.masks[static_cast<int64_t>(x.row) * a.words]) : 0;
}
// Bit i: the column sees position t + i. word0: the first word of its mask.
__device__ __forceinline__ uint32_t seen_of(const RowsArgs& a, const Item& it, const Column& x, uint64_t word0, int t) {
  uint32_t s = first_bits(clamp64(static_cast<int64_t>(x.hi) - t, 0, 32)) & ~first_bits(clamp64(static_cast<int64_t>(x.lo) - t, 0, 32));
  if (a.masks && x.row >= 0 && t + kTile > it.ctx) {
    const int64_t j = static_cast<int64_t>(t) - it.ctx;          // drafted token of bit 0, above -32
    const int64_t* m = a.masks + static_cast<int64_t>(x.row) * a.words;
    uint64_t d = 0;
    if (j < 0) {
      d = word0 << -j;
    } else if (j < 64 * static_cast<int64_t>(a.words)) {
      const int w = static_cast<int>(j >> 6), sh = static_cast<int>(j & 63);
      d = (w == 0 ? word0 : static_cast<uint64_t>(m[w])) >> sh;
      if (sh > 32 && w + 1 < a.words) d |= static_cast<uint64_t>(m[w + 1]) << (64 - sh);
    }
    s |= static_cast<uint32_t>(d) & first_bits(clamp64(static_cast<int64_t>(it.hi) - t, 0, 32));
  }
  return s;
}

// Values that are no numbers would enter columns that do not see them (0 x NaN), so
// in tiles that some columns see in part they are taken out of the product, and
// added one by one to the columns that do, as they are: no weight but that of a score of
// -infinity is nothing, however small the exponential came out. Where all columns see an
// infinity, a product is none if the weight came out as 0, or is in two terms (inf - inf),
// and so is what a later maximum scales down by 0: a wave (of k_attn_tiles a workgroup)
// whose outputs are not all numbers goes through its tiles once more, with that done in
// all of them and factors that are not 0.
template <int BITS, int PV>
__device__ __forceinline__ uint32_t odd_parts(uint32_t w) {      // ones over the parts of a word that are no numbers
  if constexpr (BITS == 8) {
    const uint32_t z = ((w & 0x7F7F7F7Fu) + 0x01010101u) & 0x80808080u;
    return (z >> 7) * 0xFFu;
  } else {
    constexpr uint32_t kExp = PV == PW_BF16 ? 0x7F80u : 0x7C00u;
    return ((w & kExp) == kExp ? 0xFFFFu : 0u) | (((w >> 16) & kExp) == kExp ? 0xFFFF0000u : 0u);
  }
}

// A factor of what is there, at least the smallest number in place of 0: infinities stay,
// and all else is nothing beside a weight of 1.
constexpr float kLeast = 0x1p-149f;

template <int D>
struct RowsLds {
  float o[kRowsWaves][16][D + 4];
  float m[kRowsWaves][16], l[kRowsWaves][16];
};

// Tiles [begin, end) of the item's span, by the workgroup's waves in turn; C x 16
// columns a wave, the same for all. whole: no other workgroup has tiles of the item,
// the result goes to the output; else to slot `slot`.
template <int ACT, int BITS, int D, int C>
__device__ __forceinline__ void attend_rows(const RowsArgs& a, RowsLds<D>& lds, const Item& it, int begin, int end, bool whole,
                                            int64_t slot) {
  constexpr int W = kRowsWaves;
  constexpr int kPv = BITS == 8 ? PW_BF16 : ACT;      // 16-bit type of the second product
  constexpr bool kByTile = kPv == PW_F16;             // exponentials against the tile's maximum
  constexpr int kLoads = D * BITS / 8 * 16 / 1024;    // 1 KB loads of 16 tokens' keys
  const int wave = __builtin_amdgcn_readfirstlane(static_cast<int>(threadIdx.x) >> 6), lane = lane_id();
  const int col = lane & 15, lg = lane >> 4;
  const int P = a.kv.block_tokens, h = it.h;
  const int first = begin + wave;                                // the wave's tiles: first, first + W, ...
  const int n_my = first < end ? (end - first + W - 1) / W : 0;
  const int g = a.n_q_heads / a.kv.n_kv_heads;

  Column x[C];
  uint64_t word0[C];                                             // (early: otherwise one more load in the chain of the last tiles)
  u32x4 q[C][D / 32];
  int all_lo = 0, all_hi = INT32_MAX;                            // all columns see [all_lo, all_hi)
#pragma unroll
  for (int c = 0; c < C; ++c) {
    const int cc = 16 * c + col;
    x[c] = column_at(a, it, cc, g);
    word0[c] = first_word(a, x[c]);
    if (x[c].row >= 0) {
      all_lo = max(all_lo, x[c].lo);
      all_hi = min(all_hi, x[c].hi);
    }
#pragma unroll
    for (int i = 0; i < D / 32; ++i) {
      q[c][i] = u32x4{0u, 0u, 0u, 0u};
      if (x[c].row >= 0)
        q[c][i] = ld16(reinterpret_cast<const uint8_t*>(a.q + static_cast<int64_t>(x[c].row) * a.ldq +
                                                        (h * g + (it.col0 + cc) % g) * a.ldqh + 32 * i + 8 * lg));
    }
  }
#pragma unroll
  for (int o = 1; o < 16; o <<= 1) {
    all_lo = max(all_lo, __shfl_xor(all_lo, o));
    all_hi = min(all_hi, __shfl_xor(all_hi, o));
  }
  all_lo = __builtin_amdgcn_readfirstlane(all_lo);
  all_hi = __builtin_amdgcn_readfirstlane(all_hi);

  // The tiles in blocks of the pool, one after the other (tiles in other blocks
  // are left out): bits of the 64 numbers at hand, then the next 64.
  const auto block_of = [&](int i) {                             // of the wave's tile i
    if (i >= n_my) return -1;
    const int64_t t = static_cast<int64_t>(it.t0 + first + W * i) * kTile;
    return static_cast<int>(a.table[it.b * a.ld_table + (t >> __builtin_ctz(P))]);
  };
  int ids, chunk;
  uint64_t todo;
  int next_t = -1, next_id = 0;                                  // first token of the next tile (-1: none), its block
  const auto advance = [&] {
    while (todo == 0 && chunk + 64 < n_my) {
      chunk += 64;
      ids = block_of(chunk + lane);
      todo = __ballot(ids >= 0 && ids < a.kv.n_blocks);
    }
    next_t = -1;
    if (todo) {
      const int l = __ffsll(static_cast<long long>(todo)) - 1;
      todo &= todo - 1;
      next_id = __builtin_amdgcn_readlane(ids, l);
      next_t = (it.t0 + first + W * (chunk + l)) * kTile;
    }
  };
  const size_t head_off = static_cast<size_t>(2 * h) * P * D * (BITS / 8);
  const size_t v_off = static_cast<size_t>(P) * D * (BITS / 8);
  const size_t sc_off = static_cast<size_t>(2) * a.kv.n_kv_heads * P * D + static_cast<size_t>(h) * P * 4;
  const size_t vs_off = static_cast<size_t>(a.kv.n_kv_heads) * P * 4;
  const float scale2 = a.scale * kLog2e;

  u32x4 k[2][kLoads], v[2 * kLoads];
  f32x4 ks[2], vs[2];
  const auto values_at = [&](int id, int t) {                    // of the tile, in memory
    return a.kv.pool + static_cast<int64_t>(id) * a.kv.block_stride + head_off + v_off +
           static_cast<size_t>(t & (P - 1)) * D * (BITS / 8);
  };
  const auto load_k = [&] {
    const int t = next_t & (P - 1);                              // in the block
    const uint8_t* blk = a.kv.pool + static_cast<int64_t>(next_id) * a.kv.block_stride;
    const uint8_t* p = blk + head_off + static_cast<size_t>(t) * D * (BITS / 8) + 16 * lane;
#pragma unroll
    for (int r = 0; r < 2; ++r)
#pragma unroll
      for (int j = 0; j < kLoads; ++j) k[r][j] = ld16(p + (r * kLoads + j) * 1024);
    if constexpr (BITS == 8) {
#pragma unroll
      for (int r = 0; r < 2; ++r) ks[r] = *reinterpret_cast<const f32x4*>(blk + sc_off + 4 * t + 16 * lg + 64 * r);
    }
  };
  const auto load_v = [&] {
    const int t = next_t & (P - 1);
    const uint8_t* p = values_at(next_id, next_t) + 16 * lane;
#pragma unroll
    for (int j = 0; j < 2 * kLoads; ++j) v[j] = ld16(p + j * 1024);
    if constexpr (BITS == 8) {
      const uint8_t* blk = a.kv.pool + static_cast<int64_t>(next_id) * a.kv.block_stride;
#pragma unroll
      for (int r = 0; r < 2; ++r) vs[r] = *reinterpret_cast<const f32x4*>(blk + sc_off + vs_off + 4 * t + 16 * lg + 64 * r);
    }
  };

  f32x4 o[C][D / 16];
  float m[C], l[C];
  for (bool careful = false;; careful = true) {
#pragma unroll
    for (int c = 0; c < C; ++c) {
#pragma unroll
      for (int j = 0; j < D / 16; ++j) o[c][j] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
      m[c] = kNoMax;
      l[c] = 0.0f;
    }

    ids = block_of(lane);
    chunk = 0;
    todo = __ballot(ids >= 0 && ids < a.kv.n_blocks);
    advance();
    if (next_t >= 0) {
      load_k();
      load_v();
    }
    while (next_t >= 0) {
      const int t = next_t, id = next_id;
      f32x4 s[C][2];
#pragma unroll
      for (int r = 0; r < 2; ++r) {
#pragma unroll
        for (int c = 0; c < C; ++c) s[c][r] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int j = 0; j < D / 32; ++j) {
          u32x4 kk;
          if constexpr (BITS == 16) kk = k[r][j];
          else kk = widen8<ACT>(k[r][j / 2][2 * (j & 1)], k[r][j / 2][2 * (j & 1) + 1]);
#pragma unroll
          for (int c = 0; c < C; ++c) s[c][r] = mma<ACT>(kk, q[c][j], s[c][r]);
        }
      }
#pragma unroll
      for (int c = 0; c < C; ++c)
#pragma unroll
        for (int r = 0; r < 2; ++r)
#pragma unroll
          for (int e = 0; e < 4; ++e) s[c][r][e] *= BITS == 8 ? scale2 * ks[r][e] : scale2;
      const bool part = t < all_lo || t + kTile > all_hi;          // some column does not see all of it
      bool odd = false;
      if (part || careful) {
        // what no column may see is left out, whatever its bits
        uint32_t keep[2][2];                                       // of four tokens' 8 or 16 bits
#pragma unroll
        for (int r = 0; r < 2; ++r) {
          keep[r][0] = keep[r][1] = 0u;
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const int tok = t + 16 * r + 4 * lg + e;
            const bool in = tok >= it.lo && tok < it.hi;
            if constexpr (BITS == 8) {
              vs[r][e] = in ? vs[r][e] : 0.0f;
              keep[r][0] |= in ? 0xFFu << (8 * e) : 0u;
            } else {
              keep[r][e / 2] |= in ? 0xFFFFu << (16 * (e & 1)) : 0u;
            }
          }
        }
        uint32_t any = 0u;
#pragma unroll
        for (int j = 0; j < 2 * kLoads; ++j)
#pragma unroll
          for (int w = 0; w < 4; ++w) {
            v[j][w] &= BITS == 8 ? keep[w & 1][0] : keep[w / 2][w & 1];
            const uint32_t z = odd_parts<BITS, kPv>(v[j][w]);
            any |= z;
            v[j][w] &= ~z;
          }
        odd = __any(any != 0u);
      }
      advance();
      if (next_t >= 0) load_k();
#pragma unroll
      for (int c = 0; c < C; ++c) {
        if (16 * c >= it.n_col) break;                           // (uniform)
        uint32_t seen = ~0u;
        if (part) {
          seen = seen_of(a, it, x[c], word0[c], t);
#pragma unroll
          for (int r = 0; r < 2; ++r)
#pragma unroll
            for (int e = 0; e < 4; ++e) s[c][r][e] = (seen >> (16 * r + 4 * lg + e)) & 1u ? s[c][r][e] : -INFINITY;
        }
        float top = s[c][0][0];
#pragma unroll
        for (int e = 1; e < 8; ++e) top = fmaxf(top, s[c][e / 4][e & 3]);
        float base = m[c];                                         // probabilities are exp2(s - base)
        float f = 1.0f, share = 1.0f;                              // factors of what is there and of this tile
        bool raise;
        if constexpr (kByTile) {
          top = fmaxf(column_max(top), kNoMax);                    // (a number, whatever the scores)
          raise = __any(top > m[c]);
          const float m_new = fmaxf(m[c], top);
          f = __builtin_amdgcn_exp2f(m[c] - m_new);
          share = __builtin_amdgcn_exp2f(top - m_new);
          base = top;
          m[c] = m_new;
        } else {
          raise = __any(top > m[c] + kSlack);
          if (raise) {
            const float m_new = fmaxf(m[c], column_max(top));
            f = __builtin_amdgcn_exp2f(m[c] - m_new);
            base = m[c] = m_new;
          }
        }
        if (raise) {
          if (BITS == 16 && careful) f = fmaxf(f, kLeast);
          l[c] *= f;
#pragma unroll
          for (int j = 0; j < D / 16; ++j)
#pragma unroll
            for (int e = 0; e < 4; ++e) o[c][j][e] *= f;
        }
        uint32_t some = 0u;                                        // of the lane's tokens, those with a weight
        if (odd) {
#pragma unroll
          for (int e = 0; e < 8; ++e) some |= s[c][e / 4][e & 3] > -INFINITY ? 1u << e : 0u;
        }
        float sum = 0.0f;
        u32x4 p_hi, p_lo;
#pragma unroll
        for (int w = 0; w < 4; ++w) {
          float p[2];
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            const int r = w / 2, y = 2 * (w & 1) + e;
            p[e] = __builtin_amdgcn_exp2f(s[c][r][y] - base);
            sum += p[e];
            if constexpr (BITS == 8) {
              p[e] *= vs[r][y];
              if (part) p[e] = (seen >> (16 * r + 4 * lg + y)) & 1u ? p[e] : 0.0f;
            }
            if constexpr (kByTile) p[e] *= kLift;
          }
          p_hi[w] = pack16<kPv>(p[0], p[1]);
          p[0] -= val16(p_hi[w] & 0xFFFFu, kPv);
          p[1] -= val16(p_hi[w] >> 16, kPv);
          p_lo[w] = kByTile ? pack16<kPv>(p[0] * kLow, p[1] * kLow) : pack16<kPv>(p[0], p[1]);
        }
        l[c] = fmaf(share, sum, l[c]);
        if (odd) {
          const uint8_t* vm = values_at(id, t);
          for (int i = 0; i < kTile; ++i) {
            const int at = 4 * (i / 16) + i % 4;                   // token i's place in lanes 16 (i / 4 mod 4) ..
            const bool none = !(__shfl(static_cast<int>(some), 16 * (i / 4 % 4) + col) >> at & 1);
            const bool on = (seen >> i) & 1u;
#pragma unroll
            for (int j = 0; j < D / 16; ++j)
#pragma unroll
              for (int e = 0; e < 4; ++e) {
                const int place = 16 * (16 * (i / 4 % 4) + 4 * lg + e);
                float y = 0.0f;
                if constexpr (BITS == 16) {
                  const uint32_t w = *reinterpret_cast<const uint16_t*>(vm + j * 1024 + place + 2 * (4 * (i / 16) + i % 4));
                  if (odd_parts<16, kPv>(w) & 0xFFFFu) y = val16(w, kPv);
                } else {
                  const uint32_t w = vm[(j / 2) * 1024 + place + 8 * (j & 1) + 4 * (i / 16) + i % 4];
                  if ((w & 0x7Fu) == 0x7Fu) y = __builtin_nanf("");
                }
                if (on && y != 0.0f) o[c][j][e] += none ? __builtin_nanf("") : y;
              }
          }
        }
        if constexpr (kByTile) share *= 1.0f / kLift;
#pragma unroll
        for (int j = 0; j < D / 16; ++j) {
          u32x4 vv;
          if constexpr (BITS == 16) vv = v[j];
          else vv = widen8<kPv>(v[j / 2][2 * (j & 1)], v[j / 2][2 * (j & 1) + 1]);
          if constexpr (kByTile) {
            const f32x4 zero{0.0f, 0.0f, 0.0f, 0.0f}, hi = mma<kPv>(vv, p_hi, zero), lo = mma<kPv>(vv, p_lo, zero);
#pragma unroll
            for (int e = 0; e < 4; ++e) o[c][j][e] = fmaf(share, fmaf(lo[e], 1.0f / kLow, hi[e]), o[c][j][e]);
            asm volatile("" : "+v"(o[c][j]));                      // (not all products before all sums: registers)
          } else {
            o[c][j] = mma<kPv>(vv, p_hi, o[c][j]);
            o[c][j] = mma<kPv>(vv, p_lo, o[c][j]);
          }
        }
      }
      if (next_t >= 0) load_v();
    }
    bool bad = false;
    if constexpr (BITS == 16) {                                  // (an 8-bit NaN gives one, however often it is added)
      if (!careful) {
#pragma unroll
        for (int c = 0; c < C; ++c)
#pragma unroll
          for (int j = 0; j < D / 16; ++j)
#pragma unroll
            for (int e = 0; e < 4; ++e) bad |= !(fabsf(o[c][j][e]) < INFINITY);
      }
    }
    if (!__any(bad)) break;
  }

  // join the waves, 16 columns at a time
#pragma unroll
  for (int c = 0; c < C; ++c) {
    const int n_col = min(16, it.n_col - 16 * c);                // (uniform)
    if (n_col <= 0) break;
    if (c) __syncthreads();                                      // what was joined before is read
    float sum_l = l[c];
    sum_l += __shfl_xor(sum_l, 16);
    sum_l += __shfl_xor(sum_l, 32);
    if (col < n_col) {
      if (lg == 0) {
        lds.m[wave][col] = m[c];
        lds.l[wave][col] = sum_l;
      }
#pragma unroll
      for (int j = 0; j < D / 16; ++j) *reinterpret_cast<f32x4*>(&lds.o[wave][col][16 * j + 4 * lg]) = o[c][j];
    }
    __syncthreads();
    for (int e = threadIdx.x; e < n_col * (D / 4); e += 64 * W) {
      const int y = e / (D / 4), d = 4 * (e % (D / 4));
      float mx = lds.m[0][y];
#pragma unroll
      for (int w = 1; w < W; ++w) mx = fmaxf(mx, lds.m[w][y]);
      f32x4 acc = {0.0f, 0.0f, 0.0f, 0.0f};
      float sum = 0.0f;
#pragma unroll
      for (int w = 0; w < W; ++w) {
        const float f = fmaxf(__builtin_amdgcn_exp2f(lds.m[w][y] - mx), kLeast);
        sum = fmaf(f, lds.l[w][y], sum);
        const f32x4 z = *reinterpret_cast<const f32x4*>(&lds.o[w][y][d]);
#pragma unroll
        for (int j = 0; j < 4; ++j) acc[j] = fmaf(f, z[j], acc[j]);
      }
      const int cc = 16 * c + y;
      if (whole) {
        const int row = it.row0 + (it.col0 + cc) / g, hq = h * g + (it.col0 + cc) % g;
        const int64_t at = static_cast<int64_t>(row) * a.n_q_heads + hq;
        const float inv = sum == 0.0f ? 0.0f : 1.0f / sum;
        *reinterpret_cast<u32x2*>(a.out + at * D + d) =
            u32x2{pack16<ACT>(acc[0] * inv, acc[1] * inv), pack16<ACT>(acc[2] * inv, acc[3] * inv)};
        if (a.lse && d == 0) a.lse[at] = sum == 0.0f ? -INFINITY : (mx + log2f(sum)) * kLn2;
      } else {
        const int64_t at = slot * (16 * C) + cc;
        *reinterpret_cast<f32x4*>(a.part_o + at * D + d) = acc;
        if (d == 0) {
          a.part_ml[2 * at] = mx;
          a.part_ml[2 * at + 1] = sum;
        }
      }
    }
  }
}

// Workgroups on a CU, by what the kernel holds in registers from tile to tile.
constexpr int rows_resident(int bits, int D, int C) {
  return C * (D / 8 + D / 4 + 8) + D / 4 * bits / 16 * 2 + 48 <= 224 ? 2 : 1;
}

template <int ACT, int BITS, int D, int C, bool LINE>
__global__ __launch_bounds__(64 * kRowsWaves, rows_resident(BITS, D, C)) void k_attn_rows(RowsArgs a) {
  __shared__ RowsLds<D> lds;
  Item it;
  Part p;
  if constexpr (!LINE) {
    if (split_of(a, 16 * C, lane_id(), &it, &p)) attend_rows<ACT, BITS, D, C>(a, lds, it, p.begin, p.end, p.whole, p.slot);
  } else {
    Walk k;
    if (!walk_begin(a, 16 * C, lane_id(), &k) || !walk_on(a, 16 * C, &k, &it, &p)) return;
    while (true) {
      attend_rows<ACT, BITS, D, C>(a, lds, it, p.begin, p.end, p.whole, p.slot);
      if (!walk_on(a, 16 * C, &k, &it, &p)) return;
      __syncthreads();                                           // the part's LDS is read
    }
  }
}

// ---------------------------------------------------------------------------
// Many columns
// ---------------------------------------------------------------------------
//
// A workgroup's four waves have columns of their own, C x 16 each, and share the
// tiles: those come into LDS by direct loads, kStages - 1 tiles ahead, in the order
// in which they lie in the cache, which is the one that the matrix instructions take
// them in: 1 KB per instruction, without bank conflicts.
// The matrix unit is the bound (busy 382 us of 4096 rows after 12288 tokens, 8 key
// heads x 4 of 128 in bf16, 0.96 TFLOP), with about as much time of vector
// instructions (exponentials, maxima, roundings) and of LDS reads beside it: 910 us,
// 1.06 PFLOP/s, where the library's product of two 8192 x 8192 matrices reaches 1.27.
// What counts is waves per SIMD that are at another of the three: C = 2 has 168
// registers and three waves, 1155 us (24 sequences of 1152 rows after 2048 tokens); with
// two waves 1360; C = 3 with two waves 1194; C = 4 spills with two waves (3029) and has
// one without (2729). All columns' maxima are compared before one branch, so that what
// follows is one block in which products and exponentials mix: 1244 us before.
// A weight is rounded once to the 16 bits of its product (a second term, as
// k_attn_rows has it, is half as many products again): in bf16 that leaves as much as
// the output's own rounding, 2.3e-3 of the result in norm together against 1.7e-3. fp16
// outputs would show it, so 8-bit caches then take two terms (several prompts of up to
// 1111 rows, heads of 64: 64 us, with one 51), and fp16 caches, whose exponentials are
// against the tile's maximum, two where a tile holds weights below 2^-29 of it.
// 8-bit codes are widened by each wave (1479 us where 16 bits take 1177).

// The scale is multiplied into the scores in one step with the maximum's subtraction: the
// largest score keeps what the maximum was rounded by, a tile that is seen in part, where
// the scale comes first, keeps nothing, and from some 2^24 on that is a factor past fp16's
// end. So a workgroup with a column whose maximum reaches kFar (the factor then being at
// most 2^(1/2048)) goes through its tiles once more, the scale first in all of them; and so
// does one with outputs that are not all numbers. (Asking costs 24 sequences of 1152 rows 1
// per cent, in fp16 2. One form for both, with a flag, cost 500 rows beside 31 single ones
// 81 us where this takes 79; a branch for large scores in every tile 15 us of 900.)
constexpr float kFar = 16384.0f;

constexpr int kStages = 3;
template <int BITS, int D>
constexpr int stage_bytes() { return 64 * D * BITS / 8 + (BITS == 8 ? 256 : 0); }

// False: not done, outputs or a maximum want the careful form. (The same for all waves.)
template <int ACT, int BITS, int D, int C, bool CAREFUL>
__device__ __forceinline__ bool attend_tiles(const RowsArgs& a, uint8_t* lds, int* again, const Item& it, int begin, int end,
                                             bool whole, int64_t slot) {
  constexpr int kPv = BITS == 8 ? PW_BF16 : ACT;
  constexpr bool kByTile = kPv == PW_F16;
  constexpr bool kTwo = BITS == 8 && ACT == PW_F16;   // weights in two terms: fp16 outputs show what one bf16 leaves
  constexpr int kLoads = D * BITS / 8 * 16 / 1024;    // 1 KB pieces of 16 tokens' keys
  constexpr int kMine = kLoads + (BITS == 8 ? 1 : 0); // loads of a wave for a tile: a quarter of the pieces, the scales
  const int wave = __builtin_amdgcn_readfirstlane(static_cast<int>(threadIdx.x) >> 6);
  int lane = lane_id();
  if constexpr (CAREFUL) asm volatile("" : "+v"(lane));         // (nothing of the other form is kept for this one)
  const int col = lane & 15, lg = lane >> 4;
  const int P = a.kv.block_tokens, h = it.h;
  const int g = a.n_q_heads / a.kv.n_kv_heads;
  const int my0 = 16 * C * wave;                                 // the wave's first column
  const bool busy = my0 < it.n_col;
  const uint32_t flip = a.scale < 0.0f ? 0x80008000u : 0u;       // queries of the other sign: maxima stay maxima
  const float scale2 = fabsf(a.scale) * kLog2e;

  Column x[C];
  u32x4 q[C][D / 32];
  int all_lo = 0, all_hi = INT32_MAX;                            // all columns of the wave see [all_lo, all_hi)
#pragma unroll
  for (int c = 0; c < C; ++c) {
    const int cc = my0 + 16 * c + col;
    x[c] = column_at(a, it, cc, g);
    if (x[c].row >= 0) {
      all_lo = max(all_lo, x[c].lo);
      all_hi = min(all_hi, x[c].hi);
    }
#pragma unroll
    for (int i = 0; i < D / 32; ++i) {
      q[c][i] = u32x4{0u, 0u, 0u, 0u};
      if (x[c].row >= 0)
        q[c][i] = ld16(reinterpret_cast<const uint8_t*>(a.q + static_cast<int64_t>(x[c].row) * a.ldq +
                                                        (h * g + (it.col0 + cc) % g) * a.ldqh + 32 * i + 8 * lg));
#pragma unroll
      for (int w = 0; w < 4; ++w) q[c][i][w] ^= flip;
    }
  }
#pragma unroll
  for (int o = 1; o < 16; o <<= 1) {
    all_lo = max(all_lo, __shfl_xor(all_lo, o));
    all_hi = min(all_hi, __shfl_xor(all_hi, o));
  }
  all_lo = __builtin_amdgcn_readfirstlane(all_lo);
  all_hi = __builtin_amdgcn_readfirstlane(all_hi);

  // tiles in blocks of the pool, in order; the same for all waves
  const int n_my = end - begin;
  const auto block_of = [&](int i) {
    if (i >= n_my) return -1;
    const int64_t t = static_cast<int64_t>(it.t0 + begin + i) * kTile;
    return static_cast<int>(a.table[it.b * a.ld_table + (t >> __builtin_ctz(P))]);
  };
  int ids, chunk;
  uint64_t todo;
  const size_t head_off = static_cast<size_t>(2 * h) * P * D * (BITS / 8);
  const size_t v_off = static_cast<size_t>(P) * D * (BITS / 8);
  const size_t sc_off = static_cast<size_t>(2) * a.kv.n_kv_heads * P * D + static_cast<size_t>(h) * P * 4;
  const uint32_t lds0 = static_cast<uint32_t>(reinterpret_cast<uintptr_t>((lds_u8_t)lds));
  const uint32_t sc_lane = (lane & 31) * 4 + (lane >= 32 ? static_cast<uint32_t>(a.kv.n_kv_heads) * P * 4 : 0u);
  // the next tile's loads into a stage; its first token, -1 where there is none
  const auto fetch = [&](int stage) {
    while (todo == 0 && chunk + 64 < n_my) {
      chunk += 64;
      ids = block_of(chunk + lane);
      todo = __ballot(ids >= 0 && ids < a.kv.n_blocks);
    }
    if (todo == 0) return -1;
    const int l = __ffsll(static_cast<long long>(todo)) - 1;
    todo &= todo - 1;
    const int id = __builtin_amdgcn_readlane(ids, l);
    const int t = (it.t0 + begin + chunk + l) * kTile;
    const uint8_t* blk = a.kv.pool + static_cast<int64_t>(id) * a.kv.block_stride;
    const uint8_t* src = uniform_ptr(blk + head_off + static_cast<size_t>(t & (P - 1)) * D * (BITS / 8));
    const uint32_t dst = lds0 + stage * stage_bytes<BITS, D>();
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
      const int piece = 4 * i + wave;                            // the keys' 2 kLoads, then the values'
      const bool is_v = piece >= 2 * kLoads;
      lds_load16(dst + piece * 1024, 16 * lane, uniform_ptr(src + (is_v ? v_off : 0) + (piece - (is_v ? 2 * kLoads : 0)) * 1024));
    }
    if constexpr (BITS == 8)                                     // (each wave the same ones)
      lds_load4(dst + 4 * kLoads * 1024, sc_lane, uniform_ptr(blk + sc_off + 4 * (t & (P - 1))));
    return t;
  };

  f32x4 o[C][D / 16];
  float m[C], l[C];
#pragma unroll
  for (int c = 0; c < C; ++c) {
#pragma unroll
    for (int j = 0; j < D / 16; ++j) o[c][j] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    m[c] = kNoMax;
    l[c] = 0.0f;
  }
  ids = block_of(lane);
  chunk = 0;
  todo = __ballot(ids >= 0 && ids < a.kv.n_blocks);
  int t = fetch(0), t1 = t < 0 ? -1 : fetch(1);
  int stage = 0;
  while (t >= 0) {
    if (t1 >= 0) wait_vm<kMine>();
    else wait_vm<0>();
    wg_barrier();                                                // the stage is there, the one before it is read
    const int t2 = t1 < 0 ? -1 : fetch(stage >= 1 ? stage - 1 : kStages - 1);
    if (busy) {
      const uint8_t* sk = lds + stage * stage_bytes<BITS, D>() + 16 * lane;
      const uint8_t* sv = sk + 2 * kLoads * 1024;
      const float* sc = reinterpret_cast<const float*>(lds + stage * stage_bytes<BITS, D>() + 4 * kLoads * 1024) + 4 * lg;
      f32x4 s[C][2];
#pragma unroll
      for (int r = 0; r < 2; ++r) {
#pragma unroll
        for (int c = 0; c < C; ++c) s[c][r] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int j = 0; j < kLoads; ++j) {
          const u32x4 kk = ld16(sk + (r * kLoads + j) * 1024);
          if constexpr (BITS == 16) {
#pragma unroll
            for (int c = 0; c < C; ++c) s[c][r] = mma<ACT>(kk, q[c][j], s[c][r]);
          } else {
#pragma unroll
            for (int e = 0; e < 2; ++e) {
              const u32x4 w = widen8<ACT>(kk[2 * e], kk[2 * e + 1]);
#pragma unroll
              for (int c = 0; c < C; ++c) s[c][r] = mma<ACT>(w, q[c][2 * j + e], s[c][r]);
            }
          }
        }
      }
      f32x4 vs[2];
      if constexpr (BITS == 8) {
#pragma unroll
        for (int r = 0; r < 2; ++r) {
          const f32x4 ks = *reinterpret_cast<const f32x4*>(sc + 16 * r);
          vs[r] = *reinterpret_cast<const f32x4*>(sc + 32 + 16 * r);
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const float f = scale2 * ks[e];
#pragma unroll
            for (int c = 0; c < C; ++c) s[c][r][e] *= f;
          }
        }
      }
      const bool part = CAREFUL || t < all_lo || t + kTile > all_hi;   // some column may not see all of it
      uint32_t seen[C];
      uint32_t some[C];                                          // CAREFUL: of the lane's tokens, those with a weight
      float mul = BITS == 8 ? 1.0f : scale2;                     // of the scores as they are
      if (part) {
#pragma unroll
        for (int c = 0; c < C; ++c) {
          seen[c] = seen_of(a, it, x[c], first_word(a, x[c]), t) >> (4 * lg);
#pragma unroll
          for (int r = 0; r < 2; ++r)
#pragma unroll
            for (int e = 0; e < 4; ++e) s[c][r][e] = (seen[c] >> (16 * r + e)) & 1u ? s[c][r][e] * mul : -INFINITY;
          if constexpr (CAREFUL) {
            some[c] = 0u;
#pragma unroll
            for (int e = 0; e < 8; ++e) some[c] |= s[c][e / 4][e & 3] > -INFINITY ? 1u << e : 0u;
          }
        }
        mul = 1.0f;
      }
      u32x4 p_hi[C], p_two[C];
      float share[C], base[C], top[C];
      bool low = false;                                          // fp16: weights that one term does not hold
      bool raise = false;
#pragma unroll
      for (int c = 0; c < C; ++c) {
        top[c] = s[c][0][0];
#pragma unroll
        for (int e = 1; e < 8; ++e) top[c] = fmaxf(top[c], s[c][e / 4][e & 3]);
        top[c] *= mul;
        if constexpr (kByTile) {
          top[c] = fmaxf(column_max(top[c]), kNoMax);
          raise |= top[c] > m[c];
        } else {
          raise |= top[c] > m[c] + kSlack;
        }
      }
      if (__any(raise)) {                                        // (all columns at once: what follows is one piece)
#pragma unroll
        for (int c = 0; c < C; ++c) {
          const float m_new = fmaxf(m[c], kByTile ? top[c] : column_max(top[c]));
          const float f = fmaxf(__builtin_amdgcn_exp2f(m[c] - m_new), CAREFUL ? kLeast : 0.0f);
          m[c] = m_new;
          l[c] *= f;
#pragma unroll
          for (int j = 0; j < D / 16; ++j)
#pragma unroll
            for (int e = 0; e < 4; ++e) o[c][j][e] *= f;
        }
      }
#pragma unroll
      for (int c = 0; c < C; ++c) {
        base[c] = kByTile ? top[c] : m[c];
        share[c] = kByTile ? __builtin_amdgcn_exp2f(top[c] - m[c]) : 1.0f;
        float sum = 0.0f;
#pragma unroll
        for (int w = 0; w < 4; ++w) {
          float p[2];
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            const int r = w / 2, y = 2 * (w & 1) + e;
            p[e] = __builtin_amdgcn_exp2f(fmaf(s[c][r][y], mul, -base[c]));
            sum += p[e];
            if constexpr (BITS == 8) {
              p[e] *= vs[r][y];
              if (part) p[e] = (seen[c] >> (16 * r + y)) & 1u ? p[e] : 0.0f;
            }
            if constexpr (kByTile) {
              p[e] *= kLift;
              low |= p[e] < 0x1p-14f;
              s[c][r][y] = p[e];
            }
          }
          p_hi[c][w] = pack16<kPv>(p[0], p[1]);
          if constexpr (kTwo)
            p_two[c][w] = pack16<kPv>(p[0] - val16(p_hi[c][w] & 0xFFFFu, kPv), p[1] - val16(p_hi[c][w] >> 16, kPv));
        }
        l[c] = fmaf(share[c], sum, l[c]);
        if constexpr (kByTile) share[c] *= 1.0f / kLift;
      }
      uint32_t keep[2][2], any = 0u;
      if (part) {
        // values that no column may see are left out, whatever their bits, and those
        // that are no numbers for now
#pragma unroll
        for (int r = 0; r < 2; ++r) {
          keep[r][0] = keep[r][1] = 0u;
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const int tok = t + 16 * r + 4 * lg + e;
            const bool in = tok >= it.lo && tok < it.hi;
            if constexpr (BITS == 8) keep[r][0] |= in ? 0xFFu << (8 * e) : 0u;
            else keep[r][e / 2] |= in ? 0xFFFFu << (16 * (e & 1)) : 0u;
          }
        }
      }
      const auto values = [&](int j) {                           // the 1 KB piece j of the values
        u32x4 v = ld16(sv + j * 1024);
        if (part) {
#pragma unroll
          for (int w = 0; w < 4; ++w) {
            v[w] &= BITS == 8 ? keep[w & 1][0] : keep[w / 2][w & 1];
            const uint32_t z = odd_parts<BITS, kPv>(v[w]);
            any |= z;
            v[w] &= ~z;
          }
        }
        return v;
      };
      if constexpr (kByTile) {
        const bool two = __any(low);
        u32x4 p_lo[C];
        if (two) {
#pragma unroll
          for (int c = 0; c < C; ++c)
#pragma unroll
            for (int w = 0; w < 4; ++w)
              p_lo[c][w] = pack16<kPv>((s[c][w / 2][2 * (w & 1)] - val16(p_hi[c][w] & 0xFFFFu, kPv)) * kLow,
                                       (s[c][w / 2][2 * (w & 1) + 1] - val16(p_hi[c][w] >> 16, kPv)) * kLow);
        }
#pragma unroll
        for (int j = 0; j < D / 16; ++j) {
          const u32x4 v = values(j);
#pragma unroll
          for (int c = 0; c < C; ++c) {
            const f32x4 zero{0.0f, 0.0f, 0.0f, 0.0f};
            f32x4 hi = mma<kPv>(v, p_hi[c], zero);
            if (two) {
              const f32x4 lo = mma<kPv>(v, p_lo[c], zero);
#pragma unroll
              for (int e = 0; e < 4; ++e) hi[e] = fabsf(hi[e]) < INFINITY ? fmaf(lo[e], 1.0f / kLow, hi[e]) : hi[e];
            }
#pragma unroll
            for (int e = 0; e < 4; ++e) o[c][j][e] = fmaf(share[c], hi[e], o[c][j][e]);
          }
        }
      } else {
#pragma unroll
        for (int j = 0; j < 2 * kLoads; ++j) {
          const u32x4 v = values(j);
          if constexpr (BITS == 16) {
#pragma unroll
            for (int c = 0; c < C; ++c) o[c][j] = mma<kPv>(v, p_hi[c], o[c][j]);
          } else {
#pragma unroll
            for (int e = 0; e < 2; ++e) {
              const u32x4 w = widen8<kPv>(v[2 * e], v[2 * e + 1]);
#pragma unroll
              for (int c = 0; c < C; ++c) {
                o[c][2 * j + e] = mma<kPv>(w, p_hi[c], o[c][2 * j + e]);
                if constexpr (kTwo) o[c][2 * j + e] = mma<kPv>(w, p_two[c], o[c][2 * j + e]);
              }
            }
          }
        }
      }
      if constexpr (BITS == 16 && !CAREFUL) {
        if (part && __any(any != 0u)) *again = 1;
      } else if (part && __any(any != 0u)) {
        // one by one, to the columns that see them
        const uint8_t* vm = lds + stage * stage_bytes<BITS, D>() + 2 * kLoads * 1024;
#pragma unroll
        for (int c = 0; c < C; ++c) {
          for (int i = 0; i < kTile; ++i) {
            const int at = 4 * (i / 16) + i % 4;                   // token i's bit in lanes 16 (i / 4 mod 4) ..
            const bool none = CAREFUL && !(__shfl(static_cast<int>(some[c]), 16 * (i / 4 % 4) + col) >> at & 1);
            const uint32_t on = static_cast<uint32_t>(__shfl(static_cast<int>(seen[c]), col)) >> i & 1u;   // (bits of lane group 0: all)
#pragma unroll
            for (int j = 0; j < D / 16; ++j)
#pragma unroll
              for (int e = 0; e < 4; ++e) {
                const int place = 16 * (16 * (i / 4 % 4) + 4 * lg + e);
                float y = 0.0f;
                if constexpr (BITS == 16) {
                  const uint32_t b = *reinterpret_cast<const any_u16*>(vm + j * 1024 + place + 2 * (4 * (i / 16) + i % 4));
                  if (odd_parts<16, kPv>(b) & 0xFFFFu) y = val16(b, kPv);
                } else {
                  const uint32_t b = vm[(j / 2) * 1024 + place + 8 * (j & 1) + 4 * (i / 16) + i % 4];
                  if ((b & 0x7Fu) == 0x7Fu) y = __builtin_nanf("");
                }
                if (on && y != 0.0f) o[c][j][e] += none ? __builtin_nanf("") : y;
              }
          }
        }
      }
    }
    t = t1;
    t1 = t2;
    stage = stage + 1 < kStages ? stage + 1 : 0;
  }
  if constexpr (BITS == 16 && !CAREFUL) {                        // (an 8-bit NaN gives one, however often it is added)
    bool bad = false;
#pragma unroll
    for (int c = 0; c < C; ++c) {
      f32x4 sum = {0.0f, 0.0f, 0.0f, 0.0f};                      // 0, NaN where an output is no number
#pragma unroll
      for (int j = 0; j < D / 16; ++j)
#pragma unroll
        for (int e = 0; e < 4; ++e) sum[e] = fmaf(o[c][j][e], 0.0f, sum[e]);
      bad |= !(sum[0] + sum[1] + sum[2] + sum[3] == 0.0f) || (fabsf(m[c]) >= kFar && m[c] > kNoMax);
    }
    if (__any(bad)) *again = 1;
    __syncthreads();                                             // (and the last stage is read)
    if (*again != 0) return false;                               // (one wave is enough: they share the tiles)
  }
  if (!busy) return true;
#pragma unroll
  for (int c = 0; c < C; ++c) {
    float sum = l[c];
    sum += __shfl_xor(sum, 16);
    sum += __shfl_xor(sum, 32);
    const int cc = my0 + 16 * c + col;
    if (cc >= it.n_col) continue;
    if (whole) {
      const int64_t at = static_cast<int64_t>(x[c].row) * a.n_q_heads + h * g + (it.col0 + cc) % g;
      const float inv = sum == 0.0f ? 0.0f : 1.0f / sum;
#pragma unroll
      for (int j = 0; j < D / 16; ++j)
        *reinterpret_cast<u32x2*>(a.out + at * D + 16 * j + 4 * lg) =
            u32x2{pack16<ACT>(o[c][j][0] * inv, o[c][j][1] * inv), pack16<ACT>(o[c][j][2] * inv, o[c][j][3] * inv)};
      if (a.lse && lg == 0) a.lse[at] = sum == 0.0f ? -INFINITY : (m[c] + log2f(sum)) * kLn2;
    } else {
      // (the lanes of a column may hold different maxima only where it has seen nothing)
      const int64_t at = slot * (64 * C) + cc;
#pragma unroll
      for (int j = 0; j < D / 16; ++j) *reinterpret_cast<f32x4*>(a.part_o + at * D + 16 * j + 4 * lg) = o[c][j];
      if (lg == 0) {
        a.part_ml[2 * at] = m[c];
        a.part_ml[2 * at + 1] = sum;
      }
    }
  }
  return true;
}

// Workgroups of k_attn_tiles on a CU, by its registers (fp16 caches: more of them)
// and LDS.
constexpr int tiles_resident(int act, int bits, int D) {
  const bool more = act == PW_F16;
  return D <= 64 ? (more ? 3 : 4) : D <= 128 ? (more ? 2 : 3) : D <= 192 ? (more && bits == 16 ? 1 : 2) : 1;
}

template <int ACT, int BITS, int D, int C>
__global__ __launch_bounds__(256, tiles_resident(ACT, BITS, D)) void k_attn_tiles(RowsArgs a) {
  __shared__ __attribute__((aligned(1024))) uint8_t lds[kStages * stage_bytes<BITS, D>()];
  __shared__ int again;
  Item it;
  Part p;
  again = 0;
  wait_lds<0>();                                                 // (a barrier of the first tile before any other write)
  if (!split_of(a, 64 * C, lane_id(), &it, &p)) return;
  const bool done = attend_tiles<ACT, BITS, D, C, false>(a, lds, &again, it, p.begin, p.end, p.whole, p.slot);
  if constexpr (BITS == 16) {
    if (!done) attend_tiles<ACT, BITS, D, C, true>(a, lds, &again, it, p.begin, p.end, p.whole, p.slot);
  }
}

// Joins the parts of 4 `per` columns of an item, `per` a wave, in a fixed order (lanes
// hold four channels, so that heads of 64 take four parts at once, of 128 two), and
// writes the rows of items that no share has.
template <int ACT, int D>
__global__ __launch_bounds__(256) void k_rows_join(RowsArgs a, int cols, int per) {
  constexpr int kLanes = D <= 64 ? 16 : D <= 128 ? 32 : 64, kAtOnce = 64 / kLanes;
  const int lane = lane_id(), wave = __builtin_amdgcn_readfirstlane(static_cast<int>(threadIdx.x) >> 6);
  const int H = a.kv.n_kv_heads, h = blockIdx.x % H, item = blockIdx.x / H, g = a.n_q_heads / H;
  Item it;
  int n = 0;
  int64_t at0 = 0;
  if (a.n_shares == 0) {
    const int rest = static_cast<int>(a.items - a.whole);
    if (!item_at(a, rest - 1 - item, h, cols, lane, &it)) return;
    n = (it.tiles + a.split_tiles - 1) / a.split_tiles;
    if (n <= 1) return;
    at0 = (h * static_cast<int64_t>(rest) + item) * a.n_splits * cols;
  } else if (!item_at(a, item, h, cols, lane, &it)) {
    return;
  } else if (it.tiles > 0) {
    const int32_t* meta = a.meta + 2 * (h * a.items + item);
    n = meta[1];
    if (n <= 1) return;
    at0 = (h * (a.n_shares + a.items) + meta[0]) * cols;
  }
  const int sub = lane / kLanes, d = 4 * (lane % kLanes);
  for (int i = 0; i < per; ++i) {
    const int c = (blockIdx.y * per + i) * 4 + wave;
    if (c >= it.n_col) return;
    const int64_t at = at0 + c;
    float mx = kNoMax;
    for (int s = lane; s < n; s += 64) mx = fmaxf(mx, a.part_ml[2 * (at + static_cast<int64_t>(s) * cols)]);
#pragma unroll
    for (int o = 32; o; o >>= 1) mx = fmaxf(mx, __shfl_xor(mx, o));
    f32x4 acc = {0.0f, 0.0f, 0.0f, 0.0f};
    float sum = 0.0f;
#pragma unroll 4
    for (int s = sub; s < n; s += kAtOnce) {
      const int64_t y = at + static_cast<int64_t>(s) * cols;
      const float f = fmaxf(__builtin_amdgcn_exp2f(a.part_ml[2 * y] - mx), kLeast);
      sum = fmaf(f, a.part_ml[2 * y + 1], sum);
      if (d < D) {
        const f32x4 x = *reinterpret_cast<const f32x4*>(a.part_o + y * D + d);
#pragma unroll
        for (int j = 0; j < 4; ++j) acc[j] = fmaf(f, x[j], acc[j]);
      }
    }
#pragma unroll
    for (int o = kLanes; o < 64; o <<= 1) {
      sum += __shfl_xor(sum, o);
#pragma unroll
      for (int j = 0; j < 4; ++j) acc[j] += __shfl_xor(acc[j], o);
    }
    const int64_t row = static_cast<int64_t>(it.row0 + (it.col0 + c) / g) * a.n_q_heads + h * g + (it.col0 + c) % g;
    const float inv = sum == 0.0f ? 0.0f : 1.0f / sum;
    if (sub == 0 && d < D)
      *reinterpret_cast<u32x2*>(a.out + row * D + d) =
          u32x2{pack16<ACT>(acc[0] * inv, acc[1] * inv), pack16<ACT>(acc[2] * inv, acc[3] * inv)};
    if (a.lse && lane == 0) a.lse[row] = sum == 0.0f ? -INFINITY : (mx + log2f(sum)) * kLn2;
  }
}

constexpr int kTileCols = 2;          // column tiles of a wave of k_attn_tiles
constexpr int kPiece = 72;            // tiles of a split in a batch

template <int ACT, int BITS, int D>
hipError_t launch_d(const RowsArgs& a, const RowsPlan& p, hipStream_t st) {
  const int64_t rest = p.items - p.whole, grid = (p.n_shares ? p.n_shares : p.whole + rest * p.n_splits) * a.kv.n_kv_heads;
  if (grid >= (1 << 23) || p.items * a.kv.n_kv_heads >= (1 << 23)) return hipErrorInvalidConfiguration;
  const uint32_t n = static_cast<uint32_t>(grid);
  constexpr int kThreads = 64 * kRowsWaves;
  constexpr int kTwo = BITS == 16 ? 2 : 1;                       // (8-bit caches have one column tile: rows_plan)
  if (p.many) k_attn_tiles<ACT, BITS, D, kTileCols><<<n, 256, 0, st>>>(a);
  else if (p.col_tiles == 1 && p.n_shares) k_attn_rows<ACT, BITS, D, 1, true><<<n, kThreads, 0, st>>>(a);
  else if (p.col_tiles == 1) k_attn_rows<ACT, BITS, D, 1, false><<<n, kThreads, 0, st>>>(a);
  else if (p.n_shares) k_attn_rows<ACT, BITS, D, kTwo, true><<<n, kThreads, 0, st>>>(a);
  else k_attn_rows<ACT, BITS, D, kTwo, false><<<n, kThreads, 0, st>>>(a);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || p.slots == 0) return e;
  const int cols = (p.many ? 64 : 16) * p.col_tiles;
  // (four columns a wave where there are many: the search for the item is most of it)
  const int per = p.many ? 4 : 1;
  k_rows_join<ACT, D><<<dim3(static_cast<uint32_t>(rest * a.kv.n_kv_heads), cols / (4 * per)), 256, 0, st>>>(a, cols, per);
  return hipGetLastError();
}

template <int ACT, int BITS>
hipError_t launch_bits(const RowsArgs& a, const RowsPlan& p, hipStream_t st) {
  switch (a.kv.head_dim) {
    case 64: return launch_d<ACT, BITS, 64>(a, p, st);
    case 128: return launch_d<ACT, BITS, 128>(a, p, st);
    case 192: return launch_d<ACT, BITS, 192>(a, p, st);
    case 256: return launch_d<ACT, BITS, 256>(a, p, st);
  }
  return hipErrorInvalidValue;
}

}  // namespace

RowsPlan rows_plan(int B, int T, int n_q_heads, int n_kv_heads, int head_dim, int act, int bits, int max_len, int window) {
  RowsPlan p{};
  p.col_tiles = p.n_splits = p.split_tiles = 1;
  if (B == 0 || T == 0) return p;
  const int64_t g = n_q_heads / n_kv_heads, rows = (static_cast<int64_t>(T) + B - 1) / B, cols = g * rows;
  p.many = g * T > 64 * static_cast<int64_t>(B);
  // 32 columns a wave where there are workgroups for the chip, 16 bits: 64 trees of up
  // to 16 tokens, as above, 135 us, with 16 columns 143; in 8 bits 128 and 116; one tree
  // of 16 after 8000 tokens 39 and 33 (27 since its join takes parts side by side).
  const auto items_of = [&](int64_t group) { return g * T / group + (B < T ? B : T); };
  if (p.many) p.col_tiles = kTileCols;
  else p.col_tiles = cols > 16 && bits == 16 && items_of(32) * n_kv_heads >= 256 ? 2 : 1;
  const int64_t group = (p.many ? 64 : 16) * p.col_tiles;
  p.items = items_of(group);
  int64_t tiles = (static_cast<int64_t>(max_len) + kTile - 1) / kTile;
  if (window > 0) {
    const int64_t w = (static_cast<int64_t>(window) + T + 2 * kTile - 2) / kTile;
    tiles = w < tiles ? w : tiles;
  }
  if (tiles == 0) tiles = 1;
  p.split_tiles = static_cast<int>(tiles);
  const int64_t items = p.items * n_kv_heads;
  if (!p.many) {
    const int64_t resident = 256 * rows_resident(bits, head_dim, p.col_tiles);
    p.least = 16;
    // Shares where items are few and long: one tree of 16 after 8000 tokens 27 us, a
    // workgroup per item 60. With an item and a half for every place on the chip the
    // second is as fast, and needs no join.
    if (items * 2 < resident * 3 && tiles >= 4 * p.least && p.items * tiles < (int64_t(1) << 31) - (1 << 20)) {
      p.n_shares = resident / n_kv_heads > 0 ? resident / n_kv_heads : 1;
      p.slots = (p.n_shares + p.items) * n_kv_heads * group;
    }
  } else if (tiles >= 8) {
    const int per_cu = tiles_resident(act, bits, head_dim);
    const int64_t resident = 256 * per_cu, most = tiles / 4;
    int64_t n = 1;
    // Splits. In a batch lengths may be unlike: pieces of kPiece tiles at most: 16 ragged trees of up to 60 tokens after up to 32768 in 8
    // bits in 1, 2, 4, 6, 12, 16 splits (us) 1434, 798, 574, 401, 372, 377; 500 rows
    // beside 31 single ones of up to 3000 tokens in 1, 2, 4, 8 splits 102, 79, 83, 88.
    // Within that the cheapest count by rounds of workgroups over the chip, the first
    // rounds whole where items are many: 4096 rows after 12288 tokens, 1024 workgroups on 768 places, unsplit 1003
    // us, all in 2, 3, 4 splits 937, 946, 965, the last round alone in 2 splits 919; 512
    // rows after 3000 tokens in 1, 2, 4, 6, 8 splits 113, 74, 58, 59, 68; 4096 rows from
    // the beginning, spans of all lengths, 151, in 2 splits 197.
    // A few rows of one sequence take small pieces, too: 7 rows x 16 heads of 256 after 644
    // tokens in 8 bits, one workgroup, 59 us whole, 28 in five.
    const bool pieces = B > 1 && items < 2 * resident;
    const double unit = (per_cu > 2 ? 0.5 * per_cu : 1.0) * head_dim / 128;   // us a tile
    const double part = group * (head_dim + 2) * 8 / 4e6;        // us to write and read a part
    const int64_t tri = rows / kTile < tiles ? rows / kTile : tiles;
    int64_t least = 1;
    if (pieces) {
      // (not more than eight rounds of them: a bound of the lengths far above the lengths
      // themselves would cost a workspace of as many parts)
      const int64_t cap = 8 * resident / items;
      least = (tiles + kPiece - 1) / kPiece;
      least = least < cap ? least : cap > 1 ? cap : 1;
    }
    const int64_t whole_step = items / resident > 0 ? items / resident : 1;
    double best = 0.0;
    for (int64_t k = least; k <= least + 31 && k <= most; ++k)
      for (int64_t whole = 0; whole <= (k > 1 && !pieces && tri <= tiles / 2 ? items / resident : 0); whole += whole_step) {
        const int64_t left = items - whole * resident, rounds = (left * k + resident - 1) / resident;
        double t = static_cast<double>(whole) * (tiles + 3) + rounds * (static_cast<double>(tiles) / k + 3);
        if (tri > tiles / 2) {                                   // spans of all lengths: short ones fill the gaps
          const double mean = (tiles - 0.5 * tri) * items / resident, longest = static_cast<double>(tiles) / k;
          t = (mean > longest ? mean : longest) + 3 * rounds;
        }
        t *= unit;
        if (k > 1) t += 5.0 + left * k * part;
        if (best == 0.0 || t < best) {
          best = t;
          n = k;
          p.whole = whole * resident / n_kv_heads;
        }
      }
    const int64_t per = (tiles + n - 1) / n;
    n = (tiles + per - 1) / per;
    if (n == 1) p.whole = 0;
    p.n_splits = static_cast<int>(n);
    p.split_tiles = static_cast<int>(per);
    if (n > 1) p.slots = (p.items - p.whole) * n_kv_heads * n * group;
  }
  if (p.slots)
    p.ws_bytes = static_cast<size_t>(p.slots) * (head_dim + 2) * sizeof(float) + static_cast<size_t>(p.items) * n_kv_heads * 8;
  return p;
}

hipError_t launch_attn_rows(const RowsArgs& a, const RowsPlan& p, hipStream_t st) {
  if (a.kv.act == PW_BF16)
    return a.kv.bits == 16 ? launch_bits<PW_BF16, 16>(a, p, st) : launch_bits<PW_BF16, 8>(a, p, st);
  return a.kv.bits == 16 ? launch_bits<PW_F16, 16>(a, p, st) : launch_bits<PW_F16, 8>(a, p, st);
}

}  // namespace pw
