// Between a projection's rows and the attention, gfx950: norms of query and key
// heads with the position rotation, into rows or (keys, with the values) into the
// paged cache (k_heads), and drafted tokens moved together in it (k_kv_keep).
#include "pw_turn.hpp"

namespace pw {
namespace {

// ---------------------------------------------------------------------------
// Norm and rotation
// ---------------------------------------------------------------------------

template <int ACT, int BITS>
__global__ __launch_bounds__(256) void k_heads(HeadsArgs a, HeadsCut k) {
  heads_wave<ACT, BITS>(a, static_cast<int64_t>(blockIdx.x) * 4 + __builtin_amdgcn_readfirstlane(static_cast<int>(threadIdx.x) >> 6),
                        k.G, k.steps, k.parts);
}

template <int ACT>
hipError_t heads(const HeadsArgs& a, hipStream_t st) {
  const int bits = a.slots ? a.kv.bits : 0;
  const HeadsCut k = heads_cut(a.T, a.D, a.n_q + (bits ? 2 : 1) * a.n_k);
  if (k.blocks > INT32_MAX) return hipErrorInvalidConfiguration;
  const dim3 g(static_cast<uint32_t>(k.blocks));
  if (bits == 0) k_heads<ACT, 0><<<g, 256, 0, st>>>(a, k);
  else if (bits == 16) k_heads<ACT, 16><<<g, 256, 0, st>>>(a, k);
  else k_heads<ACT, 8><<<g, 256, 0, st>>>(a, k);
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
// writes: one sequence 3.1 us, 64 trees of 60 tokens in 8 bits 7.8.
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
  if (a.slots && append_by_runs(a)) return launch_append_runs(a, st);
  return a.act == PW_BF16 ? heads<PW_BF16>(a, st) : heads<PW_F16>(a, st);
}

hipError_t launch_kv_keep(const KeepArgs& a, hipStream_t st) {
  const dim3 g(a.kv.n_kv_heads, a.B);
  if (a.kv.bits == 16) k_kv_keep<16><<<g, 256, 0, st>>>(a);
  else k_kv_keep<8><<<g, 256, 0, st>>>(a);
  return hipGetLastError();
}

}  // namespace pw
