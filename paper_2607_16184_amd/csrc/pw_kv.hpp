// What the kernels around the paged KV cache share (gfx950): where a token's
// elements lie, and the pieces of attention in matrix instructions.
#pragma once

#include "pw_device.hpp"
#include "pw_ops.hpp"

namespace pw {
namespace {

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

// ---------------------------------------------------------------------------
// Writing a token
// ---------------------------------------------------------------------------

__device__ __forceinline__ bool slot_ok(const KvArgs& kv, int64_t slot) {
  return slot >= 0 && slot / kv.block_tokens < kv.n_blocks;
}

// Channels 8 c .. 8 c + 7 of a token's key (is_v 0) or value (1) of head h into a
// 16-bit cache.
__device__ __forceinline__ void put16(const KvArgs& kv, u32x4 raw, int64_t slot, int h, int is_v, int c) {
  const int D = kv.head_dim, P = kv.block_tokens, t = static_cast<int>(slot % P);
  uint8_t* dst = kv.pool + slot / P * kv.block_stride + static_cast<size_t>(2 * h + is_v) * P * D * 2;
  if (8 * c >= D) return;
  if (!is_v) {
    *reinterpret_cast<u32x4*>(dst + ((t / 16) * (D / 32) + c / 4) * 1024 + 16 * (16 * (c & 3) + t % 16)) = raw;
  } else {
    uint16_t* p = reinterpret_cast<uint16_t*>(dst + ((t / 32) * (D / 16) + c / 2) * 1024) +
                  8 * (16 * (t / 4 % 4) + 8 * (c & 1)) + 4 * (t / 16 % 2) + t % 4;
#pragma unroll
    for (int j = 0; j < 8; ++j) p[8 * j] = static_cast<uint16_t>(raw[j / 2] >> (16 * (j & 1)));
  }
}

// The same into an 8-bit cache, by G neighbouring lanes (a power of two, at least
// D / 8), lane c of them with the values f of its eight channels (zeros past D).
__device__ __forceinline__ void put8(const KvArgs& kv, const float* f, int64_t slot, int h, int is_v, int c, int G) {
  const int D = kv.head_dim, P = kv.block_tokens, H = kv.n_kv_heads, t = static_cast<int>(slot % P);
  uint8_t* blk = kv.pool + slot / P * kv.block_stride;
  uint8_t* dst = blk + static_cast<size_t>(2 * h + is_v) * P * D;
  float m = 0.0f;
#pragma unroll
  for (int j = 0; j < 8; ++j) m = fmaxf(m, fabsf(f[j]));
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

template <int ACT>
__device__ __forceinline__ void unpack8(u32x4 v, float* f) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    f[2 * i] = val16(v[i], ACT);
    f[2 * i + 1] = val16(v[i] >> 16, ACT);
  }
}

// ---------------------------------------------------------------------------
// Attention
// ---------------------------------------------------------------------------

constexpr int kTile = 32;             // tokens; the columns of a tile's products are queries
constexpr float kNoMax = -3.402823466e38f;   // no finite score is below it, and exp2(-inf - it) = 0
constexpr float kSlack = 8.0f;
constexpr float kLift = 32768.0f, kLow = 4096.0f;   // factors of fp16 probabilities and of their second term

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

// Largest value of a column (lanes l, l + 16, l + 32, l + 48), in each of its
// lanes. (Rows 0 and 1, 2 and 3 trade places, then the halves.)
__device__ __forceinline__ float column_max(float x) {
  const uint32_t u = __float_as_uint(x);
  const auto a = __builtin_amdgcn_permlane16_swap(u, u, false, false);
  const uint32_t t = __float_as_uint(fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1])));
  const auto b = __builtin_amdgcn_permlane32_swap(t, t, false, false);
  return fmaxf(__uint_as_float(b[0]), __uint_as_float(b[1]));
}

}  // namespace
}  // namespace pw
