// Device helpers shared by the HIP kernels of libpagedweight.so (gfx950).
#pragma once

#include <hip/hip_runtime.h>
#include <cstdint>

#include "pw.h"

namespace pw {
namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

// ---------------------------------------------------------------------------
// 16-bit float helpers
// ---------------------------------------------------------------------------

__device__ __forceinline__ float bf16_val(uint32_t h) { return __uint_as_float(h << 16); }
__device__ __forceinline__ float f16_val(uint32_t h) {
  return static_cast<float>(__builtin_bit_cast(_Float16, static_cast<uint16_t>(h)));
}
__device__ __forceinline__ float val16(uint32_t h, int fmt) {
  return fmt == PW_BF16 ? bf16_val(h & 0xFFFFu) : f16_val(h & 0xFFFFu);
}
// round to nearest even (finite inputs)
__device__ __forceinline__ uint32_t bf16_rne(float f) {
  const uint32_t u = __float_as_uint(f);
  return (u + 0x7FFFu + ((u >> 16) & 1u)) >> 16;
}
__device__ __forceinline__ uint32_t f16_rne(float f) {
  return __builtin_bit_cast(uint16_t, static_cast<_Float16>(f));
}
__device__ __forceinline__ uint32_t rne16(float f, int fmt) {
  return fmt == PW_BF16 ? bf16_rne(f) : f16_rne(f);
}

// Directed rounding of an fp32 value to bf16: truncation moves toward zero,
// so it rounds down for positive inputs and up for negative ones.
__device__ __forceinline__ uint32_t bf16_down(float x) {
  if (x == 0.0f) return 0u;
  const uint32_t u = __float_as_uint(x), t = u >> 16;
  if ((u & 0xFFFFu) == 0u) return t;
  return (u >> 31) ? t + 1u : t;
}
__device__ __forceinline__ uint32_t bf16_up(float x) {
  if (x == 0.0f) return 0u;
  const uint32_t u = __float_as_uint(x), t = u >> 16;
  if ((u & 0xFFFFu) == 0u) return t;
  const uint32_t r = (u >> 31) ? t : t + 1u;
  return r == 0x8000u ? 0u : r;
}
// fp16: convert to nearest, then step one ulp if it landed on the wrong side.
__device__ __forceinline__ uint32_t f16_step(uint32_t h, bool up) {
  if ((h & 0x7FFFu) == 0u) return up ? 0x0001u : 0x8001u;
  const bool neg = (h >> 15) != 0;
  return (neg != up) ? h + 1u : h - 1u;
}
__device__ __forceinline__ uint32_t f16_down(float x) {
  if (x == 0.0f) return 0u;
  uint32_t h = f16_rne(x);
  if (f16_val(h) > x) h = f16_step(h, false);
  return (h & 0x7FFFu) == 0u ? 0u : h;
}
__device__ __forceinline__ uint32_t f16_up(float x) {
  if (x == 0.0f) return 0u;
  uint32_t h = f16_rne(x);
  if (f16_val(h) < x) h = f16_step(h, true);
  return (h & 0x7FFFu) == 0u ? 0u : h;
}
__device__ __forceinline__ uint32_t round_down16(float x, int fmt) {
  return fmt == PW_BF16 ? bf16_down(x) : f16_down(x);
}
__device__ __forceinline__ uint32_t round_up16(float x, int fmt) {
  return fmt == PW_BF16 ? bf16_up(x) : f16_up(x);
}

__device__ __forceinline__ int lane_id() {
  return __builtin_amdgcn_mbcnt_hi(~0u, __builtin_amdgcn_mbcnt_lo(~0u, 0u));
}

template <int ACT>
__device__ __forceinline__ f32x4 mma(u32x4 a, u32x4 b, f32x4 c) {
  if constexpr (ACT == PW_BF16)
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a),
                                                   __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
  else
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a),
                                                  __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
}

__device__ __forceinline__ u32x4 ld16(const uint8_t* p) { return *reinterpret_cast<const u32x4*>(p); }
// Weights are streamed once: nontemporal loads.
__device__ __forceinline__ u32x4 ld16_nt(const uint8_t* p) {
  return __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(p));
}

// Between writes to LDS by some lanes of a wave and reads of them by others, and
// before the next writes over what was read. The hardware keeps a wave's LDS
// accesses in order, the compiler need not: it sees one lane's addresses and types
// and may take a read for unrelated to a write. (No instruction comes of it.)
__device__ __forceinline__ void wave_exchange() {
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
  __builtin_amdgcn_wave_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}
// Parts of memory that is accessed in other types, too.
typedef uint32_t __attribute__((may_alias)) any_u32;
typedef uint16_t __attribute__((may_alias)) any_u16;

// Two values rounded to nearest even, as one 32-bit pair. NaN stays NaN (the
// hardware's conversions keep it; the bit formula of bf16_rne need not).
template <int ACT>
__device__ __forceinline__ uint32_t pack16(float a, float b) {
  typedef __bf16 bf16x2_t __attribute__((ext_vector_type(2)));
  typedef _Float16 f16x2_t __attribute__((ext_vector_type(2)));
  if constexpr (ACT == PW_BF16)
    return __builtin_bit_cast(uint32_t, bf16x2_t{static_cast<__bf16>(a), static_cast<__bf16>(b)});
  else
    return __builtin_bit_cast(uint32_t, f16x2_t{static_cast<_Float16>(a), static_cast<_Float16>(b)});
}

// ---------------------------------------------------------------------------
// 8-bit floating point (e4m3) with a scale per group
// ---------------------------------------------------------------------------

template <int CTRL>
__device__ __forceinline__ float dpp_f32(float x) {
  return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(x), CTRL, 0xF, 0xF, false));
}
// Largest value of the lane's row of 16 lanes, in every lane of it.
__device__ __forceinline__ float row16_max(float m) {
  m = fmaxf(m, dpp_f32<0xB1>(m));    // quad_perm 1,0,3,2
  m = fmaxf(m, dpp_f32<0x4E>(m));    // quad_perm 2,3,0,1
  m = fmaxf(m, dpp_f32<0x141>(m));   // row_half_mirror
  return fmaxf(m, dpp_f32<0x140>(m));   // row_mirror
}
// Scale of a group of largest magnitude m.
__device__ __forceinline__ float f8_scale(float m) { return fmaxf(m / 448.0f, 0x1p-126f); }
// The codes of eight values v of one group: e4m3 of the correctly rounded v / s
// (at most 448 (1 + 2^-23), which rounds to 448). The division's own steps are
// mostly about the divisor, so they are done once: y = 1 / s, correctly rounded;
// q = v y is off by less than two units, q + (v - q s) y (the remainder exact)
// by less than one, and the same correction of that rounds to what v / s rounds
// to (Markstein), for every v / s that is not coded 0 while no step leaves the
// normal range: elsewhere, divisions.
__device__ __forceinline__ u32x2 f8_codes8(const float* v, float s) {
  float q[8];
  if (s > 0x1p-90f && s < 0x1p90f) {
    const float y = 1.0f / s;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const float q0 = v[i] * y, q1 = fmaf(fmaf(-q0, s, v[i]), y, q0);
      q[i] = fmaf(fmaf(-q1, s, v[i]), y, q1);
    }
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) q[i] = v[i] / s;
  }
  u32x2 o;
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    int c = __builtin_amdgcn_cvt_pk_fp8_f32(q[4 * i], q[4 * i + 1], 0, false);
    c = __builtin_amdgcn_cvt_pk_fp8_f32(q[4 * i + 2], q[4 * i + 3], c, true);
    o[i] = static_cast<uint32_t>(c);
  }
  return o;
}

__device__ __forceinline__ int clampi(int v, int lo, int hi) { return v < lo ? lo : (v > hi ? hi : v); }

// Bytes of one 16-row x 128-value tile of a page at `B` bits.
template <int B> constexpr int tile_bytes() { return B == 16 ? 4096 : B == 8 ? 2048 : 1024; }

}  // namespace
}  // namespace pw
