// Product of 8-bit matrices with block scales, gfx950.
//
// One matrix instruction of 16 x 16 x 128 covers exactly one scale block of K,
// so every block's product starts from zero and enters the fp32 sum with one
// multiply-add per element. Weight rows are the row operand: their scale is one
// number per 128 rows, and a lane, which holds four rows of one token's column,
// multiplies all of them by the same w_scale * a_scale. (Both operands hold
// bytes 32 g .. 32 g + 31 of their row's block in lane group g; which k that is
// for the hardware does not matter, it is the same for both.)
#include "pw_device.hpp"
#include "pw_ops.hpp"

namespace pw {
namespace {

typedef int i32x8 __attribute__((ext_vector_type(8)));

struct F8Frag {
  u32x4 lo, hi;
};
__device__ __forceinline__ i32x8 frag(const F8Frag& f) {
  return i32x8{static_cast<int>(f.lo[0]), static_cast<int>(f.lo[1]), static_cast<int>(f.lo[2]), static_cast<int>(f.lo[3]),
               static_cast<int>(f.hi[0]), static_cast<int>(f.hi[1]), static_cast<int>(f.hi[2]), static_cast<int>(f.hi[3])};
}
// Scale operands of zero select the instruction without scales.
__device__ __forceinline__ f32x4 mma8(const F8Frag& a, const F8Frag& b) {
  return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(frag(a), frag(b), f32x4{0.0f, 0.0f, 0.0f, 0.0f}, 0, 0, 0, 0,
                                                          0, 0);
}

__device__ __forceinline__ void store_y(const Gemm8Args& a, int m, int n, float v) {
  const int64_t i = m * a.ldy + n;
  if (a.y_type == PW_F32) static_cast<float*>(a.y)[i] = v;
  else if (a.y_type == PW_BF16) static_cast<uint16_t*>(a.y)[i] = static_cast<uint16_t>(pack16<PW_BF16>(v, 0.0f));
  else static_cast<uint16_t*>(a.y)[i] = static_cast<uint16_t>(pack16<PW_F16>(v, 0.0f));
}

// Streaming kernel: 16 weight rows x 16 MT tokens per workgroup, whose four
// waves take every fourth K block and join in LDS in a fixed order.
constexpr int kStreamWaves = 4;

template <int MT>
__global__ __launch_bounds__(64 * kStreamWaves) void k_gemm8_stream(Gemm8Args a) {
  __shared__ f32x4 part[kStreamWaves][MT][64];
  const int wave = static_cast<int>(threadIdx.x) >> 6, lane = lane_id();
  const int c = lane & 15, lg = lane >> 4;
  const int n_tiles = (a.N + 15) / 16;
  const int nt = static_cast<int>(blockIdx.x) % n_tiles, m0 = static_cast<int>(blockIdx.x) / n_tiles * (16 * MT);
  const int KB = a.K / 128;
  // rows past the end repeat the last one; nothing of them is stored
  const int n_row = 16 * nt + c < a.N ? 16 * nt + c : a.N - 1;
  const uint8_t* w = a.w + n_row * a.ldw + 32 * lg;
  const float* ws = a.w_scale + static_cast<size_t>(nt / 8) * KB;
  const uint8_t* x[MT];
  const float* xs[MT];
#pragma unroll
  for (int i = 0; i < MT; ++i) {
    const int m = m0 + 16 * i + c < a.M ? m0 + 16 * i + c : a.M - 1;
    x[i] = a.a + m * a.lda + 32 * lg;
    xs[i] = a.a_scale + static_cast<size_t>(m) * KB;
  }
  f32x4 acc[MT];
#pragma unroll
  for (int i = 0; i < MT; ++i) acc[i] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
  for (int b = wave; b < KB; b += kStreamWaves) {
    const F8Frag wf = {ld16_nt(w + b * 128), ld16_nt(w + b * 128 + 16)};
    const float s = ws[b];
#pragma unroll
    for (int i = 0; i < MT; ++i) {
      const F8Frag xf = {ld16(x[i] + b * 128), ld16(x[i] + b * 128 + 16)};
      const float f = s * xs[i][b];
      const f32x4 d = mma8(wf, xf);
#pragma unroll
      for (int j = 0; j < 4; ++j) acc[i][j] = fmaf(d[j], f, acc[i][j]);
    }
  }
#pragma unroll
  for (int i = 0; i < MT; ++i) part[wave][i][lane] = acc[i];
  __syncthreads();
  for (int i = wave; i < MT; i += kStreamWaves) {
    f32x4 v = part[0][i][lane];
#pragma unroll
    for (int q = 1; q < kStreamWaves; ++q) v += part[q][i][lane];
    const int m = m0 + 16 * i + c;
    if (m >= a.M) continue;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int n = 16 * nt + 4 * lg + j;
      if (n < a.N) store_y(a, m, n, v[j]);
    }
  }
}

template <int MT>
hipError_t launch_stream(const Gemm8Args& a, hipStream_t st) {
  const int64_t grid = static_cast<int64_t>((a.N + 15) / 16) * ((a.M + 16 * MT - 1) / (16 * MT));
  if (grid > (1 << 23)) return hipErrorInvalidConfiguration;
  k_gemm8_stream<MT><<<static_cast<uint32_t>(grid), 64 * kStreamWaves, 0, st>>>(a);
  return hipGetLastError();
}

}  // namespace

size_t gemm8_workspace(int, int, int) { return 0; }

hipError_t launch_gemm8(const Gemm8Args& a, hipStream_t st) {
  if (a.M <= 16) return launch_stream<1>(a, st);
  if (a.M <= 32) return launch_stream<2>(a, st);
  return launch_stream<4>(a, st);
}

}  // namespace pw
