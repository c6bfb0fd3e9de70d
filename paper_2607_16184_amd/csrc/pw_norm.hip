// Root-mean-square norm with the residual's addition, gfx950. One pass: a row
// is read once into registers (8 values of 16 bits per lane and chunk), its
// sum of squares is joined across the row's waves, and every output is written
// from the registers. Bound by HBM; a group of 128 output columns is 16
// neighbouring lanes of 8 values, so its largest magnitude is four lane
// exchanges inside a row of 16 lanes.
//
// Measured: 4095 rows of 4096 with residual, all outputs (151 MB), over eight sets of
// buffers in turn (1.2 GB) 29.4 us (5.2 TB/s; a large copy reaches 4.9), over two
// 24.5, as the 256 MB cache before the memory then holds a part of the inputs. Four
// waves per row of 4096 take the same time as the eight used; with cached stores,
// where eight took 31 us (two sets), two took 34 and one 41.
#include "pw_device.hpp"
#include "pw_ops.hpp"

namespace pw {
namespace {

template <int ACT>
__device__ __forceinline__ void unpack8(u32x4 v, float* f) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    f[2 * i] = val16(v[i], ACT);
    f[2 * i + 1] = val16(v[i] >> 16, ACT);
  }
}

// 16-bit outputs of this size and more are stored past the caches. Past them /
// cached (us, 8 sets of buffers in turn): 2048 rows of 4096 16.8 / 18.9, 4095 29.4 /
// 32.3, 8192 53 / 58; with a kernel after it that reads both outputs 28.0 / 27.6, 47.7
// / 47.7, 88.8 / 89.0: the gain is left where what comes next takes the 8-bit rows.
// Less than that stays in the caches (64 rows 3.4 us either way). 8-bit outputs past
// the caches gained nothing.
constexpr int64_t kStreamBytes = 16 << 20;

template <bool STREAM>
__device__ __forceinline__ void store_row(uint16_t* p, u32x4 v) {
  if constexpr (STREAM) __builtin_nontemporal_store(v, reinterpret_cast<u32x4*>(p));
  else *reinterpret_cast<u32x4*>(p) = v;
}

// WPR waves share a row of at most WPR * 64 * CH * 8 values; a workgroup has
// max(WPR, 4) waves.
template <int ACT, int WPR, int CH, bool STREAM>
__global__ __launch_bounds__(64 * (WPR < 4 ? 4 : WPR)) void k_rms_norm(NormArgs a) {
  constexpr int kThreads = 64 * (WPR < 4 ? 4 : WPR);
  constexpr int kRows = kThreads / (64 * WPR);           // rows of a workgroup at once
  __shared__ float part[2][kThreads / 64];
  const int wave = static_cast<int>(threadIdx.x) >> 6, lane = lane_id();
  const int t = (wave % WPR) * 64 + lane;                // thread of the row
  const int H8 = a.H / 8;
  int turn = 0;
  for (int64_t base = static_cast<int64_t>(blockIdx.x) * kRows; base < a.T; base += static_cast<int64_t>(gridDim.x) * kRows) {
    const int64_t row = base + wave / WPR;
    const bool live = row < a.T;                         // wave-uniform
    float z[CH][8];
    float sq = 0.0f;
    if (live) {
      const uint16_t* x = a.x + row * a.ldx;
      const uint16_t* r = a.residual ? a.residual + row * a.ldr : nullptr;
#pragma unroll
      for (int c = 0; c < CH; ++c) {
        const int i = c * WPR * 64 + t;
        if (i < H8) {
          unpack8<ACT>(ld16(reinterpret_cast<const uint8_t*>(x + 8 * i)), z[c]);
          if (r) {
            float f[8];
            unpack8<ACT>(ld16(reinterpret_cast<const uint8_t*>(r + 8 * i)), f);
#pragma unroll
            for (int j = 0; j < 8; ++j) z[c][j] += f[j];
          }
        } else {
#pragma unroll
          for (int j = 0; j < 8; ++j) z[c][j] = 0.0f;
        }
#pragma unroll
        for (int j = 0; j < 8; ++j) sq = fmaf(z[c][j], z[c][j], sq);
      }
    }
#pragma unroll
    for (int o = 32; o; o >>= 1) sq += __shfl_xor(sq, o);
    if constexpr (WPR > 1) {
      // two slots in turn: the next row's sums cannot overtake this row's reads
      if (lane == 0) part[turn][wave] = sq;
      __syncthreads();
      sq = 0.0f;
#pragma unroll
      for (int w = 0; w < WPR; ++w) sq += part[turn][wave / WPR * WPR + w];
      turn ^= 1;
    }
    if (!live) continue;
    const float rstd = 1.0f / sqrtf(sq / static_cast<float>(a.H) + a.eps);
#pragma unroll
    for (int c = 0; c < CH; ++c) {
      const int i = c * WPR * 64 + t;
      if (i >= H8) continue;
      const int64_t at = row * a.H + 8 * i;
      if (a.sum_out) {
        u32x4 o;
#pragma unroll
        for (int j = 0; j < 4; ++j) o[j] = pack16<ACT>(z[c][2 * j], z[c][2 * j + 1]);
        store_row<STREAM>(a.sum_out + at, o);
      }
      float y[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) y[j] = z[c][j] * rstd;
      if (a.weight) {
        float w[8];
        unpack8<ACT>(ld16(reinterpret_cast<const uint8_t*>(a.weight + 8 * i)), w);
#pragma unroll
        for (int j = 0; j < 8; ++j) y[j] *= w[j];
      }
      if (a.y16) {
        u32x4 o;
#pragma unroll
        for (int j = 0; j < 4; ++j) o[j] = pack16<ACT>(y[2 * j], y[2 * j + 1]);
        store_row<STREAM>(a.y16 + at, o);
      }
      if (a.y8) {
        // H is a multiple of 128 here: a row of 16 lanes is in or out as one
        float m = 0.0f;
#pragma unroll
        for (int j = 0; j < 8; ++j) m = fmaxf(m, fabsf(y[j]));
        m = row16_max(m);
        const float s = f8_scale(m);
        *reinterpret_cast<u32x2*>(a.y8 + at) = f8_codes8(y, s);
        if ((lane & 15) == 0) a.y8_scale[row * (a.H / 128) + i / 16] = s;
      }
    }
  }
}

template <int ACT, int WPR, int CH>
hipError_t launch(const NormArgs& a, hipStream_t st) {
  constexpr int kThreads = 64 * (WPR < 4 ? 4 : WPR), kRows = kThreads / (64 * WPR);
  const int64_t blocks = (static_cast<int64_t>(a.T) + kRows - 1) / kRows;
  const uint32_t grid = static_cast<uint32_t>(blocks < (1 << 20) ? blocks : (1 << 20));
  if (static_cast<int64_t>(a.T) * a.H * 2 >= kStreamBytes) k_rms_norm<ACT, WPR, CH, true><<<grid, kThreads, 0, st>>>(a);
  else k_rms_norm<ACT, WPR, CH, false><<<grid, kThreads, 0, st>>>(a);
  return hipGetLastError();
}

template <int ACT>
hipError_t launch_act(const NormArgs& a, hipStream_t st) {
  if (a.H <= 512) return launch<ACT, 1, 1>(a, st);
  if (a.H <= 1024) return launch<ACT, 1, 2>(a, st);
  if (a.H <= 2048) return launch<ACT, 4, 1>(a, st);
  if (a.H <= 4096) return launch<ACT, 8, 1>(a, st);
  if (a.H <= 8192) return launch<ACT, 8, 2>(a, st);
  return launch<ACT, 16, 4>(a, st);
}

}  // namespace

hipError_t launch_rms_norm(const NormArgs& a, hipStream_t st) {
  return a.act == PW_BF16 ? launch_act<PW_BF16>(a, st) : launch_act<PW_F16>(a, st);
}

}  // namespace pw
