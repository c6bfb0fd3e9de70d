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
#include "pw_lds.hpp"
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

// Four neighbouring columns of one row, as one store where they are all there
// and aligned.
__device__ __forceinline__ void store4(const Gemm8Args& a, int m, int n, f32x4 v) {
  const int64_t i = m * a.ldy + n;
  const uintptr_t at = reinterpret_cast<uintptr_t>(a.y) + i * (a.y_type == PW_F32 ? 4 : 2);
  const int whole = a.y_type == PW_F32 ? 15 : 7;
  if (n + 4 <= a.N && (at & whole) == 0) {
    if (a.y_type == PW_F32) *reinterpret_cast<f32x4*>(at) = v;
    else if (a.y_type == PW_BF16) *reinterpret_cast<u32x2*>(at) = u32x2{pack16<PW_BF16>(v[0], v[1]), pack16<PW_BF16>(v[2], v[3])};
    else *reinterpret_cast<u32x2*>(at) = u32x2{pack16<PW_F16>(v[0], v[1]), pack16<PW_F16>(v[2], v[3])};
    return;
  }
#pragma unroll
  for (int j = 0; j < 4; ++j)
    if (n + j < a.N) store_y(a, m, n + j, v[j]);
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
    if (m < a.M) store4(a, m, 16 * nt + 4 * lg, v);
  }
}

template <int MT>
hipError_t launch_stream(const Gemm8Args& a, hipStream_t st) {
  const int64_t grid = static_cast<int64_t>((a.N + 15) / 16) * ((a.M + 16 * MT - 1) / (16 * MT));
  if (grid > (1 << 23)) return hipErrorInvalidConfiguration;
  k_gemm8_stream<MT><<<static_cast<uint32_t>(grid), 64 * kStreamWaves, 0, st>>>(a);
  return hipGetLastError();
}

// Tiled kernel: TN weight rows x TM tokens per workgroup, WN x WM waves. K
// advances by one scale block (128) per stage; two stages lie in LDS. Global
// loads write LDS directly, 8 whole 128-byte lines per load, with the 16-byte
// pieces of a row permuted by the row index so that the operand reads meet no
// bank conflict. A wave reads the column operands (tokens) of a stage once and
// the row operands tile by tile, two ahead; the multiply-adds of a row tile run
// under the next one's matrix instructions. The barrier that publishes the next
// stage stands before the last row tile, whose operands are in registers by
// then, so that the next stage's first operands arrive under it, and loads have
// a whole stage's time to land.
template <int TN, int TM, int WN, int WM>
struct Geo8 {
  static constexpr int kWaves = WN * WM;
  static constexpr int RN = TN / WN / 16, RM = TM / WM / 16;     // a wave's 16 x 16 tiles
  static constexpr int NW = TN / 8 / kWaves, NX = TM / 8 / kWaves;   // a wave's 1 KB loads of a stage
  // weights, tokens, and 256 bytes of scales per wave: 64 tokens' each, then the
  // weight blocks', then (the same again) what no one reads
  static constexpr int kX = TN * 128, kXs = kX + TM * 128, kWs = kXs + TM * 4;
  static constexpr int kSlot = kXs + kWaves * 256;
  static_assert(TM / 64 < kWaves, "a wave for the weight scales");
  static constexpr int kLds = 2 * kSlot;
};

template <int TN, int TM, int WN, int WM>
__global__ __launch_bounds__(64 * WN * WM, 2) void k_gemm8_tiled(Gemm8Args a) {
  using G = Geo8<TN, TM, WN, WM>;
  __shared__ __attribute__((aligned(1024))) uint8_t smem[G::kLds];
  lds_u8_t lds = (lds_u8_t)smem;
  const uint32_t lds0 = __builtin_amdgcn_readfirstlane(static_cast<uint32_t>(reinterpret_cast<uintptr_t>(lds)));
  const int wave = __builtin_amdgcn_readfirstlane(static_cast<int>(threadIdx.x) >> 6), lane = lane_id();
  const int wn = wave % WN, wm = wave / WN;
  const int c = lane & 15, lg = lane >> 4;
  const int KB = a.K / 128;

  // Workgroups go to the eight XCDs in turn: each XCD gets a contiguous run of
  // tiles, walked four token tiles deep so that its L2 serves both operands.
  const int tn = (a.N + TN - 1) / TN, tm = (a.M + TM - 1) / TM, total = tn * tm;
  const int id = static_cast<int>(blockIdx.x), xcd = id & 7, q8 = total >> 3, r8 = total & 7;
  const int t = xcd * q8 + (xcd < r8 ? xcd : r8) + (id >> 3);
  constexpr int kDeep = 4;
  const int grp = t / (kDeep * tn), deep = tm - kDeep * grp < kDeep ? tm - kDeep * grp : kDeep;
  const int in = t - kDeep * grp * tn;
  const int n0 = in / deep * TN, m0 = (kDeep * grp + in % deep) * TM;

  // the wave's loads: rows 8 q .. 8 q + 7 of its share, lane l the piece (l mod
  // 8) ^ (row mod 8) of row l / 8; rows past the end repeat the last one
  const int lrow = lane >> 3, piece = (lane & 7) ^ lrow;
  uint32_t woff[G::NW], xoff[G::NX];
#pragma unroll
  for (int q = 0; q < G::NW; ++q) {
    const int r = min(n0 + (wave * G::NW + q) * 8 + lrow, a.N - 1) - n0;
    woff[q] = static_cast<uint32_t>(r) * static_cast<uint32_t>(a.ldw) + 16 * piece;
  }
#pragma unroll
  for (int q = 0; q < G::NX; ++q) {
    const int r = min(m0 + (wave * G::NX + q) * 8 + lrow, a.M - 1) - m0;
    xoff[q] = static_cast<uint32_t>(r) * static_cast<uint32_t>(a.lda) + 16 * piece;
  }
  const uint8_t* wbase = uniform_ptr(a.w + n0 * a.ldw);
  const uint8_t* xbase = uniform_ptr(a.a + m0 * a.lda);
  // scales: the first TM / 64 waves load 64 tokens' each, the others the scales
  // of the tile's weight blocks (every wave one load: a branch would cut the
  // loop's schedule in two)
  uint32_t soff;
  const uint8_t* sbase;
  if (wave < TM / 64) {
    soff = static_cast<uint32_t>(min(m0 + 64 * wave + lane, a.M - 1) - m0) * static_cast<uint32_t>(KB) * 4u;
    sbase = uniform_ptr(reinterpret_cast<const uint8_t*>(a.a_scale + static_cast<size_t>(m0) * KB));
  } else {
    soff = static_cast<uint32_t>(min(n0 / 128 + min(lane, TN / 128 - 1), (a.N - 1) / 128) - n0 / 128) * static_cast<uint32_t>(KB) * 4u;
    sbase = uniform_ptr(reinterpret_cast<const uint8_t*>(a.w_scale + static_cast<size_t>(n0 / 128) * KB));
  }
  const auto load = [&](int s, int slot) {
    const int b = s < KB ? s : KB - 1;               // past the end: the last block again, not used
    const uint32_t d = lds0 + slot * G::kSlot;
#pragma unroll
    for (int q = 0; q < G::NW; ++q) lds_load16(d + (wave * G::NW + q) * 1024, woff[q], wbase + b * 128);
#pragma unroll
    for (int q = 0; q < G::NX; ++q) lds_load16(d + G::kX + (wave * G::NX + q) * 1024, xoff[q], xbase + b * 128);
    lds_load4(d + G::kXs + wave * 256, soff, sbase + b * 4);
  };

  // operand reads: row c of a 16-row tile, pieces 2 lg and 2 lg + 1
  const uint32_t p0 = 128 * c + 16 * ((2 * lg) ^ (c & 7)), p1 = 128 * c + 16 * ((2 * lg + 1) ^ (c & 7));
  const auto read = [&](int off) { return F8Frag{lds16(lds + off + p0), lds16(lds + off + p1)}; };
  const auto read_w = [&](int slot, int i) { return read(slot * G::kSlot + (wn * G::RN + i) * 2048); };
  const auto read_x = [&](int slot, int j) { return read(slot * G::kSlot + G::kX + (wm * G::RM + j) * 2048); };
  const auto lds_f32 = [&](int off) { return *reinterpret_cast<const PW_LDS float*>(lds + off); };

  F8Frag wf[2], xf[G::RM];
  f32x4 acc[G::RN][G::RM], d[2][G::RM];
  float f[G::RM], fn[G::RM], wsn = 0.0f;
#pragma unroll
  for (int i = 0; i < G::RN; ++i)
#pragma unroll
    for (int j = 0; j < G::RM; ++j) acc[i][j] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
  for (int j = 0; j < G::RM; ++j) {
    d[1][j] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    f[j] = 0.0f;
  }
  const auto read_scales = [&](int slot) {
    wsn = lds_f32(slot * G::kSlot + G::kWs + wn * G::RN * 16 / 128 * 4);
#pragma unroll
    for (int j = 0; j < G::RM; ++j) fn[j] = lds_f32(slot * G::kSlot + G::kXs + ((wm * G::RM + j) * 16 + c) * 4);
  };
  const auto add = [&](int i, int j, int p) {
#pragma unroll
    for (int e = 0; e < 4; ++e) acc[i][j][e] = fmaf(d[p][j][e], f[j], acc[i][j][e]);
  };

  load(0, 0);
  wait_vm<0>();
  wg_barrier();
  load(1, 1);
  wf[0] = read_w(0, 0);
  wf[1] = read_w(0, 1);
#pragma unroll
  for (int j = 0; j < G::RM; ++j) xf[j] = read_x(0, j);
  read_scales(0);

  for (int s = 0; s < KB; ++s) {
    const int slot = s & 1;
#pragma unroll
    for (int i = 0; i < G::RN; ++i) {
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int j = 0; j < G::RM; ++j) {
        d[i & 1][j] = mma8(wf[i & 1], xf[j]);
        if (i == G::RN - 1) xf[j] = read_x(slot ^ 1, j);
        // the tile before this one: at i = 0 the last of the previous stage
        add(i == 0 ? G::RN - 1 : i - 1, j, (i + 1) & 1);
        __builtin_amdgcn_sched_barrier(0);
      }
      if (i == 0) {
#pragma unroll
        for (int j = 0; j < G::RM; ++j) f[j] = fn[j] * wsn;
      }
      if (i == G::RN - 2) {
        // every operand of this stage has been read; the next stage is here
        wait_lds<0>();
        wait_vm<0>();
        wg_barrier();
        load(s + 2, slot);
      }
      if (i < G::RN - 2) wf[i & 1] = read_w(slot, i + 2);
      else wf[i & 1] = read_w(slot ^ 1, i + 2 - G::RN);
      if (i == G::RN - 1) read_scales(slot ^ 1);
    }
  }
#pragma unroll
  for (int j = 0; j < G::RM; ++j) add(G::RN - 1, j, (G::RN - 1) & 1);
  wait_vm<0>();

#pragma unroll
  for (int j = 0; j < G::RM; ++j) {
    const int m = m0 + (wm * G::RM + j) * 16 + c;
    if (m >= a.M) continue;
#pragma unroll
    for (int i = 0; i < G::RN; ++i) store4(a, m, n0 + (wn * G::RN + i) * 16 + 4 * lg, acc[i][j]);
  }
}

template <int TN, int TM, int WN, int WM>
hipError_t launch_tiled(const Gemm8Args& a, hipStream_t st) {
  const int64_t grid = static_cast<int64_t>((a.N + TN - 1) / TN) * ((a.M + TM - 1) / TM);
  if (grid >= (1 << 22)) return hipErrorInvalidConfiguration;
  k_gemm8_tiled<TN, TM, WN, WM><<<static_cast<uint32_t>(grid), 64 * WN * WM, 0, st>>>(a);
  return hipGetLastError();
}

}  // namespace

size_t gemm8_workspace(int, int, int) { return 0; }

hipError_t launch_gemm8(const Gemm8Args& a, hipStream_t st) {
  if (a.M <= 16) return launch_stream<1>(a, st);
  if (a.M <= 32) return launch_stream<2>(a, st);
  if (a.M <= 64) return launch_stream<4>(a, st);
  const int64_t wide = static_cast<int64_t>((a.N + 255) / 256) * ((a.M + 255) / 256);
  return wide >= 200 ? launch_tiled<256, 256, 2, 4>(a, st) : launch_tiled<128, 128, 2, 2>(a, st);
}

}  // namespace pw
