// Product of 8-bit matrices with block scales, gfx950.
//
// One matrix instruction of 16 x 16 x 128 covers exactly one scale block of K,
// so every block's product starts from zero and enters the fp32 sum with one
// multiply-add per element. Weight rows are the row operand: their scale is one
// number per 128 rows, and a lane, which holds four rows of one token's column,
// multiplies all of them by the same w_scale * a_scale. (Both operands hold
// bytes 32 g .. 32 g + 31 of their row's block in lane group g; which k that is
// for the hardware does not matter, it is the same for both.)
#include <type_traits>

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

// 16 bytes of one row's columns from n on, as one store where they are all there
// and aligned.
template <int E>
__device__ __forceinline__ void store_piece(const Gemm8Args& a, int m, int n, u32x4 v) {
  const uintptr_t at = reinterpret_cast<uintptr_t>(a.y) + (m * a.ldy + n) * E;
  if (n + 16 / E <= a.N && (at & 15) == 0) {
    __builtin_nontemporal_store(v, reinterpret_cast<u32x4*>(at));
    return;
  }
#pragma unroll
  for (int j = 0; j < 16 / E; ++j) {
    if (n + j >= a.N) break;
    if constexpr (E == 4) reinterpret_cast<uint32_t*>(at)[j] = v[j];
    else reinterpret_cast<uint16_t*>(at)[j] = static_cast<uint16_t>(v[j / 2] >> (16 * (j & 1)));
  }
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
// pieces of a row permuted by half the row index: the 16 rows that a quarter of
// an operand read takes then lie in 16 different sixteenths of the 64 banks
// (permuted by the row index itself, rows r and r + 8 share theirs and reads
// take twice the cycles). A wave reads the column operands (tokens) of a stage once and
// the row operands tile by tile, two ahead; the multiply-adds of a row tile run
// under the next one's matrix instructions. The barrier that publishes the next
// stage stands before the last row tile, whose operands are in registers by
// then, so that the next stage's first operands arrive under it. The loads of a
// stage go out over several row tiles: all at once they queue up in the address
// unit and hold the wave back.
template <int TN, int TM, int WN, int WM>
struct Geo8 {
  static constexpr int kWaves = WN * WM;
  static constexpr int RN = TN / WN / 16, RM = TM / WM / 16;     // a wave's 16 x 16 tiles
  static constexpr int NW = TN / 8 / kWaves, NX = TM / 8 / kWaves;   // a wave's 1 KB loads of a stage
  // two slots of weights and tokens, two of the tokens' scales of kSc stages
  static constexpr int kX = TN * 128, kSlot = kX + TM * 128;
  static constexpr int kSc = 8, kScSlot = TM * kSc * 4, kScOff = 2 * kSlot;
  static constexpr int NS = TM / 8 / kWaves;                     // a wave's loads of scales: 8 tokens x kSc stages each
  static constexpr int kLds = kScOff + 2 * kScSlot;
  static_assert(NS <= kSc && kSc % NS == 0, "the scales of the next stages are loaded over kSc stages");
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
  // 8) ^ (row / 2 mod 8) of row l / 8; rows past the end repeat the last one
  const int lrow = lane >> 3;
  const auto piece = [&](int q) { return (lane & 7) ^ (lrow >> 1) ^ (4 * (q & 1)); };
  uint32_t woff[G::NW], xoff[G::NX];
#pragma unroll
  for (int q = 0; q < G::NW; ++q) {
    const int r = min(n0 + (wave * G::NW + q) * 8 + lrow, a.N - 1) - n0;
    woff[q] = static_cast<uint32_t>(r) * static_cast<uint32_t>(a.ldw) + 16 * piece(wave * G::NW + q);
  }
#pragma unroll
  for (int q = 0; q < G::NX; ++q) {
    const int r = min(m0 + (wave * G::NX + q) * 8 + lrow, a.M - 1) - m0;
    xoff[q] = static_cast<uint32_t>(r) * static_cast<uint32_t>(a.lda) + 16 * piece(wave * G::NX + q);
  }
  const uint8_t* wbase = uniform_ptr(a.w + n0 * a.ldw);
  const uint8_t* xbase = uniform_ptr(a.a + m0 * a.lda);
  // Scales of the tokens come for kSc stages at a time: a load takes 8 tokens x
  // kSc stages, lane l token l mod 8 and stage l / 8 (a load for one stage would
  // touch a cache line per token, as many as all operand loads of the stage).
  // They are spread over the stages before: stage s loads a share of those of
  // the next kSc (each share more than once, so that every stage has the same
  // count of loads). The weight block's scales lie in a register, a stage in a
  // lane.
  const uint8_t* sbase = uniform_ptr(reinterpret_cast<const uint8_t*>(a.a_scale + static_cast<size_t>(m0) * KB));
  const auto load_scales = [&](int chunk, int q) {
    const int o = wave * G::NS + q;
    const int r = min(m0 + 8 * o + (lane & 7), a.M - 1) - m0, st = min(chunk * G::kSc + lrow, KB - 1);
    lds_load4(lds0 + G::kScOff + (chunk & 1) * G::kScSlot + o * 256,
              (static_cast<uint32_t>(r) * static_cast<uint32_t>(KB) + static_cast<uint32_t>(st)) * 4u, sbase);
  };
  const float* wsp = a.w_scale + static_cast<size_t>(min((n0 + wn * G::RN * 16) / 128, (a.N - 1) / 128)) * KB;
  int ws64 = 0;
  const auto fetch_ws = [&](int s) { ws64 = __float_as_int(wsp[min(s + lane, KB - 1)]); };
  // the wave's loads of stage s, one at a time
  const auto load = [&](int s, int slot, int q) {
    const int b = s < KB ? s : KB - 1;               // past the end: the last block again, not used
    const uint32_t d = lds0 + slot * G::kSlot;
    if (q < G::NX) lds_load16(d + G::kX + (wave * G::NX + q) * 1024, xoff[q], xbase + b * 128);
    else lds_load16(d + (wave * G::NW + q - G::NX) * 1024, woff[q - G::NX], wbase + b * 128);
  };
  // They go out over kOver row tiles from the barrier on, kPer at each.
  constexpr int kOver = G::RN == 8 ? 4 : 2, kPer = (G::NX + G::NW) / kOver;
  static_assert(kPer * kOver == G::NX + G::NW, "whole shares");

  // operand reads: row c of a 16-row tile, pieces lg and lg + 4
  const uint32_t p0 = 128 * c + 16 * (lg ^ (c >> 1)), p1 = p0 ^ 64;
  const auto read = [&](int off) { return F8Frag{lds16(lds + off + p0), lds16(lds + off + p1)}; };
  const auto read_w = [&](int slot, int i) { return read(slot * G::kSlot + (wn * G::RN + i) * 2048); };
  const auto read_x = [&](int slot, int j) { return read(slot * G::kSlot + G::kX + (wm * G::RM + j) * 2048); };
  const auto lds_f32 = [&](int off) { return *reinterpret_cast<const PW_LDS float*>(lds + off); };

  F8Frag wf[2], xf[G::RM];
  f32x4 acc[G::RN][G::RM], d[2][G::RM];
  float f[G::RM], fn[G::RM];
#pragma unroll
  for (int i = 0; i < G::RN; ++i)
#pragma unroll
    for (int j = 0; j < G::RM; ++j) acc[i][j] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
  for (int j = 0; j < G::RM; ++j) {
    d[1][j] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    f[j] = 0.0f;
  }
  const auto read_scales = [&](int s) {
    const int off = G::kScOff + (s / G::kSc & 1) * G::kScSlot + s % G::kSc * 32;
#pragma unroll
    for (int j = 0; j < G::RM; ++j)
      fn[j] = lds_f32(off + ((wm * G::RM + j) * 2 + (c >> 3)) * 256 + (c & 7) * 4);
  };
  const auto add = [&](int i, int j, int p) {
#pragma unroll
    for (int e = 0; e < 4; ++e) acc[i][j][e] = fmaf(d[p][j][e], f[j], acc[i][j][e]);
  };

#pragma unroll
  for (int q = 0; q < G::NS; ++q) load_scales(0, q);
#pragma unroll
  for (int q = 0; q < 8; ++q) load(0, 0, q);
#pragma unroll
  for (int q = 0; q < 2 * kPer; ++q) load(1, 1, q);
  wait_vm<2 * kPer>();
  wg_barrier();
  wf[0] = read_w(0, 0);
  wf[1] = read_w(0, 1);
#pragma unroll
  for (int j = 0; j < G::RM; ++j) xf[j] = read_x(0, j);
  read_scales(0);

  // (64 stages at a time: a branch in the loop would cut its schedule in two)
  for (int s0 = 0; s0 < KB; s0 += 64) {
  fetch_ws(s0);
  for (int s = s0; s < min(s0 + 64, KB); ++s) {
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
        const float ws = __int_as_float(__builtin_amdgcn_readlane(ws64, s & 63));
#pragma unroll
        for (int j = 0; j < G::RM; ++j) f[j] = fn[j] * ws;
      }
      if (i == G::RN - 2) {
        // every operand of this stage has been read; the next stage is here
        wait_lds<0>();
        wait_vm<0>();
        wg_barrier();
        load_scales((s + 1) / G::kSc + 1, (s + 1) % G::kSc / (G::kSc / G::NS));
      }
      // loads of the stage after next, from the barrier into the next stage
#pragma unroll
      for (int q = 0; q < kPer; ++q) {
        if (i >= G::RN - 2) load(s + 2, slot, (i - (G::RN - 2)) * kPer + q);
        else if (i + 2 < kOver) load(s + 1, slot ^ 1, (i + 2) * kPer + q);
      }
      if (i < G::RN - 2) wf[i & 1] = read_w(slot, i + 2);
      else wf[i & 1] = read_w(slot ^ 1, i + 2 - G::RN);
      if (i == G::RN - 1) read_scales(s + 1);
    }
  }
  }
#pragma unroll
  for (int j = 0; j < G::RM; ++j) add(G::RN - 1, j, (G::RN - 1) & 1);
  // Through LDS (the wave's own part of it) to rows: a store then covers whole
  // cache lines of a few tokens in place of 32 bytes of each of 16.
  wait_vm<0>();
  wg_barrier();
  const auto rows_out = [&](auto esz_tag, auto&& put) {
    constexpr int kE = decltype(esz_tag)::value;          // bytes of an element
    constexpr int kRow = G::RN * 16 * kE, kPitch = kRow + 16, kLanes = kRow / 16;
    static_assert(16 * kPitch <= G::kLds / G::kWaves, "a wave's part of LDS");
    lds_u8_t w = lds + wave * (G::kLds / G::kWaves / 16 * 16);
#pragma unroll
    for (int j = 0; j < G::RM; ++j) {
#pragma unroll
      for (int i = 0; i < G::RN; ++i) put(w + c * kPitch + (i * 16 + 4 * lg) * kE, acc[i][j]);
#pragma unroll
      for (int k = 0; k < 16 * kLanes; k += 64) {
        const int row = (k + lane) / kLanes, p = (k + lane) % kLanes;
        const u32x4 v = lds16(w + row * kPitch + 16 * p);
        const int m = m0 + (wm * G::RM + j) * 16 + row;
        if (m < a.M) store_piece<kE>(a, m, n0 + wn * G::RN * 16 + p * (16 / kE), v);
      }
    }
  };
  if (a.y_type == PW_F32)
    rows_out(std::integral_constant<int, 4>{}, [](lds_u8_t p, f32x4 v) { *reinterpret_cast<PW_LDS f32x4*>(p) = v; });
  else if (a.y_type == PW_BF16)
    rows_out(std::integral_constant<int, 2>{}, [](lds_u8_t p, f32x4 v) {
      *reinterpret_cast<PW_LDS u32x2*>(p) = u32x2{pack16<PW_BF16>(v[0], v[1]), pack16<PW_BF16>(v[2], v[3])};
    });
  else
    rows_out(std::integral_constant<int, 2>{}, [](lds_u8_t p, f32x4 v) {
      *reinterpret_cast<PW_LDS u32x2*>(p) = u32x2{pack16<PW_F16>(v[0], v[1]), pack16<PW_F16>(v[2], v[3])};
    });
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
