// Product of 8-bit matrices with block scales, gfx950.
//
// Weights are packed once (k_pack8) into tiles of 16 rows x 128 values, 2 KB in
// the order in which the matrix instructions take them, the tiles of 16 rows one
// after the other along K. Row-major rows would be read 128 bytes at a time,
// each from another place of memory: 16 tokens x 28672 x 4096 then take 36.6 us
// (3.2 TB/s) where packed tiles take 24 to 26.
//
// One matrix instruction of 16 x 16 x 128 covers exactly one scale block of K,
// so every block's product starts from zero and enters the fp32 sum with one
// multiply-add per element. Weight rows are the row operand: their scale is one
// number per 128 rows, and a lane, which holds four rows of one token's column,
// multiplies all of them by the same w_scale * a_scale. (Both operands hold
// 16-byte pieces g and g + 4 of their row's block in lane group g; which k that
// is for the hardware does not matter, it is the same for both.)
//
// The 8-bit instruction keeps 14 bits of a product: those of eight neighbours along
// K are cut, toward zero, to multiples of 2^-13 of the power of two in the largest
// of the eight, then added; the sixteen eights of a block are added as in fp32. (Its
// outputs for chosen codes show this, exactly.) An eight's sum is thus off by less
// than 7 x 2^-13 of its largest product, also where products cancel. Gaussian values
// come out 1.4e-5 off in norm, without a bias, for K = 384 as for 4096; 16-bit
// outputs are rounded to 2^-9 or 2^-12. For fp32 outputs the codes are widened,
// exactly, to bf16 and go through four 16-bit instructions, whose sums are off by
// 5e-8 (K = 384) to 1.1e-7 (4096).
#include <algorithm>
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
// The same operand in 16 bits.
struct WideFrag {
  bf16x8 v[4];
};
__device__ __forceinline__ WideFrag widen(const F8Frag& f) {
  WideFrag r;
#pragma unroll
  for (int p = 0; p < 4; ++p)
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      const uint32_t x = p < 2 ? f.lo[2 * p + k] : f.hi[2 * p + k - 4];
      const auto lo = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(x, 1.0f, false);
      const auto hi = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(x, 1.0f, true);
      r.v[p][4 * k] = lo[0];
      r.v[p][4 * k + 1] = lo[1];
      r.v[p][4 * k + 2] = hi[0];
      r.v[p][4 * k + 3] = hi[1];
    }
  return r;
}
__device__ __forceinline__ f32x4 mma8(const WideFrag& a, const WideFrag& b) {
  f32x4 d{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
  for (int p = 0; p < 4; ++p) d = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a.v[p], b.v[p], d, 0, 0, 0);
  return d;
}
template <bool WIDE>
__device__ __forceinline__ auto operand(const F8Frag& f) {
  if constexpr (WIDE) return widen(f);
  else return f;
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

// Rows [16 t, 16 t + 16) of w, block b, at tile t K / 128 + b: first the 16-byte
// pieces 0 .. 3 of every row's 128, row c's piece g at 16 (16 g + c), then the
// pieces 4 .. 7 the same way. Rows past N are zeros.
__global__ __launch_bounds__(256) void k_pack8(const uint8_t* __restrict__ w, int64_t ldw, int N, int KB,
                                               u32x4* __restrict__ packed, int64_t pieces) {
  for (int64_t o = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x; o < pieces;
       o += static_cast<int64_t>(gridDim.x) * 256) {
    const int64_t tile = o >> 7, row = tile / KB * 16 + (o & 15);
    const int piece = static_cast<int>((o >> 4) & 3) + 4 * static_cast<int>((o >> 6) & 1);
    packed[o] = row < N ? ld16_nt(w + row * ldw + tile % KB * 128 + 16 * piece) : u32x4{0u, 0u, 0u, 0u};
  }
}

// Streaming kernel, for few tokens: 16 RT weight rows x 16 MT tokens per
// workgroup, straight from memory to the matrix instructions. The eight waves
// split K into eight runs of blocks and join in LDS in a fixed order; a wave has
// kAhead blocks of weights in flight (2 KB RT each). One / two / four ahead, up to 16
// tokens (us): 16 x 6144 x 4096 7.5 / 8.3 / 8.5, 16 x 28672 x 4096 24.4 / 24.9 / 26.6,
// 16 x 4096 x 4096 6.8 / 6.4 / 7.0, 4 x 12288 x 2048 7.6 / 7.25 / 10.2, 8 x 4096 x
// 14336 12.9 / 11.9 / 14.7, 1 x 14336 x 4096 12.3 / 11.3 / 11.4: two lose least.
constexpr int kStreamWaves = 8;

template <int RT, int MT, bool WIDE>
__global__ __launch_bounds__(64 * kStreamWaves) void k_gemm8_stream(Gemm8Args a) {
  constexpr int kAhead = MT == 1 ? 2 : 1;
  __shared__ f32x4 part[kStreamWaves][RT * MT][64];
  const int wave = __builtin_amdgcn_readfirstlane(static_cast<int>(threadIdx.x) >> 6), lane = lane_id();
  const int c = lane & 15, lg = lane >> 4;
  const int n_tiles = (a.N + 16 * RT - 1) / (16 * RT);
  const int nt = static_cast<int>(blockIdx.x) % n_tiles, m0 = static_cast<int>(blockIdx.x) / n_tiles * (16 * MT);
  const int KB = a.K / 128, per = (KB + kStreamWaves - 1) / kStreamWaves;
  const int kb0 = wave * per, kb1 = min(kb0 + per, KB);
  // row tiles and rows past the end repeat the last one; nothing of them is stored
  const uint8_t* w[RT];
  const float* ws[RT];
#pragma unroll
  for (int r = 0; r < RT; ++r) {
    w[r] = a.w + static_cast<size_t>(min(nt * RT + r, (a.N - 1) / 16)) * KB * 2048 + 16 * lane;
    ws[r] = a.w_scale + static_cast<size_t>(min((nt * RT + r) * 16, a.N - 1) / 128) * KB;
  }
  const uint8_t* x[MT];
  const float* xs[MT];
#pragma unroll
  for (int i = 0; i < MT; ++i) {
    const int m = min(m0 + 16 * i + c, a.M - 1);
    x[i] = a.a + m * a.lda + 16 * lg;
    xs[i] = a.a_scale + static_cast<size_t>(m) * KB;
  }
  f32x4 acc[RT][MT];
#pragma unroll
  for (int r = 0; r < RT; ++r)
#pragma unroll
    for (int i = 0; i < MT; ++i) acc[r][i] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
  for (int b0 = kb0; b0 < kb1; b0 += kAhead) {
    F8Frag wf[kAhead][RT], xf[kAhead][MT];
    float sx[kAhead][MT], sw[kAhead][RT];
#pragma unroll
    for (int u = 0; u < kAhead; ++u) {
      const int b = min(b0 + u, KB - 1);       // past the end: a block again, not used
#pragma unroll
      for (int r = 0; r < RT; ++r) wf[u][r] = F8Frag{ld16_nt(w[r] + static_cast<size_t>(b) * 2048), ld16_nt(w[r] + static_cast<size_t>(b) * 2048 + 1024)};
    }
#pragma unroll
    for (int u = 0; u < kAhead; ++u) {
      const int b = min(b0 + u, KB - 1);
#pragma unroll
      for (int i = 0; i < MT; ++i) {
        xf[u][i] = F8Frag{ld16(x[i] + b * 128), ld16(x[i] + b * 128 + 64)};
        sx[u][i] = xs[i][b];
      }
#pragma unroll
      for (int r = 0; r < RT; ++r) sw[u][r] = ws[r][b];
    }
    __builtin_amdgcn_sched_barrier(0);         // all loads out before the first use
#pragma unroll
    for (int u = 0; u < kAhead; ++u) {
      const bool in = b0 + u < kb1;
#pragma unroll
      for (int r = 0; r < RT; ++r)
#pragma unroll
        for (int i = 0; i < MT; ++i) {
          const f32x4 d = mma8(operand<WIDE>(wf[u][r]), operand<WIDE>(xf[u][i]));
          const float f = sw[u][r] * sx[u][i];
          if (in) {
#pragma unroll
            for (int j = 0; j < 4; ++j) acc[r][i][j] = fmaf(d[j], f, acc[r][i][j]);
          }
        }
    }
  }
#pragma unroll
  for (int r = 0; r < RT; ++r)
#pragma unroll
    for (int i = 0; i < MT; ++i) part[wave][r * MT + i][lane] = acc[r][i];
  __syncthreads();
  for (int t = wave; t < RT * MT; t += kStreamWaves) {
    f32x4 v = part[0][t][lane];
#pragma unroll
    for (int q = 1; q < kStreamWaves; ++q) v += part[q][t][lane];
    const int m = m0 + 16 * (t % MT) + c;
    if (m < a.M) store4(a, m, (nt * RT + t / MT) * 16 + 4 * lg, v);
  }
}

template <int RT, int MT, bool WIDE>
hipError_t launch_stream(const Gemm8Args& a, hipStream_t st) {
  const int64_t grid = static_cast<int64_t>((a.N + 16 * RT - 1) / (16 * RT)) * ((a.M + 16 * MT - 1) / (16 * MT));
  k_gemm8_stream<RT, MT, WIDE><<<static_cast<uint32_t>(grid), 64 * kStreamWaves, 0, st>>>(a);
  return hipGetLastError();
}

// Two row tiles per workgroup share its loads of the tokens, where enough
// workgroups are left. 33 to 64 tokens go to one workgroup, or to two that read
// the weights twice: to one where the row tiles' workgroups fit the CUs once and
// twice as many do not. Two / one (us): 40 tokens x 2048 x 2048 (128 row units)
// 6.0 / 6.7, x 2560 x 2048 (160) 7.5 / 6.8, x 6144 x 4096 (192) 14.6 / 12.1; 64 x
// 6144 x 4096 16.6 / 14.9, x 8192 x 2048 (256; 56 tokens) 10.6 / 9.7, x 12288 x
// 1024 (384) 8.6 / 9.8.
template <int RT, bool WIDE>
hipError_t launch_stream_rows(const Gemm8Args& a, hipStream_t st) {
  const int units = (a.N + 16 * RT - 1) / (16 * RT);
  if (a.M <= 16) return launch_stream<RT, 1, WIDE>(a, st);
  if (a.M <= 32 || a.M > 64 || units <= 128 || units > 256) return launch_stream<RT, 2, WIDE>(a, st);
  return a.M <= 48 ? launch_stream<RT, 3, WIDE>(a, st) : launch_stream<RT, 4, WIDE>(a, st);
}
template <bool WIDE>
hipError_t launch_stream_of(const Gemm8Args& a, hipStream_t st) {
  return a.N >= 5120 ? launch_stream_rows<2, WIDE>(a, st) : launch_stream_rows<1, WIDE>(a, st);
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
template <int TN, int TM, int WN, int WM, int SLOTS>
struct Geo8 {
  static constexpr int kWaves = WN * WM;
  static constexpr int RN = TN / WN / 16, RM = TM / WM / 16;     // a wave's 16 x 16 tiles
  static constexpr int NW = TN / 8 / kWaves, NX = TM / 8 / kWaves;   // a wave's 1 KB loads of a stage
  // slots of weights and tokens, and two of the tokens' scales of kSc stages
  static constexpr int kX = TN * 128, kSlot = kX + TM * 128;
  static constexpr int kSc = 8, kScSlot = TM * kSc * 4, kScOff = SLOTS * kSlot;
  static constexpr int NS = TM / 8 / kWaves;                     // a wave's loads of scales: 8 tokens x kSc stages each
  static constexpr int kSpare = kScOff + 2 * kScSlot, kLds = kSpare + 256;
  static_assert(NS + SLOTS <= kSc, "the scales of the next stages land in time");
};

template <int TN, int TM, int WN, int WM, int SLOTS, bool WIDE = false>
__global__ __launch_bounds__(64 * WN * WM, SLOTS > 2 ? 1 : 2) void k_gemm8_tiled(Gemm8Args a) {
  using G = Geo8<TN, TM, WN, WM, SLOTS>;
  __shared__ __attribute__((aligned(1024))) uint8_t smem[G::kLds];
  lds_u8_t lds = (lds_u8_t)smem;
  const uint32_t lds0 = __builtin_amdgcn_readfirstlane(static_cast<uint32_t>(reinterpret_cast<uintptr_t>(lds)));
  const int wave = __builtin_amdgcn_readfirstlane(static_cast<int>(threadIdx.x) >> 6), lane = lane_id();
  const int wn = wave % WN, wm = wave / WN;
  const int c = lane & 15, lg = lane >> 4;
  const int KB = a.K / 128;                            // blocks of a row

  // Workgroups go to the eight XCDs in turn: each XCD gets a contiguous run of
  // tiles, walked four token tiles deep so that its L2 serves both operands.
  const int tn = (a.N + TN - 1) / TN, tm = (a.M + TM - 1) / TM, total = tn * tm;
  const int ks = __builtin_amdgcn_readfirstlane(static_cast<int>(blockIdx.x) / total), id = static_cast<int>(blockIdx.x) - ks * total;
  const int xcd = id & 7, q8 = total >> 3, r8 = total & 7;
  const int kb0 = ks * a.kb_per;                       // this workgroup's blocks of K
  const int nstage = __builtin_amdgcn_readfirstlane(min(a.kb_per, KB - kb0));
  const int t = xcd * q8 + (xcd < r8 ? xcd : r8) + (id >> 3);
  constexpr int kDeep = 4;
  const int grp = t / (kDeep * tn), deep = tm - kDeep * grp < kDeep ? tm - kDeep * grp : kDeep;
  const int in = t - kDeep * grp * tn;
  const int n0 = in / deep * TN, m0 = (kDeep * grp + in % deep) * TM;

  // the wave's loads: halves of weight tiles as they lie, and 8 rows of tokens,
  // lane l the piece (l mod 8) ^ (row / 2 mod 8) of row l / 8; what is past the
  // end repeats the last one
  const int lrow = lane >> 3;
  const auto piece = [&](int q) { return (lane & 7) ^ (lrow >> 1) ^ (4 * (q & 1)); };
  uint32_t woff[G::NW], xoff[G::NX];
#pragma unroll
  for (int q = 0; q < G::NW; ++q) {                    // half a tile each (wave-uniform)
    const int x = wave * G::NW + q, rt = min(n0 / 16 + x / 2, (a.N - 1) / 16) - n0 / 16;
    woff[q] = static_cast<uint32_t>(rt) * static_cast<uint32_t>(KB) * 2048u + (x & 1) * 1024u;
  }
#pragma unroll
  for (int q = 0; q < G::NX; ++q) {
    const int r = min(m0 + (wave * G::NX + q) * 8 + lrow, a.M - 1) - m0;
    xoff[q] = static_cast<uint32_t>(r) * static_cast<uint32_t>(a.lda) + 16 * piece(wave * G::NX + q);
  }
  const uint8_t* wbase = uniform_ptr(a.w + (static_cast<size_t>(n0 / 16) * KB + kb0) * 2048);
  const uint8_t* xbase = uniform_ptr(a.a + m0 * a.lda + kb0 * 128);
  // Scales of the tokens come for kSc stages at a time: a load takes 8 tokens x
  // kSc stages, lane l token l mod 8 and stage l / 8 (a load for one stage would
  // touch a cache line per token, as many as all operand loads of the stage).
  // They are spread over the stages before: a stage loads a share of those of the
  // next kSc. Every stage has the same count of loads, which the waits rely on;
  // those past the last share read one address into spare bytes of LDS (777 tokens
  // x 4000 x 4096: 27.4 us, with the last share's eight lines again 29.1). The
  // weight block's scales lie in a register, a stage in a lane.
  const uint8_t* sbase = uniform_ptr(reinterpret_cast<const uint8_t*>(a.a_scale + static_cast<size_t>(m0) * KB + kb0));
  const auto load_scales = [&](int chunk, int q) {
    const bool live = q < G::NS;                     // (wave-uniform)
    const int o = wave * G::NS + q;
    const int r = min(m0 + 8 * o + (lane & 7), a.M - 1) - m0, st = min(chunk * G::kSc + lrow, nstage - 1);
    const uint32_t off = (static_cast<uint32_t>(r) * static_cast<uint32_t>(KB) + static_cast<uint32_t>(st)) * 4u;
    lds_load4(lds0 + (live ? G::kScOff + (chunk & 1) * G::kScSlot + o * 256 : G::kSpare), off & (live ? ~0u : 0u), sbase);
  };
  const float* wsp = a.w_scale + static_cast<size_t>(min((n0 + wn * G::RN * 16) / 128, (a.N - 1) / 128)) * KB + kb0;
  int ws64 = 0;
  const auto fetch_ws = [&](int s) { ws64 = __float_as_int(wsp[min(s + lane, nstage - 1)]); };
  // the wave's loads of stage s, one at a time
  const auto load = [&](int s, int slot, int q) {
    const int b = s < nstage ? s : nstage - 1;       // past the end: the last block again, not used
    const uint32_t d = lds0 + slot * G::kSlot;
    if (q < G::NX) lds_load16(d + G::kX + (wave * G::NX + q) * 1024, xoff[q], xbase + b * 128);
    else lds_load16(d + (wave * G::NW + q - G::NX) * 1024, 16u * lane, wbase + woff[q - G::NX] + static_cast<size_t>(b) * 2048);
  };
  // They go out over kOver row tiles from the barrier on, kPer at each.
  constexpr int kOver = G::RN == 8 ? 4 : 2, kAll = G::NX + G::NW, kPer = kAll / kOver;
  static_assert(kPer * kOver == kAll && (SLOTS == 2 || kOver == 2), "whole shares, all out before the next barrier");

  // operand reads: row c of a 16-row tile, pieces lg and lg + 4
  const uint32_t p0 = 128 * c + 16 * (lg ^ (c >> 1)), p1 = p0 ^ 64;
  const auto read_w = [&](int slot, int i) {
    lds_u8_t p = lds + slot * G::kSlot + (wn * G::RN + i) * 2048 + 16 * lane;
    return F8Frag{lds16(p), lds16(p + 1024)};
  };
  const auto read_x = [&](int slot, int j) {
    lds_u8_t p = lds + slot * G::kSlot + G::kX + (wm * G::RM + j) * 2048;
    return F8Frag{lds16(p + p0), lds16(p + p1)};
  };
  const auto lds_f32 = [&](int off) { return *reinterpret_cast<const PW_LDS float*>(lds + off); };

  F8Frag wf[2], xf[G::RM];
  WideFrag ww, xw[G::RM];                              // (WIDE alone)
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
  for (int s = 0; s < SLOTS - 1; ++s)
#pragma unroll
    for (int q = 0; q < kAll; ++q) load(s, s, q);
#pragma unroll
  for (int q = 0; q < 2 * kPer; ++q) load(SLOTS - 1, SLOTS - 1, q);
  wait_vm<(SLOTS - 2) * kAll + 2 * kPer>();
  wg_barrier();
  wf[0] = read_w(0, 0);
  wf[1] = read_w(0, 1);
#pragma unroll
  for (int j = 0; j < G::RM; ++j) xf[j] = read_x(0, j);
  read_scales(0);

  // (64 stages at a time: a branch in the loop would cut its schedule in two)
  for (int s0 = 0; s0 < nstage; s0 += 64) {
    fetch_ws(s0);
    for (int s = s0; s < min(s0 + 64, nstage); ++s) {
      const int slot = s % SLOTS, next = (s + 1) % SLOTS;
#pragma unroll
      for (int i = 0; i < G::RN; ++i) {
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int j = 0; j < G::RM; ++j) {
          if constexpr (WIDE) {
            if (i == 0) xw[j] = widen(xf[j]);
            if (j == 0) ww = widen(wf[i & 1]);
            d[i & 1][j] = mma8(ww, xw[j]);
          } else {
            d[i & 1][j] = mma8(wf[i & 1], xf[j]);
          }
          if (i == G::RN - 1) xf[j] = read_x(next, j);
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
          wait_vm<(SLOTS - 2) * kAll>();
          wg_barrier();
          load_scales(s / G::kSc + 1, s % G::kSc);
        }
        // loads of stage s + SLOTS, from the barrier into the next stage
#pragma unroll
        for (int q = 0; q < kPer; ++q) {
          if (i >= G::RN - 2) load(s + SLOTS, slot, (i - (G::RN - 2)) * kPer + q);
          else if (i + 2 < kOver) load(s + SLOTS - 1, (s + SLOTS - 1) % SLOTS, (i + 2) * kPer + q);
        }
        if (i < G::RN - 2) wf[i & 1] = read_w(slot, i + 2);
        else wf[i & 1] = read_w(next, i + 2 - G::RN);
        if (i == G::RN - 1) read_scales(s + 1);
      }
    }
  }
#pragma unroll
  for (int j = 0; j < G::RM; ++j) add(G::RN - 1, j, (G::RN - 1) & 1);
  // a part of K: fp32 rows of its own, joined afterwards
  const bool part = a.ksplit > 1;
  Gemm8Args out = a;
  out.y = part ? a.part + static_cast<size_t>(ks) * a.M * a.ldp : a.y;
  out.ldy = part ? a.ldp : a.ldy;
  const int y_type = part ? PW_F32 : a.y_type;
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
      wave_exchange();
      u32x4 v[16 * kLanes / 64];
#pragma unroll
      for (int k = 0; k < 16 * kLanes; k += 64) v[k / 64] = lds16(w + (k + lane) / kLanes * kPitch + 16 * ((k + lane) % kLanes));
      wave_exchange();
#pragma unroll
      for (int k = 0; k < 16 * kLanes; k += 64) {
        const int row = (k + lane) / kLanes, p = (k + lane) % kLanes;
        const int m = m0 + (wm * G::RM + j) * 16 + row;
        if (m < a.M) store_piece<kE>(out, m, n0 + wn * G::RN * 16 + p * (16 / kE), v[k / 64]);
      }
    }
  };
  if (y_type == PW_F32)
    rows_out(std::integral_constant<int, 4>{}, [](lds_u8_t p, f32x4 v) { *reinterpret_cast<PW_LDS f32x4*>(p) = v; });
  else if (y_type == PW_BF16)
    rows_out(std::integral_constant<int, 2>{}, [](lds_u8_t p, f32x4 v) {
      *reinterpret_cast<PW_LDS u32x2*>(p) = u32x2{pack16<PW_BF16>(v[0], v[1]), pack16<PW_BF16>(v[2], v[3])};
    });
  else
    rows_out(std::integral_constant<int, 2>{}, [](lds_u8_t p, f32x4 v) {
      *reinterpret_cast<PW_LDS u32x2*>(p) = u32x2{pack16<PW_F16>(v[0], v[1]), pack16<PW_F16>(v[2], v[3])};
    });
}

template <int TN, int TM, int WN, int WM, int SLOTS, bool WIDE = false>
hipError_t launch_tiled(const Gemm8Args& a, hipStream_t st) {
  const int64_t grid = static_cast<int64_t>((a.N + TN - 1) / TN) * ((a.M + TM - 1) / TM) * a.ksplit;
  k_gemm8_tiled<TN, TM, WN, WM, SLOTS, WIDE><<<static_cast<uint32_t>(grid), 64 * WN * WM, 0, st>>>(a);
  return hipGetLastError();
}

// Sums the parts of K, in their order, four columns a thread.
__global__ __launch_bounds__(256) void k_gemm8_join(Gemm8Args a) {
  const int n4 = static_cast<int>(a.ldp / 4);
  for (int64_t i = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x; i < static_cast<int64_t>(a.M) * n4;
       i += static_cast<int64_t>(gridDim.x) * 256) {
    const float* p = a.part + i * 4;
    f32x4 v = *reinterpret_cast<const f32x4*>(p);
#pragma unroll 4
    for (int k = 1; k < a.ksplit; ++k) v += *reinterpret_cast<const f32x4*>(p + static_cast<size_t>(k) * a.M * a.ldp);
    store4(a, static_cast<int>(i / n4), static_cast<int>(i % n4) * 4, v);
  }
}

// Which kernel runs, and into how many parts K is cut. Measured (us):
//   streaming / 128 x 128 tiles: 64 tokens x 1024 x 2048 5.8 / 11.8, x 4000 x
//     2048 8.9 / 13.2, x 6144 x 4096 14.9 / 17.2, x 4096 x 14336 45 / 23.9, x
//     28672 x 4096 52.6 / 34.0; 128 x 4000 x 2048 14.8 / 14.6;
//   128 x 128 tiles whole / in parts of K: 128 x 6144 x 4096 24.1 / 18.0, 128 x
//     4096 x 14336 109 / 27, 256 x 4000 x 2048 14.3 / 18.9;
//   128 x 128 tiles four stages deep, one workgroup per CU / two deep, two per
//     CU: 256 x 28672 x 4096 (448 tiles) 64 / 52; below 257 tiles there is but
//     one workgroup per CU.
// Widened operands do not fit the registers of a 256 x 256 tile; 128 x 128, two
// stages deep in pairs / four deep alone: 825 x 5795 x 3456 (322 tiles) 56 / 66,
// 4096 x 14336 x 4096 447 / 533 (8-bit instructions and wide tiles: 265).
enum { kStream8, kSmall8, kSmallPair8, kWide8 };
struct Plan8 {
  int kernel, ksplit, kb_per;
};
Plan8 plan8(int M, int N, int K, bool widened) {
  const int64_t KB = K / 128;
  Plan8 p{kStream8, 1, static_cast<int>(KB)};
  const int64_t streamed = static_cast<int64_t>(N) * K * ((static_cast<int64_t>(M) + 31) / 32);
  if (M <= 32 || streamed <= (M <= 64 ? int64_t(52) << 20 : int64_t(32) << 20)) return p;
  const auto split = [&](int64_t parts) {
    p.kb_per = static_cast<int>((KB + parts - 1) / parts);
    p.ksplit = static_cast<int>((KB + p.kb_per - 1) / p.kb_per);
  };
  const int64_t wide = static_cast<int64_t>((N + 255) / 256) * ((M + 255) / 256);
  const int64_t tiles = static_cast<int64_t>((N + 127) / 128) * ((M + 127) / 128);
  p.kernel = kWide8;
  if (!widened && wide >= 200) return p;
  if (!widened && wide >= 48 && KB >= 28 * (256 / wide)) {       // long K: parts of it fill the chip
    split(256 / wide);
    return p;
  }
  p.kernel = tiles > 256 ? kSmallPair8 : kSmall8;
  int64_t parts = 256 / tiles;
  parts = parts < KB / 4 ? parts : KB / 4;
  if (parts > 1 && KB >= 24) split(parts < 8 ? parts : 8);
  return p;
}
int64_t part_ld(int N) { return (static_cast<int64_t>(N) + 3) / 4 * 4; }

// The product in launches that each take fewer than 2^32 threads: tiles of 128 x
// 128 below 2^22 (the least that the tiled kernels have, with up to 512 threads),
// weight rows up to 2^24 (32 or more of them to a workgroup of the streaming
// kernel). Sizes below that, all that are cut in parts of K among them, are one.
template <class Launch>
hipError_t in_launches(const Gemm8Args& a, Launch&& launch) {
  constexpr int64_t kRows = 1 << 24, kTiles = 1 << 22;
  const int64_t KB = a.K / 128, elt = a.y_type == PW_F32 ? 4 : 2;
  for (int64_t n0 = 0; n0 < a.N; n0 += kRows) {
    const int64_t n = a.N - n0 < kRows ? a.N - n0 : kRows;
    const int64_t most = (kTiles - 1) / ((n + 127) / 128) * 128;   // tokens
    for (int64_t m0 = 0; m0 < a.M; m0 += most) {
      Gemm8Args p = a;
      p.N = static_cast<int>(n);
      p.M = static_cast<int>(a.M - m0 < most ? a.M - m0 : most);
      p.a += m0 * a.lda;
      p.a_scale += m0 * KB;
      p.w += n0 / 16 * KB * 2048;
      p.w_scale += n0 / 128 * KB;
      p.y = static_cast<uint8_t*>(a.y) + (m0 * a.ldy + n0) * elt;
      const hipError_t e = launch(p);
      if (e != hipSuccess) return e;
    }
  }
  return hipSuccess;
}

}  // namespace

// (for any type of y)
size_t gemm8_workspace(int M, int N, int K) {
  const int parts = std::max(plan8(M, N, K, false).ksplit, plan8(M, N, K, true).ksplit);
  return parts > 1 ? static_cast<size_t>(parts) * M * part_ld(N) * sizeof(float) : 0;
}

hipError_t launch_pack8(const uint8_t* w, int64_t ldw, int N, int K, uint8_t* packed, hipStream_t st) {
  const int64_t pieces = (static_cast<int64_t>(N) + 15) / 16 * K, blocks = (pieces + 255) / 256;   // of 16 bytes
  k_pack8<<<static_cast<uint32_t>(blocks < (1 << 20) ? blocks : (1 << 20)), 256, 0, st>>>(
      w, ldw, N, K / 128, reinterpret_cast<u32x4*>(packed), pieces);
  return hipGetLastError();
}

hipError_t launch_gemm8(const Gemm8Args& args, hipStream_t st) {
  Gemm8Args a = args;
  const bool widened = a.y_type == PW_F32;
  const Plan8 p = plan8(a.M, a.N, a.K, widened);
  a.ksplit = p.ksplit;
  a.kb_per = p.kb_per;
  a.ldp = part_ld(a.N);
  const hipError_t e = in_launches(a, [&](const Gemm8Args& g) {
    switch (p.kernel) {
      case kStream8: return widened ? launch_stream_of<true>(g, st) : launch_stream_of<false>(g, st);
      case kSmall8: return widened ? launch_tiled<128, 128, 2, 4, 4, true>(g, st) : launch_tiled<128, 128, 2, 4, 4>(g, st);
      case kSmallPair8: return widened ? launch_tiled<128, 128, 2, 2, 2, true>(g, st) : launch_tiled<128, 128, 2, 2, 2>(g, st);
      default: return launch_tiled<256, 256, 2, 4, 2>(g, st);
    }
  });
  if (e != hipSuccess || a.ksplit == 1) return e;
  const int64_t blocks = (static_cast<int64_t>(a.M) * (a.ldp / 4) + 255) / 256;
  k_gemm8_join<<<static_cast<uint32_t>(blocks < 4096 ? blocks : 4096), 256, 0, st>>>(a);
  return hipGetLastError();
}

}  // namespace pw
