// Group-limited routing, gfx950: scores, groups, top-k and weights of one token
// per wave (k_route_grouped), then the expert-major permutation
// (k_permute_parts). (Both in one workgroup, for small batches, took longer
// than two launches from 9 tokens on.)
//
// The definition holds scores in 64 bits, so that the choice does not hang on
// how an exponential or a sum is rounded. Computing them so for every expert
// is the long way (16.7 us for 4096 tokens x 256 experts in 8 groups), and
// nearly never needed: the token is routed with 32-bit scores, and every
// decision is checked against a bound of their error. Experts too close to the
// last one taken, or to each other, are compared again in 64 bits, which the
// weights of those taken need anyway; where groups are too close the wave goes
// over the token again in 64 bits. So it takes 11.9 us, bound by the vector and
// lane-exchange instructions of the choice (4.2 MB of logits are read in 1), and
// the permutation of the 32768 slots 7.9; 33 tokens x 60 experts 5.7 and 3.1,
// both mostly latency.
#include "pw_device.hpp"
#include "pw_internal.hpp"
#include "pw_ops.hpp"

namespace pw {
namespace {

constexpr int kPerLane = 4;              // experts of a lane, neighbours: E <= 256
constexpr int kRouteWaves = 4;
constexpr int kMaxE = 64 * kPerLane;

// A double as an unsigned number of the same order (-0 as +0). 0 stands for
// "not eligible" and lies below every number.
__device__ __forceinline__ uint64_t order_key(double v) {
  uint64_t u = __builtin_bit_cast(uint64_t, v);
  if (u == 0x8000000000000000ull) u = 0;
  return (u >> 63) ? ~u : (u | 0x8000000000000000ull);
}
__device__ __forceinline__ double key_value(uint64_t k) {
  return __builtin_bit_cast(double, (k >> 63) ? (k & 0x7FFFFFFFFFFFFFFFull) : ~k);
}
// The same for floats as signed numbers (-0 below +0: told apart, the two are
// too close for the error bound and go to 64 bits).
__device__ __forceinline__ int order32(float v) {
  const int i = __float_as_int(v);
  return i ^ ((i >> 31) & 0x7FFFFFFF);
}
__device__ __forceinline__ float value32(int k) { return __int_as_float(k ^ ((k >> 31) & 0x7FFFFFFF)); }
constexpr int kNone32 = static_cast<int>(0x807FFFFFu);            // order32(-infinity)

__device__ __forceinline__ uint64_t max_u64(uint64_t a, uint64_t b) { return a > b ? a : b; }
__device__ __forceinline__ int max_i32(int a, int b) { return a > b ? a : b; }

template <int CTRL>
__device__ __forceinline__ int dpp_i32(int x) {
  return __builtin_amdgcn_update_dpp(0, x, CTRL, 0xF, 0xF, false);
}
template <int CTRL>
__device__ __forceinline__ uint64_t dpp_u64(uint64_t x) {
  const uint32_t lo = static_cast<uint32_t>(dpp_i32<CTRL>(static_cast<int>(static_cast<uint32_t>(x))));
  const uint32_t hi = static_cast<uint32_t>(dpp_i32<CTRL>(static_cast<int>(static_cast<uint32_t>(x >> 32))));
  return (static_cast<uint64_t>(hi) << 32) | lo;
}
__device__ __forceinline__ uint64_t lane_u64(uint64_t x, int l) {
  const uint32_t lo = __builtin_amdgcn_readlane(static_cast<uint32_t>(x), l);
  const uint32_t hi = __builtin_amdgcn_readlane(static_cast<uint32_t>(x >> 32), l);
  return (static_cast<uint64_t>(hi) << 32) | lo;
}
constexpr int kPairs = 0xB1, kQuads = 0x4E, kHalfMirror = 0x141, kMirror = 0x140;   // lane exchanges in a row of 16

// Largest value of the wave, in scalar registers.
__device__ __forceinline__ uint64_t wave_max(uint64_t k) {
  k = max_u64(k, dpp_u64<kPairs>(k));
  k = max_u64(k, dpp_u64<kQuads>(k));
  k = max_u64(k, dpp_u64<kHalfMirror>(k));
  k = max_u64(k, dpp_u64<kMirror>(k));
  return max_u64(max_u64(lane_u64(k, 0), lane_u64(k, 16)), max_u64(lane_u64(k, 32), lane_u64(k, 48)));
}
__device__ __forceinline__ int wave_max(int k) {
  k = max_i32(k, dpp_i32<kPairs>(k));
  k = max_i32(k, dpp_i32<kQuads>(k));
  k = max_i32(k, dpp_i32<kHalfMirror>(k));
  k = max_i32(k, dpp_i32<kMirror>(k));
  return max_i32(max_i32(__builtin_amdgcn_readlane(k, 0), __builtin_amdgcn_readlane(k, 16)),
                 max_i32(__builtin_amdgcn_readlane(k, 32), __builtin_amdgcn_readlane(k, 48)));
}
template <int CTRL>
__device__ __forceinline__ double dpp_f64(double x) {
  return __builtin_bit_cast(double, dpp_u64<CTRL>(__builtin_bit_cast(uint64_t, x)));
}
// Sum over the lane's row of 16 lanes, and over the wave.
__device__ __forceinline__ double row16_sum(double v) {
  v += dpp_f64<kPairs>(v);
  v += dpp_f64<kQuads>(v);
  v += dpp_f64<kHalfMirror>(v);
  return v + dpp_f64<kMirror>(v);
}
__device__ __forceinline__ double wave_sum(double v) {
  const uint64_t u = __builtin_bit_cast(uint64_t, row16_sum(v));
  return (__builtin_bit_cast(double, lane_u64(u, 0)) + __builtin_bit_cast(double, lane_u64(u, 16))) +
         (__builtin_bit_cast(double, lane_u64(u, 32)) + __builtin_bit_cast(double, lane_u64(u, 48)));
}
__device__ __forceinline__ float wave_sum(float v) {
  v += dpp_f32<kPairs>(v);
  v += dpp_f32<kQuads>(v);
  v += dpp_f32<kHalfMirror>(v);
  v += dpp_f32<kMirror>(v);
  const int i = __float_as_int(v);
  return (__int_as_float(__builtin_amdgcn_readlane(i, 0)) + __int_as_float(__builtin_amdgcn_readlane(i, 16))) +
         (__int_as_float(__builtin_amdgcn_readlane(i, 32)) + __int_as_float(__builtin_amdgcn_readlane(i, 48)));
}

template <int LT>
__device__ __forceinline__ float logit(const void* p, size_t i) {
  float x;
  if constexpr (LT == PW_F32) x = static_cast<const float*>(p)[i];
  else x = val16(static_cast<const uint16_t*>(p)[i], LT);
  return x > 3.0e38f ? 3.0e38f : x;                  // (NaN stays)
}

// What a wave knows of its token: lane l holds experts 4 l .. 4 l + 3.
struct Token {
  float x[kPerLane];       // logits; -infinity past E
  float b[kPerLane];       // bias
  float m;                 // largest eligible logit of the wave (softmax)
};
// The experts taken, one in each of the first K lanes; n > K: n that contain
// them, not in order.
struct Taken {
  int id;
  bool eligible;
  int n;
};

// Keeps the top groups: bit j of the result for group j. gk: the score of group
// `lane`, as a number that orders like it (unsigned or signed), 0 or kNone32
// where the group has no eligible expert; rank among all groups, ties to the
// lower one. `last`, `next`: the scores on both sides of the cut.
template <class T>
__device__ __forceinline__ uint64_t keep_groups(T gk, int n_groups, int top_groups, int lane, T* last, T* next) {
  int rank = 0;
  for (int j = 0; j < n_groups; ++j) {
    T o;
    if constexpr (sizeof(T) == 8) o = lane_u64(gk, j);
    else o = __builtin_amdgcn_readlane(gk, j);
    rank += (o > gk || (o == gk && j < lane)) ? 1 : 0;
  }
  const bool live = lane < n_groups;
  const auto at = [&](int r) {
    const int l = __ffsll(static_cast<long long>(__ballot(live && rank == r))) - 1;
    if constexpr (sizeof(T) == 8) return lane_u64(gk, l);
    else return __builtin_amdgcn_readlane(gk, l);
  };
  *last = at(top_groups - 1);
  *next = at(top_groups);
  return __ballot(live && rank < top_groups);
}

// The choice with 32-bit scores: the K experts, or (n > K, or n = K and *sure
// false) a few that contain them. False where this cannot be told.
//
// Error of a score (u = 2^-24; exponentials and reciprocals here are good to
// two units): sigmoid, below 4 u whatever the logit; softmax, p (2.2 d + 30) u
// with d = m - x (the exponent's two roundings and its constant's; the sum's
// terms have d below 6 on the average), below 2^-17 p up to d = 44, where p is
// below 2^-63 and b0 covers it; one more rounding, |c| u, with the bias.
// A decision between scores v1 > v2 holds if they differ by more than f (b0 +
// |v1| + |v2|): sigmoid f = 8 u, b0 = 1; softmax f = 2^-17, b0 = twice the
// largest bias (p <= |c| + |b|) + 2^-33. Sums of two get twice that, with the
// bias in b0, since their terms may cancel.
__device__ __forceinline__ bool choose32(const RouteArgs& a, const Token& tk, int lane, float* lds, Taken* out, bool* sure) {
  const int gsize = a.E / a.n_groups;
  const bool softmax = a.score == PW_SCORE_SOFTMAX;
  float p[kPerLane], bmax = 0.0f;
  if (softmax) {
    float sum = 0.0f;
#pragma unroll
    for (int q = 0; q < kPerLane; ++q) {
      p[q] = tk.x[q] > -INFINITY ? __builtin_amdgcn_exp2f((tk.x[q] - tk.m) * 1.44269504f) : 0.0f;
      sum += p[q];
    }
    const float inv = __builtin_amdgcn_rcpf(wave_sum(sum));
#pragma unroll
    for (int q = 0; q < kPerLane; ++q) p[q] *= inv;
  } else {
#pragma unroll
    for (int q = 0; q < kPerLane; ++q) p[q] = __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(tk.x[q] * -1.44269504f));
  }
  float c[kPerLane];
#pragma unroll
  for (int q = 0; q < kPerLane; ++q) {
    c[q] = p[q] + tk.b[q];
    if (!(tk.x[q] > -INFINITY) || !(c[q] > -INFINITY)) c[q] = -INFINITY;
    // the largest bias of an eligible expert
    if (c[q] > -INFINITY) bmax = fmaxf(bmax, fabsf(tk.b[q]));
  }
  if (a.bias) bmax = value32(wave_max(order32(bmax)));
  const float f = softmax ? 0x1p-17f : 0x1p-21f, b0 = softmax ? 2.0f * bmax + 0x1p-33f : 1.0f;
  const auto apart = [&](float v1, float v2, float scale, float b) { return v1 - v2 > scale * (b + fabsf(v1) + (v2 > -INFINITY ? fabsf(v2) : 0.0f)); };
  if (a.top_groups < a.n_groups) {
    float g1, g2;                        // the two largest scores of group `lane`
    const int L = gsize / kPerLane;      // lanes of a group
    if (gsize % kPerLane == 0 && L <= 16 && (L & (L - 1)) == 0) {
      const auto merge = [&](float o1, float o2) {
        g2 = fmaxf(fminf(g1, o1), fmaxf(g2, o2));
        g1 = fmaxf(g1, o1);
      };
      g1 = fmaxf(c[0], c[1]);
      g2 = fminf(c[0], c[1]);
      merge(fmaxf(c[2], c[3]), fminf(c[2], c[3]));
      // (groups whole: the exchanges pair off lanes of one group)
      if (L > 1) merge(dpp_f32<kPairs>(g1), dpp_f32<kPairs>(g2));
      if (L > 2) merge(dpp_f32<kQuads>(g1), dpp_f32<kQuads>(g2));
      if (L > 4) merge(dpp_f32<kHalfMirror>(g1), dpp_f32<kHalfMirror>(g2));
      if (L > 8) merge(dpp_f32<kMirror>(g1), dpp_f32<kMirror>(g2));
      const float h1 = __shfl(g1, (lane * L) & 63), h2 = __shfl(g2, (lane * L) & 63);
      g1 = lane < a.n_groups ? h1 : -INFINITY;
      g2 = h2;
    } else {
      *reinterpret_cast<f32x4*>(lds + 4 * lane) = f32x4{c[0], c[1], c[2], c[3]};
      wave_exchange();
      g1 = g2 = -INFINITY;
      if (lane < a.n_groups) {
        for (int i = 0; i < gsize; ++i) {
          const float v = lds[lane * gsize + i];
          g2 = fmaxf(g2, fminf(g1, v));
          g1 = fmaxf(g1, v);
        }
      }
    }
    const float score = a.group_top == 2 && g2 > -INFINITY ? g1 + g2 : g1;
    int last, next;
    const uint64_t kept = keep_groups<int>(order32(score), a.n_groups, a.top_groups, lane, &last, &next);
    if (next == kNone32 ? last == kNone32 : !apart(value32(last), value32(next), 2.0f * f, b0 + 2.0f * bmax)) return false;
#pragma unroll
    for (int q = 0; q < kPerLane; ++q) {
      const int e = kPerLane * lane + q;
      if (!((kept >> (e / gsize & 63)) & 1ull)) c[q] = -INFINITY;
    }
  }
  int key[kPerLane];
#pragma unroll
  for (int q = 0; q < kPerLane; ++q) key[q] = order32(c[q]);
  float before = INFINITY, edge = 0.0f;              // the score before, and the K-th
  *sure = true;
  int k = 0;
  for (;; ++k) {
    const int mine = max_i32(max_i32(key[0], key[1]), max_i32(key[2], key[3]));
    const int best = wave_max(mine);
    const float v = value32(best);
    if (k >= a.K && (best == kNone32 || apart(edge, v, f, b0))) break;
    if (best == kNone32 || k == 64) return false;     // fewer eligible experts than K, or many alike
    *sure = *sure && k < a.K && (k == 0 || apart(before, v, f, b0));
    before = v;
    if (k == a.K - 1) edge = v;
    const int l = __ffsll(static_cast<long long>(__ballot(mine == best))) - 1;
    const int q = key[0] == mine ? 0 : key[1] == mine ? 1 : key[2] == mine ? 2 : 3;
    const int id = __builtin_amdgcn_readlane(kPerLane * lane + q, l);
    if (lane == k) out->id = id;
#pragma unroll
    for (int j = 0; j < kPerLane; ++j)
      if (kPerLane * lane + j == id) key[j] = kNone32;
  }
  out->eligible = true;
  out->n = k;
  return true;
}

// Eligible experts' p in 64 bits: sigmoid(x), or exp(x - m), the softmax's
// numerator.
__device__ __forceinline__ double score64(const RouteArgs& a, float x, float m) {
  // (no branch around the exponential: several of them then run side by side)
  const bool in = x > -INFINITY;
  const double d = in ? static_cast<double>(x) : 0.0;
  const double e = exp(a.score == PW_SCORE_SIGMOID ? -d : d - static_cast<double>(m));
  return !in ? 0.0 : a.score == PW_SCORE_SIGMOID ? 1.0 / (1.0 + e) : e;
}

// The choice by the definition.
__device__ __forceinline__ void choose64(const RouteArgs& a, const Token& tk, int lane, uint64_t* lds, Taken* out) {
  const int E = a.E, gsize = E / a.n_groups;
  double p[kPerLane], sum = 0.0;
#pragma unroll
  for (int q = 0; q < kPerLane; ++q) {
    p[q] = score64(a, tk.x[q], tk.m);
    sum += p[q];
  }
  if (a.score == PW_SCORE_SOFTMAX) {
    sum = wave_sum(sum);
  #pragma unroll
  for (int q = 0; q < kPerLane; ++q) p[q] = sum > 0.0 ? p[q] / sum : 0.0;
  }
  uint64_t key[kPerLane];
  wave_exchange();                       // (choose32 read there)
#pragma unroll
  for (int q = 0; q < kPerLane; ++q) {
    const double c = p[q] + static_cast<double>(tk.b[q]);
    key[q] = tk.x[q] > -INFINITY && c > -__builtin_huge_val() ? order_key(c) : 0ull;
    lds[kPerLane * lane + q] = key[q];
  }
  wave_exchange();
  if (a.top_groups < a.n_groups) {
    uint64_t gk = 0;
    if (lane < a.n_groups) {
      uint64_t k1 = 0, k2 = 0;
      for (int i = 0; i < gsize; ++i) {
        const uint64_t k = lds[lane * gsize + i];
        k2 = max_u64(k2, k < k1 ? k : k1);
        k1 = max_u64(k1, k);
      }
      if (k1) gk = order_key(a.group_top == 2 && k2 ? key_value(k1) + key_value(k2) : key_value(k1));
    }
    uint64_t last, next;
    const uint64_t kept = keep_groups<uint64_t>(gk, a.n_groups, a.top_groups, lane, &last, &next);
  #pragma unroll
  for (int q = 0; q < kPerLane; ++q)
      if (!((kept >> ((kPerLane * lane + q) / gsize & 63)) & 1ull)) key[q] = 0ull;
  }
  uint32_t free4 = 0;                    // the lane's experts not taken yet
#pragma unroll
  for (int q = 0; q < kPerLane; ++q) free4 |= kPerLane * lane + q < E ? 1u << q : 0u;
  for (int k = 0; k < a.K; ++k) {
    uint64_t mine = 0;
  #pragma unroll
  for (int q = 0; q < kPerLane; ++q) mine = max_u64(mine, (free4 >> q) & 1u ? key[q] : 0ull);
    const uint64_t best = wave_max(mine);
    int q = kPerLane;                    // the lane's first free expert with that key
#pragma unroll
    for (int j = kPerLane - 1; j >= 0; --j)
      if (((free4 >> j) & 1u) && key[j] == best) q = j;
    const int l = __ffsll(static_cast<long long>(__ballot(q < kPerLane))) - 1;
    const int id = __builtin_amdgcn_readlane(kPerLane * lane + q, l);
    if (lane == k) {
      out->id = id;
      out->eligible = best != 0;
    }
    if (lane == l) free4 &= ~(1u << q);
  }
}

template <int LT>
__device__ __forceinline__ void route_token(const RouteArgs& a, int t, uint64_t* lds) {
  const int lane = lane_id(), E = a.E;
  const size_t at = static_cast<size_t>(t) * E;
  Token tk;
#pragma unroll
  for (int q = 0; q < kPerLane; ++q) {
    const int e = kPerLane * lane + q;
    tk.x[q] = e < E ? logit<LT>(a.logits, at + e) : -INFINITY;
    tk.b[q] = a.bias && e < E ? a.bias[e] : 0.0f;
  }
  tk.m = 0.0f;
  if (a.score == PW_SCORE_SOFTMAX) {
    int m = kNone32;                     // (of numbers only: NaN does not count)
#pragma unroll
    for (int q = 0; q < kPerLane; ++q) m = max_i32(m, tk.x[q] > -INFINITY ? order32(tk.x[q]) : kNone32);
    tk.m = value32(wave_max(m));
  }
  Taken got{0, false, a.K};
  bool sure = true;
  if (__builtin_expect(!choose32(a, tk, lane, reinterpret_cast<float*>(lds), &got, &sure), 0)) {
    choose64(a, tk, lane, lds, &got);
    got.n = a.K;
    sure = true;
  }
  const auto softmax_sum = [&] {
    double sum = 0.0;
#pragma unroll
    for (int q = 0; q < kPerLane; ++q) sum += score64(a, tk.x[q], tk.m);
    return wave_sum(sum);
  };
  // lane k's expert: its logit and p (the softmax's numerator)
  const auto of_mine = [&](const float* v) {
    float r = 0.0f;
#pragma unroll
    for (int q = 0; q < kPerLane; ++q) {
      const float o = __shfl(v[q], got.id / kPerLane);
      r = got.id % kPerLane == q ? o : r;
    }
    return r;
  };
  const float x = of_mine(tk.x);
  double p = score64(a, lane < got.n && got.eligible ? x : -INFINITY, tk.m);
  if (__builtin_expect(!sure, 0)) {
    // the scores that 32 bits do not tell apart, in 64 bits
    double c = p;
    if (a.bias) c = (a.score == PW_SCORE_SOFTMAX ? p / softmax_sum() : p) + static_cast<double>(of_mine(tk.b));
    const uint64_t key = order_key(c);
    int rank = 0;
    for (int j = 0; j < got.n; ++j) {
      const uint64_t o = lane_u64(key, j);
      rank += (o > key || (o == key && __builtin_amdgcn_readlane(got.id, j) < got.id)) ? 1 : 0;
    }
    const int to = 4 * (lane < got.n ? rank : lane);
    got.id = __builtin_amdgcn_ds_permute(to, got.id);
    const uint64_t u = __builtin_bit_cast(uint64_t, p);
    const uint32_t lo = static_cast<uint32_t>(__builtin_amdgcn_ds_permute(to, static_cast<int>(static_cast<uint32_t>(u))));
    const uint32_t hi = static_cast<uint32_t>(__builtin_amdgcn_ds_permute(to, static_cast<int>(static_cast<uint32_t>(u >> 32))));
    p = __builtin_bit_cast(double, (static_cast<uint64_t>(hi) << 32) | lo);
  }
  const bool mine = lane < a.K;
  if (!mine) p = 0.0;
  if (a.renorm || a.score == PW_SCORE_SOFTMAX) {
    const double sum = a.renorm ? row16_sum(p) : softmax_sum();      // K <= 16
    p = sum > 0.0 ? p / sum : 0.0;
  }
  const size_t row = static_cast<size_t>(t) * (a.K + a.n_shared);
  if (mine) {
    a.ids[row + lane] = got.id;
    a.w[row + lane] = static_cast<float>(p * static_cast<double>(a.w_scale));
  }
  for (int j = lane; j < a.n_shared; j += 64) {
    a.ids[row + a.K + j] = E + j;
    a.w[row + a.K + j] = a.gate ? a.gate[static_cast<size_t>(t) * a.n_shared + j] : 1.0f;
  }
}

template <int LT>
__global__ __launch_bounds__(64 * kRouteWaves) void k_route_grouped(RouteArgs a) {
  __shared__ __attribute__((aligned(16))) uint64_t keys[kRouteWaves][kMaxE];
  const int wave = static_cast<int>(threadIdx.x) >> 6;
  const int t = static_cast<int>(blockIdx.x) * kRouteWaves + wave;
  if (t >= a.T) return;                  // wave-uniform; no barrier follows
  route_token<LT>(a, t, keys[wave]);
}

// Permutation of the slots [s0, s1) by one workgroup of kPermWaves waves. It
// counts every expert's slots before and from s0 on (order-free LDS atomics), so
// that its experts' starts are known without a second launch, then places its
// slots in rounds of 64 per wave: a slot's rank among the wave's slots of its
// expert comes from comparing the wave's 64 ids one by one, the rounds' and
// waves' counts give the start. Nothing depends on timing. Slot numbers are
// unsigned where they may pass the last slot, which may be 2^31 - 2. Against one workgroup
// per expert, each going over all slots (the plain router's permutation): 7.7
// us in place of 9.2 for 24576 slots of 64 experts, 8.1 for 10.8 at 32768 of 256,
// equal near 16384, and 1 us slower below. The LDS atomics bound it.
constexpr int kPermWaves = 16;
constexpr int kPermRound = 64 * kPermWaves;
struct PermLds {
  int count[2 * kMaxE];                  // slots before s0, slots from s0 on
  int start[kMaxE];
  int cnt[kPermWaves][kMaxE];
  int wave_sum[kMaxE / 64];
};
__device__ __forceinline__ void permute_part(const int32_t* ids, int S, int E, int s0, int s1, PermLds& m, int32_t* offsets,
                                             int32_t* sorted_slot, int32_t* slot_pos) {
  const int tid = threadIdx.x, wave = tid >> 6, lane = lane_id();
  if (tid < 2 * kMaxE) m.count[tid] = 0;
  __syncthreads();
  const auto add = [&](uint32_t s, int id) { atomicAdd(&m.count[id + (s < static_cast<uint32_t>(s0) ? 0 : kMaxE)], 1); };
  // four ids to a load, eight loads in flight per thread (the ids come from
  // another kernel, so from beyond the L2: a round of loads is about 1 us)
  const int head = static_cast<int>(-(reinterpret_cast<uintptr_t>(ids) / 4) & 3), n4 = S > head ? (S - head) / 4 : 0;
  const int4* v = reinterpret_cast<const int4*>(ids + head);
  for (int base = tid; base < n4; base += 8 * kPermRound) {
    int4 id[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) id[j] = base + j * kPermRound < n4 ? v[base + j * kPermRound] : int4{-1, 0, 0, 0};
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const uint32_t s = head + 4u * (base + j * kPermRound);
      if (id[j].x >= 0) {
        add(s, id[j].x);
        add(s + 1, id[j].y);
        add(s + 2, id[j].z);
        add(s + 3, id[j].w);
      }
    }
  }
  if (tid < 8) {                         // what the quads leave at either end
    const uint32_t s = tid < 4 ? tid : head + 4u * n4 + (tid - 4);
    if ((tid >= 4 || tid < head) && s < static_cast<uint32_t>(S)) add(s, ids[s]);
  }
  __syncthreads();
  // exclusive sums over the experts
  int total = 0, sum = 0;
  if (tid < kMaxE) {
    total = m.count[tid] + m.count[kMaxE + tid];
    sum = total;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
      const int x = __shfl_up(sum, o);
      if (lane >= o) sum += x;
    }
    if (lane == 63) m.wave_sum[wave] = sum;
  }
  __syncthreads();
  if (tid < kMaxE) {
    for (int w = 0; w < wave; ++w) sum += m.wave_sum[w];
    m.start[tid] = sum - total + m.count[tid];
    if (s0 == 0) {
      if (tid < E) offsets[tid] = sum - total;
      if (tid == E - 1) offsets[E] = sum;
    }
  }
  for (uint32_t base = s0; base < static_cast<uint32_t>(s1); base += kPermRound) {
    for (int i = tid; i < kPermWaves * kMaxE; i += kPermRound) m.cnt[i / kMaxE][i % kMaxE] = 0;
    __syncthreads();
    const uint32_t s = base + 64 * wave + lane;
    const int id = s < static_cast<uint32_t>(s1) ? ids[s] : -1;
    int rank = 0, n = 0;
    if (base + 64 * wave < static_cast<uint32_t>(s1)) {
      // (short code: a workgroup runs it a few times, mostly from a cold
      // instruction cache)
#pragma unroll 8
      for (int j = 0; j < 64; ++j) {
        const bool same = id == __builtin_amdgcn_readlane(id, j);
        n += same;
        rank += same && lane > j;
      }
      if (id >= 0) m.cnt[wave][id] = n;            // (the same number from every slot of the expert)
    }
    __syncthreads();
    if (tid < kMaxE) {
      int at = m.start[tid];
#pragma unroll
      for (int w = 0; w < kPermWaves; ++w) {
        const int c = m.cnt[w][tid];
        m.cnt[w][tid] = at;
        at += c;
      }
      m.start[tid] = at;
    }
    __syncthreads();
    if (id >= 0) {
      const int pos = m.cnt[wave][id] + rank;
      sorted_slot[pos] = static_cast<int32_t>(s);
      slot_pos[s] = pos;
    }
    __syncthreads();
  }
}

__global__ __launch_bounds__(kPermRound) void k_permute_parts(const int32_t* __restrict__ ids, int S, int E, int part,
                                                              int32_t* __restrict__ offsets,
                                                              int32_t* __restrict__ sorted_slot,
                                                              int32_t* __restrict__ slot_pos) {
  __shared__ PermLds m;
  const int s0 = static_cast<int>(blockIdx.x) * part;
  permute_part(ids, S, E, s0, S - s0 < part ? S : s0 + part, m, offsets, sorted_slot, slot_pos);
}

constexpr int64_t kManySlots = 16384;    // where the two permutations take the same time
constexpr int kLaunchTokens = 1 << 25;   // of one launch, which takes fewer than 2^32 threads

template <int LT>
hipError_t launch_route(const RouteArgs& a, hipStream_t st) {
  const int64_t S = static_cast<int64_t>(a.T) * (a.K + a.n_shared);
  hipError_t e = hipSuccess;
  for (int64_t t0 = 0; t0 < a.T; t0 += kLaunchTokens) {
    RouteArgs p = a;
    p.T = static_cast<int>(a.T - t0 < kLaunchTokens ? a.T - t0 : kLaunchTokens);
    p.logits = static_cast<const uint8_t*>(a.logits) + t0 * a.E * (LT == PW_F32 ? 4 : 2);
    p.ids += t0 * (a.K + a.n_shared);
    p.w += t0 * (a.K + a.n_shared);
    if (a.gate) p.gate += t0 * a.n_shared;
    k_route_grouped<LT><<<static_cast<uint32_t>((p.T + kRouteWaves - 1) / kRouteWaves), 64 * kRouteWaves, 0, st>>>(p);
    e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  if (S < kManySlots)
    return launch_permute(a.ids, a.T, a.K + a.n_shared, a.E + a.n_shared, a.offsets, a.sorted_slot, a.slot_pos, st);
  // every part goes over all slots once: 512 slots to a part, and 256 parts at most
  int64_t part = (S + 255) / 256;
  part = part < 512 ? 512 : (part + 63) / 64 * 64;
  const int64_t parts = (S + part - 1) / part;
  k_permute_parts<<<static_cast<uint32_t>(parts), kPermRound, 0, st>>>(
      a.ids, static_cast<int>(S), a.E + a.n_shared, static_cast<int>(part), a.offsets, a.sorted_slot, a.slot_pos);
  return hipGetLastError();
}

}  // namespace

// (T = 0 writes the offsets alone)
hipError_t launch_route_grouped(const RouteArgs& a, hipStream_t st) {
  if (a.logit_type == PW_F32) return launch_route<PW_F32>(a, st);
  return a.logit_type == PW_BF16 ? launch_route<PW_BF16>(a, st) : launch_route<PW_F16>(a, st);
}

}  // namespace pw
