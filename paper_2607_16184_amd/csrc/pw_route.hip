// Group-limited routing, gfx950: scores, groups, top-k and weights of one token
// per wave. The permutation that follows is that of the plain router.
#include "pw_device.hpp"
#include "pw_ops.hpp"

namespace pw {
namespace {

constexpr int kPerLane = 4;              // experts of a lane: E <= 256
constexpr int kMaxTopK = 16;
constexpr int kRouteWaves = 4;

// A double as an unsigned number of the same order (-0 as +0). The choice is
// made on these 64 bits, so that it does not hang on how an exponential or a
// sum is rounded. 0 stands for "not eligible" and lies below every number.
__device__ __forceinline__ uint64_t order_key(double v) {
  uint64_t u = __builtin_bit_cast(uint64_t, v);
  if (u == 0x8000000000000000ull) u = 0;
  return (u >> 63) ? ~u : (u | 0x8000000000000000ull);
}
__device__ __forceinline__ double key_value(uint64_t k) {
  return __builtin_bit_cast(double, (k >> 63) ? (k & 0x7FFFFFFFFFFFFFFFull) : ~k);
}

__device__ __forceinline__ uint64_t max_u64(uint64_t a, uint64_t b) { return a > b ? a : b; }

template <int CTRL>
__device__ __forceinline__ uint64_t dpp_u64(uint64_t x) {
  const uint32_t lo = static_cast<uint32_t>(
      __builtin_amdgcn_update_dpp(0, static_cast<int>(static_cast<uint32_t>(x)), CTRL, 0xF, 0xF, false));
  const uint32_t hi = static_cast<uint32_t>(
      __builtin_amdgcn_update_dpp(0, static_cast<int>(static_cast<uint32_t>(x >> 32)), CTRL, 0xF, 0xF, false));
  return (static_cast<uint64_t>(hi) << 32) | lo;
}
__device__ __forceinline__ uint64_t lane_u64(uint64_t x, int l) {
  const uint32_t lo = __builtin_amdgcn_readlane(static_cast<uint32_t>(x), l);
  const uint32_t hi = __builtin_amdgcn_readlane(static_cast<uint32_t>(x >> 32), l);
  return (static_cast<uint64_t>(hi) << 32) | lo;
}
// Largest value of the wave, in scalar registers.
__device__ __forceinline__ uint64_t wave_max(uint64_t k) {
  k = max_u64(k, dpp_u64<0xB1>(k));
  k = max_u64(k, dpp_u64<0x4E>(k));
  k = max_u64(k, dpp_u64<0x141>(k));
  k = max_u64(k, dpp_u64<0x140>(k));
  return max_u64(max_u64(lane_u64(k, 0), lane_u64(k, 16)), max_u64(lane_u64(k, 32), lane_u64(k, 48)));
}
__device__ __forceinline__ double wave_sum(double v) {
#pragma unroll
  for (int o = 32; o; o >>= 1) v += __shfl_xor(v, o);
  return v;
}

template <int LT>
__device__ __forceinline__ float logit(const void* p, size_t i) {
  if constexpr (LT == PW_F32) return static_cast<const float*>(p)[i];
  else return val16(static_cast<const uint16_t*>(p)[i], LT);
}

template <int LT>
__global__ __launch_bounds__(64 * kRouteWaves) void k_route_grouped(RouteArgs a) {
  __shared__ uint64_t keys[kRouteWaves][64 * kPerLane];
  const int wave = static_cast<int>(threadIdx.x) >> 6, lane = lane_id();
  const int t = static_cast<int>(blockIdx.x) * kRouteWaves + wave;
  if (t >= a.T) return;                  // wave-uniform; no barrier follows
  const int E = a.E, gsize = E / a.n_groups;
  // lane l holds experts l, l + 64, ...
  double p[kPerLane];
  uint64_t key[kPerLane];
  float x[kPerLane];
#pragma unroll
  for (int q = 0; q < kPerLane; ++q) {
    const int e = lane + 64 * q;
    x[q] = e < E ? logit<LT>(a.logits, static_cast<size_t>(t) * E + e) : -INFINITY;
    x[q] = x[q] > 3.0e38f ? 3.0e38f : x[q];          // (NaN stays)
  }
  if (a.score == PW_SCORE_SIGMOID) {
#pragma unroll
    for (int q = 0; q < kPerLane; ++q) p[q] = x[q] > -INFINITY ? 1.0 / (1.0 + exp(-static_cast<double>(x[q]))) : 0.0;
  } else {
    float m = -INFINITY;
#pragma unroll
    for (int q = 0; q < kPerLane; ++q) m = fmaxf(m, x[q]);
#pragma unroll
    for (int o = 32; o; o >>= 1) m = fmaxf(m, __shfl_xor(m, o));
    double sum = 0.0;                    // (without an eligible expert no term is formed)
#pragma unroll
    for (int q = 0; q < kPerLane; ++q) {
      p[q] = x[q] > -INFINITY ? exp(static_cast<double>(x[q]) - static_cast<double>(m)) : 0.0;
      sum += p[q];
    }
    sum = wave_sum(sum);
#pragma unroll
    for (int q = 0; q < kPerLane; ++q) p[q] = sum > 0.0 ? p[q] / sum : 0.0;
  }
#pragma unroll
  for (int q = 0; q < kPerLane; ++q) {
    const int e = lane + 64 * q;
    const double c = a.bias && e < E ? p[q] + static_cast<double>(a.bias[e]) : p[q];
    key[q] = x[q] > -INFINITY && c > -__builtin_huge_val() ? order_key(c) : 0ull;
  }
  if (a.top_groups < a.n_groups) {
    // lane j < n_groups scores group j from the wave's keys in LDS
#pragma unroll
    for (int q = 0; q < kPerLane; ++q) keys[wave][lane + 64 * q] = key[q];
    __builtin_amdgcn_wave_barrier();
    uint64_t gk = 0;
    if (lane < a.n_groups) {
      uint64_t k1 = 0, k2 = 0;
      for (int i = 0; i < gsize; ++i) {
        const uint64_t k = keys[wave][lane * gsize + i];
        k2 = max_u64(k2, k < k1 ? k : k1);
        k1 = max_u64(k1, k);
      }
      if (k1) gk = order_key(a.group_top == 2 && k2 ? key_value(k1) + key_value(k2) : key_value(k1));
    }
    uint64_t kept = 0;                   // bit j: group j is kept
    for (int n = 0; n < a.top_groups; ++n) {
      const uint64_t free_groups = (a.n_groups == 64 ? ~0ull : (1ull << a.n_groups) - 1ull) & ~kept;
      const uint64_t best = wave_max((free_groups >> lane) & 1ull ? gk : 0ull);
      kept |= 1ull << (__ffsll(static_cast<long long>(__ballot(gk == best) & free_groups)) - 1);
    }
#pragma unroll
    for (int q = 0; q < kPerLane; ++q) {
      const int e = lane + 64 * q;
      if (e < E && !((kept >> (e / gsize)) & 1ull)) key[q] = 0ull;
    }
  }
  // K rounds: the largest key, the lowest expert that has it
  uint64_t taken[kPerLane] = {};
  int se[kMaxTopK];
  double sw[kMaxTopK], sum = 0.0;
#pragma unroll
  for (int k = 0; k < kMaxTopK; ++k) {
    if (k < a.K) {
      uint64_t mine = key[0];
#pragma unroll
      for (int q = 1; q < kPerLane; ++q) mine = max_u64(mine, key[q]);
      const uint64_t best = wave_max(mine);
      int be = -1;
      double bw = 0.0;
#pragma unroll
      for (int q = 0; q < kPerLane; ++q) {
        const int n = E - 64 * q;
        const uint64_t in = n >= 64 ? ~0ull : n > 0 ? (1ull << n) - 1ull : 0ull;
        const uint64_t hit = __ballot(key[q] == best) & in & ~taken[q];
        if (be < 0 && hit) {
          const int l = __ffsll(static_cast<long long>(hit)) - 1;
          be = l + 64 * q;
          taken[q] |= 1ull << l;
          bw = best ? __builtin_bit_cast(double, lane_u64(__builtin_bit_cast(uint64_t, p[q]), l)) : 0.0;
          if (lane == l) key[q] = 0ull;
        }
      }
      se[k] = be;
      sw[k] = bw;
      sum += bw;
    }
  }
  if (lane != 0) return;
  const int Kt = a.K + a.n_shared;
  const size_t row = static_cast<size_t>(t) * Kt;
  const double f = a.renorm ? (sum > 0.0 ? 1.0 / sum : 0.0) : 1.0;
#pragma unroll
  for (int k = 0; k < kMaxTopK; ++k) {
    if (k < a.K) {
      a.ids[row + k] = se[k];
      a.w[row + k] = static_cast<float>(sw[k] * f * static_cast<double>(a.w_scale));
    }
  }
  for (int j = 0; j < a.n_shared; ++j) {
    a.ids[row + a.K + j] = E + j;
    a.w[row + a.K + j] = a.gate ? a.gate[static_cast<size_t>(t) * a.n_shared + j] : 1.0f;
  }
}

}  // namespace

hipError_t launch_route_grouped(const RouteArgs& a, hipStream_t st) {
  if (a.T == 0) return hipSuccess;
  const uint32_t grid = static_cast<uint32_t>((a.T + kRouteWaves - 1) / kRouteWaves);
  if (a.logit_type == PW_F32) k_route_grouped<PW_F32><<<grid, 64 * kRouteWaves, 0, st>>>(a);
  else if (a.logit_type == PW_BF16) k_route_grouped<PW_BF16><<<grid, 64 * kRouteWaves, 0, st>>>(a);
  else k_route_grouped<PW_F16><<<grid, 64 * kRouteWaves, 0, st>>>(a);
  return hipGetLastError();
}

}  // namespace pw
