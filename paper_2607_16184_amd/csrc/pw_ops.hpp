// Argument blocks and launchers of the operators around the experts (norm,
// 8-bit product, KV cache and attention, grouped routing), shared by their C
// entry points (pw_ops_api.cpp) and kernels. Internal to libpagedweight.so.
#pragma once

#include <hip/hip_runtime.h>
#include <cstddef>
#include <cstdint>

#include "pw.h"

namespace pw {

struct NormArgs {
  const uint16_t* x;
  const uint16_t* residual;
  const uint16_t* weight;
  uint16_t* sum_out;
  uint16_t* y16;
  uint8_t* y8;
  float* y8_scale;
  int64_t ldx, ldr;
  int T, H;
  float eps;
  int act;
};

struct Gemm8Args {
  const uint8_t* a;
  const float* a_scale;
  const uint8_t* w;        // packed tiles
  const float* w_scale;
  void* y;
  float* part;             // sums of K's parts [ksplit][M][ldp] fp32
  int64_t lda, ldy, ldp;
  int M, N, K;
  int y_type;
  int ksplit, kb_per;      // parts of K and their 128-blocks
};

struct KvArgs {
  uint8_t* pool;
  int64_t block_stride;
  int n_blocks, block_tokens, n_kv_heads, head_dim;
  int act, bits;
};

struct AppendArgs {
  KvArgs kv;
  const uint16_t* k;
  const uint16_t* v;
  int64_t ld, ldh;
  const int64_t* slots;
  int T;
};

// A sequence's attended positions are cut into tiles of 32 tokens, at multiples
// of 32.
struct AttnArgs {
  KvArgs kv;
  const uint16_t* q;
  int64_t ldq, ldqh;
  int n_q_heads;
  const int32_t* table;
  int64_t ld_table;
  const int32_t* lens;
  int B, max_len, window;
  float scale;
  uint16_t* out;
  float* lse;
  int n_splits, split_tiles, n_shares, many_waves;
  float* part_o;           // [slots][min(16, query heads per key head)][D], not normalised
  float* part_ml;          // [slots][the same][2]: maximum (base 2), sum
};

struct RouteArgs {
  const void* logits;
  const float* bias;
  const float* gate;
  int32_t* ids;
  float* w;
  int32_t* offsets;
  int32_t* sorted_slot;
  int32_t* slot_pos;
  int T, E, K;
  int logit_type, score, n_groups, top_groups, group_top, renorm, n_shared;
  float w_scale;
};

struct AttnPlan {
  int n_splits, split_tiles;  // n_splits 0: equal shares of all tiles
  int n_shares;
  int many_waves;             // eight waves per workgroup, else four
  size_t ws_bytes;            // a slot's rows of head_dim + 2 floats each
};
AttnPlan attn_plan(int B, int n_q_heads, int n_kv_heads, int head_dim, int bits, int max_len, int window);

size_t gemm8_workspace(int M, int N, int K);

hipError_t launch_rms_norm(const NormArgs& a, hipStream_t st);
hipError_t launch_pack8(const uint8_t* w, int64_t ldw, int N, int K, uint8_t* packed, hipStream_t st);
hipError_t launch_gemm8(const Gemm8Args& a, hipStream_t st);
hipError_t launch_kv_append(const AppendArgs& a, hipStream_t st);
hipError_t launch_attn(const AttnArgs& a, hipStream_t st);
hipError_t launch_route_grouped(const RouteArgs& a, hipStream_t st);

}  // namespace pw
