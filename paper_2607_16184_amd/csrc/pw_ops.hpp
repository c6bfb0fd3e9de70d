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

struct Rotate {
  const double* inv_freq;  // [R / 2], radians a position
  const int32_t* positions;
  int64_t offset;          // added to each
  int R, interleaved;
  float amplitude;
};

struct HeadsArgs {
  Rotate rot;
  const uint16_t* q;
  const uint16_t* k;
  const uint16_t* v;       // strides as k; with a cache
  const uint16_t* q_weight;
  const uint16_t* k_weight;
  uint16_t* q_out;
  uint16_t* k_out;         // without one
  int64_t ldq, ldqh, ldk, ldkh, ldqo, ldqoh, ldko, ldkoh;
  int n_q, n_k, T, D, act, norm;
  float eps;
  KvArgs kv;
  const int64_t* slots;    // nullptr: no cache
};

struct KeepArgs {
  KvArgs kv;
  const int32_t* starts;
  const int32_t* table;
  int64_t ld_table;
  const int32_t* lens;
  const int64_t* chosen;   // [B][words]
  int32_t* new_lens;
  int B, max_len, words;
};

// Attention of several rows per sequence. An item is a sequence, a key head and a
// group of col_tiles x 16 columns: column c of a sequence is query head c mod g of
// the key head's g, of row c / g.
struct RowsArgs {
  KvArgs kv;
  const uint16_t* q;
  int64_t ldq, ldqh;
  int n_q_heads;
  const int32_t* starts;
  const int32_t* table;
  int64_t ld_table;
  const int32_t* lens;
  const int64_t* masks;    // [T][words], nullptr: causal
  int words;
  int B, T, max_len, window;
  float scale;
  uint16_t* out;
  float* lse;
  uint32_t over_g;         // floor(2^32 / g), for g = 1 the largest number
  int64_t whole;           // splits: items that are not split, the first ones
  int n_splits, split_tiles;   // of the others
  int n_shares, least;     // shares per key head (0: splits), tiles of one at least
  int64_t items;           // at most
  float* part_o;           // [key heads][shares + items][columns][D], not normalised
  float* part_ml;          // [the same][2]: maximum (base 2), sum
  int32_t* meta;           // [key heads][items][2]: first slot, parts
};

struct RowsPlan {
  int many;                // waves with columns of their own, else tiles of their own
  int col_tiles;           // of a wave
  int64_t items, whole, n_shares;
  int n_splits, split_tiles, least;
  int64_t slots;           // rows of head_dim + 2 floats of the workspace
  size_t ws_bytes;
};
RowsPlan rows_plan(int B, int T, int n_q_heads, int n_kv_heads, int head_dim, int act, int bits, int max_len,
                   int window);

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
hipError_t launch_heads(const HeadsArgs& a, hipStream_t st);
bool append_by_runs(const HeadsArgs& a);
hipError_t launch_append_runs(const HeadsArgs& a, hipStream_t st);
hipError_t launch_kv_keep(const KeepArgs& a, hipStream_t st);
hipError_t launch_attn_rows(const RowsArgs& a, const RowsPlan& p, hipStream_t st);
hipError_t launch_route_grouped(const RouteArgs& a, hipStream_t st);

}  // namespace pw
