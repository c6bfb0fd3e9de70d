// C entry points of the operators around the experts (declared in
// include/pw.h): checks of the arguments on the host, then a launch.
#include <cmath>
#include <string>

#include "pw.h"
#include "pw_internal.hpp"
#include "pw_ops.hpp"

namespace {

using pw::set_error;

pw_status launched(hipError_t e, const char* what) {
  if (e == hipSuccess) return PW_OK;
  return set_error(PW_EHIP, std::string(what) + ": " + hipGetErrorString(e));
}
bool aligned(const void* p, uintptr_t n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; }
bool act_ok(int t) { return t == PW_F16 || t == PW_BF16; }
bool rows_ok(int64_t ld, int64_t width) { return ld >= width && ld % 8 == 0; }

// What is wrong with a packed matrix's shape, or nullptr.
const char* packed_fault(int N, int K) {
  if (N < 1 || N > (1 << 30) || K < 128 || K % 128 != 0) return "need 1 <= N <= 2^30 and K a positive multiple of 128";
  if (K > (1 << 22) || (static_cast<int64_t>(N) + 15) / 16 * 16 * K >= (int64_t(1) << 40)) return "K above 2^22, or the matrix above 2^40 bytes";
  return nullptr;
}

// What is wrong with a cache's description, or nullptr.
const char* kv_fault(const pw_kv_cache* c) {
  if (!c) return "null cache";
  if (c->head_dim != 64 && c->head_dim != 128 && c->head_dim != 192 && c->head_dim != 256)
    return "head_dim must be 64, 128, 192 or 256";
  if (c->block_tokens != 32 && c->block_tokens != 64 && c->block_tokens != 128 && c->block_tokens != 256)
    return "block_tokens must be 32, 64, 128 or 256";
  if (c->n_kv_heads < 1 || c->n_kv_heads > 1024) return "need 1 <= n_kv_heads <= 1024";
  if (!act_ok(c->act)) return "act must be PW_F16 or PW_BF16";
  if (c->bits != 16 && c->bits != 8) return "bits must be 16 or 8";
  return nullptr;
}
const char* kv_memory_fault(const pw_kv_cache* c) {
  if (c->n_blocks < 1) return "need n_blocks >= 1";
  if (c->block_stride < 256 || c->block_stride % 256 != 0 || c->block_stride >= (int64_t(1) << 40))
    return "block_stride must be a positive multiple of 256 below 2^40";
  if (!c->pool || !aligned(c->pool, 256)) return "pool must be 256-byte aligned device memory";
  return nullptr;
}
pw::KvArgs kv_args(const pw_kv_cache* c) {
  return pw::KvArgs{static_cast<uint8_t*>(c->pool), c->block_stride, c->n_blocks, c->block_tokens,
                    c->n_kv_heads, c->head_dim, c->act, c->bits};
}
// The shape of an attention call, or what is wrong with it.
const char* attn_fault(const pw_kv_cache* c, int B, int n_q_heads, int max_len, int window) {
  if (const char* f = kv_fault(c)) return f;
  if (B < 0 || n_q_heads < 1 || n_q_heads % c->n_kv_heads != 0) return "need B >= 0 and n_q_heads a multiple of n_kv_heads";
  if (max_len < 0 || max_len > INT32_MAX - 256 || window < 0) return "need 0 <= max_len < 2^31 - 256 and window >= 0";
  return nullptr;
}
bool attn_too_wide(int B, int n_q_heads) { return B > 65535 || n_q_heads > 65535 || static_cast<int64_t>(B) * n_q_heads >= (int64_t(1) << 23); }

}  // namespace

extern "C" {

pw_status pw_rms_norm(const void* x, int64_t ldx, const void* residual, int64_t ldr, const void* weight, int T, int H,
                      float eps, int act, void* sum_out, void* y16, void* y8, float* y8_scale, void* stream) {
  if (T < 0 || H < 1 || H > 32768 || H % 8 != 0) return set_error(PW_EINVAL, "need T >= 0 and 1 <= H <= 32768, a multiple of 8");
  if (!act_ok(act)) return set_error(PW_EINVAL, "act must be PW_F16 or PW_BF16");
  if (!(eps >= 0.0f) || std::isinf(eps)) return set_error(PW_EINVAL, "eps must be finite and not negative");
  if (!rows_ok(ldx, H) || (residual && !rows_ok(ldr, H)))
    return set_error(PW_EINVAL, "row strides must be at least H and multiples of 8");
  if (!y8 != !y8_scale) return set_error(PW_EINVAL, "y8 and y8_scale go together");
  if (y8 && H % 128 != 0) return set_error(PW_EINVAL, "8-bit rows need H a multiple of 128");
  if (T == 0) return PW_OK;
  if (!sum_out && !y16 && !y8) return set_error(PW_EINVAL, "no output");
  if (!x) return set_error(PW_EINVAL, "null argument");
  if (!aligned(x, 16) || !aligned(residual, 16) || !aligned(weight, 16) || !aligned(sum_out, 16) || !aligned(y16, 16) ||
      !aligned(y8, 16) || !aligned(y8_scale, 4))
    return set_error(PW_EINVAL, "buffers must be 16-byte aligned");
  // an output's packed rows over an input's own: row by row, or the write of one
  // row meets the read of another
  const auto over_rows = [&](const void* out) { return out && ((out == x && ldx != H) || (out == residual && ldr != H)); };
  if (T > 1 && (over_rows(sum_out) || over_rows(y16)))
    return set_error(PW_EINVAL, "an output over x or residual needs that one's rows packed");
  if (sum_out && sum_out == y16) return set_error(PW_EINVAL, "sum_out and y16 need buffers of their own");
  const pw::NormArgs a{static_cast<const uint16_t*>(x), static_cast<const uint16_t*>(residual),
                       static_cast<const uint16_t*>(weight), static_cast<uint16_t*>(sum_out), static_cast<uint16_t*>(y16),
                       static_cast<uint8_t*>(y8), y8_scale, ldx, ldr, T, H, eps, act};
  return launched(pw::launch_rms_norm(a, static_cast<hipStream_t>(stream)), "norm launch");
}

pw_status pw_gemm_fp8_workspace(int M, int N, int K, size_t* ws_bytes) {
  if (!ws_bytes) return set_error(PW_EINVAL, "null argument");
  if (M < 0 || M > (1 << 30)) return set_error(PW_EINVAL, "need 0 <= M <= 2^30");
  if (const char* f = packed_fault(N, K)) return set_error(PW_EINVAL, f);
  *ws_bytes = pw::gemm8_workspace(M, N, K);
  return PW_OK;
}

pw_status pw_gemm_fp8_packed_bytes(int N, int K, size_t* bytes) {
  if (const char* f = packed_fault(N, K)) return set_error(PW_EINVAL, f);
  if (!bytes) return set_error(PW_EINVAL, "null argument");
  *bytes = (static_cast<size_t>(N) + 15) / 16 * 16 * K;
  return PW_OK;
}

pw_status pw_gemm_fp8_pack(const void* w, int64_t ldw, int N, int K, void* packed, void* stream) {
  if (const char* f = packed_fault(N, K)) return set_error(PW_EINVAL, f);
  if (ldw < K || ldw % 16 != 0) return set_error(PW_EINVAL, "ldw must be at least K and a multiple of 16");
  if (!w || !packed) return set_error(PW_EINVAL, "null argument");
  if (!aligned(w, 16) || !aligned(packed, 16)) return set_error(PW_EINVAL, "w and packed must be 16-byte aligned");
  return launched(pw::launch_pack8(static_cast<const uint8_t*>(w), ldw, N, K, static_cast<uint8_t*>(packed),
                                   static_cast<hipStream_t>(stream)), "pack launch");
}

pw_status pw_gemm_fp8(const void* a, int64_t lda, const float* a_scale, const void* w_packed, const float* w_scale, int M,
                      int N, int K, void* y, int64_t ldy, int y_type, void* ws, size_t ws_bytes, void* stream) {
  if (M < 0 || M > (1 << 30)) return set_error(PW_EINVAL, "need 0 <= M <= 2^30");
  if (const char* f = packed_fault(N, K)) return set_error(PW_EINVAL, f);
  if (y_type != PW_F16 && y_type != PW_BF16 && y_type != PW_F32)
    return set_error(PW_EINVAL, "y_type must be PW_F16, PW_BF16 or PW_F32");
  if (lda < K || lda % 16 != 0 || lda > (int64_t(1) << 22))
    return set_error(PW_EINVAL, "lda must be at least K, a multiple of 16 and at most 2^22");
  if (ldy < N) return set_error(PW_EINVAL, "ldy must be at least N");
  if (M == 0) return PW_OK;
  if (!a || !a_scale || !w_packed || !w_scale || !y) return set_error(PW_EINVAL, "null argument");
  if (!aligned(a, 16) || !aligned(w_packed, 16)) return set_error(PW_EINVAL, "a and w_packed must be 16-byte aligned");
  if (!aligned(a_scale, 4) || !aligned(w_scale, 4) || !aligned(y, y_type == PW_F32 ? 4 : 2))
    return set_error(PW_EINVAL, "scales and y must be aligned to their elements");
  const size_t need = pw::gemm8_workspace(M, N, K);
  if (need && (!ws || ws_bytes < need)) return set_error(PW_ENOMEM, "workspace too small (pw_gemm_fp8_workspace)");
  if (need && !aligned(ws, 16)) return set_error(PW_EINVAL, "the workspace must be 16-byte aligned");
  const pw::Gemm8Args g{static_cast<const uint8_t*>(a), a_scale, static_cast<const uint8_t*>(w_packed), w_scale, y,
                        static_cast<float*>(ws), lda, ldy, 0, M, N, K, y_type, 1, K / 128};
  return launched(pw::launch_gemm8(g, static_cast<hipStream_t>(stream)), "8-bit product launch");
}

pw_status pw_kv_block_bytes(const pw_kv_cache* c, size_t* bytes) {
  if (const char* f = kv_fault(c)) return set_error(PW_EINVAL, f);
  if (!bytes) return set_error(PW_EINVAL, "null argument");
  const size_t n = static_cast<size_t>(c->n_kv_heads) * c->block_tokens;
  *bytes = 2 * n * c->head_dim * (c->bits / 8) + (c->bits == 8 ? 8 * n : 0);
  return PW_OK;
}

pw_status pw_kv_append(const pw_kv_cache* c, const void* k, const void* v, int64_t ld, int64_t ldh, const int64_t* slots,
                       int T, void* stream) {
  if (const char* f = kv_fault(c)) return set_error(PW_EINVAL, f);
  if (const char* f = kv_memory_fault(c)) return set_error(PW_EINVAL, f);
  if (T < 0 || T > (1 << 30)) return set_error(PW_EINVAL, "need 0 <= T <= 2^30");
  if (static_cast<int64_t>(T) * c->n_kv_heads >= (int64_t(1) << 28)) return set_error(PW_EUNSUPPORTED, "T * n_kv_heads must stay below 2^28");
  if (ld % 8 != 0 || ldh % 8 != 0) return set_error(PW_EINVAL, "strides must be multiples of 8");
  if (T == 0) return PW_OK;
  if (!k || !v || !slots) return set_error(PW_EINVAL, "null argument");
  if (!aligned(k, 16) || !aligned(v, 16) || !aligned(slots, 8)) return set_error(PW_EINVAL, "k and v must be 16-byte aligned, slots 8-byte");
  const pw::AppendArgs a{kv_args(c), static_cast<const uint16_t*>(k), static_cast<const uint16_t*>(v), ld, ldh, slots, T};
  return launched(pw::launch_kv_append(a, static_cast<hipStream_t>(stream)), "append launch");
}

pw_status pw_attn_workspace(const pw_kv_cache* c, int B, int n_q_heads, int max_len, int window, size_t* ws_bytes) {
  if (const char* f = attn_fault(c, B, n_q_heads, max_len, window)) return set_error(PW_EINVAL, f);
  if (!ws_bytes) return set_error(PW_EINVAL, "null argument");
  if (attn_too_wide(B, n_q_heads)) return set_error(PW_EUNSUPPORTED, "B and n_q_heads must stay below 65536, their product below 2^23");
  *ws_bytes = pw::attn_plan(B, n_q_heads, c->n_kv_heads, c->head_dim, c->bits, max_len, window).ws_bytes;
  return PW_OK;
}

pw_status pw_attn_decode(const pw_kv_cache* c, const void* q, int64_t ldq, int64_t ldqh, int n_q_heads,
                         const int32_t* block_table, int64_t ld_table, const int32_t* seq_lens, int B, int max_len,
                         float scale, int window, void* out, float* lse, void* ws, size_t ws_bytes, void* stream) {
  if (const char* f = attn_fault(c, B, n_q_heads, max_len, window)) return set_error(PW_EINVAL, f);
  if (const char* f = kv_memory_fault(c)) return set_error(PW_EINVAL, f);
  if (attn_too_wide(B, n_q_heads)) return set_error(PW_EUNSUPPORTED, "B and n_q_heads must stay below 65536, their product below 2^23");
  if (ldq % 8 != 0 || ldqh % 8 != 0) return set_error(PW_EINVAL, "strides must be multiples of 8");
  if (!std::isfinite(scale)) return set_error(PW_EINVAL, "scale must be finite");
  const int64_t blocks = (static_cast<int64_t>(max_len) + c->block_tokens - 1) / c->block_tokens;
  if (ld_table < blocks) return set_error(PW_EINVAL, "the block table's rows are shorter than max_len");
  if (B == 0) return PW_OK;
  if (!q || !seq_lens || !out || (max_len > 0 && !block_table)) return set_error(PW_EINVAL, "null argument");
  if (!aligned(q, 16) || !aligned(out, 16) || !aligned(block_table, 4) || !aligned(seq_lens, 4) || !aligned(lse, 4))
    return set_error(PW_EINVAL, "q and out must be 16-byte aligned, the other buffers 4-byte");
  const pw::AttnPlan p = pw::attn_plan(B, n_q_heads, c->n_kv_heads, c->head_dim, c->bits, max_len, window);
  if (p.ws_bytes && (!ws || ws_bytes < p.ws_bytes)) return set_error(PW_ENOMEM, "workspace too small (pw_attn_workspace)");
  if (p.ws_bytes && !aligned(ws, 16)) return set_error(PW_EINVAL, "the workspace must be 16-byte aligned");
  pw::AttnArgs a{};
  a.kv = kv_args(c);
  a.q = static_cast<const uint16_t*>(q);
  a.ldq = ldq;
  a.ldqh = ldqh;
  a.n_q_heads = n_q_heads;
  a.table = block_table;
  a.ld_table = ld_table;
  a.lens = seq_lens;
  a.B = B;
  a.max_len = max_len;
  a.window = window;
  a.scale = scale;
  a.out = static_cast<uint16_t*>(out);
  a.lse = lse;
  a.n_splits = p.n_splits;
  a.split_tiles = p.split_tiles;
  a.n_shares = p.n_shares;
  a.many_waves = p.many_waves;
  a.part_o = static_cast<float*>(ws);
  a.part_ml = a.part_o + p.ws_bytes / sizeof(float) / (c->head_dim + 2) * c->head_dim;
  return launched(pw::launch_attn(a, static_cast<hipStream_t>(stream)), "attention launch");
}

pw_status pw_route_grouped(const void* logits, int logit_type, const float* bias, int T, int E, int K, int score,
                           int n_groups, int top_groups, int group_top, int renorm, float w_scale, int n_shared,
                           const float* shared_gate, int32_t* ids, float* w, int32_t* offsets, int32_t* sorted_slot,
                           int32_t* slot_pos, void* stream) {
  if (T < 0 || E < 1 || K < 1 || K > E || K > 16 || n_shared < 0 || E + n_shared > 256)
    return set_error(PW_EINVAL, "need 1 <= K <= E, K <= 16, n_shared >= 0, E + n_shared <= 256, T >= 0");
  if (logit_type != PW_F32 && !act_ok(logit_type)) return set_error(PW_EINVAL, "logit_type must be PW_F32, PW_F16 or PW_BF16");
  if (score != PW_SCORE_SOFTMAX && score != PW_SCORE_SIGMOID)
    return set_error(PW_EINVAL, "score must be PW_SCORE_SOFTMAX or PW_SCORE_SIGMOID");
  if (n_groups < 1 || n_groups > 64 || E % n_groups != 0 || top_groups < 1 || top_groups > n_groups)
    return set_error(PW_EINVAL, "need 1 <= n_groups <= 64 dividing E and 1 <= top_groups <= n_groups");
  if (group_top != 1 && group_top != 2) return set_error(PW_EINVAL, "group_top must be 1 or 2");
  if (K > top_groups * (E / n_groups)) return set_error(PW_EINVAL, "K exceeds the experts of top_groups groups");
  if (!std::isfinite(w_scale)) return set_error(PW_EINVAL, "w_scale must be finite");
  const int Kt = K + n_shared;
  if (T > (1 << 30) || static_cast<int64_t>(T) * Kt >= (int64_t(1) << 31)) return set_error(PW_EINVAL, "need T <= 2^30 and T * (K + n_shared) < 2^31");
  if (!offsets || (T > 0 && (!logits || !ids || !w || !sorted_slot || !slot_pos))) return set_error(PW_EINVAL, "null argument");
  pw::RouteArgs a{};
  a.logits = logits;
  a.bias = bias;
  a.gate = shared_gate;
  a.ids = ids;
  a.w = w;
  a.offsets = offsets;
  a.sorted_slot = sorted_slot;
  a.slot_pos = slot_pos;
  a.T = T;
  a.E = E;
  a.K = K;
  a.logit_type = logit_type;
  a.score = score;
  a.n_groups = n_groups;
  a.top_groups = top_groups;
  a.group_top = group_top;
  a.renorm = renorm;
  a.n_shared = n_shared;
  a.w_scale = w_scale;
  return launched(pw::launch_route_grouped(a, static_cast<hipStream_t>(stream)), "router launch");
}

}  // extern "C"
