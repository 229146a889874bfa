// C-ABI entry points of qqq_layer.h: argument validation (host code only).
#include <math.h>

#include "qqq_kv8.h"

namespace qqq {

int launch_rmsnorm(const void* x, int64_t ldx, const void* residual, int64_t ldr, int residual_type, const void* gain, float eps, int64_t M,
                   int64_t K, void* sum_out, int64_t lds, void* y, int8_t* a_q, float* s_a, hipStream_t st);
int launch_gated_act(const void* gate, int64_t ldg, const void* up, int64_t ldu, int act, int64_t M, int64_t F, int8_t* a_q, float* s_a,
                     hipStream_t st);
int launch_kv8_append(const Kv8& c, int D, int P, int sequences, const void* k, int64_t k_token, int64_t k_head, const void* v,
                      int64_t v_token, int64_t v_head, hipStream_t st);
int launch_kv8_read(const Kv8& c, int D, int P, int sequences, void* k, void* v, hipStream_t st);
int launch_attention_kv8(const Kv8& c, int D, int P, int sequences, const void* q, int64_t q_token, int64_t q_head, int q_heads, float scale,
                         int causal, int window, void* out, float* lse, void* workspace, size_t workspace_bytes, hipStream_t st);
size_t attention_kv8_bytes(int heads, int q_heads, int D, int sequences, int max_new, int max_len, int64_t tokens);

namespace {

constexpr int64_t kMaxRow = 131072;     // values of a row, as K of the GEMMs
constexpr int64_t kMaxTokens = 1 << 30; // of a sequence, and rows of a call: positions stay in 32 bits

bool aligned(const void* p, uintptr_t to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) == 0; }

bool row_stride_ok(int64_t ld, int64_t K) { return ld >= K && ld % 8 == 0; }

int check_rows(const char* name, int64_t M, int64_t K) {
  if (M < 0 || M > 0x7FFFFFFF || K < 8 || K % 8 != 0 || K > kMaxRow)
    return set_error(QQQ_ERR_SHAPE, "%s: unsupported %lld rows of %lld values", name, (long long)M, (long long)K);
  return QQQ_OK;
}

int rmsnorm(const char* name, const void* x, int64_t ldx, const void* residual, int64_t ldr, int residual_type, const void* gain, float eps,
            int64_t M, int64_t K, void* sum_out, int64_t lds, void* y, int8_t* a_q, float* s_a, bool quantise, void* stream) {
  if (int rc = check_rows(name, M, K)) return rc;
  if (residual_type < QQQ_RESIDUAL_NONE || residual_type > QQQ_RESIDUAL_FP32) return set_error(QQQ_ERR_SHAPE, "%s: residual type %d", name, residual_type);
  const bool has = residual_type != QQQ_RESIDUAL_NONE;
  if (!row_stride_ok(ldx, K) || (has && (!row_stride_ok(ldr, K) || !row_stride_ok(lds, K))))
    return set_error(QQQ_ERR_SHAPE, "%s: row strides %lld, %lld, %lld for %lld values", name, (long long)ldx, (long long)ldr, (long long)lds, (long long)K);
  if (!(eps >= 0.0f) || isinf(eps)) return set_error(QQQ_ERR_SHAPE, "%s: eps %g", name, (double)eps);
  if (M == 0) return QQQ_OK;
  if (!x || !gain || (quantise ? !a_q || !s_a : !y) || (has && (!residual || !sum_out))) return set_error(QQQ_ERR_NULL, "%s: NULL pointer", name);
  if (!has && (residual || sum_out)) return set_error(QQQ_ERR_SHAPE, "%s: a residual without its type", name);
  if (!aligned(x, 16) || !aligned(gain, 16) || !aligned(residual, 16) || !aligned(sum_out, 16) || !aligned(y, 16) || !aligned(a_q, 16) || !aligned(s_a, 4))
    return set_error(QQQ_ERR_SHAPE, "%s: misaligned pointer", name);
  if (has && sum_out == residual && lds != ldr) return set_error(QQQ_ERR_SHAPE, "%s: sum in the residual's place with another stride", name);
  route_reset();
  return launch_rmsnorm(x, ldx, residual, ldr, residual_type, gain, eps, M, K, sum_out, lds, y, a_q, s_a, (hipStream_t)stream);
}

int check_cache(const char* name, const qqq_kv8_cache* c, const qqq_kv8_batch* b, int64_t tokens) {
  if (!c || !b) return set_error(QQQ_ERR_NULL, "%s: NULL struct", name);
  if ((c->page_tokens != 16 && c->page_tokens != 32 && c->page_tokens != 64) || (c->head_dim != 64 && c->head_dim != 128 && c->head_dim != 256) ||
      c->kv_heads < 1 || c->pages < 1 || c->pages > 0x7FFFFFFF / c->kv_heads || c->slots < 1)
    return set_error(QQQ_ERR_SHAPE, "%s: unsupported cache: %lld pages of %d tokens, %d heads of %d, %d slots", name, (long long)c->pages,
                     c->page_tokens, c->kv_heads, c->head_dim, c->slots);
  if (b->sequences < 0 || tokens < 0 || tokens > kMaxTokens || b->max_new < 0 || b->max_new > kMaxTokens || b->max_len < 0 || b->max_len > kMaxTokens ||
      b->columns < 0 || b->table_stride < b->columns || b->max_len / c->page_tokens > b->columns)
    return set_error(QQQ_ERR_SHAPE, "%s: unsupported batch: %d sequences, %lld rows, at most %d new of %d tokens, %d page columns of stride %lld", name,
                     b->sequences, (long long)tokens, b->max_new, b->max_len, b->columns, (long long)b->table_stride);
  return QQQ_OK;
}
bool nothing(const qqq_kv8_batch* b, int64_t tokens) { return b->sequences == 0 || b->max_new == 0 || tokens == 0; }
int check_pointers(const char* name, const qqq_kv8_cache* c, const qqq_kv8_batch* b) {
  if (!c->k_codes || !c->v_codes || !c->k_scale || !c->v_scale || !c->k_tail || !c->v_tail || !b->kv_len || !b->cu || (!b->page_table && b->columns > 0))
    return set_error(QQQ_ERR_NULL, "%s: NULL pointer in a struct", name);
  if (!b->page_table && b->max_len >= c->page_tokens) return set_error(QQQ_ERR_NULL, "%s: no page table", name);
  if (!aligned(c->k_codes, 16) || !aligned(c->v_codes, 16) || !aligned(c->k_tail, 16) || !aligned(c->v_tail, 16) || !aligned(c->k_scale, 4) ||
      !aligned(c->v_scale, 4) || !aligned(b->page_table, 4) || !aligned(b->kv_len, 4) || !aligned(b->cu, 4) || !aligned(b->slots, 4))
    return set_error(QQQ_ERR_SHAPE, "%s: misaligned pointer in a struct", name);
  return QQQ_OK;
}
Kv8 kernel_args(const qqq_kv8_cache* c, const qqq_kv8_batch* b, int64_t tokens) {
  Kv8 k;
  k.k_codes = c->k_codes;
  k.v_codes = c->v_codes;
  k.k_scale = c->k_scale;
  k.v_scale = c->v_scale;
  k.k_tail = (const uint16_t*)c->k_tail;
  k.v_tail = (const uint16_t*)c->v_tail;
  k.table = b->page_table;
  k.kv_len = b->kv_len;
  k.cu = b->cu;
  k.slots = b->slots;
  k.table_stride = b->table_stride;
  k.pages = c->pages;
  k.nslots = c->slots;
  k.heads = c->kv_heads;
  k.max_new = b->max_new;
  k.max_len = b->max_len;
  k.tokens = tokens;
  return k;
}

}  // namespace
}  // namespace qqq

using namespace qqq;

extern "C" {

int qqq_add_rmsnorm(const void* x_fp16, int64_t ldx, const void* residual, int64_t ldr, int residual_type, const void* gain_fp16, float eps,
                    int64_t M, int64_t K, void* sum_out, int64_t lds, void* y_fp16, void* stream) {
  return rmsnorm("qqq_add_rmsnorm", x_fp16, ldx, residual, ldr, residual_type, gain_fp16, eps, M, K, sum_out, lds, y_fp16, nullptr, nullptr, false,
                 stream);
}

int qqq_add_rmsnorm_quant(const void* x_fp16, int64_t ldx, const void* residual, int64_t ldr, int residual_type, const void* gain_fp16, float eps,
                          int64_t M, int64_t K, void* sum_out, int64_t lds, int8_t* a_q, float* s_a, void* stream) {
  return rmsnorm("qqq_add_rmsnorm_quant", x_fp16, ldx, residual, ldr, residual_type, gain_fp16, eps, M, K, sum_out, lds, nullptr, a_q, s_a, true,
                 stream);
}

int qqq_gated_act_quant(const void* gate_fp16, int64_t ldg, const void* up_fp16, int64_t ldu, int act, int64_t M, int64_t F, int8_t* a_q, float* s_a,
                        void* stream) {
  const char* name = "qqq_gated_act_quant";
  if (int rc = check_rows(name, M, F)) return rc;
  if (act != QQQ_ACT_SILU && act != QQQ_ACT_GELU_TANH) return set_error(QQQ_ERR_SHAPE, "%s: activation %d", name, act);
  if (!row_stride_ok(ldg, F) || !row_stride_ok(ldu, F))
    return set_error(QQQ_ERR_SHAPE, "%s: row strides %lld, %lld for %lld values", name, (long long)ldg, (long long)ldu, (long long)F);
  if (M == 0) return QQQ_OK;
  if (!gate_fp16 || !up_fp16 || !a_q || !s_a) return set_error(QQQ_ERR_NULL, "%s: NULL pointer", name);
  if (!aligned(gate_fp16, 16) || !aligned(up_fp16, 16) || !aligned(a_q, 16) || !aligned(s_a, 4)) return set_error(QQQ_ERR_SHAPE, "%s: misaligned pointer", name);
  route_reset();
  return launch_gated_act(gate_fp16, ldg, up_fp16, ldu, act, M, F, a_q, s_a, (hipStream_t)stream);
}

int qqq_kv8_append(const qqq_kv8_cache* cache, const qqq_kv8_batch* batch, const void* k_fp16, int64_t k_token_stride, int64_t k_head_stride,
                   const void* v_fp16, int64_t v_token_stride, int64_t v_head_stride, int64_t tokens, void* stream) {
  const char* name = "qqq_kv8_append";
  if (int rc = check_cache(name, cache, batch, tokens)) return rc;
  if (k_token_stride % 8 || k_head_stride % 8 || v_token_stride % 8 || v_head_stride % 8 || k_token_stride < 0 || k_head_stride < 0 ||
      v_token_stride < 0 || v_head_stride < 0)
    return set_error(QQQ_ERR_SHAPE, "%s: strides %lld, %lld, %lld, %lld", name, (long long)k_token_stride, (long long)k_head_stride,
                     (long long)v_token_stride, (long long)v_head_stride);
  if (nothing(batch, tokens)) return QQQ_OK;
  if (!k_fp16 || !v_fp16) return set_error(QQQ_ERR_NULL, "%s: NULL pointer", name);
  if (!aligned(k_fp16, 16) || !aligned(v_fp16, 16)) return set_error(QQQ_ERR_SHAPE, "%s: misaligned pointer", name);
  if (int rc = check_pointers(name, cache, batch)) return rc;
  route_reset();
  return launch_kv8_append(kernel_args(cache, batch, tokens), cache->head_dim, cache->page_tokens, batch->sequences, k_fp16, k_token_stride,
                           k_head_stride, v_fp16, v_token_stride, v_head_stride, (hipStream_t)stream);
}

int qqq_kv8_read(const qqq_kv8_cache* cache, const qqq_kv8_batch* batch, void* k_fp16, void* v_fp16, int64_t tokens, void* stream) {
  const char* name = "qqq_kv8_read";
  if (int rc = check_cache(name, cache, batch, tokens)) return rc;
  if (nothing(batch, tokens)) return QQQ_OK;
  if (!k_fp16 || !v_fp16) return set_error(QQQ_ERR_NULL, "%s: NULL pointer", name);
  if (!aligned(k_fp16, 16) || !aligned(v_fp16, 16)) return set_error(QQQ_ERR_SHAPE, "%s: misaligned pointer", name);
  if (int rc = check_pointers(name, cache, batch)) return rc;
  route_reset();
  return launch_kv8_read(kernel_args(cache, batch, tokens), cache->head_dim, cache->page_tokens, batch->sequences, k_fp16, v_fp16, (hipStream_t)stream);
}

size_t qqq_attention_kv8_workspace_bytes(const qqq_kv8_cache* cache, const qqq_kv8_batch* batch, int q_heads, int64_t tokens) {
  if (check_cache("qqq_attention_kv8_workspace_bytes", cache, batch, tokens) || q_heads < 1 || q_heads % cache->kv_heads || nothing(batch, tokens)) return 0;
  return attention_kv8_bytes(cache->kv_heads, q_heads, cache->head_dim, batch->sequences, batch->max_new, batch->max_len, tokens);
}

int qqq_attention_kv8(const qqq_kv8_cache* cache, const qqq_kv8_batch* batch, const void* q_fp16, int64_t q_token_stride, int64_t q_head_stride,
                      int q_heads, int64_t tokens, float scale, int causal, int window, void* out_fp16, float* lse, void* workspace,
                      size_t workspace_bytes, void* stream) {
  const char* name = "qqq_attention_kv8";
  if (int rc = check_cache(name, cache, batch, tokens)) return rc;
  if (q_heads < 1 || q_heads % cache->kv_heads || (int64_t)batch->max_new * (q_heads / cache->kv_heads) > kMaxTokens)
    return set_error(QQQ_ERR_SHAPE, "%s: %d query heads for %d", name, q_heads, cache->kv_heads);
  if (q_token_stride % 8 || q_head_stride % 8 || q_token_stride < 0 || q_head_stride < 0)
    return set_error(QQQ_ERR_SHAPE, "%s: strides %lld, %lld", name, (long long)q_token_stride, (long long)q_head_stride);
  if (!(scale > 0.0f) || isinf(scale)) return set_error(QQQ_ERR_SHAPE, "%s: scale %g", name, (double)scale);
  if (window < 0 || (window > 0 && !causal)) return set_error(QQQ_ERR_SHAPE, "%s: window %d%s", name, window, causal ? "" : " without causal");
  if (nothing(batch, tokens)) return QQQ_OK;
  if (!q_fp16 || !out_fp16) return set_error(QQQ_ERR_NULL, "%s: NULL pointer", name);
  if (!aligned(q_fp16, 16) || !aligned(out_fp16, 16) || !aligned(lse, 4) || !aligned(workspace, 16)) return set_error(QQQ_ERR_SHAPE, "%s: misaligned pointer", name);
  if (int rc = check_pointers(name, cache, batch)) return rc;
  route_reset();
  return launch_attention_kv8(kernel_args(cache, batch, tokens), cache->head_dim, cache->page_tokens, batch->sequences, q_fp16, q_token_stride,
                              q_head_stride, q_heads, scale, causal, window, out_fp16, lse, workspace, workspace ? workspace_bytes : 0,
                              (hipStream_t)stream);
}

}  // extern "C"
