/*
 * qqq_layer.h — C ABI of what a decoder layer does between the W4A8 linear calls of qqq.h, MI355X (gfx950):
 *
 *   fp16 output of a linear call --qqq_add_rmsnorm_quant--> residual stream, int8 codes + per-token scale   (next linear call's GEMM)
 *   fp16 gate and up projections --qqq_gated_act_quant--> int8 codes + per-token scale                     (down projection's GEMM)
 *   fp16 keys and values --qqq_kv8_append--> 8-bit paged cache --qqq_attention_kv8--> fp16 attention output
 *                                                              --qqq_kv8_read--> fp16 keys and values again
 *
 * Conventions as in qqq.h: every pointer inside is a DEVICE pointer owned by the caller (16-byte aligned unless stated),
 * `stream` is a hipStream_t passed as void*, a call only enqueues kernels, never allocates, synchronises or throws; return
 * QQQ_OK or an error code with nothing enqueued.  Codes and scales are what qqq_quant_act gives: symmetric, codes in [-127,127],
 * scale = largest magnitude / 127.  Forward only: the path serves quantised weights, nothing on it has a gradient.
 */
#ifndef QQQ_LAYER_H_
#define QQQ_LAYER_H_

#include "qqq.h"

#ifdef __cplusplus
extern "C" {
#endif

/*
 * Residual addition and root-mean-square norm of M rows of K values.
 *   h[m,k]   = x[m,k] + residual[m,k], rounded to the residual's type (h = x without a residual); written to sum_out
 *   rho[m]   = 1 / sqrt(mean_k h[m,k]^2 + eps)                                                       (fp32; 0 where that root is 0)
 *   qqq_add_rmsnorm:        y[m,k] = fp16_rne(h[m,k] * gain[k] * rho[m])
 *   qqq_add_rmsnorm_quant:  rho is the same for a whole row, so it goes into the scale: t[m,k] = fp32(h[m,k] * gain[k]),
 *                           S = max_k |t[m,k]| / 127,  a_q[m,k] = rne(t[m,k] / S),  s_a[m] = S * rho[m]
 *                           (the codes depend on h and gain alone; a row with S < 2^-120 gives s_a = 0 and codes 0)
 * Non-finite inputs are undefined.
 *   x_fp16 [M,ldx]; residual [M,ldr] fp16 or fp32 by residual_type, or NULL with QQQ_RESIDUAL_NONE; sum_out [M,lds] of the residual's
 *   type, required with a residual and NULL without; it may be the residual's own place (same pointer and stride), not otherwise
 *   overlap an input.  gain_fp16 [K].  K % 8 == 0, 8 <= K <= 131072, strides >= K and % 8 == 0 (elements).  eps >= 0, finite.
 *   y_fp16 [M,K], a_q [M,K] int8, s_a [M] fp32, dense.
 */
#define QQQ_RESIDUAL_NONE 0
#define QQQ_RESIDUAL_FP16 1
#define QQQ_RESIDUAL_FP32 2
int qqq_add_rmsnorm(const void* x_fp16, int64_t ldx, const void* residual, int64_t ldr, int residual_type,
                    const void* gain_fp16, float eps, int64_t M, int64_t K, void* sum_out, int64_t lds, void* y_fp16,
                    void* stream);
int qqq_add_rmsnorm_quant(const void* x_fp16, int64_t ldx, const void* residual, int64_t ldr, int residual_type,
                          const void* gain_fp16, float eps, int64_t M, int64_t K, void* sum_out, int64_t lds,
                          int8_t* a_q, float* s_a, void* stream);

/*
 * Gated activation of a feed-forward block, straight to the down projection's codes.
 *   h[m,f] = act(gate[m,f]) * up[m,f]  (fp32, never rounded to fp16, so products past 65504 are kept),  S = max_f |h[m,f]| / 127,
 *   a_q[m,f] = rne(h[m,f] / S),  s_a[m] = S  (a row with S < 2^-120 gives s_a = 0 and codes 0).  Non-finite inputs are undefined.
 *   act: QQQ_ACT_SILU  g / (1 + exp(-g)),  QQQ_ACT_GELU_TANH  g (1 + tanh(sqrt(2/pi) (g + 0.044715 g^3))) / 2.
 *   gate_fp16 [M,ldg], up_fp16 [M,ldu] (two halves of one linear call's output: strides 2F); F % 8 == 0, 8 <= F <= 131072,
 *   strides >= F and % 8 == 0.
 */
#define QQQ_ACT_SILU 0
#define QQQ_ACT_GELU_TANH 1
int qqq_gated_act_quant(const void* gate_fp16, int64_t ldg, const void* up_fp16, int64_t ldu, int act, int64_t M,
                        int64_t F, int8_t* a_q, float* s_a, void* stream);

/*
 * A key/value cache of one layer, in 8 bits with a scale for each page and head.
 * A sequence's tokens 0, 1, 2, .. lie in pages of page_tokens tokens; a page that is full is "closed" and held as codes, the tokens of
 * the page that is not yet full are held in fp16 in the sequence's tail slot, so that every token is quantised exactly once,
 * from its fp16 value, and what the cache holds does not depend on the pieces it was filled in.
 *   closed page p, head h:  s = max over the page |x| / 127,  code = 128 + rne(x / s)  (offset binary; s = 0 gives codes 128)
 *   value = s * (code - 128).  A NaN is taken as 0 and an infinity as +-65504 when appended, in the tail slots too.
 *   k_codes [pages, kv_heads, page_tokens, head_dim],  v_codes [pages, kv_heads, head_dim, page_tokens]  uint8
 *   k_scale, v_scale [pages, kv_heads] fp32
 *   k_tail [slots, kv_heads, page_tokens, head_dim],  v_tail [slots, kv_heads, head_dim, page_tokens]  fp16
 * page_tokens 16, 32 or 64; head_dim 64, 128 or 256; kv_heads >= 1; pages * kv_heads < 2^31.  (Values lie token by token: eight values of one channel are
 * then an operand of the matrix instruction as they are.)
 */
typedef struct qqq_kv8_cache {
  uint8_t* k_codes;
  float* k_scale;
  uint8_t* v_codes;
  float* v_scale;
  void* k_tail;
  void* v_tail;
  int64_t pages;
  int32_t slots, kv_heads, head_dim, page_tokens;
} qqq_kv8_cache;

/*
 * The sequences of a step.  Sequence b holds kv_len[b] tokens, the last n_b = cu[b+1] - cu[b] of which are this call's: rows
 * cu[b] .. cu[b+1]-1 of the token-major tensors beside it, at positions kv_len[b] - n_b .. kv_len[b] - 1.
 *   page_table [sequences, table_stride] int32, the first `columns` entries of a row being the sequence's pages in order (the entry of a
 *   page is read once it is closed); kv_len [sequences], cu [sequences + 1], slots [sequences] int32 (device, 4-byte aligned; slots NULL:
 *   sequence b has tail slot b).
 *   max_new, max_len: host-side bounds of n_b and kv_len[b]; max_len / page_tokens <= columns.  n_b may be 0.  Attention's work is laid out by these bounds, so its
 *   time depends on them: a token behind 8000 (64 heads of 128 over 8) takes 11 us where max_len is 8000 and 19 where it is 131072, and 47 single tokens
 *   in one call with a piece of 500 take 543 us, in a call of their own 79 and the piece 153.
 * The lengths and tables are read on the device only, so a captured step can be replayed with others.  What is out of bounds there
 * gives wrong results, never an access outside: lengths are cut to the bounds, a page or slot that does not exist is taken as
 * the last one when read and skipped when written, rows outside the tensors are skipped.
 */
typedef struct qqq_kv8_batch {
  const int32_t* page_table;
  int64_t table_stride;
  const int32_t* kv_len;
  const int32_t* cu;
  const int32_t* slots;
  int32_t columns, sequences, max_new, max_len;
} qqq_kv8_batch;

/*
 * Puts the step's new keys and values into the cache: pages that they fill are closed (quantised, together with what their tail slot
 * held), the rest goes to the tail slots.  Both structs are host structs, read before the call returns.
 *   k_fp16, v_fp16: token t, head h at t * token_stride + h * head_stride (elements, % 8 == 0), head_dim values; tokens rows.
 * No two sequences of a call may share a slot or a page that is closed by it.
 */
int qqq_kv8_append(const qqq_kv8_cache* cache, const qqq_kv8_batch* batch, const void* k_fp16, int64_t k_token_stride,
                   int64_t k_head_stride, const void* v_fp16, int64_t v_token_stride, int64_t v_head_stride,
                   int64_t tokens, void* stream);

/*
 * The last n_b tokens of every sequence as the cache holds them: fp16_rne(s * (code - 128)) from closed pages, the tail's values as they
 * are.  k_fp16, v_fp16 [tokens, kv_heads, head_dim], dense.
 */
int qqq_kv8_read(const qqq_kv8_cache* cache, const qqq_kv8_batch* batch, void* k_fp16, void* v_fp16, int64_t tokens,
                 void* stream);

/*
 * Attention of the step's new tokens (whose keys and values are in the cache already) over the cache.
 * Query i of sequence b stands at position pos = kv_len[b] - n_b + i and sees key j iff
 *   0 <= j < kv_len[b],  j <= pos if causal,  j > pos - window if window > 0.
 *   out[t,h,:] = sum_j softmax_j(scale * <q[t,h], k_j>) v_j,   lse[t,h] = log sum_j exp(scale * <q[t,h], k_j>);
 *   a query that sees nothing gives out = 0, lse = -infinity, one with a NaN gives NaN in its row; rows that belong to no sequence are
 *   left as they are.  q_heads / kv_heads query heads in a row share a key/value head.
 * Products of fp16 and of codes with fp32 accumulation; probabilities are rounded to fp16 (relative to the row's largest
 * contribution) for the second product, their sum is not.
 *   q_fp16: token t, head h at t * q_token_stride + h * q_head_stride (elements, % 8 == 0); out_fp16 [tokens, q_heads, head_dim] dense;
 *   lse [tokens, q_heads] fp32 or NULL.  scale > 0, finite.  window needs causal.
 *   q_heads % kv_heads == 0.  At most 65535 sequences where a key/value head has up to 32 rows (max_new * q_heads / kv_heads).
 *   workspace: qqq_attention_kv8_workspace_bytes() bytes (partial results of calls that split the keys; 0 where none is needed; enough for every window), its
 *   contents irrelevant on entry; not shared by calls that may run concurrently.
 */
size_t qqq_attention_kv8_workspace_bytes(const qqq_kv8_cache* cache, const qqq_kv8_batch* batch, int q_heads,
                                         int64_t tokens);
int qqq_attention_kv8(const qqq_kv8_cache* cache, const qqq_kv8_batch* batch, const void* q_fp16, int64_t q_token_stride,
                      int64_t q_head_stride, int q_heads, int64_t tokens, float scale, int causal, int window,
                      void* out_fp16, float* lse, void* workspace, size_t workspace_bytes, void* stream);

#ifdef __cplusplus
}
#endif
#endif /* QQQ_LAYER_H_ */
