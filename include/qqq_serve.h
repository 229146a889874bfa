/*
 * qqq_serve.h — C ABI of the two ends of a serving step, before the first decoder layer and behind the last, MI355X (gfx950):
 *
 *   what sessions hold and bring --qqq_kv8_plan--> page tables, lengths, places of the rows (the qqq_kv8_batch of qqq_layer.h); --qqq_kv8_release--> pages free again
 *   int8 codes of the last norm (qqq_add_rmsnorm_quant) --qqq_gemm_w8a8--> logits --qqq_logprobs--> log probabilities, entropies, likeliest tokens
 *
 * Conventions as in qqq.h: every pointer inside is a DEVICE pointer owned by the caller, `stream` is a hipStream_t passed as void*, a call only enqueues
 * kernels, never allocates, synchronises or throws; return QQQ_OK or an error code with nothing enqueued.  Forward only: the path serves quantised
 * weights, nothing on it has a gradient.  Results do not depend on the order in which workgroups run.
 */
#ifndef QQQ_SERVE_H_
#define QQQ_SERVE_H_

#include "qqq_layer.h"

#ifdef __cplusplus
extern "C" {
#endif

/*
 * What a program keeps of its sessions on the GPU, so that a step's tables can be made there (and a captured step replayed) without the host.
 *   pages [sessions, pages_stride] int32: the first held / page_tokens of a row's `columns` entries are the session's closed pages in order
 *   held [sessions] int32: tokens in the cache
 *   free_pages [pool] int32, free_count [1] int32: the pages that no session has, a stack; the last of the first free_count entries is taken first.  They need not be all
 *   of the cache's pages, nor the lowest: any numbers from 0 on
 *   held_after, free_count_after: where a call writes what holds after it; the same pointers, or others (then held and free_count stay as they are, and of
 *   held_after only the step's sessions are written)
 * All 4-byte aligned.  page_tokens 16, 32 or 64, as in qqq_kv8_cache.  The struct is a host struct, read before the call returns.
 */
typedef struct qqq_kv8_sessions {
  int32_t* pages;
  int64_t pages_stride;
  const int32_t* held;
  int32_t* held_after;
  int32_t* free_pages;
  const int32_t* free_count;
  int32_t* free_count_after;
  int64_t pool;
  int32_t sessions, columns, page_tokens;
} qqq_kv8_sessions;

/*
 * The tables of a step in which sequence b is session batch->slots[b] (slots NULL: session b) and brings new_tokens[b] tokens, in the order of the sequences:
 *   n_b = new_tokens[b], cut to 0 .. max_new, to max_len - held and to the rows that are left;  len_b = held + n_b;  cu[b] = n_0 + .. + n_(b-1)
 *   fresh_b = len_b / page_tokens - held / page_tokens pages come from the stack's top, the first sequence's first
 * Written: batch->kv_len [sequences], batch->cu [sequences + 1], batch->page_table (of row b the first len_b / page_tokens entries: the session's pages, then the
 * fresh ones), the fresh ones in sessions->pages too, held_after, free_count_after, and, where they are not NULL,
 *   sequence [tokens], positions [tokens] int32: of each row its sequence in the step and its place in it, held .. len_b - 1; rows behind cu[sequences] are left as they are
 *   lacking [1] int32: pages that were wanted and not there.  Their entries are -1, which is no page: append drops what it would write to them, and attention reads the cache's last
 *   page in their place, whosever it is, in this step and in all that follow.  So a program either wants no more than free_count covers (the sequences in order, fresh_b each), or gives
 *   held_after and free_count_after of their own, looks at lacking before anything is appended, and makes the plan again for fewer tokens: pages, held and free_count still say
 *   what they said of all that the sessions hold.  After a plan in place a session with such an entry can only end.
 * batch is a qqq_kv8_batch as the calls of qqq_layer.h take it, its tensors written here.  page_table may be sessions->pages itself (with its stride) where slots is NULL;
 * no other outputs may overlap.  max_len / page_tokens <= columns of both tables; sequences < 2^24.  A session that does not exist brings nothing; one that is there twice, or held and free_count
 * that are out of bounds, give wrong tables, never an access outside.
 *   workspace: qqq_kv8_plan_workspace_bytes() bytes (of the call with these pointers: most calls with held_after and free_count_after of their own need none), 4-byte aligned, contents irrelevant on entry; not shared by calls that may run concurrently.
 */
size_t qqq_kv8_plan_workspace_bytes(const qqq_kv8_sessions* sessions, const qqq_kv8_batch* batch);
int qqq_kv8_plan(const qqq_kv8_sessions* sessions, const qqq_kv8_batch* batch, const int32_t* new_tokens, int64_t tokens,
                 int32_t* sequence, int32_t* positions, int32_t* lacking, void* workspace, size_t workspace_bytes, void* stream);

/*
 * Sessions ids[0 .. count-1] (NULL: 0 .. count-1) end: their pages go to the stack in that order, a session's in their own, and they hold nothing.  In place only: held_after is
 * held and free_count_after is free_count.  Entries that are no page (below 0) are dropped, and so is what the stack has no room for; a session that does not exist
 * is skipped, one that is there twice is released once, in the first of its places.
 */
int qqq_kv8_release(const qqq_kv8_sessions* sessions, const int32_t* ids, int64_t count, void* stream);

/*
 * Weights in 8 bits.  Codes and scales of fp16 weights [N,K] are what qqq_quant_act gives for them, a row for an output channel: symmetric, codes in
 * [-127,127], one fp32 scale a channel.
 *   w_codes [N,ldw] int8, 16-byte aligned, ldw >= K, ldw % 16 == 0.  1 <= N <= 2^24, K % 128 == 0, 128 <= K <= 131072, N K <= 2^35.
 *   w_packed: qqq_packed_w8_bytes(N,K) = K * (N rounded up to 16) bytes, opaque device tile layout, 16-byte aligned: 2 KiB chunks of 16 channels x 128 k in the order of
 *   the matrix instruction's operands; channels past N are zeros.  qqq_unpack_w8 is the exact inverse ([N,K], dense).
 */
size_t qqq_packed_w8_bytes(int64_t N, int64_t K); /* 0 for unsupported shapes */
int qqq_pack_w8(const int8_t* w_codes, int64_t N, int64_t K, int64_t ldw, void* w_packed, void* stream);
int qqq_unpack_w8(const void* w_packed, int64_t N, int64_t K, int8_t* w_codes, void* stream);

/*
 * W8A8 GEMM:  acc[m,n] = sum_k a_q[m,k] * w[n,k]  (int32, exact),  t = fp32_rne(float(acc) * s_a[m]),
 *   y[m,n] = fp16_rne(t * s_w[n])  or  fp32_rne(t * s_w[n])  by y_type.
 *   a_q [M,K] int8, dense, 16-byte aligned, codes in [-127,127]; s_a [M] fp32; w_packed as above; s_w [N] fp32; y [M,ldy] of the type, ldy >= N, aligned to its type;
 *   acc_out [M,N] int32 dense or NULL (parity/debug).  N and K as above, M <= 2^30, M == 0 is a no-op.
 *   workspace: qqq_gemm_w8a8_workspace_bytes() bytes, 16-byte aligned (partial sums of calls that split K; 0 where none is needed), contents irrelevant on entry;
 *   not shared by calls that may run concurrently.
 */
#define QQQ_OUT_FP16 0
#define QQQ_OUT_FP32 1
size_t qqq_gemm_w8a8_workspace_bytes(int64_t M, int64_t N, int64_t K);
int qqq_gemm_w8a8(const int8_t* a_q, const float* s_a, const void* w_packed, const float* s_w, void* y, int y_type, int64_t ldy,
                  int32_t* acc_out, int64_t M, int64_t N, int64_t K, void* workspace, size_t workspace_bytes, void* stream);

/*
 * What is asked of the logits x[m, 0 .. V-1] of M rows:
 *   lse[m] = log sum_v exp(x[m,v]);  logprob[m] = x[m, tokens[m]] - lse[m];  entropy[m] = -sum_v p_v log p_v,  p_v = exp(x[m,v] - lse[m])
 *   top_tokens[m, 0 .. top-1]: the largest logits' places, in falling order, of equal ones (-0 and 0 are equal) the lowest place first; top_logprobs: their x - lse.  Places that V
 *   does not have give -1 and -infinity.
 * A logit of -infinity is masked: its probability is 0 and it adds nothing to the entropy.  A row of nothing else gives lse = -infinity, entropy 0 and log probabilities of
 * -infinity.  A row with a NaN or +infinity gives NaN in all its numbers; among the top tokens NaN counts as larger than everything.  A token below 0 is none: its logprob is 0,
 * whatever the row holds; one past V - 1 gives NaN.  All sums are fp32, relative to the largest logit.
 *   logits [M,ld] fp16 or fp32 by type, aligned to it, ld >= V; 1 <= V < 2^30, M < 2^24; tokens [M] int32 or NULL (then logprob is NULL); 0 <= top <= QQQ_MAX_TOP, top_tokens [M,top] int32
 *   and top_logprobs [M,top] fp32 where top > 0; logprob, entropy, lse [M] fp32, each may be NULL.
 *   workspace: qqq_logprobs_workspace_bytes() bytes, 16-byte aligned (0 where rows are not split over workgroups), contents irrelevant on entry; not shared by calls
 *   that may run concurrently.
 */
#define QQQ_LOGITS_FP16 0
#define QQQ_LOGITS_FP32 1
#define QQQ_MAX_TOP 64
size_t qqq_logprobs_workspace_bytes(int64_t M, int64_t V, int type);
int qqq_logprobs(const void* logits, int64_t ld, int type, int64_t M, int64_t V, const int32_t* tokens, int top, float* logprob,
                 float* entropy, float* lse, int32_t* top_tokens, float* top_logprobs, void* workspace, size_t workspace_bytes,
                 void* stream);

#ifdef __cplusplus
}
#endif
#endif /* QQQ_SERVE_H_ */
