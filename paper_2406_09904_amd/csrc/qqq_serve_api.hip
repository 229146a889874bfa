// C-ABI entry points of qqq_serve.h: argument validation (host code only).
#include "qqq_plan.h"
#include "qqq_serve.h"
#include "qqq_w8a8.h"

namespace qqq {

size_t logprobs_bytes(int64_t M, int64_t V, int type);
int launch_logprobs(const void* logits, int64_t ld, int type, int64_t M, int64_t V, const int32_t* tokens, int top, float* logprob, float* entropy,
                    float* lse, int32_t* top_tokens, float* top_logprobs, void* workspace, hipStream_t st);

namespace {

constexpr int64_t kMost = 1 << 30;      // tokens of a sequence, rows of a call, pages: places stay in 32 bits
constexpr int64_t kMostGroups = (1 << 24) - 1;  // workgroups of 256 threads: a launch takes fewer than 2^32 threads

bool aligned(const void* p, uintptr_t to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) == 0; }

int check_sessions(const char* name, const qqq_kv8_sessions* s) {
  if (!s) return set_error(QQQ_ERR_NULL, "%s: NULL struct", name);
  if ((s->page_tokens != 16 && s->page_tokens != 32 && s->page_tokens != 64) || s->sessions < 1 || s->columns < 0 || s->pages_stride < s->columns ||
      s->pool < 0 || s->pool > kMost)
    return set_error(QQQ_ERR_SHAPE, "%s: unsupported sessions: %d of %d page columns of stride %lld, pages of %d tokens, a stack of %lld", name, s->sessions,
                     s->columns, (long long)s->pages_stride, s->page_tokens, (long long)s->pool);
  return QQQ_OK;
}
int check_session_pointers(const char* name, const qqq_kv8_sessions* s) {
  if (!s->held || !s->held_after || !s->free_count || !s->free_count_after || (s->columns > 0 && !s->pages) || (s->pool > 0 && !s->free_pages))
    return set_error(QQQ_ERR_NULL, "%s: NULL pointer in a struct", name);
  if (!aligned(s->pages, 4) || !aligned(s->held, 4) || !aligned(s->held_after, 4) || !aligned(s->free_pages, 4) || !aligned(s->free_count, 4) ||
      !aligned(s->free_count_after, 4))
    return set_error(QQQ_ERR_SHAPE, "%s: misaligned pointer in a struct", name);
  return QQQ_OK;
}
int check_plan(const char* name, const qqq_kv8_sessions* s, const qqq_kv8_batch* b) {
  if (int rc = check_sessions(name, s)) return rc;
  if (!b) return set_error(QQQ_ERR_NULL, "%s: NULL struct", name);
  if (b->sequences < 0 || b->sequences > kMostGroups || b->max_new < 0 || b->max_new > kMost || b->max_len < 0 || b->max_len > kMost || b->columns < 0 || b->table_stride < b->columns ||
      b->max_len / s->page_tokens > b->columns || b->max_len / s->page_tokens > s->columns)
    return set_error(QQQ_ERR_SHAPE, "%s: unsupported batch: %d sequences, at most %d new of %d tokens, %d page columns of stride %lld (the sessions' table: %d)", name,
                     b->sequences, b->max_new, b->max_len, b->columns, (long long)b->table_stride, s->columns);
  if (!b->slots && b->sequences > s->sessions) return set_error(QQQ_ERR_SHAPE, "%s: %d sequences of %d sessions", name, b->sequences, s->sessions);
  return QQQ_OK;
}
PlanArgs session_args(const qqq_kv8_sessions* s) {
  PlanArgs p = {};
  p.pages = s->pages;
  p.pages_stride = s->pages_stride;
  p.held = s->held;
  p.free_pages = s->free_pages;
  p.free_count = s->free_count;
  p.held_after = s->held_after;
  p.free_count_after = s->free_count_after;
  p.free_out = s->free_pages;
  p.pool = (int32_t)s->pool;
  p.sessions = s->sessions;
  p.columns = s->columns;
  p.shift = s->page_tokens == 16 ? 4 : s->page_tokens == 32 ? 5 : 6;
  return p;
}
// The call's arguments but for the rows, which the workspace does not depend on
PlanArgs plan_args(const qqq_kv8_sessions* s, const qqq_kv8_batch* b) {
  PlanArgs p = session_args(s);
  p.ids = b->slots;
  p.table = const_cast<int32_t*>(b->page_table);
  p.table_stride = b->table_stride;
  p.kv_len = const_cast<int32_t*>(b->kv_len);
  p.cu = const_cast<int32_t*>(b->cu);
  p.sequences = b->sequences;
  p.max_new = b->max_new;
  p.max_len = b->max_len;
  p.same_table = b->page_table == s->pages;
  return p;
}

constexpr int64_t kMostK = 131072, kMostN = 1 << 24;  // 127 * 127 * K stays below 2^31

int check_product(const char* name, int64_t N, int64_t K) {
  if (N < 1 || N > kMostN || K < 128 || K % 128 != 0 || K > kMostK || N * K > 1ll << 35)
    return set_error(QQQ_ERR_SHAPE, "%s: unsupported N=%lld K=%lld (need 1 <= N <= 2^24, K%%128==0, 128 <= K <= 131072, N K <= 2^35)", name, (long long)N, (long long)K);
  return QQQ_OK;
}

int check_logits(const char* name, int64_t M, int64_t V, int type) {
  if (M < 0 || M > kMostGroups || V < 1 || V >= kMost) return set_error(QQQ_ERR_SHAPE, "%s: unsupported %lld rows of %lld logits", name, (long long)M, (long long)V);
  if (type != QQQ_LOGITS_FP16 && type != QQQ_LOGITS_FP32) return set_error(QQQ_ERR_SHAPE, "%s: logits of type %d", name, type);
  return QQQ_OK;
}

}  // namespace
}  // namespace qqq

using namespace qqq;

extern "C" {

size_t qqq_kv8_plan_workspace_bytes(const qqq_kv8_sessions* sessions, const qqq_kv8_batch* batch) {
  if (check_plan("qqq_kv8_plan_workspace_bytes", sessions, batch)) return 0;
  return kv8_plan_bytes(plan_args(sessions, batch));
}

int qqq_kv8_plan(const qqq_kv8_sessions* sessions, const qqq_kv8_batch* batch, const int32_t* new_tokens, int64_t tokens, int32_t* sequence,
                 int32_t* positions, int32_t* lacking, void* workspace, size_t workspace_bytes, void* stream) {
  const char* name = "qqq_kv8_plan";
  if (int rc = check_plan(name, sessions, batch)) return rc;
  if (tokens < 0 || tokens > kMost) return set_error(QQQ_ERR_SHAPE, "%s: %lld rows", name, (long long)tokens);
  if (int rc = check_session_pointers(name, sessions)) return rc;
  if (!batch->cu || (batch->sequences > 0 && (!batch->kv_len || !new_tokens || (!batch->page_table && batch->max_len >= sessions->page_tokens))))
    return set_error(QQQ_ERR_NULL, "%s: NULL pointer", name);
  if (!aligned(batch->page_table, 4) || !aligned(batch->kv_len, 4) || !aligned(batch->cu, 4) || !aligned(batch->slots, 4) || !aligned(new_tokens, 4) ||
      !aligned(sequence, 4) || !aligned(positions, 4) || !aligned(lacking, 4) || !aligned(workspace, 4))
    return set_error(QQQ_ERR_SHAPE, "%s: misaligned pointer", name);
  PlanArgs p = plan_args(sessions, batch);
  if (p.same_table && p.table && (p.ids || p.table_stride != p.pages_stride))
    return set_error(QQQ_ERR_SHAPE, "%s: the sessions' own table with %s", name, p.ids ? "slots" : "another stride");
  p.new_tokens = new_tokens;
  p.tokens = (int32_t)tokens;
  p.sequence = sequence;
  p.positions = positions;
  p.lacking = lacking;
  p.top = static_cast<int32_t*>(workspace);
  const size_t need = kv8_plan_bytes(p);
  if (need && (!workspace || workspace_bytes < need))
    return set_error(QQQ_ERR_WORKSPACE, "%s: workspace %zu bytes < %zu needed", name, workspace ? workspace_bytes : 0, need);
  route_reset();
  return launch_kv8_plan(p, (hipStream_t)stream);
}

int qqq_kv8_release(const qqq_kv8_sessions* sessions, const int32_t* ids, int64_t count, void* stream) {
  const char* name = "qqq_kv8_release";
  if (int rc = check_sessions(name, sessions)) return rc;
  if (count < 0 || count > kMost || (!ids && count > sessions->sessions)) return set_error(QQQ_ERR_SHAPE, "%s: %lld of %d sessions", name, (long long)count, sessions->sessions);
  if (count == 0) return QQQ_OK;
  if (int rc = check_session_pointers(name, sessions)) return rc;
  if (!aligned(ids, 4)) return set_error(QQQ_ERR_SHAPE, "%s: misaligned pointer", name);
  if (sessions->held != sessions->held_after || sessions->free_count != sessions->free_count_after)
    return set_error(QQQ_ERR_SHAPE, "%s: not in place", name);
  PlanArgs p = session_args(sessions);
  p.ids = ids;
  p.sequences = (int32_t)count;
  route_reset();
  return launch_kv8_release(p, (hipStream_t)stream);
}

size_t qqq_packed_w8_bytes(int64_t N, int64_t K) { return check_product("qqq_packed_w8_bytes", N, K) ? 0 : (size_t)((N + 15) / 16 * 16 * K); }

int qqq_pack_w8(const int8_t* w_codes, int64_t N, int64_t K, int64_t ldw, void* w_packed, void* stream) {
  const char* name = "qqq_pack_w8";
  if (int rc = check_product(name, N, K)) return rc;
  if (ldw < K || ldw % 16) return set_error(QQQ_ERR_SHAPE, "%s: row stride %lld for %lld codes", name, (long long)ldw, (long long)K);
  if (!w_codes || !w_packed) return set_error(QQQ_ERR_NULL, "%s: NULL pointer", name);
  if (!aligned(w_codes, 16) || !aligned(w_packed, 16) || w_codes == w_packed) return set_error(QQQ_ERR_SHAPE, "%s: misaligned pointer, or in place", name);
  route_reset();
  return launch_pack_w8(w_codes, N, K, ldw, static_cast<int8_t*>(w_packed), (hipStream_t)stream);
}

int qqq_unpack_w8(const void* w_packed, int64_t N, int64_t K, int8_t* w_codes, void* stream) {
  const char* name = "qqq_unpack_w8";
  if (int rc = check_product(name, N, K)) return rc;
  if (!w_codes || !w_packed) return set_error(QQQ_ERR_NULL, "%s: NULL pointer", name);
  if (!aligned(w_codes, 16) || !aligned(w_packed, 16) || w_codes == w_packed) return set_error(QQQ_ERR_SHAPE, "%s: misaligned pointer, or in place", name);
  route_reset();
  return launch_unpack_w8(static_cast<const int8_t*>(w_packed), N, K, w_codes, (hipStream_t)stream);
}

size_t qqq_gemm_w8a8_workspace_bytes(int64_t M, int64_t N, int64_t K) {
  if (check_product("qqq_gemm_w8a8_workspace_bytes", N, K) || M < 1 || M > kMost) return 0;
  const W8Plan plan = w8_plan(M, N, K);
  return plan.k_splits > 1 ? (size_t)plan.k_splits * M * N * sizeof(int32_t) : 0;
}

int qqq_gemm_w8a8(const int8_t* a_q, const float* s_a, const void* w_packed, const float* s_w, void* y, int y_type, int64_t ldy, int32_t* acc_out, int64_t M,
                  int64_t N, int64_t K, void* workspace, size_t workspace_bytes, void* stream) {
  const char* name = "qqq_gemm_w8a8";
  if (int rc = check_product(name, N, K)) return rc;
  if (M < 0 || M > kMost) return set_error(QQQ_ERR_SHAPE, "%s: M=%lld", name, (long long)M);
  if (y_type != QQQ_OUT_FP16 && y_type != QQQ_OUT_FP32) return set_error(QQQ_ERR_SHAPE, "%s: outputs of type %d", name, y_type);
  if (ldy < N) return set_error(QQQ_ERR_SHAPE, "%s: row stride %lld for %lld outputs", name, (long long)ldy, (long long)N);
  if (M == 0) return QQQ_OK;
  if (!a_q || !s_a || !w_packed || !s_w || !y) return set_error(QQQ_ERR_NULL, "%s: NULL pointer", name);
  const int size = y_type == QQQ_OUT_FP32 ? 4 : 2;
  if (!aligned(a_q, 16) || !aligned(w_packed, 16) || !aligned(workspace, 16) || !aligned(s_a, 4) || !aligned(s_w, 4) || !aligned(acc_out, 4) || !aligned(y, size))
    return set_error(QQQ_ERR_SHAPE, "%s: misaligned pointer", name);
  const W8Plan plan = w8_plan(M, N, K);
  const size_t need = plan.k_splits > 1 ? (size_t)plan.k_splits * M * N * sizeof(int32_t) : 0;
  if (need && (!workspace || workspace_bytes < need))
    return set_error(QQQ_ERR_WORKSPACE, "%s: workspace %zu bytes < %zu needed", name, workspace ? workspace_bytes : 0, need);
  W8Params p = {};
  p.a_q = a_q;
  p.s_a = s_a;
  p.w = static_cast<const int8_t*>(w_packed);
  p.s_w = s_w;
  p.y = y;
  p.ldy = ldy;
  p.acc_out = acc_out;
  p.part = static_cast<int32_t*>(workspace);
  p.M = (int)M;
  p.N = (int)N;
  p.K = (int)K;
  p.k_splits = plan.k_splits;
  p.f32 = y_type == QQQ_OUT_FP32;
  route_reset();
  if (int rc = plan.shape == kW8Few ? launch_w8_few(p, (hipStream_t)stream) : launch_w8_tiles(p, plan.shape, (hipStream_t)stream)) return rc;
  return plan.k_splits > 1 ? launch_w8_sum(p, (hipStream_t)stream) : QQQ_OK;
}

size_t qqq_logprobs_workspace_bytes(int64_t M, int64_t V, int type) {
  return check_logits("qqq_logprobs_workspace_bytes", M, V, type) || M == 0 ? 0 : logprobs_bytes(M, V, type);
}

int qqq_logprobs(const void* logits, int64_t ld, int type, int64_t M, int64_t V, const int32_t* tokens, int top, float* logprob, float* entropy, float* lse,
                 int32_t* top_tokens, float* top_logprobs, void* workspace, size_t workspace_bytes, void* stream) {
  const char* name = "qqq_logprobs";
  if (int rc = check_logits(name, M, V, type)) return rc;
  if (ld < V) return set_error(QQQ_ERR_SHAPE, "%s: row stride %lld for %lld logits", name, (long long)ld, (long long)V);
  if (top < 0 || top > QQQ_MAX_TOP) return set_error(QQQ_ERR_SHAPE, "%s: the largest %d logits, %d at most", name, top, QQQ_MAX_TOP);
  if (M == 0) return QQQ_OK;
  if (!logits || (top > 0 && (!top_tokens || !top_logprobs)) || (logprob && !tokens)) return set_error(QQQ_ERR_NULL, "%s: NULL pointer", name);
  if (tokens && !logprob) return set_error(QQQ_ERR_NULL, "%s: tokens without their log probabilities", name);
  if (!aligned(logits, type == QQQ_LOGITS_FP32 ? 4 : 2) || !aligned(tokens, 4) || !aligned(logprob, 4) || !aligned(entropy, 4) || !aligned(lse, 4) ||
      !aligned(top_tokens, 4) || !aligned(top_logprobs, 4) || !aligned(workspace, 16))
    return set_error(QQQ_ERR_SHAPE, "%s: misaligned pointer", name);
  const size_t need = logprobs_bytes(M, V, type);
  if (need && (!workspace || workspace_bytes < need))
    return set_error(QQQ_ERR_WORKSPACE, "%s: workspace %zu bytes < %zu needed", name, workspace ? workspace_bytes : 0, need);
  route_reset();
  return launch_logprobs(logits, ld, type, M, V, tokens, top, logprob, entropy, lse, top_tokens, top_logprobs, workspace, (hipStream_t)stream);
}

}  // extern "C"
