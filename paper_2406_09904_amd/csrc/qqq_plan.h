// What the kernels of a step's tables are given (qqq_kv8_plan.hip; the sessions' layout is in qqq_serve.h).
#pragma once

#include "qqq_internal.h"

namespace qqq {

struct PlanArgs {
  int32_t* pages;
  int64_t pages_stride;
  const int32_t *held, *free_pages, *free_count;
  int32_t *held_after, *free_count_after, *free_out;
  const int32_t *ids, *new_tokens;
  int32_t *table, *kv_len, *cu, *sequence, *positions, *lacking;
  int64_t table_stride;
  int32_t* top;  // workspace: what is left of the stack at each sequence's turn
  int32_t pool, sessions, columns, sequences, max_new, max_len, tokens, shift;
  bool same_table;  // the batch's table is the sessions' own
};

constexpr int64_t kPlanSmall = 8192;

size_t kv8_plan_bytes(const PlanArgs& p);
int launch_kv8_plan(const PlanArgs& p, hipStream_t st);
int launch_kv8_release(const PlanArgs& p, hipStream_t st);

}  // namespace qqq
