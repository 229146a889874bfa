// Loads and stores past the caches (PAST), for data that no cache holds or need hold.
#pragma once

#include "qqq_internal.h"

namespace qqq {

// A call of the norm, the activation or the cache (append, read) whose operands are more than the last-level cache reads its inputs past it: none of them can be
// there still, and what it writes then is, for the call that reads that.  (Attention over few rows has a rule of its own, by how it splits the keys: see plan_of.)
constexpr int64_t kLastCacheBytes = 256 << 20;

typedef uint32_t u2v __attribute__((ext_vector_type(2)));
typedef uint32_t u4v __attribute__((ext_vector_type(4)));

template <bool PAST>
__device__ __forceinline__ uint4 load16(const void* from) {
  const u4v* at = reinterpret_cast<const u4v*>(from);
  u4v v;
  if constexpr (PAST) v = __builtin_nontemporal_load(at);
  else v = *at;
  return make_uint4(v.x, v.y, v.z, v.w);
}
template <bool PAST>
__device__ __forceinline__ uint2 load8(const void* from) {
  const u2v* at = reinterpret_cast<const u2v*>(from);
  u2v v;
  if constexpr (PAST) v = __builtin_nontemporal_load(at);
  else v = *at;
  return make_uint2(v.x, v.y);
}
template <bool PAST>
__device__ __forceinline__ void store16(void* to, uint4 x) {
  const u4v v = {x.x, x.y, x.z, x.w};
  if constexpr (PAST) __builtin_nontemporal_store(v, reinterpret_cast<u4v*>(to));
  else *reinterpret_cast<u4v*>(to) = v;
}

}  // namespace qqq
