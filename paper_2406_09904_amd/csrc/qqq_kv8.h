// The 8-bit key/value cache as the kernels see it (layout: qqq_layer.h).
#pragma once

#include "qqq_internal.h"
#include "qqq_layer.h"

namespace qqq {

struct Kv8 {
  const uint8_t *k_codes, *v_codes;
  const float *k_scale, *v_scale;
  const uint16_t *k_tail, *v_tail;  // fp16 bits
  const int32_t *table, *kv_len, *cu, *slots;
  int64_t table_stride, pages;
  int32_t nslots, heads, max_new, max_len;
  int64_t tokens;
};

// One sequence of a step, within the bounds that the host knows whatever the device tensors hold.
struct Kv8Seq {
  int64_t row;  // of its first new token
  int n, len;   // new tokens, tokens in all
  int slot;
};
__device__ __forceinline__ Kv8Seq kv8_sequence(const Kv8& c, int b) {
  Kv8Seq s;
  const int from = c.cu[b], to = c.cu[b + 1];
  s.row = from;
  s.n = to > from ? (int)min((uint32_t)to - (uint32_t)from, (uint32_t)c.max_new) : 0;
  s.len = min(max(c.kv_len[b], 0), c.max_len);
  s.slot = c.slots ? c.slots[b] : b;
  return s;
}
__device__ __forceinline__ bool kv8_has_page(const Kv8& c, int page) { return (uint32_t)page < (uint32_t)c.pages; }
// for reads: one that exists in the place of one that does not
__device__ __forceinline__ uint32_t kv8_page(const Kv8& c, int page) { return min((uint32_t)page, (uint32_t)c.pages - 1u); }
// a page's place for a head, in units of P * D values and of scales (pages * heads is below 2^31)
__device__ __forceinline__ int64_t kv8_block(const Kv8& c, int page, int head) { return kv8_page(c, page) * (uint32_t)c.heads + (uint32_t)head; }
__device__ __forceinline__ int kv8_slot(const Kv8& c, int slot) { return (uint32_t)slot < (uint32_t)c.nslots ? slot : c.nslots - 1; }

// Four codes (offset binary bytes) as fp16 code values: byte u under the exponent of 1024 is 1024 + u, less 1152 it is u - 128, exactly.
__device__ __forceinline__ uint2 codes4_to_halves(uint32_t u) {
  const h2 off = {(_Float16)1152.0f, (_Float16)1152.0f};
  // v_perm_b32: selector bytes 0-3 pick from the second source, 4-7 from the first
  const uint32_t lo = __builtin_amdgcn_perm(0x64646464u, u, 0x04010400u), hi = __builtin_amdgcn_perm(0x64646464u, u, 0x04030402u);
  return make_uint2(as_u32(as_h2(lo) - off), as_u32(as_h2(hi) - off));
}

}  // namespace qqq
