// qqq_kv8_append, qqq_kv8_read: new keys and values into the 8-bit paged cache, and out of it again.
//
// One workgroup for a page of one head of keys or of values.  Append: the page's fp16 values (the open page's from the tail slot, the
// others from the new rows) are read once into registers, |max| is reduced over the workgroup, and codes = 128 + rne(x / s) are written.
// Values are turned token-minor on the way, through LDS.
#include "qqq_kv8.h"

namespace qqq {

namespace {

constexpr int kThreads = 256;

__device__ __forceinline__ uint16_t finite_half(uint32_t h) {  // NaN as 0, an infinity as the largest value of its sign
  const uint32_t mag = h & 0x7FFFu;
  return (uint16_t)(mag < 0x7C00u ? h : mag > 0x7C00u ? 0u : (h & 0x8000u) | 0x7BFFu);
}
__device__ __forceinline__ uint4 finite_halves(uint4 v) {
  if (absmax_bits(v, 0) >= 0x7C00u) {
    auto both = [](uint32_t w) { return (uint32_t)finite_half(w & 0xFFFFu) | (uint32_t)finite_half(w >> 16) << 16; };
    v = make_uint4(both(v.x), both(v.y), both(v.z), both(v.w));
  }
  return v;
}

template <int T>
__device__ __forceinline__ uint32_t block_max_bits(uint32_t v, uint32_t* smem) {
  v = wave_max_u32(v);
  if ((threadIdx.x & 63) == 0) smem[threadIdx.x >> 6] = v;
  __syncthreads();
  uint32_t r = 0;
#pragma unroll
  for (int i = 0; i < T / 64; ++i) r = max(r, smem[i]);
  return r;
}

// A page turned in LDS: value (d, t) lies in row d, whose 16-byte chunks are permuted by d so that neither eight channels of a token
// nor eight tokens of a channel meet in the same banks.
template <int P>
__device__ __forceinline__ int turned(int d, int t) {
  return d * P + ((((t >> 3) ^ (d >> 3)) & (P / 8 - 1)) << 3) + (t & 7);
}

struct AppendParams {
  Kv8 c;
  const uint16_t *k, *v;
  int64_t k_token, k_head, v_token, v_head;
  int units;  // pages a sequence may touch
};

template <int D, int P>
__global__ __launch_bounds__(kThreads) void kv8_append_kernel(const AppendParams p) {
  constexpr int NV = P * D / 8, VPT = (NV + kThreads - 1) / kThreads;  // vectors of 8 values of a page; of a thread
  __shared__ uint32_t smem[kThreads / 64];
  __shared__ uint16_t page_lds[P * D];
  const Kv8& c = p.c;
  const int unit = blockIdx.x % p.units, head = (blockIdx.x / p.units) % c.heads;
  const bool values = blockIdx.y != 0;
  const int b = blockIdx.x / p.units / c.heads;
  Kv8Seq s = kv8_sequence(c, b);
  if (s.n > s.len) {  // tokens before position 0 do not exist
    s.row += s.n - s.len;
    s.n = s.len;
  }
  const int start = s.len - s.n, closed = s.len / P, page = start / P + unit;
  if (s.n == 0 || s.slot < 0 || s.slot >= c.nslots) return;
  const uint16_t* in = values ? p.v + head * p.v_head : p.k + head * p.k_head;
  const int64_t token_stride = values ? p.v_token : p.k_token;
  uint16_t* tail = const_cast<uint16_t*>(values ? c.v_tail : c.k_tail) + ((int64_t)s.slot * c.heads + head) * (P * D);
  auto new_values = [&](int pos, int d8) {  // eight values of a new token; a row outside the tensor reads as zeros
    const int64_t row = s.row + (pos - start);
    return row >= 0 && row < c.tokens ? finite_halves(*reinterpret_cast<const uint4*>(in + row * token_stride + d8 * 8)) : make_uint4(0, 0, 0, 0);
  };

  if (page < closed) {
    uint4 v[VPT];
    uint32_t amax_bits = 0;
    if (!values) {
#pragma unroll
      for (int j = 0; j < VPT; ++j) {
        const int i = threadIdx.x + kThreads * j, t = i / (D / 8), d8 = i % (D / 8), pos = page * P + t;
        v[j] = make_uint4(0, 0, 0, 0);
        if (i < NV) v[j] = pos < start ? reinterpret_cast<const uint4*>(tail)[i] : new_values(pos, d8);
        amax_bits = absmax_bits(v[j], amax_bits);
      }
    } else {
      const int held = max(0, start - page * P);  // tokens of the page that its tail slot holds, token-minor already
#pragma unroll
      for (int j = 0; j < VPT; ++j) {
        const int i = threadIdx.x + kThreads * j, t = i / (D / 8), d8 = i % (D / 8);
        if (i < NV && t >= held) {
          const uint4 w = new_values(page * P + t, d8);
          const uint32_t ws[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
          for (int e = 0; e < 8; ++e) page_lds[turned<P>(d8 * 8 + e, t)] = (uint16_t)(e & 1 ? ws[e >> 1] >> 16 : ws[e >> 1]);
        }
      }
      for (int i = threadIdx.x; i < D * held; i += kThreads) {
        const int d = i / held, t = i % held;
        page_lds[turned<P>(d, t)] = tail[d * P + t];
      }
      __syncthreads();
#pragma unroll
      for (int j = 0; j < VPT; ++j) {
        const int i = threadIdx.x + kThreads * j;
        v[j] = make_uint4(0, 0, 0, 0);
        if (i < NV) v[j] = *reinterpret_cast<const uint4*>(&page_lds[turned<P>(i / (P / 8), i % (P / 8) * 8)]);
        amax_bits = absmax_bits(v[j], amax_bits);
      }
    }
    amax_bits = block_max_bits<kThreads>(amax_bits, smem);
    const float amax = half_bits_to_float(amax_bits), scale = amax / 127.0f, inv = reciprocal_near(scale);
    const int id = c.table[b * c.table_stride + page];
    if (kv8_has_page(c, id)) {
      const int64_t at = (int64_t)id * c.heads + head;
      uint2* codes = reinterpret_cast<uint2*>(const_cast<uint8_t*>(values ? c.v_codes : c.k_codes)) + at * NV;
      if (threadIdx.x == 0) const_cast<float*>(values ? c.v_scale : c.k_scale)[at] = scale;
#pragma unroll
      for (int j = 0; j < VPT; ++j) {
        const int i = threadIdx.x + kThreads * j;
        uint2 o = make_uint2(0, 0);
        if (amax_bits != 0) o = quant8_act(v[j], scale, inv);
        if (i < NV) codes[i] = make_uint2(o.x ^ 0x80808080u, o.y ^ 0x80808080u);
      }
    }
    __syncthreads();  // the tail slot has been read: its first tokens may be written over below
  }
  // the new tokens of the page that stays open: by the workgroup of the sequence's first page, which is the one that reads the tail slot
  if (unit != 0 || closed * P >= s.len) return;
  const int from = max(start, closed * P), count = s.len - from;
  for (int i = threadIdx.x; i < count * (D / 8); i += kThreads) {
    const int pos = from + i / (D / 8), t = pos - closed * P, d8 = i % (D / 8);
    const uint4 w = new_values(pos, d8);
    if (!values) {
      reinterpret_cast<uint4*>(tail)[t * (D / 8) + d8] = w;
    } else {
      const uint32_t ws[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
      for (int e = 0; e < 8; ++e) tail[(d8 * 8 + e) * P + t] = (uint16_t)(e & 1 ? ws[e >> 1] >> 16 : ws[e >> 1]);
    }
  }
}

struct ReadParams {
  Kv8 c;
  uint16_t *k, *v;  // [tokens, heads, D]
  int units;
};

__device__ __forceinline__ uint4 scaled_halves(uint2 codes, float s) {
  const uint2 a = codes4_to_halves(codes.x), b = codes4_to_halves(codes.y);
  auto mul = [&](uint32_t w) {
    const h2 x = as_h2(w);
    return as_u32(h2{(_Float16)((float)x[0] * s), (_Float16)((float)x[1] * s)});
  };
  return make_uint4(mul(a.x), mul(a.y), mul(b.x), mul(b.y));
}

template <int D, int P>
__global__ __launch_bounds__(kThreads) void kv8_read_kernel(const ReadParams p) {
  constexpr int NV = P * D / 8, VPT = (NV + kThreads - 1) / kThreads;
  __shared__ uint16_t page_lds[P * D];
  const Kv8& c = p.c;
  const int unit = blockIdx.x % p.units, head = (blockIdx.x / p.units) % c.heads;
  const bool values = blockIdx.y != 0;
  const int b = blockIdx.x / p.units / c.heads;
  Kv8Seq s = kv8_sequence(c, b);
  if (s.n > s.len) {
    s.row += s.n - s.len;
    s.n = s.len;
  }
  const int start = s.len - s.n, closed = s.len / P, page = start / P + unit;
  if (s.n == 0 || page * P >= s.len) return;
  const bool is_tail = page >= closed;
  const int64_t at = is_tail ? (int64_t)kv8_slot(c, s.slot) * c.heads + head : kv8_block(c, c.table[b * c.table_stride + page], head);
  uint16_t* out = (values ? p.v : p.k) + head * D;
  auto put = [&](int t, int d8, uint4 w) {
    const int pos = page * P + t;
    const int64_t row = s.row + (pos - start);
    if (pos >= start && pos < s.len && row >= 0 && row < c.tokens) *reinterpret_cast<uint4*>(out + row * c.heads * D + d8 * 8) = w;
  };
  uint4 v[VPT];
  if (is_tail) {
    const uint4* from = reinterpret_cast<const uint4*>(values ? c.v_tail : c.k_tail) + at * NV;
#pragma unroll
    for (int j = 0; j < VPT; ++j) {
      const int i = threadIdx.x + kThreads * j;
      if (i < NV) v[j] = from[i];
    }
  } else {
    const uint2* from = reinterpret_cast<const uint2*>(values ? c.v_codes : c.k_codes) + at * NV;
    const float scale = (values ? c.v_scale : c.k_scale)[at];
#pragma unroll
    for (int j = 0; j < VPT; ++j) {
      const int i = threadIdx.x + kThreads * j;
      if (i < NV) v[j] = scaled_halves(from[i], scale);
    }
  }
  if (!values) {
#pragma unroll
    for (int j = 0; j < VPT; ++j) {
      const int i = threadIdx.x + kThreads * j;
      if (i < NV) put(i / (D / 8), i % (D / 8), v[j]);
    }
  } else {
#pragma unroll
    for (int j = 0; j < VPT; ++j) {
      const int i = threadIdx.x + kThreads * j;
      if (i < NV) *reinterpret_cast<uint4*>(&page_lds[turned<P>(i / (P / 8), i % (P / 8) * 8)]) = v[j];
    }
    __syncthreads();
#pragma unroll
    for (int j = 0; j < VPT; ++j) {
      const int i = threadIdx.x + kThreads * j, t = i / (D / 8), d8 = i % (D / 8);
      if (i < NV) {
        uint32_t w[4];
#pragma unroll
        for (int e = 0; e < 4; ++e)
          w[e] = (uint32_t)page_lds[turned<P>(d8 * 8 + 2 * e, t)] | (uint32_t)page_lds[turned<P>(d8 * 8 + 2 * e + 1, t)] << 16;
        put(t, d8, make_uint4(w[0], w[1], w[2], w[3]));
      }
    }
  }
}

template <typename Params, typename Kernel>
int launch_pages(Kernel kernel, const Params& p, int sequences, const char* name, hipStream_t st) {
  const int64_t blocks = (int64_t)p.units * p.c.heads * sequences;
  if (blocks > 0x7FFFFFFF) return set_error(QQQ_ERR_SHAPE, "%s: %lld workgroups", name, (long long)blocks);
  hipLaunchKernelGGL(kernel, dim3((unsigned)blocks, 2), dim3(kThreads), 0, st, p);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return set_error(QQQ_ERR_HIP, "%s launch: %s", name, hipGetErrorString(e));
  route_note("%s", name);
  return QQQ_OK;
}

// pages that max_new tokens in a row can touch
int units_of(int max_new, int P) { return (max_new + P - 2) / P + 1; }

}  // namespace

#define QQQ_KV8_SHAPES(F)                                                                                                        \
  if (D == 64) { if (P == 16) F(64, 16); if (P == 32) F(64, 32); F(64, 64); }                                                    \
  if (D == 128) { if (P == 16) F(128, 16); if (P == 32) F(128, 32); F(128, 64); }                                                \
  if (P == 16) F(256, 16);                                                                                                       \
  if (P == 32) F(256, 32);                                                                                                       \
  F(256, 64);

int launch_kv8_append(const Kv8& c, int D, int P, int sequences, const void* k, int64_t k_token, int64_t k_head, const void* v,
                      int64_t v_token, int64_t v_head, hipStream_t st) {
  const AppendParams p = {c, (const uint16_t*)k, (const uint16_t*)v, k_token, k_head, v_token, v_head, units_of(c.max_new, P)};
#define QQQ_APPEND(D_, P_) return launch_pages(kv8_append_kernel<D_, P_>, p, sequences, "kv8_append", st)
  QQQ_KV8_SHAPES(QQQ_APPEND)
#undef QQQ_APPEND
}

int launch_kv8_read(const Kv8& c, int D, int P, int sequences, void* k, void* v, hipStream_t st) {
  const ReadParams p = {c, (uint16_t*)k, (uint16_t*)v, units_of(c.max_new, P)};
#define QQQ_READ(D_, P_) return launch_pages(kv8_read_kernel<D_, P_>, p, sequences, "kv8_read", st)
  QQQ_KV8_SHAPES(QQQ_READ)
#undef QQQ_READ
}

}  // namespace qqq
