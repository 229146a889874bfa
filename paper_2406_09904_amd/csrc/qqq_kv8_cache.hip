// qqq_kv8_append, qqq_kv8_read: new keys and values into the 8-bit paged cache, and out of it again.
//
// Many pages: one wave for a page of one head of keys or of values, four such waves a workgroup, nothing shared between them: what bounds
// both calls then is how many bytes are on their way, so a wave requests its whole page at once and never waits for another.  Few pages (a
// step of single tokens): the workgroup's four waves share a page, since a call lasts as long as its slowest page.  Append: the page's fp16
// values (the open page's from the tail slot, the others from the new rows) are read once into registers, |max| is reduced over the
// wave, and codes = 128 + rne(x / s) are written.  A lane holds four tokens of eight channels; values are turned token-minor as codes, in
// registers (4 x 4 bytes) and through LDS.  12000 tokens of 40 heads of 128 in pages of 16: appended (376 MB) in 79 us, 4.7 TB/s, read back (445 MB)
// in 62, 7.1 TB/s with the codes still in the last-level cache; a token each of 64 sequences, 8 heads, pages of 64: 6.1 us.
#include "qqq_kv8.h"
#include "qqq_past.h"

namespace qqq {

namespace {

constexpr int kWaves = 4;

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

// Four tokens' eight bytes (channels) as eight dwords of four tokens, and back.
__device__ __forceinline__ void turn4(uint32_t a, uint32_t b, uint32_t c, uint32_t d, uint32_t* out) {  // 4 x 4 bytes
  // v_perm_b32: selector bytes 0-3 pick from the second source, 4-7 from the first
  const uint32_t ab0 = __builtin_amdgcn_perm(b, a, 0x05010400u), ab1 = __builtin_amdgcn_perm(b, a, 0x07030602u);
  const uint32_t cd0 = __builtin_amdgcn_perm(d, c, 0x05010400u), cd1 = __builtin_amdgcn_perm(d, c, 0x07030602u);
  out[0] = __builtin_amdgcn_perm(cd0, ab0, 0x05040100u);
  out[1] = __builtin_amdgcn_perm(cd0, ab0, 0x07060302u);
  out[2] = __builtin_amdgcn_perm(cd1, ab1, 0x05040100u);
  out[3] = __builtin_amdgcn_perm(cd1, ab1, 0x07060302u);
}

// A page of a head as the lanes of a wave hold it: quad i = 64 j + lane is tokens 4 (i / (D / 8)) .. + 3 of channels 8 (i % (D / 8)) .. + 7.
// (C waves to a page: i = 64 C j + ...)
template <int D, int P, int C>
struct PageShape {
  static constexpr int kStep = 64 * C, kQuads = P / 4 * (D / 8), kPerLane = (kQuads + kStep - 1) / kStep, kBytes = P * D, kRow = P + 4;  // (a row of LDS: 4 bytes over)
  static constexpr int kVectors = (kBytes / 16 + kStep - 1) / kStep;  // of 16 codes, of a lane
};

// Of a tail slot's values [D][P]: four tokens from t on of eight channels from d on, a vector of channels each.
template <int P>
__device__ __forceinline__ void tail_quad(const uint16_t* tail, int d, int t, uint4* v) {
  uint2 w[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) w[e] = *reinterpret_cast<const uint2*>(tail + (d + e) * P + t);
  auto pair = [](uint32_t a, uint32_t b, bool upper) { return upper ? __builtin_amdgcn_perm(b, a, 0x07060302u) : __builtin_amdgcn_perm(b, a, 0x05040100u); };
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    uint32_t o[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) o[e] = k < 2 ? pair(w[2 * e].x, w[2 * e + 1].x, k & 1) : pair(w[2 * e].y, w[2 * e + 1].y, k & 1);
    v[k] = make_uint4(o[0], o[1], o[2], o[3]);
  }
}

struct PageOf {  // a wave's work
  int unit, head, b;
  bool values, there;
};
template <int C>
__device__ __forceinline__ PageOf page_of_wave(const Kv8& c, int units, int sequences) {
  const int64_t id = C == 1 ? (int64_t)blockIdx.x * kWaves + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) : blockIdx.x;
  PageOf w;
  w.head = (int)(id % c.heads);
  w.unit = (int)(id / c.heads % units);
  const int64_t b = id / c.heads / units;
  w.there = b < sequences;
  w.b = w.there ? (int)b : 0;
  w.values = blockIdx.y != 0;
  return w;
}

// Between writing a page's codes to LDS and reading them.
template <int C>
__device__ __forceinline__ void page_barrier() {
  if constexpr (C > 1) {
    __syncthreads();
  } else {
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
  }
}

struct AppendParams {
  Kv8 c;
  const uint16_t *k, *v;
  int64_t k_token, k_head, v_token, v_head;
  int units, sequences;  // pages a sequence may touch
};

template <int D, int P, int C, bool PAST>
__global__ __launch_bounds__(64 * kWaves) void kv8_append_kernel(const AppendParams p) {
  using S = PageShape<D, P, C>;
  __shared__ uint32_t turned[kWaves / C][D * S::kRow / 4];
  const Kv8& c = p.c;
  const PageOf w = page_of_wave<C>(c, p.units, p.sequences);
  if (!w.there) return;
  Kv8Seq s = kv8_sequence(c, w.b);
  if (s.n > s.len) {  // tokens before position 0 do not exist
    s.row += s.n - s.len;
    s.n = s.len;
  }
  const int lane = C == 1 ? threadIdx.x & 63 : threadIdx.x;
  const int start = s.len - s.n, closed = s.len / P, page = start / P + w.unit;
  if (s.n == 0 || s.slot < 0 || s.slot >= c.nslots) return;
  const uint16_t* in = w.values ? p.v + w.head * p.v_head : p.k + w.head * p.k_head;
  const int64_t token_stride = w.values ? p.v_token : p.k_token;
  uint16_t* tail = const_cast<uint16_t*>(w.values ? c.v_tail : c.k_tail) + ((int64_t)s.slot * c.heads + w.head) * (P * D);
  auto new_values = [&](int pos, int d8) {  // eight values of a new token as they came; a row outside the tensor reads as zeros
    const int64_t row = s.row + (pos - start);
    return row >= 0 && row < c.tokens ? load16<PAST>(in + row * token_stride + d8 * 8) : make_uint4(0, 0, 0, 0);
  };

  if (page < closed) {
    const int id = c.table[w.b * c.table_stride + page];
    uint4 v[S::kPerLane][4];
#pragma unroll
    for (int j = 0; j < S::kPerLane; ++j) {
      const int i = lane + S::kStep * j, t = i / (D / 8) * 4, d8 = i % (D / 8), pos = page * P + t;
#pragma unroll
      for (int k = 0; k < 4; ++k) v[j][k] = make_uint4(0, 0, 0, 0);
      if (i >= S::kQuads) continue;
      if (pos < start) {  // (the sequence's first page only)
        if (w.values) {
          tail_quad<P>(tail, d8 * 8, t, v[j]);
        } else {
#pragma unroll
          for (int k = 0; k < 4; ++k) v[j][k] = reinterpret_cast<const uint4*>(tail)[(t + k) * (D / 8) + d8];
        }
      }
#pragma unroll
      for (int k = 0; k < 4; ++k)
        if (pos + k >= start) v[j][k] = new_values(pos + k, d8);
    }
    uint32_t amax_bits = 0;
#pragma unroll
    for (int j = 0; j < S::kPerLane; ++j)
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        v[j][k] = finite_halves(v[j][k]);
        amax_bits = absmax_bits(v[j][k], amax_bits);
      }
    amax_bits = wave_max_u32(amax_bits);
    if constexpr (C > 1) {
      __shared__ uint32_t most[kWaves];
      if ((threadIdx.x & 63) == 0) most[threadIdx.x >> 6] = amax_bits;
      __syncthreads();  // (and all of the tail slot that this page needs has been read)
#pragma unroll
      for (int i = 0; i < kWaves; ++i) amax_bits = max(amax_bits, most[i]);
    }
    const float amax = half_bits_to_float(amax_bits), scale = amax / 127.0f, inv = reciprocal_near(scale);
    if (kv8_has_page(c, id)) {
      const int64_t at = kv8_block(c, id, w.head);
      if (lane == 0) const_cast<float*>(w.values ? c.v_scale : c.k_scale)[at] = scale;
      uint8_t* codes = const_cast<uint8_t*>(w.values ? c.v_codes : c.k_codes) + at * S::kBytes;
      uint32_t* lds = turned[C == 1 ? threadIdx.x >> 6 : 0];
#pragma unroll
      for (int j = 0; j < S::kPerLane; ++j) {
        const int i = lane + S::kStep * j, t = i / (D / 8) * 4, d8 = i % (D / 8);
        if (i >= S::kQuads) continue;
        uint2 q[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          q[k] = make_uint2(0, 0);
          if (amax_bits != 0) q[k] = quant8_act(v[j][k], scale, inv);
          q[k] = make_uint2(q[k].x ^ 0x80808080u, q[k].y ^ 0x80808080u);
          if (!w.values) reinterpret_cast<uint2*>(codes)[(t + k) * (D / 8) + d8] = q[k];
        }
        if (w.values) {
          uint32_t o[8];
          turn4(q[0].x, q[1].x, q[2].x, q[3].x, o);
          turn4(q[0].y, q[1].y, q[2].y, q[3].y, o + 4);
#pragma unroll
          for (int e = 0; e < 8; ++e) lds[((d8 * 8 + e) * S::kRow + t) / 4] = o[e];
        }
      }
      if (w.values) {
        page_barrier<C>();
#pragma unroll
        for (int j = 0; j < S::kVectors; ++j) {
          const int i = lane + S::kStep * j, d = i / (P / 16), t = i % (P / 16) * 16;
          if (i >= S::kBytes / 16) continue;
          const uint32_t* from = &lds[(d * S::kRow + t) / 4];
          reinterpret_cast<uint4*>(codes)[i] = make_uint4(from[0], from[1], from[2], from[3]);
        }
      }
    }
  }
  // the new tokens of the page that stays open: by those of the sequence's first page, who have read the tail slot
  if (w.unit != 0 || closed * P >= s.len) return;
  const int from = max(start, closed * P), count = s.len - from;
  for (int i = lane; i < count * (D / 8); i += S::kStep) {
    const int pos = from + i / (D / 8), t = pos - closed * P, d8 = i % (D / 8);
    const uint4 x = finite_halves(new_values(pos, d8));
    if (!w.values) {
      reinterpret_cast<uint4*>(tail)[t * (D / 8) + d8] = x;
    } else {
      const uint32_t xs[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
      for (int e = 0; e < 8; ++e) tail[(d8 * 8 + e) * P + t] = (uint16_t)(e & 1 ? xs[e >> 1] >> 16 : xs[e >> 1]);
    }
  }
}

struct ReadParams {
  Kv8 c;
  uint16_t *k, *v;  // [tokens, heads, D]
  int units, sequences;
};

__device__ __forceinline__ uint4 scaled_halves(uint2 codes, float s) {
  const uint2 a = codes4_to_halves(codes.x), b = codes4_to_halves(codes.y);
  auto mul = [&](uint32_t w) {
    const h2 x = as_h2(w);
    return as_u32(h2{(_Float16)((float)x[0] * s), (_Float16)((float)x[1] * s)});
  };
  return make_uint4(mul(a.x), mul(a.y), mul(b.x), mul(b.y));
}

template <int D, int P, int C, bool PAST>
__global__ __launch_bounds__(64 * kWaves) void kv8_read_kernel(const ReadParams p) {
  using S = PageShape<D, P, C>;
  __shared__ uint32_t turned[kWaves / C][D * S::kRow / 4];
  const Kv8& c = p.c;
  const PageOf w = page_of_wave<C>(c, p.units, p.sequences);
  if (!w.there) return;
  Kv8Seq s = kv8_sequence(c, w.b);
  if (s.n > s.len) {
    s.row += s.n - s.len;
    s.n = s.len;
  }
  const int lane = C == 1 ? threadIdx.x & 63 : threadIdx.x;
  const int start = s.len - s.n, closed = s.len / P, page = start / P + w.unit;
  if (s.n == 0 || page * P >= s.len) return;
  const bool is_tail = page >= closed;
  uint16_t* out = (w.values ? p.v : p.k) + w.head * D;
  auto put = [&](int t, int d8, uint4 x) {
    const int pos = page * P + t;
    const int64_t row = s.row + (pos - start);
    if (pos >= start && pos < s.len && row >= 0 && row < c.tokens) store16<PAST>(out + row * c.heads * D + d8 * 8, x);
  };
  if (is_tail) {
    const uint16_t* tail = (w.values ? c.v_tail : c.k_tail) + ((int64_t)kv8_slot(c, s.slot) * c.heads + w.head) * (P * D);
#pragma unroll
    for (int j = 0; j < S::kPerLane; ++j) {
      const int i = lane + S::kStep * j, t = i / (D / 8) * 4, d8 = i % (D / 8);
      if (i >= S::kQuads || page * P + t >= s.len) continue;
      uint4 v[4];
      if (w.values) {
        tail_quad<P>(tail, d8 * 8, t, v);
      } else {
#pragma unroll
        for (int k = 0; k < 4; ++k) v[k] = reinterpret_cast<const uint4*>(tail)[(t + k) * (D / 8) + d8];
      }
#pragma unroll
      for (int k = 0; k < 4; ++k) put(t + k, d8, v[k]);
    }
    return;
  }
  const int64_t at = kv8_block(c, c.table[w.b * c.table_stride + page], w.head);
  const uint8_t* codes = (w.values ? c.v_codes : c.k_codes) + at * S::kBytes;
  const float scale = (w.values ? c.v_scale : c.k_scale)[at];
  if (!w.values) {
    uint2 q[S::kPerLane][4];
#pragma unroll
    for (int j = 0; j < S::kPerLane; ++j) {
      const int i = lane + S::kStep * j, t = i / (D / 8) * 4, d8 = i % (D / 8);
#pragma unroll
      for (int k = 0; k < 4; ++k)
        if (i < S::kQuads) q[j][k] = load8<PAST>(codes + ((t + k) * (D / 8) + d8) * 8);
    }
#pragma unroll
    for (int j = 0; j < S::kPerLane; ++j) {
      const int i = lane + S::kStep * j, t = i / (D / 8) * 4, d8 = i % (D / 8);
#pragma unroll
      for (int k = 0; k < 4; ++k)
        if (i < S::kQuads) put(t + k, d8, scaled_halves(q[j][k], scale));
    }
    return;
  }
  uint32_t* lds = turned[C == 1 ? threadIdx.x >> 6 : 0];
  uint4 raw[S::kVectors];
#pragma unroll
  for (int j = 0; j < S::kVectors; ++j) {
    const int i = lane + S::kStep * j;
    if (i < S::kBytes / 16) raw[j] = load16<PAST>(codes + i * 16);
  }
#pragma unroll
  for (int j = 0; j < S::kVectors; ++j) {
    const int i = lane + S::kStep * j, d = i / (P / 16), t = i % (P / 16) * 16;
    if (i >= S::kBytes / 16) continue;
    uint32_t* to = &lds[(d * S::kRow + t) / 4];
    to[0] = raw[j].x;
    to[1] = raw[j].y;
    to[2] = raw[j].z;
    to[3] = raw[j].w;
  }
  page_barrier<C>();
#pragma unroll
  for (int j = 0; j < S::kPerLane; ++j) {
    const int i = lane + S::kStep * j, t = i / (D / 8) * 4, d8 = i % (D / 8);
    if (i >= S::kQuads) continue;
    uint32_t x[8], lo[4], hi[4];
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = lds[((d8 * 8 + e) * S::kRow + t) / 4];
    turn4(x[0], x[1], x[2], x[3], lo);
    turn4(x[4], x[5], x[6], x[7], hi);
#pragma unroll
    for (int k = 0; k < 4; ++k) put(t + k, d8, scaled_halves(make_uint2(lo[k], hi[k]), scale));
  }
}

// Whether a page is shared: while that gives a CU eight workgroups at most, keys' and values' (64 sequences, 8 heads of 128, pages of 64: a token
// appended 6.1 us against 9.9, 65 read 9.8 against 11.4; 12000 tokens of 40 heads in pages of 16: 140 and 117 us against 102 and 68, before either went past the caches)
bool shared_pages(int64_t pages) { return pages <= (int64_t)num_cus() * 4; }
// Whether fp16 values and codes read go past the caches (codes that are written do not: attention reads them next): where a call's operands,
// fp16 and codes of `tokens` keys and values, are more than the last of them.  12000 tokens of 40 heads, 376 MB appended and 445 MB read: 79 and 62 us against 102 and 67.
bool past_caches(const Kv8& c, int D) { return c.tokens * c.heads * D * 6 > kLastCacheBytes; }

template <typename Params, typename Kernel>
int launch_pages(Kernel kernel, const Params& p, bool shared, const char* name, hipStream_t st) {
  const int64_t pages = (int64_t)p.units * p.c.heads * p.sequences, blocks = shared ? pages : (pages + kWaves - 1) / kWaves;
  if (blocks > 0x7FFFFFFF) return set_error(QQQ_ERR_SHAPE, "%s: %lld workgroups", name, (long long)blocks);
  hipLaunchKernelGGL(kernel, dim3((unsigned)blocks, 2), dim3(64 * kWaves), 0, st, p);
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
  const AppendParams p = {c, (const uint16_t*)k, (const uint16_t*)v, k_token, k_head, v_token, v_head, units_of(c.max_new, P), sequences};
  const bool shared = shared_pages((int64_t)p.units * c.heads * sequences);
  const bool past = past_caches(c, D);
#define QQQ_APPEND(D_, P_)                                                                                    \
  return shared ? launch_pages(kv8_append_kernel<D_, P_, kWaves, false>, p, true, "kv8_append", st)          \
         : past ? launch_pages(kv8_append_kernel<D_, P_, 1, true>, p, false, "kv8_append", st)               \
                : launch_pages(kv8_append_kernel<D_, P_, 1, false>, p, false, "kv8_append", st)
  QQQ_KV8_SHAPES(QQQ_APPEND)
#undef QQQ_APPEND
}

int launch_kv8_read(const Kv8& c, int D, int P, int sequences, void* k, void* v, hipStream_t st) {
  const ReadParams p = {c, (uint16_t*)k, (uint16_t*)v, units_of(c.max_new, P), sequences};
  const bool shared = shared_pages((int64_t)p.units * c.heads * sequences);
  const bool past = past_caches(c, D);
#define QQQ_READ(D_, P_)                                                                                      \
  return shared ? launch_pages(kv8_read_kernel<D_, P_, kWaves, false>, p, true, "kv8_read", st)              \
         : past ? launch_pages(kv8_read_kernel<D_, P_, 1, true>, p, false, "kv8_read", st)                   \
                : launch_pages(kv8_read_kernel<D_, P_, 1, false>, p, false, "kv8_read", st)
  QQQ_KV8_SHAPES(QQQ_READ)
#undef QQQ_READ
}

}  // namespace qqq
