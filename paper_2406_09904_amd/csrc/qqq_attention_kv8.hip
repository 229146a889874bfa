// qqq_attention_kv8: attention of a step's new tokens over the 8-bit paged cache.
//
// With ks, vs a page's scales and k, v its integer codes,  s_ij = scale ks <q_i, k_j>  and  o_i = sum_j p_ij vs v_j / sum_j p_ij,
// p_ij = exp(s_ij - m_i).  Both products run on the fp16 matrix instructions with the codes as they are (integers up to 127 are exact
// in fp16) and q as it came; ks goes into the factor of the exponent.  vs goes into the exponent itself: with
//   z_ij = s_ij log2(e) + log2(vs),   m_i = the running maximum of z,   w_ij = 2^(z_ij - m_i),
// o_i = sum_j w_ij v_j / sum_j (w_ij / vs): a tile's weights are relative to the row's largest CONTRIBUTION, so rounding them to fp16
// loses the same whatever the scales of its pages are, and a page costs one multiplication per row instead of one per element.
//
// S is computed transposed (keys x rows), and so is O (channels x rows): a lane of S^T's accumulator holds keys of ONE row, which is
// how the second product wants its operand, so that the weights go from the one to the other in registers.  What makes that fit is
// which token each row of the first product's operand is taken from (token_of_row below).
#include "qqq_kv8.h"

namespace qqq {

namespace {

typedef _Float16 h8 __attribute__((ext_vector_type(8)));
typedef float f4 __attribute__((ext_vector_type(4)));
typedef float f16v __attribute__((ext_vector_type(16)));

constexpr int kTile = 64;         // tokens of a step over the keys
constexpr float kShift = 6.0f;    // weights are up to 2^6: fp16 keeps all their bits down to 2^-20 of the largest
constexpr float kLog2e = 1.44269504088896340736f, kLn2 = 0.69314718055994530942f;

struct AttnParams {
  Kv8 c;
  const uint16_t* q;
  int64_t q_token, q_head;
  uint16_t* out;
  float* lse;
  float* part_o;     // [splits][tokens][q_heads][D], where the keys are split
  float2* part_ml;   // [splits][tokens][q_heads]
  float scale_log2;  // scale * log2(e)
  int group, q_heads, causal, window;
  int lp;            // log2(page_tokens)
  int splits, chunk; // workgroups that share a row's keys, tiles of each
  int row_blocks;    // of the largest sequence
  int sequences;
};

__device__ __forceinline__ h8 as_h8(uint4 v) { return __builtin_bit_cast(h8, v); }
__device__ __forceinline__ h8 codes8_to_halves(uint32_t a, uint32_t b) {
  const uint2 lo = codes4_to_halves(a), hi = codes4_to_halves(b);
  return as_h8(make_uint4(lo.x, lo.y, hi.x, hi.y));
}

// maximum / sum over the lanes l, l ^ 16, l ^ 32, l ^ 48 and over l, l ^ 32
template <typename F>
__device__ __forceinline__ float across32(float v, F f) {
  const auto r = __builtin_amdgcn_permlane32_swap(__builtin_bit_cast(uint32_t, v), __builtin_bit_cast(uint32_t, v), false, false);
  return f(__builtin_bit_cast(float, (uint32_t)r[0]), __builtin_bit_cast(float, (uint32_t)r[1]));
}
template <typename F>
__device__ __forceinline__ float across16(float v, F f) {
  const auto r = __builtin_amdgcn_permlane16_swap(__builtin_bit_cast(uint32_t, v), __builtin_bit_cast(uint32_t, v), false, false);
  return f(__builtin_bit_cast(float, (uint32_t)r[0]), __builtin_bit_cast(float, (uint32_t)r[1]));
}
__device__ __forceinline__ float fmax2(float a, float b) { return fmaxf(a, b); }
__device__ __forceinline__ float fadd2(float a, float b) { return a + b; }

// The keys that rows [i0, i1] (tokens of the sequence) see, in tiles, and where all of them see every key.
struct Range {
  int tile0, tiles;       // first tile, how many
  int whole_lo, whole_hi; // keys that every row sees
};
__device__ __forceinline__ Range range_of(const AttnParams& p, const Kv8Seq& s, int i0, int i1) {
  const int pos0 = s.len - s.n + i0, pos1 = s.len - s.n + i1;
  const int hi = p.causal ? max(0, min(s.len, pos1 + 1)) : s.len, lo = p.window ? max(0, pos0 - p.window + 1) : 0;
  Range r;
  r.tile0 = lo / kTile;
  r.tiles = hi > lo ? (hi + kTile - 1) / kTile - r.tile0 : 0;
  r.whole_hi = p.causal ? max(0, min(s.len, pos0 + 1)) : s.len;
  r.whole_lo = p.window ? max(0, pos1 - p.window + 1) : 0;
  return r;
}

// A page's factors: of the exponent, log2 of the values' scale, and one over it.  A scale of zero stands for codes that are all zero.
struct Factors {
  float c, lv, rv;
};
__device__ __forceinline__ Factors factors_of(float ks, float vs, float scale_log2) {
  Factors f;
  f.c = fmaxf(ks * scale_log2, 0x1p-100f);
  const float v = vs > 0.0f ? vs : 1.0f;
  f.lv = __builtin_amdgcn_logf(v);
  f.rv = 1.0f / v;
  return f;
}

// ---- a few rows: up to 16 * NT of them a key/value head -----------------------------------------------------------------------------
//
// Bound by the cache's bytes: every code is read once, straight into registers, and used by up to 16 * NT rows; a wave takes every W-th
// tile of its workgroup's chunk by itself, the waves' results are joined through LDS.
// A tile of 64 tokens, 16 x 16 x 32 products.  Lane l = 16 g + n.  S^T: operand row r of 16-token subtile t is token
// 16 (r / 4) + 4 t + r % 4, so that lane (g, n) gets the scores of row n with tokens 16 g + 4 t + i, i = 0..3: over t, the 16 tokens
// from 16 g on.  They are its operand of the second product, whose other operand is 16 consecutive tokens of a channel: one 16-byte
// load of the token-minor codes.  Along the channels of the first product the same holds: a lane loads 16 consecutive ones, the
// halves of which belong to two steps; the queries are laid out alike.
template <int D, int NT, int W>
__global__ __launch_bounds__(64 * W) void attn_rows_kernel(const AttnParams p) {
  constexpr int J = D / 64, DT = D / 16;
  __shared__ float join_o[(W / 2) * NT * DT * 4 * 64];
  __shared__ float join_m[(W / 2) * NT * 64], join_l[(W / 2) * NT * 64];
  const Kv8& c = p.c;
  const int split = blockIdx.x % p.splits, head = (blockIdx.x / p.splits) % c.heads, b = blockIdx.x / p.splits / c.heads;
  const Kv8Seq s = kv8_sequence(c, b);
  if (s.n == 0) return;
  const Range range = range_of(p, s, 0, s.n - 1);
  const int from = split * p.chunk, tiles = min(p.chunk, range.tiles - from);
  if (tiles <= 0 && split > 0) return;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, n = lane & 15, g = lane >> 4;
  const int P = 1 << p.lp, closed = s.len >> p.lp, slot = kv8_slot(c, s.slot);

  // queries, and each row's keys [lo, hi)
  h8 q[NT][J * 2];
  int lo[NT], hi[NT];
  int64_t out_at[NT];  // (token, head) of the row, or -1
#pragma unroll
  for (int nt = 0; nt < NT; ++nt) {
    const int r = nt * 16 + n, i = r / p.group, hq = head * p.group + r % p.group;
    const int64_t row = s.row + i;
    const bool there = i < s.n && row >= 0 && row < c.tokens;
    const int pos = s.len - s.n + i;
    hi[nt] = !there ? 0 : p.causal ? min(s.len, pos + 1) : s.len;
    lo[nt] = p.window ? pos - p.window + 1 : 0;
    out_at[nt] = there ? row * p.q_heads + hq : -1;
    const uint4* from_q = reinterpret_cast<const uint4*>(p.q + (there ? row * p.q_token + hq * p.q_head : 0));
#pragma unroll
    for (int j = 0; j < J; ++j)
#pragma unroll
      for (int h = 0; h < 2; ++h) q[nt][2 * j + h] = there ? as_h8(from_q[8 * j + 2 * g + h]) : as_h8(make_uint4(0, 0, 0, 0));
  }

  float m[NT], l[NT];
  f4 o[NT][DT];
#pragma unroll
  for (int nt = 0; nt < NT; ++nt) {
    m[nt] = -__builtin_inff();
    l[nt] = 0.0f;
#pragma unroll
    for (int dt = 0; dt < DT; ++dt) o[nt][dt] = f4{0, 0, 0, 0};
  }

  const int gk = n >> 2;  // 16-token group that this lane's row of the first operand is taken from
  const int32_t* table = c.table + b * c.table_stride;
  auto page_of = [&](int tile, int group) {
    const int at = (tile * kTile + 16 * group) >> p.lp;
    return closed > 0 ? kv8_page(c, table[min(at, closed - 1)]) : (int64_t)0;
  };
  uint4 kraw[4][J], vraw[DT];
  float ks, vs;
  auto request_k = [&](int64_t page) {
    const uint8_t* at = c.k_codes + ((page * c.heads + head) * P + ((16 * gk) & (P - 1)) + (n & 3)) * D + 16 * g;
#pragma unroll
    for (int t = 0; t < 4; ++t)
#pragma unroll
      for (int j = 0; j < J; ++j) kraw[t][j] = *reinterpret_cast<const uint4*>(at + 4 * t * D + 64 * j);
  };
  auto request_v = [&](int64_t page) {
    const int64_t of = page * c.heads + head;
    const uint8_t* at = c.v_codes + of * P * D + n * P + ((16 * g) & (P - 1));
#pragma unroll
    for (int dt = 0; dt < DT; ++dt) vraw[dt] = *reinterpret_cast<const uint4*>(at + dt * 16 * P);
    ks = c.k_scale[of];
    vs = c.v_scale[of];
  };

  const int first = range.tile0 + from + wave, end = range.tile0 + from + tiles;
  if (first < end) {
    request_k(page_of(first, gk));
    request_v(page_of(first, g));
  }
  for (int tile = first; tile < end; tile += W) {
    const int next = min(tile + W, end - 1);
    const int64_t next_k = page_of(next, gk), next_v = page_of(next, g);
    const bool open = (tile + 1) * kTile > closed << p.lp;           // some of its tokens are in the tail slot, or nowhere
    const bool edge = (tile + 1) * kTile > range.whole_hi || tile * kTile < range.whole_lo;
    const bool k_open = open && (tile * kTile + 16 * gk) >> p.lp >= closed, v_open = open && (tile * kTile + 16 * g) >> p.lp >= closed;

    f4 st[NT][4];
#pragma unroll
    for (int t = 0; t < 4; ++t) {
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) st[nt][t] = f4{0, 0, 0, 0};
#pragma unroll
      for (int j = 0; j < J; ++j) {
        h8 k0 = codes8_to_halves(kraw[t][j].x, kraw[t][j].y), k1 = codes8_to_halves(kraw[t][j].z, kraw[t][j].w);
        if (open && k_open) {
          const int row = ((16 * gk) & (P - 1)) + 4 * t + (n & 3);
          const uint4* at = reinterpret_cast<const uint4*>(c.k_tail + (((int64_t)slot * c.heads + head) * P + row) * D + 64 * j + 16 * g);
          k0 = as_h8(at[0]);
          k1 = as_h8(at[1]);
        }
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
          st[nt][t] = __builtin_amdgcn_mfma_f32_16x16x32_f16(k0, q[nt][2 * j], st[nt][t], 0, 0, 0);
          st[nt][t] = __builtin_amdgcn_mfma_f32_16x16x32_f16(k1, q[nt][2 * j + 1], st[nt][t], 0, 0, 0);
        }
      }
    }
    const Factors f = factors_of(v_open ? 1.0f : ks, v_open ? 1.0f : vs, p.scale_log2);
    request_k(next_k);

    h8 w[NT][2];
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      if (edge) {
#pragma unroll
        for (int t = 0; t < 4; ++t)
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const int key = tile * kTile + 16 * g + 4 * t + i;
            if (!(key >= lo[nt] && key < hi[nt])) st[nt][t][i] = -__builtin_inff();
          }
      }
      float top = -__builtin_inff();
#pragma unroll
      for (int t = 0; t < 4; ++t)
#pragma unroll
        for (int i = 0; i < 4; ++i) top = fmaxf(top, st[nt][t][i]);
      top = __builtin_fmaf(top, f.c, f.lv);
      top = across16(across32(top, fmax2), fmax2);
      const float was = m[nt], now = fmaxf(was, top);
      const float base = now == -__builtin_inff() ? 0.0f : now;   // a row that has seen nothing yet: weights 2^-inf = 0
      const float alpha = __builtin_amdgcn_exp2f(was - base), add = f.lv - base + kShift;
      m[nt] = now;
      float sum = 0.0f;
#pragma unroll
      for (int t = 0; t < 4; ++t)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float e = __builtin_amdgcn_exp2f(__builtin_fmaf(st[nt][t][i], f.c, add));
          sum += e;
          w[nt][t >> 1][(t & 1) * 4 + i] = (_Float16)e;
        }
      l[nt] = __builtin_fmaf(l[nt], alpha, sum * f.rv);
#pragma unroll
      for (int dt = 0; dt < DT; ++dt) o[nt][dt] *= alpha;
    }
#pragma unroll
    for (int dt = 0; dt < DT; ++dt) {
      h8 v0 = codes8_to_halves(vraw[dt].x, vraw[dt].y), v1 = codes8_to_halves(vraw[dt].z, vraw[dt].w);
      if (open && v_open) {
        const int t0 = (16 * g) & (P - 1), left = s.len - (tile * kTile + 16 * g);  // tokens of the group that exist
        const uint4* at = reinterpret_cast<const uint4*>(c.v_tail + (((int64_t)slot * c.heads + head) * D + dt * 16 + n) * P + t0);
        v0 = as_h8(at[0]);
        v1 = as_h8(at[1]);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          if (e >= left) v0[e] = (_Float16)0.0f;
          if (e + 8 >= left) v1[e] = (_Float16)0.0f;
        }
      }
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) {
        o[nt][dt] = __builtin_amdgcn_mfma_f32_16x16x32_f16(v0, w[nt][0], o[nt][dt], 0, 0, 0);
        o[nt][dt] = __builtin_amdgcn_mfma_f32_16x16x32_f16(v1, w[nt][1], o[nt][dt], 0, 0, 0);
      }
    }
    request_v(next_v);
  }

  // join the waves: the upper half of those left hands its results to the lower half, register by register
#pragma unroll
  for (int nt = 0; nt < NT; ++nt) l[nt] = across16(across32(l[nt], fadd2), fadd2);
#pragma unroll
  for (int half = W / 2; half >= 1; half /= 2) {
    __syncthreads();
    if (wave >= half && wave < 2 * half) {
      const int at = wave - half;
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) {
        join_m[(at * NT + nt) * 64 + lane] = m[nt];
        join_l[(at * NT + nt) * 64 + lane] = l[nt];
#pragma unroll
        for (int dt = 0; dt < DT; ++dt)
#pragma unroll
          for (int i = 0; i < 4; ++i) join_o[(((at * NT + nt) * DT + dt) * 4 + i) * 64 + lane] = o[nt][dt][i];
      }
    }
    __syncthreads();
    if (wave < half) {
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) {
        const float m2 = join_m[(wave * NT + nt) * 64 + lane], l2 = join_l[(wave * NT + nt) * 64 + lane];
        const float now = fmaxf(m[nt], m2), base = now == -__builtin_inff() ? 0.0f : now;
        const float a1 = __builtin_amdgcn_exp2f(m[nt] - base), a2 = __builtin_amdgcn_exp2f(m2 - base);
        m[nt] = now;
        l[nt] = l[nt] * a1 + l2 * a2;
#pragma unroll
        for (int dt = 0; dt < DT; ++dt)
#pragma unroll
          for (int i = 0; i < 4; ++i) o[nt][dt][i] = o[nt][dt][i] * a1 + join_o[(((wave * NT + nt) * DT + dt) * 4 + i) * 64 + lane] * a2;
      }
    }
  }
  if (wave != 0) return;
#pragma unroll
  for (int nt = 0; nt < NT; ++nt) {
    if (out_at[nt] < 0) continue;
    if (p.splits == 1) {
      const float inv = l[nt] > 0.0f ? 1.0f / l[nt] : 0.0f;
#pragma unroll
      for (int dt = 0; dt < DT; ++dt) {
        const uint2 v = make_uint2(as_u32(h2{(_Float16)(o[nt][dt][0] * inv), (_Float16)(o[nt][dt][1] * inv)}),
                                   as_u32(h2{(_Float16)(o[nt][dt][2] * inv), (_Float16)(o[nt][dt][3] * inv)}));
        *reinterpret_cast<uint2*>(p.out + out_at[nt] * D + dt * 16 + 4 * g) = v;
      }
      if (p.lse && g == 0) p.lse[out_at[nt]] = l[nt] > 0.0f ? kLn2 * (__builtin_amdgcn_logf(l[nt]) + (m[nt] - kShift)) : -__builtin_inff();
    } else {
      const int64_t at = (int64_t)split * c.tokens * p.q_heads + out_at[nt];
#pragma unroll
      for (int dt = 0; dt < DT; ++dt) *reinterpret_cast<f4*>(p.part_o + at * D + dt * 16 + 4 * g) = o[nt][dt];
      if (g == 0) p.part_ml[at] = make_float2(m[nt], l[nt]);
    }
  }
}

// ---- many rows ----------------------------------------------------------------------------------------------------------------------
//
// Bound by the matrix instructions and, as much, by the exponentials beside them: 128 rows of one key/value head (tokens times the
// heads that share it) a workgroup, 32 a wave, over tiles of 64 tokens that the workgroup converts to fp16 in LDS once for its four
// waves (two buffers, one barrier a tile, the next tile's codes on their way meanwhile).
// 32 x 32 x 16 products, lane l = 32 h + n.  S^T: operand row r of a 32-token subtile is token 16 (r / 16) + 8 ((r / 4) % 2) + 4 ((r / 8) % 2)
// + r % 4, so that lane (h, n) gets the scores of row n with tokens 16 s + 8 h + 0..7 in registers 8 s .. 8 s + 7: its operand of step s
// of the second product.
constexpr int kBlockRows = 128, kBlockThreads = 256;

template <int D>
struct TileLds {
  static constexpr int kRowK = D + 8, kRowV = kTile + 8;  // halves; 16 bytes over, so that the lanes' rows start in different banks
  uint16_t k[kTile * kRowK];
  uint16_t v[D * kRowV];
  float c[4], lv[4], rv[4];
};

template <int D>
__global__ __launch_bounds__(kBlockThreads, D <= 128 ? 2 : 1) void attn_block_kernel(const AttnParams p) {
  constexpr int KC = D / 64, VC = D / 64;  // chunks of 16 codes of a thread, of each tile's keys and values
  constexpr int KS = D / 16, DT = D / 32;
  __shared__ TileLds<D> lds[2];
  const Kv8& c = p.c;
  const int head = blockIdx.x % c.heads, split = blockIdx.x / c.heads % p.splits;
  const int block = p.row_blocks - 1 - (int)(blockIdx.x / c.heads / p.splits % p.row_blocks);  // the longest first
  const int b = blockIdx.x / c.heads / p.splits / p.row_blocks;
  const Kv8Seq s = kv8_sequence(c, b);
  const int rows = s.n * p.group, row0 = block * kBlockRows;
  if (row0 >= rows) return;
  const Range range = range_of(p, s, row0 / p.group, min(row0 + kBlockRows - 1, rows - 1) / p.group);
  const int from = split * p.chunk, tiles = min(p.chunk, range.tiles - from);
  if (tiles <= 0 && split > 0) return;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, n = lane & 31, h = lane >> 5;
  const int P = 1 << p.lp, closed = s.len >> p.lp, slot = kv8_slot(c, s.slot);

  const int r = row0 + wave * 32 + n, i = r / p.group, hq = head * p.group + r % p.group;
  const int64_t row = s.row + i;
  const bool there = i < s.n && row >= 0 && row < c.tokens;
  const int pos = s.len - s.n + i;
  const int hi = !there ? 0 : p.causal ? min(s.len, pos + 1) : s.len, lo = p.window ? pos - p.window + 1 : 0;
  h8 q[KS];
  {
    const uint4* from_q = reinterpret_cast<const uint4*>(p.q + (there ? row * p.q_token + hq * p.q_head : 0));
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) q[ks] = there ? as_h8(from_q[2 * ks + h]) : as_h8(make_uint4(0, 0, 0, 0));
  }

  // staging: thread's chunks of 16 codes
  const int32_t* table = c.table + b * c.table_stride;
  auto page_of = [&](int tile, int group) {
    const int at = (tile * kTile + 16 * group) >> p.lp;
    return closed > 0 ? kv8_page(c, table[min(at, closed - 1)]) : (int64_t)0;
  };
  uint4 kraw[KC], vraw[VC];
  float ks_raw = 0.0f, vs_raw = 0.0f;
  auto request = [&](int tile) {
#pragma unroll
    for (int j = 0; j < KC; ++j) {
      const int at = tid + kBlockThreads * j, t = at / (D / 16), d = at % (D / 16) * 16;
      kraw[j] = *reinterpret_cast<const uint4*>(c.k_codes + ((page_of(tile, t >> 4) * c.heads + head) * P + (t & (P - 1))) * D + d);
    }
#pragma unroll
    for (int j = 0; j < VC; ++j) {
      const int at = tid + kBlockThreads * j, d = at >> 2, grp = at & 3;
      vraw[j] = *reinterpret_cast<const uint4*>(c.v_codes + ((page_of(tile, grp) * c.heads + head) * D + d) * P + ((16 * grp) & (P - 1)));
    }
    if (tid < 4) {
      const int64_t of = page_of(tile, tid) * c.heads + head;
      ks_raw = c.k_scale[of];
      vs_raw = c.v_scale[of];
    }
  };
  auto stage = [&](int tile, TileLds<D>& to) {
    const bool open = (tile + 1) * kTile > closed << p.lp;
#pragma unroll
    for (int j = 0; j < KC; ++j) {
      const int at = tid + kBlockThreads * j, t = at / (D / 16), d = at % (D / 16) * 16;
      h8 a = codes8_to_halves(kraw[j].x, kraw[j].y), e = codes8_to_halves(kraw[j].z, kraw[j].w);
      if (open && (tile * kTile + t) >> p.lp >= closed) {
        const uint4* tail = reinterpret_cast<const uint4*>(c.k_tail + (((int64_t)slot * c.heads + head) * P + (t & (P - 1))) * D + d);
        a = as_h8(tail[0]);
        e = as_h8(tail[1]);
      }
      uint4* put = reinterpret_cast<uint4*>(&to.k[t * TileLds<D>::kRowK + d]);
      put[0] = __builtin_bit_cast(uint4, a);
      put[1] = __builtin_bit_cast(uint4, e);
    }
#pragma unroll
    for (int j = 0; j < VC; ++j) {
      const int at = tid + kBlockThreads * j, d = at >> 2, grp = at & 3;
      h8 a = codes8_to_halves(vraw[j].x, vraw[j].y), e = codes8_to_halves(vraw[j].z, vraw[j].w);
      if (open && (tile * kTile + 16 * grp) >> p.lp >= closed) {
        const int left = s.len - (tile * kTile + 16 * grp);
        const uint4* tail = reinterpret_cast<const uint4*>(c.v_tail + (((int64_t)slot * c.heads + head) * D + d) * P + ((16 * grp) & (P - 1)));
        a = as_h8(tail[0]);
        e = as_h8(tail[1]);
#pragma unroll
        for (int x = 0; x < 8; ++x) {
          if (x >= left) a[x] = (_Float16)0.0f;
          if (x + 8 >= left) e[x] = (_Float16)0.0f;
        }
      }
      uint4* put = reinterpret_cast<uint4*>(&to.v[d * TileLds<D>::kRowV + 16 * grp]);
      put[0] = __builtin_bit_cast(uint4, a);
      put[1] = __builtin_bit_cast(uint4, e);
    }
    if (tid < 4) {
      const bool tail = open && (tile * kTile + 16 * tid) >> p.lp >= closed;
      const Factors f = factors_of(tail ? 1.0f : ks_raw, tail ? 1.0f : vs_raw, p.scale_log2);
      to.c[tid] = f.c;
      to.lv[tid] = f.lv;
      to.rv[tid] = f.rv;
    }
  };

  float m = -__builtin_inff(), l = 0.0f;
  f16v o[DT];
#pragma unroll
  for (int dt = 0; dt < DT; ++dt)
#pragma unroll
    for (int x = 0; x < 16; ++x) o[dt][x] = 0.0f;

  const int first = range.tile0 + from, end = first + tiles;
  if (tiles > 0) {
    request(first);
    stage(first, lds[0]);
    request(min(first + 1, end - 1));
    lds_barrier();
  }
  const int token_of_row = 16 * (n >> 4) + 8 * ((n >> 2) & 1) + 4 * ((n >> 3) & 1) + (n & 3);
  for (int tile = first; tile < end; ++tile) {
    const TileLds<D>& t = lds[(tile - first) & 1];
    f16v sc[2];
#pragma unroll
    for (int u = 0; u < 2; ++u) {
#pragma unroll
      for (int x = 0; x < 16; ++x) sc[u][x] = 0.0f;
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) {
        const h8 a = as_h8(*reinterpret_cast<const uint4*>(&t.k[(32 * u + token_of_row) * TileLds<D>::kRowK + 16 * ks + 8 * h]));
        sc[u] = __builtin_amdgcn_mfma_f32_32x32x16_f16(a, q[ks], sc[u], 0, 0, 0);
      }
    }
    if ((tile + 1) * kTile > range.whole_hi || tile * kTile < range.whole_lo) {
#pragma unroll
      for (int u = 0; u < 2; ++u)
#pragma unroll
        for (int x = 0; x < 16; ++x) {
          const int key = tile * kTile + 32 * u + 16 * (x >> 3) + 8 * h + (x & 7);
          if (!(key >= lo && key < hi)) sc[u][x] = -__builtin_inff();
        }
    }
    float top = -__builtin_inff();
#pragma unroll
    for (int g = 0; g < 4; ++g) {
      float tg = sc[g >> 1][8 * (g & 1)];
#pragma unroll
      for (int x = 1; x < 8; ++x) tg = fmaxf(tg, sc[g >> 1][8 * (g & 1) + x]);
      top = fmaxf(top, __builtin_fmaf(tg, t.c[g], t.lv[g]));
    }
    top = across32(top, fmax2);
    const float was = m, now = fmaxf(was, top), base = now == -__builtin_inff() ? 0.0f : now;
    const float alpha = __builtin_amdgcn_exp2f(was - base);
    m = now;
    h8 w[4];
    l *= alpha;
#pragma unroll
    for (int g = 0; g < 4; ++g) {
      const float add = t.lv[g] - base + kShift, cg = t.c[g];
      float sum = 0.0f;
#pragma unroll
      for (int x = 0; x < 8; ++x) {
        const float e = __builtin_amdgcn_exp2f(__builtin_fmaf(sc[g >> 1][8 * (g & 1) + x], cg, add));
        sum += e;
        w[g][x] = (_Float16)e;
      }
      l = __builtin_fmaf(sum, t.rv[g], l);
    }
    if (__any(alpha != 1.0f)) {
#pragma unroll
      for (int dt = 0; dt < DT; ++dt) o[dt] *= alpha;
    }
#pragma unroll
    for (int g = 0; g < 4; ++g)
#pragma unroll
      for (int dt = 0; dt < DT; ++dt) {
        const h8 a = as_h8(*reinterpret_cast<const uint4*>(&t.v[(32 * dt + n) * TileLds<D>::kRowV + 16 * g + 8 * h]));
        o[dt] = __builtin_amdgcn_mfma_f32_32x32x16_f16(a, w[g], o[dt], 0, 0, 0);
      }
    if (tile + 1 < end) {
      stage(tile + 1, lds[(tile + 1 - first) & 1]);
      request(min(tile + 2, end - 1));
    }
    lds_barrier();
  }
  l = across32(l, fadd2);
  if (!there) return;
  const int64_t at = row * p.q_heads + hq;
  if (p.splits == 1) {
    const float inv = l > 0.0f ? 1.0f / l : 0.0f;
#pragma unroll
    for (int dt = 0; dt < DT; ++dt)
#pragma unroll
      for (int x = 0; x < 16; x += 4) {
        const uint2 v = make_uint2(as_u32(h2{(_Float16)(o[dt][x] * inv), (_Float16)(o[dt][x + 1] * inv)}),
                                   as_u32(h2{(_Float16)(o[dt][x + 2] * inv), (_Float16)(o[dt][x + 3] * inv)}));
        *reinterpret_cast<uint2*>(p.out + at * D + 32 * dt + 2 * x + 4 * h) = v;
      }
    if (p.lse && h == 0) p.lse[at] = l > 0.0f ? kLn2 * (__builtin_amdgcn_logf(l) + (m - kShift)) : -__builtin_inff();
  } else {
    const int64_t part = (int64_t)split * c.tokens * p.q_heads + at;
#pragma unroll
    for (int dt = 0; dt < DT; ++dt)
#pragma unroll
      for (int x = 0; x < 16; x += 4)
        *reinterpret_cast<f4*>(p.part_o + part * D + 32 * dt + 2 * x + 4 * h) = f4{o[dt][x], o[dt][x + 1], o[dt][x + 2], o[dt][x + 3]};
    if (h == 0) p.part_ml[part] = make_float2(m, l);
  }
}

// Joins the splits of every row, in their order.  One wave a row.
constexpr int kJoinRows = 4;
template <int D>
__global__ __launch_bounds__(64 * kJoinRows) void attn_join_kernel(const AttnParams p, int block_rows) {
  const Kv8& c = p.c;
  const int lane = threadIdx.x & 63;
  const int64_t id = (int64_t)blockIdx.x * kJoinRows + (threadIdx.x >> 6);  // (sequence, new token, head)
  const int hq = (int)(id % p.q_heads), i = (int)(id / p.q_heads % c.max_new);
  const int64_t b = id / p.q_heads / c.max_new;
  if (b >= p.sequences) return;
  const Kv8Seq s = kv8_sequence(c, (int)b);
  const int64_t row = s.row + i;
  if (i >= s.n || row < 0 || row >= c.tokens) return;
  // the tiles of the row's workgroup, as that one counted them
  const int r = i * p.group + hq % p.group, row0 = block_rows ? r / block_rows * block_rows : 0;
  const int last = block_rows ? min(row0 + block_rows, s.n * p.group) - 1 : s.n * p.group - 1;
  const Range range = range_of(p, s, row0 / p.group, last / p.group);
  const int parts = max(1, (range.tiles + p.chunk - 1) / p.chunk);
  const int64_t at = row * p.q_heads + hq, step = c.tokens * p.q_heads;
  float m = -__builtin_inff();
  for (int k = lane; k < parts; k += 64) m = fmaxf(m, p.part_ml[at + k * step].x);
#pragma unroll
  for (int x = 1; x < 64; x *= 2) m = fmaxf(m, __shfl_xor(m, x));
  const float base = m == -__builtin_inff() ? 0.0f : m;
  float l = 0.0f, o[D / 64];
#pragma unroll
  for (int j = 0; j < D / 64; ++j) o[j] = 0.0f;
  for (int k = 0; k < parts; ++k) {
    const float2 ml = p.part_ml[at + k * step];
    const float a = __builtin_amdgcn_exp2f(ml.x - base);
    l = __builtin_fmaf(ml.y, a, l);
    const float* from = p.part_o + (at + k * step) * D + lane * (D / 64);
#pragma unroll
    for (int j = 0; j < D / 64; ++j) o[j] = __builtin_fmaf(from[j], a, o[j]);
  }
  const float inv = l > 0.0f ? 1.0f / l : 0.0f;
  uint16_t* out = p.out + at * D + lane * (D / 64);
#pragma unroll
  for (int j = 0; j < D / 64; ++j) out[j] = __builtin_bit_cast(uint16_t, (_Float16)(o[j] * inv));
  if (p.lse && lane == 0) p.lse[at] = l > 0.0f ? kLn2 * (__builtin_amdgcn_logf(l) + (m - kShift)) : -__builtin_inff();
}

// What a call launches, from sizes that the host knows.
struct Plan {
  int nt;          // 16-row tiles of the few-rows kernel, or 0: the many-rows kernel
  int row_blocks;
  int splits, chunk;
  int most;        // splits that no call of a smaller span exceeds
};
constexpr int kRowsWaves = 4;

Plan plan_of(int heads, int group, int sequences, int max_new, int max_len, int window, int D) {
  Plan f;
  const int64_t rows = (int64_t)max_new * group;
  f.nt = rows <= 16 ? 1 : rows <= 32 && D <= 128 ? 2 : 0;
  f.row_blocks = f.nt ? 1 : (int)((rows + kBlockRows - 1) / kBlockRows);
  const int64_t span = window > 0 && (int64_t)window + max_new < max_len ? (int64_t)window + max_new : max_len;
  const int64_t tiles = (span + kTile - 1) / kTile + 1;  // (a window's keys may start inside a tile)
  const int64_t groups = (int64_t)sequences * heads * f.row_blocks;
  // enough workgroups to fill the chip, but at least two tiles for each wave
  const int64_t want = (int64_t)num_cus() * (f.nt ? 6 : 2), least = f.nt ? 2 * kRowsWaves : 8;
  int64_t splits = groups >= want ? 1 : (want + groups - 1) / groups;
  f.most = (int)(splits < (tiles + least - 1) / least ? splits : (tiles + least - 1) / least);
  int64_t chunk = (tiles + splits - 1) / splits;
  if (chunk < least) chunk = least;
  if (chunk >= tiles) chunk = tiles;
  f.chunk = (int)chunk;
  f.splits = (int)((tiles + chunk - 1) / chunk);
  return f;
}

template <int D>
int launch_attention_t(const AttnParams& p, const Plan& f, hipStream_t st) {
  const int64_t blocks = (int64_t)p.sequences * p.c.heads * f.row_blocks * f.splits;
  const int64_t joins = ((int64_t)p.sequences * p.c.max_new * p.q_heads + kJoinRows - 1) / kJoinRows;
  if (blocks > 0x7FFFFFFF || joins > 0x7FFFFFFF) return set_error(QQQ_ERR_SHAPE, "attention_kv8: too many workgroups");
  if (f.nt == 1) hipLaunchKernelGGL((attn_rows_kernel<D, 1, kRowsWaves>), dim3((unsigned)blocks), dim3(64 * kRowsWaves), 0, st, p);
  else if (f.nt == 2) {
    if constexpr (D <= 128) hipLaunchKernelGGL((attn_rows_kernel<D, 2, kRowsWaves>), dim3((unsigned)blocks), dim3(64 * kRowsWaves), 0, st, p);
  } else hipLaunchKernelGGL((attn_block_kernel<D>), dim3((unsigned)blocks), dim3(kBlockThreads), 0, st, p);
  if (f.splits > 1) hipLaunchKernelGGL((attn_join_kernel<D>), dim3((unsigned)joins), dim3(64 * kJoinRows), 0, st, p, f.nt ? 0 : kBlockRows);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return set_error(QQQ_ERR_HIP, "attention_kv8 launch: %s", hipGetErrorString(e));
  route_note("attention_kv8 %s x%d%s", f.nt ? "rows" : "blocks", f.splits, f.splits > 1 ? " + join" : "");
  return QQQ_OK;
}

size_t partial_bytes(int splits, int64_t tokens, int q_heads, int D) {
  return splits > 1 ? (size_t)splits * (size_t)tokens * (size_t)q_heads * ((size_t)D * 4 + 8) : 0;
}

}  // namespace

size_t attention_kv8_bytes(int heads, int q_heads, int D, int sequences, int max_new, int max_len, int64_t tokens) {
  return partial_bytes(plan_of(heads, q_heads / heads, sequences, max_new, max_len, 0, D).most, tokens, q_heads, D);
}

int launch_attention_kv8(const Kv8& c, int D, int P, int sequences, const void* q, int64_t q_token, int64_t q_head, int q_heads, float scale,
                         int causal, int window, void* out, float* lse, void* workspace, size_t workspace_bytes, hipStream_t st) {
  const Plan f = plan_of(c.heads, q_heads / c.heads, sequences, c.max_new, c.max_len, window, D);
  if (partial_bytes(f.splits, c.tokens, q_heads, D) > workspace_bytes)
    return set_error(QQQ_ERR_WORKSPACE, "attention_kv8: workspace of %zu bytes, %zu needed", workspace_bytes, partial_bytes(f.splits, c.tokens, q_heads, D));
  AttnParams p;
  p.c = c;
  p.q = (const uint16_t*)q;
  p.q_token = q_token;
  p.q_head = q_head;
  p.out = (uint16_t*)out;
  p.lse = lse;
  p.part_o = (float*)workspace;
  p.part_ml = (float2*)((char*)workspace + (size_t)f.splits * c.tokens * q_heads * D * 4);
  p.scale_log2 = scale * kLog2e;
  p.group = q_heads / c.heads;
  p.q_heads = q_heads;
  p.causal = causal;
  p.window = window;
  p.lp = P == 16 ? 4 : P == 32 ? 5 : 6;
  p.splits = f.splits;
  p.chunk = f.chunk;
  p.row_blocks = f.row_blocks;
  p.sequences = sequences;
  return D == 64 ? launch_attention_t<64>(p, f, st) : D == 128 ? launch_attention_t<128>(p, f, st) : launch_attention_t<256>(p, f, st);
}

}  // namespace qqq
