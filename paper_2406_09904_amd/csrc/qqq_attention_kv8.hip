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
#include <algorithm>
#include <type_traits>

#include "qqq_kv8.h"
#include "qqq_past.h"

namespace qqq {

namespace {

typedef _Float16 h8 __attribute__((ext_vector_type(8)));
typedef float f4 __attribute__((ext_vector_type(4)));
typedef float f16v __attribute__((ext_vector_type(16)));

constexpr int kTile = 64;         // tokens of a step over the keys
constexpr int kJoinMost = 1024;   // parts of a row
constexpr float kShift = 6.0f;    // weights are up to 2^6: fp16 keeps all their bits down to 2^-20 of the largest
constexpr float kMost = 0x1p14f;  // sums of weights up to which the many-rows kernel leaves its reference alone (fp16 ends at 2^16)
constexpr float kLog2e = 1.44269504088896340736f, kLn2 = 0.69314718055994530942f;

struct AttnParams {
  Kv8 c;
  const uint16_t* q;
  int64_t q_token, q_head;
  uint16_t* out;
  float* lse;
  // where the keys are split; many rows: [splits][tokens][q_heads], few: [2 * splits][rows of a key/value head][heads] (see Share)
  float* part_o;     // [..][D]
  float2* part_ml;
  int2* part_of;     // few rows: a sequence's first workgroup, twice, + 1 if its second place; how many share it  [sequences]
  float scale_log2;  // scale * log2(e)
  int group, q_heads, causal, window;
  int splits, chunk; // many rows: workgroups that share a row's keys, tiles of each; few rows: workgroups of a head, where parts are written; tiles of each
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

// A page's factors: of the exponent, log2 of the values' scale, and one over it.  A scale of zero stands for codes that are all zero: whatever it
// is taken for, they add nothing.  It is taken for the least that a page has (2^-24 / 127), so that such a page's scores do not stand for the row's
// largest contribution, beside which the others' weights would lose their bits (as 1, with values of 1e-3 and scores 10 below the zeros': half of the result).
struct Factors {
  float c, lv, rv;
};
__device__ __forceinline__ Factors factors_of(float ks, float vs, float scale_log2) {
  Factors f;
  f.c = fmaxf(ks * scale_log2, 0x1p-100f);
  const float v = vs > 0.0f ? vs : 0x1p-31f;
  f.lv = __builtin_amdgcn_logf(v);
  f.rv = __builtin_amdgcn_rcpf(v);
  return f;
}

// The pages of a tile of 64 tokens (64 / P of them): where they lie in units of a page and head, and their scales.  The tile is the same
// for a whole wave, so these are scalar loads.  `closed` pages exist; past them any page that does stands in (its codes are not used).
template <int P>
struct Pages {
  static constexpr int N = kTile / P;
  int32_t id[N];
};
template <int P>
__device__ __forceinline__ Pages<P> pages_of(const Kv8& c, int b, int tile, int closed) {
  // (always a load, so that the requests behind it are the same on every path)
  typedef const int32_t __attribute__((address_space(4))) * Constant;  // (scalar loads, whatever stands between them)
  const Constant table = (Constant)(uintptr_t)(closed > 0 ? c.table + b * c.table_stride : c.kv_len + b);
  Pages<P> g;
#pragma unroll
  for (int i = 0; i < Pages<P>::N; ++i) g.id[i] = table[max(0, min(tile * Pages<P>::N + i, closed - 1))];
  return g;
}
// of a 16-token group's page, by the lane's group
template <int P, typename T>
__device__ __forceinline__ T of_group(const T* v, int group) {
  constexpr int N = Pages<P>::N;
  const T a = v[0], b = v[1 % N], c = v[2 % N], d = v[3 % N];  // (all of them read, so that they stay in registers)
  if constexpr (P == 64) return a;
  else if constexpr (P == 32) return group & 2 ? b : a;
  else {
    const T lo = group & 1 ? b : a, hi = group & 1 ? d : c;
    return group & 2 ? hi : lo;
  }
}

// What a workgroup of the few-rows kernel has of a head's keys, all sequences' tiles in a row and cut into equal shares: so every workgroup
// ends at the same time whatever the lengths are, which the host does not know.  A sequence counts one tile at least, for what is written of it.  A
// workgroup that has all of a sequence writes its result; of one that it shares it writes a part, into its first place where its share starts with
// it, otherwise (the share ends with it) into its second.
struct Share {
  int b, from, tiles;  // first sequence, its tiles that others have, tiles in all
  int start;           // among all
  int each, longer;    // shares of each tiles, the first `longer` of them of one more
};
__device__ __forceinline__ int weight_of(const AttnParams& p, int b) {
  const Kv8Seq s = kv8_sequence(p.c, b);
  return s.n > 0 ? max(1, range_of(p, s, 0, s.n - 1).tiles) : 0;
}
__device__ __forceinline__ int share_at(const Share& s, int x) {  // the workgroup that has tile x
  const int of_longer = s.longer * (s.each + 1);
  return x < of_longer ? x / (s.each + 1) : s.longer + (x - of_longer) / s.each;
}
template <int T>
__device__ __forceinline__ Share share_of(const AttnParams& p, int w) {
  __shared__ int sums[T / 64], found[2];
  Share s;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  int weight = 0, upto = 0, total = 0;
  if (tid == 0) found[0] = p.sequences;  // (none: should the lengths change under the call)
  auto scan = [&](int base) {  // weights of T sequences, their running sum in each wave, each wave's sum
    weight = base + tid < p.sequences ? weight_of(p, base + tid) : 0;
    upto = weight;
#pragma unroll
    for (int x = 1; x < 64; x *= 2) {
      const int v = __shfl_up(upto, x);
      upto += lane >= x ? v : 0;
    }
    __syncthreads();
    if (lane == 63) sums[wave] = upto;
    __syncthreads();
  };
  auto before = [&](int waves) {
    int sum = 0;
    for (int x = 0; x < waves; ++x) sum += sums[x];
    return sum;
  };
  for (int base = 0; base < p.sequences; base += T) {
    scan(base);
    total += before(T / 64);
  }
  total = __builtin_amdgcn_readfirstlane(total);
  const int shares = max(1, min(p.splits, max(total / 4, p.sequences)));
  s.each = total / shares;
  s.longer = total - s.each * shares;
  s.start = w * s.each + min(w, s.longer);
  s.tiles = w < shares ? s.each + (w < s.longer ? 1 : 0) : 0;
  s.b = 0;
  s.from = s.start;
  if (s.tiles > 0) {
    int at = 0;
    for (int base = 0; base < p.sequences; base += T) {
      if (p.sequences > T) scan(base);
      const int first = at + before(wave) + upto - weight;
      if (first <= s.start && s.start < first + weight) {
        found[0] = base + tid;
        found[1] = s.start - first;
      }
      at += before(T / 64);
    }
    __syncthreads();
    s.b = __builtin_amdgcn_readfirstlane(found[0]);
    s.from = __builtin_amdgcn_readfirstlane(found[1]);
  }
  return s;
}

// ---- a few rows: up to 16 * NT of them a key/value head -----------------------------------------------------------------------------
//
// Bound by the cache's bytes: every code is read once, straight into registers, and used by up to 16 * NT rows; a wave takes every fourth
// tile of its workgroup's chunk by itself, the waves' results are joined through LDS.  One token of a session of 131000, 8 heads of 128
// read by 64: 48 us, 5.6 TB/s (a plain read stream reaches 6.2); of 48 sessions of 17 to 8000: 77 us, 5.2 TB/s, the rest being where a share
// goes from one sequence to the next.  A short past is latency: 500 tokens 7.8 to 8.1 us, of which 1.6 are an empty launch, and 0.3 a tile; with eight waves
// instead of four, so that no wave has two tiles, 8.5, since a compute unit's four SIMDs issue the same instructions either way.
// A tile of 64 tokens, 16 x 16 x 32 products.  Lane l = 16 g + n.  S^T: operand row r of 16-token subtile t is token
// 16 (r / 4) + 4 t + r % 4, so that lane (g, n) gets the scores of row n with tokens 16 g + 4 t + i, i = 0..3: over t, the 16 tokens
// from 16 g on.  They are its operand of the second product, whose other operand is 16 consecutive tokens of a channel: one 16-byte
// load of the token-minor codes.  Along the channels of the first product the same holds: a lane loads 16 consecutive ones, the
// halves of which belong to two steps; the queries are laid out alike.
//
// What is in flight is what counts: the next tile's keys are requested as soon as this tile's are in the scores, its values as soon as
// this tile's are in the result, and nothing that a request depends on is waited for there (loads return in order): page numbers
// are fetched two tiles ahead, scales one.
constexpr int W = 4, kRowsThreads = 64 * W;
template <int D, int P, int NT, bool SHARED, bool PAST>
__global__ __launch_bounds__(kRowsThreads, D <= 128 ? 2 : 1) void attn_rows_kernel(const AttnParams p) {
  constexpr int J = D / 64, DT = D / 16, NP = Pages<P>::N;
  constexpr int kRowO = D + 4;  // (16 bytes over: the lanes' rows start in different banks)
  __shared__ float join_o[W * 16 * NT * kRowO];
  __shared__ float2 join_ml[W][16 * NT];
  const Kv8& c = p.c;
  const int head = blockIdx.x;
  Share share = {};
  share.b = blockIdx.z;
  if constexpr (SHARED) {
    share = share_of<kRowsThreads>(p, blockIdx.y);
    if (share.tiles == 0) return;
  }
  int left = share.tiles;
  for (int b = share.b; b < p.sequences; ++b) {
    const Kv8Seq s = kv8_sequence(c, b);
    if (s.n == 0) {
      if constexpr (SHARED) continue;
      return;
    }
    const Range range = range_of(p, s, 0, s.n - 1);
    const int weight = max(1, range.tiles), from = SHARED ? (b == share.b ? share.from : 0) : (int)blockIdx.y * p.chunk;
    const int take = min(SHARED ? left : p.chunk, weight - from);
    if (take <= 0) return;
    const int tiles = min(take, range.tiles - from);  // (0 of a sequence that has none)
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), n = lane & 15, g = lane >> 4;
    const int closed = s.len / P, slot = kv8_slot(c, s.slot);
    const int open_tile = s.len > closed * P ? closed * P / kTile : -1;  // the one with tokens in the tail slot

    const int gk = n >> 2;  // 16-token group that this lane's row of the first operand is taken from
    uint4 kraw[4][J], vraw[DT];
    const uint32_t k_lane = (((16 * gk) & (P - 1)) + (n & 3)) * D + 16 * g, v_lane = n * P + ((16 * g) & (P - 1));
    auto offsets = [&](const Pages<P>& of, int64_t* at) {
#pragma unroll
      for (int i = 0; i < NP; ++i) at[i] = kv8_block(c, of.id[i], head) * (P * D);
    };
    auto request_k = [&](const Pages<P>& of) {
      int64_t offset[NP];
      offsets(of, offset);
      const uint8_t* at = c.k_codes + of_group<P>(offset, gk) + k_lane;
#pragma unroll
      for (int t = 0; t < 4; ++t)
#pragma unroll
        for (int j = 0; j < J; ++j) kraw[t][j] = load16<PAST>(at + 4 * t * D + 64 * j);
    };
    auto request_v = [&](const Pages<P>& of) {
      int64_t offset[NP];
      offsets(of, offset);
      const uint8_t* at = c.v_codes + of_group<P>(offset, g) + v_lane;
#pragma unroll
      for (int dt = 0; dt < DT; ++dt) vraw[dt] = load16<PAST>(at + dt * 16 * P);
    };
    float ks[NP], vs[NP];
    auto scales = [&](const Pages<P>& of) {
#pragma unroll
      for (int i = 0; i < NP; ++i) {
        const int64_t at = kv8_block(c, of.id[i], head);
        ks[i] = c.k_scale[at];
        vs[i] = c.v_scale[at];
      }
    };

    // queries, and each row's keys [lo, hi).  (Requested first: what is waited for in the loop must not lie behind the codes in flight.)
    h8 q[NT][J * 2];
    int lo[NT], hi[NT];
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      const int r = nt * 16 + n, i = r / p.group, hq = head * p.group + r % p.group;
      const int64_t row = s.row + i;
      const bool there = i < s.n && row >= 0 && row < c.tokens;
      const int pos = s.len - s.n + i;
      hi[nt] = !there ? 0 : p.causal ? min(s.len, pos + 1) : s.len;
      lo[nt] = p.window ? pos - p.window + 1 : 0;
      const uint4* from_q = reinterpret_cast<const uint4*>(p.q + (there ? row * p.q_token + hq * p.q_head : 0));
#pragma unroll
      for (int j = 0; j < J; ++j)
#pragma unroll
        for (int h = 0; h < 2; ++h) q[nt][2 * j + h] = as_h8(from_q[8 * j + 2 * g + h]);  // (a row that is not there: another's, never written)
    }

    const int first = range.tile0 + from + wave, end = range.tile0 + from + tiles;
    Pages<P> pages = pages_of<P>(c, b, min(first, end - 1), closed);

    float m[NT], l[NT];
    f4 o[NT][DT];
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      m[nt] = -__builtin_inff();
      l[nt] = 0.0f;
#pragma unroll
      for (int dt = 0; dt < DT; ++dt) o[nt][dt] = f4{0, 0, 0, 0};
    }

    // one tile's keys from `key_lo` and up to `key_hi`: k_of(t, j, half) and v_of(dt, half) give the codes' operands; next() requests after the scores
    // and after the result
    auto step = [&](int tile, int key_lo, int key_hi, const Factors& f, auto k_of, auto v_of, auto next_k, auto next_v) {
      f4 st[NT][4];
#pragma unroll
      for (int t = 0; t < 4; ++t) {
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) st[nt][t] = f4{0, 0, 0, 0};
#pragma unroll
        for (int j = 0; j < J; ++j) {
          const h8 k0 = k_of(t, j, 0), k1 = k_of(t, j, 1);
#pragma unroll
          for (int nt = 0; nt < NT; ++nt) {
            st[nt][t] = __builtin_amdgcn_mfma_f32_16x16x32_f16(k0, q[nt][2 * j], st[nt][t], 0, 0, 0);
            st[nt][t] = __builtin_amdgcn_mfma_f32_16x16x32_f16(k1, q[nt][2 * j + 1], st[nt][t], 0, 0, 0);
          }
        }
      }
      next_k();
      const bool edge = (tile + 1) * kTile > range.whole_hi || tile * kTile < range.whole_lo;
      h8 w[NT][2];
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) {
        if (edge) {
          const int least = max(lo[nt], key_lo), most = min(hi[nt], key_hi);
#pragma unroll
          for (int t = 0; t < 4; ++t)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              const int key = tile * kTile + 16 * g + 4 * t + i;
              if (!(key >= least && key < most)) st[nt][t][i] = -__builtin_inff();
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
        if (__any(alpha != 1.0f)) {
#pragma unroll
          for (int dt = 0; dt < DT; ++dt) o[nt][dt] *= alpha;
        }
      }
#pragma unroll
      for (int dt = 0; dt < DT; ++dt) {
        const h8 v0 = v_of(dt, 0), v1 = v_of(dt, 1);
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
          o[nt][dt] = __builtin_amdgcn_mfma_f32_16x16x32_f16(v0, w[nt][0], o[nt][dt], 0, 0, 0);
          o[nt][dt] = __builtin_amdgcn_mfma_f32_16x16x32_f16(v1, w[nt][1], o[nt][dt], 0, 0, 0);
        }
      }
      next_v();
    };
    auto k_codes = [&](int t, int j, int half) { return half ? codes8_to_halves(kraw[t][j].z, kraw[t][j].w) : codes8_to_halves(kraw[t][j].x, kraw[t][j].y); };
    auto v_codes = [&](int dt, int half) { return half ? codes8_to_halves(vraw[dt].z, vraw[dt].w) : codes8_to_halves(vraw[dt].x, vraw[dt].y); };

    // Tokens in the tail slot are a step of their own, a wave's last: their values are not relative to a page's scale, and in one step with closed pages of
    // small values (pages shorter than a tile) their scores would stand for more than they contribute and take those pages' weights their bits (values of
    // 1e-4 to 1e-3: 0.3 % of the result).  The step costs a short call in small pages 0.4 us (500 tokens 8.0 us); codes and slot never share registers (four tokens
    // of 48 sequences in pages of 16 109 us, 116 in one step; one of 16 sequences, heads of 64 18.5, 23.3).
    const bool has_tail = open_tile >= first && open_tile < end && (open_tile - first) % W == 0;
    const int code_end = min(end, (closed * P + kTile - 1) / kTile);
    if (first < code_end) {  // (a wave that has but the tail slot goes there at once: 500 tokens 9.0 us, 9.4 through codes that it does not use)
      __builtin_amdgcn_sched_barrier(0);
      scales(pages);
      request_k(pages);
      __builtin_amdgcn_sched_barrier(0);
      request_v(pages);
      __builtin_amdgcn_sched_barrier(0);
      pages = pages_of<P>(c, b, min(first + W, end - 1), closed);
      for (int tile = first; tile < code_end; tile += W) {
        const Factors f = factors_of(of_group<P>(ks, g), of_group<P>(vs, g), p.scale_log2);
        const Pages<P> after = pages_of<P>(c, b, min(tile + 2 * W, end - 1), closed);
        step(tile, 0, closed * P, f, k_codes, v_codes,
             [&]() {
               __builtin_amdgcn_sched_barrier(0);
               scales(pages);
               request_k(pages);
               __builtin_amdgcn_sched_barrier(0);
             },
             [&]() {
               __builtin_amdgcn_sched_barrier(0);
               request_v(pages);
               __builtin_amdgcn_sched_barrier(0);
             });
        pages = after;
      }
    }
    if (has_tail) {
      const int64_t tail = ((int64_t)slot * c.heads + head) * (P * D);
      h8 kt[4][J][2], vt[DT][2];
#pragma unroll
      for (int t = 0; t < 4; ++t)
#pragma unroll
        for (int j = 0; j < J; ++j)
#pragma unroll
          for (int half = 0; half < 2; ++half)
            kt[t][j][half] = as_h8(*reinterpret_cast<const uint4*>(c.k_tail + tail + k_lane + 4 * t * D + 64 * j + 8 * half));
#pragma unroll
      for (int dt = 0; dt < DT; ++dt)
#pragma unroll
        for (int half = 0; half < 2; ++half) vt[dt][half] = as_h8(*reinterpret_cast<const uint4*>(c.v_tail + tail + v_lane + dt * 16 * P + 8 * half));
      // tokens of the lane's group that are in the slot: what lies past them may be anything
      const int left = open_tile * kTile + 16 * g >= closed * P ? s.len - (open_tile * kTile + 16 * g) : 0;
      uint4 there[2];
#pragma unroll
      for (int half = 0; half < 2; ++half) {
        auto pair = [&](int e) { return (8 * half + e < left ? 0xFFFFu : 0u) | (8 * half + e + 1 < left ? 0xFFFF0000u : 0u); };
        there[half] = make_uint4(pair(0), pair(2), pair(4), pair(6));
      }
      step(open_tile, closed * P, s.len, factors_of(1.0f, 1.0f, p.scale_log2), [&](int t, int j, int half) { return kt[t][j][half]; },
           [&](int dt, int half) {
             const uint4 v = __builtin_bit_cast(uint4, vt[dt][half]);
             return as_h8(make_uint4(v.x & there[half].x, v.y & there[half].y, v.z & there[half].z, v.w & there[half].w));
           },
           []() {}, []() {});
    }

    // join the waves: each puts its rows into LDS, four channels of a row are then a thread's
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      l[nt] = across16(across32(l[nt], fadd2), fadd2);
      if (g == 0) join_ml[wave][nt * 16 + n] = make_float2(m[nt], l[nt]);
#pragma unroll
      for (int dt = 0; dt < DT; ++dt) *reinterpret_cast<f4*>(&join_o[(wave * 16 * NT + nt * 16 + n) * kRowO + dt * 16 + 4 * g]) = o[nt][dt];
    }
    __syncthreads();
    const int rows = s.n * p.group;
    const bool whole = take == weight;
    const int place = SHARED ? 2 * (int)blockIdx.y + (b == share.b ? 0 : 1) : 2 * (int)(blockIdx.z * gridDim.y + blockIdx.y);
    for (int at = threadIdx.x; at < rows * (D / 4); at += kRowsThreads) {
      const int r = at / (D / 4), d = at % (D / 4) * 4, i = r / p.group, hq = head * p.group + r % p.group;
      const int64_t row = s.row + i;
      float top = -__builtin_inff(), sum = 0.0f;
#pragma unroll
      for (int x = 0; x < W; ++x) top = fmaxf(top, join_ml[x][r].x);
      const float base = top == -__builtin_inff() ? 0.0f : top;
      f4 all = {0, 0, 0, 0};
#pragma unroll
      for (int x = 0; x < W; ++x) {
        const float2 ml = join_ml[x][r];
        const float a = __builtin_amdgcn_exp2f(ml.x - base);
        sum = __builtin_fmaf(ml.y, a, sum);
        all += *reinterpret_cast<const f4*>(&join_o[(x * 16 * NT + r) * kRowO + d]) * a;
      }
      if (row < 0 || row >= c.tokens) continue;
      const int64_t to = row * p.q_heads + hq;
      if (whole) {
        const float inv = sum == 0.0f ? 0.0f : 1.0f / sum;  // (0: it sees nothing; a NaN stays one)
        *reinterpret_cast<uint2*>(p.out + to * D + d) = make_uint2(as_u32(h2{(_Float16)(all[0] * inv), (_Float16)(all[1] * inv)}),
                                                                   as_u32(h2{(_Float16)(all[2] * inv), (_Float16)(all[3] * inv)}));
        if (p.lse && d == 0) p.lse[to] = sum == 0.0f ? -__builtin_inff() : kLn2 * (__builtin_amdgcn_logf(sum) + (top - kShift));
      } else {
        const int64_t part = ((int64_t)place * (c.max_new * p.group) + r) * c.heads + head;
        *reinterpret_cast<f4*>(p.part_o + part * D + d) = all;
        if (d == 0) p.part_ml[part] = make_float2(top, sum);
      }
    }
    if (p.splits > 1 && from == 0 && head == 0 && threadIdx.x == 0) {
      const int last = SHARED ? share_at(share, share.start + share.tiles - left + weight - 1) : (weight - 1) / p.chunk;
      p.part_of[b] = make_int2(place, last - (int)blockIdx.y + 1);
    }
    if constexpr (!SHARED) return;
    left -= take;
    if (left <= 0) return;
    __syncthreads();  // (the joined rows have been read)
  }
}

// ---- many rows ----------------------------------------------------------------------------------------------------------------------
//
// 128 rows of one key/value head (tokens times the heads that share it) a workgroup, 32 a wave, over tiles of 64 tokens that the
// workgroup converts to fp16 in LDS once for its four waves (two buffers, one barrier a tile, the next tile's codes on their way
// meanwhile).  A prompt of 8000 tokens, 64 heads of 128 over 8: 1.07 to 1.13 ms, 930 to 980 TFLOP/s, where a large library product of
// fp16 reaches 1411.  The matrix units are busy half of the cycles: the exponentials and conversions beside them take their issue.  Power is the rest: the
// same instructions on data of zeros take 0.88 ms.  Heads of 64 have twice the exponentials for a product: 800 TFLOP/s; heads of 256 (32 over 4) fit but one wave
// a SIMD, with 60 to 70 registers spilled and copies between the register files: 710.  64 rows a wave (accumulators in the other register file, and copies to and fro) took 1.41 ms, values straight from memory
// instead of through LDS 2.6 (spilled), the two products of neighbouring tiles interleaved 1.21.
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

template <int D, int P>
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
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), n = lane & 31, h = lane >> 5;
  const int closed = s.len / P, slot = kv8_slot(c, s.slot);

  const int r = row0 + wave * 32 + n, i = r / p.group, hq = head * p.group + r % p.group;
  const int64_t row = s.row + i;
  const bool there = i < s.n && row >= 0 && row < c.tokens;
  const int pos = s.len - s.n + i;
  const int hi = !there ? 0 : p.causal ? min(s.len, pos + 1) : s.len, lo = p.window ? pos - p.window + 1 : 0;
  h8 q[KS];
  {
    const uint4* from_q = reinterpret_cast<const uint4*>(p.q + (there ? row * p.q_token + hq * p.q_head : 0));
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) q[ks] = as_h8(from_q[2 * ks + h]);  // (a row that is not there: another's, never written)
  }

  // staging: thread's chunks of 16 codes
  constexpr int NP = Pages<P>::N;
  uint4 kraw[KC], vraw[VC];
  float ks_raw = 0.0f, vs_raw = 0.0f;
  auto request = [&](const Pages<P>& of) {
    int64_t offset[NP];
#pragma unroll
    for (int x = 0; x < NP; ++x) offset[x] = kv8_block(c, of.id[x], head) * (P * D);
#pragma unroll
    for (int j = 0; j < KC; ++j) {
      const int at = tid + kBlockThreads * j, t = at / (D / 16), d = at % (D / 16) * 16;
      kraw[j] = *reinterpret_cast<const uint4*>(c.k_codes + of_group<P>(offset, t >> 4) + (t & (P - 1)) * D + d);
    }
#pragma unroll
    for (int j = 0; j < VC; ++j) {
      const int at = tid + kBlockThreads * j, d = at >> 2, grp = at & 3;
      vraw[j] = *reinterpret_cast<const uint4*>(c.v_codes + of_group<P>(offset, grp) + d * P + ((16 * grp) & (P - 1)));
    }
    if (tid < 4) {
      const int64_t at = kv8_block(c, of_group<P>(of.id, tid), head);
      ks_raw = c.k_scale[at];
      vs_raw = c.v_scale[at];
    }
  };
  // codes to fp16, into LDS
  auto stage = [&](TileLds<D>& to) {
#pragma unroll
    for (int j = 0; j < KC; ++j) {
      const int at = tid + kBlockThreads * j, t = at / (D / 16), d = at % (D / 16) * 16;
      uint4* put = reinterpret_cast<uint4*>(&to.k[t * TileLds<D>::kRowK + d]);
      put[0] = __builtin_bit_cast(uint4, codes8_to_halves(kraw[j].x, kraw[j].y));
      put[1] = __builtin_bit_cast(uint4, codes8_to_halves(kraw[j].z, kraw[j].w));
    }
#pragma unroll
    for (int j = 0; j < VC; ++j) {
      const int at = tid + kBlockThreads * j, d = at >> 2, grp = at & 3;
      uint4* put = reinterpret_cast<uint4*>(&to.v[d * TileLds<D>::kRowV + 16 * grp]);
      put[0] = __builtin_bit_cast(uint4, codes8_to_halves(vraw[j].x, vraw[j].y));
      put[1] = __builtin_bit_cast(uint4, codes8_to_halves(vraw[j].z, vraw[j].w));
    }
    if (tid < 4) {
      const Factors f = factors_of(ks_raw, vs_raw, p.scale_log2);
      to.c[tid] = f.c;
      to.lv[tid] = f.lv;
      to.rv[tid] = f.rv;
    }
  };
  // and over it what the tail slot holds of the tile that the sequence ends in (each thread over its own chunks): where that tile has closed pages too, in
  // a step of its own after theirs (see the few-rows kernel)
  const int open_tile = s.len > closed * P ? closed * P / kTile : -1;
  auto stage_tail = [&](TileLds<D>& to) {
    const int64_t tail = ((int64_t)slot * c.heads + head) * (P * D);
    uint4 kt[KC][2], vt[VC][2];
#pragma unroll
    for (int j = 0; j < KC; ++j) {
      const int at = tid + kBlockThreads * j, t = at / (D / 16), d = at % (D / 16) * 16;
#pragma unroll
      for (int half = 0; half < 2; ++half) kt[j][half] = *reinterpret_cast<const uint4*>(c.k_tail + tail + (t & (P - 1)) * D + d + 8 * half);
    }
#pragma unroll
    for (int j = 0; j < VC; ++j) {
      const int at = tid + kBlockThreads * j, d = at >> 2, grp = at & 3;
#pragma unroll
      for (int half = 0; half < 2; ++half) vt[j][half] = *reinterpret_cast<const uint4*>(c.v_tail + tail + d * P + ((16 * grp) & (P - 1)) + 8 * half);
    }
#pragma unroll
    for (int j = 0; j < KC; ++j) {
      const int at = tid + kBlockThreads * j, t = at / (D / 16), d = at % (D / 16) * 16;
      if ((open_tile * kTile + t) / P < closed) continue;
      uint4* put = reinterpret_cast<uint4*>(&to.k[t * TileLds<D>::kRowK + d]);
      put[0] = kt[j][0];
      put[1] = kt[j][1];
    }
#pragma unroll
    for (int j = 0; j < VC; ++j) {
      const int at = tid + kBlockThreads * j, d = at >> 2, grp = at & 3;
      if ((open_tile * kTile + 16 * grp) / P < closed) continue;
      const int left = s.len - (open_tile * kTile + 16 * grp);  // tokens that exist: what lies past them may be anything
      auto pair = [&](uint32_t w, int e) { return w & ((e < left ? 0xFFFFu : 0u) | (e + 1 < left ? 0xFFFF0000u : 0u)); };
      uint4* put = reinterpret_cast<uint4*>(&to.v[d * TileLds<D>::kRowV + 16 * grp]);
#pragma unroll
      for (int half = 0; half < 2; ++half)
        put[half] = make_uint4(pair(vt[j][half].x, 8 * half), pair(vt[j][half].y, 8 * half + 2), pair(vt[j][half].z, 8 * half + 4), pair(vt[j][half].w, 8 * half + 6));
    }
    if (tid < 4 && (open_tile * kTile + 16 * tid) / P >= closed) {
      to.c[tid] = p.scale_log2;
      to.lv[tid] = 0.0f;
      to.rv[tid] = 1.0f;
    }
  };

  float m = -__builtin_inff(), l = 0.0f;
  f16v o[DT];
#pragma unroll
  for (int dt = 0; dt < DT; ++dt)
#pragma unroll
    for (int x = 0; x < 16; ++x) o[dt][x] = 0.0f;

  const int first = range.tile0 + from, last = first + tiles;
  const int tail_step = open_tile < first || open_tile >= last ? -1 : P < kTile && closed * P > open_tile * kTile ? open_tile + 1 : open_tile;
  const int end = max(last, tail_step + 1);  // steps are tiles, but for the tail slot's
  auto pages_at = [&](int tile) { return pages_of<P>(c, b, min(tile, end - 1), closed); };
  Pages<P> pages = pages_at(first);   // of the tile after the one whose codes are on their way
  request(pages);
  pages = pages_at(first + 1);
  // everything so far, the queries too: left to the loop, their wait would be one for the codes in flight in every tile
  __builtin_amdgcn_s_waitcnt(0x0F70);  // vmcnt(0)
  __builtin_amdgcn_sched_barrier(0);
  stage(lds[0]);
  if (first == tail_step) stage_tail(lds[0]);
  request(pages);
  pages = pages_at(first + 2);
  lds_barrier();
  const int token_of_row = 16 * (n >> 4) + 8 * ((n >> 2) & 1) + 4 * ((n >> 3) & 1) + (n & 3);
  bool unseen = true;  // some row of the wave has seen nothing yet
  auto step = [&](int at, auto buffer) {
    const bool is_tail = at == tail_step;
    const int tile = is_tail ? open_tile : at;
    const TileLds<D>& t = lds[decltype(buffer)::value];
    TileLds<D>& next = lds[1 - decltype(buffer)::value];
    auto k_of = [&](int x) {  // x: step and 32-token subtile (in turn, so that no product waits for the one before it)
      return as_h8(*reinterpret_cast<const uint4*>(&t.k[(32 * (x & 1) + token_of_row) * TileLds<D>::kRowK + 16 * (x >> 1) + 8 * h]));
    };
    auto v_of = [&](int x) {  // x: step of 16 tokens and 32 channels
      return as_h8(*reinterpret_cast<const uint4*>(&t.v[(32 * (x % DT) + n) * TileLds<D>::kRowV + 16 * (x / DT) + 8 * h]));
    };
    constexpr int kAhead = 4;  // operands on their way from LDS
    const f16v zero = {};
    f16v sc[2];
    {
      h8 a[2 * KS];
#pragma unroll
      for (int x = 0; x < kAhead; ++x) a[x] = k_of(x);
#pragma unroll
      for (int x = 0; x < 2 * KS; ++x) {
        if (x + kAhead < 2 * KS) a[x + kAhead] = k_of(x + kAhead);
        sc[x & 1] = __builtin_amdgcn_mfma_f32_32x32x16_f16(a[x], q[x >> 1], x < 2 ? zero : sc[x & 1], 0, 0, 0);
      }
      __builtin_amdgcn_sched_group_barrier(0x100, kAhead, 0);
#pragma unroll
      for (int x = 0; x < 2 * KS; ++x) {
        __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
        if (x + kAhead < 2 * KS) __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
      }
    }
    __builtin_amdgcn_sched_barrier(0);
    h8 v[4 * DT];
#pragma unroll
    for (int x = 0; x < kAhead; ++x) v[x] = v_of(x);  // on their way while the weights are made
    float fc[4], flv[4], frv[4];
#pragma unroll
    for (int g = 0; g < 4; ++g) {
      fc[g] = t.c[g];
      flv[g] = t.lv[g];
      frv[g] = t.rv[g];
    }
    __builtin_amdgcn_sched_barrier(0);
    if ((tile + 1) * kTile > range.whole_hi || tile * kTile < range.whole_lo) {
      const int least = P < kTile && is_tail ? max(lo, closed * P) : lo, most = P < kTile && !is_tail ? min(hi, closed * P) : hi;
#pragma unroll
      for (int u = 0; u < 2; ++u)
#pragma unroll
        for (int x = 0; x < 16; ++x) {
          const int key = tile * kTile + 32 * u + 16 * (x >> 3) + 8 * h + (x & 7);
          if (!(key >= least && key < most)) sc[u][x] = -__builtin_inff();
        }
    }
    // Weights relative to the reference as it stands.  Sums of a lane's weights that stay small say that each of them does; where they do not, or
    // where a row has seen nothing yet, the reference is raised to the row's largest contribution, and they are made again.
    h8 w[4];
    float sums[4];
    auto weigh = [&]() {
      const float base = m == -__builtin_inff() ? 0.0f : m;   // a row that has seen nothing yet: weights 2^-inf = 0
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        const float add = flv[g] - base + kShift;
        sums[g] = 0.0f;
#pragma unroll
        for (int x = 0; x < 8; ++x) {
          const float e = __builtin_amdgcn_exp2f(__builtin_fmaf(sc[g >> 1][8 * (g & 1) + x], fc[g], add));
          sums[g] += e;
          w[g][x] = (_Float16)e;
        }
      }
    };
    weigh();
    if (unseen || __any(fmaxf(fmaxf(sums[0], sums[1]), fmaxf(sums[2], sums[3])) > kMost)) {
      float top = -__builtin_inff();
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        float tg = sc[g >> 1][8 * (g & 1)];
#pragma unroll
        for (int x = 1; x < 8; ++x) tg = fmaxf(tg, sc[g >> 1][8 * (g & 1) + x]);
        top = fmaxf(top, __builtin_fmaf(tg, fc[g], flv[g]));
      }
      top = across32(top, fmax2);
      const float now = fmaxf(m, top), by = m == now ? 1.0f : __builtin_amdgcn_exp2f(m - now);
      m = now;
      l *= by;
#pragma unroll
      for (int dt = 0; dt < DT; ++dt) o[dt] *= by;
      unseen = __any(m == -__builtin_inff());
      weigh();
    }
#pragma unroll
    for (int g = 0; g < 4; ++g) l = __builtin_fmaf(sums[g], frv[g], l);
    // the second product; beside it the next tile's codes become fp16 (past the last tile: some codes again, never read)
#pragma unroll
    for (int x = 0; x < 4 * DT; ++x) {
      if (x + kAhead < 4 * DT) v[x + kAhead] = v_of(x + kAhead);
      o[x % DT] = __builtin_amdgcn_mfma_f32_32x32x16_f16(v[x], w[x / DT], o[x % DT], 0, 0, 0);
    }
    stage(next);
    if (at + 1 == tail_step) stage_tail(next);
    request(pages);
    pages = pages_at(at + 3);
    lds_barrier();
  };
  // (two at a time: which buffer is which is then a constant, and LDS addresses offsets of the instructions)
  for (int at = first; at < end; at += 2) {
    step(at, std::integral_constant<int, 0>{});
    if (at + 1 < end) step(at + 1, std::integral_constant<int, 1>{});
  }
  l = across32(l, fadd2);
  if (!there) return;
  const int64_t at = row * p.q_heads + hq;
  if (p.splits == 1) {
    const float inv = l == 0.0f ? 0.0f : 1.0f / l;
#pragma unroll
    for (int dt = 0; dt < DT; ++dt)
#pragma unroll
      for (int x = 0; x < 16; x += 4) {
        const uint2 v = make_uint2(as_u32(h2{(_Float16)(o[dt][x] * inv), (_Float16)(o[dt][x + 1] * inv)}),
                                   as_u32(h2{(_Float16)(o[dt][x + 2] * inv), (_Float16)(o[dt][x + 3] * inv)}));
        *reinterpret_cast<uint2*>(p.out + at * D + 32 * dt + 2 * x + 4 * h) = v;
      }
    if (p.lse && h == 0) p.lse[at] = l == 0.0f ? -__builtin_inff() : kLn2 * (__builtin_amdgcn_logf(l) + (m - kShift));
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

// Where the parts of a row (new token i, head hq) lie: the first, and the others at equal distances.
struct RowParts {
  int n;
  int64_t first, second, step;
  __device__ __forceinline__ int64_t operator[](int k) const { return k == 0 ? first : second + (k - 1) * step; }
};
__device__ __forceinline__ RowParts parts_of(const AttnParams& p, const Kv8Seq& s, int b, int i, int hq, int64_t at, int block_rows) {
  RowParts parts;
  const int r = i * p.group + hq % p.group;
  if (block_rows) {  // of the many-rows kernel: its workgroup's tiles as that one counted them
    const int row0 = r / block_rows * block_rows;
    const Range range = range_of(p, s, row0 / p.group, (min(row0 + block_rows, s.n * p.group) - 1) / p.group);
    parts.n = min(max(1, (range.tiles + p.chunk - 1) / p.chunk), p.splits);
    parts.first = at;
    parts.step = p.c.tokens * p.q_heads;
    parts.second = at + parts.step;
  } else {  // (one: it is written already)
    const int2 of = p.part_of[b];
    const int rows = p.c.max_new * p.group, head = hq / p.group;
    const int place = (int)min((uint32_t)of.x, 2u * p.splits - 1u);
    parts.n = of.y > 1 ? min(min(of.y, p.splits - place / 2), kJoinMost) : 0;
    parts.step = (int64_t)2 * rows * p.c.heads;
    parts.first = ((int64_t)place * rows + r) * p.c.heads + head;
    parts.second = ((int64_t)(place / 2 + 1) * 2 * rows + r) * p.c.heads + head;
  }
  return parts;
}

// Joins the splits of every row, one workgroup a row: each wave sums every kJoinWaves-th split, always in the same order.  64 splits of
// 64 rows: 6 us (55 by one wave that takes them one after another).
constexpr int kJoinWaves = 8;
template <int D>
__global__ __launch_bounds__(64 * kJoinWaves) void attn_join_kernel(const AttnParams p, int block_rows) {
  constexpr int E = D / 64;
  typedef float fe __attribute__((ext_vector_type(E)));
  __shared__ float weight[kJoinMost];
  __shared__ float2 most[kJoinWaves];
  __shared__ float sums[kJoinWaves][D];
  const Kv8& c = p.c;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int hq = (int)(blockIdx.x % p.q_heads), i = (int)(blockIdx.x / p.q_heads % c.max_new), b = (int)(blockIdx.x / p.q_heads / c.max_new);
  const Kv8Seq s = kv8_sequence(c, b);
  const int64_t row = s.row + i;
  if (i >= s.n || row < 0 || row >= c.tokens) return;
  const int64_t at = row * p.q_heads + hq;
  const RowParts place = parts_of(p, s, b, i, hq, at, block_rows);
  const int parts = place.n;
  if (parts == 0) return;
  const float* part = p.part_o + lane * E;
  fe first = {};  // (on its way while the weights are made)
  if (wave < parts) first = *reinterpret_cast<const fe*>(part + place[wave] * D);
  float2 ml[kJoinMost / 64 / kJoinWaves];
  float m = -__builtin_inff(), l = 0.0f;
#pragma unroll
  for (int j = 0; j < kJoinMost / 64 / kJoinWaves; ++j) {
    const int k = tid + 64 * kJoinWaves * j;
    ml[j] = k < parts ? p.part_ml[place[k]] : make_float2(-__builtin_inff(), 0.0f);
    m = fmaxf(m, ml[j].x);
  }
#pragma unroll
  for (int x = 1; x < 64; x *= 2) m = fmaxf(m, __shfl_xor(m, x));
  if (lane == 0) most[wave].x = m;
  __syncthreads();
#pragma unroll
  for (int j = 0; j < kJoinWaves; ++j) m = fmaxf(m, most[j].x);
  const float base = m == -__builtin_inff() ? 0.0f : m;
#pragma unroll
  for (int j = 0; j < kJoinMost / 64 / kJoinWaves; ++j) {
    const int k = tid + 64 * kJoinWaves * j;
    const float a = __builtin_amdgcn_exp2f(ml[j].x - base);
    if (k < parts) weight[k] = a;
    l = __builtin_fmaf(ml[j].y, a, l);
  }
#pragma unroll
  for (int x = 1; x < 64; x *= 2) l += __shfl_xor(l, x);
  if (lane == 0) most[wave].y = l;
  __syncthreads();
  fe o = first * (wave < parts ? weight[wave] : 0.0f);
#pragma unroll 8
  for (int k = wave + kJoinWaves; k < parts; k += kJoinWaves) o += *reinterpret_cast<const fe*>(part + place[k] * D) * weight[k];
#pragma unroll
  for (int j = 0; j < E; ++j) sums[wave][lane * E + j] = o[j];
  __syncthreads();
  if (tid >= D) return;
  l = 0.0f;
  float sum = 0.0f;
#pragma unroll
  for (int j = 0; j < kJoinWaves; ++j) {
    l += most[j].y;
    sum += sums[j][tid];
  }
  p.out[at * D + tid] = __builtin_bit_cast(uint16_t, (_Float16)(l == 0.0f ? 0.0f : sum / l));
  if (p.lse && tid == 0) p.lse[at] = l == 0.0f ? -__builtin_inff() : kLn2 * (__builtin_amdgcn_logf(l) + (m - kShift));
}

// The same of few splits or many rows: one wave a row, eight splits at a time.
constexpr int kJoinFew = 8;
template <int D>
__global__ __launch_bounds__(256) void attn_join_few_kernel(const AttnParams p, int block_rows) {
  constexpr int E = D / 64;
  typedef float fe __attribute__((ext_vector_type(E)));
  typedef _Float16 he __attribute__((ext_vector_type(E)));
  const Kv8& c = p.c;
  const int lane = threadIdx.x & 63;
  const int64_t id = (int64_t)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int hq = (int)(id % p.q_heads), i = (int)(id / p.q_heads % c.max_new);
  const int64_t b = id / p.q_heads / c.max_new;
  if (b >= p.sequences) return;
  const Kv8Seq s = kv8_sequence(c, (int)b);
  const int64_t row = s.row + i;
  if (i >= s.n || row < 0 || row >= c.tokens) return;
  const int64_t at = row * p.q_heads + hq;
  const RowParts place = parts_of(p, s, (int)b, i, hq, at, block_rows);
  const int parts = place.n;
  if (parts == 0) return;
  float m = -__builtin_inff(), l = 0.0f;
  fe sum = {};
  for (int k0 = 0; k0 < parts; k0 += kJoinFew) {
    fe o[kJoinFew];
    float2 ml[kJoinFew];
#pragma unroll
    for (int k = 0; k < kJoinFew; ++k) {
      const int64_t from = place[k0 + k < parts ? k0 + k : k0];
      ml[k] = p.part_ml[from];
      o[k] = *reinterpret_cast<const fe*>(p.part_o + from * D + lane * E);
    }
    const float was = m;
#pragma unroll
    for (int k = 0; k < kJoinFew; ++k) m = fmaxf(m, ml[k].x);
    const float base = m == -__builtin_inff() ? 0.0f : m, by = __builtin_amdgcn_exp2f(was - base);
    l *= by;
    sum *= by;
#pragma unroll
    for (int k = 0; k < kJoinFew; ++k) {
      const float a = k0 + k < parts ? __builtin_amdgcn_exp2f(ml[k].x - base) : 0.0f;
      l = __builtin_fmaf(ml[k].y, a, l);
      sum += o[k] * a;
    }
  }
  const float inv = l == 0.0f ? 0.0f : 1.0f / l;
  he out;
#pragma unroll
  for (int j = 0; j < E; ++j) out[j] = (_Float16)(sum[j] * inv);
  *reinterpret_cast<he*>(p.out + at * D + lane * E) = out;
  if (p.lse && lane == 0) p.lse[at] = l == 0.0f ? -__builtin_inff() : kLn2 * (__builtin_amdgcn_logf(l) + (m - kShift));
}

// What a call launches, from sizes that the host knows.
struct Plan {
  int nt;          // 16-row tiles of the few-rows kernel, or 0: the many-rows kernel
  int row_blocks;
  int splits, chunk;
  bool shared;     // few rows: whether workgroups take equal shares of all sequences' keys
  bool past;       // few rows: codes past the caches (of shares always)
  int most;        // splits that no call of a smaller span exceeds
};

Plan plan_of(int heads, int group, int sequences, int max_new, int max_len, int window) {
  Plan f;
  const int64_t rows = (int64_t)max_new * group;
  // Up to 32 rows the codes go to the few-rows kernel (32 rows of 8 heads of 128, 8 sequences of 4000: 22.9 us against 33.2 in the many-rows one;
  // 48 of them 98 against 147; 20 rows, 400 tokens 9.0 against 14.9).  More are not worth a third tile of registers.
  f.nt = rows <= 16 ? 1 : rows <= 32 ? 2 : 0;
  f.row_blocks = f.nt ? 1 : (int)((rows + kBlockRows - 1) / kBlockRows);
  const bool windowed = window > 0 && (int64_t)window + max_new < max_len;
  // (a window's keys may start inside a tile, but there are no more of them than of all keys)
  const int64_t all_tiles = ((int64_t)max_len + kTile - 1) / kTile;
  const int64_t tiles = windowed ? std::min(((int64_t)window + max_new + kTile - 1) / kTile + 1, all_tiles) : all_tiles;
  const int64_t groups = (int64_t)sequences * heads * f.row_blocks;
  // How the keys are split.  Up to 32 tiles for a workgroup a CU: one a CU, in pieces of four tiles at least (one a wave), and only into three or
  // more, since a join costs as much as some seven tiles.  One sequence, 8 heads of 128 read by 64: 1000 tokens 8.5 us (whole 10.1, pieces
  // of eight tiles or more 10.2), 8000 10.3 (10.9); 16 sequences of 1000 11.0 (pieces of eight 12.6); 128 new tokens behind 8000 36 (49
  // with two workgroups a CU).
  // Beyond, two workgroups a CU, so that the bytes in flight last (131000 tokens 49.0, one 55.0, four 60); few rows of several sequences in equal
  // shares: 48 of 17 to 8000 tokens 82 us (pieces of each sequence, eight workgroups a CU 92, four 95, two 105; shares for one workgroup a CU 86,
  // four 91), 64 of 50 to 16000 89 (103), eight of 1000 and one of 60000 37 (43).  Of equal lengths pieces would do (16 of 8000: 47, shares 53),
  // but the host knows only the longest; and short ones are better off with them (six of 300 to 900: 8.7, 13.4).
  // Codes past the caches: 192000 tokens 70.0 us (76.0), 48 sequences 82 (87); a workgroup that waits for each of its loads is the better for
  // what a cache may have kept (16 sequences of 2000, read a moment before, 16.5 us; past the caches 20.6).
  const int64_t cus = num_cus(), per_cu = (tiles * groups + cus - 1) / cus;
  const bool few = per_cu <= 32;
  int64_t chunk = per_cu, splits = groups >= 2 * cus ? 1 : (2 * cus + groups - 1) / groups;
  if (splits > kJoinMost) splits = kJoinMost;
  if (few) {
    if (chunk < 4) chunk = 4;
    if (tiles <= 2 * chunk) chunk = tiles;
  } else {
    chunk = (tiles + splits - 1) / splits;
    if (chunk < 8) chunk = 8;
  }
  if (chunk < 1) chunk = 1;
  f.chunk = (int)chunk;
  f.splits = tiles > 0 ? (int)((tiles + chunk - 1) / chunk) : 1;
  // (neither rule makes more of a shorter span: a workgroup a CU is at most `splits` for a head, pieces are four tiles or more, two of them are one)
  f.most = (int)(tiles <= 8 ? 1 : splits < (tiles + 3) / 4 ? splits : (tiles + 3) / 4);
  f.shared = false;
  f.past = sequences == 1 && per_cu >= 8;
  if (f.nt && sequences > 1) {
    // (shares of many sequences: at 8 workgroups a CU there are enough of whole ones; of 2^31 tiles they could not be counted, but of a window's they may)
    const bool enough = groups >= 8 * cus, many = enough || tiles * sequences > 0x7FFFFFFF;
    const int64_t shares = std::min<int64_t>((2 * cus + heads - 1) / heads, kJoinMost);
    if (!few) {
      f.shared = !many;
      if (many) f.chunk = (int)tiles;
    }
    f.splits = f.shared ? (int)shares : many || f.splits == 1 ? 1 : f.splits * sequences;
    f.most = enough ? 1 : (int)std::max(few ? 1 : shares, f.most > 1 ? (int64_t)f.most * sequences : 1);
  }
  return f;
}

template <int D, int P>
int launch_attention_t(const AttnParams& p, const Plan& f, hipStream_t st) {
  const int64_t blocks = (int64_t)p.sequences * p.c.heads * f.row_blocks * f.splits;
  const int64_t joins = (int64_t)p.sequences * p.c.max_new * p.q_heads;
  if (blocks > 0x7FFFFFFF || (f.splits > 1 && joins > 0x7FFFFFFF)) return set_error(QQQ_ERR_SHAPE, "attention_kv8: too many workgroups");
  if (f.nt && !f.shared && p.sequences > 65535) return set_error(QQQ_ERR_SHAPE, "attention_kv8: %d sequences", p.sequences);
  const dim3 grid(p.c.heads, f.shared ? f.splits : std::max(1, f.splits / p.sequences), f.shared ? 1 : p.sequences);
#define QQQ_ROWS(SHARED, PAST)                                                                                                  \
  do {                                                                                                                          \
    if (f.nt == 1) hipLaunchKernelGGL((attn_rows_kernel<D, P, 1, SHARED, PAST>), grid, dim3(kRowsThreads), 0, st, p);           \
    else hipLaunchKernelGGL((attn_rows_kernel<D, P, 2, SHARED, PAST>), grid, dim3(kRowsThreads), 0, st, p);                     \
  } while (0)
  if (f.nt == 0) hipLaunchKernelGGL((attn_block_kernel<D, P>), dim3((unsigned)blocks), dim3(kBlockThreads), 0, st, p);
  else if (f.shared) QQQ_ROWS(true, true);
  else if (f.past) QQQ_ROWS(false, true);
  else QQQ_ROWS(false, false);
#undef QQQ_ROWS
  const int block_rows = f.nt ? 0 : kBlockRows;
  // (many rows have waves enough: 4096 rows of 16 splits, 16000 keys, 55 us in all against 65 with a workgroup a row)
  const int parts = f.nt && !f.shared ? f.splits / p.sequences : f.splits;  // (of a row, at most)
  if (parts > kJoinFew && joins < 4 * (int64_t)num_cus()) hipLaunchKernelGGL((attn_join_kernel<D>), dim3((unsigned)joins), dim3(64 * kJoinWaves), 0, st, p, block_rows);
  else if (f.splits > 1) hipLaunchKernelGGL((attn_join_few_kernel<D>), dim3((unsigned)((joins + 3) / 4)), dim3(256), 0, st, p, block_rows);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return set_error(QQQ_ERR_HIP, "attention_kv8 launch: %s", hipGetErrorString(e));
  route_note("attention_kv8 %s x%d%s", f.nt ? "rows" : "blocks", f.splits, f.splits > 1 ? " + join" : "");
  return QQQ_OK;
}

template <int D>
int launch_attention_p(const AttnParams& p, int P, const Plan& f, hipStream_t st) {
  return P == 16 ? launch_attention_t<D, 16>(p, f, st) : P == 32 ? launch_attention_t<D, 32>(p, f, st) : launch_attention_t<D, 64>(p, f, st);
}

// Parts of rows, of D and two floats each, and for few rows where each sequence's are.
size_t parts_rows(const Plan& f, int splits, int64_t tokens, int max_new, int q_heads) {
  return splits == 1 ? 0 : (size_t)splits * (size_t)q_heads * (f.nt ? 2 * (size_t)max_new : (size_t)tokens);
}
size_t partial_bytes(const Plan& f, int splits, int64_t tokens, int sequences, int max_new, int q_heads, int D) {
  return splits == 1 ? 0 : parts_rows(f, splits, tokens, max_new, q_heads) * ((size_t)D * 4 + 8) + (f.nt ? (size_t)sequences * 8 : 0);
}

}  // namespace

size_t attention_kv8_bytes(int heads, int q_heads, int D, int sequences, int max_new, int max_len, int64_t tokens) {
  const Plan f = plan_of(heads, q_heads / heads, sequences, max_new, max_len, 0);
  return partial_bytes(f, f.most, tokens, sequences, max_new, q_heads, D);
}

int launch_attention_kv8(const Kv8& c, int D, int P, int sequences, const void* q, int64_t q_token, int64_t q_head, int q_heads, float scale,
                         int causal, int window, void* out, float* lse, void* workspace, size_t workspace_bytes, hipStream_t st) {
  const Plan f = plan_of(c.heads, q_heads / c.heads, sequences, c.max_new, c.max_len, window);
  const size_t need = partial_bytes(f, f.splits, c.tokens, sequences, c.max_new, q_heads, D), rows = parts_rows(f, f.splits, c.tokens, c.max_new, q_heads);
  if (need > workspace_bytes) return set_error(QQQ_ERR_WORKSPACE, "attention_kv8: workspace of %zu bytes, %zu needed", workspace_bytes, need);
  AttnParams p;
  p.c = c;
  p.q = (const uint16_t*)q;
  p.q_token = q_token;
  p.q_head = q_head;
  p.out = (uint16_t*)out;
  p.lse = lse;
  p.part_o = (float*)workspace;
  p.part_ml = (float2*)(p.part_o + rows * D);
  p.part_of = (int2*)(p.part_ml + rows);
  p.scale_log2 = scale * kLog2e;
  p.group = q_heads / c.heads;
  p.q_heads = q_heads;
  p.causal = causal;
  p.window = window;
  p.splits = f.splits;
  p.chunk = f.chunk;
  p.row_blocks = f.row_blocks;
  p.sequences = sequences;
  return D == 64 ? launch_attention_p<64>(p, P, f, st) : D == 128 ? launch_attention_p<128>(p, P, f, st) : launch_attention_p<256>(p, P, f, st);
}

}  // namespace qqq
