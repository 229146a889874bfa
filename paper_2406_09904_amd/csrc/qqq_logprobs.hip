// Log probabilities, entropy and the largest logits of rows of V values (qqq_serve.h): each logit is read once.
//
// One pass keeps, per thread and relative to the largest logit m it has met,  z = sum e^(x-m)  and  t = sum (x-m) e^(x-m);  a larger m' turns them into
// z f  and  (t + (m-m') z) f,  f = e^(m-m').  Then  lse = m + log z,  H = log z - t / z: no difference of large numbers is left in either.
// For fp16 logits all of it is in powers of two and the reference is c, the integer above m log2 e: x log2 e - c is one mixed multiply-add, rounded once, and a change of c scales by
// a power of two, exactly.  fp32 logits reach where x log2 e overflows, so x - m comes first.
//
// The largest `top` logits need nothing in that pass but the threads' maxima.  128 groups of threads hold disjoint parts of the row, so the top-th largest of the groups' maxima is
// a lower bound of the row's top-th largest value, and only the blocks of threads with a maximum of at least that are looked at again: in a row without order the bound lets
// 128 log(128 / (128 - top)) values pass, 22 for the largest 20, 89 for 64, whatever V is.  Values that reach the bound are gathered in LDS, and each one's rank is the number of larger ones.  Where they are too many, because
// most of the row is masked or equal, those above the bound are gathered, and then the row's first values that are the bound.  Where these are too many as well (rising values) they go
// through lists, of up to 64 entries in a wave's lanes in falling order.  Entries are ordered by (value, lower place first), so equal values have
// one order and no result depends on which wave came first.
//
// Many rows: a workgroup a row, read in turns.  Up to as many as CUs, of up to 256 KB: the same with the row in registers, its largest known before the first exponential.  Few long
// rows: each is split, the parts leave their sums and their groups' maxima in the workspace, and a second kernel joins them and looks again at the groups that pass.
//
// What bounds it: many rows the bytes (4096 rows of 256 KB, log probabilities and the likeliest token, 164 us, 6.4 TB/s; 777 of 131 KB 23 us, 4.4 TB/s, three rows a CU); few the launch and a
// chain of steps that wait for each other (one row of 64 KB in a graph: sums 4.2 us, with the likeliest 5.5, with the largest 20 6.7; one CU's 32000 exponentials, 16 cycles for 64 on each of four
// SIMDs, are under 0.9 of them; 48 of 200 KB, the largest 5, 8.5).
#include <float.h>

#include <algorithm>
#include <type_traits>

#include "qqq_past.h"
#include "qqq_serve.h"

namespace qqq {

namespace {

constexpr int kSplitThreads = 256, kJoinThreads = 512;
constexpr int kBound = 128;              // groups of a workgroup's threads, whose maxima give the bound
constexpr int kGroups = 64;              // of the threads of a part of a row
constexpr int kOddEach = 4;              // values a thread takes one by one, at most: a row of no more than that is spread over all threads, or its blocks would be in too few groups
constexpr float kLog2e = 1.4426950408889634f;
constexpr float kFar = -1000.0f;         // e^kFar is 0: further than that is as far, and stays finite

struct LogprobArgs {
  const char* logits;
  int64_t row_bytes;
  const int32_t* tokens;
  float *logprob, *entropy, *lse, *top_logprobs;
  int32_t* top_tokens;
  float* parts;   // split rows: of each part its sums (3 values), then its groups' maxima (kGroups)
  int V, top, splits, blocks_per_part;
};
constexpr int kPartValues = 3 + kGroups;

// fp16: 8 values in 16 bytes; fp32: 4
template <bool F32>
struct Row {
  static constexpr int kVec = F32 ? 4 : 8, kSize = F32 ? 4 : 2;
  const char* at;
  int lead, blocks, tail;  // values before the first whole 16 aligned bytes, those 16 bytes, values behind the last
  // one_by_one: a short row, all of whose values are taken as the lead's
  __device__ __forceinline__ Row(const LogprobArgs& p, int64_t row, bool one_by_one = false) {
    at = p.logits + row * p.row_bytes;
    lead = one_by_one ? p.V : min((int)((16 - (reinterpret_cast<uintptr_t>(at) & 15)) & 15) / kSize, p.V);
    blocks = (p.V - lead) / kVec;
    tail = p.V - lead - blocks * kVec;
  }
  __device__ __forceinline__ float value(int i) const {
    if constexpr (F32) return reinterpret_cast<const float*>(at)[i];
    else return (float)reinterpret_cast<const _Float16*>(at)[i];
  }
  // the i-th of the lead's and the tail's values, and its place
  __device__ __forceinline__ int place_of_odd(int i) const { return i < lead ? i : i + blocks * kVec; }
  template <bool PAST>
  __device__ __forceinline__ uint4 block(int b) const { return load16<PAST>(at + lead * kSize + (uint32_t)b * 16u); }
  __device__ __forceinline__ int place_of_block(int b) const { return lead + b * kVec; }
  static __device__ __forceinline__ uint4 masked_block() {
    constexpr uint32_t w = F32 ? 0xFF800000u : 0xFC00FC00u;  // -infinity
    return make_uint4(w, w, w, w);
  }
  static __device__ __forceinline__ void unpack(uint4 v, float* x) {
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int i = 0; i < kVec; ++i)
      x[i] = F32 ? __builtin_bit_cast(float, w[i]) : half_bits_to_float(i & 1 ? w[i >> 1] >> 16 : w[i >> 1] & 0xFFFFu);
  }
  template <int U>
  static __device__ __forceinline__ float largest(const uint4* v) {  // of U blocks; not a NaN unless all are
    if constexpr (F32) {
      float m = __builtin_bit_cast(float, v[0].x);
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const uint32_t w[4] = {v[u].x, v[u].y, v[u].z, v[u].w};
#pragma unroll
        for (int i = 0; i < 4; ++i) m = fmaxf(m, __builtin_bit_cast(float, w[i]));
      }
      return m;
    } else {
      // (the instruction itself, which takes three operands and gives a NaN where there is one: the compiler would quiet every operand first)
      uint32_t m = v[0].x;
#pragma unroll
      for (int u = 0; u < U; ++u)
        asm("v_pk_maximum3_f16 %0, %0, %1, %2\n\tv_pk_maximum3_f16 %0, %0, %3, %4" : "+v"(m) : "v"(v[u].x), "v"(v[u].y), "v"(v[u].z), "v"(v[u].w));
      const h2 pair = as_h2(m);
      return fmaxf((float)pair[0], (float)pair[1]);
    }
  }
};

template <bool F32>
struct Sums {
  static constexpr float kUnit = F32 ? 1.0f : 0.6931471805599453f;   // of m and t, in natural logarithms
  static constexpr float kToTwo = F32 ? kLog2e : 1.0f;               // and in powers of two
  float largest = -FLT_MAX;                      // value met (a NaN is not one)
  float m = F32 ? -FLT_MAX : -94505.0f;          // reference: of fp32 the largest value, of fp16 the integer above its log2 e times
  float z = 0.0f, t = 0.0f;
  // TRACK: the largest value of all batches of blocks but the one that has the largest, and which that is (below 0: of none)
  float others = -FLT_MAX;
  int at = -1;
  __device__ __forceinline__ void refer_to(float to) {
    const float higher = fmaxf(m, to), d = fmaxf(m - higher, kFar), f = __builtin_amdgcn_exp2f(d * kToTwo);
    t = (t + d * z) * f;
    z *= f;
    m = higher;
  }
  template <bool TRACK>
  __device__ __forceinline__ void meet(float x, int batch) {
    if constexpr (TRACK) {
      others = __builtin_amdgcn_fmed3f(others, largest, x);
      at = x > largest ? batch : at;
    }
    largest = fmaxf(largest, x);
    refer_to(F32 ? largest : ceilf(largest * kLog2e));
  }
  // for the bound: the largest value, or infinity where there may be a NaN
  __device__ __forceinline__ float reached() const { return z != z ? __builtin_inff() : z == 0.0f ? -__builtin_inff() : largest; }
  // of a value no larger than the largest; a NaN or infinity gives a NaN
  __device__ __forceinline__ float below(float x) const { return F32 ? x - m : __builtin_fmaf(x, kLog2e, -m); }
  static __device__ __forceinline__ float power(float d) { return __builtin_amdgcn_exp2f(d * kToTwo); }
  __device__ __forceinline__ void add(float x) {
    const float d = below(x), e = power(d);
    z += e;
    t = __builtin_fmaf(fmaxf(d, kFar), e, t);
  }
  // One block's values, none of them larger than the largest.  whole: all lanes have one (a lane without one has masked values)
  __device__ __forceinline__ void add_block(const uint4& v, bool whole) {
    float x[Row<F32>::kVec];
    Row<F32>::unpack(v, x);
    const float t_before = t;
    if (whole) {
#pragma unroll
      for (int i = 0; i < Row<F32>::kVec; ++i) {
        const float d = below(x[i]), e = power(d);
        z += e;
        t = __builtin_fmaf(d, e, t);
      }
      if (__builtin_expect(!__ballot(t != t), 1)) return;
      t = t_before;
#pragma unroll
      for (int i = 0; i < Row<F32>::kVec; ++i) {
        const float d = below(x[i]);
        t = __builtin_fmaf(fmaxf(d, kFar), power(d), t);
      }
    } else {
#pragma unroll
      for (int i = 0; i < Row<F32>::kVec; ++i) add(x[i]);
    }
  }
  template <int U, bool TRACK>
  __device__ __forceinline__ void add_blocks(const uint4* v, int batch) {
    meet<TRACK>(Row<F32>::template largest<U>(v), batch);
    const float t_before = t;
#pragma unroll
    for (int u = 0; u < U; ++u) {
      float x[Row<F32>::kVec];
      Row<F32>::unpack(v[u], x);
#pragma unroll
      for (int i = 0; i < Row<F32>::kVec; ++i) {
        const float d = below(x[i]), e = power(d);
        z += e;
        t = __builtin_fmaf(d, e, t);
      }
    }
    asm volatile("" : "+v"(z));  // (here: else every power is kept until behind the branch)
    if (__builtin_expect(__ballot(t != t), 0)) {  // -infinity times 0: a masked value, whose part is 0 (or there is a NaN, which z has too)
      t = t_before;
#pragma unroll
      for (int u = 0; u < U; ++u) {
        uint4 again = v[u];
        asm("" : "+v"(again.x), "+v"(again.y), "+v"(again.z), "+v"(again.w));  // (else every difference and power is kept for this branch: 64 registers)
        float x[Row<F32>::kVec];
        Row<F32>::unpack(again, x);
#pragma unroll
        for (int i = 0; i < Row<F32>::kVec; ++i) {
          const float d = below(x[i]);
          t = __builtin_fmaf(fmaxf(d, kFar), power(d), t);
        }
      }
    }
  }
};

template <int CTRL>
__device__ __forceinline__ float moved(float v) {
  return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), CTRL, 0xF, 0xF, false));
}
// over groups of G lanes, in each of them
template <int G>
__device__ __forceinline__ float group_max(float v) {
  if constexpr (G >= 2) v = fmaxf(v, moved<0xB1>(v));   // quad_perm [1,0,3,2]
  if constexpr (G >= 4) v = fmaxf(v, moved<0x4E>(v));   // quad_perm [2,3,0,1]
  if constexpr (G >= 8) v = fmaxf(v, moved<0x141>(v));  // row_half_mirror
  if constexpr (G >= 16) v = fmaxf(v, moved<0x140>(v)); // row_mirror
  return v;
}
__device__ __forceinline__ float lane_value(float v, int lane) { return __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, v), lane)); }
__device__ __forceinline__ float wave_max(float v) {
  v = group_max<16>(v);
  return fmaxf(fmaxf(lane_value(v, 0), lane_value(v, 16)), fmaxf(lane_value(v, 32), lane_value(v, 48)));
}
__device__ __forceinline__ float wave_sum(float v) {
  v += moved<0xB1>(v);
  v += moved<0x4E>(v);
  v += moved<0x141>(v);
  v += moved<0x140>(v);
  return (lane_value(v, 0) + lane_value(v, 16)) + (lane_value(v, 32) + lane_value(v, 48));
}
// of all lanes, in each of them; the order is fixed
template <bool F32>
__device__ __forceinline__ Sums<F32> wave_sums(Sums<F32> s) {
  s.refer_to(wave_max(s.m));
  s.z = wave_sum(s.z);
  s.t = wave_sum(s.t);
  return s;
}
template <bool F32, int WAVES>
__device__ __forceinline__ Sums<F32> join_waves(const float (*of_wave)[3]) {  // a wave's sums a lane
  Sums<F32> s;
  const int lane = threadIdx.x & 63;
  if (lane < WAVES) {
    s.m = of_wave[lane][0];
    s.z = of_wave[lane][1];
    s.t = of_wave[lane][2];
  }
  return wave_sums(s);
}

// ---- order.  Values by 32 bits that order as they do: a NaN above everything, -0 as 0
__device__ __forceinline__ uint32_t order_of(float x) {
  const uint32_t b = __builtin_bit_cast(uint32_t, x + 0.0f);
  return x != x ? 0xFFFFFFFFu : b ^ ((uint32_t)((int32_t)b >> 31) | 0x80000000u);
}
__device__ __forceinline__ float value_of(uint32_t order) {
  return __builtin_bit_cast(float, order & 0x80000000u ? order ^ 0x80000000u : ~order);
}

// The top-th largest of the workgroup's kBound values (none of them a NaN), in all its threads.  Each wave counts, for every value, the larger ones among its share of them.
template <int T>
__device__ __forceinline__ float bound_of(const float* of_group, int (*larger)[kBound], int top) {
  constexpr int W = T / 64, kShare = kBound / W;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const float v[2] = {of_group[lane], of_group[64 + lane]};
  if (top == 1) return wave_max(fmaxf(v[0], v[1]));  // the largest of all
  int n[2] = {0, 0};
#pragma unroll
  for (int i = 0; i < kShare; ++i)
#pragma unroll
    for (int h = 0; h < 2; ++h) n[h] += of_group[wave * kShare + i] > v[h];
#pragma unroll
  for (int h = 0; h < 2; ++h) larger[wave][64 * h + lane] = n[h];
  __syncthreads();
  float least = __builtin_inff();
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    n[h] = 0;
#pragma unroll
    for (int w = 0; w < W; ++w) n[h] += larger[w][64 * h + lane];
    if (n[h] < top) least = fminf(least, v[h]);
  }
  return -wave_max(-least);
}

// The largest entries so far, in the wave's lanes in falling order: (order of the value, bits of the place inverted); 0, 0: none
struct List {
  uint32_t order = 0, place = 0;
  __device__ __forceinline__ static bool above(uint32_t a_order, uint32_t a_place, uint32_t b_order, uint32_t b_place) {
    return a_order > b_order || (a_order == b_order && a_place > b_place);
  }
  // Lanes offer a value each: those that belong into the first `top` are put there, one after the other.
  __device__ __forceinline__ void offer(bool has, float x, int at, int top, float& bound) {
    if (!__ballot(has && !(x < bound))) return;
    const uint32_t o = order_of(x), q = ~(uint32_t)at;
    uint64_t some;
    while ((some = __ballot(has && above(o, q, (uint32_t)__builtin_amdgcn_readlane((int)order, top - 1), (uint32_t)__builtin_amdgcn_readlane((int)place, top - 1)) && !(x < bound)))) {
      const int from = __builtin_ctzll(some), lane = threadIdx.x & 63;
      const uint32_t new_order = (uint32_t)__builtin_amdgcn_readlane((int)o, from), new_place = (uint32_t)__builtin_amdgcn_readlane((int)q, from);
      const int to = __popcll(__ballot(above(order, place, new_order, new_place)));
      const uint32_t order_before = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)order, 0x138, 0xF, 0xF, false);  // wave_shr:1
      const uint32_t place_before = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)place, 0x138, 0xF, 0xF, false);
      order = lane < to ? order : lane == to ? new_order : order_before;
      place = lane < to ? place : lane == to ? new_place : place_before;
      if (lane == from) has = false;
    }
    // what is below the last of a full list need not be offered
    const uint32_t last = (uint32_t)__builtin_amdgcn_readlane((int)order, top - 1);
    if (last != 0 && last != 0xFFFFFFFFu) bound = fmaxf(bound, value_of(last));
  }
};

// What a workgroup has found of the largest values
template <int T>
struct Found {
  uint64_t entries[T];  // order of the value, then bits of the place inverted
  int ranks[128];
  int count;         // (also of those that found no room)
  __device__ __forceinline__ void add(uint32_t order, uint32_t place) {
    const int at = atomicAdd(&count, 1);  // (which entry lies where decides nothing)
    if (at < T) entries[at] = (uint64_t)order << 32 | place;
  }
  __device__ __forceinline__ bool is_full() const { return *const_cast<const volatile int*>(&count) > T; }  // (then nothing more need be added)
  __device__ __forceinline__ void add_list(const List& list, int top) {
    if ((int)(threadIdx.x & 63) < top && (list.order | list.place) != 0) add(list.order, list.place);
  }
};
// What lanes do with the values that they look at: gather those that reach the bound, or those above it, or offer them to the wave's list
enum { kReach, kAbove, kList };
template <int MODE>
__device__ __forceinline__ bool wanted(float x, float bound) {
  return MODE == kAbove ? !(x <= bound) : !(x < bound);  // (and a NaN)
}
template <bool F32, int T, int MODE>
__device__ __forceinline__ void look_at_block(const Row<F32>& r, int b, bool has, int top, float& bound, List& list, Found<T>& found) {
  uint4 v = Row<F32>::masked_block();
  if (has) v = r.template block<false>(b);
  float x[Row<F32>::kVec];
  Row<F32>::unpack(v, x);
  bool some = false;
#pragma unroll
  for (int i = 0; i < Row<F32>::kVec; ++i) some |= wanted<MODE>(x[i], bound);
  some &= has;
  if (!__ballot(some)) return;
#pragma unroll
  for (int i = 0; i < Row<F32>::kVec; ++i) {
    if constexpr (MODE == kList) list.offer(some, x[i], r.place_of_block(b) + i, top, bound);
    else if (some && wanted<MODE>(x[i], bound)) found.add(order_of(x[i]), ~(uint32_t)(r.place_of_block(b) + i));
  }
}
template <bool F32, int T, int MODE>
__device__ __forceinline__ void look_at_value(const Row<F32>& r, int place, bool has, int top, float& bound, List& list, Found<T>& found) {
  const float x = has ? r.value(place) : 0.0f;
  if constexpr (MODE == kList) list.offer(has, x, place, top, bound);
  else if (has && wanted<MODE>(x, bound)) found.add(order_of(x), ~(uint32_t)place);
}

// Whether a thread that reached that much has values to look at
__device__ __forceinline__ bool passes(float reached, float level, bool above) { return (above ? reached > level : reached >= level) || reached == __builtin_inff(); }

// The first `want` of the row's values that equal `value`: T blocks at a time, from the row's begin on
template <bool F32, int T>
__device__ __forceinline__ void find_equal(const Row<F32>& r, float value, int want, Found<T>& found) {
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  int got = 0;
  auto turn = [&](uint32_t hits, int place) {
    int sum = __popc(hits);
#pragma unroll
    for (int d = 1; d < 64; d *= 2) {
      const int other = __shfl_up(sum, d);
      if (lane >= d) sum += other;
    }
    if (lane == 63) found.ranks[wave] = sum;
    __syncthreads();
    int at = got + sum - __popc(hits);
    for (int w = 0; w < T / 64; ++w) {
      at += w < wave ? found.ranks[w] : 0;
      got += found.ranks[w];
    }
    for (; hits && at < want; hits &= hits - 1, ++at) found.add(order_of(value), ~(uint32_t)(place + __builtin_ctz(hits)));
    __syncthreads();
  };
  for (int i = 0; i < r.lead && got < want; i += T) turn(i + tid < r.lead && r.value(i + tid) == value, i + tid);
  for (int b0 = 0; b0 < r.blocks && got < want; b0 += T) {
    uint32_t hits = 0;
    if (b0 + tid < r.blocks) {
      float x[Row<F32>::kVec];
      Row<F32>::unpack(r.template block<false>(b0 + tid), x);
#pragma unroll
      for (int i = 0; i < Row<F32>::kVec; ++i) hits |= (uint32_t)(x[i] == value) << i;
    }
    turn(hits, r.place_of_block(b0 + tid));
  }
  if (got < want) turn(tid < r.tail && r.value(r.place_of_odd(r.lead + tid)) == value, r.place_of_odd(r.lead + tid));
  if (tid < 128) found.ranks[tid] = 0;
}

// The row's largest.  pass(level, above): the threads (or groups of them) that met a value of the level, or above it, are listed (LISTED); look(mode, level, list): what they met is.
template <bool F32, int T, bool LISTED, class Pass, class Look>
__device__ __forceinline__ void find_top(const Row<F32>& r, int top, float bound, int& passing, int& passing_once, Found<T>& found, Pass pass, Look look) {
  auto again = [&] {
    __syncthreads();
    if (threadIdx.x == 0) found.count = passing = passing_once = 0;
    __syncthreads();
  };
  auto start = [&](bool above) {
    if constexpr (LISTED) {
      pass(bound, above);
      __syncthreads();
    }
  };
  List list;
  start(false);
  look(std::integral_constant<int, kReach>{}, bound, list);
  __syncthreads();
  if (found.count <= T) return;  // (the same in every thread)
  // Too many: of those that are the bound itself only the first few can be wanted, and few are above it
  again();
  start(true);
  look(std::integral_constant<int, kAbove>{}, bound, list);
  __syncthreads();
  if (found.count <= T) {
    const int want = top - found.count;
    if (want > 0) find_equal<F32, T>(r, bound, want, found);
  } else {
    again();
    start(false);
    look(std::integral_constant<int, kList>{}, bound, list);
    again();
    found.add_list(list, top);
  }
  __syncthreads();
}

// Each entry's rank counted, the first `top` written.
template <bool F32, int T>
__device__ __forceinline__ void write_top(const LogprobArgs& p, int64_t row, const Sums<F32>& all, float log_z, Found<T>& found) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, n = found.count;
  auto write = [&](uint64_t entry, int rank) {
    if (rank >= p.top) return;
    p.top_tokens[row * p.top + rank] = (int32_t)~(uint32_t)entry;
    p.top_logprobs[row * p.top + rank] = all.z == 0.0f ? -__builtin_inff() : all.below(value_of((uint32_t)(entry >> 32))) * all.kUnit - log_z;
  };
  if (n <= 128) {  // a wave compares all of them with its share
    const uint64_t mine[2] = {lane < n ? found.entries[lane] : 0, 64 + lane < n ? found.entries[64 + lane] : 0};
    int rank[2] = {0, 0};
    for (int j = wave; j < n; j += T / 64) {
      const uint64_t other = found.entries[j];
      rank[0] += other > mine[0];
      rank[1] += other > mine[1];
    }
    if (rank[0]) atomicAdd(&found.ranks[lane], rank[0]);
    if (rank[1] && n > 64) atomicAdd(&found.ranks[64 + lane], rank[1]);
    __syncthreads();
    if (wave < 2 && 64 * wave + lane < n) write(mine[wave], found.ranks[64 * wave + lane]);
  } else {
    for (int i = threadIdx.x; i < n; i += T) {
      const uint64_t mine = found.entries[i];
      int rank = 0;
#pragma unroll 8
      for (int j = 0; j < n; ++j) rank += found.entries[j] > mine;
      write(mine, rank);
    }
  }
  for (int i = n + (int)threadIdx.x; i < p.top; i += T) {  // fewer values than that
    p.top_tokens[row * p.top + i] = -1;
    p.top_logprobs[row * p.top + i] = -__builtin_inff();
  }
}

// The row's given token and its logit, requested long before they are used
struct Given {
  int token = -1;
  float x = 0.0f;
  template <bool F32>
  __device__ __forceinline__ void request(const LogprobArgs& p, int64_t row, const Row<F32>& r) {
    if (!p.tokens) return;
    token = p.tokens[row];
    x = r.value(min(max(token, 0), p.V - 1));  // (no branch, which would wait for the token here)
  }
};

template <bool F32>
__device__ __forceinline__ void write_numbers(const LogprobArgs& p, int64_t row, const Given& given, const Sums<F32>& all, float log_z) {
  const bool none = all.z == 0.0f;  // everything masked
  if (p.lse) p.lse[row] = none ? -__builtin_inff() : (float)((double)all.m * (F32 ? 1.0 : 0.69314718055994531) + (double)log_z);
  if (p.entropy) p.entropy[row] = none ? 0.0f : log_z - all.t / all.z * all.kUnit;
  if (p.logprob) {
    float y = given.token < 0 ? 0.0f : __builtin_nanf("");
    if (given.token >= 0 && given.token < p.V) y = none ? -__builtin_inff() : all.below(given.x) * all.kUnit - log_z;
    p.logprob[row] = y;
  }
}

// One thread's part of blocks [from, to): every T-th, and one of the lead's and tail's values where `odd` says so.
template <bool F32, int T, int U, bool PAST, bool TRACK>
__device__ __forceinline__ Sums<F32> stream(const Row<F32>& r, int from, int to, bool odd) {
  Sums<F32> s;
  const int tid = threadIdx.x;
  float x[kOddEach];
#pragma unroll
  for (int i = 0; i < kOddEach; ++i) {
    const int at = tid + T * i;
    x[i] = odd && at < r.lead + r.tail ? r.value(r.place_of_odd(at)) : -__builtin_inff();
  }
  auto request = [&](int b0, uint4* v) {
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int b = b0 + tid + T * u;
      v[u] = Row<F32>::masked_block();
      if (b < to) v[u] = r.template block<PAST>(b);
    }
  };
  uint4 v[U], w[U];
  request(from, v);
  for (int b0 = from; b0 < to; b0 += 2 * T * U) {
    request(b0 + T * U, w);
    s.template add_blocks<U, TRACK>(v, b0);
    if (b0 + T * U >= to) break;
    request(b0 + 2 * T * U, v);
    s.template add_blocks<U, TRACK>(w, b0 + T * U);
  }
#pragma unroll
  for (int i = 0; i < kOddEach; ++i)
    if (odd && tid + T * i < r.lead + r.tail) {
      s.template meet<TRACK>(x[i], -1);
      s.add(x[i]);
    }
  return s;
}

// ---- a workgroup a row
template <bool F32, int T, int U, bool PAST, bool TRACK>
__global__ __launch_bounds__(T, 8) void logprobs_kernel(const LogprobArgs p) {
  __shared__ float of_wave[T / 64][3], of_group[kBound];
  __shared__ int larger[T / 64][kBound];
  __shared__ Found<T> found;
  __shared__ int passed[T], passing, passing_once;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int64_t row = blockIdx.x;
  const Row<F32> r(p, row, p.V <= kOddEach * T);
  Given given;
  given.request(p, row, r);
  const Sums<F32> mine = stream<F32, T, U, PAST, TRACK>(r, 0, r.blocks, true);
  if (p.top) {
    const float g = group_max<T / kBound>(mine.reached());
    if (tid % (T / kBound) == 0) of_group[tid / (T / kBound)] = g;
    if (tid < 128) found.ranks[tid] = 0;
    if (tid == 0) found.count = passing = passing_once = 0;
  }
  const Sums<F32> w = wave_sums(mine);
  if (lane == 0) {
    of_wave[wave][0] = w.m;
    of_wave[wave][1] = w.z;
    of_wave[wave][2] = w.t;
  }
  __syncthreads();
  if (!p.top) {
    if (wave > 0) return;
    const Sums<F32> all = join_waves<F32, T / 64>(of_wave);
    if (tid == 0) write_numbers<F32>(p, row, given, all, logf(all.z));
    return;
  }

  // Threads with such a value, and then their blocks spread over all waves: a thread's own, one after the other, would be as many memory latencies.  TRACK: where one batch of a
  // thread's blocks alone has one, as most do, no other is read again.
  auto pass = [&](float level, bool above) {
    if (!passes(mine.reached(), level, above)) return;
    if (!TRACK || mine.z != mine.z || passes(mine.others, level, above)) passed[atomicAdd(&passing, 1)] = tid;
    else if (mine.at >= 0) passed[T - 1 - atomicAdd(&passing_once, 1)] = mine.at + tid;
  };
  const int each = (r.blocks + T - 1) / T;
  auto look = [&](auto mode, float level, List& list) {
    constexpr int MODE = decltype(mode)::value;
    const int whole = passing * each, items = TRACK ? whole + passing_once * U : whole;
    for (int i0 = wave; i0 < items; i0 += T) {
      if (MODE != kList && found.is_full()) return;
      const int i = i0 + lane * (T / 64);
      int b = r.blocks;
      if (i < whole) b = passed[i / each] + i % each * T;
      else if (TRACK && i < items) b = passed[T - 1 - (i - whole) / U] + (i - whole) % U * T;
      look_at_block<F32, T, MODE>(r, b, b < r.blocks, p.top, level, list, found);
    }
    for (int i0 = wave * 64; i0 < r.lead + r.tail; i0 += T) {
      const int i = i0 + lane;
      const bool odd = i < r.lead + r.tail;
      look_at_value<F32, T, MODE>(r, odd ? r.place_of_odd(i) : 0, odd, p.top, level, list, found);
    }
  };
  find_top<F32, T, true>(r, p.top, bound_of<T>(of_group, larger, p.top), passing, passing_once, found, pass, look);
  const Sums<F32> all = join_waves<F32, T / 64>(of_wave);
  const float log_z = logf(all.z);
  write_top<F32, T>(p, row, all, log_z, found);
  if (tid == T - 1) write_numbers<F32>(p, row, given, all, log_z);
}

// ---- a workgroup a row that its registers hold: U blocks a thread (and its share of the lead and tail), so nothing is read twice
template <bool F32, int T, int U>
__global__ __launch_bounds__(T) void logprobs_short_kernel(const LogprobArgs p) {
  __shared__ float of_wave[T / 64][3], of_group[kBound];
  __shared__ int larger[T / 64][kBound];
  __shared__ Found<T> found;
  __shared__ int passed[T], passing;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int64_t row = blockIdx.x;
  const Row<F32> r(p, row, p.V <= kOddEach * T);
  const int odd = r.lead + r.tail;
  uint4 kept[U];
  float kept_odd[kOddEach];
#pragma unroll
  for (int u = 0; u < U; ++u) {
    kept[u] = Row<F32>::masked_block();
    if (tid + T * u < r.blocks) kept[u] = r.template block<false>(tid + T * u);
  }
#pragma unroll
  for (int i = 0; i < kOddEach; ++i) kept_odd[i] = tid + T * i < odd ? r.value(r.place_of_odd(tid + T * i)) : -__builtin_inff();
  Given given;
  given.request(p, row, r);

  Sums<F32> mine;
  mine.template meet<false>(Row<F32>::template largest<U>(kept), 0);
#pragma unroll
  for (int i = 0; i < kOddEach; ++i)
    if (64 * wave + T * i < odd) mine.template meet<false>(kept_odd[i], 0);
#pragma unroll
  for (int u = 0; u < U; ++u)
    if (64 * wave + T * u < r.blocks) mine.add_block(kept[u], 64 * wave + T * u + 64 <= r.blocks);
#pragma unroll
  for (int i = 0; i < kOddEach; ++i)
    if (64 * wave + T * i < odd) mine.add(kept_odd[i]);
  const float reached = mine.reached();
  if (p.top) {
    const float g = group_max<T / kBound>(reached);
    if (tid % (T / kBound) == 0) of_group[tid / (T / kBound)] = g;
    if (tid < 128) found.ranks[tid] = 0;
    if (tid == 0) found.count = passing = 0;
  }
  const Sums<F32> w = wave_sums(mine);
  if (lane == 0) {
    of_wave[wave][0] = w.m;
    of_wave[wave][1] = w.z;
    of_wave[wave][2] = w.t;
  }
  __syncthreads();
  if (!p.top) {
    if (wave > 0) return;
    const Sums<F32> all = join_waves<F32, T / 64>(of_wave);
    if (tid == 0) write_numbers<F32>(p, row, given, all, logf(all.z));
    return;
  }
  // More than one block a thread: as in the kernel above.  Looked for in these registers they took 1 to 2 us longer, since a wave's threads have theirs in different blocks.
  auto pass = [&](float level, bool above) {
    if (passes(reached, level, above)) passed[atomicAdd(&passing, 1)] = tid;
  };
  auto look = [&](auto mode, float level, List& list) {
    constexpr int MODE = decltype(mode)::value;
    auto see = [&](bool has, float x, int place) {
      if constexpr (MODE == kList) list.offer(has, x, place, p.top, level);
      else if (has && wanted<MODE>(x, level)) found.add(order_of(x), ~(uint32_t)place);
    };
    if constexpr (U == 1) {
      if (MODE == kList || passes(reached, level, MODE == kAbove)) {
        float x[Row<F32>::kVec];
        Row<F32>::unpack(kept[0], x);
#pragma unroll
        for (int i = 0; i < Row<F32>::kVec; ++i) see(tid < r.blocks, x[i], r.place_of_block(tid) + i);
      }
    } else {
      const int items = passing * U;
      for (int i0 = wave; i0 < items; i0 += T) {
        if (MODE != kList && found.is_full()) return;
        const int i = i0 + lane * (T / 64), b = i < items ? passed[i / U] + i % U * T : r.blocks;
        look_at_block<F32, T, MODE>(r, b, b < r.blocks, p.top, level, list, found);
      }
    }
#pragma unroll
    for (int i = 0; i < kOddEach; ++i)
      if (64 * wave + T * i < odd) see(tid + T * i < odd, kept_odd[i], r.place_of_odd(tid + T * i));
  };
  find_top<F32, T, (U > 1)>(r, p.top, bound_of<T>(of_group, larger, p.top), passing, passing, found, pass, look);
  const Sums<F32> all = join_waves<F32, T / 64>(of_wave);
  const float log_z = logf(all.z);
  write_top<F32, T>(p, row, all, log_z, found);
  if (tid == T - 1) write_numbers<F32>(p, row, given, all, log_z);
}

// ---- few rows: parts of them
template <bool F32>
__global__ __launch_bounds__(kSplitThreads) void logprobs_part_kernel(const LogprobArgs p) {
  __shared__ float of_wave[kSplitThreads / 64][3];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, part = blockIdx.x;
  const int64_t row = blockIdx.y;
  const Row<F32> r(p, row);
  const int from = min((int64_t)part * p.blocks_per_part, (int64_t)r.blocks), to = min((int64_t)from + p.blocks_per_part, (int64_t)r.blocks);
  const Sums<F32> mine = stream<F32, kSplitThreads, 2, false, false>(r, from, to, part == 0);
  float* out = p.parts + (row * p.splits + part) * kPartValues;
  if (p.top) {
    const float g = group_max<kSplitThreads / kGroups>(mine.reached());
    if (tid % (kSplitThreads / kGroups) == 0) out[3 + tid / (kSplitThreads / kGroups)] = g;
  }
  const Sums<F32> w = wave_sums(mine);
  if (lane == 0) {
    of_wave[wave][0] = w.m;
    of_wave[wave][1] = w.z;
    of_wave[wave][2] = w.t;
  }
  __syncthreads();
  if (wave > 0) return;
  const Sums<F32> all = join_waves<F32, kSplitThreads / 64>(of_wave);
  if (lane == 0) {
    out[0] = all.m;
    out[1] = all.z;
    out[2] = all.t;
  }
}

// the most groups of all parts of a row
constexpr int kMostParts = 128, kJoinGroups = kMostParts * kGroups / kJoinThreads;

template <bool F32, bool TOP>
__global__ __launch_bounds__(TOP ? kJoinThreads : 64) void logprobs_join_kernel(const LogprobArgs p) {
  constexpr int T = TOP ? kJoinThreads : 64, kWaves = T / 64;
  __shared__ float of_wave[kWaves][3], of_group[kBound];
  __shared__ int larger[TOP ? kWaves : 1][kBound];
  __shared__ Found<T> found;
  __shared__ int passing;
  __shared__ uint16_t passed[TOP ? kMostParts * kGroups : 1];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int64_t row = blockIdx.x;
  const Row<F32> r(p, row);
  const float* parts = p.parts + row * p.splits * kPartValues;
  float g[kJoinGroups];
  if constexpr (TOP) {
    float most = -__builtin_inff();
#pragma unroll
    for (int i = 0; i < kJoinGroups; ++i) {  // a wave: the groups of part wave + kWaves * i
      const int part = wave + kWaves * i;
      g[i] = part < p.splits ? parts[part * kPartValues + 3 + lane] : -__builtin_inff();
      most = fmaxf(most, g[i]);
    }
    most = group_max<T / kBound>(most);
    if (tid % (T / kBound) == 0) of_group[tid / (T / kBound)] = most;
    if (tid < 128) found.ranks[tid] = 0;
    if (tid == 0) found.count = passing = 0;
  }
  Given given;
  given.request(p, row, r);
  Sums<F32> s;
  for (int part = tid; part < p.splits; part += T) {
    Sums<F32> q;
    q.m = parts[part * kPartValues];
    q.z = parts[part * kPartValues + 1];
    q.t = parts[part * kPartValues + 2];
    const float m = fmaxf(s.m, q.m);
    s.refer_to(m);
    q.refer_to(m);
    s.z += q.z;
    s.t += q.t;
  }
  s = wave_sums(s);
  if constexpr (!TOP) {
    if (tid == 0) write_numbers<F32>(p, row, given, s, logf(s.z));
  } else {
    if (lane == 0) {
      of_wave[wave][0] = s.m;
      of_wave[wave][1] = s.z;
      of_wave[wave][2] = s.t;
    }
    __syncthreads();
    auto pass = [&](float level, bool above) {
#pragma unroll
      for (int i = 0; i < kJoinGroups; ++i) {
        const int part = wave + kWaves * i;
        if (part < p.splits && passes(g[i], level, above)) passed[atomicAdd(&passing, 1)] = (uint16_t)(part * kGroups + lane);
      }
    };
    // the values of each group that passed, kLanes threads of its part, by as many lanes: a wave takes 64 / kLanes groups at a time, neighbours of the list going to different waves
    constexpr int kLanes = kSplitThreads / kGroups;
    auto look = [&](auto mode, float level, List& list) {
      constexpr int MODE = decltype(mode)::value;
      const int n = passing;
      for (int e0 = wave; e0 < n; e0 += kWaves * (64 / kLanes)) {
        if (MODE != kList && found.is_full()) return;
        const int e = e0 + lane / kLanes * kWaves;
        const int id = e < n ? passed[e] : 0, part = id / kGroups, thread = id % kGroups * kLanes + lane % kLanes;
        const int from = min((int64_t)part * p.blocks_per_part, (int64_t)r.blocks), to = e < n ? min((int64_t)from + p.blocks_per_part, (int64_t)r.blocks) : 0;
        for (int j = thread; j < p.blocks_per_part; j += kSplitThreads)  // (blocks_per_part is a multiple of kSplitThreads: every lane turns as often)
          look_at_block<F32, T, MODE>(r, from + j, from + j < to, p.top, level, list, found);
        const bool odd = e < n && part == 0 && thread < r.lead + r.tail;
        look_at_value<F32, T, MODE>(r, odd ? r.place_of_odd(thread) : 0, odd, p.top, level, list, found);
      }
    };
    find_top<F32, T, true>(r, p.top, bound_of<T>(of_group, larger, p.top), passing, passing, found, pass, look);
    const Sums<F32> all = join_waves<F32, kWaves>(of_wave);
    const float log_z = logf(all.z);
    write_top<F32, T>(p, row, all, log_z, found);
    if (tid == T - 1) write_numbers<F32>(p, row, given, all, log_z);
  }
}

// Parts of a row: 1 (a workgroup a row) where the rows alone keep the CUs busy.
struct Split {
  int parts, blocks;
};
Split split_of(int64_t M, int64_t V, int type) {
  const int64_t blocks = V / (type == QQQ_LOGITS_FP32 ? 4 : 8);
  // us in a graph, split / whole, the largest 5 asked for.  fp16: one row of 48000 7.9 / 7.4, of 64000 7.8 / 8.3; 16 of 64000 8.7 / 8.8, of 100000 9.8 / 11.0; 32 of 64000 9.6 / 8.8, of 100000 9.5 / 11.0;
  // 64 of 100000 10.7 / 11.1.  fp32: one of 32000 7.4 / 6.6, of 42000 7.4 / 7.7; 16 of 50000 8.7 / 8.4; 32 of 64000 8.8 / 9.0; 64 of 64000 10.3 / 9.1.  (An fp32 value counts for 1.4.)
  if (M > 64 || V * (type == QQQ_LOGITS_FP32 ? 7 : 5) * 64 <= 5 * 56000 * (64 + M)) return {1, 0};
  // a block a thread where that leaves no more than four workgroups a CU
  int64_t each = 1;
  while (each < 64 && M * ((blocks + each * kSplitThreads - 1) / (each * kSplitThreads)) > 4 * num_cus()) each *= 2;
  while ((blocks + each * kSplitThreads - 1) / (each * kSplitThreads) > kMostParts) each *= 2;
  const int64_t parts = (blocks + each * kSplitThreads - 1) / (each * kSplitThreads);
  if (parts < 2) return {1, 0};
  return {(int)parts, (int)(each * kSplitThreads)};
}

template <bool F32>
int launch_typed(LogprobArgs& p, int64_t M, const Split& s, hipStream_t st) {
  const char* way = "logprobs in parts";
  if (s.parts == 1) {
    const bool past = M * p.V * (F32 ? 4 : 2) > kLastCacheBytes;
#define QQQ_LP(T, U, PAST, TRACK)                                                                                              \
  do {                                                                                                                       \
    hipLaunchKernelGGL((logprobs_kernel<F32, T, U, PAST, TRACK>), dim3((unsigned)M), dim3(T), 0, st, p);                     \
    way = "logprobs in turns threads=" #T " past=" #PAST " tracked=" #TRACK;                                                 \
  } while (0)
    // Threads a row, us (256 / 512 / 1024): a row a CU or less 400 KB 35.9 / 20.9 / 17.5 (100 rows, top 20); many rows 40 KB 62 / 87 / 180
    // (8000 rows, top 5), 256 KB 248 / 203 / 190 (4096 rows, top 20), 166 / 161 / 167 (top 1); 777 rows of 131 KB, sums only, 24.8 / 26.6 / 31.0
    const int64_t bytes = (int64_t)p.V * (F32 ? 4 : 2);
    // Rows of up to 256 KB, no more of them than CUs, in registers.  us in a graph with 512 / 1024 threads: one of 64 KB, the largest 20 6.9 / 7.3, the largest 64 8.4 / 8.1; of 120 KB, sums
    // 6.0 / 5.6, 5 8.2 / 8.4, 64 11.0 / 9.6; 48 of 200 KB, 5 8.7 / 8.5, 64 12.4 / 10.0; read in turns (the kernel above) 4.7, 7.2, 9.6 for 64 KB, 9.0, 12.3 for the last
    const int64_t row_blocks = p.V / (F32 ? 4 : 8), a_thread = std::max<int64_t>((row_blocks + 511) / 512, 1);
    // Twice as many of up to 64 KB: 400 of 64 KB, the largest 20 10.2, in turns 11.6; more of them, or longer ones, are sooner in turns (777 of 64 KB 16.6 and 16.4, 400 of 131 KB 22.0 and 17.2)
    if (a_thread <= (M <= num_cus() ? 32 : M <= 2 * num_cus() ? 8 : 0)) {
#define QQQ_LP_SHORT(T, U)                                                                                                   \
  do {                                                                                                                       \
    hipLaunchKernelGGL((logprobs_short_kernel<F32, T, U>), dim3((unsigned)M), dim3(T), 0, st, p);                            \
    way = "logprobs in registers threads=" #T " blocks=" #U;                                                                 \
  } while (0)
      if (a_thread <= 1) QQQ_LP_SHORT(512, 1);
      else if (a_thread <= 2) QQQ_LP_SHORT(512, 2);
      else if (a_thread <= 4) QQQ_LP_SHORT(512, 4);
      else if (a_thread <= 8) QQQ_LP_SHORT(512, 8);
      else if (a_thread <= 16 && p.top <= 32) QQQ_LP_SHORT(512, 16);
      else if (a_thread <= 16) QQQ_LP_SHORT(1024, 8);
      else QQQ_LP_SHORT(1024, 16);
#undef QQQ_LP_SHORT
    } else if (M <= num_cus()) {
      QQQ_LP(1024, 4, false, false);
    } else if (bytes > 64 << 10 && p.top * bytes >= 1800 << 10) {
      // (TRACK, us without / with: 4096 rows of 256 KB, top 4 167 / 165, 8 172 / 166, 20 195 / 171, 64 276 / 183; of 128 KB, top 8 90 / 91, 20 99 / 93; 2100 rows of 80 KB, top 20
      // 40 / 43, 64 49 / 48)
      if (past) QQQ_LP(512, 2, true, true);
      else QQQ_LP(512, 2, false, true);
    } else if (bytes > 64 << 10 && (p.top > 0 || M >= 8 * num_cus())) {
      if (past) QQQ_LP(512, 2, true, false);
      else QQQ_LP(512, 2, false, false);
    } else if (past) {
      QQQ_LP(256, 2, true, false);
    } else {
      QQQ_LP(256, 2, false, false);
    }
#undef QQQ_LP
  } else {
    p.splits = s.parts;
    p.blocks_per_part = s.blocks;
    hipLaunchKernelGGL((logprobs_part_kernel<F32>), dim3((unsigned)s.parts, (unsigned)M), dim3(kSplitThreads), 0, st, p);
    if (p.top) hipLaunchKernelGGL((logprobs_join_kernel<F32, true>), dim3((unsigned)M), dim3(kJoinThreads), 0, st, p);
    else hipLaunchKernelGGL((logprobs_join_kernel<F32, false>), dim3((unsigned)M), dim3(64), 0, st, p);
  }
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return set_error(QQQ_ERR_HIP, "logprobs launch: %s", hipGetErrorString(e));
  if (s.parts > 1) route_note("%s=%d", way, s.parts);
  else route_note("%s", way);
  return QQQ_OK;
}

}  // namespace

size_t logprobs_bytes(int64_t M, int64_t V, int type) {
  const Split s = split_of(M, V, type);
  return s.parts == 1 ? 0 : (size_t)M * s.parts * kPartValues * sizeof(float);
}

int launch_logprobs(const void* logits, int64_t ld, int type, int64_t M, int64_t V, const int32_t* tokens, int top, float* logprob, float* entropy,
                    float* lse, int32_t* top_tokens, float* top_logprobs, void* workspace, hipStream_t st) {
  LogprobArgs p = {};
  p.logits = static_cast<const char*>(logits);
  p.row_bytes = ld * (type == QQQ_LOGITS_FP32 ? 4 : 2);
  p.tokens = tokens;
  p.logprob = logprob;
  p.entropy = entropy;
  p.lse = lse;
  p.top_tokens = top_tokens;
  p.top_logprobs = top_logprobs;
  p.parts = static_cast<float*>(workspace);
  p.V = (int)V;
  p.top = top;
  const Split s = split_of(M, V, type);
  return type == QQQ_LOGITS_FP32 ? launch_typed<true>(p, M, s, st) : launch_typed<false>(p, M, s, st);
}

}  // namespace qqq
