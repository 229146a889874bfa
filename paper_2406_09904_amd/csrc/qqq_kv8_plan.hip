// The tables of a serving step from what its sessions hold and bring, and the return of a session's pages (qqq_serve.h).
//
// Sequence b brings n_b tokens: cu is the sequences' prefix sum of n_b, and the places of its fresh pages in the stack are a prefix sum of
// fresh_b = len_b / P - held_b / P.  Both sums saturate at 2^30 (no count that is used passes it), so they stay in 32 bits whatever the tensors hold.
// The sums are made in registers by lane moves; the tables' entries and the rows' places are then copies, 8 bytes moved for each.  A workgroup may fill what its sums tell only where
// no other still reads what it writes: held_after in place asks for one workgroup, or for a launch of its own for the sums.
// What bounds it: up to 1024 sequences the time that a launch and four dependent reads take (ids, held, entries, the stack: 2.1 us for one sequence, 2.7 for 64 of 125 entries, 3.5
// for 200 of 1000); for more the sums' one workgroup (2048 sequences: 4.3 us) and the copies (2048 tables of about 1000 entries, 17 MB: 6.1 us).
#include <limits.h>

#include <algorithm>

#include "qqq_plan.h"

namespace qqq {

namespace {

constexpr int kScanThreads = 1024, kFillThreads = 256;
constexpr int kMost = 1 << 30;

__device__ __forceinline__ int add_saturating(int a, int b) { return (int)min((uint32_t)a + (uint32_t)b, (uint32_t)kMost); }

// Sum of the lanes up to this one, saturating (0 <= v <= kMost)
__device__ __forceinline__ int wave_inclusive_sum(int v) {
  auto add = [&](int moved) { v = add_saturating(v, moved); };
  add(__builtin_amdgcn_update_dpp(0, v, 0x111, 0xF, 0xF, false));  // row_shr:1, 2, 4, 8 in rows of 16 lanes (none: 0)
  add(__builtin_amdgcn_update_dpp(0, v, 0x112, 0xF, 0xF, false));
  add(__builtin_amdgcn_update_dpp(0, v, 0x114, 0xF, 0xF, false));
  add(__builtin_amdgcn_update_dpp(0, v, 0x118, 0xF, 0xF, false));
  add(__builtin_amdgcn_update_dpp(0, v, 0x142, 0xA, 0xF, false));  // row_bcast:15: a row's last to the next, rows 1 and 3
  add(__builtin_amdgcn_update_dpp(0, v, 0x143, 0xC, 0xF, false));  // row_bcast:31: the second row's last to rows 2 and 3
  return v;
}

// Sum of the values of the T threads before this one, and of all, saturating.  T of 64: of a wave, without a barrier.
template <int T>
__device__ __forceinline__ int block_exclusive_sum(int v, int* smem, int& total) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int sum = wave_inclusive_sum(v);
  int before = __builtin_amdgcn_update_dpp(0, sum, 0x138, 0xF, 0xF, false);  // wave_shr:1
  if constexpr (T == 64) {
    total = __builtin_amdgcn_readlane(sum, 63);
    return before;
  }
  if (lane == 63) smem[wave] = sum;
  __syncthreads();
  // the waves' sums the same way, in each of them
  const int waves = wave_inclusive_sum(lane < T / 64 ? smem[lane] : 0);
  total = __builtin_amdgcn_readlane(waves, 63);
  if (wave > 0) before = add_saturating(before, __builtin_amdgcn_readlane(waves, wave - 1));
  __syncthreads();
  return before;
}

struct Sequence {
  int session, held, len, row, top;  // top: entries of the stack that are left when its turn comes (below 0: lacking)
};

// One sequence's entries and rows, every `step`-th from `from` on.  early: what the session's entries from, from + step, .. hold, as far as it was read before.
template <int EARLY = 0>
__device__ __forceinline__ void fill(const PlanArgs& p, int b, const Sequence& s, int64_t from, int64_t step, const int* early = nullptr) {
  const int closed = s.len >> p.shift, had = s.held >> p.shift, n = s.len - s.held;
  if (closed > 0) {
    int32_t* own = p.pages + (int64_t)s.session * p.pages_stride;
    int32_t* table = p.table + (int64_t)b * p.table_stride;
    auto entry = [&](int64_t j, int held_page) {
      int page = held_page;
      if (j >= had) {
        const int64_t place = s.top - 1 - (j - had);
        page = place >= 0 ? p.free_pages[place] : -1;
        own[j] = page;
      }
      table[j] = page;
    };
    int64_t j = (p.same_table ? had : 0) + from;
    if (!p.same_table) {
#pragma unroll
      for (int e = 0; e < EARLY; ++e, j += step)
        if (j < closed) entry(j, early[e]);
    }
    for (; j < closed; j += step) entry(j, j < had ? own[j] : 0);
  }
  if (p.sequence)
    for (int64_t i = from; i < n; i += step) p.sequence[s.row + i] = b;
  if (p.positions)
    for (int64_t i = from; i < n; i += step) p.positions[s.row + i] = s.held + (int)i;
}

// The sums over sequences 0 .. until - 1 by T threads, kEach consecutive sequences each: met(b, its numbers) for all of them, in the thread that has it.
struct Totals {
  int rows = 0, taken = 0;
};
template <int T, int kEach, class Met>
__device__ __forceinline__ Totals make_sums(const PlanArgs& p, int64_t until, int* smem, Met met) {
  const int tid = threadIdx.x, count = min(max(*p.free_count, 0), p.pool);
  Totals sum;  // of the sequences before this turn's
  for (int64_t first = 0; first < until; first += T * kEach) {
    int session[kEach], held[kEach], n[kEach], all_n = 0;
#pragma unroll
    for (int e = 0; e < kEach; ++e) {
      const int64_t b = first + (int64_t)tid * kEach + e;
      session[e] = b >= until ? -1 : p.ids ? p.ids[b] : (int)b;
      n[e] = b >= until ? 0 : p.new_tokens[b];
      if ((uint32_t)session[e] >= (uint32_t)p.sessions) session[e] = -1;
    }
#pragma unroll
    for (int e = 0; e < kEach; ++e) {
      held[e] = session[e] >= 0 ? min(max(p.held[session[e]], 0), p.max_len) : 0;
      n[e] = session[e] >= 0 ? min(min(max(n[e], 0), p.max_new), p.max_len - held[e]) : 0;
      all_n = add_saturating(all_n, n[e]);
    }
    int all;
    int row = add_saturating(sum.rows, block_exclusive_sum<T>(all_n, smem, all));
    sum.rows = add_saturating(sum.rows, all);
    int row_of[kEach], fresh[kEach], all_fresh = 0;
#pragma unroll
    for (int e = 0; e < kEach; ++e) {
      row_of[e] = min(row, p.tokens);
      row = add_saturating(row, n[e]);
      n[e] = min(n[e], p.tokens - row_of[e]);  // rows that the step's tensors do not have are not taken
      fresh[e] = (held[e] + n[e] >> p.shift) - (held[e] >> p.shift);
      all_fresh = add_saturating(all_fresh, fresh[e]);
    }
    int before = add_saturating(sum.taken, block_exclusive_sum<T>(all_fresh, smem, all));
    sum.taken = add_saturating(sum.taken, all);
#pragma unroll
    for (int e = 0; e < kEach; ++e) {
      const int64_t b = first + (int64_t)tid * kEach + e;
      if (b < until) met(b, Sequence{session[e], held[e], held[e] + n[e], row_of[e], count - before});
      before = add_saturating(before, fresh[e]);
    }
  }
  return sum;
}
__device__ __forceinline__ void write_sequence(const PlanArgs& p, int64_t b, const Sequence& s) {
  p.kv_len[b] = s.len;
  p.cu[b] = s.row;
  if (s.session >= 0) p.held_after[s.session] = s.len;
}
__device__ __forceinline__ void write_totals(const PlanArgs& p, const Totals& sum) {
  const int count = min(max(*p.free_count, 0), p.pool);
  p.cu[p.sequences] = min(sum.rows, p.tokens);
  *p.free_count_after = max(count - sum.taken, 0);
  if (p.lacking) *p.lacking = max(sum.taken - count, 0);
}

// Few sequences and entries: all by one workgroup, the sums by its first wave
__global__ __launch_bounds__(kScanThreads) void kv8_plan_small_kernel(const PlanArgs p) {
  __shared__ Sequence seqs[64];
  const int tid = threadIdx.x;
  // as many threads for a sequence's tables as there are, a wave at least
  const int lanes = p.sequences <= 1 ? kScanThreads : max(64, kScanThreads >> (32 - __clz(p.sequences - 1)));
  // A group of threads has up to four sequences, and their first entries are on their way before the sums are known
  constexpr int kMine = 4, kEarly = 2;
  int early[kMine][kEarly], session[kMine];
#pragma unroll
  for (int i = 0; i < kMine; ++i) {
    const int b = tid / lanes + kScanThreads / lanes * i;
    session[i] = b >= p.sequences ? -1 : p.ids ? p.ids[b] : b;
  }
#pragma unroll
  for (int i = 0; i < kMine; ++i)
#pragma unroll
    for (int e = 0; e < kEarly; ++e) {
      const int j = tid % lanes + lanes * e;
      early[i][e] = 0;
      if ((uint32_t)session[i] < (uint32_t)p.sessions && j < p.columns && !p.same_table) early[i][e] = p.pages[(int64_t)session[i] * p.pages_stride + j];
    }
  if (tid < 64) {
    const Totals sum = make_sums<64, 1>(p, p.sequences, nullptr, [&](int64_t b, const Sequence& s) {
      write_sequence(p, b, s);
      seqs[b] = s;
    });
    if (tid == 0) write_totals(p, sum);
  }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < kMine; ++i) {
    const int b = tid / lanes + kScanThreads / lanes * i;
    if (b < p.sequences) fill<kEarly>(p, b, seqs[b], tid % lanes, lanes, early[i]);
  }
}

// More: the sums by one workgroup of T threads, then the fill kernel
template <int T, int E>
__global__ __launch_bounds__(T) void kv8_plan_sums_kernel(const PlanArgs p) {
  __shared__ int smem[T / 64];
  const Totals sum = make_sums<T, E>(p, p.sequences, smem, [&](int64_t b, const Sequence& s) {
    write_sequence(p, b, s);
    p.top[b] = s.top;
  });
  if (threadIdx.x == 0) write_totals(p, sum);
}

// Where what holds after the step goes to other memory, so that held and the stack's height stay as they are: one launch, in which each workgroup makes the sums up to its
// sequence by itself (T of its threads do)
template <int T, int E>
__global__ __launch_bounds__(kFillThreads) void kv8_plan_each_kernel(const PlanArgs p) {
  __shared__ int smem[T / 64];
  __shared__ Sequence mine;
  const int64_t b = blockIdx.x;
  if (T == kFillThreads || threadIdx.x < T) {
    const Totals sum = make_sums<T, E>(p, b + 1, smem, [&](int64_t i, const Sequence& s) {
      if (i < b) return;
      mine = s;
      if (blockIdx.y == 0) write_sequence(p, b, s);
    });
    if (blockIdx.y == 0 && b == p.sequences - 1 && threadIdx.x == 0) write_totals(p, sum);
  }
  __syncthreads();
  fill(p, (int)b, mine, (int64_t)blockIdx.y * kFillThreads + threadIdx.x, (int64_t)gridDim.y * kFillThreads);
}

// The tables and rows of many sequences, gridDim.y workgroups for each
__global__ __launch_bounds__(kFillThreads) void kv8_plan_fill_kernel(const PlanArgs p) {
  const int b = blockIdx.x;
  Sequence s;
  s.session = p.ids ? p.ids[b] : b;
  if ((uint32_t)s.session >= (uint32_t)p.sessions) return;
  s.len = p.kv_len[b];
  s.row = p.cu[b];
  s.held = s.len - (p.cu[b + 1] - s.row);
  s.top = p.top[b];
  fill(p, b, s, (int64_t)blockIdx.y * kFillThreads + threadIdx.x, (int64_t)gridDim.y * kFillThreads);
}

// The pages of sessions that end.  A wave a session counts its pages and later, when their place in the stack is known, copies them: a row may hold entries
// that are no page.  One workgroup, bound by its own loads in flight: 4 sessions of 2000 pages 12 us in a graph, 64 of 125 6.9, 2500 of 100 175.
__global__ __launch_bounds__(kScanThreads) void kv8_release_kernel(const PlanArgs p) {
  __shared__ int smem[kScanThreads / 64];
  __shared__ int session_of[kScanThreads], closed_of[kScanThreads], pages_of[kScanThreads];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  constexpr int kWaves = kScanThreads / 64;
  auto is_page = [&](int page) { return page >= 0; };  // (any of the cache: the stack may hold a part of its pages)
  int count = min(max(*p.free_count, 0), p.pool);
  for (int64_t first = 0; first < p.sequences; first += kScanThreads) {
    const int here = (int)min((int64_t)kScanThreads, p.sequences - first);
    // A session may be listed twice: the first place in the list has its pages.  Every place goes to where the session's length was, as a number below all lengths, the least stays, and
    // who met the length itself hands it to that place.
    int session = -1, length = 0;
    if (tid < here) {
      session = p.ids ? p.ids[first + tid] : (int)first + tid;
      if ((uint32_t)session >= (uint32_t)p.sessions) session = -1;
      session_of[tid] = max(session, 0);
      closed_of[tid] = 0;
      if (session >= 0) length = atomicMin(&p.held_after[session], INT_MIN + tid);
    }
    __syncthreads();
    if (session >= 0 && length >= 0) closed_of[atomicExch(&p.held_after[session], 0) & (kScanThreads - 1)] = min(length >> p.shift, p.columns);
    __syncthreads();
    if (length < 0) {  // listed before, or a length below 0
      atomicExch(&p.held_after[session], 0);
      __threadfence();
    }
    for (int i = wave; i < here; i += kWaves) {
      const int32_t* own = p.pages + (int64_t)session_of[i] * p.pages_stride;
      int n = 0;
      for (int j = lane; j < closed_of[i]; j += 64) n += is_page(own[j]);
#pragma unroll
      for (int d = 32; d; d >>= 1) n += __shfl_xor(n, d);
      if (lane == 0) pages_of[i] = n;
    }
    __syncthreads();
    int all;
    const int before = block_exclusive_sum<kScanThreads>(tid < here ? pages_of[tid] : 0, smem, all);
    if (tid < here) pages_of[tid] = add_saturating(count, before);
    __syncthreads();
    for (int i = wave; i < here; i += kWaves) {
      const int32_t* own = p.pages + (int64_t)session_of[i] * p.pages_stride;
      int at = pages_of[i];
      for (int j0 = 0; j0 < closed_of[i]; j0 += 64) {
        const int page = j0 + lane < closed_of[i] ? own[j0 + lane] : -1;
        const uint64_t have = __ballot(is_page(page));
        const int place = at + __popcll(have & ((1ull << lane) - 1));
        if (is_page(page) && place < p.pool) p.free_out[place] = page;
        at = add_saturating(at, __popcll(have));
      }
    }
    count = min(add_saturating(count, all), p.pool);
    __syncthreads();
  }
  if (tid == 0) *p.free_count_after = count;
}

// What holds afterwards in other memory: a workgroup a sequence, up to 1024 of them (a turn of 256 threads; each reads what all before it hold).  us in a graph, this and two
// launches: one sequence of one entry 2.1 and 3.4, of 16384 2.8 and 4.4; 64 of 128 2.7 and 4.2, of 4096 3.1 and 4.7; 200 of 1024 3.5 and 5.2; 1000 of 128 4.9 and 5.2, of 1024 5.7 and
// 6.1; 1500 of 128 7.8 and 6.3; 2500 of 128 13 and 8.6.
bool each_by_itself(const PlanArgs& p) {
  return p.sequences > 0 && p.sequences <= 4 * kFillThreads && p.held_after != p.held && p.free_count_after != p.free_count;
}
// In place, where a workgroup's sums must be there before another's are written: one workgroup while it moves the entries and rows about as soon as a second launch would.  Measured in
// a graph, us with one launch and with two: one sequence of 1 entry 2.4 and 3.4, of 4096 3.1 and 4.2, of 16384 5.8 and 4.3; 37 of 256 4.9 and 4.2; 64 of 16 4.2 and 4.2, of 1024 16.7
// and 4.5.  Outside a graph a second launch also costs the host 2 us.  More than 64 sequences, whose sums take barriers, are behind in one workgroup at every length (200 of one
// entry 6.0 and 4.2, 1024 of one 21 and 4.4).
bool in_one_workgroup(const PlanArgs& p) {
  return p.sequences <= 64 && (int64_t)p.sequences * ((p.max_len >> p.shift) + (int64_t)p.max_new) <= kPlanSmall;
}

int launched(const char* what, const char* name) {
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return set_error(QQQ_ERR_HIP, "%s launch: %s", what, hipGetErrorString(e));
  route_note("%s", name);
  return QQQ_OK;
}

}  // namespace

size_t kv8_plan_bytes(const PlanArgs& p) { return in_one_workgroup(p) || each_by_itself(p) ? 0 : (size_t)p.sequences * sizeof(int32_t); }

int launch_kv8_plan(const PlanArgs& p, hipStream_t st) {
  if (!each_by_itself(p) && in_one_workgroup(p)) {
    hipLaunchKernelGGL(kv8_plan_small_kernel, dim3(1), dim3(kScanThreads), 0, st, p);
    return launched("plan", "plan one workgroup");
  }
  const int64_t most = std::max(p.max_len >> p.shift, std::min(p.max_new, p.tokens));  // entries or rows of a sequence
  const int64_t parts = std::min<int64_t>(std::max<int64_t>((most + 4 * kFillThreads - 1) / (4 * kFillThreads), 1), std::max(8 * num_cus() / p.sequences, 1));
  const dim3 grid((unsigned)p.sequences, (unsigned)parts);
  if (each_by_itself(p)) {
    // (a sequence a thread where that covers them, us in a graph with 1, 2 and 4: 200 of one entry 2.9, 3.1, 3.6; 512 of one 3.8, 3.3, 3.8; 1000 of one 5.7, 4.9, 4.5)
    if (p.sequences <= 64) hipLaunchKernelGGL((kv8_plan_each_kernel<64, 1>), grid, dim3(kFillThreads), 0, st, p);
    else if (p.sequences <= kFillThreads) hipLaunchKernelGGL((kv8_plan_each_kernel<kFillThreads, 1>), grid, dim3(kFillThreads), 0, st, p);
    else if (p.sequences <= 2 * kFillThreads) hipLaunchKernelGGL((kv8_plan_each_kernel<kFillThreads, 2>), grid, dim3(kFillThreads), 0, st, p);
    else hipLaunchKernelGGL((kv8_plan_each_kernel<kFillThreads, 4>), grid, dim3(kFillThreads), 0, st, p);
    return launched("plan", "plan one launch");
  }
  // (1000 of one entry, fill kernel too, 4.4, 4.8, 6.0; 2048 of one 6.4, 6.1, 7.5; 4000 of one 9.4, 9.1, 10.5)
  if (p.sequences <= 64) hipLaunchKernelGGL((kv8_plan_sums_kernel<64, 1>), dim3(1), dim3(64), 0, st, p);
  else if (p.sequences <= kScanThreads) hipLaunchKernelGGL((kv8_plan_sums_kernel<kScanThreads, 1>), dim3(1), dim3(kScanThreads), 0, st, p);
  else hipLaunchKernelGGL((kv8_plan_sums_kernel<kScanThreads, 2>), dim3(1), dim3(kScanThreads), 0, st, p);
  if (int rc = launched("plan", "plan sums")) return rc;
  hipLaunchKernelGGL(kv8_plan_fill_kernel, grid, dim3(kFillThreads), 0, st, p);
  return launched("plan", "fill");
}

int launch_kv8_release(const PlanArgs& p, hipStream_t st) {
  hipLaunchKernelGGL(kv8_release_kernel, dim3(1), dim3(kScanThreads), 0, st, p);
  return launched("release", "release");
}

}  // namespace qqq
