// The tables of a serving step from what its sessions hold and bring, and the return of a session's pages (qqq_serve.h).
//
// Sequence b brings n_b tokens: cu is the sequences' prefix sum of n_b, and the places of its fresh pages in the stack are a prefix sum of
// fresh_b = len_b / P - held_b / P.  Both sums saturate at 2^30 (no count that is used passes it), so they stay in 32 bits whatever the tensors hold.
// One workgroup makes the sums, a sequence a thread; the tables' entries and the rows' places are then copies, 8 bytes moved for each.
#include <algorithm>

#include "qqq_plan.h"

namespace qqq {

namespace {

constexpr int kScanThreads = 1024, kFillThreads = 256;
constexpr int kMost = 1 << 30;

__device__ __forceinline__ int add_saturating(int a, int b) { return (int)min((uint32_t)a + (uint32_t)b, (uint32_t)kMost); }

// Sum of the values of the threads before this one, and of all (0 <= v <= kMost), saturating.  smem: one value a wave.
__device__ __forceinline__ int block_exclusive_sum(int v, int* smem, int& total) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  int sum = v;
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const int below = __shfl_up(sum, d);
    if (lane >= d) sum = add_saturating(sum, below);
  }
  if (lane == 63) smem[wave] = sum;
  int before = __shfl_up(sum, 1);
  if (lane == 0) before = 0;
  __syncthreads();
  int waves = 0, all = 0;
#pragma unroll
  for (int w = 0; w < kScanThreads / 64; ++w) {
    const int x = smem[w];
    if (w < wave) waves = add_saturating(waves, x);
    all = add_saturating(all, x);
  }
  __syncthreads();
  total = all;
  return add_saturating(waves, before);
}

struct Sequence {
  int session, held, len, row, top;  // top: entries of the stack that are left when its turn comes (below 0: lacking)
};

// One sequence's entries and rows, every `step`-th from `from` on.
__device__ __forceinline__ void fill(const PlanArgs& p, int b, const Sequence& s, int64_t from, int64_t step) {
  const int closed = s.len >> p.shift, had = s.held >> p.shift, n = s.len - s.held;
  if (closed > 0) {
    int32_t* own = p.pages + (int64_t)s.session * p.pages_stride;
    int32_t* table = p.table + (int64_t)b * p.table_stride;
    for (int64_t j = (p.same_table ? had : 0) + from; j < closed; j += step) {
      int page;
      if (j < had) {
        page = own[j];
      } else {
        const int64_t place = s.top - 1 - (j - had);
        page = place >= 0 ? p.free_pages[place] : -1;
        own[j] = page;
      }
      table[j] = page;
    }
  }
  if (p.sequence)
    for (int64_t i = from; i < n; i += step) p.sequence[s.row + i] = b;
  if (p.positions)
    for (int64_t i = from; i < n; i += step) p.positions[s.row + i] = s.held + (int)i;
}

// The sums; FILL (up to kScanThreads sequences, a thread each): the tables and rows too.
template <bool FILL>
__global__ __launch_bounds__(kScanThreads) void kv8_plan_kernel(const PlanArgs p) {
  __shared__ int smem[kScanThreads / 64];
  __shared__ Sequence seqs[FILL ? kScanThreads : 1];
  const int tid = threadIdx.x;
  const int count = min(max(*p.free_count, 0), p.pool);
  int rows = 0, taken = 0;  // of the sequences before this turn's
  for (int first = 0; first < p.sequences; first += kScanThreads) {
    const int b = first + tid;
    int session = -1, held = 0, n = 0;
    if (b < p.sequences) {
      session = p.ids ? p.ids[b] : b;
      if ((uint32_t)session < (uint32_t)p.sessions) {
        held = min(max(p.held[session], 0), p.max_len);
        n = min(min(max(p.new_tokens[b], 0), p.max_new), p.max_len - held);
      } else {
        session = -1;
      }
    }
    int all;
    const int row = min(add_saturating(rows, block_exclusive_sum(n, smem, all)), p.tokens);
    n = min(n, p.tokens - row);  // rows that the step's tensors do not have are not taken
    rows = add_saturating(rows, all);
    const int len = held + n, fresh = (len >> p.shift) - (held >> p.shift);
    const int before = add_saturating(taken, block_exclusive_sum(fresh, smem, all));
    taken = add_saturating(taken, all);
    if (b < p.sequences) {
      p.kv_len[b] = len;
      p.cu[b] = row;
      if (session >= 0) p.held_after[session] = len;
      if constexpr (FILL) seqs[tid] = Sequence{session, held, len, row, count - before};
      else p.top[b] = count - before;
    }
  }
  if (tid == 0) {
    p.cu[p.sequences] = min(rows, p.tokens);
    *p.free_count_after = max(count - taken, 0);
    if (p.lacking) *p.lacking = max(taken - count, 0);
  }
  if constexpr (FILL) {
    __syncthreads();
    // as many threads for a sequence as there are, a wave at least
    const int lanes = p.sequences <= 1 ? kScanThreads : max(64, kScanThreads >> (32 - __clz(p.sequences - 1)));
    for (int b = tid / lanes; b < p.sequences; b += kScanThreads / lanes) fill(p, b, seqs[b], tid % lanes, lanes);
  }
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
// that are no page.
__global__ __launch_bounds__(kScanThreads) void kv8_release_kernel(const PlanArgs p) {
  __shared__ int smem[kScanThreads / 64];
  __shared__ int session_of[kScanThreads], closed_of[kScanThreads], pages_of[kScanThreads];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  constexpr int kWaves = kScanThreads / 64;
  auto is_page = [&](int page) { return (uint32_t)page < (uint32_t)p.pool; };
  int count = min(max(*p.free_count, 0), p.pool);
  for (int64_t first = 0; first < p.sequences; first += kScanThreads) {
    const int here = (int)min((int64_t)kScanThreads, p.sequences - first);
    if (tid < here) {
      int session = p.ids ? p.ids[first + tid] : (int)first + tid, closed = 0;
      if ((uint32_t)session < (uint32_t)p.sessions)
        closed = min(max(atomicExch(&p.held_after[session], 0), 0) >> p.shift, p.columns);  // (there twice: the second finds nothing)
      else
        session = 0;
      session_of[tid] = session;
      closed_of[tid] = closed;
    }
    __syncthreads();
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
    const int before = block_exclusive_sum(tid < here ? pages_of[tid] : 0, smem, all);
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

// One launch while a single workgroup moves the entries and rows sooner than a second launch starts
bool in_one_launch(const PlanArgs& p) {
  return p.sequences <= kScanThreads && (int64_t)p.sequences * ((p.max_len >> p.shift) + (int64_t)p.max_new) <= kPlanOneLaunch;
}

int launched(const char* what, const char* name) {
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return set_error(QQQ_ERR_HIP, "%s launch: %s", what, hipGetErrorString(e));
  route_note("%s", name);
  return QQQ_OK;
}

}  // namespace

size_t kv8_plan_bytes(const PlanArgs& p) { return in_one_launch(p) ? 0 : (size_t)p.sequences * sizeof(int32_t); }

int launch_kv8_plan(const PlanArgs& p, hipStream_t st) {
  if (in_one_launch(p)) {
    hipLaunchKernelGGL((kv8_plan_kernel<true>), dim3(1), dim3(kScanThreads), 0, st, p);
    return launched("plan", "plan one launch");
  }
  hipLaunchKernelGGL((kv8_plan_kernel<false>), dim3(1), dim3(kScanThreads), 0, st, p);
  if (int rc = launched("plan", "plan sums")) return rc;
  const int64_t most = std::max(p.max_len >> p.shift, std::min(p.max_new, p.tokens));  // entries or rows of a sequence
  const int64_t parts = std::min<int64_t>(std::max<int64_t>((most + 4 * kFillThreads - 1) / (4 * kFillThreads), 1), std::max(8 * num_cus() / p.sequences, 1));
  hipLaunchKernelGGL(kv8_plan_fill_kernel, dim3((unsigned)p.sequences, (unsigned)parts), dim3(kFillThreads), 0, st, p);
  return launched("plan", "fill");
}

int launch_kv8_release(const PlanArgs& p, hipStream_t st) {
  hipLaunchKernelGGL(kv8_release_kernel, dim3(1), dim3(kScanThreads), 0, st, p);
  return launched("release", "release");
}

}  // namespace qqq
