// W8A8 GEMM, tiles: WM x WN waves of 16 TM x 16 TN outputs each, v_mfma_i32_16x16x64_i8.
//
// Both operands come through LDS, filled by DMA (global_load_lds_dwordx4) ahead of the products.  A step is 64 k.  Activations are fetched 128 k at a time (whole
// 128-byte lines of their rows) into (NB + 2) / 2 slots, weights 64 k at a time (the packed layout's 1 KiB halves of chunks, lane by lane as the operand is) into NB.  Every
// step requests the weights of a later step and half of the activations' rows of a later 128 k, into slots that are free: the same number of requests each step, so
// "all but the newest NB - 2 steps' requests have landed" is one wait count.
//   256 x 256: the wait and the workgroup's barrier stand kAhead row tiles before the step's end.  The products still to come have their operands in registers, and the
//   fragments read after the barrier are the next step's.  2 waves a SIMD of 128 accumulators each leave no room for more.
//   FULL, the smaller tiles: the wait and the barrier stand at the step's start, and every fragment of the next step is read in this one, so a slot is free a step sooner and LDS's
//   latency is covered where there is little else to cover it.  On 256 x 256 it is 1 to 2 % slower.
// Activations lie in rows of 128 bytes, 16-byte chunk c of row r in slot c ^ ((r/2)%8), so that the 16 rows of a fragment read fall into different banks (as in
// the W4A8 tiles); the exchange is made on the global side of the DMA.
//
// What bounds it: long prompts the board's power (4096 x 28672 x 8192 in 680 to 690 us, 2.8 POP/s: matrix units busy 75 % of the cycles at some 1.72 GHz; the library's int8 product with 32-bit
// output takes 848); 64 to 600 rows the shares of CUs that tiles fill, and the step's barrier (333 x 13824 x 5120 in 30 us from the last-level cache, 37 from memory, 162 tiles on 256 CUs; at the
// long prompts' rate 17); 33 to 64 rows over a wide N the weights' bytes (48 x 50001 x 5120 in 41 us, 6.3 TB/s).  Not kept: an outer ring of 2, 4 or 5 row tiles ahead (level to 2 % slower),
// 16 row tiles to a group (2 %), wave priorities (2 %), weights straight to registers without LDS (slower everywhere), tiles of 96, 160 and 224 rows.
#include <math.h>

#include "qqq_prefill_common.h"
#include "qqq_w8a8.h"

// The DMA helper names M0 as clobbered (it rewrites it before every use), a reserved register, which the compiler remarks on.
#pragma clang diagnostic ignored "-Winline-asm"

namespace qqq {

namespace {

enum W8Out : int { kF16, kF32, kPart };  // what a tile writes: outputs, or its part of the sums

// A wave's patch of the output on its way out: 16 rows, padded by 16 bytes, and its rows' scales
template <int TM, int TN>
constexpr int w8_patch_bytes() {
  return 16 * (16 * TN * 4 + 16) + 16 * TM * 4;
}

// A wave's 16 TM x 16 TN results from row0 and col0 on.  Requests into LDS may still be landing: it is free (ep: this wave's part) once the whole workgroup's have.
template <int TM, int TN, int OUT>
__device__ __forceinline__ void w8_write(const W8Params& p, const v4i (&acc)[TM][TN], int row0, int col0, int split, int8_t* ep) {
  const int lane = threadIdx.x & 63, lcol = lane & 15, kblk = lane >> 4, M = p.M, N = p.N;
  constexpr int kRowLoads = (16 * TM + 63) / 64, kOutRow = 16 * TN * 4 + 16;
  float sa_own[kRowLoads], sw[TN];  // (requested before the wait)
  if constexpr (OUT != kPart) {
#pragma unroll
    for (int i = 0; i < kRowLoads; ++i) sa_own[i] = p.s_a[min(row0 + lane + 64 * i, M - 1)];
#pragma unroll
    for (int c = 0; c < TN; ++c) sw[c] = p.s_w[min(col0 + 16 * c + lcol, N - 1)];
  }
  asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");

  if (OUT == kPart || p.acc_out) {
    int32_t* out = OUT == kPart ? p.part + (int64_t)split * M * N : p.acc_out;
#pragma unroll
    for (int i = 0; i < TM; ++i)
#pragma unroll
      for (int v = 0; v < 4; ++v) {
        const int m = row0 + 16 * i + 4 * kblk + v;
        if (m >= M) continue;
#pragma unroll
        for (int c = 0; c < TN; ++c)
          if (col0 + 16 * c + lcol < N) out[(int64_t)m * N + col0 + 16 * c + lcol] = acc[i][c][v];
      }
  }
  if constexpr (OUT != kPart) {
    // 16 rows of the patch at a time through LDS (one wave's accesses are served in order: no barrier), out as whole rows
    float* const sa_lds = reinterpret_cast<float*>(ep + 16 * kOutRow);
#pragma unroll
    for (int i = 0; i < kRowLoads; ++i)
      if (16 * TM % 64 == 0 || lane + 64 * i < 16 * TM) sa_lds[lane + 64 * i] = sa_own[i];
    constexpr int kSize = OUT == kF32 ? 4 : 2, kPerRow = TN * kSize;  // 16-byte pieces of a row
    const int64_t pitch = p.ldy * kSize;
    const bool whole = col0 + 16 * TN <= N;
#pragma unroll
    for (int i = 0; i < TM; ++i) {
      typedef float v4f __attribute__((ext_vector_type(4)));
      const v4f sa = *reinterpret_cast<const v4f*>(sa_lds + 16 * i + 4 * kblk);
#pragma unroll
      for (int v = 0; v < 4; ++v) {
        const int r = 4 * kblk + v;
#pragma unroll
        for (int c = 0; c < TN; ++c) {
          if constexpr (OUT == kF32) *reinterpret_cast<float*>(ep + r * kOutRow + (16 * c + lcol) * 4) = w8_scaled(acc[i][c][v], sa[v], sw[c]);
          else *reinterpret_cast<_Float16*>(ep + r * kOutRow + (16 * c + lcol) * 2) = dequant(acc[i][c][v], sa[v], sw[c]);
        }
      }
      const int rows = min(16, M - (row0 + 16 * i));
      char* const to = static_cast<char*>(p.y) + ((int64_t)(row0 + 16 * i) * p.ldy + col0) * kSize;
      if (whole) {
#pragma unroll
        for (int q = 0; q < (16 * kPerRow + 63) / 64; ++q) {
          const int piece = lane + 64 * q, r = piece / kPerRow, c = piece % kPerRow;
          if (r < rows) {
            const v4i d = *reinterpret_cast<const v4i*>(ep + r * kOutRow + c * 16);
            __builtin_memcpy(to + r * pitch + c * 16, &d, 16);  // (rows may lie at any place of their type: one store all the same)
          }
        }
      } else {
        constexpr int kRows = 64 / (16 * TN);  // of a store
#pragma unroll
        for (int r0 = 0; r0 < 16; r0 += kRows) {
          const int r = r0 + lane / (16 * TN), c = lane % (16 * TN);
          if (r < rows && col0 + c < N) {
            if constexpr (OUT == kF32) *reinterpret_cast<float*>(to + r * pitch + c * 4) = *reinterpret_cast<const float*>(ep + r * kOutRow + c * 4);
            else *reinterpret_cast<_Float16*>(to + r * pitch + c * 2) = *reinterpret_cast<const _Float16*>(ep + r * kOutRow + c * 2);
          }
        }
      }
    }
  }
}

// Workgroup to tile: consecutive workgroups go to different XCDs, so each XCD gets a contiguous run of tiles, walked in groups of 4 row tiles (rows fastest): those that
// run together on an XCD share their operands in its L2.
__device__ __forceinline__ void w8_tile_of(int pid, int tiles_m, int tiles_n, int& tm, int& tn) {
  const int per = tiles_m * tiles_n / 8;
  if (pid < per * 8) pid = (pid % 8) * per + pid / 8;
  constexpr int kGroupM = 4;
  const int width = kGroupM * tiles_n, first_m = pid / width * kGroupM, gsize = min(tiles_m - first_m, kGroupM);
  tm = first_m + pid % width % gsize;
  tn = pid % width / gsize;
}

// NB: weight slots of 64 k; activation slots of 128 k are (NB + 2) / 2
template <int WM, int WN, int TM, int TN, int NB, bool FULL>
struct W8Shape {
  static constexpr int kWaves = WM * WN, kBM = 16 * WM * TM, kBN = 16 * WN * TN;
  static constexpr int kASlot = kBM * 128, kBSlot = kBN * 64;
  static constexpr int kASlots = (NB + 2) / 2;
  static constexpr int kLds = kASlots * kASlot + NB * kBSlot;
  static constexpr int kAPieces = kBM / 16, kBPieces = kBN / 16;  // 1 KiB requests of a step: 8 rows of 128 bytes, 16 channels of 64 k
  static constexpr int kPieces = kAPieces + kBPieces, kRounds = (kPieces + kWaves - 1) / kWaves;  // a wave takes every kWaves-th: kRounds of them, or one less
  static constexpr int kMany = kPieces - (kRounds - 1) * kWaves;  // waves that take kRounds
  static constexpr int kFlight = NB - 2;  // steps whose requests may be on their way when a step's are waited for
  static constexpr int kAhead = FULL ? 0 : TM >= 8 ? 3 : 2;
  static constexpr int kPerSlot = (kRounds + TM - kAhead - 1) / (TM - kAhead);
  static constexpr int kOutWave = w8_patch_bytes<TM, TN>();
  static_assert(NB % 2 == 0 && kBM % 32 == 0 && (kFlight + 1) * kRounds < 63, "pairs of slots, halves of whole requests, a wait count that fits");
  static_assert(kLds <= 160 * 1024 && kWaves * kOutWave <= kLds, "LDS");
};

template <int WM, int WN, int TM, int TN, int NB, bool FULL, int OUT>
__global__ __launch_bounds__(WM * WN * 64, 2) void w8_tile_kernel(const W8Params p, const int tiles_m, const int tiles_n) {
  using S = W8Shape<WM, WN, TM, TN, NB, FULL>;
  __shared__ __attribute__((aligned(1024))) int8_t lds[S::kLds];
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int wm = wave / WN, wn = wave % WN;
  const int N = p.N, M = p.M, ntiles = (N + 15) >> 4;
  const int64_t K = p.K;
  // part `split` of K, in blocks of 128
  const int split = blockIdx.y, blocks = p.K >> 7;
  const int first = (int)((int64_t)blocks * split / p.k_splits);
  const int T = (int)((int64_t)blocks * (split + 1) / p.k_splits) - first;

  int tm, tn;
  w8_tile_of(blockIdx.x, tiles_m, tiles_n, tm, tn);
  const int m0 = tm * S::kBM;

  // ---- requests: wave-uniform bases that move with k and 32-bit offsets a lane.  Rows past M repeat row M-1, channels past N the last chunk (not stored).
  // In a step of parity `par` rows of the activations' half par ^ 1 and the weights' 64-k half par are requested; this wave's piece of round r is wave + kWaves r, of the
  // activations first.
  const int chunk0 = tn * (S::kBN / 16);
  uint32_t voff[2][S::kRounds];
#pragma unroll
  for (int par = 0; par < 2; ++par)
#pragma unroll
    for (int r = 0; r < S::kRounds; ++r) {
      const int q = wave + S::kWaves * r, row = (par ^ 1) * (S::kBM / 2) + 8 * q + (lane >> 3);
      const uint32_t of_a = (uint32_t)(min(m0 + row, M - 1) - m0) * (uint32_t)K + (uint32_t)(((lane & 7) ^ ((row >> 1) & 7)) << 4);
      const uint32_t of_b = (uint32_t)(min(chunk0 + q - S::kAPieces, ntiles - 1) - chunk0) * 2048u + par * 1024u + (uint32_t)lane * 16u;
      voff[par][r] = q < S::kAPieces ? of_a : of_b;
    }
  const int64_t w_step = (int64_t)ntiles * 2048;  // between blocks of 128 k
  const int8_t* a_from = p.a_q + m0 * K + (int64_t)first * 128;  // of the block that is requested next
  const int8_t* b_from = p.w + (int64_t)chunk0 * 2048 + first * w_step;
  // to the block after `t` (past the last: it again, never read)
  auto a_on = [&](int t) { a_from += t < T - 1 ? 128 : 0; };
  auto b_on = [&](int t) { b_from += t < T - 1 ? w_step : 0; };
  const uint32_t lds_base = (uint32_t)(uintptr_t)(lds_ptr_t)lds;
  // Through inline assembly, so that the compiler does not wait for all of them before an LDS read; M0 holds the LDS place, lane l writes at M0 + 16 l;
  // such a load comes one wait state after a write of M0 at the earliest, and the compiler puts none into inline assembly.
  auto dma = [&](const int8_t* base, uint32_t voff, uint32_t to) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" ::"s"(to), "v"(voff), "s"(base) : "memory", "m0");
  };
  constexpr uint32_t kB0 = S::kASlots * S::kASlot;
  // this wave's request of round r: activations' rows into the slot at a_slot (bytes), or weights into the one at b_slot
  auto request = [&](int par, int r, uint32_t a_slot, uint32_t b_slot) {
    const uint32_t to_a = lds_base + a_slot + (par ^ 1) * (S::kASlot / 2) + (wave + S::kWaves * r) * 1024;
    const uint32_t to_b = lds_base + kB0 + b_slot + (wave + S::kWaves * r - S::kAPieces) * 1024;
    const bool of_a = S::kWaves * (r + 1) <= S::kAPieces || (S::kWaves * r < S::kAPieces && wave + S::kWaves * r < S::kAPieces);
    if (r + 1 < S::kRounds || S::kMany == S::kWaves || wave < S::kMany) dma(of_a ? a_from : b_from, voff[par][r], of_a ? to_a : to_b);
  };
  // all of this wave's requests but those of the newest `Steps` steps have landed
#define QQQ_W8_LANDED(STEPS)                                                                            \
  do {                                                                                                  \
    if (S::kMany == S::kWaves || wave < S::kMany)                                                        \
      asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"((STEPS) * S::kRounds) : "memory");               \
    else                                                                                                \
      asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"((STEPS) * (S::kRounds - 1)) : "memory");         \
    asm volatile("s_barrier" ::: "memory");                                                               \
  } while (0)
  constexpr int kAhead = S::kAhead, kRounds = S::kRounds;

  // ---- fragments
  const int lcol = lane & 15, kblk = lane >> 4;
  int a_off[2];
#pragma unroll
  for (int s = 0; s < 2; ++s) a_off[s] = (wm * TM * 16 + lcol) * 128 + (((4 * s + kblk) ^ ((lcol >> 1) & 7)) << 4);
  const int b_off = kB0 + wn * TN * 1024 + lane * 16;
  auto read_a = [&](uint32_t slot, int s, int i) { return *reinterpret_cast<const v4i*>(lds + slot + a_off[s] + i * 2048); };
  auto read_b = [&](uint32_t slot, int c) { return *reinterpret_cast<const v4i*>(lds + slot + b_off + c * 1024); };

  v4i acc[TM][TN];
#pragma unroll
  for (int i = 0; i < TM; ++i)
#pragma unroll
    for (int c = 0; c < TN; ++c) acc[i][c] = (v4i){0, 0, 0, 0};

  // the first block of the activations and step 0 of the weights, then what the next steps wait for, in their order
  constexpr int kEarly = FULL ? NB : NB - 1;  // steps requested before the first
#pragma unroll
  for (int r = 0; r < kRounds; ++r)  // (the first half of the first block's rows)
    if (wave + S::kWaves * r < S::kAPieces) dma(a_from, voff[1][r], lds_base + (wave + S::kWaves * r) * 1024);
#pragma unroll
  for (int step = 0; step < kEarly; ++step) {
    if (step % 2 == 1) a_on(step / 2);
#pragma unroll
    for (int r = 0; r < kRounds; ++r) request(step % 2, r, (step + 1) / 2 * S::kASlot, step * S::kBSlot);
    if (step % 2 == 1) b_on(step / 2);
  }
  QQQ_W8_LANDED(kEarly - 1);

  // this block's places in LDS: activation slot, first of its two weight slots
  uint32_t a_slot = 0, b_slot = 0;
  constexpr uint32_t kAEnd = (S::kASlots - 1) * S::kASlot, kBPair = 2 * S::kBSlot, kBEnd = (NB / 2 - 1) * kBPair;
  v4i b[2][TN];
#pragma unroll
  for (int c = 0; c < TN; ++c) b[0][c] = read_b(0, c);
  if constexpr (FULL) {
    // every fragment of the next step is read in this one, whose wait and barrier stand at its start: with one wave a SIMD nothing else covers LDS's latency.  The slots of a
    // step are free in it already, so it requests step NB from here, and rows of the activations' block kASlots from the last step of theirs.
    v4i a[2][TM];
#pragma unroll
    for (int i = 0; i < TM; ++i) a[0][i] = read_a(0, 0, i);
    for (int t = 0; t < T; ++t) {
      const uint32_t a_next = a_slot == kAEnd ? 0 : a_slot + S::kASlot, a_last = a_slot == 0 ? kAEnd : a_slot - S::kASlot;
      const uint32_t b_next = b_slot == kBEnd ? 0 : b_slot + kBPair;
#pragma unroll
      for (int s = 0; s < 2; ++s) {
        QQQ_W8_LANDED(S::kFlight);
        if (s == 1) a_on(t + S::kASlots - 1);
#pragma unroll
        for (int i = 0; i < TM; ++i) {
          a[s ^ 1][i] = s == 0 ? read_a(a_slot, 1, i) : read_a(a_next, 0, i);
          constexpr int kEach = (TN + TM - 1) / TM;
#pragma unroll
          for (int c = i * kEach; c < (i + 1) * kEach && c < TN; ++c) b[s ^ 1][c] = read_b(s == 0 ? b_slot + S::kBSlot : b_next, c);
#pragma unroll
          for (int r = i * S::kPerSlot; r < (i + 1) * S::kPerSlot && r < kRounds; ++r) request(s, r, s == 0 ? a_last : a_slot, b_slot + s * S::kBSlot);
#pragma unroll
          for (int c = 0; c < TN; ++c) acc[i][c] = __builtin_amdgcn_mfma_i32_16x16x64_i8(a[s][i], b[s][c], acc[i][c], 0, 0, 0);
          __builtin_amdgcn_sched_barrier(0);
        }
      }
      b_on(t + NB / 2);
      a_slot = a_next;
      b_slot = b_next;
    }
  } else {
    constexpr int kBufs = TM > 4 ? 8 : 4;
    static_assert(TM % kBufs == 0, "a step starts with the first register again");
    static_assert(kAhead < TM && kAhead < kBufs, "schedule");
    v4i abuf[kBufs];
#pragma unroll
    for (int i = 0; i < kAhead; ++i) abuf[i] = read_a(0, 0, i);
    a_on(S::kASlots - 2);
    for (int t = 0; t < T; ++t) {
      const uint32_t a_next = a_slot == kAEnd ? 0 : a_slot + S::kASlot, a_last = a_slot == 0 ? kAEnd : a_slot - S::kASlot;
      const uint32_t b_next = b_slot == kBEnd ? 0 : b_slot + kBPair, b_last = b_slot == 0 ? kBEnd : b_slot - kBPair;
#pragma unroll
      for (int s = 0; s < 2; ++s) {
        if (s == 1) b_on(t + NB / 2 - 1);
#pragma unroll
        for (int i = 0; i < TM; ++i) {
          if (i == TM - kAhead) QQQ_W8_LANDED(S::kFlight);
          // the fragment kAhead row tiles on
          if (i + kAhead < TM) abuf[(i + kAhead) % kBufs] = read_a(a_slot, s, i + kAhead);
          else abuf[(i + kAhead) % kBufs] = s == 0 ? read_a(a_slot, 1, i + kAhead - TM) : read_a(a_next, 0, i + kAhead - TM);
          if (i >= TM - kAhead) {  // and the next step's weights
            constexpr int kEach = (TN + kAhead - 1) / (kAhead > 0 ? kAhead : 1);
#pragma unroll
            for (int c = (i - (TM - kAhead)) * kEach; c < (i - (TM - kAhead) + 1) * kEach && c < TN; ++c)
              b[s ^ 1][c] = read_b(s == 0 ? b_slot + S::kBSlot : b_next, c);
          }
          // this step's requests, into the slots that the step before has left: rows of the activations' block kASlots - 1 from here, the weights of step NB - 1 from here
#pragma unroll
          for (int r = i * S::kPerSlot; r < (i + 1) * S::kPerSlot && r < kRounds; ++r) request(s ^ 1, r, a_last, s == 0 ? b_last + S::kBSlot : b_slot);
#pragma unroll
          for (int c = 0; c < TN; ++c) acc[i][c] = __builtin_amdgcn_mfma_i32_16x16x64_i8(abuf[i % kBufs], b[s][c], acc[i][c], 0, 0, 0);
          __builtin_amdgcn_sched_barrier(0);
        }
      }
      a_on(t + S::kASlots - 1);
      a_slot = a_next;
      b_slot = b_next;
    }
  }
  w8_write<TM, TN, OUT>(p, acc, m0 + wm * TM * 16, tn * S::kBN + wn * TN * 16, split, lds + wave * S::kOutWave);
}

// Second launch of a call that splits K: the parts' sums, an output a thread
__global__ __launch_bounds__(256) void w8_sum_kernel(const W8Params p) {
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x, slab = (int64_t)p.M * p.N;
  if (i >= slab) return;
  int x = 0;
  for (int s = 0; s < p.k_splits; ++s) x += p.part[s * slab + i];
  const int m = (int)(i / p.N), n = (int)(i % p.N);
  w8_store(p, m, n, x, p.s_a[m], p.s_w[n]);
}

template <int WM, int WN, int TM, int TN, int NB, bool FULL>
int launch_tile(const W8Params& p, hipStream_t st) {
  using S = W8Shape<WM, WN, TM, TN, NB, FULL>;
  const int tiles_m = (p.M + S::kBM - 1) / S::kBM, tiles_n = (p.N + S::kBN - 1) / S::kBN;
  if ((int64_t)tiles_m * tiles_n * (S::kWaves * 64) > 0xFFFFFFFFll) return set_error(QQQ_ERR_SHAPE, "w8a8: too many output tiles for one launch");
  const dim3 grid((unsigned)(tiles_m * tiles_n), (unsigned)p.k_splits), block(S::kWaves * 64);
  if (p.k_splits > 1) hipLaunchKernelGGL((w8_tile_kernel<WM, WN, TM, TN, NB, FULL, kPart>), grid, block, 0, st, p, tiles_m, tiles_n);
  else if (p.f32) hipLaunchKernelGGL((w8_tile_kernel<WM, WN, TM, TN, NB, FULL, kF32>), grid, block, 0, st, p, tiles_m, tiles_n);
  else hipLaunchKernelGGL((w8_tile_kernel<WM, WN, TM, TN, NB, FULL, kF16>), grid, block, 0, st, p, tiles_m, tiles_n);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return set_error(QQQ_ERR_HIP, "w8a8 launch: %s", hipGetErrorString(e));
  route_note("w8a8 tile=%dx%d slots=%d ksplit=%d", S::kBM, S::kBN, NB, p.k_splits);
  return QQQ_OK;
}

}  // namespace

int launch_w8_tiles(const W8Params& p, int shape, hipStream_t st) {
  switch (shape) {
    case kW8Tile256x256: return launch_tile<2, 4, 8, 4, 4, false>(p, st);
    case kW8Tile192x256: return launch_tile<2, 4, 6, 4, 4, true>(p, st);
    case kW8Tile128x256: return launch_tile<2, 4, 4, 4, 6, true>(p, st);
    case kW8Tile128x128: return launch_tile<2, 2, 4, 4, 4, true>(p, st);
  }
  return launch_tile<1, 4, 4, 2, 6, true>(p, st);
}

int launch_w8_sum(const W8Params& p, hipStream_t st) {
  hipLaunchKernelGGL(w8_sum_kernel, dim3((unsigned)(((int64_t)p.M * p.N + 255) / 256)), dim3(256), 0, st, p);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return set_error(QQQ_ERR_HIP, "w8a8 sum launch: %s", hipGetErrorString(e));
  route_note("sum");
  return QQQ_OK;
}

// ---- which kernel, and into how many parts K is cut: the least time of a cost model, in us.  Its constants are fitted to 6600 calls (N 512 .. 50001, K 512 .. 11008, M 1 .. 2048, each
// with every kernel and up to 16 parts; rms 6 to 10 %).  Of 190 other calls of random sizes what it picks is up to 7 % behind the best of them in nine of ten, 14 % at most (M = 15, N = 55407,
// K = 1152: tiles of 128 x 256 instead of 64 x 128).
// Tiles: start + rounds * (fixed + blocks * per_block), a round being a workgroup a CU (two for the small tiles, whose blocks then take per_block_full); a last round of a share
// x of the places takes alone + rising * x a block (small tiles with more than one workgroup on some CU: from shared to per_block_full).  Never less than the weights'
// bytes at the rate that such a launch streams them, a lower one where CUs have different numbers of workgroups.
struct W8Cost {
  int bm, bn, per_cu;
  double start, fixed, alone, rising, shared, per_block_full, per_byte, per_byte_uneven;
};
constexpr W8Cost kW8Cost[] = {
    {256, 256, 1, 0.5, 7.59, 0.853, 0.465, 0, 1.458, 0.245e-6, 0.296e-6},
    {192, 256, 1, 1.72, 5.41, 0.821, 0.301, 0, 1.203, 0.235e-6, 0.29e-6},
    {128, 256, 1, 2.48, 3.41, 0.523, 0.384, 0, 0.998, 0.18e-6, 0.183e-6},
    {128, 128, 2, 2.83, 2.16, 0.304, 0.425, 0.874, 1.09, 0.177e-6, 0.182e-6},
    {64, 128, 2, 2.88, 1.39, 0.217, 0.264, 0.636, 0.746, 0.157e-6, 0.181e-6},
};
constexpr double kW8SumStart = 4.1, kW8SumPerValue = 1.7e-6;  // of the second launch that a split needs

static double w8_tile_cost(const W8Cost& c, int64_t M, int64_t N, int64_t K, int splits, int cus) {
  const double blocks = (double)((K / 128 + splits - 1) / splits), places = (double)cus * c.per_cu;
  const double tiles = (double)((M + c.bm - 1) / c.bm) * (double)((N + c.bn - 1) / c.bn) * splits;
  const double full = floor(tiles / places), x = tiles / places - full;
  double t = c.start + full * (c.fixed + blocks * c.per_block_full);
  if (x > 0) t += c.fixed + blocks * (c.per_cu == 1 || x <= 0.5 ? c.alone + c.rising * x : c.shared + (c.per_block_full - c.shared) * (2 * x - 1));
  const bool uneven = full > 0 || (c.per_cu == 2 && x > 0.5);
  const double bytes = c.start + (uneven ? c.per_byte_uneven : c.per_byte) * (double)N * (double)K;
  return t > bytes ? t : bytes;
}
// Few rows, or more of them for few channels: the weights' bytes, or what a workgroup computes where there are several a CU; every workgroup reads its rows' activations
static double w8_few_cost(const W8FewShape& s, int64_t N, int64_t K, int splits, int cus) {
  const int mt = s.mt, nt = s.nt;
  const double groups = (double)((N + 16 * nt - 1) / (16 * nt)) * s.row_groups * splits, k = (double)K / splits;
  const double rounds = groups > cus ? groups / cus : 1;
  // (the CUs with most workgroups are last)
  const double bytes = 0.129e-6 * (double)N * (double)K, work = k / 1024 * (0.043 + 0.244 * mt * nt) * ceil(rounds);
  return 2.65 + (bytes > work ? bytes : work) + 0.656 * rounds + 0.191e-6 * groups * mt * k;
}

static int g_shape = 0, g_k_splits = 0;  // qqq_set_w8a8_tuning

W8Plan w8_plan(int64_t M, int64_t N, int64_t K) {
  const int cus = num_cus();
  const W8FewShape few = w8_few_shape(M, N, cus);
  W8Plan best = {kW8Tile64x128, 1};
  double least = 1e300;
  for (int shape = kW8Few; shape <= kW8Tile64x128; ++shape) {
    if (shape == kW8Few && M > kW8FewRows) continue;
    const int64_t rows = shape == kW8Few ? 16 * few.mt : kW8Cost[shape - kW8Tile256x256].bm, cols = shape == kW8Few ? 16 * few.nt : kW8Cost[shape - kW8Tile256x256].bn;
    const bool crowded = ((M + rows - 1) / rows) * ((N + cols - 1) / cols) * 2 > cus * (shape >= kW8Tile128x128 ? 2 : 1);
    for (int splits : {1, 2, 3, 4, 6, 8, 12, 16}) {
      // (parts of two blocks of 128 at least; slabs of 256 MB at most; none where half the places are taken without)
      if (splits > 1 && (K / 128 / splits < 2 || M * N * splits > 64000000 || crowded)) break;
      double t = shape == kW8Few ? w8_few_cost(few, N, K, splits, cus) : w8_tile_cost(kW8Cost[shape - kW8Tile256x256], M, N, K, splits, cus);
      if (splits > 1) t += kW8SumStart + kW8SumPerValue * (double)M * (double)N * splits;
      if (t < least) {
        least = t;
        best = {shape, splits};
      }
    }
  }
  if (g_shape > 0 && (g_shape != kW8Few || M <= kW8FewRows)) best.shape = g_shape;
  if (g_shape > 0) best.k_splits = 1;
  if (g_k_splits > 0 && M * N <= 1 << 30) best.k_splits = (int)(g_k_splits < K / 128 ? g_k_splits : K / 128);
  return best;
}

}  // namespace qqq

extern "C" int qqq_set_w8a8_tuning(int shape, int k_splits) {
  if (shape < 0 || shape > qqq::kW8Tile64x128 || k_splits < 0) return -1;
  const int before = qqq::g_shape;
  qqq::g_shape = shape;
  qqq::g_k_splits = k_splits;
  return before;
}
