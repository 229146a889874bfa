// W8A8 GEMM, tiles: WM x WN waves of 16 TM x 16 TN outputs each, v_mfma_i32_16x16x64_i8.
//
// Both operands come through LDS, filled by DMA (global_load_lds_dwordx4) ahead of the products.  A step is 64 k.  Activations are fetched 128 k at a time (whole
// 128-byte lines of their rows) into three slots, weights 64 k at a time (the packed layout's 1 KiB halves of chunks, lane by lane as the operand is) into four.  Every
// step requests the weights of the third step after it and half of the activations' rows of the second 128 k after its own: the same number of requests each step, so
// "all but the newest two steps' requests have landed" is one wait count.  The wait and the workgroup's barrier stand kAhead row tiles before the step's end: the
// products still to come have their operands in registers, and the fragments read after the barrier are the next step's.
// Activations lie in rows of 128 bytes, 16-byte chunk c of row r in slot c ^ ((r/2)%8), so that the 16 rows of a fragment read fall into different banks (as in
// the W4A8 tiles); the exchange is made on the global side of the DMA.
#include "qqq_prefill_common.h"
#include "qqq_w8a8.h"

// The DMA helper names M0 as clobbered (it rewrites it before every use), a reserved register, which the compiler remarks on.
#pragma clang diagnostic ignored "-Winline-asm"

namespace qqq {

namespace {

template <int WM, int WN, int TM, int TN>
struct W8Shape {
  static constexpr int kWaves = WM * WN, kBM = 16 * WM * TM, kBN = 16 * WN * TN;
  static constexpr int kASlot = kBM * 128, kBSlot = kBN * 64;
  static constexpr int kASlots = 3, kBSlots = 4;
  static constexpr int kLds = kASlots * kASlot + kBSlots * kBSlot;
  static constexpr int kAPieces = kBM / 16 / kWaves;  // 1 KiB requests of a wave and step: activations (8 rows of 128 bytes each)
  static constexpr int kBPieces = kBN / 16 / kWaves;  // and weights (16 channels)
  static constexpr int kPieces = kAPieces + kBPieces;
  static constexpr int kAhead = TM >= 8 ? 3 : 2;
  static constexpr int kPerSlot = (kPieces + TM - kAhead - 1) / (TM - kAhead);
  // a wave's patch of the output on its way out: 16 rows, padded by 16 bytes
  static constexpr int kOutRow = 16 * TN * 4 + 16, kOutWave = 16 * kOutRow;
  static_assert(kAPieces * 16 * kWaves == kBM && kBPieces * 16 * kWaves == kBN, "whole requests for every wave");
  static_assert(kLds <= 160 * 1024 && kWaves * kOutWave <= kLds, "LDS");
};

template <int WM, int WN, int TM, int TN>
__global__ __launch_bounds__(WM* WN * 64, WM * WN == 8 ? 1 : 2) void w8_tile_kernel(const W8Params p, const int tiles_m, const int tiles_n) {
  using S = W8Shape<WM, WN, TM, TN>;
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

  // Consecutive workgroups go to different XCDs: each XCD gets a contiguous run of tiles, walked in groups of 8 row tiles (rows fastest), so that those that run together
  // on an XCD share their operands in its L2.
  int pid = blockIdx.x;
  {
    const int per = tiles_m * tiles_n / 8;
    if (pid < per * 8) pid = (pid % 8) * per + pid / 8;
  }
  constexpr int kGroupM = 8;
  const int width = kGroupM * tiles_n, first_m = pid / width * kGroupM, gsize = min(tiles_m - first_m, kGroupM);
  const int m0 = (first_m + pid % width % gsize) * S::kBM, tn = pid % width / gsize;

  // ---- requests: a wave-uniform base and a 32-bit offset a lane.  Rows past M repeat row M-1, channels past N the last chunk (not stored).
  uint32_t a_voff[2][S::kAPieces];
  const int8_t* b_base[S::kBPieces];
#pragma unroll
  for (int h = 0; h < 2; ++h)
#pragma unroll
    for (int i = 0; i < S::kAPieces; ++i) {
      const int r = h * (S::kBM / 2) + 8 * (S::kAPieces * wave + i) + (lane >> 3);
      a_voff[h][i] = (uint32_t)(min(m0 + r, M - 1) - m0) * (uint32_t)K + (uint32_t)(((lane & 7) ^ ((r >> 1) & 7)) << 4);
    }
  const int8_t* a_base = p.a_q + m0 * K + (int64_t)first * 128;
  const int64_t w_step = (int64_t)ntiles * 2048;  // between blocks of 128 k
#pragma unroll
  for (int j = 0; j < S::kBPieces; ++j)
    b_base[j] = p.w + (int64_t)min(tn * (S::kBN / 16) + S::kBPieces * wave + j, ntiles - 1) * 2048 + first * w_step;
  const uint32_t b_voff = (uint32_t)lane * 16u;
  const uint32_t lds_base = (uint32_t)(uintptr_t)(lds_ptr_t)lds;
  // Through inline assembly, so that the compiler does not wait for all of them before an LDS read; M0 holds the LDS place, lane l writes at M0 + 16 l.
  auto dma = [&](const int8_t* base, uint32_t voff, uint32_t to) {
    asm volatile("s_mov_b32 m0, %0\n\tglobal_load_lds_dwordx4 %1, %2" ::"s"(to), "v"(voff), "s"(base) : "memory", "m0");
  };
  constexpr uint32_t kB0 = S::kASlots * S::kASlot;
  // rows' half h of 128-k block t into activation slot `slot`
  auto dma_a = [&](int t, int h, int slot, int i) {
    dma(a_base + (int64_t)min(t, T - 1) * 128, a_voff[h][i], lds_base + slot * S::kASlot + h * (S::kASlot / 2) + (S::kAPieces * wave + i) * 1024);
  };
  // 64-k half h of block t into weight slot `slot`
  auto dma_b = [&](int t, int h, int slot, int j) {
    dma(b_base[j] + (int64_t)min(t, T - 1) * w_step + h * 1024, b_voff, lds_base + kB0 + slot * S::kBSlot + (S::kBPieces * wave + j) * 1024);
  };
  constexpr int kPieces = S::kPieces, kAhead = S::kAhead;

  // ---- fragments
  const int lcol = lane & 15, kblk = lane >> 4;
  int a_off[2];
#pragma unroll
  for (int s = 0; s < 2; ++s) a_off[s] = (wm * TM * 16 + lcol) * 128 + (((4 * s + kblk) ^ ((lcol >> 1) & 7)) << 4);
  const int b_off = kB0 + wn * TN * 1024 + lane * 16;
  auto read_a = [&](int slot, int s, int i) { return *reinterpret_cast<const v4i*>(lds + slot * S::kASlot + a_off[s] + i * 2048); };
  auto read_b = [&](int slot, int c) { return *reinterpret_cast<const v4i*>(lds + slot * S::kBSlot + b_off + c * 1024); };

  v4i acc[TM][TN];
#pragma unroll
  for (int i = 0; i < TM; ++i)
#pragma unroll
    for (int c = 0; c < TN; ++c) acc[i][c] = (v4i){0, 0, 0, 0};

  // blocks 0 and 1 of the activations and steps 0, 1, 2 of the weights, in the order in which the steps wait for them
#pragma unroll
  for (int h = 0; h < 2; ++h)
#pragma unroll
    for (int i = 0; i < S::kAPieces; ++i) dma_a(0, h, 0, i);
#pragma unroll
  for (int j = 0; j < S::kBPieces; ++j) dma_b(0, 0, 0, j);
#pragma unroll
  for (int h = 0; h < 2; ++h) {
#pragma unroll
    for (int i = 0; i < S::kAPieces; ++i) dma_a(1, h, 1, i);
#pragma unroll
    for (int j = 0; j < S::kBPieces; ++j) dma_b(h, 1 - h, 1 + h, j);
  }
  auto wait_and_meet = [&]() { asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(2 * kPieces) : "memory"); };
  wait_and_meet();

  constexpr int kBufs = TM > 4 ? 8 : 4;
  static_assert(TM % kBufs == 0 || TM == kBufs, "a step starts with the first register again");
  static_assert(kAhead < TM && kAhead < kBufs, "schedule");
  v4i abuf[kBufs], b[2][TN];
#pragma unroll
  for (int i = 0; i < kAhead; ++i) abuf[i] = read_a(0, 0, i);
#pragma unroll
  for (int c = 0; c < TN; ++c) b[0][c] = read_b(0, c);

  int a_slot = 0, b_pair = 0;  // of this block: activation slot, first of its two weight slots / 2
  for (int t = 0; t < T; ++t) {
    const int a_next = a_slot == 2 ? 0 : a_slot + 1, a_then = a_slot == 0 ? 2 : a_slot - 1;
#pragma unroll
    for (int s = 0; s < 2; ++s) {
      const int b_slot_next = s == 0 ? 2 * b_pair + 1 : 2 * (b_pair ^ 1);
#pragma unroll
      for (int i = 0; i < TM; ++i) {
        if (i == TM - kAhead) wait_and_meet();
        // the fragment kAhead row tiles on
        if (i + kAhead < TM) abuf[(i + kAhead) % kBufs] = read_a(a_slot, s, i + kAhead);
        else abuf[(i + kAhead) % kBufs] = s == 0 ? read_a(a_slot, 1, i + kAhead - TM) : read_a(a_next, 0, i + kAhead - TM);
        if (i >= TM - kAhead) {  // and the next step's weights
          constexpr int kEach = (TN + kAhead - 1) / kAhead;
#pragma unroll
          for (int c = (i - (TM - kAhead)) * kEach; c < (i - (TM - kAhead) + 1) * kEach && c < TN; ++c) b[s ^ 1][c] = read_b(b_slot_next, c);
        }
        // this step's requests: half of the activations of block t + 2, the weights of the third step from here
#pragma unroll
        for (int q = i * S::kPerSlot; q < (i + 1) * S::kPerSlot && q < kPieces; ++q) {
          if (q < S::kAPieces) dma_a(t + 2, s, a_then, q);
          else if (s == 0) dma_b(t + 1, 1, 2 * (b_pair ^ 1) + 1, q - S::kAPieces);
          else dma_b(t + 2, 0, 2 * b_pair, q - S::kAPieces);
        }
#pragma unroll
        for (int c = 0; c < TN; ++c) acc[i][c] = __builtin_amdgcn_mfma_i32_16x16x64_i8(abuf[i % kBufs], b[s][c], acc[i][c], 0, 0, 0);
        __builtin_amdgcn_sched_barrier(0);
      }
    }
    a_slot = a_next;
    b_pair ^= 1;
  }
  // requests past the last step (repeats of it) may still be landing: LDS is free once all have
  asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");

  const int row0 = m0 + wm * TM * 16, col0 = tn * S::kBN + wn * TN * 16;
  if (p.k_splits > 1 || p.acc_out) {
    int32_t* out = p.k_splits > 1 ? p.part + (int64_t)split * M * N : p.acc_out;
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
    if (p.k_splits > 1) return;
  }
  float sw[TN];
#pragma unroll
  for (int c = 0; c < TN; ++c) sw[c] = p.s_w[min(col0 + 16 * c + lcol, N - 1)];
  // 16 rows of the wave's patch at a time through its own LDS (served in order: no barrier), out as whole rows
  int8_t* const ep = lds + wave * S::kOutWave;
  const int size = p.f32 ? 4 : 2;
#pragma unroll
  for (int i = 0; i < TM; ++i) {
#pragma unroll
    for (int v = 0; v < 4; ++v) {
      const int r = 4 * kblk + v;
      const float sa = p.s_a[min(row0 + 16 * i + r, M - 1)];
#pragma unroll
      for (int c = 0; c < TN; ++c) {
        if (p.f32) *reinterpret_cast<float*>(ep + r * S::kOutRow + (16 * c + lcol) * 4) = w8_scaled(acc[i][c][v], sa, sw[c]);
        else *reinterpret_cast<_Float16*>(ep + r * S::kOutRow + (16 * c + lcol) * 2) = dequant(acc[i][c][v], sa, sw[c]);
      }
    }
    const int rows = min(16, M - (row0 + 16 * i));
    char* const to = static_cast<char*>(p.y) + ((int64_t)(row0 + 16 * i) * p.ldy + col0) * size;
    const int64_t pitch = p.ldy * size;
    if (p.wide && col0 + 16 * TN <= N) {
      const int per_row = TN * size;  // 16-byte pieces
#pragma unroll
      for (int q = 0; q < 16 * TN * 4 / 64; ++q) {
        const int piece = lane + 64 * q, r = piece / per_row, c = piece % per_row;
        if (r < rows) *reinterpret_cast<v4i*>(to + r * pitch + c * 16) = *reinterpret_cast<const v4i*>(ep + r * S::kOutRow + c * 16);
      }
    } else {
      constexpr int kRows = 64 / (16 * TN) > 0 ? 64 / (16 * TN) : 1;  // of a store
#pragma unroll
      for (int r0 = 0; r0 < 16; r0 += kRows) {
#pragma unroll
        for (int c0 = 0; c0 < 16 * TN; c0 += 64) {
          const int r = r0 + lane / (16 * TN), c = c0 + lane % (16 * TN);
          if (r < rows && col0 + c < N) {
            if (p.f32) *reinterpret_cast<float*>(to + r * pitch + c * 4) = *reinterpret_cast<const float*>(ep + r * S::kOutRow + c * 4);
            else *reinterpret_cast<_Float16*>(to + r * pitch + c * 2) = *reinterpret_cast<const _Float16*>(ep + r * S::kOutRow + c * 2);
          }
        }
      }
    }
  }
}

// Second launch of a call that splits K: the parts' sums, four channels a thread
__global__ __launch_bounds__(256) void w8_sum_kernel(const W8Params p) {
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x, slab = (int64_t)p.M * p.N;
  if (i >= slab) return;
  int x = 0;
  for (int s = 0; s < p.k_splits; ++s) x += p.part[s * slab + i];
  const int m = (int)(i / p.N), n = (int)(i % p.N);
  w8_store(p, m, n, x, p.s_a[m], p.s_w[n]);
}

template <int WM, int WN, int TM, int TN>
int launch_tile(const W8Params& p, hipStream_t st) {
  using S = W8Shape<WM, WN, TM, TN>;
  const int tiles_m = (p.M + S::kBM - 1) / S::kBM, tiles_n = (p.N + S::kBN - 1) / S::kBN;
  if ((int64_t)tiles_m * tiles_n > 0x7FFFFFFF) return set_error(QQQ_ERR_SHAPE, "w8a8: too many output tiles for one launch");
  hipLaunchKernelGGL((w8_tile_kernel<WM, WN, TM, TN>), dim3((unsigned)(tiles_m * tiles_n), (unsigned)p.k_splits), dim3(S::kWaves * 64), 0, st, p, tiles_m, tiles_n);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return set_error(QQQ_ERR_HIP, "w8a8 launch: %s", hipGetErrorString(e));
  route_note("w8a8 tile=%dx%d ksplit=%d", S::kBM, S::kBN, p.k_splits);
  return QQQ_OK;
}

}  // namespace

int launch_w8_tiles(const W8Params& p, int shape, hipStream_t st) {
  switch (shape) {
    case kW8Tile256x256: return launch_tile<2, 4, 8, 4>(p, st);
    case kW8Tile128x256: return launch_tile<2, 4, 4, 4>(p, st);
    case kW8Tile128x128: return launch_tile<2, 2, 4, 4>(p, st);
  }
  return launch_tile<1, 4, 4, 2>(p, st);
}

int launch_w8_sum(const W8Params& p, hipStream_t st) {
  hipLaunchKernelGGL(w8_sum_kernel, dim3((unsigned)(((int64_t)p.M * p.N + 255) / 256)), dim3(256), 0, st, p);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return set_error(QQQ_ERR_HIP, "w8a8 sum launch: %s", hipGetErrorString(e));
  route_note("sum");
  return QQQ_OK;
}

static int g_shape = 0, g_k_splits = 0;  // qqq_set_w8a8_tuning

W8Plan w8_plan(int64_t M, int64_t N, int64_t K) {
  auto automatic = [&]() -> W8Plan {
    if (M <= kW8FewRows) return {kW8Few, 1};
    auto tiles = [&](int bm, int bn) { return ((M + bm - 1) / bm) * ((N + bn - 1) / bn); };
    if (tiles(256, 256) >= num_cus()) return {kW8Tile256x256, 1};
    if (tiles(128, 256) >= num_cus()) return {kW8Tile128x256, 1};
    if (tiles(128, 128) >= num_cus()) return {kW8Tile128x128, 1};
    return {kW8Tile64x128, 1};
  };
  W8Plan plan = automatic();
  if (g_shape > 0 && (g_shape != kW8Few || M <= kW8FewRows)) plan.shape = g_shape;
  if (g_k_splits > 0) plan.k_splits = (int)(g_k_splits < K / 128 ? g_k_splits : K / 128);
  return plan;
}

}  // namespace qqq

extern "C" int qqq_set_w8a8_tuning(int shape, int k_splits) {
  if (shape < 0 || shape > qqq::kW8Tile64x128 || k_splits < 0) return -1;
  const int before = qqq::g_shape;
  qqq::g_shape = shape;
  qqq::g_k_splits = k_splits;
  return before;
}
