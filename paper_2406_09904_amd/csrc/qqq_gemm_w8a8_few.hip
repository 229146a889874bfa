// W8A8 GEMM, few rows (up to 64 a workgroup): the packed weights are streamed once, so up to 64 rows it is bound by their bytes.  More rows are taken while they and the channels
// are few: with eight waves that share K it ends sooner than a tile does (us in a graph: 100 x 600 x 4096 5.9, by tiles 11.8; 670 x 141 x 2944 4.4 and 10.0).
//
// A workgroup of W waves owns 16 NT channels (and one of k_splits parts of K); its waves take the k-steps (128 k) in turn and their int32 sums meet in LDS.  A lane's 16 bytes of a
// chunk are its operand of v_mfma_i32_16x16x64_i8 as they are: no conversion, so nothing but loads stands between memory and the matrix units.  Two batches of
// k-steps are in flight per wave.  Integer sums are the same in any order.
// One row of 32000 x 4096: 20.6 us, 6.4 TB/s.
// Activations: up to eight rows come in operand order (a lane's 16 bytes of row l%16), more row by row (whole 128-byte lines) with a turn through the wave's own LDS; rows
// past M repeat row M-1 and are not stored.
#include "qqq_w8a8.h"

namespace qqq {

namespace {

template <int NT, int MT, int U>
struct W8Batch {
  v4i w[U][NT][2];
  v4i a[U][MT][2];
};

// Every call issues the same loads: k-steps past the end repeat the last one's (their products are skipped).
template <int NT, int MT, int U>
__device__ __forceinline__ void w8_load(W8Batch<NT, MT, U>& b, const W8Params& p, const int8_t* a_q, int ntiles, int tb, int stride, int t1, const uint32_t (&wtile)[NT], uint32_t lane,
                                        const uint32_t (&aoff)[MT][2]) {
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const int t = min(tb + stride * u, t1 - 1);
    const int8_t* wt = p.w + (int64_t)t * ntiles * 2048;
#pragma unroll
    for (int i = 0; i < NT; ++i)
#pragma unroll
      for (int s = 0; s < 2; ++s)  // (streamed once: non-temporal, so that they do not drive the activations from L2)
        b.w[u][i][s] = __builtin_nontemporal_load(reinterpret_cast<const v4i*>(wt + wtile[i] + s * 1024u + lane * 16u));
    const int8_t* at = a_q + (int64_t)t * 128;
#pragma unroll
    for (int mt = 0; mt < MT; ++mt)
#pragma unroll
      for (int s = 0; s < 2; ++s) b.a[u][mt][s] = *reinterpret_cast<const v4i*>(at + aoff[mt][s]);
  }
  __builtin_amdgcn_sched_barrier(0);  // all of them ahead of the products that follow
}

template <int NT, int MT, int U>
__device__ __forceinline__ void w8_multiply(const W8Batch<NT, MT, U>& b, v4i (&acc)[MT][NT], int tb, int stride, int t1, int8_t* turn, const uint32_t (&woff)[2],
                                            const uint32_t (&roff)[2]) {
#pragma unroll
  for (int u = 0; u < U; ++u) {
    if (tb + stride * u >= t1) break;
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) {
      v4i a[2] = {b.a[u][mt][0], b.a[u][mt][1]};
      if (turn) {  // wave-uniform; one wave's LDS accesses are served in order
        *reinterpret_cast<v4i*>(turn + woff[0]) = a[0];
        *reinterpret_cast<v4i*>(turn + woff[1]) = a[1];
        a[0] = *reinterpret_cast<const v4i*>(turn + roff[0]);
        a[1] = *reinterpret_cast<const v4i*>(turn + roff[1]);
      }
#pragma unroll
      for (int i = 0; i < NT; ++i)
#pragma unroll
        for (int s = 0; s < 2; ++s) acc[mt][i] = __builtin_amdgcn_mfma_i32_16x16x64_i8(a[s], b.w[u][i][s], acc[mt][i], 0, 0, 0);
    }
  }
}

template <int NT, int MT, int W, int U>
__global__ __launch_bounds__(W * 64) void w8_few_kernel(const W8Params p, const int groups) {
  constexpr int kElems = MT * NT * 256, kThreads = W * 64, kPer = (kElems + kThreads - 1) / kThreads;
  __shared__ __attribute__((aligned(16))) int sums[W * kElems];
  __shared__ __attribute__((aligned(16))) int8_t turns[W * 2048];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int nl = lane & 15, kc = lane >> 4;
  const int row0 = blockIdx.y * 16 * MT;
  const int T = p.K >> 7, ntiles = (p.N + 15) >> 4, M = min(p.M - row0, 16 * MT), N = p.N;  // this workgroup's rows
  const int group = blockIdx.x % groups, split = blockIdx.x / groups;  // neighbours sweep one window of the weights
  const int t0 = (int)((int64_t)split * T / p.k_splits), t1 = (int)((int64_t)(split + 1) * T / p.k_splits);

  v4i acc[MT][NT];
#pragma unroll
  for (int mt = 0; mt < MT; ++mt)
#pragma unroll
    for (int i = 0; i < NT; ++i) acc[mt][i] = (v4i){0, 0, 0, 0};
  if (t0 + wave < t1) {
    uint32_t wtile[NT], aoff[MT][2], woff[2], roff[2];
#pragma unroll
    for (int i = 0; i < NT; ++i) wtile[i] = (uint32_t)min(group * NT + i, ntiles - 1) * 2048u;  // (past the last: it again, not stored)
    const bool row_major = MT > 1 || M > 8;
    const uint32_t r = lane >> 3, c = lane & 7;
#pragma unroll
    for (int s = 0; s < 2; ++s) {
      // chunk c of row r lies in slot c ^ ((r/2)%8): neither the rows' writes nor the operands' reads collide
      woff[s] = (r + 8 * s) * 128 + ((c ^ (((r + 8 * s) >> 1) & 7)) << 4);
      roff[s] = nl * 128 + (((4 * s + kc) ^ ((nl >> 1) & 7)) << 4);
#pragma unroll
      for (int mt = 0; mt < MT; ++mt)
        aoff[mt][s] = row_major ? (uint32_t)min(mt * 16 + 8 * s + (int)r, M - 1) * (uint32_t)p.K + c * 16u
                                : (uint32_t)min(mt * 16 + nl, M - 1) * (uint32_t)p.K + 64u * s + 16u * kc;
    }
    int8_t* const turn = row_major ? turns + wave * 2048 : nullptr;
    const int8_t* const a_q = p.a_q + (int64_t)row0 * p.K;
    constexpr int kStep = W * U;
    W8Batch<NT, MT, U> b0, b1;
    int tb = t0 + wave;
    int more = (t1 - tb - 1) / kStep;  // batches after the first
    w8_load(b0, p, a_q, ntiles, tb, W, t1, wtile, lane, aoff);
    for (; more >= 2; more -= 2) {
      w8_load(b1, p, a_q, ntiles, tb + kStep, W, t1, wtile, lane, aoff);
      w8_multiply(b0, acc, tb, W, t1, turn, woff, roff);
      w8_load(b0, p, a_q, ntiles, tb + 2 * kStep, W, t1, wtile, lane, aoff);
      w8_multiply(b1, acc, tb + kStep, W, t1, turn, woff, roff);
      tb += 2 * kStep;
    }
    if (more == 1) {
      w8_load(b1, p, a_q, ntiles, tb + kStep, W, t1, wtile, lane, aoff);
      w8_multiply(b0, acc, tb, W, t1, turn, woff, roff);
      w8_multiply(b1, acc, tb + kStep, W, t1, turn, woff, roff);
    } else {
      w8_multiply(b0, acc, tb, W, t1, turn, woff, roff);
    }
  }
  // the waves' sums, [wave][row tile][channel tile][register][lane]
#pragma unroll
  for (int mt = 0; mt < MT; ++mt)
#pragma unroll
    for (int i = 0; i < NT; ++i)
#pragma unroll
      for (int v = 0; v < 4; ++v) sums[wave * kElems + ((mt * NT + i) * 4 + v) * 64 + lane] = acc[mt][i][v];
  __syncthreads();
#pragma unroll
  for (int j = 0; j < kPer; ++j) {
    // thread to output: channels of a row side by side
    const int e = tid + kThreads * j, ch = e % (16 * NT), m = e / (16 * NT), n = group * 16 * NT + ch;
    if (e >= kElems || m >= M || n >= N) continue;
    const int at = ((((m >> 4) * NT + (ch >> 4)) * 4 + (m & 3)) << 6) + ((m & 15) >> 2) * 16 + (ch & 15);
    int x = 0;
#pragma unroll
    for (int w = 0; w < W; ++w) x += sums[w * kElems + at];
    if (p.k_splits > 1) p.part[((int64_t)split * p.M + row0 + m) * N + n] = x;
    else w8_store(p, row0 + m, n, x, p.s_a[row0 + m], p.s_w[n]);
  }
}

template <int NT, int MT, int W, int U>
int launch_few(const W8Params& p, hipStream_t st) {
  const int groups = (p.N + 16 * NT - 1) / (16 * NT);
  hipLaunchKernelGGL((w8_few_kernel<NT, MT, W, U>), dim3((unsigned)(groups * p.k_splits), (unsigned)((p.M + 16 * MT - 1) / (16 * MT))), dim3(W * 64), 0, st, p, groups);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return set_error(QQQ_ERR_HIP, "w8a8 launch: %s", hipGetErrorString(e));
  route_note("w8a8 few rows channels=%d rows=%dx%d waves=%d ksplit=%d", 16 * NT, (p.M + 16 * MT - 1) / (16 * MT), 16 * MT, W, p.k_splits);
  return QQQ_OK;
}

}  // namespace

// Rows in workgroups of up to 64, and of fewer while that fills CUs, as even as 16-row tiles allow (us in a graph, by 64 / by fewer: 200 x 128 x 8192 9.8 / 5.6, 50 x 222 x 5120 7.7 / 5.3,
// 64 x 1500 x 2048 5.0 / 4.0); channel tiles: as many as leave two workgroups for three CUs
W8FewShape w8_few_shape(int64_t M, int64_t N, int cus) {
  W8FewShape s;
  const int64_t fill = cus / ((N + 15) / 16), most = (M + 15) / 16, least = (M + 63) / 64;
  s.row_groups = (int)(fill > most ? most : fill > least ? fill : least);
  s.mt = (int)((M + 16 * s.row_groups - 1) / (16 * s.row_groups));
  s.row_groups = (int)((M + 16 * s.mt - 1) / (16 * s.mt));
  s.nt = s.mt <= 2 ? 4 : 2;
  while (s.nt > 1 && (N + 16 * s.nt - 1) / (16 * s.nt) * s.row_groups * 3 < 2 * (int64_t)cus) s.nt >>= 1;
  // Two instead of four where the CU with most channels then has fewer.  us, four / two, one row: 17616 x 10752 39.5 / 34.5, 24000 x 4096 17.6 / 16.2, 40000 x 4096 27.0 / 25.6; where it
  // has as many, 16384 x 4096 11.6 / 12.4, 28672 x 8192 35.9 / 39.4
  auto share = [&](int nt) { return ((N + 16 * nt - 1) / (16 * nt) * s.row_groups + cus - 1) / cus * nt; };
  if (s.nt == 4 && share(2) < share(4)) s.nt = 2;
  return s;
}

int launch_w8_few(const W8Params& p, hipStream_t st) {
  const W8FewShape shape = w8_few_shape(p.M, p.N, num_cus());
  const int mt = shape.mt, nt = shape.nt;
  if (mt == 1) return nt == 4 ? launch_few<4, 1, 8, 1>(p, st) : nt == 2 ? launch_few<2, 1, 8, 2>(p, st) : launch_few<1, 1, 8, 2>(p, st);
  if (mt == 2) return nt == 4 ? launch_few<4, 2, 8, 1>(p, st) : nt == 2 ? launch_few<2, 2, 8, 1>(p, st) : launch_few<1, 2, 8, 2>(p, st);
  if (mt == 3) return nt == 2 ? launch_few<2, 3, 8, 1>(p, st) : launch_few<1, 3, 8, 1>(p, st);
  return nt == 2 ? launch_few<2, 4, 8, 1>(p, st) : launch_few<1, 4, 8, 1>(p, st);
}

// ---- layout

namespace {

__global__ __launch_bounds__(256) void pack_w8_kernel(const int8_t* w, int N, int64_t ldw, int ntiles, int64_t vectors, uint4* packed) {
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (i >= vectors) return;
  const int lane = (int)(i & 63), half = (int)(i >> 6 & 1);
  const int64_t chunk = i >> 7;
  const int64_t n = chunk % ntiles * 16 + (lane & 15), k = chunk / ntiles * 128 + half * 64 + (lane >> 4) * 16;
  packed[i] = n < N ? *reinterpret_cast<const uint4*>(w + n * ldw + k) : make_uint4(0, 0, 0, 0);
}
__global__ __launch_bounds__(256) void unpack_w8_kernel(const uint4* packed, int N, int64_t K, int ntiles, int64_t vectors, int8_t* w) {
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (i >= vectors) return;
  const int lane = (int)(i & 63), half = (int)(i >> 6 & 1);
  const int64_t chunk = i >> 7;
  const int64_t n = chunk % ntiles * 16 + (lane & 15), k = chunk / ntiles * 128 + half * 64 + (lane >> 4) * 16;
  if (n < N) *reinterpret_cast<uint4*>(w + n * K + k) = packed[i];
}

int launched(const char* what) {
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return set_error(QQQ_ERR_HIP, "%s launch: %s", what, hipGetErrorString(e));
  route_note("%s", what);
  return QQQ_OK;
}

}  // namespace

int launch_pack_w8(const int8_t* w, int64_t N, int64_t K, int64_t ldw, int8_t* packed, hipStream_t st) {
  const int64_t ntiles = (N + 15) / 16, vectors = ntiles * K;
  hipLaunchKernelGGL(pack_w8_kernel, dim3((unsigned)((vectors + 255) / 256)), dim3(256), 0, st, w, (int)N, ldw, (int)ntiles, vectors, reinterpret_cast<uint4*>(packed));
  return launched("pack_w8");
}
int launch_unpack_w8(const int8_t* packed, int64_t N, int64_t K, int8_t* w, hipStream_t st) {
  const int64_t ntiles = (N + 15) / 16, vectors = ntiles * K;
  hipLaunchKernelGGL(unpack_w8_kernel, dim3((unsigned)((vectors + 255) / 256)), dim3(256), 0, st, reinterpret_cast<const uint4*>(packed), (int)N, K, (int)ntiles, vectors, w);
  return launched("unpack_w8");
}

}  // namespace qqq
