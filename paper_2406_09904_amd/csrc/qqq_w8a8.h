// What the W8A8 kernels are given, and their last step (qqq_gemm_w8a8_few.hip, qqq_gemm_w8a8_tiles.hip; layout and formula: qqq_serve.h).
#pragma once

#include "qqq_internal.h"
#include "qqq_serve.h"

namespace qqq {

struct W8Params {
  const int8_t* a_q;   // [M,K]
  const float* s_a;    // [M]
  const int8_t* w;     // packed: 2 KiB chunks [K/128][ceil(N/16)], each two 1 KiB halves of 64 k: lane l's 16 bytes are channel l%16, k 16 (l/16) ..
  const float* s_w;    // [N]
  void* y;             // [M,ldy] fp16 or fp32
  int64_t ldy;
  int32_t* acc_out;    // [M,N] or nullptr
  int32_t* part;       // k_splits > 1: [k_splits][M][N] partial sums
  int M, N, K, k_splits;
  bool f32;            // the output's type
};

// One product rounded once to the output's type
__device__ __forceinline__ float w8_scaled(int acc, float sa, float sw) { return (float)acc * sa * sw; }

__device__ __forceinline__ void w8_store(const W8Params& p, int m, int n, int acc, float sa, float sw) {
  const int64_t at = (int64_t)m * p.ldy + n;
  if (p.f32) static_cast<float*>(p.y)[at] = w8_scaled(acc, sa, sw);
  else static_cast<_Float16*>(p.y)[at] = dequant(acc, sa, sw);
  if (p.acc_out) p.acc_out[(int64_t)m * p.N + n] = acc;
}

constexpr int kW8FewRows = 4096;  // rows that the few-rows kernel is considered for (64 a workgroup)

int launch_pack_w8(const int8_t* w, int64_t N, int64_t K, int64_t ldw, int8_t* packed, hipStream_t st);
int launch_unpack_w8(const int8_t* packed, int64_t N, int64_t K, int8_t* w, hipStream_t st);

// How a call is launched: a rule on the sizes (w8_plan in qqq_gemm_w8a8_tiles.hip)
enum W8ShapeId : int { kW8Few = 1, kW8Tile256x256, kW8Tile192x256, kW8Tile128x256, kW8Tile128x128, kW8Tile64x128 };  // (numbered as in qqq_tuning.h)
struct W8Plan {
  int shape, k_splits;
};
W8Plan w8_plan(int64_t M, int64_t N, int64_t K);
struct W8FewShape {
  int row_groups, mt, nt;  // workgroups over the rows; row tiles and channel tiles of 16 each
};
W8FewShape w8_few_shape(int64_t M, int64_t N, int cus);
int launch_w8_few(const W8Params& p, hipStream_t st);
int launch_w8_tiles(const W8Params& p, int shape, hipStream_t st);
int launch_w8_sum(const W8Params& p, hipStream_t st);

}  // namespace qqq
