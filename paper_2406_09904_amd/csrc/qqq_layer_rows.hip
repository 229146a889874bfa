// Row operators between the linear calls: residual addition + root-mean-square norm, and the gated activation, each straight to int8
// codes with a scale a row (or, the norm, to fp16).  One workgroup a row, the row in registers between the reduction and the rounding:
// each input is read once and each output written once.
//
// Norm: y = h rho gain, rho = 1/sqrt(mean h^2 + eps).  rho is common to a row, so codes = rne(h gain / S), S = max |h gain| / 127,
// and s_a = S rho: the sum of squares and the maximum come out of the same pass, and no code depends on how the sum was ordered.
// h gain is exact in fp32 where h is fp16 (11 + 11 bits).
//
// Both are bound by their bytes from some hundred rows on, below that by how soon a row is done (a launch from a graph alone is 1.6 us).
// Norm, fp16 residual, codes: M = 1, K = 4096 2.2 to 2.4 us; M = 777, K = 5120 6.2; M = 4096, K = 8192 37 to 44 (5.3 to 6.3 TB/s, by what the last-level
// cache still holds); fp32 residual, fp16 output: M = 777, K = 5120 9.7 to 10.8, M = 4096, K = 8192 66.  Gated activation: M = 16, F = 11008 3.8 to 4.0 us;
// M = 4096, F = 28672 108 (5.4 TB/s).
//
// Inputs are read past the caches (qqq_past.h) where all operands are more than the last of them: gated activation, M = 4096, F = 28672 (587 MB)
// and a reader of its codes 356 us, 424 otherwise; norm, fp32 residual, M = 4096, K = 8192 (403 MB) 66 against 74.  Smaller calls would lose what
// the call before them has left there: gated, F = 11008 (225 MB) 41 against 34, norm, fp16 residual (235 MB) 43 against 37.
#include "qqq_past.h"
#include "qqq_layer.h"

namespace qqq {

namespace {


constexpr float kLeastScale = 0x1p-120f;  // below it a reciprocal would leave fp32's range: the row counts as zero

__device__ __forceinline__ float wave_sum(float v) {
  auto add = [&](int moved) { v += __builtin_bit_cast(float, moved); };
  add(__builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), 0xB1, 0xF, 0xF, false));   // quad_perm [1,0,3,2]
  add(__builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), 0x4E, 0xF, 0xF, false));   // quad_perm [2,3,0,1]
  add(__builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), 0x141, 0xF, 0xF, false));  // row_half_mirror
  add(__builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), 0x140, 0xF, 0xF, false));  // row_mirror
  auto lane = [&](int l) { return __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, v), l)); };
  return (lane(0) + lane(16)) + (lane(32) + lane(48));
}

// Largest magnitude and sum over the workgroup, in every thread; the order of the sum is fixed.
template <int T>
__device__ __forceinline__ void block_max_sum(float& amax, float& sum, float2* smem) {
  const float m = __builtin_bit_cast(float, wave_max_u32(__builtin_bit_cast(uint32_t, amax)));  // (not negative: ordered as its bits are)
  const float s = wave_sum(sum);
  if constexpr (T == 64) {
    amax = m;
    sum = s;
    return;
  }
  if ((threadIdx.x & 63) == 0) smem[threadIdx.x >> 6] = make_float2(m, s);
  __syncthreads();
  amax = sum = 0.0f;
#pragma unroll
  for (int i = 0; i < T / 64; ++i) {
    const float2 v = smem[i];
    amax = fmaxf(amax, v.x);
    sum += v.y;
  }
}

__device__ __forceinline__ void halves_to_floats(uint4 v, float* f) {
  const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
  for (int i = 0; i < 8; ++i) f[i] = half_bits_to_float(i & 1 ? w[i >> 1] >> 16 : w[i >> 1] & 0xFFFFu);
}
__device__ __forceinline__ uint4 floats_to_halves(const float* f) {
  uint32_t w[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) w[i] = as_u32(h2{(_Float16)f[2 * i], (_Float16)f[2 * i + 1]});
  return make_uint4(w[0], w[1], w[2], w[3]);
}

// rne(t / S) of eight values, |t| <= 127 S (1 + 2^-23): the correctly rounded quotient, rounded to an integer by adding 1.5 * 2^23, whose
// low byte is the code (see quant8_act)
__device__ __forceinline__ uint2 quant8_f32(const float* t, float s, float y) {
  uint32_t b[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) b[i] = __builtin_bit_cast(uint32_t, quotient(t[i], s, y) + 12582912.0f);
  auto bytes = [&](int i) {  // v_perm_b32: selector bytes 0-3 pick from the second source, 4-7 from the first
    return __builtin_amdgcn_perm(__builtin_amdgcn_perm(b[i + 3], b[i + 2], 0x0C0C0400u), __builtin_amdgcn_perm(b[i + 1], b[i], 0x0C0C0400u), 0x05040100u);
  };
  return make_uint2(bytes(0), bytes(4));
}

struct NormParams {
  const uint4* x;
  const uint4* residual;  // fp16: a vector holds 8 values, fp32: two vectors do
  const uint4* gain;
  uint4* sum_out;
  uint4* y;      // fp16 output, or
  uint2* a_q;    // codes and
  float* s_a;    // scales
  int64_t ldx, ldr, lds;  // in units of 8 values
  float eps, inv_k;
  int nvec;
};

// RES: QQQ_RESIDUAL_*.  VPT > 0: the row is VPT vectors of 8 values per thread; VPT == 0: any K, the row is read twice.
template <int RES, bool QUANT, int VPT, int T, bool PAST>
__global__ __launch_bounds__(T) void rmsnorm_kernel(const NormParams p) {
  __shared__ float2 smem[T / 64];
  const int64_t m = blockIdx.x;
  const uint4* x = p.x + m * p.ldx;
  const uint4* res = RES == QQQ_RESIDUAL_NONE ? nullptr : p.residual + m * p.ldr * (RES == QQQ_RESIDUAL_FP32 ? 2 : 1);
  uint4* out = RES == QQQ_RESIDUAL_NONE ? nullptr : p.sum_out + m * p.lds * (RES == QQQ_RESIDUAL_FP32 ? 2 : 1);

  constexpr int RV = RES == QQQ_RESIDUAL_FP32 ? 2 : 1;
  struct Raw {
    uint4 x, r[RV];
  };
  auto request = [&](int idx, Raw& w) {
    w.x = load16<PAST>(x + idx);
    if constexpr (RES != QQQ_RESIDUAL_NONE) {
#pragma unroll
      for (int i = 0; i < RV; ++i) w.r[i] = load16<PAST>(res + (int64_t)idx * RV + i);
    }
  };
  // the sum as it is stored, in fp32
  auto add = [&](int idx, const Raw& w, float* h, bool store) {
    halves_to_floats(w.x, h);
    if constexpr (RES == QQQ_RESIDUAL_FP16) {
      float r[8];
      halves_to_floats(w.r[0], r);
#pragma unroll
      for (int i = 0; i < 8; ++i) h[i] += r[i];
      const uint4 s = floats_to_halves(h);
      if (store) out[idx] = s;
      halves_to_floats(s, h);
    } else if constexpr (RES == QQQ_RESIDUAL_FP32) {
      const uint32_t r[8] = {w.r[0].x, w.r[0].y, w.r[0].z, w.r[0].w, w.r[RV - 1].x, w.r[RV - 1].y, w.r[RV - 1].z, w.r[RV - 1].w};
#pragma unroll
      for (int i = 0; i < 8; ++i) h[i] += __builtin_bit_cast(float, r[i]);
      if (store) {
#pragma unroll
        for (int i = 0; i < 2; ++i)
          out[(int64_t)idx * 2 + i] = make_uint4(__builtin_bit_cast(uint32_t, h[4 * i]), __builtin_bit_cast(uint32_t, h[4 * i + 1]),
                                                 __builtin_bit_cast(uint32_t, h[4 * i + 2]), __builtin_bit_cast(uint32_t, h[4 * i + 3]));
      }
    }
  };
  float amax = 0.0f, sum = 0.0f;
  auto gather = [&](int idx, float* h) {  // h becomes h * gain
    float g[8];
    halves_to_floats(p.gain[idx], g);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      sum = __builtin_fmaf(h[i], h[i], sum);
      h[i] *= g[i];
      if constexpr (QUANT) amax = fmaxf(amax, fabsf(h[i]));
    }
  };
  float rho = 0.0f, s = 0.0f, inv = 0.0f;
  auto reduced = [&]() {
    block_max_sum<T>(amax, sum, smem);
    const float root = __builtin_sqrtf(__builtin_fmaf(sum, p.inv_k, p.eps));
    rho = root > 0.0f ? 1.0f / root : 0.0f;
    if constexpr (QUANT) {
      s = amax / 127.0f;
      if (!(s >= kLeastScale)) s = 0.0f;
      inv = reciprocal_near(s);
      if (threadIdx.x == 0) p.s_a[m] = s * rho;
    }
  };
  auto emit = [&](int idx, float* t) {
    if constexpr (QUANT) {
      p.a_q[m * p.nvec + idx] = s == 0.0f ? make_uint2(0, 0) : quant8_f32(t, s, inv);
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) t[i] *= rho;
      p.y[m * p.nvec + idx] = floats_to_halves(t);
    }
  };
  if constexpr (VPT > 0) {
    Raw raw[VPT];
    float t[VPT][8];
#pragma unroll
    for (int j = 0; j < VPT; ++j) {
      const int idx = threadIdx.x + T * j;
      if (idx < p.nvec) request(idx, raw[j]);
    }
#pragma unroll
    for (int j = 0; j < VPT; ++j) {
      const int idx = threadIdx.x + T * j;
      if (idx < p.nvec) {
        add(idx, raw[j], t[j], true);
        gather(idx, t[j]);
      }
    }
    reduced();
#pragma unroll
    for (int j = 0; j < VPT; ++j) {
      const int idx = threadIdx.x + T * j;
      if (idx < p.nvec) emit(idx, t[j]);
    }
  } else {
    for (int idx = threadIdx.x; idx < p.nvec; idx += T) {
      Raw w;
      float h[8];
      request(idx, w);
      add(idx, w, h, true);
      gather(idx, h);
    }
    reduced();
    for (int idx = threadIdx.x; idx < p.nvec; idx += T) {
      // the stored sum: sum_out may be the residual's place, so adding again would count x twice
      float h[8], g[8];
      if constexpr (RES == QQQ_RESIDUAL_FP32) {
        const uint4 a = out[(int64_t)idx * 2], b = out[(int64_t)idx * 2 + 1];
        const uint32_t r[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
#pragma unroll
        for (int i = 0; i < 8; ++i) h[i] = __builtin_bit_cast(float, r[i]);
      } else {
        halves_to_floats(RES == QQQ_RESIDUAL_NONE ? x[idx] : out[idx], h);
      }
      halves_to_floats(p.gain[idx], g);
#pragma unroll
      for (int i = 0; i < 8; ++i) h[i] *= g[i];
      emit(idx, h);
    }
  }
}

template <int RES, bool QUANT>
void launch_rmsnorm_t(const NormParams& p, int64_t M, bool past, hipStream_t st) {
#define QQQ_NORM(V, T)                                                                                                  \
  do {                                                                                                                  \
    if (V == 0 || !past) hipLaunchKernelGGL((rmsnorm_kernel<RES, QUANT, V, T, false>), dim3((unsigned)M), dim3(T), 0, st, p); \
    else hipLaunchKernelGGL((rmsnorm_kernel<RES, QUANT, V, T, V != 0>), dim3((unsigned)M), dim3(T), 0, st, p);              \
  } while (0)
  if (p.nvec <= 64) QQQ_NORM(1, 64);
  else if (p.nvec <= 256) QQQ_NORM(1, 256);
  else if (M <= num_cus() && p.nvec <= 2048) {
    // A row per CU at most: what counts is how soon it is done (M = 1, K = 8192 3.1 us against 3.6 with 256 threads; M = 200 4.2 against 4.5)
    if (p.nvec <= 512) QQQ_NORM(1, 512);
    else if (p.nvec <= 1024) QQQ_NORM(1, 1024);
    else QQQ_NORM(2, 1024);
  } else if (p.nvec <= 512) QQQ_NORM(2, 256);
  else if (p.nvec <= 1024) QQQ_NORM(4, 256);
  else if (p.nvec <= 2048) QQQ_NORM(4, 512);
  else if (p.nvec <= 4096) QQQ_NORM(4, 1024);
  else QQQ_NORM(0, 1024);
#undef QQQ_NORM
}

template <int ACT>
__device__ __forceinline__ float gate_act(float g) {
  if constexpr (ACT == QQQ_ACT_SILU) {
    return g * __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(g * -1.44269504088896340736f));
  } else {
    // (1 + tanh(u)) / 2 = 1 / (1 + exp(-2u)), u = sqrt(2/pi) (g + 0.044715 g^3)
    const float u = g * __builtin_fmaf(0.044715f * g, g, 1.0f);
    return g * __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(u * (-2.0f * 1.44269504088896340736f * 0.79788456080286535588f)));
  }
}

struct GatedParams {
  const uint4 *gate, *up;
  uint2* a_q;
  float* s_a;
  int64_t ldg, ldu;  // in units of 8 values
  int nvec;
};

template <int ACT, int VPT, int T, bool PAST>
__global__ __launch_bounds__(T) void gated_act_kernel(const GatedParams p) {
  __shared__ float2 smem[T / 64];
  const int64_t m = blockIdx.x;
  const uint4 *gate = p.gate + m * p.ldg, *up = p.up + m * p.ldu;
  float amax = 0.0f, none = 0.0f;
  auto product = [&](uint4 vg, uint4 vu, float* h) {
    float u[8];
    halves_to_floats(vg, h);
    halves_to_floats(vu, u);
#pragma unroll
    for (int i = 0; i < 8; ++i) h[i] = gate_act<ACT>(h[i]) * u[i];
  };
  auto largest = [&](const float* h) {
#pragma unroll
    for (int i = 0; i < 8; ++i) amax = fmaxf(amax, fabsf(h[i]));
  };
  float s = 0.0f, inv = 0.0f;
  auto reduced = [&]() {
    block_max_sum<T>(amax, none, smem);
    s = amax / 127.0f;
    if (!(s >= kLeastScale)) s = 0.0f;
    inv = reciprocal_near(s);
    if (threadIdx.x == 0) p.s_a[m] = s;
  };
  auto emit = [&](int idx, const float* h) { p.a_q[m * p.nvec + idx] = s == 0.0f ? make_uint2(0, 0) : quant8_f32(h, s, inv); };
  if constexpr (VPT > 0) {
    uint4 vg[VPT], vu[VPT];
    float h[VPT][8];
#pragma unroll
    for (int j = 0; j < VPT; ++j) {
      const int idx = threadIdx.x + T * j;
      if (idx < p.nvec) {
        vg[j] = load16<PAST>(gate + idx);
        vu[j] = load16<PAST>(up + idx);
      }
    }
#pragma unroll
    for (int j = 0; j < VPT; ++j) {
      const int idx = threadIdx.x + T * j;
      if (idx < p.nvec) {
        product(vg[j], vu[j], h[j]);
        largest(h[j]);
      }
    }
    reduced();
#pragma unroll
    for (int j = 0; j < VPT; ++j) {
      const int idx = threadIdx.x + T * j;
      if (idx < p.nvec) emit(idx, h[j]);
    }
  } else {
    for (int idx = threadIdx.x; idx < p.nvec; idx += T) {
      float h[8];
      product(gate[idx], up[idx], h);
      largest(h);
    }
    reduced();
    for (int idx = threadIdx.x; idx < p.nvec; idx += T) {
      float h[8];
      product(gate[idx], up[idx], h);
      emit(idx, h);
    }
  }
}

template <int ACT>
void launch_gated_t(const GatedParams& p, int64_t M, bool past, hipStream_t st) {
#define QQQ_GATED(V, T)                                                                                             \
  do {                                                                                                              \
    if (V == 0 || !past) hipLaunchKernelGGL((gated_act_kernel<ACT, V, T, false>), dim3((unsigned)M), dim3(T), 0, st, p); \
    else hipLaunchKernelGGL((gated_act_kernel<ACT, V, T, V != 0>), dim3((unsigned)M), dim3(T), 0, st, p);                \
  } while (0)
  if (p.nvec <= 64) QQQ_GATED(1, 64);
  else if (p.nvec <= 256) QQQ_GATED(1, 256);
  else if (p.nvec <= 512) QQQ_GATED(2, 256);
  else if (p.nvec <= 1024) QQQ_GATED(4, 256);
  else if (p.nvec <= 2048) QQQ_GATED(4, 512);
  else if (p.nvec <= 4096) QQQ_GATED(4, 1024);
  else QQQ_GATED(0, 1024);
#undef QQQ_GATED
}

}  // namespace

int launch_rmsnorm(const void* x, int64_t ldx, const void* residual, int64_t ldr, int residual_type, const void* gain, float eps, int64_t M,
                   int64_t K, void* sum_out, int64_t lds, void* y, int8_t* a_q, float* s_a, hipStream_t st) {
  NormParams p;
  p.x = (const uint4*)x;
  p.residual = (const uint4*)residual;
  p.gain = (const uint4*)gain;
  p.sum_out = (uint4*)sum_out;
  p.y = (uint4*)y;
  p.a_q = (uint2*)a_q;
  p.s_a = s_a;
  p.ldx = ldx / 8;
  p.ldr = ldr / 8;
  p.lds = lds / 8;
  p.eps = eps;
  p.inv_k = 1.0f / (float)K;
  p.nvec = (int)(K / 8);
  const bool q = a_q != nullptr;
  const int of_residual = residual_type == QQQ_RESIDUAL_NONE ? 0 : residual_type == QQQ_RESIDUAL_FP16 ? 4 : 8;  // bytes read and written of a value
  const bool past = M * K * (2 + of_residual + (q ? 1 : 2)) > kLastCacheBytes;
  if (residual_type == QQQ_RESIDUAL_NONE) q ? launch_rmsnorm_t<QQQ_RESIDUAL_NONE, true>(p, M, past, st) : launch_rmsnorm_t<QQQ_RESIDUAL_NONE, false>(p, M, past, st);
  else if (residual_type == QQQ_RESIDUAL_FP16) q ? launch_rmsnorm_t<QQQ_RESIDUAL_FP16, true>(p, M, past, st) : launch_rmsnorm_t<QQQ_RESIDUAL_FP16, false>(p, M, past, st);
  else q ? launch_rmsnorm_t<QQQ_RESIDUAL_FP32, true>(p, M, past, st) : launch_rmsnorm_t<QQQ_RESIDUAL_FP32, false>(p, M, past, st);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return set_error(QQQ_ERR_HIP, "rmsnorm launch: %s", hipGetErrorString(e));
  route_note("rmsnorm");
  return QQQ_OK;
}

int launch_gated_act(const void* gate, int64_t ldg, const void* up, int64_t ldu, int act, int64_t M, int64_t F, int8_t* a_q, float* s_a,
                     hipStream_t st) {
  GatedParams p;
  p.gate = (const uint4*)gate;
  p.up = (const uint4*)up;
  p.a_q = (uint2*)a_q;
  p.s_a = s_a;
  p.ldg = ldg / 8;
  p.ldu = ldu / 8;
  p.nvec = (int)(F / 8);
  const bool past = M * F * 5 > kLastCacheBytes;
  act == QQQ_ACT_SILU ? launch_gated_t<QQQ_ACT_SILU>(p, M, past, st) : launch_gated_t<QQQ_ACT_GELU_TANH>(p, M, past, st);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return set_error(QQQ_ERR_HIP, "gated_act launch: %s", hipGetErrorString(e));
  route_note("gated_act");
  return QQQ_OK;
}

}  // namespace qqq
