// Linear layers in 8-bit integers (gfx950): rows quantised with a scale each,
// integer products on v_mfma_i32_16x16x64_i8 (exact in 32 bits), and the scales,
// bias, activation and residual add on the way out.
//
// The weights are the MFMA's A operand and the points its B operand, so that a
// lane of a 16 x 16 result tile holds four consecutive channels of one point.
#include "pa_device.hpp"
#include "pa_ops_internal.h"

namespace pa {
namespace {

typedef int i32x4 __attribute__((ext_vector_type(4)));

__device__ __forceinline__ float gelu_exact(float x) {
  return 0.5f * x * (1.f + erff(x * 0.7071067811865476f));
}

template <typename T>
__device__ __forceinline__ float finish(const I8Args& a, int64_t n, int f, int sum, float s) {
  float u = (float)sum * (s * a.sw[f]);
  if (a.bias) u += a.bias[f];
  if (a.act == PA_ACT_GELU) u = gelu_exact(u);
  if (a.C) u += to_f<T>(reinterpret_cast<const T*>(a.C)[n * a.F + f]);
  return u;
}

// 16 points x 64 channels per wave, operands straight from memory; points past
// N and channels past F read the last one and are not stored.
template <typename T>
__global__ void __launch_bounds__(256) k_gemm_i8(I8Args a) {
  const int lane = lane_id(), r = lane & 15, g = lane >> 4;
  const int64_t n0 = (int64_t)blockIdx.x * 16;
  const int f0 = ((int)blockIdx.y * 4 + (int)(threadIdx.x >> 6)) * 64;
  if (f0 >= a.F) return;
  const int64_t n = n0 + r < a.N ? n0 + r : a.N - 1;
  i32x4 acc[4];
  for (int t = 0; t < 4; ++t) acc[t] = i32x4{0, 0, 0, 0};
  for (int k = 16 * g; k < (a.Kp + 63) / 64 * 64; k += 64) {
    const i32x4 zero = {0, 0, 0, 0};
    const bool in = k < a.Kp;
    const i32x4 x = in ? *reinterpret_cast<const i32x4*>(a.q + n * a.Kp + k) : zero;
    for (int t = 0; t < 4; ++t) {
      const int f = f0 + 16 * t + r < a.F ? f0 + 16 * t + r : a.F - 1;
      const i32x4 w = in ? *reinterpret_cast<const i32x4*>(a.w + (int64_t)f * a.Kp + k) : zero;
      acc[t] = __builtin_amdgcn_mfma_i32_16x16x64_i8(w, x, acc[t], 0, 0, 0);
    }
  }
  if (n0 + r >= a.N) return;
  const float s = a.s[n];
  for (int t = 0; t < 4; ++t)
    for (int i = 0; i < 4; ++i) {
      const int f = f0 + 16 * t + 4 * g + i;
      if (f < a.F) reinterpret_cast<T*>(a.D)[n * a.F + f] = from_f<T>(finish<T>(a, n, f, acc[t][i], s));
    }
}

// A block per row.
template <typename T>
__global__ void __launch_bounds__(256) k_quant_rows(int64_t N, int K, int Kp, const T* x,
                                                    int8_t* q, float* s) {
  __shared__ uint32_t red[4];
  for (int64_t n = blockIdx.x; n < N; n += gridDim.x) {
    uint32_t big = 0;
    for (int k = threadIdx.x; k < K; k += blockDim.x)
      big = max(big, __builtin_bit_cast(uint32_t, fabsf(to_f<T>(x[n * K + k]))));
    for (int o = 1; o < 64; o <<= 1) big = max(big, (uint32_t)__shfl_xor((int)big, o));
    __syncthreads();
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = big;
    __syncthreads();
    const QuantScale c = quant_scale(max(max(red[0], red[1]), max(red[2], red[3])));
    for (int k = threadIdx.x; k < Kp; k += blockDim.x)
      q[n * Kp + k] = k < K ? (int8_t)quant1(to_f<T>(x[n * K + k]), c.inv) : (int8_t)0;
    if (threadIdx.x == 0) s[n] = c.s;
  }
}

// A block per 64 channels: column maxima, then the columns turned into rows.
template <typename T>
__global__ void __launch_bounds__(256) k_quant_weight(int K, int Kp, int F, const T* W,
                                                      int8_t* q, float* sw) {
  __shared__ uint32_t red[4][64];
  const int fl = threadIdx.x & 63, part = threadIdx.x >> 6;
  const int f = blockIdx.x * 64 + fl;
  uint32_t big = 0;
  if (f < F)
    for (int k = part; k < K; k += 4)
      big = max(big, __builtin_bit_cast(uint32_t, fabsf(to_f<T>(W[(int64_t)k * F + f]))));
  red[part][fl] = big;
  __syncthreads();
  if (f >= F) return;
  const QuantScale c =
      quant_scale(max(max(red[0][fl], red[1][fl]), max(red[2][fl], red[3][fl])));
  for (int k = part; k < Kp; k += 4)
    q[(int64_t)f * Kp + k] =
        k < K ? (int8_t)quant1(to_f<T>(W[(int64_t)k * F + f]), c.inv) : (int8_t)0;
  if (part == 0) sw[f] = c.s;
}

}  // namespace

bool gemm_i8_fused_quant(int64_t N, int F, int K) { return false; }

hipError_t launch_gemm_i8(const I8Args& a, int d_dtype, hipStream_t st) {
  const int64_t gx = (a.N + 15) / 16, gy = (a.F + 255) / 256;
  if (a.N < 1 || a.F < 1 || gx > 0x7fffffff || gy > 65535) return hipErrorInvalidValue;
  const dim3 grid((unsigned)gx, (unsigned)gy);
  if (d_dtype == 1)
    hipLaunchKernelGGL(k_gemm_i8<bf16>, grid, dim3(256), 0, st, a);
  else
    hipLaunchKernelGGL(k_gemm_i8<float>, grid, dim3(256), 0, st, a);
  return hipGetLastError();
}

hipError_t launch_quant_rows(int64_t N, int K, int dtype, const void* x, int8_t* q, float* s,
                             hipStream_t st) {
  const int Kp = (K + 15) / 16 * 16;
  const dim3 grid((unsigned)(N < 65536 ? N : 65536));
  if (dtype == 1)
    hipLaunchKernelGGL(k_quant_rows<bf16>, grid, dim3(256), 0, st, N, K, Kp, (const bf16*)x, q, s);
  else
    hipLaunchKernelGGL(k_quant_rows<float>, grid, dim3(256), 0, st, N, K, Kp, (const float*)x, q, s);
  return hipGetLastError();
}

hipError_t launch_quant_weight(int K, int F, int dtype, const void* W, int8_t* Wq, float* sw,
                               hipStream_t st) {
  const int Kp = (K + 15) / 16 * 16;
  const dim3 grid((unsigned)((F + 63) / 64));
  if (dtype == 1)
    hipLaunchKernelGGL(k_quant_weight<bf16>, grid, dim3(256), 0, st, K, Kp, F, (const bf16*)W, Wq, sw);
  else
    hipLaunchKernelGGL(k_quant_weight<float>, grid, dim3(256), 0, st, K, Kp, F, (const float*)W, Wq,
                       sw);
  return hipGetLastError();
}

}  // namespace pa
