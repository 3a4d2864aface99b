// Device helpers of the 8-bit integer products (gfx950): the activation, and rows
// of bf16 or fp32 turned into integers.
#pragma once

#include <type_traits>

#include "pa_device.hpp"
#include "pa_ops_internal.h"

namespace pa {

typedef int i32x4 __attribute__((ext_vector_type(4)));

// GELU: x Phi(x) = max(x, 0) - z Q(z), z = |x|, the upper tail Q(z) = 1 - Phi(z) as exp2
// of a polynomial, fitted for these kernels (weighted minimax, linear programming
// over 4,001 points).  Half of the kernels' vector instructions: one exp2, the time of
// four others, and a few more than the polynomial's.
//
// bf16 results: degree 7 over [0, 9].  In fp32 against 64 bits: relative 1.8e-5 for
// x > -3, 3.6e-5 down to -4, 1.1e-4 to -6, 3.8e-4 to -9, below that 1.1e-18 absolute;
// half a bf16 step is 2e-3 to 3.9e-3.  (Degree 6 is 1% off at -7, 32% at -9.)
//
// fp32 results: degree 10 over [0, 8].  Relative 6e-7 for x > -2, 1.1e-6 down to -4,
// 6e-6 to -5, 1.2e-4 to -6, below that 1e-10 absolute (0.5 x (1 + erf) in fp32, which
// cancels there, is 5e-4 off at -4 and takes longer: 29,205 rows, 64 to 2496, 128 us and 92).
__device__ __forceinline__ float tail_of(float x, float z, float p) {
  return fmaf(-z, fast_exp2(p), __builtin_elementwise_maximum(x, 0.f));
}
template <typename T> __device__ __forceinline__ float gelu_for(float x) {
  if constexpr (sizeof(T) == 2) {
    const float z = __builtin_elementwise_minimum(fabsf(x), 9.f);
    float p = -1.2643212130569736e-06f;
    p = fmaf(p, z, 4.878497202298604e-05f);
    p = fmaf(p, z, -0.0008188498904928565f);
    p = fmaf(p, z, 0.008031141944229603f);
    p = fmaf(p, z, -0.05292445048689842f);
    p = fmaf(p, z, -0.45953628420829773f);
    p = fmaf(p, z, -1.1508264541625977f);
    return tail_of(x, z, fmaf(p, z, -1.0000252723693848f));
  } else {
    const float z = __builtin_elementwise_minimum(fabsf(x), 8.f);
    float p = -2.5640650491709494e-08f;
    p = fmaf(p, z, 7.68178097132477e-07f);
    p = fmaf(p, z, -9.893834430840798e-06f);
    p = fmaf(p, z, 6.959781603654847e-05f);
    p = fmaf(p, z, -0.00025399887817911804f);
    p = fmaf(p, z, -5.7297507737530395e-05f);
    p = fmaf(p, z, 0.007021773606538773f);
    p = fmaf(p, z, -0.05249564349651337f);
    p = fmaf(p, z, -0.4592008888721466f);
    p = fmaf(p, z, -1.1511073112487793f);
    return tail_of(x, z, fmaf(p, z, -0.9999998807907104f));
  }
}

template <typename T> struct Row16 {
  static constexpr int E = 16 / (int)sizeof(T);
  T v[E];
};
// Chunk c of a row of K elements, without a branch around the load (which would be
// waited for at once).  ODD: K, at least E, is no multiple of E and rows start
// anywhere; of a chunk that is cut short, or lies behind the row's end, the row's
// last E elements (put_chunk moves them).  Otherwise zeros behind the end.
template <bool ODD, typename T>
__device__ __forceinline__ Row16<T> row_chunk(const T* row, int K, int c) {
  constexpr int E = Row16<T>::E;
  Row16<T> o;
  if constexpr (!ODD) {
    const bool in = E * c < K;
    const uint4 q = *reinterpret_cast<const uint4*>(row + (in ? E * c : 0));
    return __builtin_bit_cast(Row16<T>, in ? q : uint4{0, 0, 0, 0});
  } else {
    __builtin_memcpy(&o, row + (E * c + E <= K ? E * c : K - E), 16);
    return o;
  }
}
// The bits of a chunk's largest magnitude as an fp32 number.
__device__ __forceinline__ uint32_t largest(const Row16<float>& c) {
  uint32_t big = 0;
#pragma unroll
  for (int e = 0; e < 4; ++e) big = max(big, __builtin_bit_cast(uint32_t, c.v[e]) & 0x7fffffffu);
  return big;
}
__device__ __forceinline__ uint32_t largest(const Row16<bf16>& c) {  // two at a time
  typedef unsigned short u16x2 __attribute__((ext_vector_type(2)));
  uint32_t w[4];
  __builtin_memcpy(w, &c, 16);
  u16x2 m = __builtin_bit_cast(u16x2, w[0] & 0x7fff7fffu);
#pragma unroll
  for (int i = 1; i < 4; ++i)
    m = __builtin_elementwise_max(m, __builtin_bit_cast(u16x2, w[i] & 0x7fff7fffu));
  return (uint32_t)max(m[0], m[1]) << 16;
}
// ... over the 16 lanes of a row of lanes.
__device__ __forceinline__ uint32_t row16_max(uint32_t v) {
  const auto step = [&](auto ctrl) {
    v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, decltype(ctrl)::value, 0xF, 0xF, false));
  };
  step(std::integral_constant<int, kQuadSwap1>{});
  step(std::integral_constant<int, kQuadSwap2>{});
  step(std::integral_constant<int, kHalfMirror>{});
  step(std::integral_constant<int, kMirror>{});
  return v;
}
// Chunk c in integers, at q.  ODD: of the row's last E elements those that belong
// there, in place, and zeros.
template <bool ODD, typename T>
__device__ __forceinline__ void put_chunk(int8_t* q, const Row16<T>& x, float inv, int K, int c) {
  constexpr int E = Row16<T>::E;
  typedef typename std::conditional<E == 8, uint64_t, uint32_t>::type W;
  W w = quant4(to_f<T>(x.v[0]), to_f<T>(x.v[1]), to_f<T>(x.v[2]), to_f<T>(x.v[3]), inv);
  if constexpr (E == 8)
    w |= (W)quant4(to_f<T>(x.v[4]), to_f<T>(x.v[5]), to_f<T>(x.v[6]), to_f<T>(x.v[7]), inv) << 32;
  if constexpr (ODD) {
    const int over = E * c + E - K;  // elements behind the end
    w = over >= E ? 0 : over > 0 ? w >> 8 * over : w;
  }
  *reinterpret_cast<W*>(q) = w;
}

}  // namespace pa
