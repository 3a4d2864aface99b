// Dropout from a counter-based generator with the residual add (gfx950):
//   out = r + y 65536 / (65536 - T) where an element's 16 bits are at least T, r elsewhere
// The bits are Philox-4x32-10 (J. Salmon, M. Moraes, R. Dror, D. Shaw, "Parallel random
// numbers: as easy as 1, 2, 3", 2011) of the counter (element / 8, offset) under the key
// seed: a counter's four words are the bits of eight elements, which is what a lane
// works on, so no mask is stored and the backward, the same kernel on the gradient
// without r, draws it again.
//
// What bounds it: memory.  A million rows of 256 in bf16 with the residual take 298 us, 5.15
// TB/s, more than a copy's 4.9; 100,003 rows of 95 in fp32 without it 17.4 us, 4.4 TB/s.  The
// ten rounds are 20 products of 32 bits, of which there are two instructions each (lower
// and upper half), for eight elements: 5 a element, hidden behind the loads.  (16 bits an element, so
// that a call of the generator serves eight: a P is off by at most 2^-17 from what was asked
// for, and the scale is that of the P in use.)
#include "pa_ops_internal.h"
#include "pa_stream.hpp"

namespace pa {
namespace {

struct Words {
  uint32_t w[4];
};
__device__ __forceinline__ Words philox(uint64_t counter, uint64_t offset, uint64_t seed) {
  uint32_t c0 = (uint32_t)counter, c1 = (uint32_t)(counter >> 32);
  uint32_t c2 = (uint32_t)offset, c3 = (uint32_t)(offset >> 32);
  uint32_t k0 = (uint32_t)seed, k1 = (uint32_t)(seed >> 32);
#pragma unroll
  for (int i = 0; i < 10; ++i) {
    const uint64_t a = (uint64_t)0xD2511F53u * c0, b = (uint64_t)0xCD9E8D57u * c2;
    c0 = (uint32_t)(b >> 32) ^ c1 ^ k0;
    c1 = (uint32_t)b;
    c2 = (uint32_t)(a >> 32) ^ c3 ^ k1;
    c3 = (uint32_t)a;
    k0 += 0x9E3779B9u;
    k1 += 0xBB67AE85u;
  }
  return {{c0, c1, c2, c3}};
}

template <typename T> __device__ __forceinline__ void load8(const T* p, float (&v)[8]) {
  if constexpr (sizeof(T) == 2) {
    const bf16x8 b = __builtin_bit_cast(bf16x8, ld_global16<true>(p));
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = (float)b[e];
  } else {
    const f32x4 lo = __builtin_bit_cast(f32x4, ld_global16<true>(p));
    const f32x4 hi = __builtin_bit_cast(f32x4, ld_global16<true>(p + 4));
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      v[e] = lo[e];
      v[e + 4] = hi[e];
    }
  }
}
template <typename T> __device__ __forceinline__ void store8(T* p, const float (&v)[8]) {
  if constexpr (sizeof(T) == 2) {
    bf16x8 b;
#pragma unroll
    for (int e = 0; e < 8; ++e) b[e] = (bf16)v[e];
    st_global16(p, __builtin_bit_cast(uint4, b));
  } else {
    const f32x4 lo{v[0], v[1], v[2], v[3]}, hi{v[4], v[5], v[6], v[7]};
    st_global16(p, __builtin_bit_cast(uint4, lo));
    st_global16(p + 4, __builtin_bit_cast(uint4, hi));
  }
}

template <typename T, bool RES> __global__ void __launch_bounds__(256) k_dropout(DropArgs a) {
  const T* y = reinterpret_cast<const T*>(a.y);
  const T* r = reinterpret_cast<const T*>(a.r);
  T* out = reinterpret_cast<T*>(a.out);
  const uint64_t offset = a.offset + (a.offset_dev ? (uint64_t)a.offset_dev[0] : 0);
  const int64_t step = (int64_t)gridDim.x * 256;
  for (int64_t c = (int64_t)blockIdx.x * 256 + threadIdx.x; c * 8 < a.n; c += step) {
    const int64_t e0 = c * 8;
    const bool whole = e0 + 8 <= a.n;
    float v[8], b[8];
    if (whole) {
      load8(y + e0, v);
      if constexpr (RES) load8(r + e0, b);
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        v[e] = e0 + e < a.n ? to_f<T>(y[e0 + e]) : 0.f;
        if constexpr (RES) b[e] = e0 + e < a.n ? to_f<T>(r[e0 + e]) : 0.f;
      }
    }
    const Words x = philox((uint64_t)c, offset, a.seed);
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const uint32_t bits = e & 1 ? x.w[e / 2] >> 16 : x.w[e / 2] & 0xffffu;
      // (chosen, not multiplied: what is dropped may be an infinity or a NaN)
      const float kept = RES ? fmaf(v[e], a.scale, b[e]) : v[e] * a.scale;
      v[e] = bits >= a.threshold ? kept : RES ? b[e] : 0.f;
    }
    if (whole) {
      store8(out + e0, v);
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e)
        if (e0 + e < a.n) out[e0 + e] = from_f<T>(v[e]);
    }
  }
}

}  // namespace

hipError_t launch_dropout(const DropArgs& a, int dtype, hipStream_t st) {
  const int64_t need = ((a.n + 7) / 8 + 255) / 256;
  const dim3 grid((uint32_t)(need < 2048 ? need : 2048));
  auto go = [&](auto* k) { hipLaunchKernelGGL(k, grid, dim3(256), 0, st, a); };
  if (dtype == 1) a.r ? go(k_dropout<bf16, true>) : go(k_dropout<bf16, false>);
  else a.r ? go(k_dropout<float, true>) : go(k_dropout<float, false>);
  return hipGetLastError();
}

}  // namespace pa
