// One AdamW step over many tensors (gfx950), moments in fp32 or in 8 bits; the
// formulas and the 8-bit code are in include/pa_ops.h.
//
// A launch takes up to kAdamMax tensors, described in its arguments.  A block
// works on 16 units of 256 consecutive elements of one tensor, a wave on four of
// them, four elements per lane: a unit is a block of the 8-bit moments, whose
// largest magnitude is a reduction within the wave.
#include "pa_device.hpp"
#include "pa_ops_internal.h"

namespace pa {

// (host and device)
__host__ __device__ static inline uint32_t fmix32(uint32_t h) {
  h = (h ^ (h >> 16)) * 0x85EBCA6Bu;
  h = (h ^ (h >> 13)) * 0xC2B2AE35u;
  return h ^ (h >> 16);
}
__host__ __device__ static inline uint32_t mix32(uint32_t a, uint32_t b) {
  return fmix32(a ^ (b * 0x9E3779B9u));
}
uint32_t adam_mix(uint32_t a, uint32_t b) { return mix32(a, b); }

namespace {

constexpr int kUnit = 256;   // elements of a unit (of a scale of the 8-bit moments)
constexpr int kWaveUnits = 4;
constexpr int kBlockElems = kUnit * kWaveUnits * 4;

// The launch's arguments where the kernel was given them: indexing the
// by-value copy at run time would move it to scratch memory.
typedef const __attribute__((address_space(4))) AdamBatch* ArgPtr;
__device__ __forceinline__ ArgPtr kernel_args() {
  return (ArgPtr)__builtin_amdgcn_kernarg_segment_ptr();
}

__device__ __forceinline__ float level(uint32_t c, uint32_t lo) {
  return c ? __builtin_bit_cast(float, (c + lo) << 20) : 0.f;
}
constexpr uint32_t kLoM = 889, kLoV = 761;

// The block's scale from the bits of its largest magnitude.
__device__ __forceinline__ float block_scale(uint32_t big) {
  if (big >= 0x7f800000u) return __builtin_nanf("");
  if (big == 0) return 0.f;
  uint32_t up = (big & 0x7f800000u) + ((big & 0x7fffffu) ? 0x800000u : 0u);
  up = up < 0x00800000u ? 0x00800000u : up > 0x7F000000u ? 0x7F000000u : up;
  return __builtin_bit_cast(float, up);
}
__device__ __forceinline__ int code_of(float mag, float inv, uint32_t h, uint32_t lo) {
  return (int)((__builtin_bit_cast(uint32_t, mag * inv) + 16 * h + 8) >> 20) - (int)lo;
}

struct Consts {
  float b1, b2, c1, c2, gs, ss, rs, eps, lrwd;
};

// p, m, v of one element after the step (the moments without fused
// multiply-adds, as documented).
__device__ __forceinline__ void update(const Consts& k, float g, float& p, float& m, float& v) {
  {
#pragma clang fp contract(off)
    g = g * k.gs;
    m = m * k.b1 + g * k.c1;
    v = v * k.b2 + (g * g) * k.c2;
  }
  const float den = fmaf(sqrtf(v), k.rs, k.eps);
  p -= fmaf(k.lrwd, p, k.ss * (m / den));
}

__global__ void __launch_bounds__(256) k_adamw(AdamBatch by_value) {
  const ArgPtr A = kernel_args();
  // the item of this block: the last one that starts at or before it
  const uint32_t b = blockIdx.x;
  int lo = 0, hi = A->n;
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (A->first[mid] <= b) lo = mid;
    else hi = mid;
  }
  const int k = lo;
  const int64_t n = A->it[k].n;
  float* P = A->it[k].p;
  bf16* CP = reinterpret_cast<bf16*>(A->it[k].copy);
  const void* G = A->it[k].g;
  void* M = A->it[k].m;
  void* V = A->it[k].v;
  float* MS = A->it[k].ms;
  float* VS = A->it[k].vs;
  const uint32_t bits = A->it[k].bits;

  Consts c;
  c.b1 = A->b1; c.b2 = A->b2; c.c1 = A->c1; c.c2 = A->c2;
  c.gs = A->gscale ? *A->gscale : 1.f;
  const double lr = A->lr_dev ? (double)*A->lr_dev : A->lr;
  const int64_t step = A->step_dev ? *A->step_dev : A->step;
  c.ss = (float)(lr / (1.0 - exp2((double)step * A->log2b1)));
  c.rs = (float)(1.0 / sqrt(1.0 - exp2((double)step * A->log2b2)));
  c.eps = (float)A->eps;
  c.lrwd = (float)(lr * (double)A->it[k].wd);
  const uint32_t key = mix32(mix32(A->seed_key, (uint32_t)step), (uint32_t)(A->base + k));

  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  for (int w = 0; w < kWaveUnits; ++w) {
    const int64_t unit = ((int64_t)(b - A->first[k]) * 4 + wave) * kWaveUnits + w;
    const int64_t i0 = unit * kUnit + 4 * lane;
    if (unit * kUnit >= n) break;
    const int live = n - i0 >= 4 ? 4 : n > i0 ? (int)(n - i0) : 0;  // of this lane's four
    float p[4], g[4], m[4], v[4];
    uint32_t mc = 0, vc = 0;
    float sm = 0.f, sv = 0.f;
    if (bits & 2) {
      sm = MS[unit];
      sv = VS[unit];
    }
    for (int e = 0; e < 4; ++e) {
      p[e] = g[e] = m[e] = v[e] = 0.f;
      if (e < live) {
        p[e] = P[i0 + e];
        g[e] = bits & 1 ? (float)reinterpret_cast<const bf16*>(G)[i0 + e]
                        : reinterpret_cast<const float*>(G)[i0 + e];
        if (bits & 2) {
          const uint32_t x = reinterpret_cast<const uint8_t*>(M)[i0 + e];
          const float mag = level(x & 127, kLoM) * sm;
          m[e] = x & 128 ? -mag : mag;
          v[e] = level(reinterpret_cast<const uint8_t*>(V)[i0 + e], kLoV) * sv;
        } else {
          m[e] = reinterpret_cast<const float*>(M)[i0 + e];
          v[e] = reinterpret_cast<const float*>(V)[i0 + e];
        }
      }
    }
    for (int e = 0; e < 4; ++e) update(c, g[e], p[e], m[e], v[e]);
    for (int e = 0; e < live; ++e) {
      P[i0 + e] = p[e];
      if (CP) CP[i0 + e] = (bf16)p[e];
    }
    if (!(bits & 2)) {
      for (int e = 0; e < live; ++e) {
        reinterpret_cast<float*>(M)[i0 + e] = m[e];
        reinterpret_cast<float*>(V)[i0 + e] = v[e];
      }
      continue;
    }
    uint32_t bm = 0, bv = 0;
    for (int e = 0; e < 4; ++e)
      if (e < live) {
        bm = max(bm, __builtin_bit_cast(uint32_t, fabsf(m[e])));
        bv = max(bv, __builtin_bit_cast(uint32_t, v[e]));
      }
    for (int o = 1; o < 64; o <<= 1) {
      bm = max(bm, (uint32_t)__shfl_xor((int)bm, o));
      bv = max(bv, (uint32_t)__shfl_xor((int)bv, o));
    }
    sm = block_scale(bm);
    sv = block_scale(bv);
    const float im = sm == 0.f ? 0.f : __fdiv_rn(1.f, sm), iv = sv == 0.f ? 0.f : __fdiv_rn(1.f, sv);
    const uint32_t kb = mix32(key, (uint32_t)unit);
    for (int e = 0; e < live; ++e) {
      const uint32_t h = fmix32(kb + (uint32_t)(4 * lane + e));
      int x = code_of(fabsf(m[e]), im, h & 0xffffu, kLoM);
      x = x < 0 ? 0 : x > 127 ? 127 : x;
      if (x && m[e] < 0.f) x |= 128;
      int y = code_of(v[e], iv, h >> 16, kLoV);
      y = v[e] == 0.f ? 0 : y < 1 ? 1 : y > 255 ? 255 : y;
      reinterpret_cast<uint8_t*>(M)[i0 + e] = (uint8_t)x;
      reinterpret_cast<uint8_t*>(V)[i0 + e] = (uint8_t)y;
    }
    if (lane == 0) {
      MS[unit] = sm;
      VS[unit] = sv;
    }
  }
}

__global__ void __launch_bounds__(256) k_adam_unpack(int64_t n, const uint8_t* codes,
                                                     const float* scales, int sgn, float* out) {
  const int64_t stride = (int64_t)gridDim.x * blockDim.x;
  for (int64_t i = (int64_t)blockIdx.x * blockDim.x + threadIdx.x; i < n; i += stride) {
    const uint32_t x = codes[i], c = sgn ? x & 127 : x;
    const float mag = level(c, sgn ? kLoM : kLoV) * scales[i / kUnit];
    out[i] = sgn && (x & 128) ? -mag : mag;
  }
}

}  // namespace

uint32_t adam_blocks(int64_t n) { return (uint32_t)((n + kBlockElems - 1) / kBlockElems); }

hipError_t launch_adamw(const AdamBatch& b, hipStream_t st) {
  if (b.n < 1 || b.n > kAdamMax || b.first[b.n] < 1) return hipErrorInvalidValue;
  hipLaunchKernelGGL(k_adamw, dim3(b.first[b.n]), dim3(256), 0, st, b);
  return hipGetLastError();
}

hipError_t launch_adam_unpack(int64_t n, const uint8_t* codes, const float* scales, bool sgn,
                              float* out, hipStream_t st) {
  const int64_t need = (n + 255) / 256;
  hipLaunchKernelGGL(k_adam_unpack, dim3((unsigned)(need < 8192 ? need : 8192)), dim3(256), 0, st,
                     n, codes, scales, sgn ? 1 : 0, out);
  return hipGetLastError();
}

}  // namespace pa
