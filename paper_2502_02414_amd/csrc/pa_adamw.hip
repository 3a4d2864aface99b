// One AdamW step over many tensors (gfx950), moments in fp32 or in 8 bits; the
// formulas and the 8-bit code are in include/pa_ops.h.
//
// A launch takes the tensors of a table in device memory, or up to kAdamMax of
// them that are described in its arguments.  A block
// works on 16 units of 256 consecutive elements of one tensor, a wave on four of
// them, four elements per lane: a unit is a block of the 8-bit moments, whose
// largest magnitude is a reduction within the wave.
//
// Bound by memory: per element 28 bytes with fp32 gradients and moments, 16 with
// 8-bit moments, 2 more for a bf16 copy.  110 million parameters in 168 tensors
// with bf16 gradients and copies 576 us (3.07 GB, 5.3 TB/s; a copy reaches 4.85);
// 7 million in 168 with 8-bit moments and copies 25 us (5.0 TB/s) through a table, 50
// with the tensors in the arguments of four launches (where gradients are new tensors
// every step).  A first form with one element at a time took 1008 us.  The 8-bit code takes about 60 vector instructions an
// element: the rounding is an integer addition and a shift, since a code is the top
// of a float's bits, and the scale a power of two, so that dividing by it is exact
// and cheap.
#include <cmath>
#include <type_traits>

#include "pa_device.hpp"
#include "pa_ops_internal.h"

namespace pa {

// The hash of the random bits (host and device).
__host__ __device__ static inline uint32_t scramble(uint32_t h) {
  h = (h ^ (h >> 16)) * 0x85EBCA6Bu;
  h = (h ^ (h >> 13)) * 0xC2B2AE35u;
  return h ^ (h >> 16);
}
__host__ __device__ static inline uint32_t mix32(uint32_t a, uint32_t b) {
  return scramble(a ^ (b * 0x9E3779B9u));
}
uint32_t adam_mix(uint32_t a, uint32_t b) { return mix32(a, b); }

// lr / (1 - b1^step) and 1 / sqrt(1 - b2^step): the same operations of 64 bits on
// the host and on the device, so that both give the same step.
__host__ __device__ static inline double whole_power(double b, int64_t n) {
#pragma clang fp contract(off)
  double r = 1.0;
  for (; n > 0; n >>= 1, b = b * b)
    if (n & 1) r = r * b;
  return r;
}
__host__ __device__ static inline void adam_step_consts(double lr, double b1, double b2,
                                                        int64_t step, float& ss, float& rs) {
#pragma clang fp contract(off)
  ss = (float)(lr / (1.0 - whole_power(b1, step)));
  rs = (float)(1.0 / sqrt(1.0 - whole_power(b2, step)));
}
void adam_consts(double lr, double b1, double b2, int64_t step, float* ss, float* rs) {
  adam_step_consts(lr, b1, b2, step, *ss, *rs);
}

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
// 1 / S of a power of two from 2^-126 to 2^127 (its exponent mirrored; 2^-127 is
// subnormal); a NaN stays one.
__device__ __forceinline__ float fast_rcp_pow2(float S) {
  const uint32_t b = __builtin_bit_cast(uint32_t, S);
  return S != S ? S : __builtin_bit_cast(float, b == 0x7F000000u ? 0x00400000u : 0x7F000000u - b);
}
__device__ __forceinline__ int code_of(float mag, float inv, uint32_t h, uint32_t lo) {
  return (int)((__builtin_bit_cast(uint32_t, mag * inv) + 16 * h + 8) >> 20) - (int)lo;
}

struct Consts {
  float b1, b2, c1, c2, gs, ss, rs, eps, lrwd;
};

// p, m, v of one element after the step (the moments without fused
// multiply-adds, as documented).  The root and the reciprocal are the
// hardware's, good to one step of fp32 each; it takes a subnormal v for zero, so
// such ones are scaled.
__device__ __forceinline__ void update(const Consts& k, float g, float& p, float& m, float& v) {
  {
#pragma clang fp contract(off)
    g = g * k.gs;
    m = m * k.b1 + g * k.c1;
    v = v * k.b2 + (g * g) * k.c2;
  }
  const bool tiny = v < 0x1p-96f;
  const float root = __builtin_amdgcn_sqrtf(tiny ? v * 0x1p64f : v) * (tiny ? 0x1p-32f : 1.f);
  const float den = fmaf(root, k.rs, k.eps);
  p -= fmaf(k.lrwd, p, k.ss * (m * fast_rcp(den)));
}

// The tensors of an item.
struct Item {
  float* p;
  bf16* copy;
  const void* g;
  void *m, *v;
  float *ms, *vs;
  int64_t n;
};

// Four elements of one unit, this lane's.
struct Four {
  float p[4], g[4], m[4], v[4];
};

template <typename V> __device__ __forceinline__ V get(const void* base, int64_t i) {
  return reinterpret_cast<const V*>(base)[i];
}

// WHOLE: units that lie inside of the tensor, with 16-byte accesses; otherwise
// element by element up to its end.
template <bool Q8, bool GB, bool WHOLE>
__device__ __forceinline__ void load_unit(const Item& t, int64_t i0, int live, Four& x, uint32_t& mc,
                                          uint32_t& vc) {
  if constexpr (WHOLE) {
    const f32x4 p = get<f32x4>(t.p, i0 / 4);
    f32x4 m, v;
    if constexpr (Q8) {
      mc = get<uint32_t>(t.m, i0 / 4);
      vc = get<uint32_t>(t.v, i0 / 4);
    } else {
      m = get<f32x4>(t.m, i0 / 4);
      v = get<f32x4>(t.v, i0 / 4);
    }
    if constexpr (GB) {
      const bf16x4 g = get<bf16x4>(t.g, i0 / 4);
#pragma unroll
      for (int e = 0; e < 4; ++e) x.g[e] = (float)g[e];
    } else {
      const f32x4 g = get<f32x4>(t.g, i0 / 4);
#pragma unroll
      for (int e = 0; e < 4; ++e) x.g[e] = g[e];
    }
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      x.p[e] = p[e];
      if constexpr (!Q8) {
        x.m[e] = m[e];
        x.v[e] = v[e];
      }
    }
  } else {
    mc = vc = 0;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int64_t i = i0 + e;
      const bool in = e < live;
      x.p[e] = in ? t.p[i] : 0.f;
      x.g[e] = !in ? 0.f : GB ? (float)get<bf16>(t.g, i) : get<float>(t.g, i);
      if constexpr (Q8) {
        if (in) {
          mc |= (uint32_t)get<uint8_t>(t.m, i) << 8 * e;
          vc |= (uint32_t)get<uint8_t>(t.v, i) << 8 * e;
        }
      } else {
        x.m[e] = in ? get<float>(t.m, i) : 0.f;
        x.v[e] = in ? get<float>(t.v, i) : 0.f;
      }
    }
  }
}

__device__ __forceinline__ uint32_t wave_max(uint32_t v) {
  const auto step = [&](auto ctrl) {
    v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, decltype(ctrl)::value, 0xF, 0xF, false));
  };
  step(std::integral_constant<int, kQuadSwap1>{});
  step(std::integral_constant<int, kQuadSwap2>{});
  step(std::integral_constant<int, kHalfMirror>{});
  step(std::integral_constant<int, kMirror>{});
  // (the four rows of 16 lanes)
  return max(max(__builtin_amdgcn_readlane(v, 0), __builtin_amdgcn_readlane(v, 16)),
             max(__builtin_amdgcn_readlane(v, 32), __builtin_amdgcn_readlane(v, 48)));
}

// Codes of a unit's new moments (lanes behind the end: zeros).
__device__ __forceinline__ void encode(const Four& x, uint32_t kb, int lane, float& sm, float& sv,
                                       uint32_t& mc, uint32_t& vc) {
  uint32_t bm = 0, bv = 0;
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    bm = max(bm, __builtin_bit_cast(uint32_t, x.m[e]) & 0x7fffffffu);
    bv = max(bv, __builtin_bit_cast(uint32_t, x.v[e]));
  }
  sm = block_scale(wave_max(bm));
  sv = block_scale(wave_max(bv));
  // (powers of two: exact; a NaN stays one)
  const float im = sm == 0.f ? 0.f : fast_rcp_pow2(sm), iv = sv == 0.f ? 0.f : fast_rcp_pow2(sv);
  mc = vc = 0;
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const uint32_t h = scramble(kb + (uint32_t)(4 * lane + e));
    int c = code_of(fabsf(x.m[e]), im, h & 0xffffu, kLoM);
    c = min(max(c, 0), 127);
    c |= c && x.m[e] < 0.f ? 128 : 0;
    int d = code_of(x.v[e], iv, h >> 16, kLoV);
    d = x.v[e] == 0.f ? 0 : min(max(d, 1), 255);
    mc |= (uint32_t)c << 8 * e;
    vc |= (uint32_t)d << 8 * e;
  }
}

template <bool Q8, bool GB, bool WHOLE, int U>
__device__ __forceinline__ void units(const Item& t, int64_t unit0, const Consts& k, uint32_t key) {
  const int lane = lane_id();
  Four x[U];
  uint32_t mc[U], vc[U];
  float sm[U], sv[U];
  int live[U];
#pragma unroll
  for (int w = 0; w < U; ++w) {
    const int64_t i0 = (unit0 + w) * kUnit + 4 * lane, left = t.n - i0;
    live[w] = WHOLE ? 4 : left >= 4 ? 4 : left > 0 ? (int)left : 0;
    load_unit<Q8, GB, WHOLE>(t, i0, live[w], x[w], mc[w], vc[w]);
    if constexpr (Q8) {
      sm[w] = t.ms[unit0 + w];
      sv[w] = t.vs[unit0 + w];
    }
  }
#pragma unroll
  for (int w = 0; w < U; ++w) {
    const int64_t unit = unit0 + w, i0 = unit * kUnit + 4 * lane;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      if constexpr (Q8) {
        const uint32_t c = mc[w] >> 8 * e & 0xffu;
        const float mag = level(c & 127u, kLoM) * sm[w];
        x[w].m[e] = c & 128u ? -mag : mag;
        x[w].v[e] = level(vc[w] >> 8 * e & 0xffu, kLoV) * sv[w];
      }
      update(k, x[w].g[e], x[w].p[e], x[w].m[e], x[w].v[e]);
      if (!WHOLE && e >= live[w]) x[w].m[e] = x[w].v[e] = 0.f;
    }
    if constexpr (Q8) encode(x[w], mix32(key, (uint32_t)unit), lane, sm[w], sv[w], mc[w], vc[w]);
    if constexpr (WHOLE) {
      reinterpret_cast<f32x4*>(t.p)[i0 / 4] = f32x4{x[w].p[0], x[w].p[1], x[w].p[2], x[w].p[3]};
      if (t.copy)
        reinterpret_cast<bf16x4*>(t.copy)[i0 / 4] =
            bf16x4{(bf16)x[w].p[0], (bf16)x[w].p[1], (bf16)x[w].p[2], (bf16)x[w].p[3]};
      if constexpr (Q8) {
        reinterpret_cast<uint32_t*>(t.m)[i0 / 4] = mc[w];
        reinterpret_cast<uint32_t*>(t.v)[i0 / 4] = vc[w];
      } else {
        reinterpret_cast<f32x4*>(t.m)[i0 / 4] = f32x4{x[w].m[0], x[w].m[1], x[w].m[2], x[w].m[3]};
        reinterpret_cast<f32x4*>(t.v)[i0 / 4] = f32x4{x[w].v[0], x[w].v[1], x[w].v[2], x[w].v[3]};
      }
    } else {
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (e < live[w]) {
          t.p[i0 + e] = x[w].p[e];
          if (t.copy) t.copy[i0 + e] = (bf16)x[w].p[e];
          if constexpr (Q8) {
            reinterpret_cast<uint8_t*>(t.m)[i0 + e] = (uint8_t)(mc[w] >> 8 * e);
            reinterpret_cast<uint8_t*>(t.v)[i0 + e] = (uint8_t)(vc[w] >> 8 * e);
          } else {
            reinterpret_cast<float*>(t.m)[i0 + e] = x[w].m[e];
            reinterpret_cast<float*>(t.v)[i0 + e] = x[w].v[e];
          }
        }
    }
    if constexpr (Q8)
      if (lane == 0) {
        t.ms[unit] = sm[w];
        t.vs[unit] = sv[w];
      }
  }
}

template <bool Q8, bool GB>
__device__ __forceinline__ void wave_units(const Item& t, int64_t unit0, const Consts& k,
                                           uint32_t key) {
  if ((unit0 + kWaveUnits) * kUnit <= t.n) {
    units<Q8, GB, true, kWaveUnits>(t, unit0, k, key);
  } else {
    for (int w = 0; w < kWaveUnits && (unit0 + w) * kUnit < t.n; ++w)
      units<Q8, GB, false, 1>(t, unit0 + w, k, key);
  }
}

// Block `b` of an item whose first block is `first`; A: where the step's constants
// are (the launch's arguments).
template <typename Step>
__device__ __forceinline__ void item_block(Step A, const Item& t, float wd, uint32_t bits,
                                           uint32_t index, uint32_t b) {
  Consts k;
  k.b1 = A->b1; k.b2 = A->b2; k.c1 = A->c1; k.c2 = A->c2;
  k.gs = A->gscale ? *A->gscale : 1.f;
  k.eps = A->eps;
  double lr = A->lr;
  uint32_t step_key = A->step_key;
  k.ss = A->ss;
  k.rs = A->rs;
  if (A->lr_dev || A->step_dev) {  // a captured graph's: as the host forms them
    if (A->lr_dev) lr = (double)*A->lr_dev;
    const int64_t step = A->step_dev ? *A->step_dev : A->step;
    adam_step_consts(lr, A->beta1, A->beta2, step, k.ss, k.rs);
    step_key = mix32(A->seed_key, (uint32_t)step);
  }
  k.lrwd = (float)(lr * (double)wd);
  const uint32_t key = mix32(step_key, index);
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int64_t unit0 = ((int64_t)b * 4 + wave) * kWaveUnits;
  if (bits & 2) {
    if (bits & 1) wave_units<true, true>(t, unit0, k, key);
    else wave_units<true, false>(t, unit0, k, key);
  } else {
    if (bits & 1) wave_units<false, true>(t, unit0, k, key);
    else wave_units<false, false>(t, unit0, k, key);
  }
}

template <typename I> __device__ __forceinline__ Item tensors(const I& i) {
  return {i.p, reinterpret_cast<bf16*>(i.copy), i.g, i.m, i.v, i.ms, i.vs, i.n};
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
  item_block(&A->s, tensors(A->it[lo]), A->it[lo].wd, A->it[lo].bits, (uint32_t)(A->base + lo),
             b - A->first[lo]);
}

__global__ void __launch_bounds__(256) k_adamw_table(AdamStep s, const AdamEntry* entries,
                                                     const uint32_t* map) {
  const AdamEntry* e = entries + map[blockIdx.x];
  item_block(&s, tensors(e->it), e->it.wd, e->it.bits, e->index, blockIdx.x - e->first);
}

// Four codes per thread (the last ones one by one).
__global__ void __launch_bounds__(256) k_adam_unpack(int64_t n, const uint8_t* codes,
                                                     const float* scales, int sgn, float* out) {
  const int64_t stride = (int64_t)gridDim.x * blockDim.x;
  for (int64_t q = (int64_t)blockIdx.x * blockDim.x + threadIdx.x; 4 * q < n; q += stride) {
    const bool whole = 4 * q + 4 <= n;
    uint32_t w = 0;
    if (whole) {
      w = reinterpret_cast<const uint32_t*>(codes)[q];
    } else {
      for (int e = 0; 4 * q + e < n; ++e) w |= (uint32_t)codes[4 * q + e] << 8 * e;
    }
    const float s = scales[q / (kUnit / 4)];
    f32x4 o;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const uint32_t x = w >> 8 * e & 0xffu, c = sgn ? x & 127u : x;
      const float mag = level(c, sgn ? kLoM : kLoV) * s;
      o[e] = sgn && (x & 128u) ? -mag : mag;
    }
    if (whole) {
      reinterpret_cast<f32x4*>(out)[q] = o;
    } else {
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (4 * q + e < n) out[4 * q + e] = o[e];
    }
  }
}

}  // namespace

uint32_t adam_blocks(int64_t n) { return (uint32_t)((n + kBlockElems - 1) / kBlockElems); }

hipError_t launch_adamw(const AdamBatch& b, hipStream_t st) {
  if (b.n < 1 || b.n > kAdamMax || b.first[b.n] < 1) return hipErrorInvalidValue;
  hipLaunchKernelGGL(k_adamw, dim3(b.first[b.n]), dim3(256), 0, st, b);
  return hipGetLastError();
}

hipError_t launch_adamw_table(const AdamStep& s, const AdamEntry* entries, const uint32_t* map,
                              uint32_t blocks, hipStream_t st) {
  hipLaunchKernelGGL(k_adamw_table, dim3(blocks), dim3(256), 0, st, s, entries, map);
  return hipGetLastError();
}

hipError_t launch_adam_unpack(int64_t n, const uint8_t* codes, const float* scales, bool sgn,
                              float* out, hipStream_t st) {
  const int64_t need = (n + 1023) / 1024;
  hipLaunchKernelGGL(k_adam_unpack, dim3((unsigned)(need < 8192 ? need : 8192)), dim3(256), 0, st,
                     n, codes, scales, sgn ? 1 : 0, out);
  return hipGetLastError();
}

}  // namespace pa
