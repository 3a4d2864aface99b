// The joint between two blocks (gfx950):
//   u = post(y),  x1 = alpha x + scale m u,  h = pre(x1)
// with post and pre a LayerNorm, an RMSNorm or nothing and m a gate t,
// sigmoid(t) or 1; and its backward.
//
// With yhat, xhat the rows normalised by post and pre and ry, rx their 1 / size,
//   e  = dx1 + rx (gh - mean_c(gh) - xhat mean_c(gh xhat)),   gh = dh pre_g
//   dx = alpha e,   du = scale m e,   dt = scale e u m',   gu = du post_g
//   dy = ry (gu - mean_c(gu) - yhat mean_c(gu yhat))
// (RMSNorm: without the plain means), and sums over the rows of du yhat, du,
// e m u, dh xhat and dh for post_g, post_b, scale, pre_g and pre_b.
//
// A lane holds 16 bytes of a row (8 bf16 or 4 fp32 channels).  Rows of up to
// 64 such chunks are shared by the smallest power of two of lanes that holds
// them, several rows per wave, the sums over a row by lane exchanges; wider rows
// take a block of one wave per 64 chunks and sums through LDS.  Lanes behind a
// row's end read its first chunk and count as zeros.
#include <type_traits>

#include "pa_device.hpp"
#include "pa_ops_internal.h"

namespace pa {
namespace {

template <typename T> struct Chunk16 { static constexpr int E = 16 / (int)sizeof(T); };

template <typename T>
__device__ __forceinline__ void load_chunk(const void* base, int64_t at,
                                           float (&v)[Chunk16<T>::E]) {
  const T* p = reinterpret_cast<const T*>(base) + at;
  if constexpr (sizeof(T) == 2) {
    const bf16x8 b = *reinterpret_cast<const bf16x8*>(p);
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = (float)b[e];
  } else {
    const f32x4 f = *reinterpret_cast<const f32x4*>(p);
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] = f[e];
  }
}
template <typename T>
__device__ __forceinline__ void store_chunk(void* base, int64_t at,
                                            const float (&v)[Chunk16<T>::E]) {
  T* p = reinterpret_cast<T*>(base) + at;
  if constexpr (sizeof(T) == 2) {
    bf16x8 b;
#pragma unroll
    for (int e = 0; e < 8; ++e) b[e] = (bf16)v[e];
    *reinterpret_cast<bf16x8*>(p) = b;
  } else {
    f32x4 f;
#pragma unroll
    for (int e = 0; e < 4; ++e) f[e] = v[e];
    *reinterpret_cast<f32x4*>(p) = f;
  }
}

// The lanes that share a row: L lanes of a wave (narrow), or the block.
template <bool WIDE>
struct RowGroup {
  int L;
  float* red;  // [waves] (wide)
  __device__ __forceinline__ float sum(float v) const {
    if constexpr (!WIDE) {
      for (int o = 1; o < L; o <<= 1) v += __shfl_xor(v, o);
      return v;
    } else {
      for (int o = 1; o < 64; o <<= 1) v += __shfl_xor(v, o);
      __syncthreads();  // the sums before have been read
      if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
      __syncthreads();
      float s = 0.f;
      for (int w = 0; w < (int)(blockDim.x >> 6); ++w) s += red[w];
      return s;
    }
  }
  __device__ __forceinline__ uint32_t max(uint32_t v) const {
    if constexpr (!WIDE) {
      for (int o = 1; o < L; o <<= 1) v = ::max(v, (uint32_t)__shfl_xor((int)v, o));
      return v;
    } else {
      for (int o = 1; o < 64; o <<= 1) v = ::max(v, (uint32_t)__shfl_xor((int)v, o));
      uint32_t* r = reinterpret_cast<uint32_t*>(red);
      __syncthreads();
      if ((threadIdx.x & 63) == 0) r[threadIdx.x >> 6] = v;
      __syncthreads();
      uint32_t s = 0;
      for (int w = 0; w < (int)(blockDim.x >> 6); ++w) s = ::max(s, r[w]);
      return s;
    }
  }
};

// v <- the row normalised (lanes off the row: zeros); returns 1 / its size.
template <int E, bool WIDE>
__device__ __forceinline__ float normalise(float (&v)[E], bool on, int kind, float eps, float invC,
                                           const RowGroup<WIDE>& grp) {
  if (kind == PA_NORM_LAYER) {
    float s = 0.f;
#pragma unroll
    for (int e = 0; e < E; ++e) s += v[e];
    const float mean = grp.sum(on ? s : 0.f) * invC;
#pragma unroll
    for (int e = 0; e < E; ++e) v[e] = v[e] - mean;
  }
  float q = 0.f;
#pragma unroll
  for (int e = 0; e < E; ++e) q += v[e] * v[e];
  const float r = 1.0f / sqrtf(grp.sum(on ? q : 0.f) * invC + eps);
#pragma unroll
  for (int e = 0; e < E; ++e) v[e] = on ? v[e] * r : 0.f;
  return r;
}

// z's gradient from that of its normalised form: d <- r (d - [mean d] - zhat
// mean(d zhat)).
template <int E, bool WIDE>
__device__ __forceinline__ void pull_back(float (&d)[E], const float (&zh)[E], float r, bool on,
                                          int kind, float invC, const RowGroup<WIDE>& grp) {
  float sd = 0.f, sz = 0.f;
#pragma unroll
  for (int e = 0; e < E; ++e) {
    sd += d[e];
    sz += d[e] * zh[e];
  }
  const float md = kind == PA_NORM_LAYER ? grp.sum(on ? sd : 0.f) * invC : 0.f;
  const float mz = grp.sum(on ? sz : 0.f) * invC;
#pragma unroll
  for (int e = 0; e < E; ++e) d[e] = r * (d[e] - md - zh[e] * mz);
}

// The gate and its slope; exp of -|t| alone, so that nothing overflows.
__device__ __forceinline__ float gate_of(float t, int kind, float& slope) {
  if (kind == PA_GATE_LINEAR) {
    slope = 1.f;
    return t;
  }
  const float q = expf(-fabsf(t)), s = 1.f / (1.f + q);
  slope = q * s * s;
  return t >= 0.f ? s : q * s;
}

// A row's channels [c0, c0 + E) of an fp32 vector, or `none`.
template <int E>
__device__ __forceinline__ void gains(const float* p, int c0, float none, float (&v)[E]) {
#pragma unroll
  for (int e = 0; e < E; ++e) v[e] = p ? p[c0 + e] : none;
}

template <typename T, bool WIDE>
__global__ void __launch_bounds__(WIDE ? 1024 : 256) k_resnorm(ResNormArgs a) {
  constexpr int E = Chunk16<T>::E;
  __shared__ float red[16];
  const int L = WIDE ? blockDim.x : a.L;
  const RowGroup<WIDE> grp{L, red};
  const int rows = WIDE ? 1 : blockDim.x / L;  // rows per block and turn
  const int c = (threadIdx.x % L) * E;
  const bool on = c < a.C;
  const int c0 = on ? c : 0;
  const float invC = 1.f / (float)a.C;
  float pg[E], pb[E], sc[E], qg[E], qb[E];
  gains(a.post_g, c0, 1.f, pg);
  gains(a.post_b, c0, 0.f, pb);
  gains(a.scale, c0, 1.f, sc);
  gains(a.pre_g, c0, 1.f, qg);
  gains(a.pre_b, c0, 0.f, qb);
  const int64_t step = (int64_t)gridDim.x * rows;
  for (int64_t base = (int64_t)blockIdx.x * rows; base < a.N; base += step) {
    const int64_t row = base + (WIDE ? 0 : threadIdx.x / L);
    const bool ok = row < a.N;
    const int64_t at = (ok ? row : a.N - 1) * a.C + c0;
    float u[E], v[E];
    load_chunk<T>(a.y, at, u);
    load_chunk<T>(a.x, at, v);
    if (a.post != PA_NORM_NONE) {
      normalise(u, on, a.post, a.post_eps, invC, grp);
#pragma unroll
      for (int e = 0; e < E; ++e) u[e] = u[e] * pg[e] + pb[e];
    }
    if (a.t) {
      float t[E], slope;
      load_chunk<T>(a.t, at, t);
#pragma unroll
      for (int e = 0; e < E; ++e) u[e] *= gate_of(t[e], a.gate, slope);
    }
#pragma unroll
    for (int e = 0; e < E; ++e) v[e] = to_f<T>(from_f<T>(fmaf(a.alpha, v[e], sc[e] * u[e])));
    if (ok && on) store_chunk<T>(a.x1, at, v);
    if (a.pre == PA_NORM_NONE) continue;
    normalise(v, on, a.pre, a.pre_eps, invC, grp);
#pragma unroll
    for (int e = 0; e < E; ++e) v[e] = v[e] * qg[e] + qb[e];
    if (a.h && ok && on) store_chunk<T>(a.h, at, v);
    if (a.hq) {
      uint32_t big = 0;
#pragma unroll
      for (int e = 0; e < E; ++e) big = ::max(big, __builtin_bit_cast(uint32_t, fabsf(v[e])));
      const QuantScale q = quant_scale(grp.max(on ? big : 0u));
      uint32_t w[E / 4];
#pragma unroll
      for (int e = 0; e < E; e += 4)
        w[e / 4] = on ? quant4(v[e], v[e + 1], v[e + 2], v[e + 3], q.inv) : 0u;
      const int Kp = (a.C + 15) / 16 * 16;
      if (ok && c < Kp) {
        uint32_t* o = reinterpret_cast<uint32_t*>(a.hq + row * Kp + c);
#pragma unroll
        for (int e = 0; e < E / 4; ++e) o[e] = w[e];
        if (c == 0) a.hs[row] = q.s;
      }
    }
  }
}

template <typename T, bool WIDE>
__global__ void __launch_bounds__(WIDE ? 1024 : 256) k_resnorm_bwd(ResNormArgs a) {
  constexpr int E = Chunk16<T>::E;
  __shared__ float red[16];
  extern __shared__ float fold[];  // [rows][C] (narrow)
  const int L = WIDE ? blockDim.x : a.L;
  const RowGroup<WIDE> grp{L, red};
  const int rows = WIDE ? 1 : blockDim.x / L;
  const int c = (threadIdx.x % L) * E;
  const bool on = c < a.C;
  const int c0 = on ? c : 0;
  const float invC = 1.f / (float)a.C;
  float pg[E], pb[E], sc[E], qg[E];
  gains(a.post_g, c0, 1.f, pg);
  gains(a.post_b, c0, 0.f, pb);
  gains(a.scale, c0, 1.f, sc);
  gains(a.pre_g, c0, 1.f, qg);
  float acc[5][E];
#pragma unroll
  for (int k = 0; k < 5; ++k)
#pragma unroll
    for (int e = 0; e < E; ++e) acc[k][e] = 0.f;
  const int64_t step = (int64_t)gridDim.x * rows;
  for (int64_t base = (int64_t)blockIdx.x * rows; base < a.N; base += step) {
    const int64_t row = base + (WIDE ? 0 : threadIdx.x / L);
    const bool ok = row < a.N;
    const int64_t at = (ok ? row : a.N - 1) * a.C + c0;
    float d[E];
    if (a.dx1) {
      load_chunk<T>(a.dx1, at, d);
    } else {
#pragma unroll
      for (int e = 0; e < E; ++e) d[e] = 0.f;
    }
    if (a.dh) {
      float xh[E], gh[E];
      load_chunk<T>(a.x1, at, xh);
      load_chunk<T>(a.dh, at, gh);
      const float rx = normalise(xh, on, a.pre, a.pre_eps, invC, grp);
#pragma unroll
      for (int e = 0; e < E; ++e) {
        if (ok) {
          acc[3][e] += gh[e] * xh[e];
          acc[4][e] += gh[e];
        }
        gh[e] *= qg[e];
      }
      pull_back(gh, xh, rx, on, a.pre, invC, grp);
#pragma unroll
      for (int e = 0; e < E; ++e) d[e] += gh[e];
    }
    // d: e of the header.  u: post(y); yh its normalised row
    float yh[E], u[E], o[E];
    load_chunk<T>(a.y, at, yh);
    float ry = 1.f;
    if (a.post != PA_NORM_NONE) ry = normalise(yh, on, a.post, a.post_eps, invC, grp);
#pragma unroll
    for (int e = 0; e < E; ++e) {
      u[e] = a.post != PA_NORM_NONE ? yh[e] * pg[e] + pb[e] : yh[e];
      o[e] = a.alpha * d[e];
    }
    if (ok && on) store_chunk<T>(a.dx, at, o);
    float m[E];
#pragma unroll
    for (int e = 0; e < E; ++e) m[e] = 1.f;
    if (a.t) {
      float t[E];
      load_chunk<T>(a.t, at, t);
#pragma unroll
      for (int e = 0; e < E; ++e) {
        float slope;
        m[e] = gate_of(t[e], a.gate, slope);
        t[e] = sc[e] * d[e] * u[e] * slope;
      }
      if (ok && on) store_chunk<T>(a.dt, at, t);
    }
#pragma unroll
    for (int e = 0; e < E; ++e) {
      const float du = d[e] * sc[e] * m[e];
      if (ok) {
        acc[2][e] += d[e] * m[e] * u[e];
        acc[0][e] += du * yh[e];
        acc[1][e] += du;
      }
      u[e] = du * pg[e];
    }
    if (a.post != PA_NORM_NONE) {
      pull_back(u, yh, ry, on, a.post, invC, grp);
      if (ok && on) store_chunk<T>(a.dy, at, u);
    } else if (ok && on) {
#pragma unroll
      for (int e = 0; e < E; ++e) o[e] = d[e] * sc[e] * m[e];
      store_chunk<T>(a.dy, at, o);
    }
  }
  if (!a.partials) return;
  // the block's record [5][C]: its rows added in order
  float* rec = a.partials + (int64_t)blockIdx.x * 5 * a.C;
#pragma unroll
  for (int k = 0; k < 5; ++k) {
    if constexpr (WIDE) {
      if (on)
#pragma unroll
        for (int e = 0; e < E; ++e) rec[k * a.C + c + e] = acc[k][e];
    } else {
      __syncthreads();
      if (on)
#pragma unroll
        for (int e = 0; e < E; ++e) fold[(threadIdx.x / L) * a.C + c + e] = acc[k][e];
      __syncthreads();
      for (int i = threadIdx.x; i < a.C; i += blockDim.x) {
        float s = 0.f;
        for (int r = 0; r < rows; ++r) s += fold[r * a.C + i];
        rec[k * a.C + i] = s;
      }
    }
  }
}

struct ResNormGeo {
  bool wide;
  int threads, L, rows;  // rows per block and turn
};
ResNormGeo geo(int C, int dtype) {
  const int E = dtype == 1 ? 8 : 4, chunks = (C + E - 1) / E;
  ResNormGeo g;
  g.wide = chunks > 64;
  g.L = 1;
  while (g.L < chunks && !g.wide) g.L <<= 1;
  g.threads = g.wide ? (chunks + 63) / 64 * 64 : 256;
  if (g.wide) g.L = g.threads;
  g.rows = g.threads / g.L;
  return g;
}

}  // namespace

int resnorm_blocks(int64_t N, int C, int dtype, bool bwd) {
  const ResNormGeo g = geo(C, dtype);
  const int64_t need = (N + g.rows - 1) / g.rows;
  const int64_t cap = g.wide ? 512 : bwd ? 1024 : 2048;
  return (int)(need < cap ? need : cap);
}

hipError_t launch_resnorm(const ResNormArgs& a0, int dtype, bool bwd, hipStream_t st) {
  ResNormArgs a = a0;
  const int most = dtype == 1 ? 8192 : 4096;
  if (a.N < 1 || a.C < 16 || a.C % 8 || a.C > most) return hipErrorInvalidValue;
  const ResNormGeo g = geo(a.C, dtype);
  a.L = g.L;
  const dim3 grid(resnorm_blocks(a.N, a.C, dtype, bwd)), block(g.threads);
  const size_t lds = bwd && !g.wide ? (size_t)g.rows * a.C * sizeof(float) : 0;
  auto go = [&](auto* k) { hipLaunchKernelGGL(k, grid, block, lds, st, a); };
  if (dtype == 1) {
    if (g.wide) bwd ? go(k_resnorm_bwd<bf16, true>) : go(k_resnorm<bf16, true>);
    else bwd ? go(k_resnorm_bwd<bf16, false>) : go(k_resnorm<bf16, false>);
  } else {
    if (g.wide) bwd ? go(k_resnorm_bwd<float, true>) : go(k_resnorm<float, true>);
    else bwd ? go(k_resnorm_bwd<float, false>) : go(k_resnorm<float, false>);
  }
  return hipGetLastError();
}

}  // namespace pa
