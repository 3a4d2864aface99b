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
//
// Bound by memory (4 to 8 rows of C elements read or written per row, some 20 and
// 45 operations an element).  A million rows of 256 in bf16: forward 373 us (5.5
// TB/s), to int8 rows 358 (5.0), backward with a gate 782 to 794 us (5.2 TB/s); in fp32
// 801, 683 and, without a gate, 1173 us (4.9 to 5.2 TB/s); a copy reaches 4.85.  A first form
// with one row at a time, its tensors loaded where they were needed, and sums by
// ds_bpermute took 415 and 1371 us.  Sums share their exchanges two at a time:
// four rounds for a backward row.  Rows that do not fill their lanes or cache
// lines are slower: 500,000 of 264 332 and 581 us with a gate (4.0 and 3.6 TB/s),
// 26,648 of 2,920 210 and 375 us (3.7 and 3.3 TB/s).
#include <algorithm>
#include <type_traits>

#include "pa_ops_internal.h"
#include "pa_stream.hpp"

namespace pa {
namespace {

template <typename T> struct Chunk16 {
  static constexpr int E = 16 / (int)sizeof(T);
  uint4 q;
};
template <typename T>
__device__ __forceinline__ Chunk16<T> fetch(const void* base, int64_t at) {
  return {ld_global16<true>(reinterpret_cast<const T*>(base) + at)};
}
template <typename T>
__device__ __forceinline__ void unpack(const Chunk16<T>& c, float (&v)[Chunk16<T>::E]) {
  if constexpr (sizeof(T) == 2) {
    const bf16x8 b = __builtin_bit_cast(bf16x8, c.q);
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = (float)b[e];
  } else {
    const f32x4 f = __builtin_bit_cast(f32x4, c.q);
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] = f[e];
  }
}
template <typename T>
__device__ __forceinline__ void store_chunk(void* base, int64_t at,
                                            const float (&v)[Chunk16<T>::E]) {
  uint4 q;
  if constexpr (sizeof(T) == 2) {
    bf16x8 b;
#pragma unroll
    for (int e = 0; e < 8; ++e) b[e] = (bf16)v[e];
    q = __builtin_bit_cast(uint4, b);
  } else {
    f32x4 f;
#pragma unroll
    for (int e = 0; e < 4; ++e) f[e] = v[e];
    q = __builtin_bit_cast(uint4, f);
  }
  st_global16(reinterpret_cast<T*>(base) + at, q);
}

// Sums and maxima over the lanes that share a row: L lanes of a wave (narrow), by
// lane exchanges without LDS, or the block's waves (wide), which meet in LDS, in
// two places in turn, so that a sum takes one barrier.
template <int WIDE>
struct RowGroup {
  int L;
  float2* red;  // [2][16] (wide)
  int turn = 0;

  __device__ __forceinline__ float lanes_sum(float v) const {
    if (WIDE || L > 1) v += dpp<kQuadSwap1>(v);
    if (WIDE || L > 2) v += dpp<kQuadSwap2>(v);
    if (WIDE || L > 4) v += dpp<kHalfMirror>(v);
    if (WIDE || L > 8) v += dpp<kMirror>(v);
    if (WIDE || L > 16) {
      float a = v, b = v;
      lane_swap16(a, b);
      v = a + b;
    }
    if (WIDE || L > 32) {
      float a = v, b = v;
      lane_swap32(a, b);
      v = a + b;
    }
    return v;
  }
  // a and b summed, together
  __device__ __forceinline__ void sum2(float& a, float& b) {
    a = lanes_sum(a);
    b = lanes_sum(b);
    if constexpr (WIDE) {
      float2* r = red + 16 * turn;
      turn ^= 1;
      if ((threadIdx.x & 63) == 0) r[threadIdx.x >> 6] = {a, b};
      block_sync();
      a = b = 0.f;
      for (int w = 0; w < (int)(blockDim.x >> 6); ++w) {
        a += r[w].x;
        b += r[w].y;
      }
    }
  }
  __device__ __forceinline__ uint32_t max(uint32_t v) {
    for (int o = 1; o < (WIDE ? 64 : L); o <<= 1) v = ::max(v, (uint32_t)__shfl_xor((int)v, o));
    if constexpr (WIDE) {
      float2* r = red + 16 * turn;
      turn ^= 1;
      if ((threadIdx.x & 63) == 0) r[threadIdx.x >> 6].x = __builtin_bit_cast(float, v);
      block_sync();
      v = 0;
      for (int w = 0; w < (int)(blockDim.x >> 6); ++w)
        v = ::max(v, __builtin_bit_cast(uint32_t, r[w].x));
    }
    return v;
  }
};

template <int E> __device__ __forceinline__ float total(const float (&v)[E]) {
  float s = 0.f;
#pragma unroll
  for (int e = 0; e < E; ++e) s += v[e];
  return s;
}
template <int E>
__device__ __forceinline__ float dot(const float (&v)[E], const float (&w)[E]) {
  float s = 0.f;
#pragma unroll
  for (int e = 0; e < E; ++e) s = fmaf(v[e], w[e], s);
  return s;
}

// Two rows normalised together (their sums share the exchanges): a <- its
// deviation from the mean (LayerNorm) over its size, on the lanes of the row,
// zeros on the others; ra = 1 / size.  NONE leaves a row as it is, r = 1.
template <int E, int WIDE>
__device__ __forceinline__ void normalise2(float (&a)[E], int ka, float ea, float& ra, float (&b)[E],
                                           int kb, float eb, float& rb, bool on, float invC,
                                           RowGroup<WIDE>& grp) {
  if (ka == PA_NORM_LAYER || kb == PA_NORM_LAYER) {
    float sa = on ? total(a) : 0.f, sb = on ? total(b) : 0.f;
    grp.sum2(sa, sb);
    const float ma = ka == PA_NORM_LAYER ? sa * invC : 0.f, mb = kb == PA_NORM_LAYER ? sb * invC : 0.f;
#pragma unroll
    for (int e = 0; e < E; ++e) {
      a[e] -= ma;
      b[e] -= mb;
    }
  }
  ra = rb = 1.f;
  if (ka != PA_NORM_NONE || kb != PA_NORM_NONE) {
    float qa = on ? dot(a, a) : 0.f, qb = on ? dot(b, b) : 0.f;
    grp.sum2(qa, qb);
    if (ka != PA_NORM_NONE) ra = 1.0f / sqrtf(fmaf(qa, invC, ea));
    if (kb != PA_NORM_NONE) rb = 1.0f / sqrtf(fmaf(qb, invC, eb));
  }
  const float fa = on ? ra : 0.f, fb = on ? rb : 0.f;
#pragma unroll
  for (int e = 0; e < E; ++e) {
    a[e] *= fa;
    b[e] *= fb;
  }
}

// z's gradient from that of its normalised form: d <- r (d - [mean d] - zhat
// mean(d zhat)).  (zhat and d are finite or the row's are not.)
template <int E, int WIDE>
__device__ __forceinline__ void pull_back(float (&d)[E], const float (&zh)[E], float r, bool on,
                                          int kind, float invC, RowGroup<WIDE>& grp) {
  float sd = on ? total(d) : 0.f, sz = on ? dot(d, zh) : 0.f;
  grp.sum2(sd, sz);
  const float md = kind == PA_NORM_LAYER ? sd * invC : 0.f, mz = sz * invC;
#pragma unroll
  for (int e = 0; e < E; ++e) d[e] = r * (d[e] - md - zh[e] * mz);
}

// The gate and its slope; exp of -|t| alone, so that nothing overflows.
// (bf16: the hardware's exp2 and reciprocal, good to a few steps of fp32.)
template <typename T>
__device__ __forceinline__ float gate_of(float t, int kind, float& slope) {
  if (kind == PA_GATE_LINEAR) {
    slope = 1.f;
    return t;
  }
  const float q = sizeof(T) == 2 ? fast_exp2(-kLog2e * fabsf(t)) : expf(-fabsf(t));
  const float s = sizeof(T) == 2 ? fast_rcp(1.f + q) : 1.f / (1.f + q);
  slope = q * s * s;
  return t >= 0.f ? s : q * s;
}

// A row's channels [c0, c0 + E) of an fp32 vector, or `none`.
template <int E>
__device__ __forceinline__ void gains(const float* p, int c0, float none, float (&v)[E]) {
#pragma unroll
  for (int e = 0; e < E; ++e) v[e] = p ? p[c0 + e] : none;
}

template <typename T, int WIDE, bool AHEAD, bool GATE>
__global__ void __launch_bounds__(WIDE ? WIDE : 256) k_resnorm(ResNormArgs a) {
  constexpr int E = Chunk16<T>::E, U = WIDE ? 1 : 2;  // rows in turn per group
  __shared__ float2 red[32];
  const int L = WIDE ? blockDim.x : a.L;
  RowGroup<WIDE> grp{L, red};
  const int rows = WIDE ? 1 : blockDim.x / L;  // groups per block
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
  struct Rows {
    Chunk16<T> x[U], y[U], t[U];
  };
  const int64_t step = (int64_t)gridDim.x * rows * U;
  // (rows past N: the last one)
  auto place = [&](int64_t row) { return (row < a.N ? row : a.N - 1) * a.C + c0; };
  auto load = [&](int64_t base, Rows& w) __attribute__((always_inline)) {
#pragma unroll
    for (int k = 0; k < U; ++k) {
      const int64_t at = place(base + k * rows + (WIDE ? 0 : threadIdx.x / L));
      w.y[k] = fetch<T>(a.y, at);
      w.x[k] = fetch<T>(a.x, at);
      if constexpr (GATE) w.t[k] = fetch<T>(a.t, at);
    }
  };
  auto work = [&](int64_t base, const Rows& w) __attribute__((always_inline)) {
    int64_t row[U], at[U];
#pragma unroll
    for (int k = 0; k < U; ++k) {
      row[k] = base + k * rows + (WIDE ? 0 : threadIdx.x / L);
      at[k] = place(row[k]);
    }
    float u[U][E], v[U][E], r0, r1;
#pragma unroll
    for (int k = 0; k < U; ++k) unpack<T>(w.y[k], u[k]);
    if (a.post != PA_NORM_NONE) {
      if constexpr (U == 2) {
        normalise2(u[0], a.post, a.post_eps, r0, u[1], a.post, a.post_eps, r1, on, invC, grp);
      } else {
        float none[E] = {};
        normalise2(u[0], a.post, a.post_eps, r0, none, PA_NORM_NONE, 0.f, r1, on, invC, grp);
      }
    }
#pragma unroll
    for (int k = 0; k < U; ++k) {
      float g[E];
      unpack<T>(w.x[k], v[k]);
      if constexpr (GATE) unpack<T>(w.t[k], g);
#pragma unroll
      for (int e = 0; e < E; ++e) {
        if (a.post != PA_NORM_NONE) u[k][e] = fmaf(u[k][e], pg[e], pb[e]);
        if constexpr (GATE) {
          float slope;
          u[k][e] *= gate_of<T>(g[e], a.gate, slope);
        }
        v[k][e] = to_f<T>(from_f<T>(fmaf(a.alpha, v[k][e], sc[e] * u[k][e])));
      }
      if (row[k] < a.N && on) store_chunk<T>(a.x1, at[k], v[k]);
    }
    if (a.pre == PA_NORM_NONE) return;
    if constexpr (U == 2) {
      normalise2(v[0], a.pre, a.pre_eps, r0, v[1], a.pre, a.pre_eps, r1, on, invC, grp);
    } else {
      float none[E] = {};
      normalise2(v[0], a.pre, a.pre_eps, r0, none, PA_NORM_NONE, 0.f, r1, on, invC, grp);
    }
#pragma unroll
    for (int k = 0; k < U; ++k) {
      const bool ok = row[k] < a.N;
#pragma unroll
      for (int e = 0; e < E; ++e) v[k][e] = fmaf(v[k][e], qg[e], qb[e]);
      if (a.h && ok && on) store_chunk<T>(a.h, at[k], v[k]);
      if (a.hq) {
        uint32_t big = 0;
#pragma unroll
        for (int e = 0; e < E; ++e)
          big = ::max(big, __builtin_bit_cast(uint32_t, v[k][e]) & 0x7fffffffu);
        const QuantScale q = quant_scale(grp.max(on ? big : 0u));
        const int Kp = (a.C + 15) / 16 * 16;
        if (ok && c < Kp) {
          uint32_t* o = reinterpret_cast<uint32_t*>(a.hq + row[k] * Kp + c);
#pragma unroll
          for (int e = 0; e < E; e += 4)
            o[e / 4] = on ? quant4(v[k][e], v[k][e + 1], v[k][e + 2], v[k][e + 3], q.inv) : 0u;
          if (c == 0) a.hs[row[k]] = q.s;
        }
      }
    }
  };
  int64_t base = (int64_t)blockIdx.x * rows * U;  // < N
  if constexpr (AHEAD) {  // the next rows on their way while these are worked on
    Rows r0, r1;
    load(base, r0);
    for (;;) {
      load(base + step, r1);
      work(base, r0);
      if ((base += step) >= a.N) break;
      load(base + step, r0);
      work(base, r1);
      if ((base += step) >= a.N) break;
    }
  } else {
    for (; base < a.N; base += step) {
      Rows r;
      load(base, r);
      work(base, r);
    }
  }
}

template <typename T, int WIDE, bool AHEAD, bool GATE>
__global__ void __launch_bounds__(WIDE ? WIDE : 256, WIDE ? 1 : 3) k_resnorm_bwd(ResNormArgs a) {
  constexpr int E = Chunk16<T>::E;
  __shared__ float2 red[32];
  extern __shared__ __attribute__((aligned(16))) float fold[];  // [rows][5][C] (narrow)
  // Blocks of 1024 threads on bf16 keep the parameters in LDS, [4][C], for want of
  // registers (16,384 rows of 8192 with a gate: 638 us with them in registers, and
  // 35 of those spilled, 554 so; narrower rows lose 5 to 20% by it).
  constexpr bool LP = WIDE == 1024 && sizeof(T) == 2;
  const int L = WIDE ? blockDim.x : a.L;
  RowGroup<WIDE> grp{L, red};
  const int rows = WIDE ? 1 : blockDim.x / L;
  const int c = (threadIdx.x % L) * E;
  const bool on = c < a.C;
  const int c0 = on ? c : 0;
  const float invC = 1.f / (float)a.C;
  float kept[LP ? 1 : 4][E];
  if constexpr (LP) {
    for (int i = threadIdx.x; i < a.C; i += blockDim.x) {
      fold[i] = a.post_g ? a.post_g[i] : 1.f;
      fold[a.C + i] = a.post_b ? a.post_b[i] : 0.f;
      fold[2 * a.C + i] = a.scale ? a.scale[i] : 1.f;
      fold[3 * a.C + i] = a.pre_g ? a.pre_g[i] : 1.f;
    }
    __syncthreads();
  } else {
    gains(a.post_g, c0, 1.f, kept[0]);
    gains(a.post_b, c0, 0.f, kept[1]);
    gains(a.scale, c0, 1.f, kept[2]);
    gains(a.pre_g, c0, 1.f, kept[3]);
  }
  auto param = [&](int k, float(&v)[E]) __attribute__((always_inline)) {
#pragma unroll
    for (int e = 0; e < E; ++e) v[e] = LP ? fold[k * a.C + c0 + e] : kept[LP ? 0 : k][e];
  };
  float acc[5][E];
#pragma unroll
  for (int k = 0; k < 5; ++k)
#pragma unroll
    for (int e = 0; e < E; ++e) acc[k][e] = 0.f;
  // (a gradient that is not given: y's rows, which are read anyway, as zeros)
  const void* DX1 = a.dx1 ? a.dx1 : a.y;
  const void* DH = a.dh ? a.dh : a.y;
  const int pre = a.dh ? a.pre : PA_NORM_NONE;
  struct Rows {
    Chunk16<T> y, x, dh, dx, t;
  };
  const int64_t step = (int64_t)gridDim.x * rows;
  auto place = [&](int64_t row) { return (row < a.N ? row : a.N - 1) * a.C + c0; };
  auto load = [&](int64_t base, Rows& r) __attribute__((always_inline)) {
    const int64_t at = place(base + (WIDE ? 0 : threadIdx.x / L));
    r.y = fetch<T>(a.y, at);
    r.x = fetch<T>(a.x1, at);
    r.dh = fetch<T>(DH, at);
    r.dx = fetch<T>(DX1, at);
    if constexpr (GATE) r.t = fetch<T>(a.t, at);
  };
  auto work = [&](int64_t base, const Rows& r) __attribute__((always_inline)) {
    const int64_t row = base + (WIDE ? 0 : threadIdx.x / L);
    const bool ok = row < a.N;
    const int64_t at = place(row);
    float yh[E], xh[E], gh[E], d[E], ry, rx;
    unpack<T>(r.y, yh);
    unpack<T>(r.x, xh);
    normalise2(yh, a.post, a.post_eps, ry, xh, pre, a.pre_eps, rx, on, invC, grp);
    unpack<T>(r.dx, d);
    if (!a.dx1) {
#pragma unroll
      for (int e = 0; e < E; ++e) d[e] = 0.f;
    }
    if (a.dh) {
      unpack<T>(r.dh, gh);
      float qg[E];
      param(3, qg);
#pragma unroll
      for (int e = 0; e < E; ++e) {
        if (ok) {
          acc[3][e] = fmaf(gh[e], xh[e], acc[3][e]);
          acc[4][e] += gh[e];
        }
        gh[e] *= qg[e];
      }
      pull_back(gh, xh, rx, on, pre, invC, grp);
#pragma unroll
      for (int e = 0; e < E; ++e) d[e] += gh[e];
    }
    // d: e of the header; u: post(y)
    float u[E], o[E], m[E], pg[E], pb[E], sc[E];
    param(0, pg);
    param(1, pb);
    param(2, sc);
#pragma unroll
    for (int e = 0; e < E; ++e) {
      u[e] = a.post != PA_NORM_NONE ? fmaf(yh[e], pg[e], pb[e]) : yh[e];
      o[e] = a.alpha * d[e];
      m[e] = 1.f;
    }
    if (ok && on) store_chunk<T>(a.dx, at, o);
    if constexpr (GATE) {
      float t[E];
      unpack<T>(r.t, t);
#pragma unroll
      for (int e = 0; e < E; ++e) {
        float slope;
        m[e] = gate_of<T>(t[e], a.gate, slope);
        t[e] = sc[e] * d[e] * u[e] * slope;
      }
      if (ok && on) store_chunk<T>(a.dt, at, t);
    }
#pragma unroll
    for (int e = 0; e < E; ++e) {
      const float em = d[e] * m[e], du = em * sc[e];
      if (ok) {
        acc[2][e] = fmaf(em, u[e], acc[2][e]);
        acc[0][e] = fmaf(du, yh[e], acc[0][e]);
        acc[1][e] += du;
      }
      u[e] = a.post != PA_NORM_NONE ? du * pg[e] : du;
    }
    if (a.post != PA_NORM_NONE) pull_back(u, yh, ry, on, a.post, invC, grp);
    if (ok && on) store_chunk<T>(a.dy, at, u);
  };
  int64_t base = (int64_t)blockIdx.x * rows;  // < N
  if constexpr (AHEAD) {
    Rows r0, r1;
    load(base, r0);
    for (;;) {
      load(base + step, r1);
      work(base, r0);
      if ((base += step) >= a.N) break;
      load(base + step, r0);
      work(base, r1);
      if ((base += step) >= a.N) break;
    }
  } else {
    for (; base < a.N; base += step) {
      Rows r;
      load(base, r);
      work(base, r);
    }
  }
  if (!a.partials) return;
  // the block's record [5][C]: its rows added in order; of the only block, the gradients
  float* rec = a.partials + (int64_t)blockIdx.x * 5 * a.C;
  const bool only = gridDim.x == 1;
  auto place_of = [&](int k) {
    if (!only) return rec + k * a.C;
    return k == 0 ? a.g0 : k == 1 ? a.g1 : k == 2 ? a.g2 : k == 3 ? a.g3 : a.g4;
  };
  if constexpr (WIDE) {
    if (on)
#pragma unroll
      for (int k = 0; k < 5; ++k) {
        float* to = place_of(k);
        if (to)
#pragma unroll
          for (int e = 0; e < E; ++e) to[c + e] = acc[k][e];
      }
  } else {
    const int C5 = 5 * a.C;
    if (on)
#pragma unroll
      for (int k = 0; k < 5; ++k)
#pragma unroll
        for (int e = 0; e < E; ++e) fold[(threadIdx.x / L) * C5 + k * a.C + c + e] = acc[k][e];
    __syncthreads();
    for (int i = threadIdx.x; i < C5; i += blockDim.x) {
      float s = 0.f;
      for (int r = 0; r < rows; ++r) s += fold[r * C5 + i];
      const int k = i / a.C;
      float* to = place_of(k);
      if (to) to[i - k * a.C] = s;
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
  const int turn = g.rows * (bwd || g.wide ? 1 : 2);
  const int64_t need = (N + turn - 1) / turn;
  // (backward: up to two turns in one block, which writes the parameters' gradients
  // itself; us, two turns in one block and in two with the sum of their records: 64
  // rows of 64 bf16 9.1 and 10.0, 16 of 256 9.8 and 10.5, 8 of 256 fp32 8.9 and 9.8;
  // four turns 14.5 and 10.6)
  if (bwd && need <= 2) return 1;
  // (backward: three blocks per CU, what its registers allow, in one round; 1024
  // blocks took 934 us where these take 793, at N = 1,000,000, C = 256)
  const int waves = g.threads / 64;
  const int64_t cap = g.wide ? (bwd ? std::min(1024, std::max(1, 12 / waves) * 256)
                                    : std::min(2048, std::max(1, 20 / waves) * 256))
                             : bwd ? 768 : 2048;
  return (int)(need < cap ? need : cap);
}

hipError_t launch_resnorm(const ResNormArgs& a0, int dtype, bool bwd, hipStream_t st) {
  ResNormArgs a = a0;
  const int most = dtype == 1 ? 8192 : 4096;
  if (a.N < 1 || a.C < 16 || a.C % 8 || a.C > most) return hipErrorInvalidValue;
  const ResNormGeo g = geo(a.C, dtype);
  a.L = g.L;
  const dim3 grid(resnorm_blocks(a.N, a.C, dtype, bwd)), block(g.threads);
  const size_t lds = !bwd ? 0 : !g.wide ? (size_t)g.rows * 5 * a.C * sizeof(float)
                                        : dtype == 1 && g.threads > 512 ? (size_t)4 * a.C * sizeof(float) : 0;
  auto go = [&](auto* k) { hipLaunchKernelGGL(k, grid, block, lds, st, a); };
  auto pick = [&](auto type, auto wide, auto ahead) {
    using T = decltype(type);
    constexpr int W = decltype(wide)::value;
    constexpr bool A = decltype(ahead)::value, AB = A && !(W == 1024 && sizeof(T) == 2);
    if (a.t) bwd ? go(k_resnorm_bwd<T, W, AB, true>) : go(k_resnorm<T, W, A, true>);
    else bwd ? go(k_resnorm_bwd<T, W, AB, false>) : go(k_resnorm<T, W, A, false>);
  };
  // The next rows are requested ahead where a block meets at barriers for every row
  // (but for the backward of 1024 threads of bf16, which has no registers for it),
  // and where a fifth or more of the lanes have no part of a row and there is less in
  // flight (backward, us: 500,000 rows of 264 with a gate 686 -> 590, 1,000,000 of 96
  // 341 -> 320; rows that fill their lanes lose 5%: of 256 788 and 834).
  const int chunks = (a.C + (dtype == 1 ? 7 : 3)) / (dtype == 1 ? 8 : 4);
  auto width = [&](auto type) {
    if (!g.wide && 5 * chunks > 4 * g.L) pick(type, std::integral_constant<int, 0>{}, std::false_type{});
    else if (!g.wide) pick(type, std::integral_constant<int, 0>{}, std::true_type{});
    else if (g.threads <= 512) pick(type, std::integral_constant<int, 512>{}, std::true_type{});
    else pick(type, std::integral_constant<int, 1024>{}, std::true_type{});
  };
  if (dtype == 1) width(bf16{});
  else width(float{});
  return hipGetLastError();
}

}  // namespace pa
