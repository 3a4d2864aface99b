// Attention of query points over the states of their request, backward (gfx950).
// With p = exp(s - lse) and dp_ij = do_i.v_j,
//   dv_j = sum_i p_ij do_i,   ds_ij = p_ij (dp_ij - delta_i),   delta_i = sum_j p_ij dp_ij
//   dq_i = scale sum_j ds_ij k_j,   dk_j = scale sum_i ds_ij q_i
// in two passes, both of which form p and dp again: one over the states for each tile
// of queries (dq, delta), one over the queries for each tile of states (dk, dv).
// Sums over queries in one block go on in registers, over several they are records
// that are added in order.
//
// delta_i is do_i.o_i; of an o in bf16 that is off by some 2^-9 |do o|, and dq_i by
// that error times sum_j p_j k_j, which does not shrink where many states count, as
// dq_i does.  So dq's pass corrects it: with d0 = do.o,
//   A = sum p (dp - d0) k,  B = sum p k,  e = sum p (dp - d0):
//   dq = scale (A - e B),  delta = d0 + e.
#include "pa_ask.hpp"

namespace pa {
namespace {
using namespace ask;

template <typename T, int DP>
__global__ void __launch_bounds__(256) k_ask_dq(AskArgs a) {
  using Gm = AskGeo<T, DP>;
  constexpr bool FIX = sizeof(T) == 2;
  constexpr int TQ = 64, SHIFT = 6;
  extern __shared__ __attribute__((aligned(16))) char smem[];  // [2] k and v tiles
  __shared__ float live[2][kTile];                             // 0, or -inf where left out
  const int G = a.Hq / a.Hkv;
  const int h = blockIdx.x % a.Hkv, s = blockIdx.y;
  const int64_t slot = blockIdx.x / a.Hkv;
  const int rq = request_of(a.q_off, a.R, a.Nq, G, SHIFT, slot);
  if (rq < 0) return;
  const Range qr = range_of(a.q_off, rq, a.Nq);
  const int n = (int)(qr.e - qr.b) * G;
  const int64_t tile = slot - ((qr.b * G) >> SHIFT) - rq;
  if (tile < 0 || tile * TQ >= n) return;
  const int v0 = (int)tile * TQ;
  const Range all = range_of(a.k_off, rq, a.Nk), kr = piece(all, s, a.S);
  if (all.e - all.b <= a.few) return;

  const int lane = lane_id(), r = lane & 15, g = lane >> 4, w = threadIdx.x >> 6;
  const T* K = reinterpret_cast<const T*>(a.k) + (int64_t)h * a.D;
  const T* V = reinterpret_cast<const T*>(a.v) + (int64_t)h * a.D;
  const int vq = v0 + w * 16 + r;  // this lane's query: column r of the wave's tile
  const bool on = vq < n;
  const uint32_t v = on ? vq : n - 1, i = G == 1 ? v : v / (uint32_t)G;
  const int64_t row = qr.b + i;
  const int hq = h * G + (int)(v - i * G);
  K32<T> qf[Gm::NK], of[Gm::NK];
  row_frags<T, DP>(of, reinterpret_cast<const T*>(a.o) + row * a.ldo + (int64_t)hq * a.D, a.D, on);
  row_frags<T, DP>(qf, reinterpret_cast<const T*>(a.d_o) + row * a.lddo + (int64_t)hq * a.D, a.D, on);
  float d0 = 0.f;
#pragma unroll
  for (int k = 0; k < Gm::NK; ++k)
#pragma unroll
    for (int e = 0; e < 8; ++e) d0 = fmaf(k32_elem(of[k], e), k32_elem(qf[k], e), d0);
  d0 = groups_sum(d0);
#pragma unroll
  for (int k = 0; k < Gm::NK; ++k) of[k] = qf[k];  // do from here on
  row_frags<T, DP>(qf, reinterpret_cast<const T*>(a.q) + row * a.ldq + (int64_t)hq * a.D, a.D, on);
  const bool busy = v0 + w * 16 < n;
  const float sc = a.scale * kLog2e;
  // (a row without states: lse = -inf, weights of 0)
  float lse2 = a.lse[(int64_t)hq * a.Nq + row] * kLog2e;
  if (lse2 == -INFINITY) lse2 = INFINITY;
  f32x4 A[Gm::ND], Bk[FIX ? Gm::ND : 1];
  float e0 = 0.f;
#pragma unroll
  for (int d = 0; d < Gm::ND; ++d) {
    A[d] = zero4();
    if constexpr (FIX) Bk[d] = zero4();
  }

  TileLoad<T, DP> tk, tv;
  float alive;
  auto load = [&](int64_t p0) __attribute__((always_inline)) {
    tk.states(K, a.ldk, p0, kr.e, a.D, a.mask);
    tv.states(V, a.ldv, p0, kr.e, a.D, a.mask);
    if (threadIdx.x < kTile) {
      const int64_t p = p0 + threadIdx.x;
      alive = p < kr.e && (!a.mask || a.mask[p]) ? 0.f : -INFINITY;
    }
  };
  auto put = [&](int buf) __attribute__((always_inline)) {
    tk.put(smem + buf * 2 * Gm::TB);
    tv.put(smem + buf * 2 * Gm::TB + Gm::TB);
    if (threadIdx.x < kTile) live[buf][threadIdx.x] = alive;
  };
  const RowBase<T> rb = row_base<T>(r, Gm::RB);
  const int tb = tr_base<T>(Gm::RB);
  if (kr.b < kr.e) {
    load(kr.b);
    put(0);
  }
  int buf = 0;
  for (int64_t p0 = kr.b; p0 < kr.e; p0 += kTile, buf ^= 1) {
    block_sync();
    const bool more = p0 + kTile < kr.e;
    if (more) load(p0 + kTile);
    if (busy) {
      const char* kt = smem + buf * 2 * Gm::TB;
      const char* vt = kt + Gm::TB;
      K16<T> pf[4], sf[4];
#pragma unroll
      for (int t = 0; t < 4; ++t) {
        f32x4 x = zero4(), dp = zero4();
#pragma unroll
        for (int k = 0; k < Gm::NK; ++k) {
          K32<T> kf, vf;
          ld_row<T>(kf, kt, rb, t * 16 * Gm::RB + 32 * k * Gm::SZ);
          ld_row<T>(vf, vt, rb, t * 16 * Gm::RB + 32 * k * Gm::SZ);
          x = mma32(kf, qf[k], x);
          dp = mma32(vf, of[k], dp);
        }
        if (a.mask || p0 + kTile > kr.e) {
          const f32x4 dead = *reinterpret_cast<const f32x4*>(&live[buf][16 * t + 4 * g]);
#pragma unroll
          for (int i = 0; i < 4; ++i) x[i] = dead[i] == 0.f ? x[i] : -INFINITY;
        }
        float p[4], ds[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          p[i] = fast_exp2(fmaf(x[i], sc, -lse2));
          ds[i] = p[i] * (dp[i] - d0);
          if constexpr (FIX) e0 += ds[i];
        }
        if constexpr (FIX) set_k16(pf[t], p[0], p[1], p[2], p[3]);
        set_k16(sf[t], ds[0], ds[1], ds[2], ds[3]);
      }
#pragma unroll
      for (int d = 0; d < Gm::ND; ++d) {
#pragma unroll
        for (int t = 0; t < 4; t += 2) {
          K16<T> k0, k1;
          ld_tr<T>(k0, kt, tb, t * 16 * Gm::RB + d * 16 * Gm::SZ, Gm::RB);
          ld_tr<T>(k1, kt, tb, (t + 1) * 16 * Gm::RB + d * 16 * Gm::SZ, Gm::RB);
          A[d] = mma16x2(k0, sf[t], k1, sf[t + 1], A[d]);
          if constexpr (FIX) Bk[d] = mma16x2(k0, pf[t], k1, pf[t + 1], Bk[d]);
        }
      }
    }
    if (more) put(buf ^ 1);
  }
  if constexpr (FIX) e0 = groups_sum(e0);
  if (!on) return;
  if (a.S == 1) {
    T* DQ = reinterpret_cast<T*>(a.dq) + row * a.lddq + (int64_t)hq * a.D;
#pragma unroll
    for (int d = 0; d < Gm::ND; ++d) {
      f32x4 x = A[d];
      if constexpr (FIX) x -= Bk[d] * e0;
      if (16 * d + 4 * g < a.D) store4<T>(DQ + 16 * d + 4 * g, x * a.scale);
    }
    if (g == 0) a.delta[(int64_t)hq * a.Nq + row] = d0 + e0;
  } else {
    const int64_t at = ((int64_t)s * a.Nq + row) * a.Hq + hq;
#pragma unroll
    for (int d = 0; d < Gm::ND; ++d) {
      if (16 * d + 4 * g >= a.D) continue;
      store4<float>(a.part + at * a.D + 16 * d + 4 * g, A[d]);
      if constexpr (FIX) store4<float>(a.part_b + at * a.D + 16 * d + 4 * g, Bk[d]);
    }
    if (g == 0) {
      a.part_lse[at] = e0;
      if (s == 0) a.delta[(int64_t)hq * a.Nq + row] = d0;
    }
  }
}

// dq's pieces joined: a thread has four elements of a head of a row.
template <typename T> __global__ void __launch_bounds__(256) k_ask_dq_join(AskArgs a) {
  constexpr bool FIX = sizeof(T) == 2;
  const int per = a.D / 4;
  const int64_t t = (int64_t)blockIdx.x * 256 + threadIdx.x, rows = a.Nq * a.Hq;
  const int64_t at = t / per;
  const int c = (int)(t - at * per) * 4;
  if (at >= rows) return;
  const int64_t row = at / a.Hq;
  const int hq = (int)(at - row * a.Hq);
  if (a.q_off && (row < a.q_off[0] || row >= a.q_off[a.R])) return;
  float e = 0.f;
  f32x4 A = zero4(), B = zero4();
  for (int s = 0; s < a.S; ++s) {
    e += a.part_lse[s * rows + at];
    A += *reinterpret_cast<const f32x4*>(a.part + (s * rows + at) * a.D + c);
    if constexpr (FIX) B += *reinterpret_cast<const f32x4*>(a.part_b + (s * rows + at) * a.D + c);
  }
  if constexpr (FIX) A -= B * e;
  store4<T>(reinterpret_cast<T*>(a.dq) + row * a.lddq + (int64_t)hq * a.D + c, A * a.scale);
  if (c == 0) a.delta[(int64_t)hq * a.Nq + row] += e;
}

// dk and dv of a tile of 64 states: a wave has 16 of them as columns, and their rows
// of k and v in registers; the queries come through LDS.
template <typename T, int DP>
__global__ void __launch_bounds__(256) k_ask_dkv(AskArgs a) {
  using Gm = AskGeo<T, DP>;
  extern __shared__ __attribute__((aligned(16))) char smem[];  // [2] q and do tiles
  __shared__ float stat[2][2][kTile];                          // lse (base 2), delta
  const int G = a.Hq / a.Hkv;
  const int h = blockIdx.x % a.Hkv, s = blockIdx.y;
  const int64_t slot = blockIdx.x / a.Hkv;
  const int rq = request_of(a.k_off, a.R, a.Nk, 1, 6, slot);
  if (rq < 0) return;
  const Range kr = range_of(a.k_off, rq, a.Nk);
  const int64_t tile = slot - (kr.b >> 6) - rq;
  if (tile < 0 || tile * kTile >= kr.e - kr.b || kr.e - kr.b <= a.few) return;
  const Range qr = range_of(a.q_off, rq, a.Nq);
  const Range vr = piece(Range{0, (qr.e - qr.b) * G}, s, a.SQ);  // virtual rows
  const int n = (int)vr.e;

  const int lane = lane_id(), r = lane & 15, g = lane >> 4, w = threadIdx.x >> 6;
  const T* Q = reinterpret_cast<const T*>(a.q) + (int64_t)h * G * a.D;
  const T* DO = reinterpret_cast<const T*>(a.d_o) + (int64_t)h * G * a.D;
  const int64_t p = kr.b + tile * kTile + w * 16 + r;
  const bool in = p < kr.e;
  const int64_t pc = in ? p : kr.e - 1;
  const bool on = in && (!a.mask || a.mask[pc]);
  const bool busy = kr.b + tile * kTile + w * 16 < kr.e;
  K32<T> kf[Gm::NK], vf[Gm::NK];
  row_frags<T, DP>(kf, reinterpret_cast<const T*>(a.k) + pc * a.ldk + (int64_t)h * a.D, a.D, on);
  row_frags<T, DP>(vf, reinterpret_cast<const T*>(a.v) + pc * a.ldv + (int64_t)h * a.D, a.D, on);
  const float sc = a.scale * kLog2e;
  f32x4 dk[Gm::ND], dv[Gm::ND];
#pragma unroll
  for (int d = 0; d < Gm::ND; ++d) dk[d] = dv[d] = zero4();

  TileLoad<T, DP> tq, td;
  float ls, de;
  auto load = [&](int v0) __attribute__((always_inline)) {
    tq.queries(Q, a.ldq, qr.b, G, v0, n, a.D);
    td.queries(DO, a.lddo, qr.b, G, v0, n, a.D);
    if (threadIdx.x < kTile) {
      const uint32_t v = v0 + (int)threadIdx.x < n ? v0 + threadIdx.x : n - 1;
      const uint32_t i = G == 1 ? v : v / (uint32_t)G;
      const int64_t at = (int64_t)(h * G + (int)(v - i * G)) * a.Nq + qr.b + i;
      const bool ok = v0 + (int)threadIdx.x < n;
      ls = a.lse[at] * kLog2e;
      de = a.delta[at];
      if (!ok || ls == -INFINITY) ls = INFINITY;  // (weights of 0)
      if (!ok) de = 0.f;
    }
  };
  auto put = [&](int buf) __attribute__((always_inline)) {
    tq.put(smem + buf * 2 * Gm::TB);
    td.put(smem + buf * 2 * Gm::TB + Gm::TB);
    if (threadIdx.x < kTile) {
      stat[buf][0][threadIdx.x] = ls;
      stat[buf][1][threadIdx.x] = de;
    }
  };
  const RowBase<T> rb = row_base<T>(r, Gm::RB);
  const int tb = tr_base<T>(Gm::RB);
  const int first = (int)vr.b;
  if (first < n) {
    load(first);
    put(0);
  }
  int buf = 0;
  for (int v0 = first; v0 < n; v0 += kTile, buf ^= 1) {
    block_sync();
    const bool more = v0 + kTile < n;
    if (more) load(v0 + kTile);
    if (busy) {
      const char* qt = smem + buf * 2 * Gm::TB;
      const char* dt = qt + Gm::TB;
      K16<T> pf[4], sf[4];
#pragma unroll
      for (int t = 0; t < 4; ++t) {
        f32x4 x = zero4(), dp = zero4();
#pragma unroll
        for (int k = 0; k < Gm::NK; ++k) {
          K32<T> qf, of;
          ld_row<T>(qf, qt, rb, t * 16 * Gm::RB + 32 * k * Gm::SZ);
          ld_row<T>(of, dt, rb, t * 16 * Gm::RB + 32 * k * Gm::SZ);
          x = mma32(qf, kf[k], x);
          dp = mma32(of, vf[k], dp);
        }
        const f32x4 l = *reinterpret_cast<const f32x4*>(&stat[buf][0][16 * t + 4 * g]);
        const f32x4 de4 = *reinterpret_cast<const f32x4*>(&stat[buf][1][16 * t + 4 * g]);
        float pr[4], ds[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          pr[i] = on ? fast_exp2(fmaf(x[i], sc, -l[i])) : 0.f;
          ds[i] = pr[i] * (dp[i] - de4[i]);
        }
        set_k16(pf[t], pr[0], pr[1], pr[2], pr[3]);
        set_k16(sf[t], ds[0], ds[1], ds[2], ds[3]);
      }
#pragma unroll
      for (int d = 0; d < Gm::ND; ++d) {
#pragma unroll
        for (int t = 0; t < 4; t += 2) {
          K16<T> a0, a1;
          ld_tr<T>(a0, dt, tb, t * 16 * Gm::RB + d * 16 * Gm::SZ, Gm::RB);
          ld_tr<T>(a1, dt, tb, (t + 1) * 16 * Gm::RB + d * 16 * Gm::SZ, Gm::RB);
          dv[d] = mma16x2(a0, pf[t], a1, pf[t + 1], dv[d]);
          ld_tr<T>(a0, qt, tb, t * 16 * Gm::RB + d * 16 * Gm::SZ, Gm::RB);
          ld_tr<T>(a1, qt, tb, (t + 1) * 16 * Gm::RB + d * 16 * Gm::SZ, Gm::RB);
          dk[d] = mma16x2(a0, sf[t], a1, sf[t + 1], dk[d]);
        }
      }
    }
    if (more) put(buf ^ 1);
  }
  if (!in) return;
  if (a.SQ == 1) {
    T* DK = reinterpret_cast<T*>(a.dk) + p * a.lddk + (int64_t)h * a.D;
    T* DV = reinterpret_cast<T*>(a.dv) + p * a.lddv + (int64_t)h * a.D;
#pragma unroll
    for (int d = 0; d < Gm::ND; ++d) {
      if (16 * d + 4 * g >= a.D) continue;
      store4<T>(DK + 16 * d + 4 * g, dk[d] * a.scale);
      store4<T>(DV + 16 * d + 4 * g, dv[d]);
    }
  } else {
    const int64_t at = (((int64_t)s * a.Nk + p) * a.Hkv + h) * a.D;
#pragma unroll
    for (int d = 0; d < Gm::ND; ++d) {
      if (16 * d + 4 * g >= a.D) continue;
      store4<float>(a.part_k + at + 16 * d + 4 * g, dk[d] * a.scale);
      store4<float>(a.part_v + at + 16 * d + 4 * g, dv[d]);
    }
  }
}

// The records of the queries' pieces added in order.
template <typename T> __global__ void __launch_bounds__(256) k_ask_dkv_sum(AskArgs a) {
  const int64_t width = (int64_t)a.Hkv * a.D, all = a.Nk * width;
  const int64_t t = ((int64_t)blockIdx.x * 256 + threadIdx.x) * 4;
  if (t >= all) return;
  const int64_t row = t / width;
  const int c = (int)(t - row * width);
  if (a.k_off && (row < a.k_off[0] || row >= a.k_off[a.R])) return;
  const float* part = blockIdx.y ? a.part_v : a.part_k;
  f32x4 sum = zero4();
  for (int s = 0; s < a.SQ; ++s) sum += *reinterpret_cast<const f32x4*>(part + s * all + t);
  T* to = reinterpret_cast<T*>(blockIdx.y ? a.dv : a.dk) + row * (blockIdx.y ? a.lddv : a.lddk) + c;
  store4<T>(to, sum);
}

template <typename T, int DP> hipError_t launch(const AskArgs& a, hipStream_t st) {
  using Gm = AskGeo<T, DP>;
  const int64_t G = a.Hq / a.Hkv;
  const int64_t qs = (a.Nq * G >> 6) + a.R, ks = (a.Nk >> 6) + a.R;
  hipError_t e = hipSuccess;
  if (a.Nq) {
    hipLaunchKernelGGL((k_ask_dq<T, DP>), dim3((uint32_t)(qs * a.Hkv), a.S), dim3(256), 4 * Gm::TB,
                       st, a);
    if ((e = hipGetLastError()) != hipSuccess) return e;
  }
  if (a.Nq && a.S > 1) {
    const int64_t threads = a.Nq * a.Hq * (a.D / 4);
    hipLaunchKernelGGL(k_ask_dq_join<T>, dim3((uint32_t)((threads + 255) / 256)), dim3(256), 0, st, a);
    if ((e = hipGetLastError()) != hipSuccess) return e;
  }
  if (!a.dk || !a.Nk) return hipSuccess;
  hipLaunchKernelGGL((k_ask_dkv<T, DP>), dim3((uint32_t)(ks * a.Hkv), a.SQ), dim3(256), 4 * Gm::TB,
                     st, a);
  if ((e = hipGetLastError()) != hipSuccess || a.SQ == 1) return e;
  const int64_t threads = a.Nk * a.Hkv * a.D / 4;
  hipLaunchKernelGGL(k_ask_dkv_sum<T>, dim3((uint32_t)((threads + 255) / 256), 2), dim3(256), 0, st,
                     a);
  return hipGetLastError();
}
template <typename T> hipError_t width(const AskArgs& a, hipStream_t st) {
  if (a.D <= 32) return launch<T, 32>(a, st);
  if (a.D <= 64) return launch<T, 64>(a, st);
  if (a.D <= 96) return launch<T, 96>(a, st);
  return launch<T, 128>(a, st);
}

}  // namespace

// Pieces of the queries: with fewer blocks of all of them than the chip holds.
int ask_pieces_q(const AskArgs& a) {
  const int64_t G = a.Hq / a.Hkv, blocks = ((a.Nk >> 6) + a.R) * a.Hkv;
  const int64_t tiles = (a.Nq * G / a.R + kTile - 1) / kTile;
  int64_t S = (1024 + blocks - 1) / blocks;
  if (S > tiles / 2) S = tiles / 2;
  return (int)(S < 1 ? 1 : S > 256 ? 256 : S);
}

hipError_t launch_ask_backward(const AskArgs& a, int dtype, hipStream_t st) {
  if (!ask_few_backward_served(a, dtype)) return dtype == 1 ? width<bf16>(a, st) : width<float>(a, st);
  const hipError_t e = launch_ask_few_backward(a, st);
  if (e != hipSuccess || a.R == 1 || a.Nk <= ask_few_most(a)) return e;
  // (a request that is longer than max_k says)
  AskArgs rest = a;
  rest.few = ask_few_most(a);
  rest.S = rest.SQ = 1;
  return width<bf16>(rest, st);
}

}  // namespace pa
