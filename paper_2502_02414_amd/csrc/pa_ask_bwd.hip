// Attention of query points over the states of their request, backward (gfx950).
// With p = exp(s - lse) and dp_ij = do_i.v_j,
//   dv_j = sum_i p_ij do_i,   ds_ij = p_ij (dp_ij - delta_i),   delta_i = sum_j p_ij dp_ij
//   dq_i = scale sum_j ds_ij k_j,   dk_j = scale sum_i ds_ij q_i
// in two passes, both of which form p and dp again: one over the states for each tile
// of queries (dq, delta), one over the queries for each tile of states (dk, dv).
// Sums over queries in one block go on in registers, over several they are records
// that are added in order.
//
// delta_i is do_i.o_i; of an o in bf16 that is off by some 2^-9 |do o|, of one in fp32 by what
// its sum over the states lost, and dq_i by that error times sum_j p_j k_j, which does not
// shrink where many states count, as dq_i does.  So dq's pass corrects it: with d0 = do.o,
// ds' = p (dp - d0), and ds'' as it is rounded for the product,
//   A = sum ds'' k,  B = sum p k:   dq = scale (A - (sum ds'') B),  delta = d0 + sum ds'.
// In bf16 that also takes out of A what the roundings of ds'' add up to (times any part that
// all k have in common): dq's error is 1.3 to 1.4 times that of its own rounding to bf16, 1.4
// to 1.5 with sum ds' in its place.  In fp32 B, which is multiplied by an error, is a product
// of p and k rounded to bf16, at 1/16 of A's time.
//
// What bounds it: the products.  8,192 queries of 4 heads over 8,192 states of one of 128,
// bf16, take 505 to 535 us, dq's pass half of it: 640 to 680 TFLOP/s counting the five products
// of the formulas, 1030 to 1090 with the eight that are formed (scores and dp twice, and B),
// 85 to 90% of what a large library product reaches on this card.  The matrix cores are busy
// for 46 to 50% (dq) and 43% of the passes' cycles (a library product at 1205 TFLOP/s for 48%),
// vector instructions take 38% and 29%, LDS 38% and 50%.  One pass over the pairs would save
// two products, but adds one side's sums in memory, by atomics (in an order that changes) or
// by records of it per block: 8,192 rows of 512 fp32 for each of the 128 tiles of states are
// 2.1 GB.
// fp32: 6,001 queries of 4 heads over 3,333 states of 2 heads of 40, 9 requests, take 90 us, the
// matrix cores busy for 30% (dq) and 35% of the passes' cycles: 1/16 of bf16's rate, on one wave
// to a SIMD (0.8 and 1.0 on average).
#include <algorithm>

#include "pa_ask.hpp"

namespace pa {
namespace {
using namespace ask;

// dq and delta of a tile of 16 QT W virtual rows, as k_ask: q and do in registers, the states
// through LDS.
template <typename T, int DP, int QT, int W>
__global__ void __launch_bounds__(64 * W, W == 8 || DP * sizeof(T) <= 256 ? 2 : 1) k_ask_dq(AskArgs a) {
  using Gm = AskGeo<T, DP, W>;
  constexpr bool HALF = sizeof(T) == 2;
  constexpr int TQ = 16 * QT * W, SHIFT = TQ == 64 ? 6 : TQ == 128 ? 7 : 8;
  __shared__ __attribute__((aligned(16))) char tiles0[2 * Gm::TB], tiles1[2 * Gm::TB];
  __shared__ __attribute__((aligned(16))) float live0[kTile], live1[kTile];
  const int G = a.Hq / a.Hkv;
  const int h = block_of() % (uint32_t)a.Hkv, s = blockIdx.y;
  const int64_t slot = block_of() / (uint32_t)a.Hkv;
  Place pl;
  if (!place_of(pl, a.q_off, a.Nq, a.k_off, a.Nk, a.R, G, SHIFT, slot)) return;
  const Range qr = pl.mine, kr = piece(pl.theirs, s, a.S);
  const int n = (int)(qr.e - qr.b) * G;
  const int64_t tile = slot - ((qr.b * G) >> SHIFT) - pl.r;
  if (tile < 0 || tile * TQ >= n) return;
  const int v0 = (int)tile * TQ;

  const int lane = lane_id(), r = lane & 15, g = lane >> 4, w = threadIdx.x >> 6;
  StateTiles<T, DP, W> st;
  st.init(a, h, kr);
  if (kr.b < kr.e) st.load(kr.b, tiles0);
  // this lane's queries: column r of the wave's QT tiles of 16
  int64_t row[QT];
  int hq[QT];
  bool on[QT];
  float d0[QT], lse2[QT], e0[QT];
  f32x4 E[HALF ? QT : 1];
  WideF<T> qf[QT][Gm::NK], of[QT][Gm::NK];
  f32x4 A[QT][Gm::ND], Bk[QT][Gm::ND];
#pragma unroll
  for (int c = 0; c < QT; ++c) {
    const int vq = v0 + (w * QT + c) * 16 + r;
    on[c] = vq < n;
    const uint32_t v = on[c] ? vq : n - 1, i = G == 1 ? v : v / (uint32_t)G;
    row[c] = qr.b + i;
    hq[c] = h * G + (int)(v - i * G);
    const int64_t at = (int64_t)hq[c] * a.D;
    row_frags<T, DP>(qf[c], reinterpret_cast<const T*>(a.o) + row[c] * a.ldo + at, a.D, on[c]);
    row_frags<T, DP>(of[c], reinterpret_cast<const T*>(a.d_o) + row[c] * a.lddo + at, a.D, on[c]);
    d0[c] = e0[c] = 0.f;
#pragma unroll
    for (int k = 0; k < Gm::NK; ++k)
#pragma unroll
      for (int e = 0; e < Wide<T>::L; ++e)
        d0[c] = fmaf(wide_elem(of[c][k], e), wide_elem(qf[c][k], e), d0[c]);
    d0[c] = groups_sum(d0[c]);
    row_frags<T, DP>(qf[c], reinterpret_cast<const T*>(a.q) + row[c] * a.ldq + at, a.D, on[c]);
    // (a row without states: lse = -inf, weights of 0)
    lse2[c] = a.lse[(int64_t)hq[c] * a.Nq + row[c]] * kLog2e;
    if (lse2[c] == -INFINITY) lse2[c] = INFINITY;
#pragma unroll
    for (int d = 0; d < Gm::ND; ++d) {
      A[c][d] = Bk[c][d] = zero4();
    }
    if constexpr (HALF) E[c] = zero4();
  }
  const bool busy = v0 + w * QT * 16 < n;
  const float sc = a.scale * kLog2e;
  const TileRead<T, DP> at;
  K16<T> ones;
  set_k16(ones, 1.f, 1.f, 1.f, 1.f);
  if (kr.b < kr.e) st.put(live0);
  auto work = [&](const char* kt, const float* live) __attribute__((always_inline)) {
    const char* vt = kt + Gm::TB;
    // (all scores first: they are on their way while the first weights are formed, and a
    // half's products while the other's are)
    f32x4 x[4][QT], dp[4][QT];
    __builtin_amdgcn_s_setprio(1);
    pipelined<4 * Gm::NK, 3, WidePair<T>>(
        [&](int i, WidePair<T>& f) {
          at.rows(f.a, kt, i / Gm::NK, i % Gm::NK);
          at.rows(f.b, vt, i / Gm::NK, i % Gm::NK);
        },
        [&](int i, const WidePair<T>& f) {
          const int t = i / Gm::NK, k = i % Gm::NK;
          const f32x4 from = k ? zero4() : *reinterpret_cast<const f32x4*>(&live[16 * t + 4 * g]);
#pragma unroll
          for (int c = 0; c < QT; ++c) {
            x[t][c] = mma(f.a, qf[c][k], k ? x[t][c] : from);
            dp[t][c] = mma(f.b, of[c][k], k ? dp[t][c] : zero4());
          }
        });
    __builtin_amdgcn_s_setprio(0);
#pragma unroll
    for (int t0 = 0; t0 < 4; t0 += 2) {
      K16<bf16> pf[QT][2];
      K16<T> sf[QT][2];
#pragma unroll
      for (int u = 0; u < 2; ++u)
#pragma unroll
        for (int c = 0; c < QT; ++c) {
          float p[4], ds[4];
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            p[i] = fast_exp2(fmaf(x[t0 + u][c][i], sc, -lse2[c]));
            ds[i] = p[i] * (dp[t0 + u][c][i] - d0[c]);
            e0[c] += ds[i];
          }
          set_k16(pf[c][u], p[0], p[1], p[2], p[3]);
          set_k16(sf[c][u], ds[0], ds[1], ds[2], ds[3]);
        }
      __builtin_amdgcn_s_setprio(1);
      if constexpr (HALF) {
#pragma unroll
        for (int c = 0; c < QT; ++c) E[c] = mma16x2(ones, sf[c][0], ones, sf[c][1], E[c]);
      }
      pipelined<Gm::ND, 4, ColumnPair<T>>(
          [&](int d, ColumnPair<T>& f) {
            at.columns(f.a, kt, t0, d);
            at.columns(f.b, kt, t0 + 1, d);
          },
          [&](int d, const ColumnPair<T>& f) {
            K16<bf16> ka, kb;
            if constexpr (HALF) {
              ka = f.a;
              kb = f.b;
            } else {
              set_k16(ka, f.a.v[0], f.a.v[1], f.a.v[2], f.a.v[3]);
              set_k16(kb, f.b.v[0], f.b.v[1], f.b.v[2], f.b.v[3]);
            }
#pragma unroll
            for (int c = 0; c < QT; ++c) {
              A[c][d] = mma16x2(f.a, sf[c][0], f.b, sf[c][1], A[c][d]);
              Bk[c][d] = mma16x2(ka, pf[c][0], kb, pf[c][1], Bk[c][d]);
            }
          });
      __builtin_amdgcn_s_setprio(0);
    }
  };
  auto turn = [&](int64_t p0, const char* now, const float* live, char* next, float* live_next)
                  __attribute__((always_inline)) {
    tiles_ready();
    const bool more = p0 + kTile < kr.e;
    if (more) st.load(p0 + kTile, next);
    if (busy && st.some(live)) work(now, live);
    if (more) st.put(live_next);
  };
  for (int64_t p0 = kr.b; p0 < kr.e; p0 += 2 * kTile) {
    turn(p0, tiles0, live0, tiles1, live1);
    if (p0 + kTile < kr.e) turn(p0 + kTile, tiles1, live1, tiles0, live0);
  }
#pragma unroll
  for (int c = 0; c < QT; ++c) {
    e0[c] = groups_sum(e0[c]);
    const float rounded = HALF ? E[c][0] : e0[c];
    if (!on[c]) continue;
    // (a row without states, or whose states' infinities left it with lse = -inf: 0 times those
    // is NaN)
    const bool none = lse2[c] == INFINITY;
    if (a.S == 1) {
      T* DQ = reinterpret_cast<T*>(a.dq) + row[c] * a.lddq + (int64_t)hq[c] * a.D;
#pragma unroll
      for (int d = 0; d < Gm::ND; ++d) {
        const f32x4 x = A[c][d] - Bk[c][d] * rounded;
        if (16 * d + 4 * g < a.D) store4<T>(DQ + 16 * d + 4 * g, none ? zero4() : x * a.scale);
      }
      if (g == 0) a.delta[(int64_t)hq[c] * a.Nq + row[c]] = d0[c] + e0[c];
    } else {
      const int64_t at = ((int64_t)s * a.Nq + row[c]) * a.Hq + hq[c];
#pragma unroll
      for (int d = 0; d < Gm::ND; ++d) {
        if (16 * d + 4 * g >= a.D) continue;
        store4<float>(a.part + at * a.D + 16 * d + 4 * g, none ? zero4() : A[c][d]);
        store4<float>(a.part_b + at * a.D + 16 * d + 4 * g, none ? zero4() : Bk[c][d]);
      }
      if (g == 0) {
        a.part_lse[at] = e0[c];
        if constexpr (HALF) a.part_e[at] = rounded;
        if (s == 0) a.delta[(int64_t)hq[c] * a.Nq + row[c]] = d0[c];
      }
    }
  }
}

// dq's pieces joined as the forward's are (join_of).
template <typename T>
__device__ __forceinline__ void put_joined(const AskArgs& a, int64_t row, int hq, int c, f32x4 A,
                                           const f32x4& B, float e, float er) {
  A -= B * (sizeof(T) == 2 ? er : e);
  store4<T>(reinterpret_cast<T*>(a.dq) + row * a.lddq + (int64_t)hq * a.D + c, A * a.scale);
  if (c == 0) a.delta[(int64_t)hq * a.Nq + row] += e;
}
template <typename T> __global__ void __launch_bounds__(256) k_ask_dq_join(AskArgs a, int each) {
  constexpr bool HALF = sizeof(T) == 2;
  const int per = a.D / 4, item = threadIdx.x / per, c = (threadIdx.x % per) * 4;
  const int64_t rows = a.Nq * a.Hq, at = (int64_t)blockIdx.x * each + item, row = at / a.Hq;
  if (item >= each || at >= rows || !asked_for(a, row)) return;
  float e = 0.f, er = 0.f;
  f32x4 A = zero4(), B = zero4();
  for (int s = 0; s < a.S; ++s) {
    e += a.part_lse[s * rows + at];
    if constexpr (HALF) er += a.part_e[s * rows + at];
    A += *reinterpret_cast<const f32x4*>(a.part + (s * rows + at) * a.D + c);
    B += *reinterpret_cast<const f32x4*>(a.part_b + (s * rows + at) * a.D + c);
  }
  put_joined<T>(a, row, (int)(at - row * a.Hq), c, A, B, e, er);
}
template <typename T> __global__ void __launch_bounds__(256) k_ask_dq_join_many(AskArgs a, int P, int U) {
  constexpr bool HALF = sizeof(T) == 2;
  __shared__ float alle[4], allr[4];
  __shared__ f32x4 lds[256];
  const int64_t rows = a.Nq * a.Hq, at = blockIdx.x, row = at / a.Hq;
  if (!asked_for(a, row)) return;
  const int t = threadIdx.x, u = t / P, c = 4 * ((int)blockIdx.y * P + t % P);
  f32x4 A = zero4(), B = zero4();
  if (u < U && c < a.D) {
#pragma unroll 8
    for (int s = u; s < a.S; s += U) {
      A += *reinterpret_cast<const f32x4*>(a.part + (s * rows + at) * a.D + c);
      B += *reinterpret_cast<const f32x4*>(a.part_b + (s * rows + at) * a.D + c);
    }
  }
  const float e = block_sum(t < a.S ? a.part_lse[t * rows + at] : 0.f, alle);
  const float er = HALF ? block_sum(t < a.S ? a.part_e[t * rows + at] : 0.f, allr) : 0.f;
  A = add_groups(A, lds, u, U, t % P, P);
  B = add_groups(B, lds, u, U, t % P, P);
  if (u == 0 && c < a.D) put_joined<T>(a, row, (int)(at - row * a.Hq), c, A, B, e, er);
}

// dk and dv of a tile of 16 KT W states: a wave has KT times 16 of them as columns, and
// their rows of k and v in registers; the queries come through LDS, 16 NR rows at a time.
template <typename T, int DP, int KT, int W, int NR>
__global__ void __launch_bounds__(64 * W, W == 8 || DP * sizeof(T) <= 256 ? 2 : 1) k_ask_dkv(AskArgs a) {
  constexpr int ROWS = 16 * NR, TK = 16 * KT * W, SHIFT = TK == 64 ? 6 : TK == 128 ? 7 : 8;
  using Gm = AskGeo<T, DP, W, ROWS>;
  __shared__ __attribute__((aligned(16))) char tiles0[2 * Gm::TB], tiles1[2 * Gm::TB];
  __shared__ __attribute__((aligned(16))) float stat0[2 * kTile], stat1[2 * kTile];  // lse (base 2), delta
  const int G = a.Hq / a.Hkv;
  const int h = block_of() % (uint32_t)a.Hkv, s = blockIdx.y;
  const int64_t slot = block_of() / (uint32_t)a.Hkv;
  Place pl;
  if (!place_of(pl, a.k_off, a.Nk, a.q_off, a.Nq, a.R, 1, SHIFT, slot)) return;
  const Range kr = pl.mine, qr = pl.theirs;
  const int64_t tile = slot - (kr.b >> SHIFT) - pl.r;
  if (tile < 0 || tile * TK >= kr.e - kr.b) return;
  const Range vr = piece(Range{0, (qr.e - qr.b) * G}, s, a.SQ);  // virtual rows
  const int n = (int)vr.e;

  const int lane = lane_id(), r = lane & 15, g = lane >> 4, w = threadIdx.x >> 6;
  QueryTiles<T, DP, W, ROWS> st;
  st.init(a, h, qr.b, n);
  const int first = (int)vr.b;
  if (first < n) st.load(first, tiles0);
  const int64_t p0 = kr.b + tile * TK + w * KT * 16 + r;
  bool busy = false;  // (a state of the wave's counts)
  bool in[KT];
  bool counts[KT];
  WideF<T> kf[KT][Gm::NK], vf[KT][Gm::NK];
  f32x4 dk[KT][Gm::ND], dv[KT][Gm::ND];
#pragma unroll
  for (int c = 0; c < KT; ++c) {
    in[c] = p0 + 16 * c < kr.e;
    const int64_t p = in[c] ? p0 + 16 * c : kr.e - 1;
    const bool on = in[c] && (!a.mask || a.mask[p]);
    counts[c] = on;
    busy = busy || __any(on);
    row_frags<T, DP>(kf[c], reinterpret_cast<const T*>(a.k) + p * a.ldk + (int64_t)h * a.D, a.D, on);
    row_frags<T, DP>(vf[c], reinterpret_cast<const T*>(a.v) + p * a.ldv + (int64_t)h * a.D, a.D, on);
#pragma unroll
    for (int d = 0; d < Gm::ND; ++d) dk[c][d] = dv[c][d] = zero4();
  }
  const float sc = a.scale * kLog2e;
  const TileRead<T, DP> at;
  if (first < n) st.put(stat0);
  auto work = [&](const char* qt, const float* stat) __attribute__((always_inline)) {
    const char* dt = qt + Gm::TB;
    f32x4 x[NR][KT], dp[NR][KT];
    __builtin_amdgcn_s_setprio(1);
    pipelined<NR * Gm::NK, 3, WidePair<T>>(
        [&](int i, WidePair<T>& f) {
          at.rows(f.a, qt, i / Gm::NK, i % Gm::NK);
          at.rows(f.b, dt, i / Gm::NK, i % Gm::NK);
        },
        [&](int i, const WidePair<T>& f) {
          const int t = i / Gm::NK, k = i % Gm::NK;
#pragma unroll
          for (int c = 0; c < KT; ++c) {
            x[t][c] = mma(f.a, kf[c][k], k ? x[t][c] : zero4());
            dp[t][c] = mma(f.b, vf[c][k], k ? dp[t][c] : zero4());
          }
        });
    __builtin_amdgcn_s_setprio(0);
#pragma unroll
    for (int t0 = 0; t0 < NR; t0 += 2) {
      K16<T> pf[KT][2], sf[KT][2];
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        const int t = t0 + u;
        const f32x4 l = *reinterpret_cast<const f32x4*>(&stat[16 * t + 4 * g]);
        const f32x4 de4 = *reinterpret_cast<const f32x4*>(&stat[kTile + 16 * t + 4 * g]);
#pragma unroll
        for (int c = 0; c < KT; ++c) {
          float pr[4], ds[4];
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            pr[i] = fast_exp2(fmaf(x[t][c][i], sc, -l[i]));
            ds[i] = pr[i] * (dp[t][c][i] - de4[i]);
          }
          set_k16(pf[c][u], pr[0], pr[1], pr[2], pr[3]);
          set_k16(sf[c][u], ds[0], ds[1], ds[2], ds[3]);
        }
      }
      __builtin_amdgcn_s_setprio(1);
      // (step 2 d: do's columns for dv, 2 d + 1: q's for dk)
      pipelined<2 * Gm::ND, 4, ColumnPair<T>>(
          [&](int i, ColumnPair<T>& f) {
            at.columns(f.a, i & 1 ? qt : dt, t0, i / 2);
            at.columns(f.b, i & 1 ? qt : dt, t0 + 1, i / 2);
          },
          [&](int i, const ColumnPair<T>& f) {
            const int d = i / 2;
#pragma unroll
            for (int c = 0; c < KT; ++c) {
              if (i & 1) dk[c][d] = mma16x2(f.a, sf[c][0], f.b, sf[c][1], dk[c][d]);
              else dv[c][d] = mma16x2(f.a, pf[c][0], f.b, pf[c][1], dv[c][d]);
            }
          });
      __builtin_amdgcn_s_setprio(0);
    }
  };
  auto turn = [&](int v0, const char* now, const float* stat, char* next, float* stat_next)
                  __attribute__((always_inline)) {
    tiles_ready();
    const bool more = v0 + ROWS < n;
    if (more) st.load(v0 + ROWS, next);
    if (busy) work(now, stat);
    if (more) st.put(stat_next);
  };
  for (int v0 = first; v0 < n; v0 += 2 * ROWS) {
    turn(v0, tiles0, stat0, tiles1, stat1);
    if (v0 + ROWS < n) turn(v0 + ROWS, tiles1, stat1, tiles0, stat0);
  }
#pragma unroll
  for (int c = 0; c < KT; ++c) {
    if (!in[c]) continue;
    const int64_t p = p0 + 16 * c;
    if (!counts[c]) {  // (weights of a row of zeros: no gradient of a state that is left out)
#pragma unroll
      for (int d = 0; d < Gm::ND; ++d) dk[c][d] = dv[c][d] = zero4();
    }
    if (a.SQ == 1) {
      T* DK = reinterpret_cast<T*>(a.dk) + p * a.lddk + (int64_t)h * a.D;
      T* DV = reinterpret_cast<T*>(a.dv) + p * a.lddv + (int64_t)h * a.D;
#pragma unroll
      for (int d = 0; d < Gm::ND; ++d) {
        if (16 * d + 4 * g >= a.D) continue;
        store4<T>(DK + 16 * d + 4 * g, dk[c][d] * a.scale);
        store4<T>(DV + 16 * d + 4 * g, dv[c][d]);
      }
    } else {
      const int64_t at = (((int64_t)s * a.Nk + p) * a.Hkv + h) * a.D;
#pragma unroll
      for (int d = 0; d < Gm::ND; ++d) {
        if (16 * d + 4 * g >= a.D) continue;
        store4<float>(a.part_k + at + 16 * d + 4 * g, dk[c][d] * a.scale);
        store4<float>(a.part_v + at + 16 * d + 4 * g, dv[c][d]);
      }
    }
  }
}

// The records of the queries' pieces added, by U groups of 256 / U threads: few records by one
// thread each, many in a tree (27,615 queries over 16 states, 128 wide, in many records: 108
// us for the call with one thread, 38 so).
template <typename T> __global__ void __launch_bounds__(256) k_ask_dkv_sum(AskArgs a, int U) {
  __shared__ f32x4 lds[256];
  const int P = 256 / U, u = threadIdx.x / P, x = threadIdx.x % P;
  const int64_t width = (int64_t)a.Hkv * a.D, all = a.Nk * width;
  const int64_t t = ((int64_t)blockIdx.x * P + x) * 4;
  const float* part = blockIdx.y ? a.part_v : a.part_k;
  f32x4 sum = zero4();
  if (t < all)
    for (int s = u; s < a.SQ; s += U) sum += *reinterpret_cast<const f32x4*>(part + s * all + t);
  if (U > 1) sum = add_groups(sum, lds, u, U, x, P);
  if (u || t >= all) return;
  const int64_t row = t / width;
  const int c = (int)(t - row * width);
  if (a.k_off && (row < a.k_off[0] || row >= a.k_off[a.R])) return;
  T* to = reinterpret_cast<T*>(blockIdx.y ? a.dv : a.dk) + row * (blockIdx.y ? a.lddv : a.lddk) + c;
  store4<T>(to, sum);
}

template <typename T, int DP, int QT, int W> hipError_t launch_dq(const AskArgs& a, hipStream_t st) {
  const int64_t slots = a.Nq * (a.Hq / a.Hkv) / (16 * QT * W) + a.R;
  hipLaunchKernelGGL((k_ask_dq<T, DP, QT, W>), grid_of(slots * a.Hkv, a.S), dim3(64 * W), 0,
                     st, a);
  return hipGetLastError();
}
template <typename T, int DP, int KT, int W, int NR = 4>
hipError_t launch_dkv(const AskArgs& a, hipStream_t st) {
  const int64_t slots = a.Nk / (16 * KT * W) + a.R;
  hipLaunchKernelGGL((k_ask_dkv<T, DP, KT, W, NR>), grid_of(slots * a.Hkv, a.SQ), dim3(64 * W),
                     0, st, a);
  return hipGetLastError();
}
// Rows of a block.  Blocks of eight waves in dq's pass, as ask_large, and of as many states
// in dk and dv's, with two tiles of 16 a wave up to 64 wide (wider ones have no registers
// for two); up to 32 wide small blocks, of which more are resident, are as fast or faster
// (us, small and large: 2,080 queries of 8 heads over 17,906 states 259 and 331 to 385,
// 8,192 over 8,192 480 and 451; 64 wide and 4 heads 387 and 327).
int rows_dq(const AskArgs& a, int dtype) {
  if (ask_eight(a, dtype)) return 128;
  return a.D <= 32 || !ask_large(a, dtype, true) ? 64 : a.D <= 64 ? 256 : 128;
}
// Requests of 32 virtual rows or fewer (on average): dk and dv's pass in tiles of 32, not of 64
// (4 queries of 16 heads over 262,808 states of 4 heads of 64, fp32, the call: 394 and 507 us;
// 20 of 4 heads over 300,000, bf16: 231 and 244).
bool few_rows(const AskArgs& a) { return a.Nq * (a.Hq / a.Hkv) <= 32 * (int64_t)a.R; }
int rows_dkv(const AskArgs& a, int dtype) {
  if (few_rows(a)) return 64;
  if (ask_eight(a, dtype)) return 128;
  const int64_t rows = a.Nq * (a.Hq / a.Hkv), each = (a.Nk + a.R - 1) / a.R;
  const bool large = dtype == 1 && 5 * each >= 4 * ((each + 255) / 256 * 256) && rows / a.R >= 128 &&
                     (a.Nk + 255) / 256 * a.Hkv * (rows / a.R / kTile) >= (a.D <= 64 ? 4096 : 2048);
  return a.D <= 32 || !large ? 64 : a.D <= 64 ? 256 : 128;
}

hipError_t passes(const AskArgs& a, int dtype, hipStream_t st) {
  hipError_t e = hipSuccess;
  if (a.Nq) {
    const bool large = rows_dq(a, dtype) > 64;
    e = by_width(a.D, dtype, [&](auto type, auto dp) {
      using T = decltype(type);
      constexpr int DP = decltype(dp)::value;
      if constexpr (sizeof(T) == 2 && DP > 32)
        if (large) return launch_dq<T, DP, DP <= 64 ? 2 : 1, 8>(a, st);
      if constexpr (sizeof(T) == 4 && DP > 64)
        if (large) return launch_dq<T, DP, 1, 8>(a, st);
      return launch_dq<T, DP, 1, 4>(a, st);
    });
    if (e != hipSuccess) return e;
    if (a.S > 1) {
      const Join j = join_of(a);
      const auto go = [&](auto type) {
        using T = decltype(type);
        if (j.U) hipLaunchKernelGGL(k_ask_dq_join_many<T>, j.grid, dim3(256), 0, st, a, j.P, j.U);
        else hipLaunchKernelGGL(k_ask_dq_join<T>, j.grid, dim3(256), 0, st, a, j.P);
      };
      dtype == 1 ? go(bf16{}) : go(float{});
      if ((e = hipGetLastError()) != hipSuccess) return e;
    }
  }
  if (!a.dk || !a.Nk) return hipSuccess;
  const bool large = rows_dkv(a, dtype) > 64;
  e = by_width(a.D, dtype, [&](auto type, auto dp) {
    using T = decltype(type);
    constexpr int DP = decltype(dp)::value;
    if constexpr (sizeof(T) == 2 && DP > 32)
      if (large) return launch_dkv<T, DP, DP <= 64 ? 2 : 1, 8>(a, st);
    if constexpr (sizeof(T) == 4 && DP > 64)
      if (large) return launch_dkv<T, DP, 1, 8>(a, st);
    return few_rows(a) ? launch_dkv<T, DP, 1, 4, 2>(a, st) : launch_dkv<T, DP, 1, 4>(a, st);
  });
  if (e != hipSuccess || a.SQ == 1) return e;
  const int U = a.SQ <= 8 ? 1 : a.SQ <= 64 ? 8 : 32;
  const int64_t quads = a.Nk * a.Hkv * a.D / 4;
  const dim3 grid((uint32_t)((quads + 256 / U - 1) / (256 / U)), 2);
  if (dtype == 1) hipLaunchKernelGGL(k_ask_dkv_sum<bf16>, grid, dim3(256), 0, st, a, U);
  else hipLaunchKernelGGL(k_ask_dkv_sum<float>, grid, dim3(256), 0, st, a, U);
  return hipGetLastError();
}

}  // namespace

// Pieces of the states in dq's pass (four products, in fp32 three and one in bf16), and of the queries in
// dk and dv's (four).
int ask_pieces_dq(const AskArgs& a, int dtype) {
  const int rows = rows_dq(a, dtype), tiles_of = rows == 256 ? 2 : 1;
  const double cycles = 600 + (dtype == 1 ? 2.0 * 4 : 32.0 * 3) * a.D;
  return ask_pieces_of(ask_blocks(a.Nq * (a.Hq / a.Hkv), a.R, rows) * a.Hkv, rows > 64 ? 8 : 4,
                       ask_resident(a, dtype, rows > 64, true), tiles_of * cycles,
                       (a.Nk / a.R + kTile - 1) / kTile,
                       8.0 * a.Nq * a.Hq * (a.D + 1));
}
int ask_pieces_q(const AskArgs& a, int dtype) {
  const int rows = rows_dkv(a, dtype), tiles_of = rows == 256 ? 2 : 1;
  const double cycles = 600 + (dtype == 1 ? 2.0 : 32.0) * 4 * a.D;
  return ask_pieces_of(ask_blocks(a.Nk, a.R, rows) * a.Hkv, rows > 64 ? 8 : 4,
                       ask_resident(a, dtype, rows > 64, true), tiles_of * cycles,
                       (a.Nq * (a.Hq / a.Hkv) / a.R + kTile - 1) / kTile,
                       8.0 * a.Nk * a.Hkv * a.D);
}

hipError_t launch_ask_backward(const AskArgs& a, int dtype, hipStream_t st) {
  return ask_few_backward_served(a, dtype) ? launch_ask_few_backward(a, st) : passes(a, dtype, st);
}

}  // namespace pa
