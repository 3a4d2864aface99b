// Attention of many query points over few states, as an encoder of 16 to 64 of them leaves
// them (gfx950, bf16): a wave keeps its head's rows of k and v in registers and streams the
// queries past them, forward and backward in one pass each.
//
// Forward: scores as k q^T (states are rows, queries columns), left out states as
// -infinity in the accumulators' first value, and o^T = v^T p^T with the weights as
// they leave the first product.  v's columns are permuted so that a lane has eight
// consecutive elements of its query's row of o.
// Backward: the same for p and dp = v do^T; delta = sum_j p dp is formed here (all
// states are at hand), so that o is not read and a lone state's ds is 0; dq^T = k^T
// ds^T, less (sum_j ds) (sum_j p k) of ds as it is rounded, which would be 0 but for the
// roundings.  The sums over the queries, dv += p^T do and dk += ds^T q, need p and ds with
// queries along the product: they go through the wave's part of LDS, as do q and do.
// A block's dk and dv are a record in the workspace, added in order.
//
// What bounds them: memory.  A million queries of 8 heads of 32 over 64 states take 240 us,
// 1.02 GB of q and o and 32 MB of lse at 4.4 TB/s (a copy reaches 4.9), backward 390 to 410,
// 1.57 GB of q, do and dq with lse, at 4.0, and 14 for the 256 records.  The kernels of
// any number of states, which read the states from LDS for every tile of queries, take 395 and
// 1070.  Two tiles of queries are on their way while a wave works on two, and the blocks go
// over the rows together, so that what is read at one time lies in one region: with a
// range of the rows for every block and loads and stores past the caches 283 and 457 us.
#include "pa_ask.hpp"
#include "pa_ask_split.hpp"

namespace pa {
namespace {
using namespace ask;

// Row 4 g + i of product tile d stands for element 32 (d / 2) + 8 g + 4 (d % 2) + i.
__device__ __forceinline__ int column_of(int d, int r) {
  return 32 * (d >> 1) + 8 * (r >> 2) + 4 * (d & 1) + (r & 3);
}

// The states of one head as operands.
template <int DP, int NT> struct States {
  static constexpr int NK = DP / 32, ND = DP / 16;
  // rows: lane (r, g) elements 32 k + 8 g .. of state 16 t + r
  static __device__ __forceinline__ void rows(K32<bf16> (&f)[NT][NK], const bf16* base, int64_t ld,
                                              Range k, const uint8_t* mask, int D) {
#pragma unroll
    for (int t = 0; t < NT; ++t) {
      const int64_t p = k.b + 16 * t + (lane_id() & 15);
      bool counts = p < k.e;
      if (k.b < k.e) {
        const int64_t pc = counts ? p : k.e - 1;
        if (mask) counts = counts && mask[pc];
        row_frags<bf16, DP>(f[t], base + pc * ld, D, counts);
      } else {
#pragma unroll
        for (int c = 0; c < NK; ++c) f[t][c].v = __builtin_bit_cast(bf16x8, zero16());
      }
    }
  }
  // columns: lane (r, g) element column_of(d, r) of states 16 t + 4 g .. + 3, from rows
  // by way of the wave's part of LDS (kBytes of it)
  static constexpr int RB = 2 * DP + 32, kBytes = 16 * NT * RB;
  static __device__ __forceinline__ void columns(K16<bf16> (&f)[ND][NT],
                                                 const K32<bf16> (&rows)[NT][NK], char* mine) {
    const int r = lane_id() & 15, g = lane_id() >> 4;
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
      for (int k = 0; k < NK; ++k)
        *reinterpret_cast<bf16x8*>(mine + lds_off(16 * t + r, 64 * k + 16 * g, RB)) = rows[t][k].v;
    wave_sync();
    const int at = lds_off(4 * g + (r >> 2), 16 * (r & 3), RB);
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
      for (int d = 0; d < ND; ++d)
        ld_tr<bf16>(f[d][t], mine, at, 16 * t * RB + 64 * (d >> 1) + 8 * (d & 1), RB);
    wave_sync();
  }
  // 0, or -infinity where a state is left out; NaN in a request of more states than max_k
  // says, so that its answers are; whether one counts
  static __device__ __forceinline__ bool alive(f32x4 (&f)[NT], Range k, const uint8_t* mask) {
    const int g = lane_id() >> 4;
    bool some = false;
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int64_t p = k.b + 16 * t + 4 * g + i;
        bool counts = p < k.e;
        if (mask && k.b < k.e) counts = counts && mask[counts ? p : k.e - 1];
        f[t][i] = k.e - k.b > 16 * NT ? NAN : counts ? 0.f : -INFINITY;
        some = some || counts;
      }
    return __any(some);
  }
};

// A wave's LDS in the backward: 32 rows of q and of do, and of p and ds (before them, its
// states').
template <int DP, int NT> constexpr int few_bwd_bytes() {
  constexpr int rows = 64 * 2 * DP + 64 * 32 * NT;
  return States<DP, NT>::kBytes > rows ? States<DP, NT>::kBytes : rows;
}

// 16 bytes of virtual row `v` of a tile (32 of them from one that begins `rem` heads into a
// query's group), from column c on, in bytes from the tile's first query; kNowhere past D.
__device__ __forceinline__ int place(int v, int rem, int G, int64_t ld, int D, int c) {
  const uint32_t u = v + rem, i = G == 1 ? u : u / (uint32_t)G, g = u - i * G;
  return c < D ? (int)(i * (uint32_t)ld + g * D + c) * 2 : kNowhere;
}
// A tensor's rows of a head of a request from query i on, as many as a tile has and not
// behind query `last`.
__device__ __forceinline__ Buffer rows_from(const bf16* p, int64_t ld, int i, int last, int width) {
  return buffer_of(p + i * ld, ((last - i < 32 ? last - i : 32) * ld + width) * 2);
}
// 16 bytes of a row from two tiles, times f.
__device__ __forceinline__ void store_lane(Buffer b, int at, const f32x4& x, const f32x4& y, float f,
                                           bool none = false) {
  typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));
  bf16x8 o;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    o[i] = (bf16)(x[i] * f);
    o[i + 4] = (bf16)(y[i] * f);
  }
  const u32x4 bits = __builtin_bit_cast(u32x4, o);
  __builtin_amdgcn_raw_buffer_store_b128(none ? u32x4{0, 0, 0, 0} : bits, b, at, 0, 0);
}

// Which of the block's waves works on what: `heads` of them a head each, the others on
// other tiles of the same heads.
struct Role {
  int h, sub, subs;
};
__device__ __forceinline__ Role role_of(int Hkv) {
  const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int W = blockDim.x >> 6, heads = Hkv < W ? Hkv : W;
  return {(int)blockIdx.y * heads + w % heads, w / heads, W / heads};
}

template <int DP, int NT>
__global__ void __launch_bounds__(512, DP* NT <= 128 ? 4 : 2) k_ask_few(AskArgs a, int P) {
  constexpr int NK = DP / 32, ND = DP / 16, C = 2;  // C: tiles of 16 queries at once
  using S_ = States<DP, NT>;
  extern __shared__ __attribute__((aligned(16))) char smem[];
  const int G = a.Hq / a.Hkv;
  const Role me = role_of(a.Hkv);
  const int rq = blockIdx.x / P;
  const Range qr = range_of(a.q_off, rq, a.Nq), kr = range_of(a.k_off, rq, a.Nk);
  const int n = (int)(qr.e - qr.b) * G, pc = blockIdx.x % P;
  if (me.h >= a.Hkv || me.sub >= me.subs || 32 * (pc * me.subs + me.sub) >= n) return;
  const int lane = lane_id(), r = lane & 15, g = lane >> 4;
  const bf16* Q = reinterpret_cast<const bf16*>(a.q) + (int64_t)me.h * G * a.D + qr.b * a.ldq;
  const bf16* K = reinterpret_cast<const bf16*>(a.k) + (int64_t)me.h * a.D;
  const bf16* V = reinterpret_cast<const bf16*>(a.v) + (int64_t)me.h * a.D;
  bf16* O = reinterpret_cast<bf16*>(a.o) + (int64_t)me.h * G * a.D + qr.b * a.ldo;
  const float sc = a.scale * kLog2e;

  f32x4 none[NT];
  // of q: none is read where no state counts, so that no NaN is
  const int D = S_::alive(none, kr, a.mask) ? a.D : 0;

  // this lane's parts of a tile of 32 rows: 16 bytes for each step of the width
  const bool even = 32 % G == 0;  // (tiles begin at a query)
  const int last = (int)(qr.e - qr.b) - 1;
  int qo[C][NK], oo[C][NK];
  auto places = [&](int rem) __attribute__((always_inline)) {
#pragma unroll
    for (int c = 0; c < C; ++c)
#pragma unroll
      for (int k = 0; k < NK; ++k) {
        qo[c][k] = place(16 * c + r, rem, G, a.ldq, D, 32 * k + 8 * g);
        oo[c][k] = place(16 * c + r, rem, G, a.ldo, a.D, 32 * k + 8 * g);
      }
  };
  places(0);
  struct Tile {
    uint4 q[C][NK];
  };
  // (blocks go over the rows together; at most kRowsAhead, so that v + step is below 2^31)
  const int step = 16 * C * me.subs * P;
  auto load = [&](int v, Tile& t) __attribute__((always_inline)) {
    if (v >= n) return;
    const int i0 = G == 1 ? v : v / G;
    if (!even) places(v - i0 * G);
    const Buffer b = rows_from(Q, a.ldq, i0, last, G * a.D);
#pragma unroll
    for (int c = 0; c < C; ++c)
#pragma unroll
      for (int k = 0; k < NK; ++k) t.q[c][k] = load16(b, qo[c][k]);
  };
  K32<bf16> kf[NT][NK];
  K16<bf16> vf[ND][NT];
  auto work = [&](int v, const Tile& q) __attribute__((always_inline)) {
    const int i0 = G == 1 ? v : v / G;
    if (!even) places(v - i0 * G);
    const Buffer b = rows_from(O, a.ldo, i0, last, G * a.D);
#pragma unroll
    for (int c = 0; c < C; ++c) {
      f32x4 x[NT], o[ND];
#pragma unroll
      for (int t = 0; t < NT; ++t)
#pragma unroll
        for (int k = 0; k < NK; ++k) {
          K32<bf16> qf;
          set_wide(qf, q.q[c][k]);
          x[t] = mma32(kf[t][k], qf, k ? x[t] : none[t]);
        }
      float mx = -INFINITY;
#pragma unroll
      for (int t = 0; t < NT; ++t) mx = largest(mx, x[t]);
      mx = groups_largest(mx) * sc;
      const float base = mx == -INFINITY ? 0.f : mx;
      float sum = 0.f;
      K16<bf16> pf[NT];
#pragma unroll
      for (int t = 0; t < NT; ++t) {
        float p[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          p[i] = fast_exp2(fmaf(x[t][i], sc, -base));
          sum += p[i];
        }
        set_k16(pf[t], p[0], p[1], p[2], p[3]);
      }
#pragma unroll
      for (int d = 0; d < ND; ++d)
#pragma unroll
        for (int t = 0; t < NT; t += 2)
          o[d] = mma16x2(vf[d][t], pf[t], vf[d][t + 1], pf[t + 1], t ? o[d] : zero4());
      sum = groups_sum(sum);
      // (1 / 0: of weights that are all 0)
      const float inv = sum == 0.f ? 0.f : fast_rcp(sum);
      const bool in = v + 16 * c + r < n;
#pragma unroll
      for (int k = 0; k < NK; ++k) store_lane(b, in ? oo[c][k] : kNowhere, o[2 * k], o[2 * k + 1], inv);
      if (a.lse && g == 0 && in) {
        const uint32_t u = v + 16 * c + r, i = G == 1 ? u : u / (uint32_t)G;
        const float l = base + __builtin_amdgcn_logf(sum);
        a.lse[(int64_t)(me.h * G + (int)(u - i * G)) * a.Nq + qr.b + i] = l * kLn2;
      }
    }
  };
  int v = 16 * C * (pc * me.subs + me.sub);
  Tile t0, t1;
  load(v, t0);  // (on its way while the states come)
  {
    K32<bf16> vr_[NT][NK];
    S_::rows(kf, K, a.ldk, kr, a.mask, a.D);
    S_::rows(vr_, V, a.ldv, kr, a.mask, a.D);
    S_::columns(vf, vr_, smem + (threadIdx.x >> 6) * S_::kBytes);
  }
  for (;;) {  // the next tiles on their way while these are worked on
    load(v + step, t1);
    work(v, t0);
    if ((v += step) >= n) break;
    load(v + step, t0);
    work(v, t1);
    if ((v += step) >= n) break;
  }
}

// The same states' gradients and the queries', 32 queries of a wave's head at a time.
template <int DP, int NT, int TH>
__global__ void __launch_bounds__(TH, TH / 256) k_ask_few_bwd(AskArgs a, int P) {
  constexpr int NK = DP / 32, ND = DP / 16;
  // LDS rows of q and do in places as AskGeo's; of p and ds, which are written 8 bytes a
  // lane for 16 rows at once, so that those meet every bank once too.  (With 32 bytes of
  // padding between rows conflicts took 26% of the kernel's cycles: 300,000 queries over 20
  // states of 8 heads of 32 121 us, and 106 so; over 64, where memory is the bound, no less.)
  using Gm = AskGeo<bf16, DP>;
  constexpr int RB = 2 * DP, PB = 32 * NT;
  const auto key = [](int row) {
    return NT == 4 ? 2 * (row >> 1 & 3) + (row >> 3 & 1) : 2 * (row >> 2 & 1) + (row >> 3 & 1);
  };
  constexpr int CPR = DP / 8, NCH = CPR / 2;          // 16-byte chunks of a row; per lane of 32 rows
  using S_ = States<DP, NT>;
  extern __shared__ __attribute__((aligned(16))) char smem[];
  const int G = a.Hq / a.Hkv;
  const Role me = role_of(a.Hkv);
  const int rq = blockIdx.x / P;
  const Range qr = range_of(a.q_off, rq, a.Nq), kr = range_of(a.k_off, rq, a.Nk);
  const int n = (int)(qr.e - qr.b) * G, pc = blockIdx.x % P;
  if (me.h >= a.Hkv || me.sub >= me.subs) return;
  const int lane = lane_id(), r = lane & 15, g = lane >> 4;
  const int64_t head = (int64_t)me.h * G * a.D;
  const bf16* Q = reinterpret_cast<const bf16*>(a.q) + head + qr.b * a.ldq;
  const bf16* DO = reinterpret_cast<const bf16*>(a.d_o) + head + qr.b * a.lddo;
  bf16* DQ = reinterpret_cast<bf16*>(a.dq) + head + qr.b * a.lddq;
  const float sc = a.scale * kLog2e;
  char* qt = smem + (threadIdx.x >> 6) * few_bwd_bytes<DP, NT>();
  char* dt = qt + 32 * RB;
  char* pt = qt + 64 * RB;
  char* st = pt + 32 * PB;

  K32<bf16> kf[NT][NK], vf[NT][NK];
  K16<bf16> kc[ND][NT];
  f32x4 none[NT], dk[NT][ND], dv[NT][ND];
  const int D = S_::alive(none, kr, a.mask) ? a.D : 0;  // (of q and do, as forward)
#pragma unroll
  for (int t = 0; t < NT; ++t)
#pragma unroll
    for (int d = 0; d < ND; ++d) dk[t][d] = dv[t][d] = zero4();

  // this lane's parts of a tile of 32 rows: chunks of q and do, and of dq's rows
  const bool even = 32 % G == 0;  // (tiles begin at a query)
  const int last = (int)(qr.e - qr.b) - 1;
  int qo[NCH], od[NCH], dqo[2][NK];
  // (rows of q and do past the end are the last one again: zeros' scores would be NaN with a
  // state's infinity)
  auto places = [&](int rem, int rows) __attribute__((always_inline)) {
#pragma unroll
    for (int j = 0; j < NCH; ++j) {
      const int c = lane + 64 * j, u = rows == 32 || c / CPR < rows ? c / CPR : rows - 1;
      qo[j] = place(u, rem, G, a.ldq, D, c % CPR * 8);
      od[j] = place(u, rem, G, a.lddo, D, c % CPR * 8);
    }
#pragma unroll
    for (int c = 0; c < 2; ++c)
#pragma unroll
      for (int k = 0; k < NK; ++k) dqo[c][k] = place(16 * c + r, rem, G, a.lddq, a.D, 32 * k + 8 * g);
  };
  places(0, 32);
  struct Tile {
    uint4 q[NCH], d[NCH];
    float lse[2];
  } tl;
  auto load = [&](int v) __attribute__((always_inline)) {
    const int i0 = G == 1 ? v : v / G;
    if (n - v < 32) places(v - i0 * G, n - v);
    else if (!even) places(v - i0 * G, 32);
    const Buffer bq = rows_from(Q, a.ldq, i0, last, G * a.D), bd = rows_from(DO, a.lddo, i0, last, G * a.D);
#pragma unroll
    for (int j = 0; j < NCH; ++j) {
      tl.q[j] = load16(bq, qo[j]);
      tl.d[j] = load16(bd, od[j]);
    }
#pragma unroll
    for (int c = 0; c < 2; ++c) {
      const bool in = v + 16 * c + r < n;
      const uint32_t u = in ? v + 16 * c + r : n - 1, i = G == 1 ? u : u / (uint32_t)G;
      const float l = a.lse[(int64_t)(me.h * G + (int)(u - i * G)) * a.Nq + qr.b + i];
      tl.lse[c] = !in || l == -INFINITY ? INFINITY : l * kLog2e;  // (weights of 0)
    }
  };
  K16<bf16> ones;
  set_k16(ones, 1.f, 1.f, 1.f, 1.f);
  // (places of a tile's first 16 rows; those of step k, d or t differ by an exclusive or)
  const int rt = 4 * g + (r >> 2), half = 8 * (r & 1), odd = r >> 1 & 1;
  const int at_row = r * RB + (g ^ Gm::key(r)) * 16;
  const int at_col = rt * RB + (odd ^ Gm::key(rt)) * 16 + half;
  const int at_w = r * PB + ((g >> 1) ^ key(r)) * 16 + 8 * (g & 1);
  const int at_wcol = rt * PB + (odd ^ key(rt)) * 16 + half;
  const int at_in = lane / CPR * RB + ((lane % CPR) ^ Gm::key(lane / CPR)) * 16;
  const int step = 32 * me.subs * P;  // (blocks go over the rows together)
  int v = 32 * (pc * me.subs + me.sub);
  if (v < n) load(v);  // (on its way while the states come)
  S_::rows(kf, reinterpret_cast<const bf16*>(a.k) + (int64_t)me.h * a.D, a.ldk, kr, a.mask, a.D);
  S_::rows(vf, reinterpret_cast<const bf16*>(a.v) + (int64_t)me.h * a.D, a.ldv, kr, a.mask, a.D);
  S_::columns(kc, kf, qt);
  for (; v < n; v += step) {
#pragma unroll
    for (int j = 0; j < NCH; ++j) {
      *reinterpret_cast<uint4*>(qt + at_in + 1024 * j) = tl.q[j];
      *reinterpret_cast<uint4*>(dt + at_in + 1024 * j) = tl.d[j];
    }
    const float lse[2] = {tl.lse[0], tl.lse[1]};
    wave_sync();
    const int i0 = G == 1 ? v : v / G;
    const Buffer b = rows_from(DQ, a.lddq, i0, last, G * a.D);
    if (v + step < n) load(v + step);
    if (!even) places(v - i0 * G, 32);
    K16<bf16> sf[2][NT];
#pragma unroll
    for (int c = 0; c < 2; ++c) {
      K32<bf16> qf[NK], of[NK];
#pragma unroll
      for (int k = 0; k < NK; ++k) {
        set_wide(qf[k], *reinterpret_cast<const uint4*>(qt + (at_row ^ 64 * k) + 16 * c * RB));
        set_wide(of[k], *reinterpret_cast<const uint4*>(dt + (at_row ^ 64 * k) + 16 * c * RB));
      }
      f32x4 x[NT], dp[NT], e;
      K16<bf16> pf[NT];
      float delta = 0.f;
#pragma unroll
      for (int t = 0; t < NT; ++t) {
#pragma unroll
        for (int k = 0; k < NK; ++k) {
          x[t] = mma32(kf[t][k], qf[k], k ? x[t] : none[t]);
          dp[t] = mma32(vf[t][k], of[k], k ? dp[t] : zero4());
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          x[t][i] = fast_exp2(fmaf(x[t][i], sc, -lse[c]));
          delta = fmaf(x[t][i], dp[t][i], delta);
        }
        set_k16(pf[t], x[t][0], x[t][1], x[t][2], x[t][3]);
        *reinterpret_cast<bf16x4*>(pt + (at_w ^ 32 * t) + 16 * c * PB) = pf[t].v;
      }
      delta = groups_sum(delta);
#pragma unroll
      for (int t = 0; t < NT; ++t) {
        float ds[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) ds[i] = x[t][i] * (dp[t][i] - delta);
        set_k16(sf[c][t], ds[0], ds[1], ds[2], ds[3]);
        *reinterpret_cast<bf16x4*>(st + (at_w ^ 32 * t) + 16 * c * PB) = sf[c][t].v;
      }
      f32x4 dq[ND];
#pragma unroll
      for (int t = 0; t < NT; t += 2)
        e = mma16x2(ones, sf[c][t], ones, sf[c][t + 1], t ? e : zero4());
#pragma unroll
      for (int d = 0; d < ND; ++d) {
        f32x4 b;
#pragma unroll
        for (int t = 0; t < NT; t += 2) {
          dq[d] = mma16x2(kc[d][t], sf[c][t], kc[d][t + 1], sf[c][t + 1], t ? dq[d] : zero4());
          b = mma16x2(kc[d][t], pf[t], kc[d][t + 1], pf[t + 1], t ? b : zero4());
        }
        dq[d] -= b * e[0];
      }
      const bool in = v + 16 * c + r < n;
#pragma unroll
      for (int k = 0; k < NK; ++k)
        // (a row without states: 0 times their infinities is NaN)
        store_lane(b, in ? dqo[c][k] : kNowhere, dq[2 * k], dq[2 * k + 1], a.scale,
                   lse[c] == INFINITY);
    }
    // acc += (p or ds, in LDS)^T (rows, in LDS)
    auto add = [&](const char* weights, const char* rows, f32x4(&acc)[NT][ND])
                   __attribute__((always_inline)) {
      K16<bf16> b0[ND], b1[ND];
#pragma unroll
      for (int d = 0; d < ND; ++d) {
        ld_tr<bf16>(b0[d], rows, at_col ^ 32 * d, 0, RB);
        ld_tr<bf16>(b1[d], rows, at_col ^ 32 * d, 16 * RB, RB);
      }
#pragma unroll
      for (int t = 0; t < NT; ++t) {
        K16<bf16> a0, a1;
        ld_tr<bf16>(a0, weights, at_wcol ^ 32 * t, 0, PB);
        ld_tr<bf16>(a1, weights, at_wcol ^ 32 * t, 16 * PB, PB);
#pragma unroll
        for (int d = 0; d < ND; ++d) acc[t][d] = mma16x2(a0, b0[d], a1, b1[d], acc[t][d]);
      }
    };
    wave_sync();
    add(pt, dt, dv);
    add(st, qt, dk);
    wave_sync();
  }
  if (!a.dk) return;
  const int64_t rec = (int64_t)16 * NT * a.Hkv * a.D;
  const int64_t at = ((int64_t)blockIdx.x * me.subs + me.sub) * rec + (int64_t)me.h * a.D;
#pragma unroll
  for (int t = 0; t < NT; ++t)
#pragma unroll
    for (int d = 0; d < ND; ++d) {
      if (16 * d + r >= a.D) continue;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int64_t to = at + (int64_t)(16 * t + 4 * g + i) * a.Hkv * a.D + 16 * d + r;
        a.part_k[to] = dk[t][d][i] * a.scale;
        a.part_v[to] = dv[t][d][i];
      }
    }
}

// A request's records added, each of 8 threads every eighth and those in order: four
// elements of its states' rows.
__global__ void __launch_bounds__(256) k_ask_few_sum(AskArgs a, int per, int64_t rec, int blocks) {
  __shared__ f32x4 part[8][32];
  const int rq = blockIdx.x / blocks, u = threadIdx.x >> 5, c = threadIdx.x & 31;
  const int64_t first = ((int64_t)(blockIdx.x % blocks) * 32 + c) * 4, width = (int64_t)a.Hkv * a.D;
  const Range kr = range_of(a.k_off, rq, a.Nk);
  const int64_t n = (kr.e - kr.b) * width;
  const float* p = (blockIdx.y ? a.part_v : a.part_k) + (int64_t)rq * per * rec;
  f32x4 s = zero4();
  if (first < n)
    for (int i = u; i < per; i += 8) s += *reinterpret_cast<const f32x4*>(p + i * rec + first);
  part[u][c] = s;
  __syncthreads();
  if (u) return;
#pragma unroll
  for (int i = 1; i < 8; ++i) s += part[i][c];
  bf16* to = reinterpret_cast<bf16*>(blockIdx.y ? a.dv : a.dk);
  for (int64_t e = first; e < n; e += 128 * (int64_t)blocks) {
    if (n > rec) s = f32x4{NAN, NAN, NAN, NAN};  // (more states than max_k says)
    const int64_t row = e / width, col = e - row * width;
    // (weights of 0, of a do that is NaN, too)
    store4<bf16>(to + (kr.b + row) * (blockIdx.y ? a.lddv : a.lddk) + col,
                 a.mask && !a.mask[kr.b + row] ? zero4() : s);
  }
}

FewSplit split_of(const AskArgs& a, bool bwd) {
  return few_split(a.Nq, a.R, a.Hq, a.Hkv, a.D, a.max_k, bwd);
}
int tiles_of(const AskArgs& a) { return a.max_k <= 32 ? 2 : 4; }

template <int DP, int NT> hipError_t launch(const AskArgs& a, bool bwd, hipStream_t st) {
  const FewSplit s = split_of(a, bwd);
  const dim3 grid((uint32_t)(a.R * s.P), s.groups), block(64 * s.waves);
  constexpr int TH = DP * NT > 128 ? 256 : 512, lds = States<DP, NT>::kBytes;
  constexpr int lds_bwd = few_bwd_bytes<DP, NT>();
  if (!bwd) hipLaunchKernelGGL((k_ask_few<DP, NT>), grid, block, s.waves * lds, st, a, s.P);
  else hipLaunchKernelGGL((k_ask_few_bwd<DP, NT, TH>), grid, block, s.waves * lds_bwd, st, a, s.P);
  return hipGetLastError();
}
hipError_t sizes(const AskArgs& a, bool bwd, hipStream_t st) {
  const bool two = tiles_of(a) == 2;
  if (a.D <= 32) return two ? launch<32, 2>(a, bwd, st) : launch<32, 4>(a, bwd, st);
  return two ? launch<64, 2>(a, bwd, st) : launch<64, 4>(a, bwd, st);
}

}  // namespace

bool ask_few_served(const AskArgs& a, int dtype) {
  return dtype == 1 && a.D <= 64 && a.max_k <= 64 && a.R <= (1 << 20);
}

// Floats of the backward's records of dk, or of dv.
int64_t ask_few_records(const AskArgs& a) {
  const FewSplit s = split_of(a, true);
  return (int64_t)a.R * s.P * s.subs * 16 * tiles_of(a) * a.Hkv * a.D;
}
// (records of up to 256 MB: for more requests than that the other kernels need none)
bool ask_few_backward_served(const AskArgs& a, int dtype) {
  return ask_few_served(a, dtype) && ask_few_records(a) <= (1 << 25);
}

hipError_t launch_ask_few(const AskArgs& a, hipStream_t st) { return sizes(a, false, st); }

hipError_t launch_ask_few_backward(const AskArgs& a, hipStream_t st) {
  hipError_t e = sizes(a, true, st);
  if (e != hipSuccess || !a.dk) return e;
  const FewSplit s = split_of(a, true);
  const int64_t rec = (int64_t)16 * tiles_of(a) * a.Hkv * a.D;
  const int blocks = (int)((rec / 4 + 31) / 32);
  hipLaunchKernelGGL(k_ask_few_sum, dim3((uint32_t)(a.R * blocks), 2), dim3(256), 0, st, a,
                     s.P * s.subs, rec, blocks);
  return hipGetLastError();
}

}  // namespace pa
