// Attention of query points over the states of their request, forward (gfx950):
//   s_ij = scale q_i.k_j,  lse_i = log sum_j exp(s_ij),  o_i = sum_j exp(s_ij - lse_i) v_j
// over the states j of i's request that the mask leaves.  One pass over the states in
// tiles of 64 with the running maximum m and sum l of a softmax; scores, maxima and
// sums are fp32, and exp(s - m) is rounded to the operands' type for the product with
// v (bf16: 2^-9 of each weight, below the rounding of o, since the errors of several
// weights do not line up; l adds up the unrounded ones).
//
// What bounds it: with few queries to a request the read of k and v (64 queries in 64
// requests over a million states of 2 heads of 64, bf16: 100 us, 5.1 TB/s), with many the
// products and the weights' arithmetic on the same SIMDs (16,384 queries over 16,384 states,
// 4 heads of 64, bf16: 315 us, 870 TFLOP/s; the vector instructions take 66% of its cycles,
// the matrix cores 35%; fp32, whose products run at 1/16 of that rate, is bound by them).
// So: tiles come into LDS by loads that pass no register, one tile ahead of the products;
// whole tiles of 64 states go without a bound's check (a state that is not there or left out
// begins at -infinity in the accumulator); the maximum moves seldom; scores are scaled in
// the exponential's fused multiply-add.
#include <algorithm>

#include "pa_ask.hpp"

namespace pa {
namespace {
using namespace ask;

// A block has a tile of 16 QT W virtual rows and a head: a wave's QT tiles of 16 queries are
// columns of its products, and every wave reads all of a tile of states.  Two blocks of
// eight waves on a CU (128 VGPRs) with two tiles each took 315 us for 16,384 squared where
// four of four waves took 340 and, at 256 VGPRs, two of four 382.
template <typename T, int DP, int QT, int W>
__global__ void __launch_bounds__(64 * W, sizeof(T) == 2 && DP <= 64             ? 4
                                          : W == 8 || DP * sizeof(T) <= 256 ? 2
                                                                            : 1)
k_ask(AskArgs a) {
  using Gm = AskGeo<T, DP, W>;
  constexpr int TQ = 16 * QT * W, SHIFT = TQ == 64 ? 6 : TQ == 128 ? 7 : 8;
  // (arrays of their own: the compiler waits for the loads into the one that it reads)
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
  const T* Q = reinterpret_cast<const T*>(a.q) + (int64_t)h * G * a.D;
  StateTiles<T, DP, W> st;
  st.init(a, h, kr);
  if (kr.b < kr.e) st.load(kr.b, tiles0);
  // this lane's queries: column r of the wave's QT tiles of 16
  int vq[QT];
  int64_t row[QT];
  int head[QT];
  WideF<T> qf[QT][Gm::NK];
#pragma unroll
  for (int c = 0; c < QT; ++c) {
    vq[c] = v0 + (w * QT + c) * 16 + r;
    const uint32_t v = vq[c] < n ? vq[c] : n - 1;
    const uint32_t i = G == 1 ? v : v / (uint32_t)G;
    row[c] = qr.b + i;
    head[c] = v - i * G;
    row_frags<T, DP>(qf[c], Q + row[c] * a.ldq + (int64_t)head[c] * a.D, a.D, vq[c] < n);
  }
  const bool busy = v0 + w * QT * 16 < n;  // (of the wave; all load)
  const float sc = a.scale * kLog2e;
  f32x4 o[QT][Gm::ND];
  float m[QT], l[QT];
#pragma unroll
  for (int c = 0; c < QT; ++c) {
    m[c] = -INFINITY;
    l[c] = 0.f;
#pragma unroll
    for (int d = 0; d < Gm::ND; ++d) o[c][d] = zero4();
  }
  const TileRead<T, DP> at;
  if (kr.b < kr.e) st.put(live0);
  auto work = [&](const char* kt, const float* live) __attribute__((always_inline)) {
    const char* vt = kt + Gm::TB;
    f32x4 x[QT][4];
    __builtin_amdgcn_s_setprio(1);
    // (states that are left out begin at -infinity; their rows are zeros)
    pipelined<4 * Gm::NK, 3, WideF<T>>(
        [&](int i, WideF<T>& kf) { at.rows(kf, kt, i / Gm::NK, i % Gm::NK); },
        [&](int i, const WideF<T>& kf) {
          const int t = i / Gm::NK, k = i % Gm::NK;
          const f32x4 from = k ? zero4() : *reinterpret_cast<const f32x4*>(&live[16 * t + 4 * g]);
#pragma unroll
          for (int c = 0; c < QT; ++c) x[c][t] = mma(kf, qf[c][k], k ? x[c][t] : from);
        });
    __builtin_amdgcn_s_setprio(0);
    float base[QT];
#pragma unroll
    for (int c = 0; c < QT; ++c) {
      float mx = -INFINITY;
#pragma unroll
      for (int t = 0; t < 4; ++t) mx = largest(mx, x[c][t]);
      mx = groups_largest(mx) * sc;
      // The maximum moves only where a score is 2^8 above it: weights up to 2^8 are as
      // exact, and most tiles leave o and l as they are.
      if (__any(mx > m[c] + 8.f)) {
        const float to = largest(m[c], mx), down = fast_exp2(m[c] - (to == -INFINITY ? 0.f : to));
        m[c] = to;
        l[c] *= down;
#pragma unroll
        for (int d = 0; d < Gm::ND; ++d) o[c][d] *= down;
      }
      base[c] = m[c] == -INFINITY ? 0.f : m[c];  // (nothing yet: weights of 0)
    }
    // (half of the states at a time: a half's products run while the next one's weights
    // are formed)
#pragma unroll
    for (int t0 = 0; t0 < 4; t0 += 2) {
      K16<T> pf[QT][2];
#pragma unroll
      for (int c = 0; c < QT; ++c)
#pragma unroll
        for (int u = 0; u < 2; ++u) {
          float p[4];
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            p[i] = fast_exp2(fmaf(x[c][t0 + u][i], sc, -base[c]));
            l[c] += p[i];
          }
          set_k16(pf[c][u], p[0], p[1], p[2], p[3]);
        }
      __builtin_amdgcn_s_setprio(1);
      pipelined<Gm::ND, 4, ColumnPair<T>>(
          [&](int d, ColumnPair<T>& v) {
            at.columns(v.a, vt, t0, d);
            at.columns(v.b, vt, t0 + 1, d);
          },
          [&](int d, const ColumnPair<T>& v) {
#pragma unroll
            for (int c = 0; c < QT; ++c) o[c][d] = mma16x2(v.a, pf[c][0], v.b, pf[c][1], o[c][d]);
          });
      __builtin_amdgcn_s_setprio(0);
    }
  };
  // a tile is worked on while the next one comes into the other array
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
    const float sum = groups_sum(l[c]);
    if (vq[c] >= n) continue;
    const float inv = sum > 0.f ? 1.f / sum : sum == 0.f ? 0.f : sum;
    const float lse2 = sum == 0.f ? -INFINITY : m[c] + log2f(sum);
    const int hq = h * G + head[c];
    if (a.S == 1) {
      T* O = reinterpret_cast<T*>(a.o) + row[c] * a.ldo + (int64_t)hq * a.D;
#pragma unroll
      for (int d = 0; d < Gm::ND; ++d)
        if (16 * d + 4 * g < a.D) store4<T>(O + 16 * d + 4 * g, o[c][d] * inv);
      if (a.lse && g == 0) a.lse[(int64_t)hq * a.Nq + row[c]] = lse2 * kLn2;
    } else {
      const int64_t at = ((int64_t)s * a.Nq + row[c]) * a.Hq + hq;
#pragma unroll
      for (int d = 0; d < Gm::ND; ++d)
        if (16 * d + 4 * g < a.D) store4<float>(a.part + at * a.D + 16 * d + 4 * g, o[c][d] * inv);
      if (g == 0) a.part_lse[at] = lse2;
    }
  }
}

// A row's answer from the sum of its pieces' answers, weighted.
template <typename T>
__device__ __forceinline__ void put_joined(const AskArgs& a, int64_t row, int hq, int c, const f32x4& o,
                                           float sum, float base) {
  const float inv = sum > 0.f ? 1.f / sum : sum == 0.f ? 0.f : sum;
  store4<T>(reinterpret_cast<T*>(a.o) + row * a.ldo + (int64_t)hq * a.D + c, o * inv);
  if (a.lse && c == 0)
    a.lse[(int64_t)hq * a.Nq + row] = sum == 0.f ? -INFINITY : (base + log2f(sum)) * kLn2;
}
// The pieces of the states joined (join_of): up to 8, a thread four elements of a row.
template <typename T> __global__ void __launch_bounds__(256) k_ask_join(AskArgs a, int each) {
  const int per = a.D / 4, item = threadIdx.x / per, c = (threadIdx.x % per) * 4;
  const int64_t rows = a.Nq * a.Hq, at = (int64_t)blockIdx.x * each + item, row = at / a.Hq;
  if (item >= each || at >= rows || !asked_for(a, row)) return;
  float m = -INFINITY;
  for (int s = 0; s < a.S; ++s) m = fmaxf(m, a.part_lse[s * rows + at]);
  const float base = m == -INFINITY ? 0.f : m;
  float sum = 0.f;
  f32x4 o = zero4();
  for (int s = 0; s < a.S; ++s) {
    const float w = fast_exp2(a.part_lse[s * rows + at] - base);
    const f32x4 x = *reinterpret_cast<const f32x4*>(a.part + (s * rows + at) * a.D + c);
    sum += w;
    o += x * w;
  }
  put_joined<T>(a, row, (int)(at - row * a.Hq), c, o, sum, base);
}
// More: a block four times P elements of a row.
template <typename T> __global__ void __launch_bounds__(256) k_ask_join_many(AskArgs a, int P, int U) {
  __shared__ float top[4], all[4], weight[256];
  __shared__ f32x4 lds[256];
  const int64_t rows = a.Nq * a.Hq, at = blockIdx.x, row = at / a.Hq;
  if (!asked_for(a, row)) return;
  const int t = threadIdx.x, u = t / P, c = 4 * ((int)blockIdx.y * P + t % P);
  const float l = t < a.S ? a.part_lse[t * rows + at] : -INFINITY;
  const float m = block_largest(l, top), base = m == -INFINITY ? 0.f : m;
  const float w = t < a.S ? fast_exp2(l - base) : 0.f;
  weight[t] = w;
  const float sum = block_sum(w, all);  // (with a barrier: the weights are there)
  f32x4 o = zero4();
  if (u < U && c < a.D) {
#pragma unroll 8
    for (int s = u; s < a.S; s += U)
      o += *reinterpret_cast<const f32x4*>(a.part + (s * rows + at) * a.D + c) * weight[s];
  }
  o = add_groups(o, lds, u, U, t % P, P);
  if (u == 0 && c < a.D) put_joined<T>(a, row, (int)(at - row * a.Hq), c, o, sum, base);
}

template <typename T, int DP, int QT, int W> hipError_t launch(const AskArgs& a, hipStream_t st) {
  const int64_t G = a.Hq / a.Hkv, slots = a.Nq * G / (16 * QT * W) + a.R;
  hipLaunchKernelGGL((k_ask<T, DP, QT, W>), grid_of(slots * a.Hkv, a.S), dim3(64 * W), 0, st,
                     a);
  return hipGetLastError();
}
hipError_t width(const AskArgs& a, int dtype, hipStream_t st) {
  const bool large = ask_large(a, dtype, false), eight = ask_eight(a, dtype);
  return by_width(a.D, dtype, [&](auto type, auto dp) {
    using T = decltype(type);
    constexpr int DP = decltype(dp)::value;
    if constexpr (sizeof(T) == 2)
      if (large) return launch<T, DP, 2, 8>(a, st);
    if constexpr (sizeof(T) == 4 && DP > 64)
      if (eight) return launch<T, DP, 1, 8>(a, st);
    return launch<T, DP, 1, 4>(a, st);
  });
}

}  // namespace

// Blocks of eight waves with two tiles of 16 queries each (bf16) in place of four with one:
// a tile of states is read by them a quarter as often, from LDS half as often, where
// requests fill most of them and there is work for the chip (in pieces).  us, small and
// large, of 4 heads: 16,384 squared of 64 wide 407 and 345, 8,192 squared 112 and 97, 4,096
// squared 45 and 58, of 128 wide 59 and 53, 2,048 squared 28 and 35; dq's pass of 4,096
// squared of 64 wide 5 more and less.
bool ask_large(const AskArgs& a, int dtype, bool backward) {
  const int64_t rows = a.Nq * (a.Hq / a.Hkv), each = (rows + a.R - 1) / a.R;
  const int64_t tiles = a.Nk / a.R / kTile;
  return dtype == 1 && 5 * each >= 4 * ((each + 255) / 256 * 256) && tiles >= 2 &&
         (rows + 255) / 256 * a.Hkv * tiles >= (a.D > 64 ? 2048 : backward ? 4096 : 8192);
}

// fp32 heads wider than 64, whose tiles leave room for one block on a CU: eight waves where
// there is work for two on every SIMD (us, four and eight: 4,096 squared of 2 heads of 128 171
// and 156, backward 506 and 470; 1,000 queries over 300 states of 8 heads 28 and 38).
bool ask_eight(const AskArgs& a, int dtype) {
  const int64_t rows = (a.Nq * (a.Hq / a.Hkv) + kTile - 1) / kTile;
  return dtype == 0 && a.D > 64 && rows * a.Hkv * ((a.Nk / a.R + kTile - 1) / kTile) >= 1024;
}

// Blocks of R requests of some N rows in all (none has more than it takes on average), of `rows` each.
int64_t ask_blocks(int64_t N, int64_t R, int rows) {
  return R * (((N + R - 1) / R + rows - 1) / rows);
}
// The number of pieces whose time comes out shortest: blocks of `waves` that take `cycles`
// for each of `tiles` tiles.  n waves of a SIMD share it, up to `resident`, in n + 1 times
// one's cycles (none is faster than 2000); a block's start is 6000; what does not fit comes in
// rounds, of which the last one is one more where a CU has one block at a time, and a part
// of one where it has several, whose ends differ; several pieces are joined, `bytes` each at 1.5 KB a
// cycle, by a launch of 6000.  (us, the pieces that it chooses and others: 10,792 queries over
// 17,721 states of 4 heads of 80, 4 pieces 364, 1 450, 2 461, 8 386; 643 over 14,654 of 8 of 32,
// 16 42, 1 147, 4 53; 16,384 squared of 4 of 64, 2 333, 1 391, 4 325.)
int ask_pieces_of(int64_t blocks, int waves, int resident, double cycles, int64_t tiles,
                  double bytes) {
  int best = 1;
  double least = 0;
  const int64_t once = 1024 * resident / waves;
  for (int S = 1; S <= 256 && S <= (tiles > 1 ? tiles : 1); S *= 2) {
    const double each = (double)((tiles + S - 1) / S);
    const auto round = [&](double n) { return 6000 + each * std::max(2000.0, cycles * (n + 1)); };
    const int64_t rounds = blocks * S / once, last = blocks * S % once;
    double t = rounds * round(resident) + (S > 1 ? 6000 + S * bytes / 1500 : 0);
    if (rounds == 0 || (last && once == 256)) t += round((double)last * waves / 1024);
    else t += round(resident) * last / once;
    if (S == 1 || t < least) {
      best = S;
      least = t;
    }
  }
  return best;
}
// Waves of a SIMD that the kernels' registers and LDS leave room for.
int ask_resident(const AskArgs& a, int dtype, bool eight, bool backward) {
  if (dtype == 0) return a.D <= 32 ? 4 : a.D <= 64 || eight ? 2 : 1;
  return a.D <= 64 && !(eight && backward) ? 4 : 2;
}
int ask_pieces(const AskArgs& a, int dtype) {
  const int64_t rows = a.Nq * (a.Hq / a.Hkv), tiles = (a.Nk / a.R + kTile - 1) / kTile;
  const bool large = ask_large(a, dtype, false);
  const int block = large ? 256 : ask_eight(a, dtype) ? 128 : 64;
  const double cycles = 450 + (dtype == 1 ? 2.0 : 32.0) * 2 * a.D;  // softmax, two products
  return ask_pieces_of(ask_blocks(rows, a.R, block) * a.Hkv, block > 64 ? 8 : 4,
                       ask_resident(a, dtype, block > 64, false), large ? 2 * cycles : cycles, tiles,
                       4.0 * a.Nq * a.Hq * (a.D + 1));
}

hipError_t launch_ask(const AskArgs& a, int dtype, hipStream_t st) {
  if (ask_few_served(a, dtype)) return launch_ask_few(a, st);
  const hipError_t e = width(a, dtype, st);
  if (e != hipSuccess || a.S == 1) return e;
  const Join j = join_of(a);
  const auto go = [&](auto type) {
    using T = decltype(type);
    if (j.U) hipLaunchKernelGGL(k_ask_join_many<T>, j.grid, dim3(256), 0, st, a, j.P, j.U);
    else hipLaunchKernelGGL(k_ask_join<T>, j.grid, dim3(256), 0, st, a, j.P);
  };
  dtype == 1 ? go(bf16{}) : go(float{});
  return hipGetLastError();
}

}  // namespace pa
