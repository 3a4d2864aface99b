// A linear layer in 8-bit integers on many rows of few channels, in one pass
// (gfx950, bf16 rows in and out): the rows are quantised on the way into LDS, so
// that neither their integers nor their scales go through memory (XQ: rows that
// are integers already).
//
// A block is persistent on its CU: each of its eight waves keeps the integer
// weights of 16 NCT output channels in registers (the MFMA A operand, at most
// 128 registers), and the block walks a range of the points in tiles of 32.  A
// tile's rows come from memory a tile ahead, 16 lanes per row, which find the
// row's largest magnitude among themselves, and go into a double-buffered LDS
// tile as integers; all waves read it as the B operand: one barrier per tile.
// Results leave from the registers, 64 bytes of a point's row per instruction.
//
// Measured, a million rows of bf16: 256 to 1024 channels 514 us (5.0 TB/s, what a
// copy reaches), with GELU 665 to 690 us (once the card's clock has settled: 650 to
// 990 in the first thirty passes after a pause); 1024 to 256 with a residual 635 to
// 677 us by the card (4.5 to 4.8 TB/s); 256 to 256 214 us, 64 to 256 with GELU 209 us,
// 256 to 64 174 us.  As two launches, quantised rows through memory and tiles: 1064,
// 1200, 1217, 377, 272 and 334 us.  With GELU the vector units bound it: 17 issue slots
// an output (the exp2 takes four), 1.3M cycles of four per CU at a million rows,
// beside 0.25M of the matrix cores.  Before the loads and stores lost their
// branches the compiler waited for each at once: 1024 to 256 838 us.  Issuing the
// products among the activation's instructions, run by run, changed nothing; with
// two halves' sums in registers it spilled (970 us).  Waves in their products come
// first: 1 to 3% (128 to 512 with GELU 314 -> 305 us).
//
// LDS rows hold 64 KS bytes without padding; the 16-byte chunks of row j lie at
// c ^ key(j), so that the lanes of an operand read meet different banks.
#include <type_traits>

#include "pa_i8.hpp"
#include "pa_stream.hpp"

namespace pa {
namespace {

template <bool XQ, int KS, int NCT>
struct FusedGeo {
  static constexpr int FCB = 128 * NCT;               // channels of a block
  static constexpr int PTS = 32, RB = 64 * KS;        // points of a tile, bytes of a row
  static constexpr int TILE = PTS * RB;
  // 16-byte chunks of a row per lane (XQ: of integers)
  static constexpr int NC = XQ ? (4 * KS + 15) / 16 : (8 * KS + 15) / 16;
  static constexpr int RUNS = (NCT + 1) / 2;          // runs of 8 (NCT = 1: 4) channels
};
template <int KS> __device__ __forceinline__ int key_of(int row) {
  return KS == 1 ? (row >> 1) & 3 : row & 7;
}

template <bool XQ, int ACT, int KS, int NCT>
__global__ void __launch_bounds__(512) k_linear_i8(I8Args a, int PG) {
  using G = FusedGeo<XQ, KS, NCT>;
  constexpr int V = NCT == 1 ? 4 : 8;
  __shared__ __attribute__((aligned(16))) char xs[2][G::TILE];
  __shared__ float ss[2][G::PTS];
  __shared__ __attribute__((aligned(16))) float sws[G::FCB], bs[G::FCB];
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int lane = lane_id(), r = lane & 15, g = lane >> 4;
  const int F = a.F, K = a.K, ncg = (F + G::FCB - 1) / G::FCB;
  // blocks are dealt to the XCDs round robin: the column blocks of one range of
  // points share an XCD's L2
  const int nb = gridDim.x, bl = blockIdx.x;
  const int l = nb % 8 == 0 ? (bl % 8) * (nb / 8) + bl / 8 : bl;
  const int pg = l / ncg, f0 = (l - pg * ncg) * G::FCB;
  const int64_t tiles = (a.N + G::PTS - 1) / G::PTS;
  const int64_t t0 = tiles * pg / PG, t1 = tiles * (pg + 1) / PG;  // t0 < t1 (PG <= tiles)
  const int fw = f0 + 16 * NCT * wave;  // the wave's first channel
  const bool on = fw < F;

  // Rows, results and residuals go by buffer instructions, which leave out (or read
  // as zeros) what lies behind the rows of the tile, or at an offset behind them:
  // with no branch around a load or a store, the wait for a tile's rows is neither
  // where they are requested nor one for results that were stored after that.
  auto tile_of = [&](const void* p, int64_t t, int width) {  // rows of `width` bytes
    const int64_t left = a.N - t * G::PTS;
    return __builtin_amdgcn_make_buffer_rsrc(
        const_cast<char*>(reinterpret_cast<const char*>(p)) + t * G::PTS * width, 0,
        (int)(left < G::PTS ? left : G::PTS) * width, 0x00027000);
  };
  constexpr int NOWHERE = 0x7fffff00;
  // the tile's row and chunks of this thread
  const int row = threadIdx.x >> 4, c0 = threadIdx.x & 15;
  i32x4 xr[G::NC];
  float xscale = 0.f;
  auto load = [&](int64_t t) __attribute__((always_inline)) {
    const int64_t tc = t < t1 ? t : t1 - 1;
    if constexpr (XQ) {
      const auto rx = tile_of(a.q, tc, a.Kp), rs = tile_of(a.s, tc, 4);
#pragma unroll
      for (int j = 0; j < G::NC; ++j) {
        const int c = 16 * (c0 + 16 * j);
        xr[j] = __builtin_bit_cast(
            i32x4,
            __builtin_amdgcn_raw_buffer_load_b128(rx, c < a.Kp ? row * a.Kp + c : NOWHERE, 0, 0));
      }
      xscale = __builtin_bit_cast(float, __builtin_amdgcn_raw_buffer_load_b32(rs, row * 4, 0, 0));
    } else {
      const auto rx = tile_of(a.x, tc, K * 2);
#pragma unroll
      for (int j = 0; j < G::NC; ++j) {
        const int c = 8 * (c0 + 16 * j);  // K is a multiple of 8
        xr[j] = __builtin_bit_cast(
            i32x4,
            __builtin_amdgcn_raw_buffer_load_b128(rx, c < K ? (row * K + c) * 2 : NOWHERE, 0, 0));
      }
    }
  };
  // a lane's chunk j: 8 integers, half a 16-byte chunk (XQ: 16, a whole one)
  const int put = row * G::RB + (XQ ? 16 * (c0 ^ key_of<KS>(row))
                                    : 16 * ((c0 >> 1) ^ key_of<KS>(row)) + 8 * (c0 & 1));
  auto store = [&](int buf) __attribute__((always_inline)) {
    if constexpr (XQ) {
#pragma unroll
      for (int j = 0; j < G::NC; ++j)
        if (16 * (c0 + 16 * j) < G::RB)
          *reinterpret_cast<i32x4*>(xs[buf] + put + 256 * j) = xr[j];
      if (c0 == 0) ss[buf][row] = xscale;
    } else {
      uint32_t big = 0;
#pragma unroll
      for (int j = 0; j < G::NC; ++j) big = max(big, largest(__builtin_bit_cast(Row16<bf16>, xr[j])));
      const QuantScale q = quant_scale(row16_max(big));
#pragma unroll
      for (int j = 0; j < G::NC; ++j) {
        if (8 * (c0 + 16 * j) < G::RB)
          put_chunk<false>(reinterpret_cast<int8_t*>(xs[buf] + put + 128 * j),
                           __builtin_bit_cast(Row16<bf16>, xr[j]), q.inv, 0, 0);
        if (G::NC > 2) __builtin_amdgcn_sched_barrier(0);  // (all at once would spill)
      }
      if (c0 == 0) ss[buf][row] = q.s;
    }
  };

  // weights: MFMA row r of tile i is channel fw + step(i) + 8 (r / 4) + r % 4 (NCT
  // = 1: r itself), so that a lane's results of a tile pair are 8 channels in order
  auto step = [](int i) { return NCT == 1 ? 0 : 32 * (i / 2) + 4 * (i & 1); };
  const int fr = NCT == 1 ? r : 8 * (r >> 2) + (r & 3);
  const auto rw = __builtin_amdgcn_make_buffer_rsrc(
      const_cast<int8_t*>(a.w) + (int64_t)f0 * a.Kp, 0,
      (F - f0 < G::FCB ? F - f0 : G::FCB) * a.Kp, 0x00027000);
  i32x4 w[NCT][KS];
#pragma unroll
  for (int i = 0; i < NCT; ++i) {
    const int f = fw + step(i) + fr;
#pragma unroll
    for (int s = 0; s < KS; ++s) {
      const int k = 64 * s + 16 * g;
      w[i][s] = __builtin_bit_cast(
          i32x4, __builtin_amdgcn_raw_buffer_load_b128(
                     rw, f < F && k < a.Kp ? (f - f0) * a.Kp + k : NOWHERE, 0, 0));
    }
  }
  for (int f = threadIdx.x; f < G::FCB; f += 512) {
    const bool in = f0 + f < F;
    sws[f] = in ? a.sw[f0 + f] : 0.f;
    bs[f] = in && a.bias ? a.bias[f0 + f] : 0.f;
  }
  load(t0);
  store(0);
  load(t0 + 1);

  // operand chunk 4 s + g of rows r and 16 + r (the same key)
  const int at[2] = {r * G::RB + 16 * (g ^ key_of<KS>(r)), r * G::RB + 16 * ((4 + g) ^ key_of<KS>(r))};
  // A tile's results; residuals (RES; up to two runs a half) are requested before the
  // rows of the tile after next, so that they do not wait for those.
  typedef bf16 BV __attribute__((ext_vector_type(V)));
  auto channel = [&](int q) { return 16 * NCT * wave + (NCT == 1 ? 4 * g : 32 * q + 8 * g); };
  auto place = [&](int u, int q) {  // F is a multiple of V
    const int f = f0 + channel(q);
    return f < F ? ((16 * u + r) * F + f) * 2 : NOWHERE;
  };
  auto residual = [&](__amdgpu_buffer_rsrc_t rc, int u, int q) {
    if constexpr (V == 8)
      return __builtin_bit_cast(BV, __builtin_amdgcn_raw_buffer_load_b128(rc, place(u, q), 0, 0));
    else
      return __builtin_bit_cast(BV, __builtin_amdgcn_raw_buffer_load_b64(rc, place(u, q), 0, 0));
  };
  auto tile = [&](int64_t t, int buf, auto RES) __attribute__((always_inline)) {
    constexpr bool res = decltype(RES)::value;
    const auto rd = tile_of(a.D, t, F * 2), rc = tile_of(res ? a.C : a.D, t, F * 2);
    BV c[2][G::RUNS];
    if constexpr (res)
#pragma unroll
      for (int u = 0; u < 2; ++u)
#pragma unroll
        for (int q = 0; q < G::RUNS; ++q) c[u][q] = residual(rc, u, q);
    load(t + 2);
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      const char* xb = xs[buf] + 16 * u * G::RB;
      i32x4 acc[NCT];
#pragma unroll
      for (int i = 0; i < NCT; ++i) acc[i] = i32x4{0, 0, 0, 0};
      __builtin_amdgcn_s_setprio(1);  // (products first: they run beside another wave's activation)
#pragma unroll
      for (int s = 0; s < KS; ++s) {
        const i32x4 x = *reinterpret_cast<const i32x4*>(xb + at[s & 1] + 128 * (s / 2));
#pragma unroll
        for (int i = 0; i < NCT; ++i)
          acc[i] = __builtin_amdgcn_mfma_i32_16x16x64_i8(w[i][s], x, acc[i], 0, 0, 0);
        if (KS > 4 && s % 4 == 3) __builtin_amdgcn_sched_barrier(0);  // (all at once would spill)
      }
      __builtin_amdgcn_s_setprio(0);
      const float sn = ss[buf][16 * u + r];
#pragma unroll
      for (int q = 0; q < G::RUNS; ++q) {
        const int fl = channel(q);
        BV o;
#pragma unroll
        for (int e = 0; e < V; ++e) {
          float y = fmaf((float)acc[2 * q + e / 4][e % 4], sn * sws[fl + e], bs[fl + e]);
          if constexpr (ACT == PA_ACT_GELU) y = gelu_for<bf16>(y);
          if constexpr (res) y += (float)c[u][q][e];
          o[e] = (bf16)y;
        }
        typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
        typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
        if constexpr (V == 8)
          __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4, o), rd, place(u, q), 0, 0);
        else
          __builtin_amdgcn_raw_buffer_store_b64(__builtin_bit_cast(u32x2, o), rd, place(u, q), 0, 0);
        __builtin_amdgcn_sched_barrier(0);  // (more runs at once would spill)
      }
    }
  };
  // One loop each for waves with channels, with and without residuals, and for
  // those without, and nothing in flight before it: a wait in a loop has to suit
  // every way into it.
  __builtin_amdgcn_sched_barrier(0);
  __builtin_amdgcn_s_waitcnt(0x0f70);  // vmcnt(0)
  auto walk = [&](auto body) __attribute__((always_inline)) {
    for (int64_t t = t0; t < t1; ++t) {
      const int buf = (int)(t - t0) & 1;
      block_sync();    // tile t is in LDS, tile t - 1 is read
      store(buf ^ 1);  // (behind the last tile: rows that nothing reads)
      body(t, buf);
    }
  };
  if (!on) walk([&](int64_t t, int) { load(t + 2); });
  else if (G::RUNS > 2 || !a.C) walk([&](int64_t t, int buf) { tile(t, buf, std::false_type{}); });
  else if constexpr (G::RUNS <= 2)
    walk([&](int64_t t, int buf) { tile(t, buf, std::true_type{}); });
}

template <bool XQ, int KS, int NCT>
hipError_t run(const I8Args& a, hipStream_t st) {
  using G = FusedGeo<XQ, KS, NCT>;
  if (a.C && G::RUNS > 2) return hipErrorInvalidValue;
  const int ncg = (a.F + G::FCB - 1) / G::FCB;
  const int64_t tiles = (a.N + G::PTS - 1) / G::PTS;
  const int PG = (int)(tiles < 256 / ncg ? tiles : 256 / ncg);
  const dim3 grid(PG * ncg), block(512);
  if (a.act == PA_ACT_GELU)
    hipLaunchKernelGGL((k_linear_i8<XQ, PA_ACT_GELU, KS, NCT>), grid, block, 0, st, a, PG);
  else
    hipLaunchKernelGGL((k_linear_i8<XQ, PA_ACT_NONE, KS, NCT>), grid, block, 0, st, a, PG);
  return hipGetLastError();
}
template <bool XQ>
hipError_t by_size(const I8Args& a, hipStream_t st) {
  if (a.K <= 64) return run<XQ, 1, 4>(a, st);
  if (a.K <= 128) return run<XQ, 2, 4>(a, st);
  if (a.K <= 256) {
    if (a.F <= 256) return run<XQ, 4, 2>(a, st);
    // (128 channels to a wave, so that 1024 share their rows, leave no registers for
    // residuals, which then wait for each other, and fewer, longer turns: 256 to 1024,
    // us, with 64 and 128: a million rows 607 and 519, with residuals 827 and 971;
    // 100,000 65 and 56; 50,000 30 and 32; 10,000 13 and 18)
    return a.F <= 512 || a.C || a.N < 65536 ? run<XQ, 4, 4>(a, st) : run<XQ, 4, 8>(a, st);
  }
  if (a.K <= 512) return a.F <= 128 ? run<XQ, 8, 1>(a, st) : run<XQ, 8, 4>(a, st);
  return run<XQ, 16, 2>(a, st);
}

}  // namespace

// Every block first fetches its weights: above 128 KiB of more than 256 inputs that
// takes about as long as all of the two launches on few rows.  (Two launches against
// this, us: 256 to 1024 9.5 and 8.3 at 2,048 rows, 13.2 and 8.9 at 4,096; 512 to 1024
// 10.7 and 12.3, 15.4 and 13.1; 1024 to 256 11.3 and 13.1 at 4,096, 16.4 and 13.4
// at 6,144; 256 to 256 7.9 and 5.4 at 512; 128 to 1024 7.5 and 5.9 at 512.)
bool linear_i8_fused(int64_t N, int F, int K) {
  if (F % 8 || K > 1024) return false;
  const int most = K <= 128 ? 1024 : K <= 256 ? 2048 : K <= 512 ? 1024 : 512;
  return F <= most && (K <= 256 || K * F <= 131072 || N >= (K <= 512 ? 4096 : 6144));
}

hipError_t launch_linear_i8(const I8Args& a, hipStream_t st) {
  return a.q ? by_size<true>(a, st) : by_size<false>(a, st);
}

}  // namespace pa
