// Linear layers in 8-bit integers (gfx950): rows quantised with a scale each,
// integer products on v_mfma_i32_16x16x64_i8 (exact in 32 bits), and the scales,
// bias, activation and residual add on the way out.
//
// The weights are the MFMA's A operand and the points its B operand, so that a
// lane of a 16 x 16 result tile holds four consecutive channels of one point.
//
// Large products: 8192^3 456 to 474 us (2.3 to 2.4 PFLOP/s' worth of operations; a
// library product of plain integers 2.07), 4096^3 64 to 74 us by the card, on a first
// form whose operands came straight from memory, without LDS, 640 us.  Bound by waits,
// not by a unit: counters at 4096^3 (72.5 us at 2.27 GHz) have the matrix cores busy 40%
// of the cycles and LDS 15%, without bank conflicts, and the waves waiting 42% of
// theirs (for loads one step ahead, at a barrier per step; before the first products
// and behind the last, 12 us by the constants of the tiles' model).  Also built, exact and
// within 3% (not kept): two groups of four waves that take turns between the
// products and the operand reads, with raised wave priority and four buffers of 64
// bytes of K (4096^3 75 us where this form takes 74 on the same card; 8192^3 463
// and 474).  Small products are bound by latency: 333 x 1000 x 517 5.0 us with
// four buffers under the tiles of 64 x 64, 9.8 us with two.  Four groups of waves
// that share K gained 0 to 15% there (128 x 4096 x 4096 10.8 -> 9.2 us) and lost
// as much below K = 1024: not kept.
#include <type_traits>

#include "pa_i8.hpp"

namespace pa {
namespace {

// All but the wave's last LATER loads are done, and all its LDS reads, for all
// waves of the block.
template <int LATER> __device__ __forceinline__ void tile_ready() {
  asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"i"(LATER) : "memory");
}

// ---------------------------------------------------------------------------
// Tiled product.  A block of WF x WN waves forms a tile of TF channels x TN
// points, each wave MF x MN MFMA tiles of 16 x 16, over steps of 128 bytes of
// K.  A step's rows come from memory straight into LDS (16 bytes per lane), NB - 1
// steps ahead, in NB buffers.  A buffer load past the last row or past a row's
// end (K is no multiple of 128) leaves zeros.
//
// LDS rows are 128 bytes, without padding (a wave's load fills 1 KB in order);
// the 16-byte chunks of row j lie at c ^ key(j), so that the lanes of an operand
// read (one chunk of 16 rows) meet different banks.
//
// Channels go to MFMA rows so that a lane's results are 16 bytes of a point's
// row: bf16: tile pairs (2 j, 2 j + 1) hold channels 32 j + 8 g + 4 (i & 1) ..
// of lane group g; fp32: tile i holds channels 16 i + 4 g ..
// ---------------------------------------------------------------------------
template <int WF, int WN, int MF, int MN, int NB>
struct I8Geo {
  static constexpr int W = WF * WN, TF = 16 * MF * WF, TN = 16 * MN * WN, BK = 128;
  static constexpr int LF = TF / 8 / W, LN = TN / 8 / W;  // 1 KB loads per wave and step
  static constexpr int BUF = (TF + TN) * BK;
  static_assert(LF * W * 8 == TF && LN * W * 8 == TN, "whole loads");
  static_assert(NB * BUF <= 160 * 1024, "the buffers fit");
};

template <typename T>
__device__ __forceinline__ int key_f(int row) {  // of a row of weights
  if constexpr (sizeof(T) == 2) return (row & 3) | ((row >> 3) & 1) << 2;
  else return row & 7;
}
__device__ __forceinline__ int key_n(int row) { return row & 7; }

// A wave's results: acc[i][j] is MFMA tile i of its channels, from f1 on, and j of
// its points, n1 + 16 j; in runs of V channels of one point.  (A row's start, and
// so a run, need not be aligned: F is any number.)
template <typename T, int ACT, int MF, int MN>
__device__ __forceinline__ void results(const I8Args& a, const i32x4 (&acc)[MF][MN], int64_t n1,
                                        int f1, int g) {
  constexpr int V = sizeof(T) == 2 ? 8 : 4, RUN = V / 4;
  typedef T TV __attribute__((ext_vector_type(V)));
  T* D = reinterpret_cast<T*>(a.D);
  const T* Cr = reinterpret_cast<const T*>(a.C);
  // Residuals of MN runs are requested together, the next ones before these are worked
  // on.  (From the start of C where there is no whole run.)
  const bool some = Cr && a.N * a.F >= V;
  auto residuals = [&](int i, TV(&c)[MN]) __attribute__((always_inline)) {
    const int f = f1 + (sizeof(T) == 2 ? 16 * i + 8 * g : 16 * i + 4 * g);
#pragma unroll
    for (int j = 0; j < MN; ++j) {
      const int64_t n = n1 + 16 * j;
      __builtin_memcpy(&c[j], Cr + (n < a.N && f + V <= a.F ? n * a.F + f : 0), 16);
    }
  };
  TV c[2][MN];
  if (some) residuals(0, c[0]);
  float sn[MN];
#pragma unroll
  for (int j = 0; j < MN; ++j) sn[j] = a.s[n1 + 16 * j < a.N ? n1 + 16 * j : a.N - 1];
#pragma unroll
  for (int i = 0; i < MF; i += RUN) {
    const int f = f1 + (sizeof(T) == 2 ? 16 * i + 8 * g : 16 * i + 4 * g);
    float sw[V], b[V];
#pragma unroll
    for (int e = 0; e < V; ++e) {
      const int fe = f + e < a.F ? f + e : a.F - 1;
      sw[e] = a.sw[fe];
      b[e] = a.bias ? a.bias[fe] : 0.f;
    }
    if (some && i + RUN < MF) residuals(i + RUN, c[(i / RUN + 1) & 1]);
#pragma unroll
    for (int j = 0; j < MN; ++j) {
      const int64_t n = n1 + 16 * j, at = n * a.F + f;
      float u[V];
#pragma unroll
      for (int e = 0; e < V; ++e) {
        u[e] = fmaf((float)acc[i + e / 4][j][e % 4], sn[j] * sw[e], b[e]);
        if constexpr (ACT == PA_ACT_GELU) u[e] = gelu_for<T>(u[e]);
      }
      if (n < a.N && f + V <= a.F) {
        if (Cr) {
#pragma unroll
          for (int e = 0; e < V; ++e) u[e] += (float)c[(i / RUN) & 1][j][e];
        }
        TV o;
#pragma unroll
        for (int e = 0; e < V; ++e) o[e] = (T)u[e];
        __builtin_memcpy(D + at, &o, 16);
      } else if (n < a.N) {
#pragma unroll
        for (int e = 0; e < V; ++e)
          if (f + e < a.F) D[at + e] = from_f<T>(Cr ? u[e] + to_f<T>(Cr[at + e]) : u[e]);
      }
      __builtin_amdgcn_sched_barrier(0);  // (more runs at once would spill)
    }
  }
}

template <typename T, int ACT, int WF, int WN, int MF, int MN, int NB>
__global__ void __launch_bounds__(64 * WF * WN, 2) k_gemm_i8(I8Args a) {
  using G = I8Geo<WF, WN, MF, MN, NB>;
  constexpr int BK = G::BK;
  __shared__ __attribute__((aligned(16))) char buf0[G::BUF];
  __shared__ __attribute__((aligned(16))) char buf1[G::BUF];
  __shared__ __attribute__((aligned(16))) char buf2[NB > 2 ? G::BUF : 16];
  __shared__ __attribute__((aligned(16))) char buf3[NB > 3 ? G::BUF : 16];
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int lane = lane_id(), r = lane & 15, g = lane >> 4;
  const int wf = wave % WF, wn = wave / WF;
  // Blocks are dealt to the XCDs round robin: each gets a run of tiles in an order that
  // goes over all channels for GROUP tiles of points at a time, so that both operands'
  // rows are found in its L2 (in order of blockIdx: 13,426 x 4096 to 223 56 us in place
  // of 28, 100,000 x 1040 to 300 84 in place of 65; squares of 4096 and 8192 the same).
  constexpr unsigned GROUP = 8;
  const unsigned ftiles = (unsigned)(a.F + G::TF - 1) / G::TF, ntiles = gridDim.x / ftiles;
  const unsigned xcd = blockIdx.x % 8, per = gridDim.x / 8, more = gridDim.x % 8;
  const unsigned l = xcd * per + (xcd < more ? xcd : more) + blockIdx.x / 8;
  const unsigned grp = l / (GROUP * ftiles), in = l - grp * GROUP * ftiles;
  const unsigned wide = ntiles - grp * GROUP < GROUP ? ntiles - grp * GROUP : GROUP;
  const int64_t n0 = (int64_t)(grp * GROUP + in % wide) * G::TN;
  const int f0 = (int)(in / wide) * G::TF;
  const int rows_n = (int)(a.N - n0 < G::TN ? a.N - n0 : G::TN);
  const int rows_f = a.F - f0 < G::TF ? a.F - f0 : G::TF;

  const auto rw = __builtin_amdgcn_make_buffer_rsrc(
      const_cast<int8_t*>(a.w) + (int64_t)f0 * a.Kp, 0, rows_f * a.Kp, 0x00027000);
  const auto rq = __builtin_amdgcn_make_buffer_rsrc(
      const_cast<int8_t*>(a.q) + n0 * a.Kp, 0, rows_n * a.Kp, 0x00027000);

  // this lane's row and chunk in each of its wave's loads
  int off[G::LF + G::LN], chunk[G::LF + G::LN];
#pragma unroll
  for (int j = 0; j < G::LF + G::LN; ++j) {
    const bool isf = j < G::LF;
    const int row = 8 * ((isf ? j : j - G::LF) * G::W + wave) + (lane >> 3);
    chunk[j] = 16 * ((lane & 7) ^ (isf ? key_f<T>(row) : key_n(row)));
    off[j] = row * a.Kp + chunk[j];
  }
  auto load = [&](char* buf, int k0) {
#pragma unroll
    for (int j = 0; j < G::LF + G::LN; ++j) {
      const bool isf = j < G::LF;
      char* dst = buf + (isf ? 0 : G::TF * BK) + 1024 * ((isf ? j : j - G::LF) * G::W + wave);
      const int o = k0 + chunk[j] < a.Kp ? off[j] + k0 : 0x7fffff00;
      __builtin_amdgcn_raw_ptr_buffer_load_lds(
          isf ? rw : rq, (__attribute__((address_space(3))) void*)dst, 16, o, 0, 0, 0);
    }
    __builtin_amdgcn_sched_barrier(0);  // (before the products of the step before, not behind them)
  };

  i32x4 acc[MF][MN];
#pragma unroll
  for (int i = 0; i < MF; ++i)
#pragma unroll
    for (int j = 0; j < MN; ++j) acc[i][j] = i32x4{0, 0, 0, 0};

  // operand reads: row of MFMA row r of the wave's first tile, then constants
  const int row_f = wf * 16 * MF + (sizeof(T) == 2 ? 8 * (r >> 2) + (r & 3) : r);
  const int row_n = wn * 16 * MN + r;
  const int kf = key_f<T>(row_f), kn = key_n(row_n);
  auto step_f = [](int i) { return sizeof(T) == 2 ? 32 * (i / 2) + 4 * (i & 1) : 16 * i; };
  auto compute = [&](const char* buf) {
#pragma unroll
    for (int s = 0; s < 2; ++s) {
      i32x4 x[MN], w[MF];
      const char* pf = buf + row_f * BK + 16 * ((4 * s + g) ^ kf);
      const char* pn = buf + (G::TF + row_n) * BK + 16 * ((4 * s + g) ^ kn);
#pragma unroll
      for (int j = 0; j < MN; ++j) x[j] = *reinterpret_cast<const i32x4*>(pn + 16 * BK * j);
#pragma unroll
      for (int i = 0; i < MF; ++i) w[i] = *reinterpret_cast<const i32x4*>(pf + BK * step_f(i));
#pragma unroll
      for (int i = 0; i < MF; ++i)
#pragma unroll
        for (int j = 0; j < MN; ++j)
          acc[i][j] = __builtin_amdgcn_mfma_i32_16x16x64_i8(w[i], x[j], acc[i][j], 0, 0, 0);
    }
  };

  // step k is computed while the NB - 1 next ones come into the other buffers, the
  // last of which every wave has read before the barrier.  (Separate arrays, not
  // one: the compiler waits for the loads into the array that it reads.  Loads
  // behind the last step put zeros where nothing is read.)
  constexpr int PER = G::LF + G::LN;
  const int steps = (a.Kp + BK - 1) / BK;
  if constexpr (NB == 2) {
    load(buf0, 0);
    int s = 0;
    for (; s + 1 < steps; s += 2) {
      tile_ready<0>();
      load(buf1, (s + 1) * BK);
      compute(buf0);
      tile_ready<0>();
      if (s + 2 < steps) load(buf0, (s + 2) * BK);
      compute(buf1);
    }
    if (s < steps) {
      tile_ready<0>();
      compute(buf0);
    }
  } else {
    static_assert(NB == 4, "two or four buffers");
    load(buf0, 0);
    load(buf1, BK);
    load(buf2, 2 * BK);
    auto step = [&](int s, char* next, const char* now) __attribute__((always_inline)) {
      if (s < steps) {
        tile_ready<2 * PER>();
        load(next, (s + 3) * BK);
        compute(now);
      }
    };
    for (int s = 0; s < steps; s += 4) {
      step(s, buf3, buf0);
      step(s + 1, buf0, buf1);
      step(s + 2, buf1, buf2);
      step(s + 3, buf2, buf3);
    }
    __builtin_amdgcn_s_waitcnt(0x0f70);  // vmcnt(0): nothing comes into LDS once it is given back
  }

  results<T, ACT, MF, MN>(a, acc, n0 + row_n, f0 + wf * 16 * MF, g);
}

// ---------------------------------------------------------------------------
// Rows quantised.  A lane holds chunks of 16 bytes of a row in registers (the
// last one of a row may be cut short; rows need not be aligned), so that a row is
// read once: rows of up to 64 chunks are shared by the smallest power of two of
// lanes, U rows each in turn with all their loads first; longer ones take a wave
// and NC chunks per lane.  Bound by memory: 4096 rows of 4096 bf16 9.7 us (5.2
// TB/s), a million of 256 147 us (5.2 TB/s); unaligned rows touch more lines:
// 100,000 of 257 23 us where 256 take 17, 50,000 of 1001 fp32 38 us.  (With the shift
// of a cut chunk on the row's elements, for every chunk, in place of one on its
// integers those took 20 to 60% longer.)  Rows beyond 1024 chunks take a block and
// are read twice.
// ---------------------------------------------------------------------------
template <typename T, bool ODD, int NC, int U>
__global__ void __launch_bounds__(256) k_quant_rows(int64_t N, int K, int Kp, int L, const T* x,
                                                    int8_t* q, float* s) {
  constexpr int E = Row16<T>::E;
  const int per = 256 / L, slot = threadIdx.x / L, c0 = threadIdx.x % L, CP = Kp / E;
  const int64_t step = (int64_t)gridDim.x * per * U;
  for (int64_t base = (int64_t)blockIdx.x * per * U; base < N; base += step) {
    Row16<T> v[U][NC];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int64_t n = base + u * per + slot;
#pragma unroll
      for (int j = 0; j < NC; ++j)
        v[u][j] = row_chunk<ODD>(x + (n < N ? n : N - 1) * K, K, c0 + j * L);
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int64_t n = base + u * per + slot;
      uint32_t big = 0;
#pragma unroll
      for (int j = 0; j < NC; ++j) big = max(big, largest(v[u][j]));
      for (int o = 1; o < L; o <<= 1) big = max(big, (uint32_t)__shfl_xor((int)big, o));
      const QuantScale c = quant_scale(big);
      if (n >= N) continue;
#pragma unroll
      for (int j = 0; j < NC; ++j)
        if (c0 + j * L < CP)
          put_chunk<ODD>(q + n * Kp + E * (c0 + j * L), v[u][j], c.inv, K, c0 + j * L);
      if (c0 == 0) s[n] = c.s;
    }
  }
}

// Rows shorter than a chunk: a row per thread.
template <typename T>
__global__ void __launch_bounds__(256) k_quant_short(int64_t N, int K, const T* x, int8_t* q,
                                                     float* s) {
  const int64_t step = (int64_t)gridDim.x * 256;
  for (int64_t n = (int64_t)blockIdx.x * 256 + threadIdx.x; n < N; n += step) {
    float v[8];
    uint32_t big = 0;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      v[e] = e < K ? to_f<T>(x[n * K + e]) : 0.f;
      big = max(big, __builtin_bit_cast(uint32_t, v[e]) & 0x7fffffffu);
    }
    const QuantScale c = quant_scale(big);
    *reinterpret_cast<uint4*>(q + n * 16) = {quant4(v[0], v[1], v[2], v[3], c.inv),
                                             quant4(v[4], v[5], v[6], v[7], c.inv), 0u, 0u};
    s[n] = c.s;
  }
}

template <typename T, bool ODD>
__global__ void __launch_bounds__(512) k_quant_long(int64_t N, int K, int Kp, const T* x,
                                                    int8_t* q, float* s) {
  constexpr int E = Row16<T>::E;
  __shared__ uint32_t red[8];
  const int CP = Kp / E;
  for (int64_t n = blockIdx.x; n < N; n += gridDim.x) {
    uint32_t big = 0;
    for (int c = threadIdx.x; c < CP; c += 512) big = max(big, largest(row_chunk<ODD>(x + n * K, K, c)));
    for (int o = 1; o < 64; o <<= 1) big = max(big, (uint32_t)__shfl_xor((int)big, o));
    __syncthreads();
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = big;
    __syncthreads();
    for (int w = 0; w < 8; ++w) big = max(big, red[w]);
    const QuantScale k = quant_scale(big);
    for (int c = threadIdx.x; c < CP; c += 512)
      put_chunk<ODD>(q + n * Kp + E * c, row_chunk<ODD>(x + n * K, K, c), k.inv, K, c);
    if (threadIdx.x == 0) s[n] = k.s;
  }
}

// Weights, a block per 64 channels: the columns' maxima, then their integers, four
// rows to a thread, turned into rows by LDS.  WHOLE: 16 bytes at a time.  4096 to 4096
// bf16 28 us (a first form with 256 threads that took an element at a time 601).
template <typename T, bool WHOLE>
__global__ void __launch_bounds__(1024) k_quant_weight(int K, int Kp, int F, const T* W,
                                                       int8_t* q, float* sw) {
  constexpr int E = Row16<T>::E, CL = 64 / E, R = 1024 / CL, KB = 4 * R, RB = KB + 16;
  __shared__ __attribute__((aligned(16))) int8_t xs[64 * RB];
  __shared__ uint32_t big[64];
  const int tid = threadIdx.x, cl = tid % CL, r = tid / CL, f0 = blockIdx.x * 64, f = f0 + E * cl;
  // this thread's four rows of a turn; behind the last row and channel the last ones
  auto load = [&](int k0, Row16<T>(&v)[4]) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int k = k0 + 4 * r + i;
      const T* row = W + (int64_t)(k < K ? k : K - 1) * F;
      if constexpr (WHOLE) {
        v[i] = __builtin_bit_cast(Row16<T>, *reinterpret_cast<const uint4*>(row + (f < F ? f : F - E)));
      } else {
#pragma unroll
        for (int e = 0; e < E; ++e) v[i].v[e] = row[f + e < F ? f + e : F - 1];
      }
    }
  };
  if (tid < 64) big[tid] = 0;
  __syncthreads();
  uint32_t m[E];
#pragma unroll
  for (int e = 0; e < E; ++e) m[e] = 0;
  auto largest4 = [&](const Row16<T>(&v)[4]) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int e = 0; e < E; ++e)
        m[e] = max(m[e], __builtin_bit_cast(uint32_t, to_f<T>(v[i].v[e])) & 0x7fffffffu);
  };
  for (int k0 = 0; k0 < K; k0 += 2 * KB) {
    Row16<T> v[4], u[4];
    load(k0, v);
    load(k0 + KB, u);
    largest4(v);
    largest4(u);
  }
#pragma unroll
  for (int e = 0; e < E; ++e) {
    for (int o = CL; o < 64; o <<= 1) m[e] = max(m[e], (uint32_t)__shfl_xor((int)m[e], o));
    if ((tid & 63) < CL) atomicMax(&big[E * cl + e], m[e]);
  }
  __syncthreads();
  float inv[E];
#pragma unroll
  for (int e = 0; e < E; ++e) {
    const QuantScale c = quant_scale(big[E * cl + e]);
    inv[e] = c.inv;
    if (r == 0 && f + e < F) sw[f + e] = c.s;
  }
  for (int k0 = 0; k0 < Kp; k0 += KB) {
    Row16<T> v[4];
    load(k0, v);
    __syncthreads();  // (the turn before is written)
#pragma unroll
    for (int e = 0; e < E; ++e) {
      float x[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) x[i] = k0 + 4 * r + i < K ? to_f<T>(v[i].v[e]) : 0.f;
      *reinterpret_cast<uint32_t*>(xs + (E * cl + e) * RB + 4 * r) = quant4(x[0], x[1], x[2], x[3], inv[e]);
    }
    __syncthreads();
    for (int c = tid; c < 64 * (KB / 16); c += 1024) {
      const int col = c / (KB / 16), k = 16 * (c % (KB / 16));
      if (f0 + col < F && k0 + k < Kp)
        *reinterpret_cast<uint4*>(q + (int64_t)(f0 + col) * Kp + k0 + k) =
            *reinterpret_cast<const uint4*>(xs + col * RB + k);
    }
  }
}

}  // namespace

namespace {
template <typename T, int WF, int WN, int MF, int MN, int NB>
hipError_t run_tiled(const I8Args& a, hipStream_t st) {
  using G = I8Geo<WF, WN, MF, MN, NB>;
  // a launch takes fewer than 2^32 threads: beyond them (2^30 rows at F = 1) the rows go in parts
  const int64_t ftiles = (a.F + G::TF - 1) / G::TF;
  const int64_t most = 0xffffffff / (64 * G::W) / ftiles * G::TN;
  hipError_t e = hipSuccess;
  for (int64_t n = 0; n < a.N && e == hipSuccess; n += most) {
    I8Args b = a;
    b.N = a.N - n < most ? a.N - n : most;
    b.q += n * a.Kp;
    b.s += n;
    if (a.C) b.C = reinterpret_cast<const T*>(a.C) + n * a.F;
    b.D = reinterpret_cast<T*>(a.D) + n * a.F;
    const dim3 grid((unsigned)((b.N + G::TN - 1) / G::TN * ftiles)), block(64 * G::W);
    if (a.act == PA_ACT_GELU)
      hipLaunchKernelGGL((k_gemm_i8<T, PA_ACT_GELU, WF, WN, MF, MN, NB>), grid, block, 0, st, b);
    else
      hipLaunchKernelGGL((k_gemm_i8<T, PA_ACT_NONE, WF, WN, MF, MN, NB>), grid, block, 0, st, b);
    e = hipGetLastError();
  }
  return e;
}
template <typename T>
hipError_t run_gemm(const I8Args& a, hipStream_t st) {
  // The tile that takes the least time, by a model of its measured ones (us): a block to
  // each CU takes `first` and, for a step of 128 of K, `step`; each further block of a CU
  // `more` and `more_step`.  (Within 10% of the best tile over N from 333 to 100,000, F
  // from 76 to 8188, K from 64 to 4096: 4096^3 65, 70 and 106 us with tiles of 256,
  // 128 and 64; 4096 x 256 to 4092 18, 14 and 24; 2000 x 1040 to 2001 27, 13 and 15;
  // 2000 x 4096 to 2001 60, 32 and 29.)
  const int steps = (a.Kp + 127) / 128;
  const auto cost = [&](int t, double first, double step, double more, double more_step) {
    const int64_t n = (a.N + t - 1) / t * ((a.F + t - 1) / t);
    return first + step * steps + (double)((n + 255) / 256 - 1) * (more + more_step * steps);
  };
  const double c256 = cost(256, 12.0, 1.45, 8.5, 1.6), c128 = cost(128, 5.5, 0.8, 1.4, 0.46),
               c64 = cost(64, 3.9, 0.27, 1.2, 0.14);
  const int want = c256 <= c128 && c256 <= c64 ? 256 : c128 <= c64 ? 128 : 64;
  if (want == 256) return run_tiled<T, 2, 4, 8, 4, 2>(a, st);
  if (want == 128) return run_tiled<T, 2, 2, 4, 4, 2>(a, st);
  return run_tiled<T, 2, 2, 2, 2, 4>(a, st);
}
}  // namespace

hipError_t launch_gemm_i8(const I8Args& a, int d_dtype, hipStream_t st) {
  if (a.N < 1 || a.F < 1 || a.Kp < 16) return hipErrorInvalidValue;
  return d_dtype == 1 ? run_gemm<bf16>(a, st) : run_gemm<float>(a, st);
}

namespace {
template <typename T, bool ODD>
hipError_t run_quant(int64_t N, int K, const T* x, int8_t* q, float* s, hipStream_t st) {
  const int Kp = (K + 15) / 16 * 16, CP = Kp / Row16<T>::E;
  int L = 1;
  while (L < CP && L < 64) L <<= 1;
  auto go = [&](auto* k, int U) {
    const int64_t rows = 256 / L * U, need = (N + rows - 1) / rows;
    hipLaunchKernelGGL(k, dim3((unsigned)(need < 4096 ? need : 4096)), dim3(256), 0, st, N, K, Kp, L,
                       x, q, s);
  };
  if (CP <= 64) go(k_quant_rows<T, ODD, 1, 4>, 4);
  else if (CP <= 128) go(k_quant_rows<T, ODD, 2, 2>, 2);
  else if (CP <= 256) go(k_quant_rows<T, ODD, 4, 1>, 1);
  else if (CP <= 512) go(k_quant_rows<T, ODD, 8, 1>, 1);
  else if (CP <= 1024) go(k_quant_rows<T, ODD, 16, 1>, 1);
  else
    hipLaunchKernelGGL((k_quant_long<T, ODD>), dim3((unsigned)(N < 4096 ? N : 4096)), dim3(512), 0, st,
                       N, K, Kp, x, q, s);
  return hipGetLastError();
}
template <typename T>
hipError_t run_quant(int64_t N, int K, const void* x, int8_t* q, float* s, hipStream_t st) {
  const T* p = reinterpret_cast<const T*>(x);
  if (K < Row16<T>::E) {
    const int64_t need = (N + 255) / 256;
    hipLaunchKernelGGL(k_quant_short<T>, dim3((unsigned)(need < 4096 ? need : 4096)), dim3(256), 0, st,
                       N, K, p, q, s);
    return hipGetLastError();
  }
  return K % Row16<T>::E ? run_quant<T, true>(N, K, p, q, s, st) : run_quant<T, false>(N, K, p, q, s, st);
}
}  // namespace

hipError_t launch_quant_rows(int64_t N, int K, int dtype, const void* x, int8_t* q, float* s,
                             hipStream_t st) {
  return dtype == 1 ? run_quant<bf16>(N, K, x, q, s, st) : run_quant<float>(N, K, x, q, s, st);
}

hipError_t launch_quant_weight(int K, int F, int dtype, const void* W, int8_t* Wq, float* sw,
                               hipStream_t st) {
  const int Kp = (K + 15) / 16 * 16;
  const dim3 grid((unsigned)((F + 63) / 64)), block(1024);
  auto go = [&](auto* k, auto* w) { hipLaunchKernelGGL(k, grid, block, 0, st, K, Kp, F, w, Wq, sw); };
  if (dtype == 1) {
    const bf16* w = (const bf16*)W;
    F % 8 ? go(k_quant_weight<bf16, false>, w) : go(k_quant_weight<bf16, true>, w);
  } else {
    const float* w = (const float*)W;
    F % 4 ? go(k_quant_weight<float, false>, w) : go(k_quant_weight<float, true>, w);
  }
  return hipGetLastError();
}

}  // namespace pa
