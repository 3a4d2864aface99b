// A linear layer in 8-bit integers on few rows, or where one round of blocks does it
// (gfx950): one launch, bound by latency and the weights' way from memory.
//
// A block of eight waves takes up to 16 or 32 rows and 16 output channels per KW
// waves, which share the contraction; every wave requests its weights (MFMA
// operands straight from memory, up to eight steps of 64 in flight) before anything
// else.  Meanwhile the block quantises its rows into LDS, each by 512 / (the rows'
// next power of two) threads, which find its largest magnitude together.  The
// waves' integer sums (exact, so their order does not matter) meet in LDS.
//
// With more rows than 16 every block of channels quantises them again, which costs
// less than a second launch while all the blocks run at once.  Measured, the least of
// some, us, as two launches (quantiser, tiles) and as one: 333 rows of 1000 to 517 fp32 8.3 and
// 6.7; bf16 32 rows of 1024 to 4096 7.9 and 5.8, 333 of 256 to 517 7.8 and 5.5, 1024
// of 1024 to 256 8.8 and 6.6, 512 of 4096 to 256 15.4 and 13.2.  Medians of 60 in a row:
// these 7.3, 6.4, 5.8, 7.1 and 14.5; one row of 4096 to 4096 5.9 us (16.8 MB of
// weights, from the last cache in these figures), 2 of them 6.3, 16 10.1, 16 of 1024 to
// 4096 5.4.
#include "pa_i8.hpp"

namespace pa {
namespace {

constexpr int kFewRows = 16;

// Bytes between rows in LDS: an odd number of 16-byte chunks, so that the 16 rows
// of an operand read lie in different banks.
__host__ __device__ constexpr int row_bytes(int Kp) { return Kp % 32 ? Kp : Kp + 16; }

// RT: tiles of 16 rows that a block takes.
template <int RT> struct FewGeo {
  static constexpr int ROWS = kFewRows * RT;
  static constexpr int OWN = 8 * ROWS * 64 + 8 * ROWS + 1024 + 256;  // LDS beside the rows
};

// H: a thread's chunks of a row in flight.
template <typename TX, typename TD, bool ODD, int RT, int H>
__global__ void __launch_bounds__(512) k_linear_few(I8Args a, int KW, int G, int rows_first) {
  constexpr int E = Row16<TX>::E, U = 8, NOWHERE = 0x7fffff00;
  constexpr int ROWS = FewGeo<RT>::ROWS;
  extern __shared__ __attribute__((aligned(16))) char xs[];  // [N][RB]
  __shared__ __attribute__((aligned(16))) int red[8][ROWS][16];
  __shared__ uint32_t big[ROWS];
  __shared__ float ss[ROWS], sws[128], bs[128];
  const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int lane = lane_id(), r = lane & 15, g = lane >> 4;
  const int64_t n0 = (int64_t)(rows_first ? blockIdx.x : blockIdx.y) * ROWS;
  const int N = (int)(a.N - n0 < ROWS ? a.N - n0 : ROWS);  // the block's rows
  const int F = a.F, K = a.K, Kp = a.Kp, RB = row_bytes(Kp);
  const int FB = 16 * (8 / KW), f0 = (rows_first ? blockIdx.y : blockIdx.x) * FB;

  // the wave's weights: channel f0 + 16 (wave / KW) + r, steps [s0, s1)
  const int steps = (Kp + 63) / 64, per = (steps + KW - 1) / KW;
  const int s0 = wave % KW * per, s1 = s0 + per < steps ? s0 + per : steps;
  const auto rw = __builtin_amdgcn_make_buffer_rsrc(
      const_cast<int8_t*>(a.w) + (int64_t)f0 * Kp, 0, (F - f0 < FB ? F - f0 : FB) * Kp, 0x00027000);
  const int fr = 16 * (wave / KW) + r;
  auto weight = [&](int s) {  // zeros behind the wave's steps, a row's end and the last channel
    const int k = 64 * s + 16 * g;
    return __builtin_bit_cast(i32x4, __builtin_amdgcn_raw_buffer_load_b128(
                                         rw, s < s1 && k < Kp ? fr * Kp + k : NOWHERE, 0, 0));
  };
  i32x4 w[U];
#pragma unroll
  for (int j = 0; j < U; ++j) w[j] = weight(s0 + j);

  // the rows: G threads each, chunk c of E channels by thread c % G, the first H of
  // them kept in registers, the others in turns of H
  const int n = tid / G, tg = tid % G, CP = Kp / E;
  const bool mine = n < N;
  const TX* X = reinterpret_cast<const TX*>(a.x) + (n0 + (mine ? n : 0)) * K;
  if (tid < ROWS) big[tid] = 0;
  if (tid < FB) {
    const int f = f0 + tid < F ? f0 + tid : F - 1;
    sws[tid] = a.sw[f];
    bs[tid] = a.bias ? a.bias[f] : 0.f;
  }
  auto fetch = [&](int c0, Row16<TX>(&v)[H]) __attribute__((always_inline)) {
#pragma unroll
    for (int j = 0; j < H; ++j) v[j] = row_chunk<ODD>(X, K, c0 + tg + j * G);
  };
  Row16<TX> v[H];
  fetch(0, v);
  __syncthreads();
  uint32_t m = 0;
#pragma unroll
  for (int j = 0; j < H; ++j) m = max(m, largest(v[j]));
  for (int c = H * G; c < CP; c += H * G) {
    Row16<TX> u[H];
    fetch(c, u);
#pragma unroll
    for (int j = 0; j < H; ++j) m = max(m, largest(u[j]));
  }
  if (mine) atomicMax(&big[n], m);
  __syncthreads();
  if (mine) {
    const QuantScale q = quant_scale(big[n]);
    int8_t* row = reinterpret_cast<int8_t*>(xs) + n * RB;
    auto put = [&](int c0, const Row16<TX>(&v)[H]) __attribute__((always_inline)) {
#pragma unroll
      for (int j = 0; j < H; ++j) {
        const int c = c0 + tg + j * G;
        if (c < CP) put_chunk<ODD>(row + E * c, v[j], q.inv, K, c);
      }
    };
    put(0, v);
    for (int c = H * G; c < CP; c += H * G) {
      Row16<TX> u[H];
      fetch(c, u);
      put(c, u);
    }
    if (tg == 0) ss[n] = q.s;
  }
  __syncthreads();

  i32x4 acc[RT];
  const char* xr[RT];
#pragma unroll
  for (int t = 0; t < RT; ++t) {
    acc[t] = i32x4{0, 0, 0, 0};
    const int p = 16 * t + r;  // (columns past N are not used)
    xr[t] = xs + (p < N ? p : N - 1) * RB;
  }
  auto product = [&](int s, i32x4 ws) {
    const int k = 64 * s + 16 * g, at = k < Kp ? k : Kp - 16;  // (behind a row's end the weights are zeros)
#pragma unroll
    for (int t = 0; t < RT; ++t) {
      const i32x4 x = *reinterpret_cast<const i32x4*>(xr[t] + at);
      acc[t] = __builtin_amdgcn_mfma_i32_16x16x64_i8(ws, x, acc[t], 0, 0, 0);
    }
  };
#pragma unroll
  for (int j = 0; j < U; ++j) product(s0 + j, w[j]);
  for (int s = s0 + U; s < s1; s += U) {
#pragma unroll
    for (int j = 0; j < U; ++j) w[j] = weight(s + j);
#pragma unroll
    for (int j = 0; j < U; ++j) product(s + j, w[j]);
  }
#pragma unroll
  for (int t = 0; t < RT; ++t) *reinterpret_cast<i32x4*>(&red[wave][16 * t + r][4 * g]) = acc[t];
  __syncthreads();
  for (int t = tid; t < N * FB; t += 512) {
    const int p = t / FB, fl = t % FB, f = f0 + fl;
    if (f >= F) continue;
    int sum = 0;
    for (int k = 0; k < KW; ++k) sum += red[fl / 16 * KW + k][p][fl % 16];
    float u = fmaf((float)sum, ss[p] * sws[fl], bs[fl]);
    if (a.act == PA_ACT_GELU) u = gelu_for<TD>(u);
    const int64_t at = (n0 + p) * F + f;
    if (a.C) u += to_f<TD>(reinterpret_cast<const TD*>(a.C)[at]);
    reinterpret_cast<TD*>(a.D)[at] = from_f<TD>(u);
  }
}

// The waves that share a contraction; 0: not served.  Beyond 16 rows: as many as let
// all the blocks run at once (a block takes a CU), if each wave's weights fit its
// registers; and rows short enough to be read again by every block of channels (us,
// two launches and one: bf16 32 rows of 4096 to 1024 13.7 and 12.2; fp32 of 2048 to
// 1024 9.4 and 10.0, of 4096 13.9 and 15.8; bf16 128 of 3695, whose rows are not aligned, to
// 1500 14.8 and 16.5), longer than 2 KB only where few
// channels to a block make up for it (fp32 512 rows of 1024 to 1024 8.2 and, at KW =
// 2, 8.6).
template <int RT> int few_split(int64_t N, int F, int K, int x_dtype) {
  constexpr int ROWS = FewGeo<RT>::ROWS;
  const int Kp = (K + 15) / 16 * 16, steps = (Kp + 63) / 64, E = x_dtype == 1 ? 8 : 4;
  const int64_t rows = N < ROWS ? N : ROWS, nb = (N + ROWS - 1) / ROWS;
  if (K < E || rows * row_bytes(Kp) + FewGeo<RT>::OWN > 160 * 1024) return 0;
  int KW = 8;
  // (waves without a step cost nothing while there are CUs for the blocks)
  while (KW && nb * ((F + 128 / KW - 1) / (128 / KW)) > 256 && (RT == 2 || KW > steps)) KW /= 2;
  if (RT == 1) return KW;
  const int bytes = x_dtype == 1 ? 2 * K : 4 * K;
  return 8 * KW < steps || bytes > (x_dtype == 1 && K % 8 == 0 ? 8192 : 4096) || (bytes > 2048 && KW < 4) ? 0 : KW;
}

template <typename TX, typename TD, int RT, int H>
hipError_t run(const I8Args& a, hipStream_t st) {
  constexpr int ROWS = FewGeo<RT>::ROWS;
  const int rows = a.N < ROWS ? (int)a.N : ROWS, KW = few_split<RT>(a.N, a.F, a.K, a.x_dtype);
  if (!KW) return hipErrorInvalidValue;
  int NP = 1;
  while (NP < rows) NP *= 2;
  const int FB = 128 / KW;
  const size_t lds = (size_t)rows * row_bytes(a.Kp);
  // Blocks are dealt to the XCDs round robin: those with the larger operand in common
  // a multiple of the other count apart, in one L2.
  const unsigned nf = (a.F + FB - 1) / FB, nb = (unsigned)((a.N + ROWS - 1) / ROWS);
  const int rows_first = a.N * (int64_t)sizeof(TX) > a.F && nf <= 65535;
  const dim3 grid(rows_first ? nb : nf, rows_first ? nf : nb), block(512);
  if (a.K % Row16<TX>::E)
    hipLaunchKernelGGL((k_linear_few<TX, TD, true, RT, H>), grid, block, lds, st, a, KW, 512 / NP,
                       rows_first);
  else
    hipLaunchKernelGGL((k_linear_few<TX, TD, false, RT, H>), grid, block, lds, st, a, KW, 512 / NP,
                       rows_first);
  return hipGetLastError();
}
template <typename TX, typename TD>
hipError_t by_rows(const I8Args& a, hipStream_t st) {
  if (a.N <= kFewRows) return run<TX, TD, 1, 4>(a, st);
  // (32 rows have 16 threads each, to which 8 chunks are 2 KB of a row and 16 are 4; us, 333
  // rows to 517 with 8 and 16: 1000 fp32 7.5 and 6.7, 1542 bf16 9.0 and 7.9; to 64, 3000
  // bf16 9.7 and 11.0)
  const int bytes = a.K * (int)sizeof(TX);
  return bytes > 2048 && bytes <= 4096 ? run<TX, TD, 2, 16>(a, st) : run<TX, TD, 2, 8>(a, st);
}

}  // namespace

bool linear_i8_few(int64_t N, int F, int K, int x_dtype) {
  return (N <= kFewRows ? few_split<1>(N, F, K, x_dtype) : few_split<2>(N, F, K, x_dtype)) > 0;
}

hipError_t launch_linear_few(const I8Args& a, int d_dtype, hipStream_t st) {
  if (a.x_dtype == 1) return d_dtype == 1 ? by_rows<bf16, bf16>(a, st) : by_rows<bf16, float>(a, st);
  return d_dtype == 1 ? by_rows<float, bf16>(a, st) : by_rows<float, float>(a, st);
}

}  // namespace pa
