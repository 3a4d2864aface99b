// A linear layer in 8-bit integers on up to 16 rows (gfx950): one launch, bound by
// the weights' way from memory.
//
// A block of eight waves takes 16 output channels per KW waves, which share the
// contraction; every wave requests its weights (MFMA operands straight from
// memory, up to eight steps of 64 in flight) before anything else.  Meanwhile
// the block quantises all the rows into LDS, each by 512 / (N's next power of
// two) threads, which find its largest magnitude together.  The waves' integer
// sums (exact, so their order does not matter) meet in LDS.
#include "pa_i8.hpp"

namespace pa {
namespace {

constexpr int kFewRows = 16, kFewLds = 144 * 1024;

template <typename TX, typename TD, bool ODD>
__global__ void __launch_bounds__(512) k_linear_few(I8Args a, int KW, int G) {
  constexpr int E = Row16<TX>::E, U = 8, NOWHERE = 0x7fffff00;
  extern __shared__ __attribute__((aligned(16))) char xs[];  // [N][Kp + 16]
  __shared__ int red[8][16][16];
  __shared__ uint32_t big[kFewRows];
  __shared__ float ss[kFewRows];
  const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int lane = lane_id(), r = lane & 15, g = lane >> 4;
  const int N = (int)a.N, F = a.F, K = a.K, Kp = a.Kp, RB = Kp + 16;
  const int FB = 16 * (8 / KW), f0 = blockIdx.x * FB;

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
  // them in registers
  constexpr int H = 4;
  const int n = tid / G, tg = tid % G, CP = Kp / E;
  const bool mine = n < N;
  const TX* X = reinterpret_cast<const TX*>(a.x) + (int64_t)(mine ? n : 0) * K;
  if (tid < kFewRows) big[tid] = 0;
  Row16<TX> v[H];
#pragma unroll
  for (int j = 0; j < H; ++j) v[j] = row_chunk<ODD>(X, K, tg + j * G);
  __syncthreads();
  uint32_t m = 0;
#pragma unroll
  for (int j = 0; j < H; ++j) m = max(m, largest(v[j]));
  for (int c = tg + H * G; c < CP; c += G) m = max(m, largest(row_chunk<ODD>(X, K, c)));
  if (mine) atomicMax(&big[n], m);
  __syncthreads();
  if (mine) {
    const QuantScale q = quant_scale(big[n]);
    int8_t* row = reinterpret_cast<int8_t*>(xs) + n * RB;
#pragma unroll
    for (int j = 0; j < H; ++j)
      if (tg + j * G < CP) put_chunk(row + E * (tg + j * G), v[j], q.inv);
    for (int c = tg + H * G; c < CP; c += G) put_chunk(row + E * c, row_chunk<ODD>(X, K, c), q.inv);
    if (tg == 0) ss[n] = q.s;
  }
  __syncthreads();

  i32x4 acc = {0, 0, 0, 0};
  const char* xr = xs + (r < N ? r : N - 1) * RB;  // (columns past N are not used)
  auto product = [&](int s, i32x4 ws) {
    const int k = 64 * s + 16 * g;  // (behind a row's end the weights are zeros)
    const i32x4 x = *reinterpret_cast<const i32x4*>(xr + (k < Kp ? k : Kp - 16));
    acc = __builtin_amdgcn_mfma_i32_16x16x64_i8(ws, x, acc, 0, 0, 0);
  };
#pragma unroll
  for (int j = 0; j < U; ++j) product(s0 + j, w[j]);
  for (int s = s0 + U; s < s1; s += U) {
#pragma unroll
    for (int j = 0; j < U; ++j) w[j] = weight(s + j);
#pragma unroll
    for (int j = 0; j < U; ++j) product(s + j, w[j]);
  }
  *reinterpret_cast<i32x4*>(&red[wave][r][4 * g]) = acc;
  __syncthreads();
  for (int t = tid; t < N * FB; t += 512) {
    const int p = t / FB, fl = t % FB, f = f0 + fl;
    if (f >= F) continue;
    int sum = 0;
    for (int k = 0; k < KW; ++k) sum += red[fl / 16 * KW + k][p][fl % 16];
    float u = fmaf((float)sum, ss[p] * a.sw[f], a.bias ? a.bias[f] : 0.f);
    if (a.act == PA_ACT_GELU) u = gelu_for<TD>(u);
    const int64_t at = (int64_t)p * F + f;
    if (a.C) u += to_f<TD>(reinterpret_cast<const TD*>(a.C)[at]);
    reinterpret_cast<TD*>(a.D)[at] = from_f<TD>(u);
  }
}

template <typename TX, typename TD>
hipError_t run(const I8Args& a, hipStream_t st) {
  const int steps = (a.Kp + 63) / 64;
  int KW = 1, NP = 1;
  while (KW < 8 && 2 * KW <= steps) KW *= 2;
  while (NP < a.N) NP *= 2;
  const int FB = 16 * (8 / KW);
  const size_t lds = (size_t)a.N * (a.Kp + 16);
  const dim3 grid((a.F + FB - 1) / FB), block(512);
  if (a.K % Row16<TX>::E)
    hipLaunchKernelGGL((k_linear_few<TX, TD, true>), grid, block, lds, st, a, KW, 512 / NP);
  else
    hipLaunchKernelGGL((k_linear_few<TX, TD, false>), grid, block, lds, st, a, KW, 512 / NP);
  return hipGetLastError();
}

}  // namespace

bool linear_i8_few(int64_t N, int K) {
  return N <= kFewRows && N * ((K + 15) / 16 * 16 + 16) <= kFewLds;
}

hipError_t launch_linear_few(const I8Args& a, int d_dtype, hipStream_t st) {
  if (a.x_dtype == 1) return d_dtype == 1 ? run<bf16, bf16>(a, st) : run<bf16, float>(a, st);
  return d_dtype == 1 ? run<float, bf16>(a, st) : run<float, float>(a, st);
}

}  // namespace pa
