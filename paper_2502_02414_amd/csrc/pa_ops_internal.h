// Internal launch interface of the operators of include/pa_ops.h, between
// pa_ops_api.cpp and the kernels (pa_resnorm.hip, pa_adamw.hip, pa_i8.hip).
#pragma once

#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include "pa_ops.h"

namespace pa {

// ---- the joint between two blocks (pa_resnorm.hip) ----
struct ResNormArgs {
  int64_t N = 0;
  int C = 0, L = 0;  // L: lanes per row (set by the launch)
  int post = 0, pre = 0, gate = 0;
  float post_eps = 0.f, pre_eps = 0.f, alpha = 1.f;
  const float *post_g = nullptr, *post_b = nullptr, *scale = nullptr;
  const float *pre_g = nullptr, *pre_b = nullptr;
  const void *x = nullptr, *y = nullptr, *t = nullptr;
  void *x1 = nullptr, *h = nullptr;  // (x1: read by the backward)
  int8_t* hq = nullptr;
  float* hs = nullptr;
  const void *dx1 = nullptr, *dh = nullptr;
  void *dx = nullptr, *dy = nullptr, *dt = nullptr;
  float* partials = nullptr;  // resnorm_blocks records [5][C], nullable
  // one block: the gradients that the record is for, in its place, each nullable
  float *g0 = nullptr, *g1 = nullptr, *g2 = nullptr, *g3 = nullptr, *g4 = nullptr;
};
int resnorm_blocks(int64_t N, int C, int dtype, bool bwd);
hipError_t launch_resnorm(const ResNormArgs& a, int dtype, bool bwd, hipStream_t st);

// ---- AdamW (pa_adamw.hip) ----
struct AdamItem {
  float* p;
  void* copy;
  const void* g;
  void *m, *v;
  float *ms, *vs;
  int64_t n;
  float wd;
  uint32_t bits;  // 1: bf16 gradient, 2: 8-bit moments
};
// What all tensors of a step have in common.
struct AdamStep {
  double lr, beta1, beta2;
  const float* gscale;
  const float* lr_dev;
  const int64_t* step_dev;
  int64_t step;
  float ss, rs;               // adam_consts of lr and step
  uint32_t seed_key, step_key;  // mix(seed, seed >> 32), mix(that, step)
  float b1, b2, c1, c2, eps;  // c = 1 - b
};
// Tensors in a launch's arguments, at most kAdamMax; first[i]: the launch's first
// block that works on item i.
constexpr int kAdamMax = 52;
struct AdamBatch {
  AdamStep s;
  int n, base;  // items; the index of item 0 in the call
  uint32_t first[kAdamMax + 1];
  AdamItem it[kAdamMax];
};
static_assert(sizeof(AdamBatch) <= 4096, "a launch's arguments");
// Tensors in a table in device memory: the entries, then the entry of each block.
struct AdamEntry {
  AdamItem it;
  uint32_t first;  // the first block that works on it
  uint32_t index;  // in the call's list
};
hipError_t launch_adamw_table(const AdamStep& s, const AdamEntry* entries, const uint32_t* map,
                              uint32_t blocks, hipStream_t st);
void adam_consts(double lr, double b1, double b2, int64_t step, float* ss, float* rs);
uint32_t adam_mix(uint32_t a, uint32_t b);
uint32_t adam_blocks(int64_t n);  // blocks that an item of n elements takes
hipError_t launch_adamw(const AdamBatch& b, hipStream_t st);
hipError_t launch_adam_unpack(int64_t n, const uint8_t* codes, const float* scales, bool sgn,
                              float* out, hipStream_t st);

// ---- 8-bit integer products (pa_i8.hip) ----
struct I8Args {
  int64_t N = 0;
  int F = 0, K = 0, Kp = 0;
  const int8_t* q = nullptr;   // [N,Kp]
  const float* s = nullptr;    // [N]
  const void* x = nullptr;     // [N,K] x_dtype: rows that the product quantises itself
  int x_dtype = 0;
  const int8_t* w = nullptr;   // [F,Kp]
  const float* sw = nullptr;   // [F]
  const float* bias = nullptr;
  int act = 0;
  const void* C = nullptr;
  void* D = nullptr;
};
hipError_t launch_gemm_i8(const I8Args& a, int d_dtype, hipStream_t st);
// Products of many rows that keep their weights in registers (pa_i8_fused.hip; bf16
// results), of integers, or of bf16 rows that they quantise: served, and faster
// than the tiles.
bool linear_i8_fused(int64_t N, int F, int K);
hipError_t launch_linear_i8(const I8Args& a, hipStream_t st);
// Few rows, or few blocks (pa_i8_few.hip): served.
bool linear_i8_few(int64_t N, int F, int K, int x_dtype);
hipError_t launch_linear_few(const I8Args& a, int d_dtype, hipStream_t st);
hipError_t launch_quant_rows(int64_t N, int K, int dtype, const void* x, int8_t* q, float* s,
                             hipStream_t st);
hipError_t launch_quant_weight(int K, int F, int dtype, const void* W, int8_t* Wq, float* sw,
                               hipStream_t st);

#ifdef __HIPCC__
// A row's scale from the bits of its largest magnitude (as integers, so that
// an infinity or a NaN comes out on top): q = rne(x inv), s = max / 127.  Rows
// below 1e-36, whose 127 / max nears the end of fp32, are zeros.
struct QuantScale {
  float inv, s;
};
__device__ __forceinline__ QuantScale quant_scale(uint32_t big) {
  const float m = __builtin_bit_cast(float, big);
  const bool zero = m < 1e-36f, bad = big >= 0x7f800000u;
  const float inv = __fdiv_rn(127.f, m), s = __fdiv_rn(m, 127.f);
  return {zero || bad ? 0.f : inv, bad ? __builtin_nanf("") : zero ? 0.f : s};
}
// Four integers of a row in one word.  |x inv| <= 127 (1 + 2^-23): rounded to
// even they stay within +-127; 1.5 2^23 added leaves the integer in the lowest
// bits.  inv = 0 (zeros, or a row that is not finite): zeros.
__device__ __forceinline__ uint32_t quant4(float a, float b, float c, float d, float inv) {
  const float v[4] = {a, b, c, d};
  uint32_t t[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
#pragma clang fp contract(off)
    t[i] = __builtin_bit_cast(uint32_t, v[i] * inv + 12582912.f);
  }
  const uint32_t lo = __builtin_amdgcn_perm(t[1], t[0], 0x0c0c0400u);
  const uint32_t hi = __builtin_amdgcn_perm(t[3], t[2], 0x04000c0cu);
  return inv == 0.f ? 0u : lo | hi;
}
#endif

}  // namespace pa
