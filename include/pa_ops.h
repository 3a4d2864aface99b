/*
 * pa_ops.h -- operators around the block stack of pa.h, in the same library
 * (libpa.so) and under the conventions that pa.h states for its calls: device
 * pointers owned by the caller, row-major, contiguous and 16-byte aligned
 * (fp32 vectors of block scales: 4-byte); asynchronous on `stream`, whose
 * device has to be the current one; nothing is allocated, freed or
 * synchronised, so every call may be captured into a HIP graph; the host
 * validates the arguments before anything is launched (PA_ERR_INVALID,
 * PA_ERR_UNSUPPORTED, PA_ERR_WORKSPACE, pa_last_error()); results are
 * deterministic; outputs and workspaces must not overlap inputs or each other
 * unless said otherwise (PA_ERR_INVALID); a workspace belongs to one call at a
 * time (calls on two streams, or in two graphs that may run together, need one
 * each).
 *
 *   pa_residual_norm   the joint between a block and the next one: a norm
 *                      after the block, its gate and residual scale, the
 *                      residual add, the norm before the next block; and its
 *                      backward
 *   pa_adamw           one AdamW step over many tensors, moments in 32 or 8
 *                      bits
 *   pa_linear_i8       a linear layer in 8-bit integers with scales per row
 *                      (token) and per output channel
 */
#ifndef PA_OPS_H
#define PA_OPS_H

#include "pa.h"

#ifdef __cplusplus
extern "C" {
#endif

#define PA_OPS_VERSION 1
int pa_ops_version(void);

/* ---------------------------------------------------------------------
 * The joint between two blocks.  For every row i of x, y [N,C]:
 *   u  = post(y)                   post: nothing, LayerNorm or RMSNorm
 *   m  = t, sigmoid(t), or 1 without t
 *   x1 = alpha x + scale m u       rounded to dtype, written
 *   h  = pre(x1)                   of the rounded x1
 * with LayerNorm(z) = (z - mean) / sqrt(var + eps) g + b (biased variance)
 * and RMSNorm(z) = z / sqrt(mean(z^2) + eps) g + b, over the C channels.
 * post_g, post_b, pre_g, pre_b and scale are [C] fp32, each nullable (1, 0,
 * 1, 0, 1); t [N,C] dtype, nullable.  C a multiple of 8 in [16, 8192] (bf16)
 * or [16, 4096] (fp32).  Sums are fp32, the squares' deviations from the
 * row's own mean.  A row's statistics are not kept: the backward forms them
 * again from y and x1, which it reads anyway.
 * --------------------------------------------------------------------- */
typedef enum { PA_NORM_NONE = 0, PA_NORM_LAYER = 1, PA_NORM_RMS = 2 } pa_norm;
typedef enum { PA_GATE_LINEAR = 0, PA_GATE_SIGMOID = 1 } pa_gate;

typedef struct {
  int32_t post, pre;         /* pa_norm                                        */
  int32_t gate;              /* pa_gate: how t becomes the gate (with t only)  */
  float post_eps, pre_eps;   /* > 0 (unused without the norm)                  */
  float alpha;               /* scale of the residual stream                   */
  const float *post_g, *post_b;
  const float* scale;
  const float *pre_g, *pre_b;
} pa_residual_norm_params;

/* x1 [N,C] dtype and, with a pre norm, h [N,C] dtype and / or h in 8-bit
 * integers with a scale per row, as pa_quant_rows would form them from the
 * unrounded h: hq [N,Kp] int8 (Kp = C rounded up to 16, the rest zeros), hs
 * [N] fp32.  h, hq and hs nullable (hq and hs together); without a pre norm
 * all are NULL. */
pa_status pa_residual_norm(int64_t N, int C, pa_dtype dtype, const pa_residual_norm_params* p,
                           const void* x, const void* y, const void* t, void* x1, void* h,
                           int8_t* hq, float* hs, void* stream);

/* Gradients of the parameters, fp32 [C], each nullable.  Sums over the rows
 * as partial sums per block, added in block order. */
typedef struct {
  float *dpost_g, *dpost_b;  /* written with a post norm only */
  float* dscale;
  float *dpre_g, *dpre_b;    /* written with a pre norm only  */
} pa_residual_norm_grads;

/* Chain rule, from the gradients dx1 (x1 in the residual stream) and dh, both
 * [N,C] dtype; either may be NULL (0), not both; dh needs a pre norm:
 *   e  = dx1 + pre'(dh; x1),   dx = alpha e,   dy = post'(scale m e; y),
 *   dt = scale e u m'(t)
 * dx, dy and, with t, dt [N,C] dtype; *gr nullable.  Workspace for the
 * parameters' gradients: pa_residual_norm_workspace bytes (0 without). */
pa_status pa_residual_norm_backward(int64_t N, int C, pa_dtype dtype,
                                    const pa_residual_norm_params* p, const void* x1,
                                    const void* y, const void* t, const void* dx1,
                                    const void* dh, void* dx, void* dy, void* dt,
                                    const pa_residual_norm_grads* gr, void* ws, size_t ws_bytes,
                                    void* stream);
pa_status pa_residual_norm_workspace(int64_t N, int C, pa_dtype dtype, size_t* bytes);

/* ---------------------------------------------------------------------
 * AdamW over many tensors:
 *   g  = gscale gradient
 *   m <- b1 m + (1 - b1) g,   v <- b2 v + (1 - b2) g^2
 *   p <- p - (lr wd p + lr / (1 - b1^step) m / (sqrt(v) / sqrt(1 - b2^step) + eps))
 * in fp32, every product and sum of m and v rounded to nearest (no fused
 * multiply-add), so that the moments can be reproduced bit for bit.
 *
 * Moments in 8 bits (m_scale and v_scale given): m and v are [n] bytes, with
 * a scale per block of 256 consecutive elements ([ceil(n / 256)] fp32).  S is
 * the smallest power of two not below the block's largest magnitude (at least
 * 2^-126, at most 2^127; 0 for a block of zeros; NaN for a block with an
 * infinity or NaN).  A code c > 0 stands for S times the fp32 number whose
 * upper 12 bits are c + 889 (m: c the code's lower 7 bits, bit 7 the sign) or
 * c + 761 (v: all 8), c = 0 for 0: steps of 1/8 within an octave, 16 and 32
 * octaves.  A moment is coded by adding 16 h + 8 to the bits of its magnitude
 * over S, h 16 random bits, and dropping the lower 20: an unbiased rounding.
 * (Rounded to nearest, v would stand still: at b2 = 0.999 a step moves it by
 * less than half a code.)  Below the last code m becomes 0, a positive v the
 * last code, so that no parameter is divided by a v that was lost.  The random
 * bits, in 32-bit arithmetic: with A. Appleby's published finaliser
 *   f(h): h ^= h >> 16, h *= 0x85EBCA6B, h ^= h >> 13, h *= 0xC2B2AE35, h ^= h >> 16
 * and mix(a, b) = f(a ^ (b 0x9E3779B9)), element j of block k of the call's
 * tensor i takes r = f(mix(mix(mix(mix(seed, seed >> 32), step), i), k) + j),
 * the lower half for m, the upper half for v.  Zeroed codes and scales are zero
 * moments.
 * --------------------------------------------------------------------- */
typedef struct {
  int64_t n;             /* elements, >= 0 (0: skipped), at most 2^36          */
  float* p;              /* the parameters, updated in place                   */
  void* copy;            /* nullable: p rounded to bf16, written               */
  const void* g;         /* the gradient, g_dtype                              */
  void *m, *v;           /* the moments, updated in place: fp32, or codes      */
  float *m_scale, *v_scale; /* both NULL: fp32 moments                         */
  float wd;              /* weight decay of this tensor                        */
  int32_t g_dtype;       /* pa_dtype                                           */
} pa_adamw_item;

typedef struct {
  double lr, beta1, beta2, eps;  /* betas in [0, 1), eps a normal fp32 > 0      */
  int64_t step;                  /* of this update, from 1                     */
  uint64_t seed;                 /* of the 8-bit moments' rounding             */
  const float* gscale;           /* nullable device scalar (1): clipping       */
  /* For a captured graph, whose host values stand still: nullable device
   * scalars, read when the step runs, in place of lr and step. */
  const float* lr_dev;
  const int64_t* step_dev;
} pa_adamw_args;

/* items is a host array, read before the call returns.  The tensors of one
 * call must not overlap: whatever is written (p, copy, m, v and the scales) is
 * checked; gradients may be shared. */
pa_status pa_adamw(int n_items, const pa_adamw_item* items, const pa_adamw_args* args,
                   void* stream);

/* The same step over a table that a program keeps where its tensors stay where
 * they are: one launch however many tensors there are, and nothing to check or
 * copy per step.  pa_adamw_table_size: the table's bytes and its blocks;
 * pa_adamw_table fills `host` (host memory, 8-byte aligned) with it, which the
 * caller copies to the device, `table` of pa_adamw_run, and fills anew when a
 * tensor (a gradient, too) moves.  Both make pa_adamw's checks of the items;
 * pa_adamw_run takes the table on trust.  Same results, bit for bit. */
pa_status pa_adamw_table_size(int n_items, const pa_adamw_item* items, size_t* bytes,
                              int64_t* blocks);
pa_status pa_adamw_table(int n_items, const pa_adamw_item* items, void* host, size_t bytes);
pa_status pa_adamw_run(int n_items, int64_t blocks, const void* table, const pa_adamw_args* args,
                       void* stream);

/* The values that n codes stand for: out [n] fp32 (is_signed = 1: m's codes,
 * 0: v's). */
pa_status pa_adamw_unpack(int64_t n, const void* codes, const float* scales, int is_signed,
                          float* out, void* stream);

/* ---------------------------------------------------------------------
 * Products in 8-bit integers with scales per row (token) and output channel.
 * Rows of int8 matrices are Kp = K rounded up to 16 bytes apart and end in
 * zeros.  K in [1, 131072] (the sum of K products of integers up to 127 fits
 * 32 bits: exact), F >= 1, N >= 1, any sizes.
 * --------------------------------------------------------------------- */

/* q_ik = round-to-even(x_ik (127 / max_k |x_ik|)), the quotient and the
 * product in fp32, s_i = max / 127: q [N,Kp] int8, s [N] fp32 from x [N,K].  A row
 * whose largest magnitude is below 1e-36 has q = 0, s = 0; one with an
 * infinity or NaN q = 0, s = NaN, which the product passes on. */
pa_status pa_quant_rows(int64_t N, int K, pa_dtype dtype, const void* x, int8_t* q, float* s,
                        void* stream);

/* Weights, once: W [K,F] in the x W layout of pa.h -> Wq [F,Kp] int8 with a
 * scale sw [F] per output channel, each column quantised as a row above. */
pa_status pa_quant_weight(int K, int F, pa_dtype dtype, const void* W, int8_t* Wq, float* sw,
                          void* stream);

typedef enum { PA_ACT_NONE = 0, PA_ACT_GELU = 1 } pa_act;

/* D [N,F] (d_dtype) = act(s_i sw_f sum_k q_ik Wq_fk + bias_f) + C_if; bias
 * [F] fp32 and C [N,F] d_dtype nullable; GELU(u) = u Phi(u) on the fp32 value,
 * to within 2e-6 of it, or 2e-10 (bf16 results: 1e-4, or 2e-7, before rounding).
 * D may be C (the residual stream updated in place). */
pa_status pa_gemm_i8(int64_t N, int F, int K, const int8_t* q, const float* s, const int8_t* Wq,
                     const float* sw, const float* bias, pa_act act, const void* C, void* D,
                     pa_dtype d_dtype, void* stream);

/* pa_quant_rows and pa_gemm_i8, the rows quantised into the workspace or, where
 * that is faster, inside of the product, in one launch: x [N,K] x_dtype; ws at
 * least pa_linear_i8_workspace bytes. */
pa_status pa_linear_i8(int64_t N, int F, int K, const void* x, pa_dtype x_dtype,
                       const int8_t* Wq, const float* sw, const float* bias, pa_act act,
                       const void* C, void* D, pa_dtype d_dtype, void* ws, size_t ws_bytes,
                       void* stream);
pa_status pa_linear_i8_workspace(int64_t N, int F, int K, size_t* bytes);

#ifdef __cplusplus
}
#endif
#endif /* PA_OPS_H */
