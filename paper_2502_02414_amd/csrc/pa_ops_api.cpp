// C ABI of include/pa_ops.h: host-side validation and launches.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cfloat>
#include <cmath>
#include <cstdarg>
#include <cstdio>
#include <new>
#include <vector>

#include "pa_ask_split.hpp"
#include "pa_internal.h"
#include "pa_ops_internal.h"

namespace {

pa_status err(pa_status s, const char* fmt, ...) __attribute__((format(printf, 2, 3)));
pa_status err(pa_status s, const char* fmt, ...) {
  char buf[512];
  va_list ap;
  va_start(ap, fmt);
  vsnprintf(buf, sizeof buf, fmt, ap);
  va_end(ap);
  pa::set_last_error(buf);
  return s;
}

#define PO_HIP(call, what)                                                               \
  do {                                                                                   \
    hipError_t e_ = (call);                                                              \
    if (e_ != hipSuccess) return err(PA_ERR_HIP, "%s: %s", what, hipGetErrorString(e_)); \
  } while (0)
#define PO_TRY(x)               \
  do {                          \
    pa_status s_ = (x);         \
    if (s_ != PA_OK) return s_; \
  } while (0)

hipStream_t as_stream(void* s) { return reinterpret_cast<hipStream_t>(s); }

pa_status opt(const char* who, const void* p, const char* name, unsigned align = 16) {
  if (p && ((uintptr_t)p & (align - 1)))
    return err(PA_ERR_INVALID, "%s: %s is not %u-byte aligned", who, name, align);
  return PA_OK;
}
pa_status need(const char* who, const void* p, const char* name, unsigned align = 16) {
  if (!p) return err(PA_ERR_INVALID, "%s: %s is NULL", who, name);
  return opt(who, p, name, align);
}
pa_status dtype_ok(const char* who, int dt) {
  return dt == PA_F32 || dt == PA_BF16
             ? PA_OK
             : err(PA_ERR_INVALID, "%s: dtype must be PA_F32 or PA_BF16", who);
}

// Memory of one tensor of a call (without a pointer or bytes: none).
struct Span {
  const char* name;
  const void* p;
  uint64_t bytes;
};
// Every output apart from the inputs and from the other outputs: kernels read rows
// ahead of those that they write, and again (a row past the end is the last one).
template <size_t NO, size_t NI>
pa_status apart(const char* who, const Span (&out)[NO], const Span (&in)[NI]) {
  const auto meet = [](const Span& a, const Span& b) {
    const uintptr_t x = (uintptr_t)a.p, y = (uintptr_t)b.p;
    return a.p && b.p && x < y + b.bytes && y < x + a.bytes;
  };
  for (size_t i = 0; i < NO; ++i) {
    for (size_t j = i + 1; j < NO; ++j)
      if (meet(out[i], out[j]))
        return err(PA_ERR_INVALID, "%s: %s and %s overlap", who, out[i].name, out[j].name);
    for (const Span& s : in)
      if (meet(out[i], s)) return err(PA_ERR_INVALID, "%s: %s and %s overlap", who, out[i].name, s.name);
  }
  return PA_OK;
}
uint64_t dtype_bytes(int dt) { return dt == PA_BF16 ? 2 : 4; }

// Rows of one tensor of a call: `width` bytes, `pitch` from one to the next.
struct Rows {
  const char* name;
  const void* p;
  uint64_t rows, width, pitch;
};
bool rows_meet(const Rows& a, const Rows& b) {
  if (!a.p || !b.p || !a.rows || !b.rows) return false;
  const uintptr_t x = (uintptr_t)a.p, y = (uintptr_t)b.p;
  if (x >= y + (b.rows - 1) * b.pitch + b.width || y >= x + (a.rows - 1) * a.pitch + a.width)
    return false;
  // side by side in rows of one pitch: b's columns from a's, in the row they begin in
  if (a.pitch != b.pitch) return true;
  const uint64_t off = y >= x ? (y - x) % a.pitch : (a.pitch - (x - y) % a.pitch) % a.pitch;
  return off < a.width || off + b.width > a.pitch;
}
template <size_t NO, size_t NI>
pa_status rows_apart(const char* who, const Rows (&out)[NO], const Rows (&in)[NI]) {
  for (size_t i = 0; i < NO; ++i) {
    for (size_t j = i + 1; j < NO; ++j)
      if (rows_meet(out[i], out[j]))
        return err(PA_ERR_INVALID, "%s: %s and %s overlap", who, out[i].name, out[j].name);
    for (const Rows& s : in)
      if (rows_meet(out[i], s))
        return err(PA_ERR_INVALID, "%s: %s and %s overlap", who, out[i].name, s.name);
  }
  return PA_OK;
}

// Sizes and parameters of the joint.
pa_status joint_sizes(const char* who, int64_t N, int C, int dtype) {
  PO_TRY(dtype_ok(who, dtype));
  if (N < 1 || C < 1) return err(PA_ERR_INVALID, "%s: N and C must be >= 1", who);
  const int most = dtype == PA_BF16 ? 8192 : 4096;
  if (C < 16 || C % 8 || C > most || N > ((int64_t)1 << 40) / C)
    return err(PA_ERR_UNSUPPORTED, "%s: C must be a multiple of 8 in [16, %d], N C at most 2^40",
               who, most);
  return PA_OK;
}
pa_status joint_params(const char* who, const pa_residual_norm_params* p, bool gate) {
  if (!p) return err(PA_ERR_INVALID, "%s: params is NULL", who);
  for (int k : {p->post, p->pre})
    if (k != PA_NORM_NONE && k != PA_NORM_LAYER && k != PA_NORM_RMS)
      return err(PA_ERR_INVALID, "%s: post and pre must be a pa_norm", who);
  if (gate && p->gate != PA_GATE_LINEAR && p->gate != PA_GATE_SIGMOID)
    return err(PA_ERR_INVALID, "%s: gate must be a pa_gate", who);
  if ((p->post != PA_NORM_NONE && !(p->post_eps > 0.f && std::isfinite(p->post_eps))) ||
      (p->pre != PA_NORM_NONE && !(p->pre_eps > 0.f && std::isfinite(p->pre_eps))))
    return err(PA_ERR_INVALID, "%s: eps must be > 0 and finite", who);
  if (!std::isfinite(p->alpha)) return err(PA_ERR_INVALID, "%s: alpha must be finite", who);
  if (p->post == PA_NORM_NONE && (p->post_g || p->post_b))
    return err(PA_ERR_INVALID, "%s: post_g and post_b need a post norm", who);
  if (p->pre == PA_NORM_NONE && (p->pre_g || p->pre_b))
    return err(PA_ERR_INVALID, "%s: pre_g and pre_b need a pre norm", who);
  PO_TRY(opt(who, p->post_g, "post_g"));
  PO_TRY(opt(who, p->post_b, "post_b"));
  PO_TRY(opt(who, p->scale, "scale"));
  PO_TRY(opt(who, p->pre_g, "pre_g"));
  PO_TRY(opt(who, p->pre_b, "pre_b"));
  return PA_OK;
}
pa::ResNormArgs joint_args(int64_t N, int C, const pa_residual_norm_params* p) {
  pa::ResNormArgs a;
  a.N = N; a.C = C;
  a.post = p->post; a.pre = p->pre; a.gate = p->gate;
  a.post_eps = p->post_eps; a.pre_eps = p->pre_eps; a.alpha = p->alpha;
  a.post_g = p->post_g; a.post_b = p->post_b; a.scale = p->scale;
  a.pre_g = p->pre_g; a.pre_b = p->pre_b;
  return a;
}

pa_status i8_sizes(const char* who, int64_t N, int F, int K) {
  if (N < 1 || F < 1 || K < 1) return err(PA_ERR_INVALID, "%s: N, F and K must be >= 1", who);
  if (K > 131072 || F > (1 << 20) || N > ((int64_t)1 << 34))
    return err(PA_ERR_UNSUPPORTED, "%s: K at most 131072, F at most 2^20, N at most 2^34", who);
  return PA_OK;
}
int pad16(int K) { return (K + 15) / 16 * 16; }

}  // namespace

extern "C" {

int pa_ops_version(void) { return PA_OPS_VERSION; }

pa_status pa_residual_norm(int64_t N, int C, pa_dtype dtype, const pa_residual_norm_params* p,
                           const void* x, const void* y, const void* t, void* x1, void* h,
                           int8_t* hq, float* hs, void* stream) {
  const char* who = "pa_residual_norm";
  PO_TRY(joint_sizes(who, N, C, dtype));
  PO_TRY(joint_params(who, p, t != nullptr));
  PO_TRY(need(who, x, "x"));
  PO_TRY(need(who, y, "y"));
  PO_TRY(opt(who, t, "t"));
  PO_TRY(need(who, x1, "x1"));
  PO_TRY(opt(who, h, "h"));
  PO_TRY(opt(who, hq, "hq"));
  PO_TRY(opt(who, hs, "hs", 4));
  if (!hq != !hs) return err(PA_ERR_INVALID, "%s: hq and hs go together", who);
  if (p->pre == PA_NORM_NONE && (h || hq))
    return err(PA_ERR_INVALID, "%s: h, hq and hs need a pre norm", who);
  const uint64_t n = (uint64_t)N * C * dtype_bytes(dtype), v = (uint64_t)C * 4;
  PO_TRY(apart(who, {{"x1", x1, n}, {"h", h, n}, {"hq", hq, (uint64_t)N * pad16(C)}, {"hs", hs, (uint64_t)N * 4}},
               {{"x", x, n}, {"y", y, n}, {"t", t, n}, {"post_g", p->post_g, v}, {"post_b", p->post_b, v},
                {"scale", p->scale, v}, {"pre_g", p->pre_g, v}, {"pre_b", p->pre_b, v}}));
  pa::ResNormArgs a = joint_args(N, C, p);
  a.x = x; a.y = y; a.t = t; a.x1 = x1; a.h = h; a.hq = hq; a.hs = hs;
  if (!h && !hq) a.pre = PA_NORM_NONE;
  PO_HIP(pa::launch_resnorm(a, dtype, false, as_stream(stream)), who);
  return PA_OK;
}

pa_status pa_residual_norm_workspace(int64_t N, int C, pa_dtype dtype, size_t* bytes) {
  const char* who = "pa_residual_norm_workspace";
  PO_TRY(joint_sizes(who, N, C, dtype));
  if (!bytes) return err(PA_ERR_INVALID, "%s: bytes is NULL", who);
  *bytes = (size_t)pa::resnorm_blocks(N, C, dtype, true) * 5 * C * sizeof(float);
  return PA_OK;
}

pa_status pa_residual_norm_backward(int64_t N, int C, pa_dtype dtype,
                                    const pa_residual_norm_params* p, const void* x1,
                                    const void* y, const void* t, const void* dx1,
                                    const void* dh, void* dx, void* dy, void* dt,
                                    const pa_residual_norm_grads* gr, void* ws, size_t ws_bytes,
                                    void* stream) {
  const char* who = "pa_residual_norm_backward";
  PO_TRY(joint_sizes(who, N, C, dtype));
  PO_TRY(joint_params(who, p, t != nullptr));
  PO_TRY(need(who, x1, "x1"));
  PO_TRY(need(who, y, "y"));
  PO_TRY(opt(who, t, "t"));
  PO_TRY(opt(who, dx1, "dx1"));
  PO_TRY(opt(who, dh, "dh"));
  if (!dx1 && !dh) return err(PA_ERR_INVALID, "%s: one of dx1 and dh is required", who);
  if (dh && p->pre == PA_NORM_NONE) return err(PA_ERR_INVALID, "%s: dh needs a pre norm", who);
  PO_TRY(need(who, dx, "dx"));
  PO_TRY(need(who, dy, "dy"));
  if (!t != !dt) return err(PA_ERR_INVALID, "%s: t and dt go together", who);
  PO_TRY(opt(who, dt, "dt"));
  pa::Segments seg{};
  bool sums = false;
  if (gr) {
    float* d[5] = {gr->dpost_g, gr->dpost_b, gr->dscale, gr->dpre_g, gr->dpre_b};
    const char* names[5] = {"dpost_g", "dpost_b", "dscale", "dpre_g", "dpre_b"};
    for (int i = 0; i < 5; ++i) {
      PO_TRY(opt(who, d[i], names[i], 4));
      if (i < 2 && p->post == PA_NORM_NONE) d[i] = nullptr;
      if (i > 2 && p->pre == PA_NORM_NONE) d[i] = nullptr;
      seg.dst[i] = d[i];
      seg.len[i] = C;
      sums = sums || d[i];
    }
    seg.n = 5;
  }
  const int P = pa::resnorm_blocks(N, C, dtype, true);
  const size_t bytes = sums ? (size_t)P * 5 * C * sizeof(float) : 0;
  if (sums && (!ws || ws_bytes < bytes))
    return err(PA_ERR_WORKSPACE, "%s: workspace needs %zu bytes", who, bytes);
  if (sums) PO_TRY(opt(who, ws, "ws"));
  const uint64_t n = (uint64_t)N * C * dtype_bytes(dtype), v = (uint64_t)C * 4;
  PO_TRY(apart(who,
               {{"dx", dx, n}, {"dy", dy, n}, {"dt", dt, n}, {"dpost_g", seg.dst[0], v},
                {"dpost_b", seg.dst[1], v}, {"dscale", seg.dst[2], v}, {"dpre_g", seg.dst[3], v},
                {"dpre_b", seg.dst[4], v}, {"ws", sums ? ws : nullptr, bytes}},
               {{"x1", x1, n}, {"y", y, n}, {"t", t, n}, {"dx1", dx1, n}, {"dh", dh, n},
                {"post_g", p->post_g, v}, {"post_b", p->post_b, v}, {"scale", p->scale, v},
                {"pre_g", p->pre_g, v}}));
  pa::ResNormArgs a = joint_args(N, C, p);
  a.y = y; a.t = t; a.x1 = const_cast<void*>(x1);
  a.dx1 = dx1; a.dh = dh; a.dx = dx; a.dy = dy; a.dt = dt;
  a.partials = sums ? reinterpret_cast<float*>(ws) : nullptr;
  if (sums && P == 1) {  // (nothing to add to the only block's sums)
    a.g0 = seg.dst[0]; a.g1 = seg.dst[1]; a.g2 = seg.dst[2]; a.g3 = seg.dst[3]; a.g4 = seg.dst[4];
  }
  PO_HIP(pa::launch_resnorm(a, dtype, true, as_stream(stream)), who);
  if (sums && P > 1) PO_HIP(pa::launch_reduce(a.partials, P, 5 * C, seg, as_stream(stream)), who);
  return PA_OK;
}

// Two tensors of one call that share memory: their updates would race.
static pa_status adamw_overlap(const char* who, int n, const pa_adamw_item* items) {
  struct Range { uintptr_t lo, hi; };
  try {
    std::vector<Range> r;
    r.reserve(6 * (size_t)n);
    for (int i = 0; i < n; ++i) {
      const pa_adamw_item& t = items[i];
      if (!t.n) continue;
      const uintptr_t st = t.m_scale ? 1 : 4;
      r.push_back({(uintptr_t)t.p, (uintptr_t)t.p + 4 * (uintptr_t)t.n});
      r.push_back({(uintptr_t)t.m, (uintptr_t)t.m + st * (uintptr_t)t.n});
      r.push_back({(uintptr_t)t.v, (uintptr_t)t.v + st * (uintptr_t)t.n});
      if (t.copy) r.push_back({(uintptr_t)t.copy, (uintptr_t)t.copy + 2 * (uintptr_t)t.n});
      const uintptr_t sb = 4 * (((uintptr_t)t.n + 255) / 256);
      if (t.m_scale) r.push_back({(uintptr_t)t.m_scale, (uintptr_t)t.m_scale + sb});
      if (t.v_scale) r.push_back({(uintptr_t)t.v_scale, (uintptr_t)t.v_scale + sb});
    }
    std::sort(r.begin(), r.end(), [](const Range& a, const Range& b) { return a.lo < b.lo; });
    for (size_t i = 1; i < r.size(); ++i)
      if (r[i].lo < r[i - 1].hi) return err(PA_ERR_INVALID, "%s: tensors overlap", who);
  } catch (const std::bad_alloc&) {
    return err(PA_ERR_INVALID, "%s: no host memory to check %d items", who, n);
  }
  return PA_OK;
}

static pa_status adamw_items(const char* who, int n_items, const pa_adamw_item* items) {
  if (n_items < 0 || (n_items && !items)) return err(PA_ERR_INVALID, "%s: items are required", who);
  for (int i = 0; i < n_items; ++i) {
    const pa_adamw_item& t = items[i];
    if (t.n < 0 || t.n > ((int64_t)1 << 36))
      return err(PA_ERR_INVALID, "%s: item %d has %lld elements", who, i, (long long)t.n);
    if (!t.n) continue;
    PO_TRY(dtype_ok(who, t.g_dtype));
    PO_TRY(need(who, t.p, "p"));
    PO_TRY(opt(who, t.copy, "copy"));
    PO_TRY(need(who, t.g, "g"));
    PO_TRY(need(who, t.m, "m"));
    PO_TRY(need(who, t.v, "v"));
    if (!t.m_scale != !t.v_scale)
      return err(PA_ERR_INVALID, "%s: m_scale and v_scale go together", who);
    PO_TRY(opt(who, t.m_scale, "m_scale", 4));
    PO_TRY(opt(who, t.v_scale, "v_scale", 4));
    if (!std::isfinite(t.wd)) return err(PA_ERR_INVALID, "%s: wd must be finite", who);
  }
  return adamw_overlap(who, n_items, items);
}

static pa::AdamItem adamw_item(const pa_adamw_item& t) {
  return {t.p, t.copy, t.g, t.m, t.v, t.m_scale, t.v_scale, t.n, t.wd,
          (t.g_dtype == PA_BF16 ? 1u : 0u) | (t.m_scale ? 2u : 0u)};
}

static pa_status adamw_step(const char* who, const pa_adamw_args* args, pa::AdamStep* s) {
  if (!args) return err(PA_ERR_INVALID, "%s: args is NULL", who);
  const auto unit = [](double b) { return b >= 0.0 && b < 1.0; };
  if (!std::isfinite(args->lr) || !unit(args->beta1) || !unit(args->beta2) ||
      !std::isfinite(args->eps) || !((float)args->eps >= FLT_MIN))
    return err(PA_ERR_INVALID, "%s: lr finite, betas in [0, 1), eps at least %g", who, FLT_MIN);
  if (!args->step_dev && args->step < 1) return err(PA_ERR_INVALID, "%s: step must be >= 1", who);
  PO_TRY(opt(who, args->gscale, "gscale", 4));
  PO_TRY(opt(who, args->lr_dev, "lr_dev", 4));
  PO_TRY(opt(who, args->step_dev, "step_dev", 8));
  s->lr = args->lr; s->beta1 = args->beta1; s->beta2 = args->beta2;
  s->eps = (float)args->eps;
  s->gscale = args->gscale; s->lr_dev = args->lr_dev; s->step_dev = args->step_dev;
  s->step = args->step;
  s->seed_key = pa::adam_mix((uint32_t)args->seed, (uint32_t)(args->seed >> 32));
  s->step_key = pa::adam_mix(s->seed_key, (uint32_t)args->step);
  if (!args->step_dev)
    pa::adam_consts(args->lr, args->beta1, args->beta2, args->step, &s->ss, &s->rs);
  s->b1 = (float)args->beta1; s->c1 = (float)(1.0 - args->beta1);
  s->b2 = (float)args->beta2; s->c2 = (float)(1.0 - args->beta2);
  return PA_OK;
}

pa_status pa_adamw(int n_items, const pa_adamw_item* items, const pa_adamw_args* args,
                   void* stream) {
  const char* who = "pa_adamw";
  pa::AdamBatch b{};
  PO_TRY(adamw_step(who, args, &b.s));
  PO_TRY(adamw_items(who, n_items, items));
  for (int i = 0; i < n_items;) {
    // the next items, up to kAdamMax (one without elements takes no block)
    b.n = 0;
    b.base = i;
    b.first[0] = 0;
    for (; i < n_items && b.n < pa::kAdamMax; ++i, ++b.n) {
      b.it[b.n] = adamw_item(items[i]);
      b.first[b.n + 1] = b.first[b.n] + pa::adam_blocks(items[i].n);
    }
    if (b.first[b.n]) PO_HIP(pa::launch_adamw(b, as_stream(stream)), who);
  }
  return PA_OK;
}

// A table's blocks, or -1: more than a launch takes.
static int64_t adamw_blocks(int n_items, const pa_adamw_item* items) {
  int64_t blocks = 0;
  for (int i = 0; i < n_items; ++i) blocks += pa::adam_blocks(items[i].n);
  return blocks <= 0x7fffffff ? blocks : -1;
}

pa_status pa_adamw_table_size(int n_items, const pa_adamw_item* items, size_t* bytes,
                              int64_t* blocks) {
  const char* who = "pa_adamw_table_size";
  if (!bytes || !blocks) return err(PA_ERR_INVALID, "%s: bytes and blocks are required", who);
  PO_TRY(adamw_items(who, n_items, items));
  *blocks = adamw_blocks(n_items, items);
  if (*blocks < 0) return err(PA_ERR_UNSUPPORTED, "%s: too many elements for one table", who);
  *bytes = sizeof(pa::AdamEntry) * (size_t)n_items + sizeof(uint32_t) * (size_t)*blocks;
  return PA_OK;
}

pa_status pa_adamw_table(int n_items, const pa_adamw_item* items, void* host, size_t bytes) {
  const char* who = "pa_adamw_table";
  size_t size = 0;
  int64_t blocks = 0;
  PO_TRY(pa_adamw_table_size(n_items, items, &size, &blocks));
  if (size && (!host || bytes < size))
    return err(PA_ERR_WORKSPACE, "%s: the table needs %zu bytes", who, size);
  PO_TRY(opt(who, host, "host", 8));
  pa::AdamEntry* e = reinterpret_cast<pa::AdamEntry*>(host);
  uint32_t* map = reinterpret_cast<uint32_t*>(e + n_items);
  uint32_t first = 0;
  for (int i = 0; i < n_items; ++i) {
    const uint32_t k = pa::adam_blocks(items[i].n);
    e[i] = {adamw_item(items[i]), first, (uint32_t)i};
    for (uint32_t j = 0; j < k; ++j) map[first + j] = (uint32_t)i;
    first += k;
  }
  return PA_OK;
}

pa_status pa_adamw_run(int n_items, int64_t blocks, const void* table, const pa_adamw_args* args,
                       void* stream) {
  const char* who = "pa_adamw_run";
  pa::AdamStep s{};
  PO_TRY(adamw_step(who, args, &s));
  if (n_items < 0 || blocks < 0 || blocks > 0x7fffffff)
    return err(PA_ERR_INVALID, "%s: n_items and blocks as pa_adamw_table_size gave them", who);
  if (!blocks) return PA_OK;
  PO_TRY(need(who, table, "table"));
  const pa::AdamEntry* e = reinterpret_cast<const pa::AdamEntry*>(table);
  PO_HIP(pa::launch_adamw_table(s, e, reinterpret_cast<const uint32_t*>(e + n_items),
                                (uint32_t)blocks, as_stream(stream)), who);
  return PA_OK;
}

pa_status pa_adamw_unpack(int64_t n, const void* codes, const float* scales, int is_signed,
                          float* out, void* stream) {
  const char* who = "pa_adamw_unpack";
  if (n < 1 || n > ((int64_t)1 << 40)) return err(PA_ERR_INVALID, "%s: n must be in [1, 2^40]", who);
  PO_TRY(need(who, codes, "codes"));
  PO_TRY(need(who, scales, "scales", 4));
  PO_TRY(need(who, out, "out"));
  PO_TRY(apart(who, {{"out", out, (uint64_t)n * 4}},
               {{"codes", codes, (uint64_t)n}, {"scales", scales, ((uint64_t)n + 255) / 256 * 4}}));
  PO_HIP(pa::launch_adam_unpack(n, (const uint8_t*)codes, scales, is_signed != 0, out,
                                as_stream(stream)), who);
  return PA_OK;
}

pa_status pa_quant_rows(int64_t N, int K, pa_dtype dtype, const void* x, int8_t* q, float* s,
                        void* stream) {
  const char* who = "pa_quant_rows";
  PO_TRY(i8_sizes(who, N, 1, K));
  PO_TRY(dtype_ok(who, dtype));
  PO_TRY(need(who, x, "x"));
  PO_TRY(need(who, q, "q"));
  PO_TRY(need(who, s, "s", 4));
  PO_TRY(apart(who, {{"q", q, (uint64_t)N * pad16(K)}, {"s", s, (uint64_t)N * 4}},
               {{"x", x, (uint64_t)N * K * dtype_bytes(dtype)}}));
  PO_HIP(pa::launch_quant_rows(N, K, dtype, x, q, s, as_stream(stream)), who);
  return PA_OK;
}

pa_status pa_quant_weight(int K, int F, pa_dtype dtype, const void* W, int8_t* Wq, float* sw,
                          void* stream) {
  const char* who = "pa_quant_weight";
  PO_TRY(i8_sizes(who, 1, F, K));
  PO_TRY(dtype_ok(who, dtype));
  PO_TRY(need(who, W, "W"));
  PO_TRY(need(who, Wq, "Wq"));
  PO_TRY(need(who, sw, "sw", 4));
  PO_TRY(apart(who, {{"Wq", Wq, (uint64_t)F * pad16(K)}, {"sw", sw, (uint64_t)F * 4}},
               {{"W", W, (uint64_t)K * F * dtype_bytes(dtype)}}));
  PO_HIP(pa::launch_quant_weight(K, F, dtype, W, Wq, sw, as_stream(stream)), who);
  return PA_OK;
}

static pa_status product(const char* who, pa::I8Args& a, int64_t N, int F, int K,
                         const int8_t* Wq, const float* sw, const float* bias, pa_act act,
                         const void* C, void* D, pa_dtype d_dtype) {
  PO_TRY(i8_sizes(who, N, F, K));
  PO_TRY(dtype_ok(who, d_dtype));
  if (act != PA_ACT_NONE && act != PA_ACT_GELU)
    return err(PA_ERR_INVALID, "%s: act must be a pa_act", who);
  PO_TRY(need(who, Wq, "Wq"));
  PO_TRY(need(who, sw, "sw", 4));
  PO_TRY(opt(who, bias, "bias", 4));
  PO_TRY(opt(who, C, "C"));
  PO_TRY(need(who, D, "D"));
  a.N = N; a.F = F; a.K = K; a.Kp = pad16(K);
  a.w = Wq; a.sw = sw; a.bias = bias; a.act = act; a.C = C; a.D = D;
  return PA_OK;
}

// D apart from what the product reads: its rows (of a width in bytes) and their
// scales, the weights, the bias, and C where D is not C itself; and the workspace,
// where there is one, from all of them.
static pa_status product_apart(const char* who, const pa::I8Args& a, pa_dtype d_dtype,
                               const void* rows, uint64_t width, const float* s, const void* ws,
                               uint64_t ws_bytes) {
  const uint64_t N = (uint64_t)a.N, F = (uint64_t)a.F, d = N * F * dtype_bytes(d_dtype);
  return apart(who, {{"D", a.D, d}, {"ws", ws, ws_bytes}},
               {{a.x ? "x" : "q", rows, N * width}, {"s", s, N * 4}, {"Wq", a.w, F * (uint64_t)a.Kp},
                {"sw", a.sw, F * 4}, {"bias", a.bias, F * 4}, {"C", a.C == a.D ? nullptr : a.C, d}});
}

// The product of rows that are integers.
static hipError_t integers(const pa::I8Args& a, int d_dtype, hipStream_t st) {
  return d_dtype == PA_BF16 && pa::linear_i8_fused(a.N, a.F, a.K) ? pa::launch_linear_i8(a, st)
                                                                  : pa::launch_gemm_i8(a, d_dtype, st);
}

pa_status pa_gemm_i8(int64_t N, int F, int K, const int8_t* q, const float* s, const int8_t* Wq,
                     const float* sw, const float* bias, pa_act act, const void* C, void* D,
                     pa_dtype d_dtype, void* stream) {
  const char* who = "pa_gemm_i8";
  pa::I8Args a;
  PO_TRY(product(who, a, N, F, K, Wq, sw, bias, act, C, D, d_dtype));
  PO_TRY(need(who, q, "q"));
  PO_TRY(need(who, s, "s", 4));
  a.q = q; a.s = s;
  PO_TRY(product_apart(who, a, d_dtype, q, (uint64_t)a.Kp, s, nullptr, 0));
  PO_HIP(integers(a, d_dtype, as_stream(stream)), who);
  return PA_OK;
}

pa_status pa_linear_i8_workspace(int64_t N, int F, int K, size_t* bytes) {
  const char* who = "pa_linear_i8_workspace";
  PO_TRY(i8_sizes(who, N, F, K));
  if (!bytes) return err(PA_ERR_INVALID, "%s: bytes is NULL", who);
  *bytes = (size_t)N * pad16(K) + (size_t)N * 4;
  return PA_OK;
}

pa_status pa_linear_i8(int64_t N, int F, int K, const void* x, pa_dtype x_dtype,
                       const int8_t* Wq, const float* sw, const float* bias, pa_act act,
                       const void* C, void* D, pa_dtype d_dtype, void* ws, size_t ws_bytes,
                       void* stream) {
  const char* who = "pa_linear_i8";
  pa::I8Args a;
  PO_TRY(product(who, a, N, F, K, Wq, sw, bias, act, C, D, d_dtype));
  PO_TRY(dtype_ok(who, x_dtype));
  PO_TRY(need(who, x, "x"));
  a.x = x;
  a.x_dtype = x_dtype;
  // (asked for whether the kernel of these sizes uses it or not)
  const size_t rows = (size_t)N * a.Kp;
  if (!ws || ws_bytes < rows + (size_t)N * 4)
    return err(PA_ERR_WORKSPACE, "%s: workspace needs %zu bytes", who, rows + (size_t)N * 4);
  PO_TRY(opt(who, ws, "ws"));
  PO_TRY(product_apart(who, a, d_dtype, x, (uint64_t)K * dtype_bytes(x_dtype), nullptr, ws,
                       rows + (uint64_t)N * 4));
  const bool fused =
      x_dtype == PA_BF16 && d_dtype == PA_BF16 && K % 8 == 0 && pa::linear_i8_fused(N, F, K);
  // (of both, for weights of at most 64 KiB and 512 inputs the one-pass product is as
  // fast or faster: us at 333 rows, 256 to 128 4.3 and 5.2, 512 to 128 5.9 and 5.0)
  if (pa::linear_i8_few(N, F, K, x_dtype) && (N <= 16 || !fused || K > 512 || K * F > 65536)) {
    PO_HIP(pa::launch_linear_few(a, d_dtype, as_stream(stream)), who);
    return PA_OK;
  }
  if (fused) {
    PO_HIP(pa::launch_linear_i8(a, as_stream(stream)), who);
    return PA_OK;
  }
  int8_t* q = reinterpret_cast<int8_t*>(ws);
  float* s = reinterpret_cast<float*>(q + rows);
  PO_HIP(pa::launch_quant_rows(N, K, x_dtype, x, q, s, as_stream(stream)), who);
  a.q = q;
  a.s = s;
  PO_HIP(integers(a, d_dtype, as_stream(stream)), who);
  return PA_OK;
}

// ---- attention of query points over states ----
static pa_status ask_params(const char* who, int64_t Nq, int64_t Nk, int dtype,
                            const pa_cross_attention_params* p, pa::AskArgs* a) {
  PO_TRY(dtype_ok(who, dtype));
  if (!p) return err(PA_ERR_INVALID, "%s: params is NULL", who);
  if (Nq < 0 || Nk < 0) return err(PA_ERR_INVALID, "%s: Nq and Nk must be >= 0", who);
  if (p->R < 1) return err(PA_ERR_INVALID, "%s: R must be >= 1", who);
  if (p->Hq < 1 || p->Hkv < 1 || p->Hq % p->Hkv)
    return err(PA_ERR_INVALID, "%s: Hkv must divide Hq", who);
  if (p->D < 8 || p->D % 8 || p->D > 128)
    return err(PA_ERR_UNSUPPORTED, "%s: D must be a multiple of 8 in [8, 128]", who);
  const int64_t most = pa::kMostRows;
  if (p->Hq > 4096 || p->R > (1 << 24) || Nk > most || Nq > most / (p->Hq / p->Hkv))
    return err(PA_ERR_UNSUPPORTED, "%s: Hq at most 4096, R 2^24, Nk and Nq Hq / Hkv below 2^31 - 2^21",
               who);
  if (((Nq * (p->Hq / p->Hkv) >> 6) + p->R) * p->Hkv > most || ((Nk >> 6) + p->R) * p->Hkv > most)
    return err(PA_ERR_UNSUPPORTED, "%s: too many rows times heads for one launch", who);
  // (scores are scaled for a power of 2: scale log2 e has to be finite too)
  if (!(p->scale > 0.f) || !(p->scale <= 0x1p127f))
    return err(PA_ERR_INVALID, "%s: scale must be > 0 and at most 2^127", who);
  if (!p->q_off != !p->k_off) return err(PA_ERR_INVALID, "%s: q_off and k_off go together", who);
  if (!p->q_off && p->R != 1) return err(PA_ERR_INVALID, "%s: R > 1 needs q_off and k_off", who);
  if (p->max_k < 0) return err(PA_ERR_INVALID, "%s: max_k must be >= 0", who);
  PO_TRY(opt(who, p->q_off, "q_off", 8));
  PO_TRY(opt(who, p->k_off, "k_off", 8));
  a->Nq = Nq; a->Nk = Nk; a->R = p->R; a->Hq = p->Hq; a->Hkv = p->Hkv; a->D = p->D;
  a->scale = p->scale; a->q_off = p->q_off; a->k_off = p->k_off; a->mask = p->mask;
  a->max_k = p->k_off && p->max_k && p->max_k < Nk ? p->max_k : Nk;
  return PA_OK;
}
// A tensor of N rows of H heads, given with the elements between its rows; without
// rows it may be NULL.
static pa_status ask_rows(const char* who, const char* name, const void* ptr, int64_t N, int H,
                          int D, int64_t* ld, int dtype, Rows* out) {
  const int64_t b = (int64_t)dtype_bytes(dtype), width = (int64_t)H * D;
  if (N < 2) *ld = width;
  if (*ld < width || *ld * b % 16)
    return err(PA_ERR_INVALID, "%s: ld of %s must be a multiple of 16 bytes and at least %lld", who,
               name, (long long)width);
  if (*ld >= (1 << 25) / b)  // (offsets in a tile of 64 rows are 31 bits)
    return err(PA_ERR_UNSUPPORTED, "%s: rows of %s must be less than 2^25 bytes apart", who, name);
  if (N) PO_TRY(need(who, ptr, name));
  *out = {name, ptr, (uint64_t)N, (uint64_t)(width * b), (uint64_t)(*ld * b)};
  return PA_OK;
}
static Rows flat(const char* name, const void* p, uint64_t bytes) { return {name, p, 1, bytes, bytes}; }

// The workspace's parts, of which the forward has the first two; returns the bytes.
static size_t ask_layout(pa::AskArgs* a, int dtype, bool backward, void* ws) {
  char* base = reinterpret_cast<char*>(ws);
  size_t at = 0;
  const auto take = [&](uint64_t floats) {
    float* p = base ? reinterpret_cast<float*>(base + at) : nullptr;
    at += (floats * 4 + 255) / 256 * 256;
    return p;
  };
  const uint64_t rows = (uint64_t)a->Nq * a->Hq;
  if (backward ? pa::ask_few_backward_served(*a, dtype) : pa::ask_few_served(*a, dtype)) {
    if (!backward) return at;
    const uint64_t n = (uint64_t)pa::ask_few_records(*a);
    a->part_k = take(n);
    a->part_v = take(n);
    return at;
  }
  a->S = backward ? pa::ask_pieces_dq(*a, dtype) : pa::ask_pieces(*a, dtype);
  if (a->S > 1) {
    a->part = take((uint64_t)a->S * rows * a->D);
    a->part_lse = take((uint64_t)a->S * rows);
  }
  if (!backward) return at;
  a->delta = take(rows);
  if (a->S > 1) {
    a->part_b = take((uint64_t)a->S * rows * a->D);
    if (dtype == PA_BF16) a->part_e = take((uint64_t)a->S * rows);
  }
  a->SQ = pa::ask_pieces_q(*a, dtype);
  if (a->SQ > 1) {
    const uint64_t n = (uint64_t)a->SQ * a->Nk * a->Hkv * a->D;
    a->part_k = take(n);
    a->part_v = take(n);
  }
  return at;
}

pa_status pa_cross_attention_workspace(int64_t Nq, int64_t Nk, pa_dtype dtype,
                                       const pa_cross_attention_params* p, int backward,
                                       size_t* bytes) {
  const char* who = "pa_cross_attention_workspace";
  pa::AskArgs a;
  PO_TRY(ask_params(who, Nq, Nk, dtype, p, &a));
  if (!bytes) return err(PA_ERR_INVALID, "%s: bytes is NULL", who);
  *bytes = ask_layout(&a, dtype, backward != 0, nullptr);
  return PA_OK;
}

pa_status pa_cross_attention(int64_t Nq, int64_t Nk, pa_dtype dtype,
                             const pa_cross_attention_params* p, const void* q, int64_t ldq,
                             const void* k, int64_t ldk, const void* v, int64_t ldv, void* o,
                             int64_t ldo, float* lse, void* ws, size_t ws_bytes, void* stream) {
  const char* who = "pa_cross_attention";
  pa::AskArgs a;
  Rows rq, rk, rv, ro;
  PO_TRY(ask_params(who, Nq, Nk, dtype, p, &a));
  PO_TRY(ask_rows(who, "q", q, Nq, a.Hq, a.D, &ldq, dtype, &rq));
  PO_TRY(ask_rows(who, "k", k, Nk, a.Hkv, a.D, &ldk, dtype, &rk));
  PO_TRY(ask_rows(who, "v", v, Nk, a.Hkv, a.D, &ldv, dtype, &rv));
  PO_TRY(ask_rows(who, "o", o, Nq, a.Hq, a.D, &ldo, dtype, &ro));
  PO_TRY(opt(who, lse, "lse", 4));
  const size_t bytes = ask_layout(&a, dtype, false, nullptr);
  if (bytes && (!ws || ws_bytes < bytes))
    return err(PA_ERR_WORKSPACE, "%s: workspace needs %zu bytes", who, bytes);
  if (bytes) PO_TRY(opt(who, ws, "ws"));
  const uint64_t offs = ((uint64_t)a.R + 1) * 8;
  PO_TRY(rows_apart(who, {ro, flat("lse", lse, (uint64_t)Nq * a.Hq * 4), flat("ws", bytes ? ws : nullptr, bytes)},
                    {rq, rk, rv, flat("mask", a.mask, (uint64_t)Nk), flat("q_off", a.q_off, offs),
                     flat("k_off", a.k_off, offs)}));
  if (!Nq) return PA_OK;
  ask_layout(&a, dtype, false, ws);
  a.q = q; a.k = k; a.v = v; a.o = o; a.lse = lse;
  a.ldq = ldq; a.ldk = ldk; a.ldv = ldv; a.ldo = ldo;
  PO_HIP(pa::launch_ask(a, dtype, as_stream(stream)), who);
  return PA_OK;
}

pa_status pa_cross_attention_backward(int64_t Nq, int64_t Nk, pa_dtype dtype,
                                      const pa_cross_attention_params* p, const void* q,
                                      int64_t ldq, const void* k, int64_t ldk, const void* v,
                                      int64_t ldv, const void* o, int64_t ldo, const float* lse,
                                      const void* d_o, int64_t lddo, void* dq, int64_t lddq,
                                      void* dk, int64_t lddk, void* dv, int64_t lddv, void* ws,
                                      size_t ws_bytes, void* stream) {
  const char* who = "pa_cross_attention_backward";
  pa::AskArgs a;
  Rows rq, rk, rv, ro, rd, rdq, rdk, rdv;
  PO_TRY(ask_params(who, Nq, Nk, dtype, p, &a));
  PO_TRY(ask_rows(who, "q", q, Nq, a.Hq, a.D, &ldq, dtype, &rq));
  PO_TRY(ask_rows(who, "k", k, Nk, a.Hkv, a.D, &ldk, dtype, &rk));
  PO_TRY(ask_rows(who, "v", v, Nk, a.Hkv, a.D, &ldv, dtype, &rv));
  PO_TRY(ask_rows(who, "o", o, Nq, a.Hq, a.D, &ldo, dtype, &ro));
  PO_TRY(ask_rows(who, "d_o", d_o, Nq, a.Hq, a.D, &lddo, dtype, &rd));
  PO_TRY(ask_rows(who, "dq", dq, Nq, a.Hq, a.D, &lddq, dtype, &rdq));
  if (Nk && !dk != !dv) return err(PA_ERR_INVALID, "%s: dk and dv go together", who);
  const bool states = dk && dv;
  PO_TRY(ask_rows(who, "dk", dk, states ? Nk : 0, a.Hkv, a.D, &lddk, dtype, &rdk));
  PO_TRY(ask_rows(who, "dv", dv, states ? Nk : 0, a.Hkv, a.D, &lddv, dtype, &rdv));
  if (Nq) PO_TRY(need(who, lse, "lse", 4));
  if (!Nq && !Nk) return PA_OK;
  const size_t bytes = ask_layout(&a, dtype, true, nullptr);
  if (bytes && (!ws || ws_bytes < bytes))
    return err(PA_ERR_WORKSPACE, "%s: workspace needs %zu bytes", who, bytes);
  if (bytes) PO_TRY(opt(who, ws, "ws"));
  const uint64_t offs = ((uint64_t)a.R + 1) * 8;
  PO_TRY(rows_apart(who, {rdq, rdk, rdv, flat("ws", bytes ? ws : nullptr, bytes)},
                    {rq, rk, rv, ro, rd, flat("lse", lse, (uint64_t)Nq * a.Hq * 4),
                     flat("mask", a.mask, (uint64_t)Nk), flat("q_off", a.q_off, offs),
                     flat("k_off", a.k_off, offs)}));
  ask_layout(&a, dtype, true, ws);
  a.q = q; a.k = k; a.v = v; a.o = const_cast<void*>(o); a.lse = const_cast<float*>(lse);
  a.ldq = ldq; a.ldk = ldk; a.ldv = ldv; a.ldo = ldo;
  a.d_o = d_o; a.dq = dq; a.lddo = lddo; a.lddq = lddq;
  a.dk = states ? dk : nullptr; a.dv = states ? dv : nullptr;
  a.lddk = lddk; a.lddv = lddv;
  PO_HIP(pa::launch_ask_backward(a, dtype, as_stream(stream)), who);
  return PA_OK;
}

pa_status pa_dropout(int64_t n, pa_dtype dtype, const void* y, const void* r, void* out, double p,
                     uint64_t seed, uint64_t offset, const int64_t* offset_dev, void* stream) {
  const char* who = "pa_dropout";
  PO_TRY(dtype_ok(who, dtype));
  if (n < 0 || n > ((int64_t)1 << 40)) return err(PA_ERR_INVALID, "%s: n must be in [0, 2^40]", who);
  if (!(p >= 0.0) || !(65536.0 * p < 65535.5))
    return err(PA_ERR_INVALID, "%s: p must be in [0, 1 - 2^-17)", who);
  PO_TRY(opt(who, offset_dev, "offset_dev", 8));
  if (!n) return PA_OK;
  PO_TRY(need(who, y, "y"));
  PO_TRY(opt(who, r, "r"));
  PO_TRY(need(who, out, "out"));
  const uint64_t bytes = (uint64_t)n * dtype_bytes(dtype);
  PO_TRY(apart(who, {{"out", out, bytes}},
               {{"y", y == out ? nullptr : y, bytes}, {"r", r == out ? nullptr : r, bytes},
                {"offset_dev", offset_dev, 8}}));
  pa::DropArgs a;
  a.n = n; a.y = y; a.r = r; a.out = out;
  a.threshold = (uint32_t)std::llround(65536.0 * p);
  a.scale = (float)(65536.0 / (65536.0 - a.threshold));
  a.seed = seed; a.offset = offset; a.offset_dev = offset_dev;
  PO_HIP(pa::launch_dropout(a, dtype, as_stream(stream)), who);
  return PA_OK;
}

}  // extern "C"
