"""The operators of include/pa_ops.h in 64 bits (and the parts that are defined
in 32 bits in 32), on the CPU, with the magnitudes that bound a 32-bit
evaluation's error."""
import math

import torch

U = 2.0 ** -24  # half a step of fp32, relative
LN_EPS = 1e-5


def half_step(dt):
    return torch.finfo(dt).eps / 2


# ---- the joint between two blocks ----
class Norm:
    """zh = (z - [mean]) r and the magnitude of zh's error in units of U: a row
    whose mean is large against its spread loses that ratio; the sums over C
    channels (lanes of 4 or 8 channels, then a tree) round at most 24 times."""

    def __init__(self, z, kind, eps):
        mean = z.mean(1, keepdim=True) if kind == "layer" else torch.zeros_like(z[:, :1])
        c = z - mean
        self.kind = kind
        self.r = 1 / torch.sqrt((c * c).mean(1, keepdim=True) + eps)
        self.zh = c * self.r
        big = z.abs().mean(1, keepdim=True) * self.r if kind == "layer" else 0 * self.r
        self.err = 32 * self.zh.abs() + 24 * big + 2 * (z * self.r).abs()

    def back(self, d, d_err):
        """z's gradient from zh's, and its error's magnitude (d known to d_err U)."""
        mz = (d * self.zh).mean(1, keepdim=True)
        az = (d * self.zh).abs().mean(1, keepdim=True)
        md = d.mean(1, keepdim=True) if self.kind == "layer" else 0 * mz
        ad = d.abs().mean(1, keepdim=True) if self.kind == "layer" else 0 * mz
        g = self.r * (d - md - self.zh * mz)
        ez = (d_err * self.zh.abs() + d.abs() * self.err).mean(1, keepdim=True) + 24 * az
        ed = d_err.mean(1, keepdim=True) + 24 * ad
        size = d.abs() + ad + self.zh.abs() * az
        err = self.r * (d_err + ed + self.zh.abs() * ez + self.err * az + 48 * size)
        return g, err


def vec(p, k, none):
    return p[k].double() if p.get(k) is not None else torch.full((), none, dtype=torch.float64)


def gate(t, kind):
    if t is None:
        one = torch.ones((), dtype=torch.float64)
        return one, 0 * one
    if kind == "linear":
        return t, torch.ones_like(t)
    m = torch.sigmoid(t)
    return m, m * torch.sigmoid(-t)


def joint(p, x, y, t=None):
    """x1 before rounding and its error's magnitude (in units of U)."""
    y = y.double()
    if p["post"]:
        n = Norm(y, p["post"], p.get("post_eps", LN_EPS))
        g, b = vec(p, "post_g", 1.0), vec(p, "post_b", 0.0)
        u, eu = n.zh * g + b, n.err * g.abs() + 2 * ((n.zh * g).abs() + b.abs())
    else:
        u, eu = y, 0 * y
    m, _ = gate(None if t is None else t.double(), p.get("gate", "sigmoid"))
    s = vec(p, "scale", 1.0)
    a = p.get("alpha", 1.0) * x.double()
    v = s * m * u
    return a + v, (s * m).abs() * eu + 16 * v.abs() + 4 * a.abs()


def pre(p, x1):
    """h before rounding, from the stored x1, and its error's magnitude."""
    n = Norm(x1.double(), p["pre"], p.get("pre_eps", LN_EPS))
    g, b = vec(p, "pre_g", 1.0), vec(p, "pre_b", 0.0)
    return n.zh * g + b, n.err * g.abs() + 2 * ((n.zh * g).abs() + b.abs())


def joint_backward(p, x1, y, t, dx1, dh, rows):
    """{name: (value, error's magnitude)}; rows: rows that one running sum of the
    parameters' gradients adds."""
    x1, y = x1.double(), y.double()
    o = {}

    def total(terms, err):
        return terms.sum(0), err.sum(0) + (rows + 16) * terms.abs().sum(0)

    e, ee = torch.zeros_like(x1), torch.zeros_like(x1)
    if dx1 is not None:
        e = e + dx1.double()
    if dh is not None:
        dh = dh.double()
        n = Norm(x1, p["pre"], p.get("pre_eps", LN_EPS))
        o["dpre_g"] = total(dh * n.zh, dh.abs() * n.err)
        o["dpre_b"] = total(dh, 0 * dh)
        gh = dh * vec(p, "pre_g", 1.0)
        g, ge = n.back(gh, 2 * gh.abs())
        e, ee = e + g, ee + ge + 2 * (e.abs() + g.abs())
    al = p.get("alpha", 1.0)
    o["dx"] = al * e, abs(al) * (ee + 2 * e.abs())
    m, slope = gate(None if t is None else t.double(), p.get("gate", "sigmoid"))
    s = vec(p, "scale", 1.0)
    if p["post"]:
        n = Norm(y, p["post"], p.get("post_eps", LN_EPS))
        g, b = vec(p, "post_g", 1.0), vec(p, "post_b", 0.0)
        u, eu = n.zh * g + b, n.err * g.abs() + 2 * ((n.zh * g).abs() + b.abs())
    else:
        u, eu = y, 0 * y
    if t is not None:
        v = s * e * u * slope
        o["dt"] = v, (s * slope).abs() * (ee * u.abs() + e.abs() * eu) + 24 * v.abs()
    o["dscale"] = total(e * m * u, m.abs() * (ee * u.abs() + e.abs() * eu) + 16 * (e * m * u).abs())
    du = s * m * e
    edu = (s * m).abs() * ee + 16 * du.abs()
    if not p["post"]:
        o["dy"] = du, edu
        return o
    o["dpost_b"] = total(du, edu)
    o["dpost_g"] = total(du * n.zh, edu * n.zh.abs() + du.abs() * n.err)
    o["dy"] = n.back(du * g, edu * g.abs() + 2 * (du * g).abs())
    return o


# ---- AdamW ----
def scramble(h):
    h = ((h ^ (h >> 16)) * 0x85EBCA6B) & 0xFFFFFFFF
    h = ((h ^ (h >> 13)) * 0xC2B2AE35) & 0xFFFFFFFF
    return h ^ (h >> 16)


def mix(a, b):
    return scramble(a ^ ((b * 0x9E3779B9) & 0xFFFFFFFF))


def random_bits(n, seed, step, item):
    """The 32 random bits of each of a tensor's n elements."""
    i = torch.arange(n, dtype=torch.int64)
    key = mix(mix(mix(seed & 0xFFFFFFFF, (seed >> 32) & 0xFFFFFFFF), step & 0xFFFFFFFF), item)
    return scramble((mix(torch.full_like(i, key), i // 256) + i % 256) & 0xFFFFFFFF)


def blocks(x):
    """x [n] as [ceil(n / 256), 256], zeros behind the end."""
    n = x.numel()
    o = torch.zeros(-(-n // 256) * 256, dtype=x.dtype)
    o[:n] = x
    return o.view(-1, 256)


def encode(x, h, signed):
    """Codes [n] and scales of an fp32 tensor; h: 16 random bits each."""
    n, lo, top = x.numel(), 889 if signed else 761, 127 if signed else 255
    bx = blocks(x)
    big = bx.abs().amax(1)
    bits = big.view(torch.int32).to(torch.int64)
    up = (bits & 0x7F800000) + 0x800000 * ((bits & 0x7FFFFF) > 0)
    S = up.clamp(0x00800000, 0x7F000000).to(torch.int32).view(torch.float32)
    S = torch.where(big > 0, S, torch.zeros_like(S))
    S = torch.where(torch.isfinite(bx).all(1), S, torch.full_like(S, math.nan))
    inv = torch.where(S == 0, torch.zeros_like(S), 1 / S)
    a = (bx.abs() * inv[:, None]).reshape(-1)[:n]
    c = ((a.view(torch.int32).to(torch.int64) + 16 * h + 8) >> 20) - lo
    if signed:
        c = c.clamp(0, top)
        c = c + 128 * ((x < 0) & (c > 0))
    else:
        c = torch.where(x == 0, 0, c.clamp(1, top))
    return c.to(torch.uint8), S


def decode(c, S, signed):
    c = c.to(torch.int64)
    mag = c & 127 if signed else c
    v = ((mag + (889 if signed else 761)) << 20).to(torch.int32).view(torch.float32)
    v = torch.where(mag > 0, v, torch.zeros_like(v)) * S.repeat_interleave(256)[:c.numel()]
    return torch.where(c > 127, -v, v) if signed else v


def adamw(p, g, m, v, lr, b1, b2, eps, wd, step, gscale=None):
    """The moments in 32 bits, every operation rounded, and the parameter in 64."""
    f = lambda z: torch.tensor(z, dtype=torch.float32)
    g = g.float()
    if gscale is not None:
        g = g * gscale
    m = m * f(b1) + g * f(1 - b1)
    v = v * f(b2) + (g * g) * f(1 - b2)
    upd = (m.double() / (1 - b1 ** step)) / (torch.sqrt(v.double() / (1 - b2 ** step)) + eps)
    return p.double() - lr * (wd * p.double() + upd), m, v, upd


# ---- 8-bit integer products ----
def quant(x):
    """q (as int32) and s of the rows of x [N, K]."""
    x = x.float()
    big = x.abs().amax(1)
    bad = ~torch.isfinite(x).all(1)
    small = big < 1e-36
    # (one division: torch forms 127 / big from a rounded reciprocal)
    inv = torch.div(torch.full_like(big, 127.0), big)
    inv = torch.where(small | bad, torch.zeros_like(big), inv)
    q = torch.where(inv[:, None] == 0, torch.zeros_like(x), torch.round(x * inv[:, None]))
    s = torch.where(small, torch.zeros_like(big), big / 127)
    return q.to(torch.int32), torch.where(bad, torch.full_like(s, math.nan), s)


def padded(q):
    N, K = q.shape
    o = torch.zeros(N, -(-K // 16) * 16, dtype=torch.int8)
    o[:, :K] = q.to(torch.int8)
    return o


def linear(q, s, w, sw, bias=None, act=None, C=None):
    """D before rounding and its error's magnitude (units of U; GELU's own error
    apart) from integers q [N, K], w [F, K]."""
    u = (q.double() @ w.double().t()) * s.double()[:, None] * sw.double()
    err = 4 * u.abs()
    if bias is not None:
        u = u + bias.double()
        err = err + 2 * u.abs() + bias.double().abs()
    if act == "gelu":  # |slope| at most 1.13; GELU's own arithmetic
        u = u * 0.5 * torch.erfc(-u / math.sqrt(2.0))
        err = 1.2 * err + 16 * u.abs()
    if C is not None:
        err = err + u.abs() + C.double().abs()
        u = u + C.double()
    return u, err
