"""pa_cross_attention and its backward in 64 bits on the CPU, with what bounds an
evaluation in 32 bits whose weights are rounded to the storage type; and
Philox-4x32-10 with the dropout that it decides."""
import numpy as np
import torch

U = 2.0 ** -24  # half a step of fp32, relative
# A weight below the smallest normal fp32 number, 2^-126, may become 0: with queries in
# the hundreds that is 2^-126 x 10 x 1000 in a gradient, above any bound by the value.
FLUSH = 2.0 ** -126


def half_step(dt):
    return torch.finfo(dt).eps / 2


class Out:
    """A value, the most that its evaluation can be off before the final rounding
    (every rounding at its largest, all of one sign), and what the 2-norm of the error
    can be (the weights' roundings, which are independent, by their squares)."""

    def __init__(self, shape, fill=0.0):
        self.v = torch.full(shape, fill, dtype=torch.float64)
        self.worst, self.rms = torch.zeros_like(self.v), torch.zeros_like(self.v)

    def put(self, at, v, hp, terms, squares, u_terms):
        """v with weights' roundings hp on `terms` (their sum of magnitudes; `squares`
        the root of their squares' sum) and 32-bit errors u_terms."""
        self.v[at] += v
        self.worst[at] += hp * terms + u_terms
        self.rms[at] += hp * squares + u_terms


def check(got, ref, dt, name, touched=None, before=None):
    """got against an Out; rows that are not `touched` have to be `before`."""
    got = got.detach().cpu()
    if touched is not None:
        rest = ~touched
        assert torch.equal(got[rest], before[rest]), f"{name}: rows of no request were written"
        pick = touched
    else:
        pick = torch.ones(got.shape[0], dtype=torch.bool)
    g, v, w, r = got[pick].double(), ref.v[pick], ref.worst[pick], ref.rms[pick]
    fin = torch.isfinite(v)
    assert torch.equal(g[~fin], v[~fin]), f"{name}: infinities"
    g, v, w, r = g[fin], v[fin], w[fin], r[fin]
    assert torch.isfinite(g).all(), f"{name}: not finite"
    if not g.numel():
        return
    hs = half_step(dt)
    off = (g - v).abs()
    bound = hs * (v.abs() + w) + w + 1e-37
    worst = (off / bound).max().item()
    assert worst <= 1, f"{name}: {worst:.3g} of the bound"
    # (a few values: the squares say little about the largest of them)
    if g.numel() >= 256:
        norm = (hs * v.norm() + r.norm()).item() + 1e-37
        assert off.norm().item() <= norm, f"{name}: norm {off.norm().item() / norm:.3g} of the bound"


def requests(q_off, k_off, Nq, Nk, mask):
    q_off = [0, Nq] if q_off is None else q_off
    k_off = [0, Nk] if k_off is None else k_off
    for r in range(len(q_off) - 1):
        live = torch.arange(k_off[r], k_off[r + 1])
        if mask is not None:
            live = live[mask[live] != 0]
        yield torch.arange(q_off[r], q_off[r + 1]), live


def _weights(q, k, scale):
    """Scores, lse, weights and the relative error of the weights in 32 bits: a score's
    D products and sums, its scaling and difference from the maximum, exp2 and the
    sum's roundings (the maximum is met again in the lse: both cancel but for it)."""
    D = q.shape[1]
    s = scale * (q @ k.t())
    size = scale * (q.abs() @ k.abs().t())
    lse = torch.logsumexp(s, 1, keepdim=True)
    p = torch.exp(s - lse)
    es = U * ((D + 4) * size + 4 * (s.abs() + lse.abs()) + 8)
    # (l's own error: its weights', and the roundings of a sum of k terms)
    el = (p * es).sum(1, keepdim=True) + U * (k.shape[0] / 4 + 64)
    return s, lse, p, es, el


def forward(q, k, v, scale, q_off=None, k_off=None, mask=None):
    """(o, lse, rows that belong to a request)."""
    Nq, Hq, D = q.shape
    Nk, Hkv = k.shape[:2]
    hp = 0.0 if q.dtype == torch.float32 else half_step(q.dtype)
    o, lse = Out((Nq, Hq, D)), Out((Nq, Hq), -float("inf"))
    touched = torch.zeros(Nq, dtype=torch.bool)
    for rows, live in requests(q_off, k_off, Nq, Nk, mask):
        touched[rows] = True
        if not rows.numel() or not live.numel():
            continue
        for h in range(Hq):
            kk, vv = k[live, h * Hkv // Hq].double(), v[live, h * Hkv // Hq].double()
            s, l, p, es, el = _weights(q[rows, h].double(), kk, scale)
            big = (p * es) @ vv.abs() + el * (p @ vv.abs())
            big = big + U * (live.numel() / 4 + 64) * (p @ vv.abs()) + FLUSH * vv.abs().sum(0)
            o.put((rows, h), p @ vv, hp, p @ vv.abs(), torch.sqrt((p * p) @ (vv * vv)), big)
            lse.v[rows, h] = 0
            e = (el + U * (4 * l.abs() + 8))[:, 0]
            lse.put((rows, h), l[:, 0], 0.0, 0.0, 0.0, e)
    return o, lse, touched


def backward(q, k, v, o, do, scale, q_off=None, k_off=None, mask=None):
    """({"dq", "dk", "dv"}: Out, touched rows of the queries and of the states); o: the
    forward's output in the storage type."""
    Nq, Hq, D = q.shape
    Nk, Hkv = k.shape[:2]
    hp = 0.0 if q.dtype == torch.float32 else half_step(q.dtype)
    out = {"dq": Out(q.shape), "dk": Out(k.shape), "dv": Out(v.shape)}
    tq, tk = torch.zeros(Nq, dtype=torch.bool), torch.zeros(Nk, dtype=torch.bool)
    ko = [0, Nk] if k_off is None else k_off
    for r, (rows, live) in enumerate(requests(q_off, k_off, Nq, Nk, mask)):
        tq[rows] = True
        tk[ko[r]:ko[r + 1]] = True
        if not rows.numel() or not live.numel():
            continue
        n, m = live.numel(), rows.numel()
        for h in range(Hq):
            hk = h * Hkv // Hq
            kk, vv, qq = k[live, hk].double(), v[live, hk].double(), q[rows, h].double()
            dd, oo = do[rows, h].double(), o[rows, h].double()
            s, l, p, es, el = _weights(qq, kk, scale)
            es = es + el
            dp = dd @ vv.t()
            delta = (p * dp).sum(1, keepdim=True)
            d0 = (dd * oo).sum(1, keepdim=True)
            ds = p * (dp - delta)
            # ds in 32 bits: the weight's error, dp's and delta's
            edp = U * (D + 4) * (dd.abs() @ vv.abs().t())
            edl = U * (D + 8) * (dd * oo).abs().sum(1, keepdim=True) + (p * edp).sum(1, keepdim=True)
            edl = edl + (p * es * (dp - d0).abs()).sum(1, keepdim=True)
            edl = edl + U * (n / 4 + 64) * (p * (dp - d0).abs()).sum(1, keepdim=True)
            if hp == 0:  # (delta is do.o of the rounded o as it is)
                edl = edl + (delta - d0).abs()
            eds = p * (es * (dp - delta).abs() + edp + edl) + 4 * U * ds.abs()
            eds = eds + FLUSH * (1 + (dp - delta).abs())
            s0, e0 = (p * (dp - d0)).abs(), (delta - d0).abs()
            add = U * (n / 4 + 64)
            # dq = scale (sum r k - (sum r) B) with B = sum p k, where r = ds' (1 + t), |t| <=
            # hp, are ds' = p (dp - d0) as they are rounded, and p is rounded in B.  sum ds' (k
            # - B) is dq's exact value (ds' differs from ds by p (delta - d0), and sum p (k - B)
            # = 0), so that what is off is sum ds' t (k - B), at most hp sum |ds'| (|k| + |B|),
            # and (sum r) times B's error, at most (e0 + hp sum |ds'|) hp sum p |k|.  fp32: hp =
            # 0, and B is of p and k rounded to bf16, each by 2^-8 of it at most, its sum in 32
            # bits: off by 2^-6.9 sum p |k|, times sum ds', e0 and what edl holds at most.  An
            # error of a ds' in 32 bits, eds, is in sum r as well, so it meets |k| + |B|.
            coarse = 2 ** -6.9 * (e0 + edl) if hp == 0 else 0.0
            B, pk, s1 = p @ kk, p @ kk.abs(), s0.sum(1, keepdim=True)
            q0 = s0 * s0
            spread = (q0 @ (kk * kk) - 2 * B * (q0 @ kk) + B * B * q0.sum(1, keepdim=True)).clamp(min=0)
            out["dq"].put((rows, h), scale * (ds @ kk), hp,
                          scale * (s0 @ kk.abs() + s1 * B.abs() + (e0 + hp * s1) * pk),
                          scale * (torch.sqrt(spread)
                                   + (e0 + hp * s1) * torch.sqrt((p * p) @ (kk * kk))),
                          scale * ((eds + add * (s0 + e0 * p)) @ kk.abs()
                                   + (add * s1 + eds.sum(1, keepdim=True) + coarse) * pk))
            add = U * (m / 4 + 64)
            out["dk"].put((live, hk), scale * (ds.t() @ qq), hp, scale * (ds.abs().t() @ qq.abs()),
                          scale * torch.sqrt((ds * ds).t() @ (qq * qq)),
                          scale * ((eds + add * ds.abs()).t() @ qq.abs()))
            out["dv"].put((live, hk), p.t() @ dd, hp, p.t() @ dd.abs(),
                          torch.sqrt((p * p).t() @ (dd * dd)),
                          (p * (es + add) + FLUSH).t() @ dd.abs())
    return out, tq, tk


# ---- dropout ----
def philox(counter, key):
    """Philox-4x32-10 of counters [n, 4] (uint64 arrays that hold 32-bit words)."""
    c = [np.asarray(counter, dtype=np.uint64)[:, i] for i in range(4)]
    k = [int(key[0]), int(key[1])]
    low, s32 = np.uint64(0xFFFFFFFF), np.uint64(32)
    for _ in range(10):
        a, b = c[0] * np.uint64(0xD2511F53), c[2] * np.uint64(0xCD9E8D57)
        c = [(b >> s32) ^ c[1] ^ np.uint64(k[0]), b & low, (a >> s32) ^ c[3] ^ np.uint64(k[1]),
             a & low]
        k = [(k[0] + 0x9E3779B9) & 0xFFFFFFFF, (k[1] + 0xBB67AE85) & 0xFFFFFFFF]
    return np.stack(c, 1)


def kept(e, p, seed, offset):
    """Whether the elements e (an int64 array) are kept, and the scale of those."""
    T = int(np.floor(65536 * p + 0.5))
    e = np.asarray(e, dtype=np.uint64)
    j, low = e // np.uint64(8), np.uint64(0xFFFFFFFF)
    ctr = np.stack([j & low, j >> np.uint64(32), np.full_like(j, offset & 0xFFFFFFFF),
                    np.full_like(j, (offset >> 32) & 0xFFFFFFFF)], 1)
    w = philox(ctr, (seed & 0xFFFFFFFF, (seed >> 32) & 0xFFFFFFFF))
    i = (e % np.uint64(8)).astype(np.int64)
    word = w[np.arange(len(e)), i // 2]
    bits = np.where(i % 2 == 0, word & np.uint64(0xFFFF), word >> np.uint64(16))
    return torch.from_numpy(bits.astype(np.int64) >= T), 65536 / (65536 - T)
