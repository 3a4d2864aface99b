"""Operators around the block stack as measurable cases: inputs, plain forms in
elementary torch operations, necessary work, and values in 64 bits.

Kinds of case:
  norm    the joint between a block and the next one: a norm after the block,
          its gate and residual scale, the residual add, and the norm before
          the next block; forward, or its backward (back = True)
  adamw   one AdamW step over all tensors of a block stack, moments in 32 or
          in 8 bits
  lin8    a linear layer in 8-bit integers: rows quantised with a scale each,
          an integer product with weights that have a scale per output
          channel, bias, GELU, residual add

The definitions, where they are not the usual ones:

norm    u = post(y); m = sigmoid(t) or 1; x1 = alpha x + scale m u, rounded to
        the storage type; h = pre(x1) of the rounded sum.  post and pre are
        LayerNorm, RMSNorm or nothing.  The backward takes the gradients of
        x1 (its use in the residual stream) and of h.
adamw   m <- b1 m + (1 - b1) g, v <- b2 v + (1 - b2) g^2 (g times a scale on
        the device, a clipping coefficient), p <- p - (lr wd p + lr / (1 -
        b1^step) m / (sqrt(v) / sqrt(1 - b2^step) + eps)).
        8 bits: blocks of 256 consecutive elements of a tensor; S is the
        smallest power of two that is not below a block's largest magnitude;
        a code c > 0 stands for S times the float whose upper 12 bits are c +
        889 (m; bit 7 of the code is the sign) or c + 761 (v), c = 0 for 0:
        3 mantissa bits, 16 or 32 octaves below S.  What is coded is the new
        moment in 32 bits, every product and sum above rounded to nearest:
        its magnitude over S becomes a code by adding 16 h + 8 to the float's
        bits, h 16 random bits, and dropping the lower 20 (an unbiased
        rounding); below the last code m becomes 0, a positive v the last
        code.  The random bits are murmur3's 32-bit finaliser over seed, step,
        tensor, block and element.
lin8    s_i = max_k |x_ik| / 127, q_ik = round-to-even(x_ik (127 / max)), the
        quotient and the product in 32 bits (a border between two integers is
        decided on that product); a row of zeros has q = s = 0;
        D_if = act(s_i sw_f sum_k q_ik wq_fk + b_f) + C_if.
"""
import math

import torch

own = False

DEV = "cuda"
EPS_LN, EPS_RMS = 1e-5, 1e-6
LR, B1, B2, EPS_ADAM = 1e-3, 0.9, 0.999, 1e-8
BLK = 256


# --------------------------------------------------------------------------
# The cases
# --------------------------------------------------------------------------
def listed():
    return [
        # one query point through a block's joint when serving: latency only
        {"name": "norm_1_bf16", "kind": "norm", "N": 1, "C": 256, "dtype": "bf16",
         "post": "layer", "pre": "layer", "gate": False, "alpha": 1.0, "back": False},
        # the backward on a small 2D field (64 x 64 points), full precision
        {"name": "norm_back_4k_f32", "kind": "norm", "N": 4096, "C": 64, "dtype": "f32",
         "post": "layer", "pre": "layer", "gate": False, "alpha": 1.0, "back": True},
        # a width that is no power of two, a ragged number of points, a gate
        {"name": "norm_100k_odd_bf16", "kind": "norm", "N": 100003, "C": 96, "dtype": "bf16",
         "post": "rms", "pre": "rms", "gate": True, "alpha": 0.75, "back": False},
        # the million-point car surface, forward
        {"name": "norm_1m_bf16", "kind": "norm", "N": 1000000, "C": 256, "dtype": "bf16",
         "post": "layer", "pre": "layer", "gate": False, "alpha": 1.0, "back": False},
        # its backward, with a gate
        {"name": "norm_back_1m_bf16", "kind": "norm", "N": 1000000, "C": 256, "dtype": "bf16",
         "post": "rms", "pre": "layer", "gate": True, "alpha": 1.0, "back": True},
        # the optimiser step of a small model's one block: launch bound
        {"name": "adamw_1_block_32", "kind": "adamw", "C": 64, "M": 16, "blocks": 1, "bits": 32,
         "g": "f32", "copy": False},
        # the eight-block aircraft model, moments in 8 bits, bf16 copies kept
        {"name": "adamw_8_blocks_8", "kind": "adamw", "C": 256, "M": 64, "blocks": 8, "bits": 8,
         "g": "f32", "copy": True},
        # a hundred million parameters, bf16 gradients, moments in 32 bits
        {"name": "adamw_100m_32", "kind": "adamw", "C": 1024, "M": 64, "blocks": 8, "bits": 32,
         "g": "bf16", "copy": True},
        # a single token: the weights are the traffic
        {"name": "lin8_1_bf16", "kind": "lin8", "N": 1, "K": 4096, "F": 4096, "x": "bf16",
         "out": "bf16", "gelu": False, "resid": False},
        # odd sizes throughout, full-precision rows
        {"name": "lin8_odd_f32", "kind": "lin8", "N": 333, "K": 1000, "F": 517, "x": "f32",
         "out": "f32", "gelu": False, "resid": True},
        # the first MLP product of the million-point model with its GELU
        {"name": "lin8_1m_up_bf16", "kind": "lin8", "N": 1000000, "K": 256, "F": 1024,
         "x": "bf16", "out": "bf16", "gelu": True, "resid": False},
        # a square product: the matrix cores are the bound
        {"name": "lin8_4k_bf16", "kind": "lin8", "N": 4096, "K": 4096, "F": 4096, "x": "bf16",
         "out": "bf16", "gelu": False, "resid": True},
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["norm", "adamw", "lin8"])
    if kind == "norm":
        dt = rng.choice(["bf16", "bf16", "f32"])
        C = 8 * _log_int(rng, 2, 512) if rng.random() < 0.5 else rng.choice([64, 96, 128, 256])
        cap = (1 << 27) if dt == "bf16" else (1 << 25)
        return {"kind": "norm", "N": _log_int(rng, 1, min(1000000, cap // C)), "C": C,
                "dtype": dt, "post": rng.choice(["layer", "rms", "none"]),
                "pre": rng.choice(["layer", "rms"]), "gate": rng.random() < 0.5,
                "alpha": rng.choice([1.0, 0.75, 1.5]), "back": rng.random() < 0.5}
    if kind == "adamw":
        bits = rng.choice([8, 32])
        C = rng.choice([32, 48, 64, 96, 128, 160, 256, 384])
        return {"kind": "adamw", "C": C, "M": rng.randint(4, 64), "blocks": rng.randint(1, 12),
                "bits": bits, "g": rng.choice(["f32", "bf16"]), "copy": rng.random() < 0.5}
    N = _log_int(rng, 1, 200000)
    K, F = _log_int(rng, 16, 4096), _log_int(rng, 16, 4096)
    if rng.random() < 0.5:
        K, F = 64 * max(1, K // 64), 64 * max(1, F // 64)
    N = max(1, min(N, (1 << 35) // (K * F), (1 << 28) // max(K, F)))
    dt = rng.choice(["bf16", "bf16", "f32"])
    return {"kind": "lin8", "N": N, "K": K, "F": F, "x": dt, "out": dt,
            "gelu": rng.random() < 0.4, "resid": rng.random() < 0.4}


# --------------------------------------------------------------------------
# Inputs
# --------------------------------------------------------------------------
def _t(name):
    return torch.float32 if name == "f32" else torch.bfloat16


class _Draw:
    """Seeded draws on the GPU."""

    def __init__(self, seed):
        self.g = torch.Generator(device=DEV)
        self.g.manual_seed(int(seed))

    def normal(self, *shape, dtype=torch.float32):
        return torch.randn(*shape, generator=self.g, device=DEV, dtype=torch.float32).to(dtype)

    def small(self, *shape):
        return 0.2 * (2 * torch.rand(*shape, generator=self.g, device=DEV) - 1)


def _norm_inputs(case, seed):
    """The residual stream, with a few channels much larger than the rest as
    trained networks have them, and a block's output beside it."""
    d, N, C, dt = _Draw(seed), case["N"], case["C"], _t(case["dtype"])
    chan = torch.exp(0.5 * d.normal(C))
    i = {"y": (d.normal(N, C) * chan + 0.3 * d.normal(C)).to(dt), "scale": 0.5 + d.small(C)}
    if case["post"] != "none":
        i["post_g"] = 1 + d.small(C)
    if case["post"] == "layer":
        i["post_b"] = d.small(C)
    i["pre_g"] = 1 + d.small(C)
    if case["pre"] == "layer":
        i["pre_b"] = d.small(C)
    if case["gate"]:
        i["t"] = d.normal(N, C, dtype=dt)
    x = (d.normal(N, C) * chan.flip(0) + d.normal(C)).to(dt)
    i["x1" if case["back"] else "x"] = x
    if case["back"]:  # a loss's gradient: a part common to the points, one per point
        i["dx1"] = (d.normal(N, C) + d.normal(C)).to(dt)
        i["dh"] = (d.normal(N, C) + d.normal(C)).to(dt)
    return i


def _stack_sizes(case):
    """(elements, decayed) of a block stack's tensors, block after block."""
    C, M = case["C"], case["M"]
    one = [(C, 0), (C, 0), (C * C, 1), (C, 0), (C * M, 1), (M, 0), (C, 0)]  # ln1, Project, slices
    one += [(C * C, 1), (C, 0)] * 4                                         # q, k, v, o
    one += [(C, 0), (C, 0), (4 * C * C, 1), (4 * C, 0), (4 * C * C, 1), (C, 0)]  # ln2, MLP
    return one * case["blocks"]


def _layout(case):
    """Tensors at multiples of 256 elements of flat buffers: offsets, sizes,
    decays, and the flat length."""
    off, out = 0, []
    for n, dec in _stack_sizes(case):
        out.append((off, n, 0.01 * dec))
        off += -(-n // BLK) * BLK
    return out, off


def _adamw_inputs(case, seed):
    d = _Draw(seed)
    lay, total = _layout(case)
    live = torch.zeros(total, device=DEV)
    for off, n, _ in lay:
        live[off:off + n] = 1
    # gradients whose size differs from element to element by orders of magnitude
    size = torch.exp(2 * d.normal(total) - 7)
    i = {"p": 0.1 * d.normal(total) * live, "g": (size * d.normal(total) * live).to(_t(case["g"])),
         "gscale": torch.full((1,), 0.7, device=DEV), "seed": 1000003 * (seed + 1),
         "step": 10 + seed % 7}
    m = 0.4 * size * d.normal(total) * live
    v = 0.01 * size * size * (0.1 + torch.rand(total, generator=d.g, device=DEV)) * live
    if case["bits"] == 32:
        i["m"], i["v"] = m, v
    else:
        i["mq"], i["ms"] = _encode(m.view(-1, BLK), None, True)
        i["vq"], i["vs"] = _encode(v.view(-1, BLK), None, False)
    if case["copy"]:
        i["copy"] = i["p"].to(torch.bfloat16)
    return i


def _lin8_inputs(case, seed):
    d, N, K, F = _Draw(seed), case["N"], case["K"], case["F"]
    # activations with heavier channels; weights of a trained layer's size
    x = (d.normal(N, K) * torch.exp(0.5 * d.normal(K))).to(_t(case["x"]))
    W = d.normal(F, K) * (torch.exp(0.3 * d.normal(F, 1)) / math.sqrt(K))
    amax = W.abs().amax(1)
    Kp = -(-K // 16) * 16
    wq = torch.zeros(F, Kp, dtype=torch.int8, device=DEV)   # rows padded to 16 bytes
    wq[:, :K] = torch.round(W * (127.0 / amax)[:, None]).to(torch.int8)
    i = {"x": x, "wq": wq, "sw": amax / 127.0, "b": d.small(F)}
    if case["resid"]:
        i["C"] = d.normal(N, F, dtype=_t(case["out"]))
    return i


def _inputs(case, seed):
    return {"norm": _norm_inputs, "adamw": _adamw_inputs, "lin8": _lin8_inputs}[case["kind"]](
        case, seed)


def prepare(case, seed):
    s = _inputs(case, seed)
    s["case"] = case
    if not own:
        return s
    from paper_2502_02414_amd import ops
    s["ops"] = ops
    if case["kind"] == "norm":
        N, C, dt = case["N"], case["C"], _t(case["dtype"])
        e = lambda: torch.empty(N, C, dtype=dt, device=DEV)
        s["par"] = ops.make_residual_norm_params(
            post=case["post"], pre=case["pre"], alpha=case["alpha"], scale=s["scale"],
            gate="sigmoid", post_g=s.get("post_g"), post_b=s.get("post_b"), pre_g=s["pre_g"],
            pre_b=s.get("pre_b"), post_eps=EPS_LN if case["post"] == "layer" else EPS_RMS,
            pre_eps=EPS_LN if case["pre"] == "layer" else EPS_RMS)
        if not case["back"]:
            s["o"] = {"x1": e(), "h": e()}
        else:
            f = lambda k: torch.empty(C, dtype=torch.float32, device=DEV)
            s["o"] = {"dx": e(), "dy": e()}
            if case["gate"]:
                s["o"]["dt"] = e()
            gr = {"d" + k: f(k) for k in _GAINS if k in s}
            s["o"].update(gr)
            s["gr"] = ops.make_residual_norm_grads(**gr)
            s["ws"] = ops.residual_norm_workspace(N, C, dt)
    elif case["kind"] == "adamw":
        lay, total = _layout(case)
        keys = [k for k in ("p", "g", "m", "v", "copy") if k in s]
        items = []
        for off, n, wd in lay:
            it = {k: s[k][off:off + n] for k in keys}
            it["wd"] = wd
            if case["bits"] == 8:
                b0, b1 = off // BLK, -(-(off + n) // BLK)
                it.update(m=s["mq"].view(-1)[off:off + n], v=s["vq"].view(-1)[off:off + n],
                          m_scale=s["ms"][b0:b1], v_scale=s["vs"][b0:b1])
            items.append(it)
        s["items"] = ops.make_adamw_items(items)
        if case["bits"] == 8:
            s["mo"], s["vo"] = torch.empty_like(s["p"]), torch.empty_like(s["p"])
    else:
        N, K, F = case["N"], case["K"], case["F"]
        s["D"] = torch.empty(N, F, dtype=_t(case["out"]), device=DEV)
        s["ws"] = ops.linear_i8_workspace(N, K, F)
    return s


# --------------------------------------------------------------------------
# One pass
# --------------------------------------------------------------------------
_GAINS = ("post_g", "post_b", "scale", "pre_g", "pre_b")


def _stats(x, kind, eps):
    """The centred row and 1 / its size."""
    if kind == "layer":
        x = x - x.mean(1, keepdim=True)
    return x, torch.rsqrt((x * x).mean(1, keepdim=True) + eps)


def _norm_plain(s):
    c = s["case"]
    dt, alpha = _t(c["dtype"]), c["alpha"]
    y = s["y"].float()
    eps = {"layer": EPS_LN, "rms": EPS_RMS}
    if c["post"] != "none":
        yc, ry = _stats(y, c["post"], eps[c["post"]])
        yhat = yc * ry
        u = yhat * s["post_g"]
        if "post_b" in s:
            u = u + s["post_b"]
    else:
        u = y
    gate = 1 / (1 + torch.exp(-s["t"].float())) if "t" in s else None
    mu = u if gate is None else gate * u
    if not c["back"]:
        x1 = (alpha * s["x"].float() + s["scale"] * mu).to(dt)
        xc, rx = _stats(x1.float(), c["pre"], eps[c["pre"]])
        h = xc * rx * s["pre_g"]
        if "pre_b" in s:
            h = h + s["pre_b"]
        return {"x1": x1, "h": h.to(dt)}
    xc, rx = _stats(s["x1"].float(), c["pre"], eps[c["pre"]])
    xhat = xc * rx
    dh = s["dh"].float()
    o = {"dpre_g": (dh * xhat).sum(0)}
    if "pre_b" in s:
        o["dpre_b"] = dh.sum(0)
    gh = dh * s["pre_g"]
    e = gh - xhat * (gh * xhat).mean(1, keepdim=True)
    if c["pre"] == "layer":
        e = e - gh.mean(1, keepdim=True)
    e = s["dx1"].float() + rx * e
    o["dx"] = (alpha * e).to(dt)
    o["dscale"] = (e * mu).sum(0)
    du = s["scale"] * e
    if gate is not None:
        o["dt"] = (du * u * gate * (1 - gate)).to(dt)
        du = du * gate
    if c["post"] == "none":
        o["dy"] = du.to(dt)
        return o
    o["dpost_g"] = (du * yhat).sum(0)
    if "post_b" in s:
        o["dpost_b"] = du.sum(0)
    gu = du * s["post_g"]
    dy = gu - yhat * (gu * yhat).mean(1, keepdim=True)
    if c["post"] == "layer":
        dy = dy - gu.mean(1, keepdim=True)
    o["dy"] = (ry * dy).to(dt)
    return o


def _fmix(h):
    """murmur3's 32-bit finaliser on int64 tensors that hold 32-bit values."""
    k = 0xFFFFFFFF
    h = ((h ^ (h >> 16)) * 0x85EBCA6B) & k
    h = ((h ^ (h >> 13)) * 0xC2B2AE35) & k
    return h ^ (h >> 16)


def _mix(a, b):
    return _fmix(a ^ ((b * 0x9E3779B9) & 0xFFFFFFFF))


def _random_bits(case, seed, step):
    """32 random bits for every element of the flat buffers, [blocks, 256]."""
    lay, total = _layout(case)
    item, blk = [], []
    for k, (_, n, _) in enumerate(lay):
        nb = -(-n // BLK)
        item.append(torch.full((nb,), k, dtype=torch.int64))
        blk.append(torch.arange(nb))
    item, blk = torch.cat(item).to(DEV), torch.cat(blk).to(DEV)
    word = lambda x: torch.tensor(x & 0xFFFFFFFF, dtype=torch.int64, device=DEV)
    key = _mix(_mix(word(seed), word(seed >> 32)), word(step))
    kb = _mix(_mix(key, item), blk)
    return _fmix((kb[:, None] + torch.arange(BLK, device=DEV)) & 0xFFFFFFFF)


def _encode(x, h, signed):
    """Codes and block scales of x [blocks, 256]; h: 16 random bits per
    element (None: the middle)."""
    big = x.abs().amax(1)
    bits = big.view(torch.int32)
    up = (bits & 0x7F800000) + torch.where((bits & 0x7FFFFF) > 0, 0x800000, 0)
    S = up.clamp(min=0x00800000, max=0x7F000000).to(torch.int32).view(torch.float32)
    S = torch.where(big > 0, S, torch.zeros_like(S))
    a = x.abs() * torch.where(S > 0, 1 / S, torch.zeros_like(S))[:, None]
    add = 16 * h.to(torch.int32) + 8 if h is not None else 0x80000
    lo, hi = (889, 127) if signed else (761, 255)
    c = ((a.view(torch.int32) + add) >> 20) - lo
    if signed:
        c = c.clamp(0, hi) + torch.where(x < 0, 128, 0)
        c = torch.where((c & 127) == 0, 0, c)
    else:
        c = torch.where(x > 0, c.clamp(1, hi), 0)
    return c.to(torch.uint8), S


def _decode(c, S, signed):
    c = c.to(torch.int32)
    mag = c & 127 if signed else c
    val = ((mag + (889 if signed else 761)) << 20).view(torch.float32)
    val = torch.where(mag > 0, val, torch.zeros_like(val))
    if signed:
        val = torch.where(c > 127, -val, val)
    return val * S[:, None]


def _decays(case):
    return torch.cat([torch.full((-(-n // BLK),), wd) for _, n, wd in _layout(case)[0]]).to(DEV)


def _adamw_plain(s):
    case = s["case"]
    q8 = case["bits"] == 8
    g = s["g"].float().mul(s["gscale"]).view(-1, BLK)
    m = _decode(s["mq"], s["ms"], True) if q8 else s["m"].view(-1, BLK)
    v = _decode(s["vq"], s["vs"], False) if q8 else s["v"].view(-1, BLK)
    m = m * B1 + g * (1 - B1)
    v = v * B2 + (g * g) * (1 - B2)
    den = v.sqrt() * (1 / math.sqrt(1 - B2 ** s["step"])) + EPS_ADAM
    p = s["p"].view(-1, BLK)
    p.sub_((LR * _decays(case))[:, None] * p + (LR / (1 - B1 ** s["step"])) * (m / den))
    o = {"p": s["p"]}
    if case["copy"]:
        s["copy"].copy_(s["p"])
        o["copy"] = s["copy"]
    if not q8:
        s["m"].copy_(m.view(-1))
        s["v"].copy_(v.view(-1))
        o["m"], o["v"] = s["m"], s["v"]
    else:
        h = _random_bits(case, s["seed"], s["step"])
        s["mq"], s["ms"] = _encode(m, h & 0xFFFF, True)
        s["vq"], s["vs"] = _encode(v, h >> 16, False)
        o["m"] = _decode(s["mq"], s["ms"], True).view(-1)
        o["v"] = _decode(s["vq"], s["vs"], False).view(-1)
    return o


def _erf_gelu(x):
    return 0.5 * x * (1 + torch.erf(x * math.sqrt(0.5)))


def _lin8_plain(s):
    c = s["case"]
    x, out = s["x"], []
    rows = max(1, (1 << 28) // max(c["K"], c["F"]))
    w = s["wq"][:, :c["K"]].float().t().contiguous()
    for r in range(0, c["N"], rows):
        xr = x[r:r + rows].float()
        big = xr.abs().amax(1, keepdim=True)
        # (one division: torch forms 127.0 / big from a rounded reciprocal)
        per = torch.div(torch.full_like(big, 127.0), big)
        q = torch.round(xr * torch.where(big > 0, per, torch.zeros_like(big)))
        D = (q @ w) * ((big / 127.0) * s["sw"]) + s["b"]
        if c["gelu"]:
            D = _erf_gelu(D)
        if c["resid"]:
            D = D + s["C"][r:r + rows].float()
        out.append(D.to(_t(c["out"])))
    return out[0] if len(out) == 1 else torch.cat(out)


def run(s):
    case = s["case"]
    kind = case["kind"]
    if kind == "adamw":
        s["step"] += 1
    if not own:
        return {"norm": _norm_plain, "adamw": _adamw_plain, "lin8": _lin8_plain}[kind](s)
    ops = s["ops"]
    if kind == "norm":
        o = s["o"]
        if not case["back"]:
            ops.pa_residual_norm(s["x"], s["y"], s["par"], o["x1"], o["h"], t=s.get("t"))
        else:
            ops.pa_residual_norm_backward(s["x1"], s["y"], s["par"], s["dx1"], s["dh"], o["dx"],
                                          o["dy"], s["gr"], s["ws"], t=s.get("t"),
                                          dt=o.get("dt"))
        return o
    if kind == "adamw":
        ops.pa_adamw(s["items"], lr=LR, beta1=B1, beta2=B2, eps=EPS_ADAM, step=s["step"],
                     gscale=s["gscale"], seed=s["seed"])
        o = {"p": s["p"]}
        if case["copy"]:
            o["copy"] = s["copy"]
        if case["bits"] == 32:
            o["m"], o["v"] = s["m"], s["v"]
        else:  # the values that the codes stand for
            ops.pa_adamw_unpack(s["mq"], s["ms"], s["mo"], signed=True)
            ops.pa_adamw_unpack(s["vq"], s["vs"], s["vo"], signed=False)
            o["m"], o["v"] = s["mo"], s["vo"]
        return o
    ops.pa_linear_i8(s["x"], s["wq"], s["sw"], s["D"], s["ws"], bias=s["b"],
                     act="gelu" if case["gelu"] else "none", C=s.get("C"))
    return s["D"]


# --------------------------------------------------------------------------
# Necessary work
# --------------------------------------------------------------------------
def work(case):
    kind = case["kind"]
    if kind == "norm":
        n, b = case["N"] * case["C"], 4 if case["dtype"] == "f32" else 2
        if case["back"]:  # x1, y, dx1, dh, t; dx, dy, dt; the gains and their gradients
            return {"bytes": n * b * (8 if case["gate"] else 6) + 40 * case["C"], "flops": 45 * n}
        return {"bytes": n * b * (5 if case["gate"] else 4) + 20 * case["C"], "flops": 20 * n}
    if kind == "adamw":
        n = sum(k for k, _ in _stack_sizes(case))
        b = 8 + (4 if case["g"] == "f32" else 2) + (2 if case["copy"] else 0)
        # 8 bits: codes and scales read and written, and the values given back
        b += 16 if case["bits"] == 32 else 4 + 16 / BLK + 8
        return {"bytes": int(n * b), "flops": 15 * n}
    N, K, F = case["N"], case["K"], case["F"]
    bx, bo = 4 if case["x"] == "f32" else 2, 4 if case["out"] == "f32" else 2
    return {"bytes": N * K * bx + F * K + 8 * F + N * F * bo * (2 if case["resid"] else 1),
            "flops": 2 * N * K * F}


# --------------------------------------------------------------------------
# Values in 64 bits
# --------------------------------------------------------------------------
def _exact_norm(case, i):
    f = {k: v.double() for k, v in i.items()}
    N, C = case["N"], case["C"]

    def unit(z, kind):
        if kind == "layer":
            mean = z.sum(1, keepdim=True) / C
            var = ((z - mean) ** 2).sum(1, keepdim=True) / C
            r = (var + EPS_LN) ** -0.5
            return (z - mean) * r, r
        r = ((z ** 2).sum(1, keepdim=True) / C + EPS_RMS) ** -0.5
        return z * r, r

    def pull_back(zh, r, d, kind):
        """The gradient of z from that of its unit form zh."""
        k = d - zh * (d * zh).sum(1, keepdim=True) / C
        return r * (k - d.sum(1, keepdim=True) / C) if kind == "layer" else r * k

    sig = torch.sigmoid(f["t"]) if case["gate"] else torch.ones(1, 1, dtype=torch.float64,
                                                                device=DEV)
    if case["post"] == "none":
        yh, ry, u = f["y"], None, f["y"]
    else:
        yh, ry = unit(f["y"], case["post"])
        u = yh * f["post_g"] + f.get("post_b", 0.0)
    if not case["back"]:
        x1 = case["alpha"] * f["x"] + f["scale"] * sig * u
        stored = x1.to(_t(case["dtype"])).double()
        h = unit(stored, case["pre"])[0] * f["pre_g"] + f.get("pre_b", 0.0)
        return {"x1": x1, "h": h}
    xh, rx = unit(f["x1"], case["pre"])
    e = f["dx1"] + pull_back(xh, rx, f["dh"] * f["pre_g"], case["pre"])
    o = {"dx": case["alpha"] * e}
    du = e * f["scale"] * sig
    o["dy"] = du if ry is None else pull_back(yh, ry, du * f["post_g"], case["post"])
    if case["gate"]:
        o["dt"] = e * f["scale"] * u * sig * torch.sigmoid(-f["t"])
    if "post_g" in f:
        o["dpost_g"] = (du * yh).sum(0)
    if "post_b" in f:
        o["dpost_b"] = du.sum(0)
    o["dscale"] = (e * sig * u).sum(0)
    o["dpre_g"] = (f["dh"] * xh).sum(0)
    if "pre_b" in f:
        o["dpre_b"] = f["dh"].sum(0)
    return o


def _exact_adamw(case, i):
    step = i["step"] + 1
    lay, total = _layout(case)
    o = {k: torch.zeros(total, dtype=torch.float64, device=DEV)
         for k in ("p", "copy", "m", "v") if k != "copy" or case["copy"]}

    def near(z):
        """The nearest float of 32 bits."""
        z = z if torch.is_tensor(z) else torch.tensor(z, dtype=torch.float64, device=DEV)
        return z.float().double()

    def mix(a, b=None):
        """One word after another into 32 bits."""
        if b is not None:
            a = a ^ (b * 0x9E3779B9 % (1 << 32))
        for shift, mul in ((16, 0x85EBCA6B), (13, 0xC2B2AE35)):
            a = (a ^ (a >> shift)) * mul % (1 << 32)
        return a ^ (a >> 16)

    def value(c, S, top):
        """The value of a code: octave and eighth below S."""
        k = c.double()
        octave = torch.floor((k - top) / 8)
        eighth = (k - top) - 8 * octave
        return torch.where(k > 0, S * torch.exp2(octave) * (1 + eighth / 8), 0 * k)

    def coded(x, bits, top):
        """The value that x [blocks, 256] is stored as."""
        big = x.abs().amax(1, keepdim=True)
        S = torch.exp2(torch.ceil(torch.log2(big.clamp(min=2.0 ** -126))))
        S = torch.where(big > 0, S, torch.zeros_like(S))
        a = torch.where(S > 0, x.abs() / S.clamp(min=2.0 ** -126), torch.zeros_like(x))
        _, ex = torch.frexp(a)                        # a = fraction 2^ex, fraction in [1/2, 1)
        octave = (ex - 1).double()
        eighths = (a / torch.exp2(octave) - 1) * 8     # in [0, 8)
        k = top + 8 * octave + torch.floor(eighths + (16 * bits + 8).double() / 2 ** 20)
        k = torch.where(a > 0, k.clamp(min=1.0 if top == 255 else 0.0, max=float(top)), 0 * k)
        return torch.sign(x) * value(k, S, top)

    word = lambda z: torch.tensor(z % (1 << 32), dtype=torch.int64, device=DEV)
    key = mix(mix(word(i["seed"]), word(i["seed"] >> 32)), word(step))
    for k, (off, n, wd) in enumerate(lay):
        sl = slice(off, off + -(-n // BLK) * BLK)
        g = i["g"][sl].double() * i["gscale"].double()
        if case["bits"] == 32:
            m, v = i["m"][sl].double(), i["v"][sl].double()
        else:
            bl = slice(sl.start // BLK, sl.stop // BLK)
            mc = i["mq"][bl].to(torch.int64)
            m = value(mc % 128, i["ms"][bl, None].double(), 127) * torch.where(mc > 127, -1.0, 1.0)
            v = value(i["vq"][bl], i["vs"][bl, None].double(), 255)
            m, v = m.reshape(-1), v.reshape(-1)
        if case["bits"] == 32:
            m = B1 * m + (1 - B1) * g
            v = B2 * v + (1 - B2) * g ** 2
        else:  # the moments that are coded, rounded after every operation
            m = near(near(near(B1) * m) + near(near(1 - B1) * near(g)))
            v = near(near(near(B2) * v) + near(near(1 - B2) * near(near(g) ** 2)))
        upd = (m / (1 - B1 ** step)) / (torch.sqrt(v / (1 - B2 ** step)) + EPS_ADAM)
        p = i["p"][sl].double()
        o["p"][sl] = p - LR * wd * p - LR * upd
        if case["bits"] == 8:
            nb = m.numel() // BLK
            kb = mix(mix(key, word(k)), torch.arange(nb, device=DEV))
            h = mix((kb[:, None] + torch.arange(BLK, device=DEV)) % (1 << 32))
            m = coded(m.view(nb, BLK), h % 65536, 127).reshape(-1)
            v = coded(v.view(nb, BLK), h // 65536, 255).reshape(-1)
        o["m"][sl], o["v"][sl] = m, v
    if case["copy"]:
        o["copy"] = o["p"]
    return o


def _exact_lin8(case, i):
    N, K, F = case["N"], case["K"], case["F"]
    D = torch.empty(N, F, dtype=torch.float64, device=DEV)
    w = i["wq"][:, :K].double() * i["sw"].double()[:, None]
    for r in range(0, N, 65536):
        x = i["x"][r:r + 65536].double()
        top = x.abs().max(1, keepdim=True).values
        unit = top / 127
        # the integers: the quotient and the product rounded to 32 bits, then to even
        per = (127 / top).float().double()
        q = torch.where(top > 0, torch.round((x * per).float().double()), torch.zeros_like(x))
        y = torch.matmul(q * unit, w.t().contiguous()) + i["b"].double()
        if case["gelu"]:
            y = y * 0.5 * torch.erfc(-y / math.sqrt(2.0))
        if case["resid"]:
            y = y + i["C"][r:r + 65536].double()
        D[r:r + 65536] = y
    return D


def exact(case, seed):
    i = _inputs(case, seed)
    return {"norm": _exact_norm, "adamw": _exact_adamw, "lin8": _exact_lin8}[case["kind"]](case, i)
