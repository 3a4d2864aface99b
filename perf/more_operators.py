"""Operators of a decoder that answers query points from an encoder's states, as
measurable cases: inputs, plain forms in elementary torch operations, necessary
work, and values in 64 bits.

Kinds of case:
  ask     attention of query points over the states of their request: requests are
          packed rows, each with its own number of queries and of states; forward,
          or its backward (back = True)
  drop    dropout from a counter-based generator with the residual add; forward, or
          its backward (back = True), which draws the same numbers again

The definitions, where they are not the usual ones:

ask     rows q_off[r] .. q_off[r+1] of q [Nq, Hq, D] attend to rows k_off[r] ..
        k_off[r+1] of k and v [Nk, Hkv, D]; Hq / Hkv query heads share a head of k
        and v.  s = scale q.k over the states whose mask is set; lse = log sum
        exp(s), o = sum exp(s - lse) v.  A row without a state has o = 0, lse =
        -inf and passes no gradient.  Rows behind q_off[R] (k_off[R]) belong to no
        request and are left as they were.
drop    out = r + y / (1 - P) where the element is kept, r where it is not; P = T /
        65536 with T = round(65536 p).  Element e is kept if its 16 bits are at
        least T: the (e % 2)-th half, lower first, of word (e % 8) / 2 of
        Philox-4x32-10 (Salmon et al., "Parallel random numbers: as easy as 1, 2,
        3", 2011) of the counter (e / 8, offset), 64 bits each, lower words first,
        with the key seed.
"""
import math

import torch

own = False

DEV = "cuda"


# --------------------------------------------------------------------------
# The cases
# --------------------------------------------------------------------------
def listed():
    return [
        # one query point of one geometry with 64 states: latency only
        {"name": "ask_1_bf16", "kind": "ask", "Nq": 1, "Nk": 64, "R": 1, "Hq": 8, "Hkv": 8,
         "D": 32, "dtype": "bf16", "mask": False, "fused": True, "back": False},
        # a probe point of each of 64 requests over the long caches of their states
        # (an encoder that keeps its points), heads shared
        {"name": "ask_64_requests_bf16", "kind": "ask", "Nq": 64, "Nk": 1000000, "R": 64,
         "Hq": 8, "Hkv": 2, "D": 64, "dtype": "bf16", "mask": False, "fused": True,
         "back": False},
        # a small batch of ragged requests in full precision, states left out, some
        # requests with nothing to answer or nothing to read
        {"name": "ask_ragged_f32", "kind": "ask", "Nq": 20003, "Nk": 1777, "R": 7, "Hq": 4,
         "Hkv": 4, "D": 16, "dtype": "f32", "mask": True, "fused": False, "back": False},
        # the million-point car surface queried from 64 states
        {"name": "ask_1m_bf16", "kind": "ask", "Nq": 1000000, "Nk": 64, "R": 1, "Hq": 8,
         "Hkv": 8, "D": 32, "dtype": "bf16", "mask": False, "fused": True, "back": False},
        # a mesh queried from another mesh's points: the products are the bound
        {"name": "ask_16k_bf16", "kind": "ask", "Nq": 16384, "Nk": 16384, "R": 1, "Hq": 4,
         "Hkv": 4, "D": 64, "dtype": "bf16", "mask": False, "fused": True, "back": False},
        # training: the backward of the million points
        {"name": "ask_back_1m_bf16", "kind": "ask", "Nq": 1000000, "Nk": 64, "R": 1, "Hq": 8,
         "Hkv": 8, "D": 32, "dtype": "bf16", "mask": False, "fused": True, "back": True},
        # of a mesh from another mesh's points, wide heads of which four share one
        {"name": "ask_back_8k_bf16", "kind": "ask", "Nq": 8192, "Nk": 8192, "R": 1, "Hq": 4,
         "Hkv": 1, "D": 128, "dtype": "bf16", "mask": True, "fused": True, "back": True},
        # of ragged requests in full precision, heads shared
        {"name": "ask_back_ragged_f32", "kind": "ask", "Nq": 6001, "Nk": 3333, "R": 9, "Hq": 4,
         "Hkv": 2, "D": 40, "dtype": "f32", "mask": True, "fused": True, "back": True},
        # one point's row: latency only
        {"name": "drop_1_bf16", "kind": "drop", "N": 1, "C": 256, "dtype": "bf16", "p": 0.1,
         "resid": True, "back": False},
        # the million-point car surface, with the residual stream
        {"name": "drop_1m_bf16", "kind": "drop", "N": 1000000, "C": 256, "dtype": "bf16",
         "p": 0.1, "resid": True, "back": False},
        # the backward at an odd width
        {"name": "drop_back_odd_f32", "kind": "drop", "N": 100003, "C": 95, "dtype": "f32",
         "p": 0.25, "resid": False, "back": True},
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    if rng.random() < 0.25:
        C = _log_int(rng, 1, 1030) if rng.random() < 0.5 else rng.choice([64, 96, 128, 256])
        back = rng.random() < 0.5
        return {"kind": "drop", "N": _log_int(rng, 1, min(1000000, (1 << 27) // C)), "C": C,
                "dtype": rng.choice(["bf16", "bf16", "f32"]),
                "p": rng.choice([0.05, 0.1, 0.25, 0.5]),
                "resid": not back and rng.random() < 0.7, "back": back}
    back, dt = rng.random() < 0.45, rng.choice(["bf16", "bf16", "f32"])
    D, Hkv = rng.choice([16, 24, 32, 32, 40, 64, 64, 80, 96, 128]), rng.choice([1, 2, 4, 8])
    Hq = Hkv * rng.choice([1, 1, 2, 4])
    while Hq * D > 1024:
        Hq, Hkv = (Hq // 2, Hkv // 2) if Hkv > 1 else (Hq // 2, 1)
    R = 1 if rng.random() < 0.5 else _log_int(rng, 2, 100)
    # points or meshes over few or many states, or a few points over long caches
    Nq = max(R, _log_int(rng, 1, 500000))
    # (of a lone state the gradients of q and k are nothing but zeros)
    least = 16 * R if back else R
    Nk = max(least, _log_int(rng, 1, 500000))
    # (pairs of a query and a state: by the products, and by the plain form's memory)
    most = min(((1 << 36) if dt == "bf16" else (1 << 32)) // (D * (4 if back else 1)),
               1 << 30) // Hq * R
    while Nq * Nk > most:
        if rng.random() < 0.5:
            Nq = max(R, Nq // 2)
        else:
            Nk = max(least, Nk // 2)
    Nq, Nk = min(Nq, (1 << 27) // (Hq * D)), min(Nk, (1 << 27) // (Hkv * D))
    return {"kind": "ask", "Nq": Nq, "Nk": Nk, "R": R, "Hq": Hq, "Hkv": Hkv, "D": D, "dtype": dt,
            "mask": rng.random() < 0.4, "fused": rng.random() < 0.5, "back": back}


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

    def uniform(self, *shape):
        return torch.rand(*shape, generator=self.g, device=DEV)


def _offsets(case):
    """(q_off, k_off): where the requests' rows begin and end.  The lengths differ by
    up to a factor of two; a few rows at the end belong to no request; of seven or
    more requests one has no queries and one no states."""
    R, Nq, Nk = case["R"], case["Nq"], case["Nk"]
    if R == 1:
        return [0, Nq], [0, Nk]

    def cut(N, phase, none):
        N -= 3 if N > 8 * R else 0
        if N < 2 * R:
            w = [1] * R
        else:
            w = [4 + (5 * r + phase) % 5 for r in range(R)]
            if R >= 7:
                w[none] = 0
        off, total, run = [0], sum(w), 0
        for x in w:
            run += x
            off.append(N * run // total)
        return off

    return cut(Nq, 1, 2), cut(Nk, 3, 4)


def _ask_inputs(case, seed):
    """Queries that find some states much nearer than others, states with a common
    part, and the gradient of a loss over the answers."""
    d, dt, D = _Draw(seed), _t(case["dtype"]), case["D"]
    Nq, Nk, Hq, Hkv = case["Nq"], case["Nk"], case["Hq"], case["Hkv"]
    i = {"q": d.normal(Nq, Hq, D).mul_(1.5).to(dt)}
    k = d.normal(Nk, Hkv, D).add_(0.3 * d.normal(Hkv, D)).to(dt)
    v = d.normal(Nk, Hkv, D).add_(0.5 * d.normal(Hkv, D)).to(dt)
    if case["fused"]:  # one product's rows hold both, side by side
        kv = torch.stack((k, v), 1)
        k, v = kv[:, 0], kv[:, 1]
    i.update(k=k, v=v)
    if case["mask"]:  # states left out; of several requests, all of the last one's
        i["mask"] = d.uniform(Nk) < 0.9
        if case["R"] > 1:
            i["mask"][_offsets(case)[1][-2]:] = False
    if case["back"]:
        i["do"] = d.normal(Nq, Hq, D).add_(0.5 * d.normal(Hq, D)).to(dt)
    return i


def _drop_inputs(case, seed):
    d, dt, N, C = _Draw(seed), _t(case["dtype"]), case["N"], case["C"]
    i = {"y": d.normal(N, C).mul_(torch.exp(0.5 * d.normal(C))).to(dt), "seed": 7919 * seed + 12345,
         "offset": 3 + seed % 5}
    if case["resid"]:
        i["r"] = d.normal(N, C, dtype=dt)
    return i


def prepare(case, seed):
    s = (_ask_inputs if case["kind"] == "ask" else _drop_inputs)(case, seed)
    s["case"] = case
    if own:
        from paper_2502_02414_amd import ops
        s["ops"] = ops
    if case["kind"] == "drop":
        s["out"] = torch.empty_like(s["y"])
        return s
    _plan(s)
    Nq, Nk, D = case["Nq"], case["Nk"], case["D"]
    s["o"] = torch.zeros_like(s["q"])
    s["lse"] = torch.zeros(case["Hq"], Nq, device=DEV)
    if case["back"]:  # what the forward left
        f = _ask_plain(s)
        s["o"], s["lse"] = f["o"].clone(), f["lse"].clone()
        s["dq"] = torch.zeros_like(s["q"])
        z = torch.zeros(Nk, 2, case["Hkv"], D, dtype=s["k"].dtype, device=DEV)
        s["dk"], s["dv"] = (z[:, 0], z[:, 1]) if case["fused"] else (z[:, 0].clone(),
                                                                    z[:, 1].clone())
    if own:
        several = case["R"] > 1
        s["par"] = ops.make_cross_attention(
            case["Hq"], case["Hkv"], D, q_off=s["q_off"] if several else None,
            k_off=s["k_off"] if several else None, mask=s.get("mask"), max_k=s["Lk"])
        s["ws"] = ops.cross_attention_workspace(s["par"], Nq, Nk, s["q"].dtype,
                                                backward=case["back"])
    return s


def _plan(s):
    """The requests' offsets and, for the plain form, the rows of a padded batch."""
    case = s["case"]
    qo, ko = _offsets(case)
    s["q_off"] = torch.tensor(qo, device=DEV)
    s["k_off"] = torch.tensor(ko, device=DEV)
    ql, kl = s["q_off"].diff(), s["k_off"].diff()
    s["Lq"], s["Lk"] = max(1, int(ql.max())), max(1, int(kl.max()))
    if case["R"] == 1:
        return
    pq, pk = torch.arange(s["Lq"], device=DEV), torch.arange(s["Lk"], device=DEV)
    s["q_on"], s["k_on"] = pq < ql[:, None], pk < kl[:, None]
    s["qi"] = torch.where(s["q_on"], s["q_off"][:-1, None] + pq, 0)
    s["ki"] = torch.where(s["k_on"], s["k_off"][:-1, None] + pk, 0)
    # the place of every row in the padded batch
    s["q_at"], s["k_at"] = s["q_on"].view(-1).nonzero()[:, 0], s["k_on"].view(-1).nonzero()[:, 0]


# --------------------------------------------------------------------------
# One pass
# --------------------------------------------------------------------------
def _queries(s, x):
    """Rows of the query side as [R, Hkv, Lq G, D] in 32 bits."""
    c = s["case"]
    G = c["Hq"] // c["Hkv"]
    x = x[s["qi"]] if c["R"] > 1 else x[None]
    x = x.float().view(c["R"], s["Lq"], c["Hkv"], G, c["D"]).transpose(1, 2)
    return x.reshape(c["R"], c["Hkv"], s["Lq"] * G, c["D"])


def _states(s, x, on):
    """Rows of the states as [R, Hkv, Lk, D] in 32 bits, zeros where they are left out."""
    x = x[s["ki"]] if s["case"]["R"] > 1 else x[None]
    x = x.float()
    if on is not None:
        x = torch.where(on[:, :, None, None], x, torch.zeros_like(x))
    return x.transpose(1, 2)


def _on(s):
    """Which states count, [R, Lk]."""
    on = s.get("mask")
    if s["case"]["R"] == 1:
        return None if on is None else on[None]
    return s["k_on"] if on is None else s["k_on"] & on[s["ki"]]


def _queries_back(s, x, out):
    """The inverse of _queries, rounded into the rows of out."""
    c = s["case"]
    G = c["Hq"] // c["Hkv"]
    x = x.view(c["R"], c["Hkv"], s["Lq"], G, -1).transpose(1, 2)
    x = x.reshape(c["R"] * s["Lq"], c["Hq"], -1)
    if c["R"] == 1:
        out.copy_(x)
    else:
        out[:s["q_at"].numel()] = x[s["q_at"]].to(out.dtype)


def _states_back(s, x, out):
    c = s["case"]
    x = x.transpose(1, 2).reshape(c["R"] * s["Lk"], c["Hkv"], -1)
    if c["R"] == 1:
        out.copy_(x)
    else:
        out[:s["k_at"].numel()] = x[s["k_at"]].to(out.dtype)


def _ask_plain(s):
    c, on = s["case"], _on(s)
    q, k, v = _queries(s, s["q"]), _states(s, s["k"], on), _states(s, s["v"], on)
    a = torch.matmul(q, k.transpose(2, 3).contiguous()).mul_(1 / math.sqrt(c["D"]))
    if on is not None:
        a.masked_fill_(~on[:, None, None, :], -math.inf)
    m = a.amax(3, keepdim=True)
    m = torch.where(m == -math.inf, torch.zeros_like(m), m)
    e = a.sub_(m).exp_()
    l = e.sum(3, keepdim=True)
    o = torch.matmul(e, v.contiguous()) / torch.where(l > 0, l, torch.ones_like(l))
    _queries_back(s, o, s["o"])
    _queries_back(s, m + torch.log(l), s["lse"].t().unsqueeze(2))
    return {"o": s["o"], "lse": s["lse"]}


def _ask_back_plain(s):
    c, on = s["case"], _on(s)
    scale = 1 / math.sqrt(c["D"])
    q, k, v = _queries(s, s["q"]), _states(s, s["k"], on), _states(s, s["v"], on)
    do = _queries(s, s["do"])
    a = torch.matmul(q, k.transpose(2, 3).contiguous()).mul_(scale)
    if on is not None:
        a.masked_fill_(~on[:, None, None, :], -math.inf)
    a = a.sub_(a.amax(3, keepdim=True).clamp_(min=-1e30)).exp_()
    l = a.sum(3, keepdim=True)
    p = a.div_(torch.where(l > 0, l, torch.ones_like(l)))
    if c["R"] > 1:  # (rows of the padded batch that are none)
        do = do * s["q_on"].repeat_interleave(c["Hq"] // c["Hkv"], 1)[:, None, :, None]
    dv = torch.matmul(p.transpose(2, 3), do)
    dp = torch.matmul(do, v.transpose(2, 3).contiguous())
    delta = (p * dp).sum(3, keepdim=True)
    ds = dp.sub_(delta).mul_(p).mul_(scale)
    _queries_back(s, torch.matmul(ds, k.contiguous()), s["dq"])
    _states_back(s, torch.matmul(ds.transpose(2, 3), q), s["dk"])
    _states_back(s, dv, s["dv"])
    return {"dq": s["dq"], "dk": s["dk"], "dv": s["dv"]}


def _philox(n, offset, seed):
    """Philox-4x32-10 of the counters (0 .. n - 1, offset), [n, 4]."""
    low = 0xFFFFFFFF
    c0 = torch.arange(n, device=DEV)
    c0, c1 = c0 & low, c0 >> 32
    c2, c3 = torch.full_like(c0, offset & low), torch.full_like(c0, offset >> 32)
    k0, k1 = seed & low, seed >> 32
    for _ in range(10):
        # (the products' 64 bits wrap into the sign, which the shift's mask takes off)
        a, b = c0 * 0xD2511F53, c2 * 0xCD9E8D57
        c0, c1, c2, c3 = (b >> 32 & low) ^ c1 ^ k0, b & low, (a >> 32 & low) ^ c3 ^ k1, a & low
        k0, k1 = (k0 + 0x9E3779B9) & low, (k1 + 0xBB67AE85) & low
    return torch.stack((c0, c1, c2, c3), 1)


def _drop_plain(s):
    c, y = s["case"], s["y"]
    n, T = y.numel(), round(65536 * c["p"])
    w = _philox(-(-n // 8), s["offset"], s["seed"])
    bits = torch.stack((w & 0xFFFF, w >> 16), 2).view(-1)[:n].view(y.shape)
    out = torch.where(bits >= T, y.float() * (65536 / (65536 - T)), torch.zeros((), device=DEV))
    if c["resid"]:
        out = out + s["r"].float()
    s["out"].copy_(out)
    return s["out"]


def run(s):
    case = s["case"]
    if case["kind"] == "drop":
        if not own:
            return _drop_plain(s)
        s["ops"].pa_dropout(s["y"], s["out"], case["p"], s["seed"], s["offset"], r=s.get("r"))
        return s["out"]
    if not own:
        return _ask_back_plain(s) if case["back"] else _ask_plain(s)
    if case["back"]:
        s["ops"].pa_cross_attention_backward(s["q"], s["k"], s["v"], s["o"], s["lse"], s["par"],
                                             s["do"], s["dq"], s["dk"], s["dv"], s["ws"])
        return {"dq": s["dq"], "dk": s["dk"], "dv": s["dv"]}
    s["ops"].pa_cross_attention(s["q"], s["k"], s["v"], s["par"], s["o"], s["lse"], s["ws"])
    return {"o": s["o"], "lse": s["lse"]}


# --------------------------------------------------------------------------
# Necessary work
# --------------------------------------------------------------------------
def work(case):
    b = 4 if case["dtype"] == "f32" else 2
    if case["kind"] == "drop":
        n = case["N"] * case["C"]
        # a counter's ten rounds of two products and six other steps give eight elements
        return {"bytes": n * b * (3 if case["resid"] else 2), "flops": n * (10 * 8 // 8 + 3)}
    Hq, Hkv, D, back = case["Hq"], case["Hkv"], case["D"], case["back"]
    qo, ko = _offsets(case)
    pairs = sum((qo[r + 1] - qo[r]) * (ko[r + 1] - ko[r]) for r in range(case["R"]))
    # q and o; for the backward q, o, do and dq: and k, v; dk and dv
    rows = qo[-1] * Hq * D * b * (4 if back else 2) + ko[-1] * Hkv * D * b * (4 if back else 2)
    return {"bytes": rows + 4 * Hq * qo[-1] + (ko[-1] if case["mask"] else 0),
            "flops": pairs * Hq * D * (10 if back else 4)}


# --------------------------------------------------------------------------
# Values in 64 bits
# --------------------------------------------------------------------------
def _exact_ask(case, i):
    qo, ko = _offsets(case)
    D, G, back = case["D"], case["Hq"] // case["Hkv"], case["back"]
    wide = lambda x: torch.zeros(x.shape, dtype=torch.float64, device=DEV)
    o, dk, dv = wide(i["q"]), wide(i["k"]), wide(i["v"])
    lse = torch.zeros(case["Hq"], case["Nq"], dtype=torch.float64, device=DEV)
    for r in range(case["R"]):
        rows, live = slice(qo[r], qo[r + 1]), torch.arange(ko[r], ko[r + 1], device=DEV)
        if "mask" in i:
            live = live[i["mask"][live]]
        if qo[r] == qo[r + 1]:
            continue
        if not live.numel():
            lse[:, rows] = -math.inf
            continue
        for h in range(case["Hkv"]):
            k = i["k"][live, h].double().requires_grad_(back)
            v = i["v"][live, h].double().requires_grad_(back)
            for g in range(h * G, h * G + G):
                q = i["q"][rows, g].double().requires_grad_(back)
                logits = (q @ k.t().contiguous()) / D ** 0.5
                out = torch.softmax(logits, 1) @ v
                if not back:
                    o[rows, g] = out
                    lse[g, rows] = torch.logsumexp(logits, 1)
                    continue
                a, b, c = torch.autograd.grad(out, (q, k, v), i["do"][rows, g].double())
                o[rows, g] = a
                dk[live, h] += b
                dv[live, h] += c
    return {"dq": o, "dk": dk, "dv": dv} if back else {"o": o, "lse": lse}


def _kept(n, T, offset, seed):
    """Which of n elements are kept, the generator's products by 16-bit halves."""
    M = 1 << 32
    j = torch.arange(-(-n // 8), dtype=torch.int64, device=DEV)
    x = [j % M, torch.div(j, M, rounding_mode="floor"), 0 * j + offset % M, 0 * j + offset // M]

    def times(u, m):
        """(upper, lower) 32 bits of u m."""
        p = [(u % 65536) * (m % 65536), (u % 65536) * (m // 65536), (u // 65536) * (m % 65536),
             (u // 65536) * (m // 65536)]
        mid = torch.div(p[0], 65536, rounding_mode="floor") + p[1] % 65536 + p[2] % 65536
        up = p[3] + p[1] // 65536 + p[2] // 65536 + mid // 65536
        return up, (mid % 65536) * 65536 + p[0] % 65536

    for t in range(10):
        key = [(seed % M + t * 0x9E3779B9) % M, (seed // M + t * 0xBB67AE85) % M]
        h0, l0 = times(x[0], 0xD2511F53)
        h1, l1 = times(x[2], 0xCD9E8D57)
        x = [h1 ^ x[1] ^ key[0], l1, h0 ^ x[3] ^ key[1], l0]
    halves = [w % 65536 if e % 2 == 0 else w // 65536 for w in x for e in (0, 1)]
    return (torch.stack(halves, 1) >= T).reshape(-1)[:n]


def _exact_drop(case, i):
    T = int(65536 * case["p"] + 0.5)
    keep = _kept(case["N"] * case["C"], T, i["offset"], i["seed"]).view(case["N"], case["C"])
    out = torch.where(keep, i["y"].double() / (1 - T / 65536), 0.0)
    return out + i["r"].double() if case["resid"] else out


def exact(case, seed):
    if case["kind"] == "drop":
        return _exact_drop(case, _drop_inputs(case, seed))
    return _exact_ask(case, _ask_inputs(case, seed))
