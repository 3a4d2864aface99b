"""A stack of Transolver++ blocks, forward and backward, through the C ABI.

A block is the Transformer block with Physics-Attention in place of
attention (Section 3; the block diagram of Figure 2a), read as pre-norm with
residual adds:

    x1 = x + PA(LN1(x)),    x2 = x1 + GELU(LN2(x1) W1 + b1) W2 + b2,

where PA starts with Algorithm 1's Project step x_proj = h Wp + bp.  The
Project step is folded: the slice parameters become A' = Wp A, b' = b + bp A,
a' = Wp a, b_t' = b_t + bp.a (pa_project_fold), the layer's streaming calls
run on h = LN1(x), and the states are projected, S_proj = S Wp + bp
(pa_project_states), before the token attention (whose optional Wo, bo is
the layer's output projection).  x_proj is never formed.

Every step is a call of libpa.so (the layer's calls, LayerNorm with the
residual add fused, the Project folding, the MLP's first product with its
GELU as one kernel (bf16; fp32 storage: a hipBLASLt GEMM and the GELU
kernel), and hipBLASLt GEMMs for the rest of the MLP, whose second GEMM
adds the residual).  torch only allocates the device buffers.  Per layer the
forward keeps x, LN1(x), x1, LN2(x1), GELU(u) (the backward's weight
gradient of W2 reads it) and the small per-layer state for the backward;
the pre-activation u is recomputed by the backward's fused kernel from
LN2(x1) (bf16; fp32 storage keeps u).

``infer`` is the forward alone, with nothing kept, and after ``quantize`` the
MLP's products in 8-bit integers (ops.pa_linear_i8).  ``SandwichStack`` has a
norm after each half of a block as well, and learned residual scales.  A
training step is ``forward``, ``backward`` and a step of ``adamw``'s optimizer.
``QueryDecoder`` answers at points of its own from the states that an encoder left (a
stack's points, say), for many requests at once.

Parameters per layer (dict of device tensors): fp32 ln1_g, ln1_b, Wp [C,C],
bp [C], A [C,M], b [M], a [C], Wq, bq, Wk, bk, Wv, bv (optional Wo, bo),
ln2_g, ln2_b, b1 [4C], b2 [C]; W1 [C,4C] and W2 [4C,C] in the storage dtype;
plus b_t: a float, which training leaves as it is, or an fp32 device tensor [1].
"""
from __future__ import annotations

import weakref

from . import binding as B
from . import ops

ATTN = ("Wq", "bq", "Wk", "bk", "Wv", "bv", "Wo", "bo")


class BlockStack:
    def __init__(self, N, C, H, M, params, dtype, tau0=0.5, tau_min=0.01, eps=1e-5,
                 ln_eps=1e-5, device="cuda"):
        import torch
        self.torch = torch
        self.N, self.C, self.H, self.M = N, C, H, M
        self.params = params
        self.dt = dtype                       # torch dtype of the point-side tensors
        self.pdt = B.PA_BF16 if dtype == torch.bfloat16 else B.PA_F32
        self.ln_eps = ln_eps
        self.dims = B.make_dims(N, C, H, M, tau0, tau_min, eps, self.pdt)
        self.ws = B.workspace(self.dims, device)
        # scratch of the sums over rows (LayerNorm gains, bias gradients) and of hipBLASLt
        self.ws_rows = torch.empty(1024 * 4 * C, dtype=torch.float32, device=device)
        self.ws_gemm = torch.empty(256 << 20, dtype=torch.uint8, device=device)
        self.tuned = set()  # GEMM problems already tuned (pa_gemm_prepare)
        # bf16: the MLP's first product and GELU as one kernel (pa_mlp_up)
        self.fused_mlp = self.pdt == B.PA_BF16 and C in (64, 128, 256)
        self.dev = device
        self.ws_int8 = None
        self.int8 = None  # per layer: W1 and W2 as integers with scales (quantize)
        self.int8_of = None  # what they were made from
        self.steps = 0  # of the optimizers that adamw has made

    # -- helpers ------------------------------------------------------------
    def _e(self, *shape, dt=None):
        return self.torch.empty(*shape, dtype=dt or self.dt, device=self.dev)

    def _f(self, *shape):
        return self.torch.empty(*shape, dtype=self.torch.float32, device=self.dev)

    def _gemm(self, A, Bm, D, **kw):
        # each GEMM problem is tuned once, on its first call (pa_gemm_prepare
        # synchronises); later calls never synchronise
        key = (tuple(A.shape), A.dtype, tuple(Bm.shape), Bm.dtype, D.dtype,
               tuple(sorted((k, v if isinstance(v, (bool, float, int)) else v is not None)
                            for k, v in kw.items())))
        first = key not in self.tuned
        self.tuned.add(key)
        B.pa_gemm(A, Bm, D, ws=self.ws_gemm, prepare=first, **kw)

    def _folded(self, p):
        """The folded slice parameters of a layer (pa_project_fold)."""
        C, M = self.C, self.M
        A_f, a_f = self._e(C, M), self._e(C)
        b_f, bt_f, b_t = self._f(M), self._f(1), p.get("b_t", 0.0)
        B.pa_project_fold(self.dims, p["Wp"], p["bp"], p["A"], p.get("b"), p.get("a"), A_f, b_f,
                          a_f, bt_f)
        tensor = self.torch.is_tensor(b_t)
        if tensor and b_t.numel() != 1:
            raise ValueError(f"b_t: {b_t.numel()} elements, it is one")
        if tensor and b_t.dtype == self.torch.float32 and b_t.device.type in str(self.dev):
            # (added on the device, so that nothing waits for it; others are read as floats)
            both, b_t = (bt_f, b_t), 0.0
            pair, bt_f = self._f(2), self._f(1)
            for i, t in enumerate(both):
                B.pa_heads_expand(t, pair[i:i + 1], 1, False)
            B.pa_heads_sum(pair, bt_f, 2, False)
        sp = B.make_slice_params(A_f, b_f, a_f, b_t, b_t_dev=bt_f)
        return {"A": A_f, "b": b_f, "a": a_f, "bt": bt_f, "sp": sp}

    def named_parameters(self):
        """{"<layer>.<name>": tensor} of every trained tensor (b_t among them where it
        is one)."""
        return {f"{l}.{k}": v for l, p in enumerate(self.params) for k, v in p.items()
                if self.torch.is_tensor(v)}

    def adamw(self, lr, **kw):
        """ops.AdamW over the stack's parameters: those in bf16 (W1, W2) as fp32
        ones whose rounded copies are the stack's.  step(named_grads(grads)), which
        refuses to go on where a parameter of the stack is another tensor by then, or
        W1 or W2 have been written (then ``refresh`` of the optimizer first)."""
        named = self.named_parameters()
        f32 = self.torch.float32
        copies = {k: v for k, v in named.items() if v.dtype != f32}
        where = {f"{l}.{k}": (p, k) for l, p in enumerate(self.params) for k in p}

        def after():
            self.steps += 1

        return ops.AdamW({k: v.float() if k in copies else v for k, v in named.items()}, lr,
                         copies=copies, where={k: where[k] for k in named}, after=after, **kw)

    @staticmethod
    def named_grads(grads):
        """The gradients of ``backward`` by the names of ``named_parameters``."""
        return {f"{l}.{k[1:]}": v for l, g in enumerate(grads) for k, v in g.items()}

    # -- the halves of a block ------------------------------------------------
    def _attention(self, p, c, h, G):
        """PA(h) [N,C]; c receives what the backward needs."""
        N, C, M = self.N, self.C, self.M
        fo = self._folded(p)
        num, den, S, S_proj, Sp = self._f(M, C), self._f(M), self._f(M, C), self._f(M, C), \
            self._f(M, C)
        B.pa_slice_aggregate(self.dims, h, G, fo["sp"], num, den, S, self.ws)
        B.pa_project_states(self.dims, S, p["Wp"], p["bp"], S_proj)
        apr = B.make_attn_params(**{k: p[k] for k in ATTN if p.get(k) is not None})
        B.pa_token_attention(self.dims, S_proj, apr, Sp, self.ws)
        y = self._e(N, C)
        B.pa_deslice(self.dims, h, G, fo["sp"], Sp, y, self.ws)
        c.update({"h": h, "G": G, "fold": fo, "num": num, "den": den, "S": S, "S_proj": S_proj,
                  "Sp": Sp, "apr": apr})
        return y

    def _attention_backward(self, p, c, g, dY):
        """The gradient of h from that of PA(h); g receives the parameters'."""
        N, C, M = self.N, self.C, self.M
        # Physics-Attention on h with the folded Project step
        fo = c["fold"]
        dSp, dS_proj = self._f(M, C), self._f(M, C)
        B.pa_deslice_backward(self.dims, c["h"], c["G"], fo["sp"], dY, dSp, self.ws)
        ag = {k: self._f(C, C) for k in ("dWq", "dWk", "dWv")}
        ag.update({k: self._f(C) for k in ("dbq", "dbk", "dbv")})
        if p.get("Wo") is not None:
            ag["dWo"], ag["dbo"] = self._f(C, C), self._f(C)
        B.pa_token_attention_backward(self.dims, c["S_proj"], c["apr"], dSp, dS_proj,
                                      B.make_attn_grads(**ag), self.ws)
        g.update(ag)
        dS = self._f(M, C)
        self._gemm(dS_proj, p["Wp"], dS, transB=True)         # dS = dS_proj Wp^T
        gf = {"dA": self._f(C, M), "db": self._f(M), "da": self._f(C), "db_t": self._f(1),
              "dtau0": self._f(1)}
        dh = self._e(N, C)
        B.pa_slice_aggregate_backward(self.dims, c["h"], c["G"], fo["sp"], c["num"], c["den"],
                                      dS, c["Sp"], dY, dh, B.make_slice_grads(**gf), self.ws)
        g["dWp"], g["dbp"] = self._f(C, C), self._f(C)
        g.update({"dA": self._f(C, M), "db": self._f(M), "da": self._f(C),
                  "db_t": self._f(1)})
        B.pa_project_backward(self.dims, p["Wp"], p["bp"], p["A"], p.get("a"), c["S"], dS_proj,
                              B.make_slice_grads(**gf), g["dWp"], g["dbp"], None,
                              B.make_slice_grads(dA=g["dA"], db=g["db"], da=g["da"],
                                                 db_t=g["db_t"]))
        return dh

    def _mlp(self, p, c, h2, x1=None):
        """GELU(h2 W1 + b1) W2 + b2 (+ x1: the second residual add in the GEMM)."""
        N, C = self.N, self.C
        gu = self._e(N, 4 * C)
        if self.fused_mlp:
            # GELU(h2 W1 + b1) in one kernel; u is recomputed in the backward
            u = None
            B.pa_mlp_up(h2, p["W1"], p["b1"], gu, self.ws_gemm)
        else:
            u = self._e(N, 4 * C)
            self._gemm(h2, p["W1"], u, bias=p["b1"])
            B.pa_gelu(u, gu)
        x2 = self._e(N, C)
        if x1 is not None:
            self._gemm(gu, p["W2"], x2, bias=p["b2"], beta=1.0, C=x1)
        else:
            self._gemm(gu, p["W2"], x2, bias=p["b2"])
        c.update({"h2": h2, "u": u, "gu": gu})
        return x2

    def _mlp_backward(self, p, c, g, dy):
        """The gradient of h2 from that of the MLP's output; g receives the
        parameters'."""
        N, C = self.N, self.C
        gu = c.pop("gu")                                       # GELU(u), kept by the forward
        g["dW2"] = self._f(4 * C, C)
        self._gemm(gu, dy, g["dW2"], transA=True)
        g["db2"] = self._f(C)
        B.pa_colsum(dy, g["db2"], self.ws_rows)
        if self.fused_mlp:                                     # du, in place of gu
            B.pa_mlp_up_backward(c["h2"], p["W1"], p["b1"], dy, p["W2"], gu, self.ws_gemm)
        else:
            self._gemm(dy, p["W2"], gu, transB=True)          # dGELU(u), in place of gu
            B.pa_gelu_backward(c["u"], gu, gu)                 # du
        g["dW1"] = self._f(C, 4 * C)
        self._gemm(c["h2"], gu, g["dW1"], transA=True)
        g["db1"] = self._f(4 * C)
        B.pa_colsum(gu, g["db1"], self.ws_rows)
        dh2 = self._e(N, C)
        self._gemm(gu, p["W1"], dh2, transB=True)
        return dh2

    # -- forward ------------------------------------------------------------
    def forward(self, x, Gs):
        """x [N,C] (storage dtype), Gs: one Gumbel tensor [N,M] (or None) per
        layer.  Returns the output [N,C]; keeps what the backward needs."""
        N, C = self.N, self.C
        self.caches = []
        for p, G in zip(self.params, Gs):
            c = {"x": x}
            h, m1, r1 = self._e(N, C), self._f(N), self._f(N)
            B.pa_layernorm(x, h, m1, r1, g=p["ln1_g"], b=p["ln1_b"], eps=self.ln_eps)
            y = self._attention(p, c, h, G)
            # x1 = x + y (the first residual add) fused into LN2
            x1, h2, m2, r2 = self._e(N, C), self._e(N, C), self._f(N), self._f(N)
            B.pa_layernorm(x, h2, m2, r2, g=p["ln2_g"], b=p["ln2_b"], r=y, xs=x1, eps=self.ln_eps)
            del y
            # x2 = x1 + GELU(u) W2 + b2
            x = self._mlp(p, c, h2, x1)
            c.update({"m1": m1, "r1": r1, "x1": x1, "m2": m2, "r2": r2})
            self.caches.append(c)
        return x

    # -- backward -----------------------------------------------------------
    def backward(self, dy):
        """dy [N,C]: the gradient of the stack's output.  Returns (dx,
        [grads per layer]) with fp32 parameter gradients named d<param>."""
        N, C = self.N, self.C
        grads = [None] * len(self.params)
        for l in reversed(range(len(self.params))):
            p, c = self.params[l], self.caches[l]
            g = {}
            # MLP: x2 = x1 + GELU(u) W2 + b2
            dh2 = self._mlp_backward(p, c, g, dy)
            dx1 = self._e(N, C)
            g["dln2_g"], g["dln2_b"] = self._f(C), self._f(C)
            B.pa_layernorm_backward(c["x1"], c["m2"], c["r2"], dh2, dx1, g=p["ln2_g"], dres=dy,
                                    dg=g["dln2_g"], db=g["dln2_b"], ws=self.ws_rows)
            del dh2
            dh = self._attention_backward(p, c, g, dx1)       # dY = dx1
            # LN1 and the first residual: dx = LN1'(dh) + dx1
            dx = self._e(N, C)
            g["dln1_g"], g["dln1_b"] = self._f(C), self._f(C)
            B.pa_layernorm_backward(c["x"], c["m1"], c["r1"], dh, dx, g=p["ln1_g"], dres=dx1,
                                    dg=g["dln1_g"], db=g["dln1_b"], ws=self.ws_rows)
            grads[l] = g
            dy = dx
        return dy, grads

    # -- inference ------------------------------------------------------------
    def _weights(self):
        return [p[k] for p in self.params for k in ("W1", "W2")]

    def quantize(self):
        """The MLP's weights in 8-bit integers with a scale per output channel, for
        ``infer``; again after the weights have changed: ``infer`` refuses integers of
        weights that were written since (by torch, or a step of ``adamw``'s optimizer; of
        a replayed graph's it cannot know) or of tensors that are others by then.  Every
        call writes the same tensors, so that an ``infer`` in a graph replays with the
        integers of the moment."""
        if self.int8 is None:
            self.int8 = [(*ops.empty_weight(p["W1"]), *ops.empty_weight(p["W2"]))
                         for p in self.params]
        self.int8_of = None
        for p, (w1, s1, w2, s2) in zip(self.params, self.int8):
            ops.pa_quant_weight(p["W1"], w1, s1)
            ops.pa_quant_weight(p["W2"], w2, s2)
        # (how often they were written: by adamw's optimizers, and by torch)
        self.int8_of = self.steps, [(weakref.ref(t), ops.version(t)) for t in self._weights()]
        if self.ws_int8 is None:
            self.ws_int8 = ops.linear_i8_workspace(self.N, 4 * self.C, self.C, self.dev)

    def _ready(self):
        if self.int8 is None:
            return
        steps, of = self.int8_of or (None, ())  # (None: a quantize that did not end)
        if steps != self.steps or any(ref() is not t or n != ops.version(t)
                                      for (ref, n), t in zip(of, self._weights())):
            raise ValueError("the weights have changed since quantize: call it again")

    def _mlp_infer(self, l, h2, x1=None):
        p, N, C = self.params[l], self.N, self.C
        if self.int8 is None:
            return self._mlp(p, {}, h2, x1)
        w1, s1, w2, s2 = self.int8[l]
        gu, x2 = self._e(N, 4 * C), self._e(N, C)
        ops.pa_linear_i8(h2, w1, s1, gu, self.ws_int8, bias=p["b1"], act="gelu")
        ops.pa_linear_i8(gu, w2, s2, x2, self.ws_int8, bias=p["b2"], C=x1)
        return x2

    def infer(self, x, Gs):
        """``forward`` with nothing kept for a backward and, after ``quantize``, the
        MLP in 8-bit integers."""
        self._ready()
        N, C = self.N, self.C
        m, r = self._f(N), self._f(N)
        for l, (p, G) in enumerate(zip(self.params, Gs)):
            h = self._e(N, C)
            B.pa_layernorm(x, h, m, r, g=p["ln1_g"], b=p["ln1_b"], eps=self.ln_eps)
            y = self._attention(p, {}, h, G)
            x1, h2 = self._e(N, C), h
            B.pa_layernorm(x, h2, m, r, g=p["ln2_g"], b=p["ln2_b"], r=y, xs=x1, eps=self.ln_eps)
            x = self._mlp_infer(l, h2, x1)
        return x


class SandwichStack(BlockStack):
    """Blocks with a norm before and after each half and a learned scale of
    each half's way into the residual stream:

        x1 = x + rs1 * post1(PA(LN1(x))),    x2 = x1 + rs2 * post2(MLP(LN2(x1)))

    Each residual add, the norm before it and the one that follows (LN2; the next
    block's LN1) are one pa_residual_norm call, forward and backward.  ``post``:
    "layer" or "rms".  A layer's parameters have rs1, rs2 [C], post1_g, post2_g
    [C] and, for "layer", post1_b, post2_b [C] (fp32) as well; gradients drs1,
    dpost1_g, ...  LN1 and LN2 are LayerNorms as in BlockStack."""

    def __init__(self, *args, post="rms", post_eps=1e-5, **kw):
        super().__init__(*args, **kw)
        if post not in ("layer", "rms"):
            raise ValueError("post must be \"layer\" or \"rms\"")
        self.post, self.post_eps = post, post_eps
        self.ws_joint = ops.residual_norm_workspace(self.N, self.C, self.dt, self.dev)

    def _joint(self, l, k):
        """Joint 1 of layer l: after its attention, before its MLP; joint 2: after its
        MLP, before the next layer (the last one: nothing after it)."""
        p = self.params[l]
        pre = (p, "ln2") if k == 1 else (self.params[l + 1], "ln1") if l + 1 < len(self.params) \
            else None
        kw = {}
        if pre is not None:
            kw = {"pre": "layer", "pre_g": pre[0][pre[1] + "_g"], "pre_b": pre[0][pre[1] + "_b"],
                  "pre_eps": self.ln_eps}
        return ops.make_residual_norm_params(
            post=self.post, post_g=p[f"post{k}_g"], post_b=p.get(f"post{k}_b"),
            post_eps=self.post_eps, scale=p[f"rs{k}"], **kw)

    def _first_norm(self, x, m, r):
        h, p = self._e(self.N, self.C), self.params[0]
        B.pa_layernorm(x, h, m, r, g=p["ln1_g"], b=p["ln1_b"], eps=self.ln_eps)
        return h

    def forward(self, x, Gs):
        N, C = self.N, self.C
        self.caches = []
        m, r = self._f(N), self._f(N)
        self.first = (x, m, r)
        h = self._first_norm(x, m, r)
        for l, (p, G) in enumerate(zip(self.params, Gs)):
            c = {}
            y = self._attention(p, c, h, G)
            x1, h2 = self._e(N, C), self._e(N, C)
            ops.pa_residual_norm(x, y, self._joint(l, 1), x1, h2)
            z = self._mlp(p, c, h2)
            last = l + 1 == len(self.params)
            x, h = self._e(N, C), None if last else self._e(N, C)
            ops.pa_residual_norm(x1, z, self._joint(l, 2), x, h)
            c.update({"y": y, "x1": x1, "z": z, "x2": x})
            self.caches.append(c)
        return x

    def _joint_backward(self, l, k, grads, x1, y, dx1, dh):
        """Through joint k of layer l: (dx, dy); its parameters' gradients into the
        layer's, and the next layer's, dicts."""
        N, C = self.N, self.C
        dx, dy = self._e(N, C), self._e(N, C)
        out = {"drs%d" % k: "dscale", "dpost%d_g" % k: "dpost_g"}
        if self.post == "layer":
            out["dpost%d_b" % k] = "dpost_b"
        kw = {}
        for name, field in out.items():
            kw[field] = grads[l][name] = self._f(C)
        if dh is not None:
            to, ln = (grads[l], "ln2") if k == 1 else (grads[l + 1], "ln1")
            kw["dpre_g"] = to[f"d{ln}_g"] = self._f(C)
            kw["dpre_b"] = to[f"d{ln}_b"] = self._f(C)
        ops.pa_residual_norm_backward(x1, y, self._joint(l, k), dx1, dh, dx, dy,
                                      ops.make_residual_norm_grads(**kw), self.ws_joint)
        return dx, dy

    def backward(self, dy):
        N, C = self.N, self.C
        grads = [{} for _ in self.params]
        dx, dh = dy, None  # of the residual stream, and of the norm before the next layer
        for l in reversed(range(len(self.params))):
            p, c, g = self.params[l], self.caches[l], grads[l]
            dx, dz = self._joint_backward(l, 2, grads, c["x2"], c["z"], dx, dh)
            dh2 = self._mlp_backward(p, c, g, dz)
            dx, dya = self._joint_backward(l, 1, grads, c["x1"], c["y"], dx, dh2)
            dh = self._attention_backward(p, c, g, dya)
        x, m, r = self.first
        out, g = self._e(N, C), grads[0]
        g["dln1_g"], g["dln1_b"] = self._f(C), self._f(C)
        B.pa_layernorm_backward(x, m, r, dh, out, g=self.params[0]["ln1_g"], dres=dx,
                                dg=g["dln1_g"], db=g["dln1_b"], ws=self.ws_rows)
        return out, grads

    def infer(self, x, Gs):
        self._ready()
        N, C = self.N, self.C
        h = self._first_norm(x, self._f(N), self._f(N))
        for l, (p, G) in enumerate(zip(self.params, Gs)):
            y = self._attention(p, {}, h, G)
            x1, h2 = self._e(N, C), h
            if self.int8 is None:
                ops.pa_residual_norm(x, y, self._joint(l, 1), x1, h2)
                z = self._mlp(p, {}, h2)
            else:  # the norm writes the MLP's input as integers
                hq = self.torch.empty(N, ops.padded(C), dtype=self.torch.int8, device=self.dev)
                hs = self._f(N)
                ops.pa_residual_norm(x, y, self._joint(l, 1), x1, None, hq=hq, hs=hs)
                w1, s1, w2, s2 = self.int8[l]
                gu, z = self._e(N, 4 * C), y
                ops.pa_gemm_i8(hq, hs, w1, s1, gu, K=C, bias=p["b1"], act="gelu")
                ops.pa_linear_i8(gu, w2, s2, z, self.ws_int8, bias=p["b2"])
            last = l + 1 == len(self.params)
            x = self._e(N, C)
            ops.pa_residual_norm(x1, z, self._joint(l, 2), x, None if last else h)
        return x


class QueryDecoder(BlockStack):
    """Blocks that answer at query points from an encoder's states, s [Ns,Cs] in the
    storage dtype, for one request or many.  A block stack's states are the points that
    its ``forward`` or ``infer`` answers (their gradient, of ``backward`` here, goes into
    the stack's ``backward``; the states of its slices stay inside of it); a caller's own
    encoder may leave any number of any width:

        x1 = x + drop(Ask(LN1(x), s) Wo + bo),    x2 = x1 + drop(MLP(LN2(x1)))

    where Ask is ops.pa_cross_attention of q = h Wq + bq over k, v = s Wkv + bkv (side
    by side in the rows of one product) and drop is ops.pa_dropout with the residual
    add.  N query points of C channels in all, H query heads, Hkv heads of k and v
    (default: H), each C / H wide (a multiple of 8, up to 128); drop: the probability
    that training drops an element with, seed: of its numbers.

    Parameters per layer: ln1_g, ln1_b, bq [C], bkv [2 Hkv C / H], bo, ln2_g, ln2_b, b1
    [4C], b2 fp32; Wq [C,C], Wkv [Cs, 2 Hkv C / H], Wo [C,C], W1 [C,4C], W2 [4C,C] in the
    storage dtype (Cs: the states' width)."""

    def __init__(self, N, C, H, params, dtype, Hkv=None, drop=0.0, seed=0, ln_eps=1e-5,
                 device="cuda"):
        import torch
        self.torch = torch
        Hkv = H if Hkv is None else Hkv
        if H < 1 or Hkv < 1 or C % H or H % Hkv:
            raise ValueError("H must divide C, and Hkv H")
        if C // H % 8 or not 8 <= C // H <= 128:
            raise ValueError("C / H must be a multiple of 8, up to 128")
        self.N, self.C, self.H, self.Hkv, self.D = N, C, H, Hkv, C // H
        self.params, self.dt, self.ln_eps, self.dev = params, dtype, ln_eps, device
        self.pdt = B.PA_BF16 if dtype == torch.bfloat16 else B.PA_F32
        self.drop, self.seed = drop, seed
        self.ws_rows = torch.empty(1024 * 4 * C, dtype=torch.float32, device=device)
        self.ws_gemm = torch.empty(256 << 20, dtype=torch.uint8, device=device)
        self.tuned = set()
        self.fused_mlp = self.pdt == B.PA_BF16 and C in (64, 128, 256)
        self.ws_int8 = self.int8 = self.int8_of = None
        self.steps = 0
        self.one = ops.make_cross_attention(H, Hkv, self.D)

    def requests(self, q_off, k_off, mask=None, max_k=0):
        """Which query points ask which states (ops.make_cross_attention)."""
        return ops.make_cross_attention(self.H, self.Hkv, self.D, q_off=q_off, k_off=k_off,
                                        mask=mask, max_k=max_k)

    def _kv(self, p, s):
        kv = self._e(s.shape[0], 2, self.Hkv, self.D)
        if s.shape[0]:
            self._gemm(s, p["Wkv"], kv.view(s.shape[0], -1), bias=p["bkv"])
        return kv

    def _ask(self, p, c, h, kv, par, lse=False):
        """Ask(h) Wo + bo; c receives what the backward needs."""
        N, H, D = self.N, self.H, self.D
        q, o = self._e(N, self.C), self._e(N, H, D)
        self._gemm(h, p["Wq"], q, bias=p["bq"])
        l = self._f(H, N) if lse else None
        ws = ops.cross_attention_workspace(par, N, kv.shape[0], self.dt, device=self.dev)
        if par.tensors["q_off"] is not None:
            o.zero_()  # (a point of no request asks nothing)
            if lse:
                l.zero_()
        ops.pa_cross_attention(q.view(N, H, D), kv[:, 0], kv[:, 1], par, o, l, ws)
        y = self._e(N, self.C)
        self._gemm(o.view(N, -1), p["Wo"], y, bias=p["bo"])
        c.update({"q": q, "kv": kv, "o": o, "lse": l})
        return y

    def _ask_backward(self, p, c, g, s, par, dy, ds, first):
        """The gradient of h from that of Ask(h) Wo + bo; the states' goes into ds (added,
        but for the first)."""
        N, C, H, D = self.N, self.C, self.H, self.D
        do, dq = self._e(N, C), self._e(N, C)
        o, kv = c["o"], c["kv"]
        Ns, F = kv.shape[0], 2 * self.Hkv * D
        g["dWo"], g["dbo"] = self._f(C, C), self._f(C)
        self._gemm(o.view(N, C), dy, g["dWo"], transA=True)
        B.pa_colsum(dy, g["dbo"], self.ws_rows)
        self._gemm(dy, p["Wo"], do, transB=True)
        dkv = self._e(Ns, 2, self.Hkv, D)
        if par.tensors["q_off"] is not None:
            dq.zero_()
            dkv.zero_()
        ws = ops.cross_attention_workspace(par, N, Ns, self.dt, True, self.dev)
        v3 = lambda t: t.view(N, H, D)
        ops.pa_cross_attention_backward(v3(c["q"]), kv[:, 0], kv[:, 1], o, c["lse"], par, v3(do),
                                        v3(dq), dkv[:, 0], dkv[:, 1], ws)
        g["dWq"], g["dbq"] = self._f(C, C), self._f(C)
        self._gemm(c["h"], dq, g["dWq"], transA=True)
        B.pa_colsum(dq, g["dbq"], self.ws_rows)
        dh = do
        self._gemm(dq, p["Wq"], dh, transB=True)
        g["dWkv"], g["dbkv"] = self._f(s.shape[1], F), self._f(F)
        if Ns:
            dkv = dkv.view(Ns, F)
            self._gemm(s, dkv, g["dWkv"], transA=True)
            B.pa_colsum(dkv, g["dbkv"], self.ws_rows)
            self._gemm(dkv, p["Wkv"], ds, transB=True, beta=0.0 if first else 1.0)
        else:
            g["dWkv"].zero_()
            g["dbkv"].zero_()
        return dh

    def _add(self, y, x, l, k):
        """x + drop(y), the k-th of layer l."""
        out, (at, dev) = self._e(self.N, self.C), self.at
        ops.pa_dropout(y, out, self.drop, self.seed, at + 2 * l + k, r=x, offset_dev=dev)
        return out

    def _drop_grad(self, dy, l, k):
        if not self.drop:
            return dy
        out, (at, dev) = self._e(self.N, self.C), self.at
        ops.pa_dropout(dy, out, self.drop, self.seed, at + 2 * l + k, offset_dev=dev)
        return out

    def forward(self, x, s, par=None, step=0, offset_dev=None):
        """x [N,C], s [Ns,Cs]: the answers [N,C]; par: which points ask which states
        (``requests``; None: all of them all).  step: of the training, names the dropped
        elements.  Those of a captured graph, whose step stands still, are named by
        offset_dev, a device int64 [1] that counts 2 x layers a step (its own numbers follow
        step's: 0 there) and that ``backward`` reads again, so that it moves on behind that.
        Keeps what the backward needs."""
        N, C = self.N, self.C
        par = self.one if par is None else par
        self.caches, self.states, self.par = [], s, par
        self.at = (2 * len(self.params) * step, offset_dev)
        for l, p in enumerate(self.params):
            h, m1, r1 = self._e(N, C), self._f(N), self._f(N)
            c = {"x": x, "h": h, "m1": m1, "r1": r1}
            B.pa_layernorm(x, h, m1, r1, g=p["ln1_g"], b=p["ln1_b"], eps=self.ln_eps)
            y = self._ask(p, c, h, self._kv(p, s), par, lse=True)
            h2, m2, r2 = self._e(N, C), self._f(N), self._f(N)
            if self.drop:
                x1 = self._add(y, x, l, 0)
                B.pa_layernorm(x1, h2, m2, r2, g=p["ln2_g"], b=p["ln2_b"], eps=self.ln_eps)
                x = self._add(self._mlp(p, c, h2), x1, l, 1)
            else:
                x1 = self._e(N, C)
                B.pa_layernorm(x, h2, m2, r2, g=p["ln2_g"], b=p["ln2_b"], r=y, xs=x1,
                               eps=self.ln_eps)
                x = self._mlp(p, c, h2, x1)
            c.update({"x1": x1, "m2": m2, "r2": r2})
            self.caches.append(c)
        return x

    def backward(self, dy):
        """From the gradient of the answers: (dx, the states' gradient, [gradients per
        layer])."""
        N, C = self.N, self.C
        s, par, L = self.states, self.par, len(self.params)
        grads, ds = [None] * L, self._e(*s.shape)
        if not L:
            ds.zero_()
        for l in reversed(range(L)):
            p, c, g = self.params[l], self.caches[l], {}
            dh2 = self._mlp_backward(p, c, g, self._drop_grad(dy, l, 1))
            dx1 = self._e(N, C)
            g["dln2_g"], g["dln2_b"] = self._f(C), self._f(C)
            B.pa_layernorm_backward(c["x1"], c["m2"], c["r2"], dh2, dx1, g=p["ln2_g"], dres=dy,
                                    dg=g["dln2_g"], db=g["dln2_b"], ws=self.ws_rows)
            dh = self._ask_backward(p, c, g, s, par, self._drop_grad(dx1, l, 0), ds, l == L - 1)
            dx = self._e(N, C)
            g["dln1_g"], g["dln1_b"] = self._f(C), self._f(C)
            B.pa_layernorm_backward(c["x"], c["m1"], c["r1"], dh, dx, g=p["ln1_g"], dres=dx1,
                                    dg=g["dln1_g"], db=g["dln1_b"], ws=self.ws_rows)
            grads[l], dy = g, dx
        return dy, ds, grads

    def keep(self, s):
        """k and v of every layer for states that many calls of ``infer`` ask."""
        return [self._kv(p, s) for p in self.params]

    def infer(self, x, s=None, par=None, kept=None):
        """``forward`` without dropout, nothing kept for a backward; of the states s, or of
        what ``keep`` made of them; after ``quantize`` with the MLP in 8-bit integers."""
        self._ready()
        N, C = self.N, self.C
        par = self.one if par is None else par
        m, r = self._f(N), self._f(N)
        for l, p in enumerate(self.params):
            h = self._e(N, C)
            B.pa_layernorm(x, h, m, r, g=p["ln1_g"], b=p["ln1_b"], eps=self.ln_eps)
            y = self._ask(p, {}, h, self._kv(p, s) if kept is None else kept[l], par)
            x1, h2 = self._e(N, C), h
            B.pa_layernorm(x, h2, m, r, g=p["ln2_g"], b=p["ln2_b"], r=y, xs=x1, eps=self.ln_eps)
            x = self._mlp_infer(l, h2, x1)
        return x
