"""The operators of include/pa_ops.h together, as the block stack uses them: a
training step (SandwichStack forward and backward, AdamW), and inference with
the MLP in 8-bit integers."""
import numpy as np
import pytest
import torch

import ops_ref as R
from paper_2502_02414_amd import ops
from paper_2502_02414_amd.stack import BlockStack, SandwichStack
from pa_cases import say
from test_gpu_ops import check_step

pytestmark = pytest.mark.gpu

F32, BF16 = torch.float32, torch.bfloat16


def make(N, C, M, L, dt, kind=BlockStack, seed=0, **kw):
    g = torch.Generator()
    g.manual_seed(seed)
    rnd = lambda *s, scale=1.0: scale * torch.randn(*s, generator=g)
    ps = []
    for _ in range(L):
        p = {"Wp": rnd(C, C, scale=C ** -0.5), "bp": rnd(C, scale=0.1), "A": rnd(C, M, scale=C ** -0.5),
             "b": rnd(M, scale=0.1), "a": rnd(C, scale=0.02 * C ** -0.5),
             "ln1_g": 1 + rnd(C, scale=0.1), "ln1_b": rnd(C, scale=0.1),
             "ln2_g": 1 + rnd(C, scale=0.1), "ln2_b": rnd(C, scale=0.1),
             "b1": rnd(4 * C, scale=0.1), "b2": rnd(C, scale=0.1),
             "W1": rnd(C, 4 * C, scale=C ** -0.5).to(dt), "W2": rnd(4 * C, C, scale=0.5 * C ** -0.5).to(dt)}
        for n in "qkvo":
            p["W" + n], p["b" + n] = rnd(C, C, scale=C ** -0.5), rnd(C, scale=0.1)
        if kind is SandwichStack:
            for k in "12":
                p["rs" + k] = 0.5 + rnd(C, scale=0.1)
                p[f"post{k}_g"] = 1 + rnd(C, scale=0.1)
                if kw.get("post") == "layer":
                    p[f"post{k}_b"] = rnd(C, scale=0.1)
        p = {k: v.cuda() for k, v in p.items()}
        p["b_t"] = 0.5
        ps.append(p)
    x = rnd(N, C).to(dt).cuda()
    Gs = [-torch.log(-torch.log(torch.rand(N, M, generator=g).clamp(1e-6, 1 - 1e-6))).to(dt).cuda()
          for _ in range(L)]
    return kind(N, C, 4, M, ps, dt, **kw), x, Gs, rnd(N, C).to(dt).cuda()


@pytest.mark.parametrize("post", ["rms", "layer"])
def test_sandwich_joins_as_its_parts(post):
    """Forward: each joint against 64 bits on the tensors that the stack kept."""
    s, x, Gs, _ = make(777, 64, 16, 2, F32, SandwichStack, post=post)
    out = s.forward(x, Gs)
    cpu = lambda t: None if t is None else t.cpu()
    for l, c in enumerate(s.caches):
        p = {k: cpu(v) for k, v in s.params[l].items() if torch.is_tensor(v)}
        before = x if l == 0 else s.caches[l - 1]["x2"]
        for k, (xi, y, x1) in enumerate(((before, c["y"], c["x1"]), (c["x1"], c["z"], c["x2"])), 1):
            q = {"post": post, "post_g": p[f"post{k}_g"], "post_b": p.get(f"post{k}_b"),
                 "scale": p[f"rs{k}"]}
            ref, err = R.joint(q, cpu(xi), cpu(y))
            off = (cpu(x1).double() - ref).abs()
            assert (off <= R.U * (err + ref.abs())).all(), (l, k)
        q = {"pre": "layer", "pre_g": p["ln2_g"], "pre_b": p["ln2_b"]}
        ref, err = R.pre(q, cpu(c["x1"]))
        assert ((cpu(c["h2"]).double() - ref).abs() <= R.U * (err + ref.abs())).all(), l
    assert torch.equal(out, s.caches[-1]["x2"])
    assert torch.equal(s.infer(x, Gs), out)


def test_sandwich_reads_the_parameters_of_the_moment():
    """A tensor put in a parameter's place after the stack was made."""
    s, x, Gs, dy = make(500, 64, 16, 2, F32, SandwichStack)
    fresh, *_ = make(500, 64, 16, 2, F32, SandwichStack, seed=1)
    for kind in ("rs1", "rs2", "post1_g", "post2_g", "ln1_g", "ln2_b"):
        for p, q in zip(s.params, fresh.params):
            p[kind] = q[kind].clone()
    t = SandwichStack(500, 64, 4, 16, s.params, F32)
    t.tuned = s.tuned  # (each would choose the products' algorithms by its own timing)
    assert torch.equal(s.infer(x, Gs), t.infer(x, Gs))
    assert torch.equal(s.forward(x, Gs), t.forward(x, Gs))
    for a, b in zip(s.backward(dy), t.backward(dy)):
        if torch.is_tensor(a):
            assert torch.equal(a, b)
        else:
            assert all(torch.equal(u[k], v[k]) for u, v in zip(a, b) for k in u)


@pytest.mark.parametrize("post", ["rms", "layer"])
def test_sandwich_gradients_against_differences(post):
    """Directional differences of <w, forward> for the input and every parameter.
    Two step widths tell the truncation (the quotient's error goes with the
    square of the step: the wider one has four times as much); the outputs' fp32
    rounding, at most 2^-18 of their size each after some 30 operations on a path,
    divided by the step 2^-6, is below 1e-3 of the terms' root sum of squares."""
    s, x, Gs, w = make(300, 64, 16, 2, F32, SandwichStack, post=post, seed=3)
    w = 1 + 0.5 * w
    out = s.forward(x, Gs)
    dx, grads = s.backward(w.clone())
    noise = 2.0 ** -18 * (w.double() * out.double()).norm().item() / 2.0 ** -6

    def loss():
        return (w.double() * s.forward(x, Gs).double()).sum().item()

    named = {**s.named_parameters(), "x": x}
    got = {**s.named_grads(grads), "x": dx}
    assert set(named) - set(got) == set()
    g = torch.Generator()
    g.manual_seed(5)
    for k, t in named.items():
        v = torch.randn(t.shape, generator=g).cuda()
        v = v / v.norm() * t.norm() if t.norm() > 0 else v
        keep, quot = t.clone(), {}
        for h in (2.0 ** -6, 2.0 ** -5):
            side = []
            for sign in (1, -1):
                t.copy_(keep + sign * h * v)
                side.append(loss())
            quot[h] = (side[0] - side[1]) / (2 * h)
        t.copy_(keep)
        want = (got[k].double() * v.double()).sum().item()
        tol = 2 * abs(quot[2.0 ** -5] - quot[2.0 ** -6]) + noise + 1e-3 * abs(want)
        say(f"  {k:12s} {want:12.5g} differences {quot[2.0 ** -6]:12.5g} tolerance {tol:.3g}")
        assert abs(want - quot[2.0 ** -6]) <= tol, k


@pytest.mark.parametrize("kind,dt,bits", [(BlockStack, F32, 32), (SandwichStack, F32, 8),
                                          (SandwichStack, BF16, 8), (BlockStack, BF16, 32)])
def test_training_steps(kind, dt, bits):
    """Three steps: after each, every parameter, moment and rounded copy is the
    reference's step from the gradients that the backward returned."""
    say(f"{kind.__name__} {dt} {bits} bits")
    s, x, Gs, w = make(1001, 64, 16, 2, dt, kind)
    opt = s.adamw(lr=1e-2, bits=bits, wd=0.1, seed=4)
    clip = torch.tensor([0.25], device="cuda")
    names = list(s.named_parameters())
    cpu = lambda t: t.cpu().clone() if torch.is_tensor(t) else t
    for step in (1, 2, 3):
        s.forward(x, Gs)
        _, grads = s.backward(w)
        grads = s.named_grads(grads)
        before = [{k: cpu(v) for k, v in d.items() if v is not None} for d in opt.items.tensors]
        for d, k in zip(before, names):
            d["g"] = grads[k].cpu()
            d["shape"] = d["p"].shape
        opt.step(grads, gscale=clip)
        after = [{k: v for k, v in d.items() if v is not None} for d in opt.items.tensors]
        flat = lambda ds: [{k: v.reshape(-1) if torch.is_tensor(v) else v for k, v in d.items()}
                           for d in ds]
        check_step(flat(before), flat(after), step, 4, clip.cpu(), lr=1e-2)
    for k, t in s.named_parameters().items():  # the stack computes with them
        p = opt.items.tensors[names.index(k)]["p"]
        assert torch.equal(t, p.to(t.dtype)), k
    assert torch.isfinite(s.forward(x, Gs).float()).all()


@pytest.mark.parametrize("kind,dt,bits", [(SandwichStack, F32, 8), (BlockStack, BF16, 32)])
def test_training_steps_in_a_graph(kind, dt, bits):
    """Forward, backward and the optimiser's step in one graph, replayed beside a twin
    that runs them eagerly: the same parameters after every step."""
    s, x, Gs, w = make(1001, 64, 16, 2, dt, kind)
    t, *_ = make(1001, 64, 16, 2, dt, kind)
    t.tuned = s.tuned
    count = torch.zeros(1, dtype=torch.int64, device="cuda")
    lr = torch.full((1,), 1e-2, device="cuda")
    a, b = (k.adamw(lr=1e-2, bits=bits, wd=0.1, seed=4) for k in (s, t))

    def step(k, opt, **kw):
        k.forward(x, Gs)
        opt.step(k.named_grads(k.backward(w)[1]), **kw)

    for _ in range(2):  # (the first chooses the library products' algorithms)
        step(s, a)
        step(t, b)
        count.add_(1)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        count.add_(1)
        step(s, a, step_dev=count, lr_dev=lr)
    for rep in range(4):
        step(t, b, lr=lr.item())  # (the fp32 number that the graph reads)
        graph.replay()
        torch.cuda.synchronize()
        for k, v in s.named_parameters().items():
            assert torch.equal(v, t.named_parameters()[k]), (rep, k)
    assert count.item() == 6 and a.t == 2 and b.t == 6


@pytest.mark.parametrize("kind,dt", [(BlockStack, F32), (BlockStack, BF16), (SandwichStack, F32),
                                     (SandwichStack, BF16)])
@pytest.mark.parametrize("N,C", [(1001, 64), (8192, 128)])
def test_inference_in_8_bits(kind, dt, N, C):
    """infer is forward bit for bit; with the MLP's products in integers it is
    within 3%: an element is off by at most half of max / 127, about 0.3 / 127
    max ~ 0.8% of a row's size, for the rows and the weights of two products
    (together 1.6% of the MLP's part), and the next block carries that on."""
    s, x, Gs, _ = make(N, C, 16, 2, dt, kind)
    want = s.forward(x, Gs)
    assert torch.equal(s.infer(x, Gs), want)
    s.quantize()
    got = s.infer(x, Gs)
    rel = ((got.double() - want.double()).norm() / want.double().norm()).item()
    say(f"  {kind.__name__} {dt} N={N} C={C}: {rel:.4f}")
    assert 1e-5 < rel <= 0.03
    assert torch.equal(s.infer(x, Gs), got)


@pytest.mark.parametrize("kind,dt", [(BlockStack, BF16), (SandwichStack, BF16), (SandwichStack, F32)])
def test_quantised_inference_in_a_graph(kind, dt):
    """infer captured after quantize and replayed: as the eager one, also after the
    weights have changed and been quantised again, with new tensors in the place of
    whatever the stack let go of."""
    say(f"quantised infer in a graph, {kind.__name__} {dt}")
    s, x, Gs, _ = make(1001, 64, 16, 2, dt, kind)
    s.quantize()
    s.infer(x, Gs)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = s.infer(x, Gs)
    seen, hold = [], []
    for rep in range(4):
        if rep:
            for p in s.params:
                for k in ("W1", "W2"):
                    p[k].mul_(1 + 0.25 * rep)
            s.quantize()
            hold += [torch.full_like(t, 77) for layer in s.int8 for t in layer]
        want = s.infer(x, Gs)
        for _ in range(2):
            out.zero_()
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(out, want), rep
        seen.append(want)
    assert all(not torch.equal(a, b) for a, b in zip(seen, seen[1:]))


def test_training_goes_on_from_weights_that_were_loaded():
    """bf16 weights loaded in place between two steps: refused, then, refreshed, a step
    from the loaded weights."""
    s, x, Gs, w = make(1001, 64, 16, 2, BF16, SandwichStack)
    t, *_ = make(1001, 64, 16, 2, BF16, SandwichStack, seed=1)
    opt = s.adamw(lr=1e-2, wd=0.1, seed=4)

    def grads():
        s.forward(x, Gs)
        return s.named_grads(s.backward(w)[1])

    opt.step(grads())
    for p, q in zip(s.params, t.params):
        for k in ("W1", "W2"):
            p[k].copy_(q[k])
    g = grads()
    with pytest.raises(ValueError, match="refresh"):
        opt.step(g)
    opt.refresh()
    flat = lambda: [{k: v.cpu().reshape(-1) if torch.is_tensor(v) else v for k, v in d.items()
                     if v is not None} for d in opt.items.tensors]
    before = flat()
    for d, k in zip(before, opt.names):
        d["g"] = g[k].cpu().reshape(-1)
        if k.endswith(("W1", "W2")):
            l, name = k.split(".")
            assert torch.equal(d["p"], t.params[int(l)][name].float().cpu().reshape(-1))
    opt.step(g)
    check_step(before, flat(), 2, 4, lr=1e-2)


@pytest.mark.parametrize("kind,dt,bits", [(SandwichStack, BF16, 8), (BlockStack, BF16, 32),
                                          (BlockStack, F32, 8)])
def test_training_goes_on_from_a_state(kind, dt, bits, tmp_path):
    """Parameters and the optimizer's state saved after two steps and loaded into a stack
    of its own: the next two steps bit for bit."""
    s, x, Gs, w = make(1001, 64, 16, 2, dt, kind)
    t, *_ = make(1001, 64, 16, 2, dt, kind, seed=1)
    t.tuned = s.tuned
    a, b = s.adamw(lr=1e-2, bits=bits, seed=4), t.adamw(lr=1e-2, bits=bits)

    def step(k, opt):
        k.forward(x, Gs)
        opt.step(k.named_grads(k.backward(w)[1]))

    for _ in range(2):
        step(s, a)
    torch.save({"params": s.named_parameters(), "state": a.state()}, tmp_path / "c.pt")
    got = torch.load(tmp_path / "c.pt", weights_only=True)
    for k, v in t.named_parameters().items():
        v.copy_(got["params"][k])
    b.load_state(got["state"])
    for rep in range(2):
        step(s, a)
        step(t, b)
        for k, v in s.named_parameters().items():
            assert torch.equal(v, t.named_parameters()[k]), (rep, k)
        for k in a.names:
            assert all(torch.equal(m, n) for m, n in zip(a.moments(k), b.moments(k))), (rep, k)
    assert a.t == b.t == 4


@pytest.mark.parametrize("kind,dt", [(BlockStack, BF16), (SandwichStack, F32)])
def test_quantised_inference_after_a_step(kind, dt):
    """Refused with the integers of the weights before the step; quantised again, as a
    stack that never had other weights."""
    s, x, Gs, w = make(1001, 64, 16, 2, dt, kind)
    opt = s.adamw(lr=1e-2)
    s.quantize()
    s.infer(x, Gs)
    s.forward(x, Gs)
    opt.step(s.named_grads(s.backward(w)[1]))
    with pytest.raises(ValueError, match="quantize"):
        s.infer(x, Gs)
    s.quantize()
    got = s.infer(x, Gs)
    t = kind(1001, 64, 4, 16, s.params, dt)
    t.quantize()
    assert torch.equal(got, t.infer(x, Gs))


def with_b_t(s, value=0.375):
    for p in s.params:
        p["b_t"] = torch.tensor([value], device="cuda")


@pytest.mark.parametrize("kind", [BlockStack, SandwichStack])
def test_b_t_as_a_tensor(kind):
    """The same outputs as with a float (0.375 and bp.a add to one fp32 rounding, 2^-24
    of a temperature of about 1; a weight's logarithm goes with logit / tau, here up to
    about 20: 1e-5), and its gradient against differences: a step of 2^-6, so that the
    fp32 outputs' roundings, 2^-18 of each at most, stay below the tolerance."""
    s, x, Gs, w = make(300, 64, 16, 2, F32, kind, seed=3)
    for p in s.params:
        p["b_t"] = 0.375
    want = s.forward(x, Gs)
    with_b_t(s)
    out = s.forward(x, Gs)
    assert ((out - want).double().norm() / want.double().norm()).item() <= 1e-5
    _, grads = s.backward(w)
    noise = 2.0 ** -18 * (w.double() * out.double()).norm().item() / 2.0 ** -6
    for l, p in enumerate(s.params):
        quot = {}
        for h in (2.0 ** -6, 2.0 ** -5):
            side = []
            for sign in (1, -1):
                p["b_t"].fill_(0.375 + sign * h)
                side.append((w.double() * s.forward(x, Gs).double()).sum().item())
            quot[h] = (side[0] - side[1]) / (2 * h)
        p["b_t"].fill_(0.375)
        got = grads[l]["db_t"].item()
        tol = 2 * abs(quot[2.0 ** -5] - quot[2.0 ** -6]) + noise + 1e-3 * abs(got)
        say(f"  {l}: {got:.5g} differences {quot[2.0 ** -6]:.5g} tolerance {tol:.3g}")
        assert abs(got - quot[2.0 ** -6]) <= tol


@pytest.mark.parametrize("kind,dt", [(SandwichStack, F32), (BlockStack, BF16)])
def test_b_t_is_trained(kind, dt):
    """Steps with b_t among the parameters, eagerly and in a graph: it moves, by the
    optimizer's first step lr from where it was, and both ways alike."""
    s, x, Gs, w = make(1001, 64, 16, 2, dt, kind)
    t, *_ = make(1001, 64, 16, 2, dt, kind)
    t.tuned = s.tuned
    for k in (s, t):
        with_b_t(k)
    a, b = s.adamw(lr=1e-2), t.adamw(lr=1e-2)
    count = torch.zeros(1, dtype=torch.int64, device="cuda")

    def step(k, opt, **kw):
        k.forward(x, Gs)
        opt.step(k.named_grads(k.backward(w)[1]), **kw)

    for _ in range(2):
        step(s, a)
        step(t, b)
        count.add_(1)
        if count.item() == 1:
            for p in s.params:
                assert abs(abs(p["b_t"].item() - 0.375) - 1e-2) <= 1e-5
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        count.add_(1)
        step(s, a, step_dev=count)
    for rep in range(3):
        step(t, b)
        graph.replay()
        torch.cuda.synchronize()
        for k, v in s.named_parameters().items():
            assert torch.equal(v, t.named_parameters()[k]), (rep, k)


@pytest.mark.parametrize("post", ["rms", "layer"])
def test_sandwich_backward_joins_as_its_parts_in_bf16(post, monkeypatch):
    """Every joint's backward that the stack runs, against 64 bits on what it was given;
    each from the forward's tensors of its place and with its place's parameters, the
    residual stream's gradient handed on from joint to joint, and the parameters'
    gradients under their names."""
    s, x, Gs, w = make(777, 64, 16, 2, BF16, SandwichStack, post=post)
    s.forward(x, Gs)
    calls, real = [], ops.pa_residual_norm_backward

    def record(x1, y, par, dx1, dh, dx, dy, gr, ws):
        real(x1, y, par, dx1, dh, dx, dy, gr, ws)
        calls.append(({"x1": x1, "y": y, "dx1": dx1, "dh": dh},
                      {"dx": dx.clone(), "dy": dy.clone()}, gr.tensors, ws.numel() // (20 * 64)))

    monkeypatch.setattr(ops, "pa_residual_norm_backward", record)
    import test_gpu_ops as check
    _, grads = s.backward(w)
    assert len(calls) == 4
    cpu = lambda t: None if t is None else t.cpu()
    dx = w
    for (l, k), (i, o, gr, rec) in zip(((1, 2), (1, 1), (0, 2), (0, 1)), calls):
        c, p = s.caches[l], {n: cpu(v) for n, v in s.params[l].items() if torch.is_tensor(v)}
        assert i["x1"] is c["x2" if k == 2 else "x1"] and i["y"] is c["z" if k == 2 else "y"]
        assert torch.equal(i["dx1"], dx)
        dx = o["dx"]
        q = {"post": post, "post_g": p[f"post{k}_g"], "post_b": p.get(f"post{k}_b"),
             "scale": p[f"rs{k}"], "pre": None}
        at, ln = (l, "ln2") if k == 1 else (l + 1, "ln1")
        assert (i["dh"] is None) == (at == len(s.params))
        names = {"dscale": grads[l][f"drs{k}"], "dpost_g": grads[l][f"dpost{k}_g"]}
        if post == "layer":
            names["dpost_b"] = grads[l][f"dpost{k}_b"]
        if i["dh"] is not None:
            n = s.params[at]
            q.update(pre="layer", pre_g=cpu(n[ln + "_g"]), pre_b=cpu(n[ln + "_b"]))
            names.update(dpre_g=grads[at][f"d{ln}_g"], dpre_b=grads[at][f"d{ln}_b"])
        for name, t in names.items():
            assert gr[name] is t, (l, k, name)
        ref = R.joint_backward(q, *(cpu(i[n]) for n in ("x1", "y")), None, cpu(i["dx1"]),
                               cpu(i["dh"]), 777 // rec + 300)
        for name, (v, err) in ref.items():
            if name in o or name in names:
                check.within(o.get(name, names.get(name)), v, err, BF16 if name in o else F32,
                       f"{l}.{k} {name}")


@pytest.mark.parametrize("kind", [BlockStack, SandwichStack])
def test_inference_in_8_bits_at_256_channels(kind):
    """As test_inference_in_8_bits, to its bound, at the widest stack's channels, whose
    products keep their weights in registers."""
    s, x, Gs, _ = make(5003, 256, 32, 2, BF16, kind)
    want = s.infer(x, Gs)
    s.quantize()
    got = s.infer(x, Gs)
    rel = ((got.double() - want.double()).norm() / want.double().norm()).item()
    say(f"  {kind.__name__}: {rel:.4f}")
    assert 1e-5 < rel <= 0.03
    assert torch.equal(s.infer(x, Gs), got)
