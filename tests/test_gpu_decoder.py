"""QueryDecoder: cross attention and dropout together, as a program trains and asks
them, against the same blocks in 64 bits."""
import numpy as np
import pytest
import torch

import ask_ref as R
import oracle
from paper_2502_02414_amd import inputs as I
from paper_2502_02414_amd import ops
from paper_2502_02414_amd.stack import BlockStack, QueryDecoder
from pa_cases import dev, host, rel_l2, say

pytestmark = pytest.mark.gpu

F32, BF16 = torch.float32, torch.bfloat16


def make(N, C, H, Hkv, Cs, Ns, L, dt, drop=0.0, seed=0):
    g = torch.Generator()
    g.manual_seed(seed)
    rnd = lambda *s, scale=1.0: scale * torch.randn(*s, generator=g)
    ps = []
    for _ in range(L):
        F = 2 * Hkv * (C // H)
        p = {"ln1_g": 1 + rnd(C, scale=0.1), "ln1_b": rnd(C, scale=0.1), "bq": rnd(C, scale=0.1),
             "bkv": rnd(F, scale=0.1), "bo": rnd(C, scale=0.1), "ln2_g": 1 + rnd(C, scale=0.1),
             "ln2_b": rnd(C, scale=0.1), "b1": rnd(4 * C, scale=0.1), "b2": rnd(C, scale=0.1),
             "Wq": rnd(C, C, scale=C ** -0.5).to(dt), "Wkv": rnd(Cs, F, scale=Cs ** -0.5).to(dt),
             "Wo": rnd(C, C, scale=C ** -0.5).to(dt), "W1": rnd(C, 4 * C, scale=C ** -0.5).to(dt),
             "W2": rnd(4 * C, C, scale=0.5 * C ** -0.5).to(dt)}
        ps.append({k: v.cuda() for k, v in p.items()})
    dec = QueryDecoder(N, C, H, ps, dt, Hkv=Hkv, drop=drop, seed=77)
    return dec, rnd(N, C).to(dt).cuda(), rnd(Ns, Cs).to(dt).cuda(), rnd(N, C).to(dt).cuda()


def blocks(dec, P, x, s, q_off, k_off, mask, drops):
    """The decoder's definition in 64 bits on the CPU (leaves P, x, s: autograd)."""
    H, Hkv, D = dec.H, dec.Hkv, dec.D
    norm = lambda z, g, b: torch.nn.functional.layer_norm(z, z.shape[1:], g, b, dec.ln_eps)
    gelu = lambda z: z * 0.5 * torch.erfc(-z / 2 ** 0.5)
    N, Ns = x.shape[0], s.shape[0]
    for l, p in enumerate(P):
        q = (norm(x, p["ln1_g"], p["ln1_b"]) @ p["Wq"] + p["bq"]).view(N, H, D)
        kv = (s @ p["Wkv"] + p["bkv"]).view(Ns, 2, Hkv, D)
        o = torch.zeros(N, H, D, dtype=torch.float64)
        for rows, live in R.requests(q_off, k_off, N, Ns, mask):
            if rows.numel() and live.numel():
                for h in range(H):
                    k, v = kv[live, 0, h * Hkv // H], kv[live, 1, h * Hkv // H]
                    a = torch.softmax(q[rows, h] @ k.t() * D ** -0.5, 1) @ v
                    o = o.index_put((rows, torch.tensor(h)), a)
        y = o.view(N, -1) @ p["Wo"] + p["bo"]
        x = x + (y if drops is None else y * drops[l][0])
        z = gelu(norm(x, p["ln2_g"], p["ln2_b"]) @ p["W1"] + p["b1"]) @ p["W2"] + p["b2"]
        x = x + (z if drops is None else z * drops[l][1])
    return x


def drops_of(dec, step):
    """The scales of every element (0 where it is dropped), per layer and place."""
    if not dec.drop:
        return None
    out, n = [], dec.N * dec.C
    for l in range(len(dec.params)):
        pair = []
        for k in range(2):
            keep, f = R.kept(np.arange(n), dec.drop, dec.seed, 2 * len(dec.params) * step + 2 * l + k)
            pair.append((keep.double() * f).view(dec.N, dec.C))
        out.append(pair)
    return out


def rel(a, b):
    return (a.detach().cpu().double() - b).norm().item() / (b.norm().item() + 1e-30)


# A relative 2-norm of 1e-5 in fp32 (the bar of the framework's other stacks: some 30
# roundings of 2^-24 on a path, with a hundred in hand for what sums lose).  bf16: some 10
# stored tensors on the way forward and 20 on the way back, each within 2^-8 of its
# values, by their squares sqrt(20) 2^-8 / sqrt(3) = 1%; twice that.
BAR = {F32: 1e-5, BF16: 2e-2}


@pytest.mark.parametrize("dt", [F32, BF16])
@pytest.mark.parametrize("drop", [0.0, 0.2])
@pytest.mark.parametrize("N,C,H,Hkv,Cs,Ns,ql,kl,mask", [
    (300, 64, 4, 4, 64, 40, None, None, False),
    (257, 128, 8, 2, 96, 333, (100, 0, 157), (33, 200, 100), True),
    (64, 256, 8, 8, 256, 64, None, None, False),
])
def test_decoder_against_64_bits(dt, drop, N, C, H, Hkv, Cs, Ns, ql, kl, mask):
    say(f"decoder {dt} drop={drop} N={N} C={C} H={H}/{Hkv} Ns={Ns}")
    dec, x, s, dy = make(N, C, H, Hkv, Cs, Ns, 2, dt, drop)
    off = lambda n: None if n is None else [0] + list(np.cumsum(n))
    q_off, k_off = off(ql), off(kl)
    m = torch.arange(Ns) % 7 != 3 if mask else None
    par = None
    if ql is not None:
        par = dec.requests(torch.tensor(q_off).cuda(), torch.tensor(k_off).cuda(),
                           None if m is None else m.cuda(), max(kl))
    out = dec.forward(x, s, par, step=5)
    dx, ds, grads = dec.backward(dy.clone())
    P = [{k: v.cpu().double().requires_grad_() for k, v in p.items()} for p in dec.params]
    x64, s64 = x.cpu().double().requires_grad_(), s.cpu().double().requires_grad_()
    ref = blocks(dec, P, x64, s64, q_off, k_off, m, drops_of(dec, 5))
    (ref * dy.cpu().double()).sum().backward()
    assert rel(out, ref.detach()) <= BAR[dt]
    assert rel(dx, x64.grad) <= BAR[dt] and rel(ds, s64.grad) <= BAR[dt]
    for l, g in enumerate(grads):
        assert set(g) == {"d" + k for k in P[l]}
        for k, v in g.items():
            want = P[l][k[1:]].grad
            if k == "dbkv":  # (a bias of k alone moves every score of a row alike: no gradient)
                half = want.numel() // 2
                v, want = v[half:], want[half:]
            assert rel(v, want) <= BAR[dt], (l, k, rel(v, want))
    if not drop:
        assert torch.equal(dec.infer(x, s, par), out)
        assert torch.equal(dec.infer(x, par=par, kept=dec.keep(s)), out)


def test_dropped_elements_change_from_step_to_step():
    dec, x, s, _ = make(200, 64, 4, 4, 64, 30, 1, F32, 0.3)
    a, b, c = dec.forward(x, s, step=1), dec.forward(x, s, step=2), dec.forward(x, s, step=1)
    assert torch.equal(a, c) and not torch.equal(a, b)
    assert not torch.equal(dec.infer(x, s), a)


def test_one_point_of_a_request_among_many():
    """A point asked alone and in a batch of requests, within one rounding of bf16 in
    every stored tensor (the kernels differ)."""
    C, H, n = 64, 4, 9
    dec, x, s, _ = make(n, C, H, H, C, n * 50, 1, BF16)
    off = torch.arange(n + 1).cuda()
    batch = dec.infer(x, s, dec.requests(off, 50 * off, max_k=50))
    one = QueryDecoder(1, C, H, dec.params, BF16)
    for i in range(n):
        alone = one.infer(x[i:i + 1].clone(), s[50 * i:50 * i + 50].clone())
        assert rel(alone, batch[i:i + 1].cpu().double()) <= BAR[BF16]


def test_a_training_step_in_a_graph():
    """Forward, backward and the optimizer's step captured, the step's numbers on the
    device, beside an eager twin: every replay's answers, gradients and parameters."""
    args = (500, 64, 4, 2, 64, 48, 2, F32, 0.1)
    (a, x, s, w), (b, *_) = make(*args), make(*args)
    b.tuned = a.tuned  # (each would choose the products' algorithms by its own timing)
    oa, ob = a.adamw(1e-3), b.adamw(1e-3)
    step = torch.zeros(1, dtype=torch.int64, device="cuda")
    at = torch.zeros(1, dtype=torch.int64, device="cuda")

    def train(dec, opt, dev=False, n=0):
        kw = {"offset_dev": at} if dev else {"step": n}
        out = dec.forward(x, s, **kw)
        dx, ds, grads = dec.backward(w.clone())
        opt.step(dec.named_grads(grads), **({"step_dev": step} if dev else {}))
        return out, dx, ds

    for n in range(2):  # (the products are tuned)
        train(a, oa, n=n)
        train(b, ob, n=n)
    torch.cuda.synchronize()
    step.fill_(2)
    at.fill_(2 * 2 * 2)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step.add_(1)
        outs = train(b, ob, dev=True)
        at.add_(4)
    for n in range(2, 6):
        want = train(a, oa, n=n)
        graph.replay()
        torch.cuda.synchronize()
        for u, v in zip(want, outs):
            assert torch.equal(u, v), n
        for k, v in a.named_parameters().items():
            assert torch.equal(v, b.named_parameters()[k]), (n, k)


def test_a_frozen_encoder_and_integers():
    """Inference with the MLP in 8-bit integers stays near the decoder's own: each of the
    two products a layer within the integers' steps (1/127 of a row's largest)."""
    dec, x, s, _ = make(400, 64, 4, 4, 64, 60, 2, BF16)
    plain = dec.infer(x, s)
    dec.quantize()
    q = dec.infer(x, s)
    assert not torch.equal(plain, q)
    assert rel(q, plain.cpu().double()) <= 5e-2


def test_an_encoder_that_trains_with_its_decoder():
    """A block stack's points as the states, the decoder's gradient of them into the stack's
    backward: against both in 64 bits.  The bar is that of four passes (stack and decoder,
    forward and backward), 1e-5 each."""
    n, C, H, M = 700, 64, 4, 16
    w = I.small("stack", n, C, H, M, "f32", geometry="normal")
    x, G = I.make_x(w, n), I.make_layer_gumbel(w, 0, n)
    p = I.make_block_params(w, 0)
    put = lambda k, v: float(v) if k == "b_t" else dev(v, "f32")
    enc = BlockStack(n, C, H, M, [{k: put(k, v) for k, v in p.items()}], F32, w.tau0, w.tau_min, w.eps)
    dec, xq, _, dy = make(300, C, H, H, C, 1, 2, F32)
    s = enc.forward(dev(x, "f32"), [dev(G, "f32")])
    out = dec.forward(xq, s)
    dxq, ds, grads = dec.backward(dy.clone())
    dx, egrads = enc.backward(ds)
    s64, caches = oracle.stack_forward(x, [G], [p], w.tau0, w.tau_min, w.eps, H)
    P = [{k: v.cpu().double().requires_grad_() for k, v in q.items()} for q in dec.params]
    leaf, q64 = torch.tensor(s64).double().requires_grad_(), xq.cpu().double().requires_grad_()
    ref = blocks(dec, P, q64, leaf, None, None, None, None)
    (ref * dy.cpu().double()).sum().backward()
    rdx, rgr = oracle.stack_backward(leaf.grad.numpy(), [G], [p], w.tau0, w.tau_min, w.eps, H, caches)
    assert rel(out, ref.detach()) <= 4e-5 and rel(dxq, q64.grad) <= 4e-5
    assert rel(ds, leaf.grad) <= 4e-5 and rel_l2(host(dx), rdx) <= 4e-5
    for l, g in enumerate(grads):
        for k in ("dWq", "dWo", "dW1", "dW2", "dln1_g", "dbo"):
            assert rel(g[k], P[l][k[1:]].grad) <= 4e-5, (l, k)
    for k in ("dW1", "dW2", "dWp", "dln1_g"):
        assert rel_l2(host(egrads[0][k]), rgr[0][k]) <= 4e-5, k
