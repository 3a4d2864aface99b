"""What the block stack and its optimiser keep from call to call, on the CPU (the
library's launches replaced by a recorder)."""
import gc
import weakref

import pytest
import torch

from paper_2502_02414_amd import binding as B
from paper_2502_02414_amd import ops
from paper_2502_02414_amd.stack import BlockStack, SandwichStack


class Recorder:
    """libpa.so's calls by name and arguments."""

    def __init__(self):
        self.calls = []

    def __getattr__(self, name):
        def call(*args):
            self.calls.append((name, args))
            return B.PA_OK
        return call

    def names(self):
        return [n for n, _ in self.calls]


@pytest.fixture
def fake(monkeypatch):
    rec = Recorder()
    monkeypatch.setattr(ops, "load", lambda: rec)
    monkeypatch.setattr(ops, "_dev", lambda t, name, cur=None: t.data_ptr())
    monkeypatch.setattr(ops, "_current_device", lambda: -1)  # (a CPU tensor's index)
    monkeypatch.setattr(ops, "_capturing", lambda *a: False)
    monkeypatch.setattr(B, "_stream", lambda s=None: 0)
    return rec


def params(C=64, M=16, dt=torch.bfloat16, kind=BlockStack):
    r = lambda *s: torch.randn(*s)
    p = {"Wp": r(C, C), "bp": r(C), "A": r(C, M), "b": r(M), "a": r(C), "b1": r(4 * C), "b2": r(C),
         "W1": r(C, 4 * C).to(dt), "W2": r(4 * C, C).to(dt), "b_t": 0.5}
    for n in ("ln1", "ln2"):
        p[n + "_g"], p[n + "_b"] = r(C), r(C)
    for n in "qkv":
        p["W" + n], p["b" + n] = r(C, C), r(C)
    if kind is SandwichStack:
        for k in "12":
            p["rs" + k], p[f"post{k}_g"] = r(C), r(C)
    return p


def stack(kind=BlockStack, L=2, N=100, C=64, M=16, dt=torch.bfloat16):
    return kind(N, C, 4, M, [params(C, M, dt, kind) for _ in range(L)], dt, device="cpu")


@pytest.mark.parametrize("kind", [BlockStack, SandwichStack])
def test_quantize_writes_the_same_tensors_every_time(fake, monkeypatch, kind):
    """A captured infer reads the integers and scales by their addresses: quantising
    again has to write those, and may not let go of them."""
    if kind is SandwichStack:
        monkeypatch.setattr(ops, "residual_norm_workspace", lambda *a: torch.empty(8))
    s = stack(kind)
    s.quantize()
    first = [[t.data_ptr() for t in layer] for layer in s.int8]
    sizes = [[tuple(t.shape) for t in layer] for layer in s.int8]
    assert sizes == [[(256, 64), (256,), (64, 256), (64,)]] * 2
    hold = list(fake.calls)
    fake.calls.clear()
    for p in s.params:
        p["W1"] = p["W1"] + 1
    s.quantize()
    gc.collect()
    assert [[t.data_ptr() for t in layer] for layer in s.int8] == first
    out = lambda calls: [a[4:6] for n, a in calls if n == "pa_quant_weight"]
    assert out(fake.calls) == out(hold) and len(out(hold)) == 4


def items_of(*sizes):
    z = torch.zeros
    return ops.make_adamw_items([{"p": z(n), "g": z(n), "m": z(n), "v": z(n)} for n in sizes])


@pytest.mark.parametrize("table", [False, True])
def test_gradients_that_a_graph_reads_are_kept(fake, monkeypatch, table):
    """A step captured into a graph, then a step with other gradients: the first ones'
    memory stays as long as the items."""
    monkeypatch.setattr(ops, "_capturing", lambda *a: True)
    monkeypatch.setattr(B, "_stream", lambda s=None: 1)
    it = items_of(300, 400)
    if table:
        it.dev, it.blocks, it.stream, it.ptr, it.device = torch.zeros(8), 2, 1, 4096, -1
    alive = [weakref.ref(d["g"]) for d in it.tensors]
    for _ in range(3):  # (several graphs of the same gradients keep them once)
        ops.pa_adamw(it, lr=1e-3, step_dev=torch.ones(1, dtype=torch.int64))
    assert len(it.captured_grads) == 1 and len(it.captured) == table
    monkeypatch.setattr(ops, "_capturing", lambda *a: False)
    monkeypatch.setattr(B, "_stream", lambda s=None: 0)
    it.set_grads([torch.ones(300), torch.ones(400)])
    ops.pa_adamw(it, lr=1e-3)
    gc.collect()
    assert all(r() is not None for r in alive)
    loose = [weakref.ref(d["g"]) for d in it.tensors]
    it.set_grads([torch.ones(300), torch.ones(400)])
    gc.collect()
    assert all(r() is None for r in loose)  # (those of an eager step are let go of)


def test_a_capture_is_looked_for_on_the_stream_of_the_call(fake, monkeypatch):
    """A stream handed over that is being captured, while the current one is not: the
    step needs its number on the device, makes no table (a copy and a wait, which end
    a capture), and what it reads is kept."""
    side = object()
    monkeypatch.setattr(ops, "_capturing", lambda stream=None: stream is side)
    monkeypatch.setattr(B, "_stream", lambda s=None: 7 if s is side else 0)
    w, g = {"w": torch.zeros(300)}, {"w": torch.ones(300)}
    opt = ops.AdamW(w, lr=1e-3)
    made = []
    monkeypatch.setattr(opt.items, "table", lambda: made.append(1))
    opt.step(g)
    with pytest.raises(ValueError, match="step_dev"):
        opt.step(g, stream=side)
    one = torch.ones(1, dtype=torch.int64)
    opt.step(g, stream=side, step_dev=one)  # (its gradients have stayed)
    assert not made and len(opt.items.captured_grads) == 1
    it = opt.items
    it.dev, it.blocks, it.stream, it.ptr, it.device = torch.zeros(8), 1, 0, 4096, -1
    opt.step(g, stream=side, step_dev=one)
    assert len(it.captured) == 1 and it.captured[0] is it.dev
    it.dev = None
    opt.step(g)
    assert made and fake.names() == ["pa_adamw", "pa_adamw", "pa_adamw_run", "pa_adamw"]


def test_gradients_of_a_step_on_another_stream(fake, monkeypatch):
    """The allocator hears of the stream that reads the gradients and device scalars:
    the next step lets go of the gradients while that one may not have run."""
    side = object()
    monkeypatch.setattr(B, "_stream", lambda s=None: 7 if s is side else 3)
    seen = []
    monkeypatch.setattr(torch.Tensor, "record_stream", lambda t, s: seen.append((id(t), s)))
    opt = ops.AdamW({"a": torch.zeros(300), "b": torch.zeros(20)}, lr=1e-3)
    g = {"a": torch.ones(300), "b": torch.ones(20)}
    scale = torch.ones(1)
    monkeypatch.setattr(opt.items, "table", lambda: None)
    opt.step(g)
    assert seen == []
    opt.step(g, gscale=scale, stream=side)
    assert sorted(seen) == sorted((id(t), side) for t in (g["a"], g["b"], scale))


@pytest.mark.parametrize("n", [0, 1, 3])
def test_a_gradient_for_every_item(fake, n):
    """Too few gradients left the others at the last step's, too many were passed over."""
    it = items_of(300, 400)
    had = [d["g"] for d in it.tensors]
    with pytest.raises(ValueError, match="2 items"):
        it.set_grads([torch.ones(300), torch.ones(400), torch.ones(5)][:n])
    assert all(d["g"] is g for d, g in zip(it.tensors, had))


def test_structs_of_another_device_are_refused(fake, monkeypatch):
    """Parameters, gradients and items are pointers that were checked where they were
    made: with another current device a call refuses them, with a table or without."""
    x, w = torch.zeros(10, 32), torch.ones(32)
    par, none = ops.make_residual_norm_params(pre="rms", pre_g=w), ops.make_residual_norm_params(pre="rms")
    gr = ops.make_residual_norm_grads(dpre_g=w)
    it = items_of(300)
    at = [0]
    monkeypatch.setattr(ops, "_current_device", lambda: at[0])
    monkeypatch.setattr(ops, "_in", lambda t, *a: None if t is None else t.data_ptr())
    for bad in (lambda: ops.pa_residual_norm(x, x, par, x, x),
                lambda: ops.pa_residual_norm_backward(x, x, par, x, x, x, x),
                lambda: ops.pa_residual_norm_backward(x, x, none, x, x, x, x, gr),
                lambda: ops.pa_adamw(it, lr=1e-3), it.table):
        with pytest.raises(ValueError, match="current one"):
            bad()
    it.dev, it.blocks, it.stream, it.ptr = torch.zeros(8), 1, 0, 4096
    with pytest.raises(ValueError, match="current one"):
        ops.pa_adamw(it, lr=1e-3)
    assert fake.calls == []
    ops.pa_residual_norm(x, x, none, x, x)  # (nothing that could be elsewhere)
    at[0] = -1
    ops.pa_residual_norm(x, x, par, x, x)
    ops.pa_adamw(it, lr=1e-3)
    assert fake.names() == ["pa_residual_norm"] * 2 + ["pa_adamw_run"]


def grads_of(s):
    return {k: torch.ones_like(v, dtype=torch.float32) for k, v in s.named_parameters().items()}


@pytest.mark.parametrize("dt", [torch.bfloat16, torch.float32])
def test_a_step_for_tensors_that_the_stack_has_no_more(fake, dt):
    """A tensor put in a parameter's place: the optimizer would go on with the one
    before and the stack would never see a step."""
    s = stack(dt=dt)
    opt = s.adamw(lr=1e-3)
    g = grads_of(s)
    opt.step(g)
    for name in ("W1", "bp", "ln2_g"):
        p = s.params[1]
        had, p[name] = p[name], p[name].clone()
        with pytest.raises(ValueError, match="1." + name):
            opt.step(g)
        p[name] = had
    del s.params[0]["b"]
    with pytest.raises(ValueError, match="0.b"):
        opt.step(g)
    assert fake.names() == ["pa_adamw"] and opt.t == 1


def test_a_bf16_weight_that_was_written(fake):
    """A checkpoint loaded in place: the step would write the old fp32 parameter's
    rounding over it.  Refused until refresh() has taken it over."""
    s = stack()
    opt = s.adamw(lr=1e-3)
    g = grads_of(s)
    opt.items.table = lambda: None
    opt.step(g)
    w = s.params[0]["W1"]
    master = opt.items.tensors[opt.names.index("0.W1")]["p"]
    w.copy_(torch.full_like(w, 3.0))
    with pytest.raises(ValueError, match="0.W1.*refresh"):
        opt.step(g)
    assert fake.names() == ["pa_adamw"] and not (master == 3).all()
    opt.refresh()
    assert (master == 3).all()
    s.params[0]["Wp"].add_(1)  # (fp32: the optimizer's own)
    opt.step(g)
    assert fake.names() == ["pa_adamw"] * 2 and opt.t == 2
    with torch.inference_mode():  # (their writes are not counted)
        ops.AdamW({"w": torch.zeros(20)}, lr=1e-3, copies={"w": torch.zeros(20, dtype=torch.bfloat16)})


def test_state_of_an_optimizer(fake):
    s = stack()
    a = s.adamw(lr=1e-3, bits=8, seed=5)
    for d in a.items.tensors:  # (as if after some steps)
        for k in ("m", "v", "m_scale", "v_scale"):
            if d.get(k) is not None:
                d[k].copy_(torch.randint(0, 100, d[k].shape))
    a.items.tensors[a.names.index("0.W1")]["p"].fill_(1 + 2 ** -12)
    a.t = 7
    st = a.state()
    assert "p" in st["tensors"]["0.W1"] and "p" not in st["tensors"]["0.Wp"]
    a.items.tensors[0]["m"].zero_()  # (new tensors)
    b = stack().adamw(lr=1e-3, bits=8)
    b.load_state(st)
    assert b.t == 7 and b.seed == 5
    for k, d in zip(b.names, b.items.tensors):
        for key, v in st["tensors"][k].items():
            assert torch.equal(d[key], v), (k, key)
    copy = b.items.tensors[b.names.index("0.W1")]["copy"]
    assert torch.equal(copy, torch.ones_like(copy))
    b.step({k: torch.ones_like(d["p"]) for k, d in zip(b.names, b.items.tensors)})
    had = b.state()
    for other in (stack().adamw(lr=1e-3), stack(L=1).adamw(lr=1e-3, bits=8),
                  stack(C=32).adamw(lr=1e-3, bits=8), stack(dt=torch.float32).adamw(lr=1e-3, bits=8)):
        with pytest.raises(ValueError):
            b.load_state(other.state())
    for k, d in b.state()["tensors"].items():
        assert all(torch.equal(v, had["tensors"][k][key]) for key, v in d.items())


@pytest.mark.parametrize("kind", [BlockStack, SandwichStack])
def test_infer_with_integers_of_other_weights(fake, monkeypatch, kind):
    """After an optimizer's step, a write or another tensor infer answered with the last
    quantize's integers."""
    monkeypatch.setattr(ops, "residual_norm_workspace", lambda *a: torch.empty(8))
    for name in ("pa_layernorm", "pa_mlp_up", "pa_gemm"):
        monkeypatch.setattr(B, name, lambda *a, **kw: None)
    monkeypatch.setattr(kind, "_attention", lambda self, p, c, h, G: torch.empty_like(h))
    s = stack(kind)
    x, Gs = torch.zeros(100, 64, dtype=torch.bfloat16), [None, None]
    opt = s.adamw(lr=1e-3)
    opt.items.table = lambda: None

    def put(l, k):
        s.params[l][k] = s.params[l][k].clone()

    s.infer(x, Gs)  # (no integers: the weights themselves)
    opt.step(grads_of(s))
    s.quantize()
    s.infer(x, Gs)
    s.params[0]["bp"].add_(1)  # (not quantised)
    s.infer(x, Gs)
    for change in (lambda: opt.step(grads_of(s)), lambda: s.params[1]["W2"].mul_(2),
                   lambda: put(0, "W1")):
        change()
        for _ in range(2):
            with pytest.raises(ValueError, match="quantize"):
                s.infer(x, Gs)
        s.quantize()
        s.infer(x, Gs)
        opt.refresh()


def test_b_t_as_a_tensor_stays_on_the_device(fake, monkeypatch):
    """The folded parameters take a device b_t without reading it on the host (a wait,
    and an error in a capture); a float as before."""
    def read(t):
        raise AssertionError("b_t was read on the host")

    monkeypatch.setattr(torch.Tensor, "__float__", read)
    calls = []
    for name in ("pa_project_fold", "pa_heads_expand", "pa_heads_sum"):
        monkeypatch.setattr(B, name, lambda *a, name=name: calls.append((name, a)))
    monkeypatch.setattr(B, "make_slice_params",
                        lambda A, b, a, b_t, b_t_dev: (float(b_t), b_t_dev))
    s = stack()
    assert s._folded(s.params[0])["sp"][0] == 0.5 and [n for n, _ in calls] == ["pa_project_fold"]
    bt = s.params[1]["b_t"] = torch.tensor([0.25])
    calls.clear()
    host, on_device = s._folded(s.params[1])["sp"]
    names = [n for n, _ in calls]
    assert names == ["pa_project_fold", "pa_heads_expand", "pa_heads_expand", "pa_heads_sum"]
    assert host == 0.0 and calls[2][1][0] is bt and calls[3][1][1] is on_device
    assert set(s.named_parameters()) - set(stack().named_parameters()) == {"1.b_t"}


@pytest.mark.parametrize("b_t", [torch.tensor(0.5), torch.tensor([0.5], dtype=torch.float64),
                                 torch.tensor([0.5], dtype=torch.bfloat16)])
def test_b_t_that_is_read_on_the_host(fake, monkeypatch, b_t):
    """Of another type, or (as a stack on the GPU finds them) on the CPU: as the float."""
    calls = []
    for name in ("pa_project_fold", "pa_heads_expand", "pa_heads_sum"):
        monkeypatch.setattr(B, name, lambda *a, name=name: calls.append(name))
    monkeypatch.setattr(B, "make_slice_params",
                        lambda A, b, a, b_t, b_t_dev: (float(b_t), b_t_dev))
    s = stack()
    if b_t.dtype == torch.float32:
        s._e = s._f = lambda *shape, **kw: torch.empty(*shape)
        s.dev = "cuda"
    s.params[0]["b_t"] = b_t
    assert s._folded(s.params[0])["sp"][0] == 0.5 and calls == ["pa_project_fold"]


@pytest.mark.parametrize("b_t", [torch.zeros(2), torch.zeros(16), torch.zeros(0),
                                 torch.zeros(2, dtype=torch.bfloat16)])
def test_b_t_of_another_size_is_refused(fake, monkeypatch, b_t):
    """(More than one element would be written behind the pair that is added.)"""
    calls = []
    for name in ("pa_project_fold", "pa_heads_expand", "pa_heads_sum"):
        monkeypatch.setattr(B, name, lambda *a, name=name: calls.append(name))
    s = stack()
    s.params[0]["b_t"] = b_t
    with pytest.raises(ValueError, match="b_t"):
        s._folded(s.params[0])
    assert "pa_heads_expand" not in calls


def test_gradients_from_any_iterable(fake):
    it = items_of(300, 400)
    new = [torch.ones(300), torch.ones(400)]
    it.set_grads(g for g in new)
    assert all(d["g"] is g for d, g in zip(it.tensors, new))
