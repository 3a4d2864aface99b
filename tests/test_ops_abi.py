"""The refusals of the operators of include/pa_ops.h, on the CPU: the C ABI's
host validation (every call below fails before anything is launched; the fake
addresses are never dereferenced) and the Python binding's checks (the
library replaced by a recorder)."""
import ctypes
import os
import re

import pytest
import torch

from paper_2502_02414_amd import binding as B
from paper_2502_02414_amd import ops
from test_abi import FAKE, ROOT, fake_addresses

INV, UNS, WS = B.PA_ERR_INVALID, B.PA_ERR_UNSUPPORTED, B.PA_ERR_WORKSPACE


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(B.LIB_PATH):
        from paper_2502_02414_amd import build
        build.build()
    return ops.load()


def test_every_declared_symbol_is_exported(lib):
    with open(os.path.join(ROOT, "include", "pa_ops.h")) as f:
        text = re.sub(r"/\*.*?\*/", "", f.read(), flags=re.S)
    declared = set(re.findall(r"\b(pa_[a-z_0-9]+)\s*\(", text))
    assert declared == set(ops.SYMBOLS)
    for name in declared:
        assert hasattr(lib, name), name
    assert lib.pa_ops_version() == 1


def refused(lib, status, expected, word=""):
    assert status == expected, lib.pa_last_error()
    assert word in lib.pa_last_error().decode()


def joint(**kw):
    d = dict(post=1, pre=1, gate=1, post_eps=1e-5, pre_eps=1e-5, alpha=1.0)
    d.update(kw)
    return ops.pa_residual_norm_params(**d)


@fake_addresses
@pytest.mark.parametrize("kw,over,expected,word", [
    (dict(), dict(N=0), INV, "N"),
    (dict(), dict(C=0), INV, "C"),
    (dict(), dict(C=8), UNS, "C"),
    (dict(), dict(C=60), UNS, "C"),
    (dict(), dict(C=8200), UNS, "C"),
    (dict(), dict(C=4104, dtype=0), UNS, "C"),
    (dict(), dict(N=1 << 40), UNS, "2^40"),
    (dict(), dict(dtype=2), INV, "dtype"),
    (dict(post=3), {}, INV, "post"),
    (dict(pre=-1), {}, INV, "pre"),
    (dict(gate=2), dict(t=FAKE), INV, "gate"),
    (dict(post_eps=0.0), {}, INV, "eps"),
    (dict(pre_eps=float("nan")), {}, INV, "eps"),
    (dict(pre_eps=float("inf")), {}, INV, "eps"),
    (dict(alpha=float("inf")), {}, INV, "alpha"),
    (dict(post=0, post_g=FAKE), {}, INV, "post_g"),
    (dict(pre=0, pre_b=FAKE), dict(h=None), INV, "pre_g"),
    (dict(scale=FAKE + 4), {}, INV, "scale"),
    (dict(), dict(x=None), INV, "x"),
    (dict(), dict(y=FAKE + 2), INV, "y"),
    (dict(), dict(t=FAKE + 8), INV, "t"),
    (dict(), dict(x1=None), INV, "x1"),
    (dict(), dict(hq=FAKE), INV, "hq"),
    (dict(), dict(hs=FAKE), INV, "hs"),
    (dict(pre=0), {}, INV, "pre norm"),
    (dict(pre=0), dict(h=None, hq=FAKE, hs=FAKE), INV, "pre norm"),
])
def test_joint_refusals(lib, kw, over, expected, word):
    a = dict(N=100, C=64, dtype=1, x=FAKE, y=FAKE, t=None, x1=FAKE, h=FAKE, hq=None, hs=None)
    a.update(over)
    p = joint(**kw)
    refused(lib, lib.pa_residual_norm(a["N"], a["C"], a["dtype"], ctypes.byref(p), a["x"], a["y"],
                                      a["t"], a["x1"], a["h"], a["hq"], a["hs"], None),
            expected, word)


@fake_addresses
def test_joint_null_params(lib):
    refused(lib, lib.pa_residual_norm(4, 64, 1, None, FAKE, FAKE, None, FAKE, FAKE, None, None,
                                      None), INV, "params")


@fake_addresses
@pytest.mark.parametrize("kw,over,expected,word", [
    (dict(), dict(dx1=None, dh=None), INV, "one of"),
    (dict(pre=0), {}, INV, "pre norm"),
    (dict(), dict(dx=None), INV, "dx"),
    (dict(), dict(dy=FAKE + 4), INV, "dy"),
    (dict(), dict(t=FAKE), INV, "dt"),
    (dict(), dict(dt=FAKE), INV, "dt"),
    (dict(), dict(x1=None), INV, "x1"),
    (dict(), dict(ws=None), WS, "workspace"),
    (dict(), dict(n=-4), WS, "workspace"),
    (dict(), dict(ws=FAKE + 4), INV, "ws"),
])
def test_joint_backward_refusals(lib, kw, over, expected, word):
    size = ctypes.c_size_t(0)
    assert lib.pa_residual_norm_workspace(5000, 64, 1, ctypes.byref(size)) == B.PA_OK
    a = dict(x1=FAKE, y=FAKE, t=None, dx1=FAKE, dh=FAKE, dx=FAKE, dy=FAKE, dt=None, ws=FAKE, n=0)
    a.update(over)
    p, gr = joint(**kw), ops.pa_residual_norm_grads(None, None, FAKE, None, None)
    refused(lib, lib.pa_residual_norm_backward(
        5000, 64, 1, ctypes.byref(p), a["x1"], a["y"], a["t"], a["dx1"], a["dh"], a["dx"], a["dy"],
        a["dt"], ctypes.byref(gr), a["ws"], size.value + a["n"], None), expected, word)


def test_joint_workspace(lib):
    size = ctypes.c_size_t(0)
    refused(lib, lib.pa_residual_norm_workspace(10, 64, 1, None), INV, "bytes")
    refused(lib, lib.pa_residual_norm_workspace(10, 20, 1, ctypes.byref(size)), UNS)
    for C in (16, 256, 520, 8192):  # partial records per block: nothing that grows with N for good
        assert lib.pa_residual_norm_workspace(1 << 26, C, 1, ctypes.byref(size)) == B.PA_OK
        assert 0 < size.value <= 1024 * 5 * 4 * C


def item(**kw):
    d = dict(n=1000, p=FAKE, copy=None, g=FAKE + (1 << 20), m=FAKE + (2 << 20),
             v=FAKE + (3 << 20), m_scale=None, v_scale=None, wd=0.0, g_dtype=0)
    d.update(kw)
    return ops.pa_adamw_item(**d)


def adam_args(**kw):
    d = dict(lr=1e-3, beta1=0.9, beta2=0.999, eps=1e-8, step=1, seed=0)
    d.update(kw)
    return ops.pa_adamw_args(**d)


def adamw(lib, items, args):
    arr = (ops.pa_adamw_item * len(items))(*items)
    return lib.pa_adamw(len(items), arr, ctypes.byref(args), None)


@fake_addresses
@pytest.mark.parametrize("kw,akw,word", [
    (dict(n=-1), {}, "elements"),
    (dict(n=(1 << 36) + 1), {}, "elements"),
    (dict(p=None), {}, "p is NULL"),
    (dict(p=FAKE + 4), {}, "p is not"),
    (dict(g=None), {}, "g is NULL"),
    (dict(g_dtype=3), {}, "dtype"),
    (dict(copy=FAKE + 8), {}, "copy"),
    (dict(m=None), {}, "m is NULL"),
    (dict(v=FAKE + (3 << 20) + 4), {}, "v is not"),
    (dict(m_scale=FAKE), {}, "go together"),
    (dict(m_scale=FAKE + 2, v_scale=FAKE), {}, "m_scale"),
    (dict(wd=float("nan")), {}, "wd"),
    (dict(m=FAKE + 16), {}, "overlap"),
    (dict(v=FAKE + (2 << 20) + 16), {}, "overlap"),
    (dict(copy=FAKE + 3984), {}, "overlap"),
    (dict(m_scale=FAKE + (2 << 20) + 996, v_scale=FAKE + (4 << 20)), {}, "overlap"),
    (dict(m_scale=FAKE + (4 << 20), v_scale=FAKE + (4 << 20) + 12), {}, "overlap"),
    ({}, dict(lr=float("nan")), "lr"),
    ({}, dict(beta1=1.0), "betas"),
    ({}, dict(beta2=-0.1), "betas"),
    ({}, dict(eps=0.0), "eps"),
    ({}, dict(eps=1e-60), "eps"),
    ({}, dict(step=0), "step"),
    ({}, dict(gscale=FAKE + 2), "gscale"),
    ({}, dict(step_dev=FAKE + 4), "step_dev"),
])
def test_adamw_refusals(lib, kw, akw, word):
    refused(lib, adamw(lib, [item(**kw)], adam_args(**akw)), INV, word)


@fake_addresses
def test_adamw_tensors_that_share_memory_are_refused(lib):
    far = 1 << 24
    other = lambda **kw: item(**{**dict(p=FAKE + far, m=FAKE + far + (2 << 20),
                                        v=FAKE + far + (3 << 20)), **kw})
    refused(lib, adamw(lib, [item(), item()], adam_args()), INV, "overlap")
    refused(lib, adamw(lib, [item(), other(p=FAKE + 3984)], adam_args()), INV, "overlap")
    refused(lib, adamw(lib, [other(m=FAKE + (2 << 20) + 3984)] + [item()], adam_args()), INV,
            "overlap")
    # also where the two are in different launches
    many = [item(p=FAKE + (i + 2) * far, m=FAKE + (i + 2) * far + (2 << 20),
                 v=FAKE + (i + 2) * far + (3 << 20)) for i in range(100)]
    refused(lib, adamw(lib, [item()] + many + [other(v=FAKE)], adam_args()), INV, "overlap")
    refused(lib, lib.pa_adamw(1, None, ctypes.byref(adam_args()), None), INV, "items")
    refused(lib, lib.pa_adamw(0, None, None, None), INV, "args")
    # nothing to do
    assert lib.pa_adamw(0, None, ctypes.byref(adam_args()), None) == B.PA_OK
    assert adamw(lib, [item(n=0, p=None)], adam_args()) == B.PA_OK


def test_adamw_table(lib):
    """The table holds every block's item; its sizes and refusals (host memory
    only)."""
    far = 1 << 26
    ns = [1000, 0, 4096, 4097, 100000]
    items = [item(n=n, p=FAKE + (i + 1) * far, m=FAKE + (i + 1) * far + (2 << 20),
                  v=FAKE + (i + 1) * far + (3 << 20)) for i, n in enumerate(ns)]
    arr = (ops.pa_adamw_item * len(ns))(*items)
    size, blocks = ctypes.c_size_t(0), ctypes.c_int64(0)
    assert lib.pa_adamw_table_size(5, arr, ctypes.byref(size), ctypes.byref(blocks)) == B.PA_OK
    per = [-(-n // 4096) for n in ns]
    assert blocks.value == sum(per)
    host = torch.zeros(size.value // 4 + 2, dtype=torch.int32)
    assert lib.pa_adamw_table(5, arr, host.data_ptr(), size.value) == B.PA_OK
    want = [i for i, k in enumerate(per) for _ in range(k)]
    assert host[size.value // 4 - sum(per):size.value // 4].tolist() == want
    assert host[size.value // 4:].tolist() == [0, 0]
    refused(lib, lib.pa_adamw_table(5, arr, host.data_ptr(), size.value - 1), WS, "table")
    refused(lib, lib.pa_adamw_table(5, arr, None, size.value), WS, "table")
    refused(lib, lib.pa_adamw_table(5, arr, host.data_ptr() + 4, size.value), INV, "host")
    refused(lib, lib.pa_adamw_table_size(5, arr, None, ctypes.byref(blocks)), INV, "bytes")
    arr[4].m = arr[3].p
    refused(lib, lib.pa_adamw_table_size(5, arr, ctypes.byref(size), ctypes.byref(blocks)), INV,
            "overlap")
    huge = [item(n=1 << 36, p=FAKE + (3 * i + 1) * (1 << 39), m=FAKE + (3 * i + 2) * (1 << 39),
                 v=FAKE + (3 * i + 3) * (1 << 39)) for i in range(130)]
    arr = (ops.pa_adamw_item * 130)(*huge)
    refused(lib, lib.pa_adamw_table_size(130, arr, ctypes.byref(size), ctypes.byref(blocks)), UNS,
            "table")
    a = adam_args()
    assert lib.pa_adamw_run(0, 0, None, ctypes.byref(a), None) == B.PA_OK
    refused(lib, lib.pa_adamw_run(3, -1, None, ctypes.byref(a), None), INV, "blocks")
    refused(lib, lib.pa_adamw_run(3, 5, None, ctypes.byref(a), None), INV, "table")
    refused(lib, lib.pa_adamw_run(3, 5, None, ctypes.byref(adam_args(step=0)), None), INV, "step")


@fake_addresses
def test_unpack_refusals(lib):
    refused(lib, lib.pa_adamw_unpack(0, FAKE, FAKE, 1, FAKE, None), INV, "n")
    refused(lib, lib.pa_adamw_unpack(10, None, FAKE, 1, FAKE, None), INV, "codes")
    refused(lib, lib.pa_adamw_unpack(10, FAKE, None, 1, FAKE, None), INV, "scales")
    refused(lib, lib.pa_adamw_unpack(10, FAKE, FAKE, 1, FAKE + 4, None), INV, "out")


@fake_addresses
def test_product_refusals(lib):
    def gemm(N=10, F=64, K=64, q=FAKE, s=FAKE, w=FAKE, sw=FAKE, bias=None, act=0, C=None, D=FAKE,
             dt=1):
        return lib.pa_gemm_i8(N, F, K, q, s, w, sw, bias, act, C, D, dt, None)

    for kw, expected, word in [
            (dict(N=0), INV, "N"), (dict(F=0), INV, "F"), (dict(K=0), INV, "K"),
            (dict(K=131073), UNS, "K"), (dict(F=(1 << 20) + 1), UNS, "F"),
            (dict(N=(1 << 34) + 1), UNS, "N"), (dict(q=None), INV, "q"), (dict(q=FAKE + 8), INV, "q"),
            (dict(s=None), INV, "s"), (dict(w=None), INV, "Wq"), (dict(sw=FAKE + 1), INV, "sw"),
            (dict(bias=FAKE + 2), INV, "bias"), (dict(act=2), INV, "act"),
            (dict(C=FAKE + 2), INV, "C"), (dict(D=None), INV, "D"), (dict(dt=2), INV, "dtype")]:
        refused(lib, gemm(**kw), expected, word)
    size = ctypes.c_size_t(0)
    assert lib.pa_linear_i8_workspace(1000, 64, 60, ctypes.byref(size)) == B.PA_OK
    assert size.value >= 1000 * 64 + 4000
    linear = lambda x, dt, ws, n: lib.pa_linear_i8(1000, 64, 60, x, dt, FAKE, FAKE, None, 0, None,
                                                   FAKE, 1, ws, n, None)
    refused(lib, linear(None, 1, FAKE, size.value), INV, "x")
    refused(lib, linear(FAKE, 2, FAKE, size.value), INV, "dtype")
    refused(lib, linear(FAKE, 1, None, size.value), WS, "workspace")
    refused(lib, linear(FAKE, 1, FAKE, size.value - 1), WS, "workspace")
    refused(lib, linear(FAKE, 1, FAKE + 8, size.value + 8), INV, "ws")
    refused(lib, lib.pa_linear_i8_workspace(10, 64, 64, None), INV, "bytes")
    refused(lib, lib.pa_quant_rows(10, 0, 1, FAKE, FAKE, FAKE, None), INV, "K")
    refused(lib, lib.pa_quant_rows(10, 8, 1, FAKE + 2, FAKE, FAKE, None), INV, "x")
    refused(lib, lib.pa_quant_rows(10, 8, 1, FAKE, None, FAKE, None), INV, "q")
    refused(lib, lib.pa_quant_weight(8, 0, 1, FAKE, FAKE, FAKE, None), INV, "F")
    refused(lib, lib.pa_quant_weight(8, 8, 1, FAKE, FAKE, None, None), INV, "sw")


# ---- the Python binding ----
class _Recorder:
    def __init__(self):
        self.calls = []

    def __getattr__(self, name):
        def call(*args):
            self.calls.append((name, args))
            return B.PA_OK
        return call


@pytest.fixture
def fake(monkeypatch):
    rec = _Recorder()
    monkeypatch.setattr(ops, "load", lambda: rec)
    monkeypatch.setattr(ops, "_dev", lambda t, name, cur=None: 4096)
    monkeypatch.setattr(ops, "_current_device", lambda: 0)
    monkeypatch.setattr(B, "_stream", lambda s=None: None)
    return rec


def z(*shape, dt=torch.float32):
    return torch.zeros(*shape, dtype=dt)


bf = torch.bfloat16


def test_binding_marshals_one_argument_per_parameter(fake):
    x = z(10, 24, dt=bf)
    par = ops.make_residual_norm_params(post="layer", pre="rms", post_g=z(24), scale=z(24))
    gr = ops.make_residual_norm_grads(dscale=z(24))
    ops.pa_residual_norm(x, x, par, x, x, t=x, hq=z(10, 32, dt=torch.int8), hs=z(10))
    ops.pa_residual_norm_backward(x, x, par, x, x, x, x, gr, z(8, dt=torch.uint8), t=x, dt=x)
    it = ops.make_adamw_items([{"p": z(300), "g": z(300, dt=bf), "m": z(300), "v": z(300)}])
    ops.pa_adamw(it, lr=1e-3, gscale=z(1), step_dev=z(1, dt=torch.int64), lr_dev=z(1))
    u8 = z(300, dt=torch.uint8)
    ops.pa_adamw_unpack(u8, z(2), z(300), signed=True)
    ops.pa_quant_rows(x, z(10, 32, dt=torch.int8), z(10))
    ops.pa_quant_weight(z(24, 8), z(8, 32, dt=torch.int8), z(8))
    ops.pa_gemm_i8(z(10, 32, dt=torch.int8), z(10), z(8, 32, dt=torch.int8), z(8), z(10, 8), K=24,
                   bias=z(8), act="gelu", C=z(10, 8))
    ops.pa_linear_i8(x, z(8, 32, dt=torch.int8), z(8), z(10, 8), z(500, dt=torch.uint8))
    assert {n: len(a) for n, a in fake.calls} == {
        "pa_residual_norm": 12, "pa_residual_norm_backward": 16, "pa_adamw": 4,
        "pa_adamw_unpack": 6, "pa_quant_rows": 7, "pa_quant_weight": 7, "pa_gemm_i8": 13,
        "pa_linear_i8": 15}


def test_binding_refuses_before_the_call(fake):
    x, par = z(10, 32, dt=bf), ops.make_residual_norm_params(pre="layer", pre_g=z(32))
    bad = pytest.raises(ValueError)
    with bad:
        ops.pa_residual_norm(x, x[:9], par, x, x)
    with bad:
        ops.pa_residual_norm(x, x.float(), par, x, x)
    with bad:
        ops.pa_residual_norm(x[:, :16], x[:, :16], par, x, x)
    with bad:
        ops.pa_residual_norm(x.half(), x.half(), par, x.half(), x.half())
    with bad:
        ops.pa_residual_norm(x, x, par, x, x, hq=z(10, 31, dt=torch.int8), hs=z(10))
    with bad:
        ops.make_residual_norm_params(pre="batch")
    with bad:
        ops.make_residual_norm_params(pre="layer", pre_g=z(32), pre_b=z(16))
    with bad:
        ops.make_residual_norm_params(pre="layer", pre_g=z(32, dt=bf))
    with bad:
        ops.pa_residual_norm_backward(x, x, par, x, x, x, x,
                                      ops.make_residual_norm_grads(dpre_g=z(16)))
    ok = {"p": z(300), "g": z(300), "m": z(300), "v": z(300)}
    for change in ({"p": z(300, dt=bf)}, {"g": z(299)}, {"m": z(299)}, {"v": z(300, dt=torch.uint8)},
                   {"m_scale": z(2)}, {"copy": z(300)}, {"wdecay": 1.0}, {"g": z(300).half()},
                   {"m": z(300, dt=torch.uint8), "v": z(300, dt=torch.uint8), "m_scale": z(2),
                    "v_scale": z(1)}):
        with bad:
            ops.make_adamw_items([{**ok, **change}])
    it = ops.make_adamw_items([ok])
    with bad:
        ops.pa_adamw(it, lr=1e-3, gscale=z(2))
    with bad:
        ops.pa_adamw(it, lr=1e-3, step_dev=z(1))
    with bad:
        ops.AdamW({"w": z(10)}, lr=1e-3, bits=16)
    with bad:
        ops.AdamW({"w": z(10)}, lr=1e-3, decay=["v"])
    with bad:
        ops.pa_adamw_unpack(z(300, dt=torch.uint8), z(1), z(300), signed=True)
    q, w = z(10, 32, dt=torch.int8), z(8, 32, dt=torch.int8)
    with bad:
        ops.pa_gemm_i8(q, z(9), w, z(8), z(10, 8))
    with bad:
        ops.pa_gemm_i8(q, z(10), w, z(8), z(10, 7))
    with bad:
        ops.pa_gemm_i8(q, z(10), w, z(8), z(10, 8), act="relu")
    with bad:
        ops.pa_gemm_i8(q, z(10), w, z(8), z(10, 8), C=z(10, 8, dt=bf))
    with bad:
        ops.pa_linear_i8(z(10, 24), w[:, :16], z(8), z(10, 8), z(500, dt=torch.uint8))
    with bad:
        ops.pa_linear_i8(z(9, 24), w, z(8), z(10, 8), z(500, dt=torch.uint8))
    assert fake.calls == []


def test_tensors_on_the_cpu_or_not_contiguous_are_refused():
    with pytest.raises(ValueError, match="GPU"):
        ops._dev(z(4, 32), "x", 0)
    with pytest.raises(ValueError, match="GPU"):
        ops._in(z(4, 32), 128, torch.float32, "x", True, 0)


# ---- tensors of one call that share memory ----
MB = 1 << 20


def apart(names):
    """Fake addresses a megabyte apart."""
    return {k: FAKE + (i + 1) * MB for i, k in enumerate(names)}


@fake_addresses
@pytest.mark.parametrize("out,inp", [
    (o, i) for o in ("x1", "h", "hq", "hs") for i in ("x", "y", "t", "scale", "post_g", "pre_b")])
@pytest.mark.parametrize("by", ["same", "last bytes"])
def test_joint_outputs_over_inputs_are_refused(lib, out, inp, by):
    """100 rows of 64 bf16: 12,800 bytes, int8 rows 6,400, scales 400, vectors 256."""
    a = apart(("x", "y", "t", "x1", "h", "hq", "hs", "scale", "post_g", "pre_b"))
    size = {"x1": 12800, "h": 12800, "hq": 6400, "hs": 400}[out]
    a[inp] = a[out] + (0 if by == "same" else size - 16)
    p = joint(**{k: a[k] for k in ("scale", "post_g", "pre_b")})
    refused(lib, lib.pa_residual_norm(100, 64, 1, ctypes.byref(p), a["x"], a["y"], a["t"], a["x1"],
                                      a["h"], a["hq"], a["hs"], None), INV, f"{out} and {inp} overlap")


@fake_addresses
def test_joint_backward_outputs_over_inputs_are_refused(lib):
    outs, ins = ("dx", "dy", "dt", "dscale", "ws"), ("x1", "y", "t", "dx1", "dh", "pre_g")
    size = ctypes.c_size_t(0)
    assert lib.pa_residual_norm_workspace(5000, 64, 1, ctypes.byref(size)) == B.PA_OK

    def call(a):
        p, gr = joint(pre_g=a["pre_g"]), ops.pa_residual_norm_grads(None, None, a["dscale"], None, None)
        return lib.pa_residual_norm_backward(5000, 64, 1, ctypes.byref(p), a["x1"], a["y"], a["t"],
                                             a["dx1"], a["dh"], a["dx"], a["dy"], a["dt"],
                                             ctypes.byref(gr), a["ws"], size.value, None)

    for o in outs:
        for i in ins:
            a = apart(outs + ins)
            a[i] = a[o]
            refused(lib, call(a), INV, f"{o} and {i} overlap")
    for o, q in (("dx", "dy"), ("dy", "dt"), ("dt", "ws"), ("dscale", "ws")):
        a = apart(outs + ins)
        a[q] = a[o]
        refused(lib, call(a), INV, f"{o} and {q} overlap")


@fake_addresses
def test_product_outputs_over_inputs_are_refused(lib):
    """1000 rows of 60 (int8: 64) to 64 outputs, bf16."""
    names = ("q", "s", "w", "sw", "bias", "C", "D", "x", "ws")
    size = ctypes.c_size_t(0)
    assert lib.pa_linear_i8_workspace(1000, 64, 60, ctypes.byref(size)) == B.PA_OK
    gemm = lambda a: lib.pa_gemm_i8(1000, 64, 60, a["q"], a["s"], a["w"], a["sw"], a["bias"], 0,
                                    a["C"], a["D"], 1, None)
    linear = lambda a: lib.pa_linear_i8(1000, 64, 60, a["x"], 1, a["w"], a["sw"], a["bias"], 0,
                                        a["C"], a["D"], 1, a["ws"], size.value, None)
    for call, o, i, by in ([(gemm, "D", i, 0) for i in ("q", "s", "w", "sw", "bias")] +
                           [(linear, "D", i, 0) for i in ("x", "w", "sw", "bias", "ws")] +
                           [(linear, "ws", i, 0) for i in ("x", "w", "sw", "bias", "C")] +
                           # (C may be D itself, and not a part of it)
                           [(gemm, "D", "C", 16), (linear, "D", "C", 127984), (gemm, "D", "C", -16)]):
        a = apart(names)
        a[i] = a[o] + by
        name = {"w": "Wq"}.get(i, i)
        refused(lib, call(a), INV, f"{o} and {name} overlap")
    refused(lib, lib.pa_quant_rows(10, 8, 1, FAKE, FAKE + 144, FAKE + MB, None), INV, "q and x")
    refused(lib, lib.pa_quant_rows(10, 8, 1, FAKE, FAKE + MB, FAKE + MB + 156, None), INV, "q and s")
    refused(lib, lib.pa_quant_weight(8, 8, 1, FAKE, FAKE + 112, FAKE + MB, None), INV, "Wq and W")
    refused(lib, lib.pa_quant_weight(8, 8, 1, FAKE, FAKE + MB, FAKE + 124, None), INV, "sw and W")
    refused(lib, lib.pa_adamw_unpack(300, FAKE, FAKE + MB, 1, FAKE + 288, None), INV, "out and codes")
    refused(lib, lib.pa_adamw_unpack(300, FAKE, FAKE + MB + 1196, 1, FAKE + MB, None), INV,
            "out and scales")
