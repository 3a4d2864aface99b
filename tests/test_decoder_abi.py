"""The refusals of pa_cross_attention and pa_dropout on the CPU (the C ABI's host
validation: every call fails before anything is launched, the fake addresses are never
dereferenced; the binding's checks, the library replaced by a recorder), and the
published values of the generator that dropout's definition is checked with."""
import ctypes
import os

import numpy as np
import pytest
import torch

import ask_ref as R
from paper_2502_02414_amd import binding as B
from paper_2502_02414_amd import ops
from test_abi import FAKE, fake_addresses

INV, UNS, WS = B.PA_ERR_INVALID, B.PA_ERR_UNSUPPORTED, B.PA_ERR_WORKSPACE
MB = 1 << 20


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(B.LIB_PATH):
        from paper_2502_02414_amd import build
        build.build()
    return ops.load()


def refused(lib, status, expected, word=""):
    assert status == expected, lib.pa_last_error()
    assert word in lib.pa_last_error().decode()


def params(**kw):
    d = dict(R=1, Hq=4, Hkv=2, D=32, scale=0.2, q_off=None, k_off=None, mask=None, max_k=0)
    d.update(kw)
    return ops.pa_cross_attention_params(**d)


# a call of 100 queries and 50 states, every tensor a place of its own
PLACES = {k: FAKE + i * MB for i, k in enumerate(
    ("q", "k", "v", "o", "lse", "d_o", "dq", "dk", "dv", "ws", "off"))}
SIZES = dict(Nq=100, Nk=50, dtype=1, ldq=128, ldk=64, ldv=64, ldo=128, lddo=128, lddq=128, lddk=64,
             lddv=64, bytes=MB)


def forward(lib, p, **over):
    a = {**PLACES, **SIZES, **over}
    return lib.pa_cross_attention(
        a["Nq"], a["Nk"], a["dtype"], None if p is None else ctypes.byref(p), a["q"], a["ldq"],
        a["k"], a["ldk"], a["v"], a["ldv"], a["o"], a["ldo"], a["lse"], a["ws"], a["bytes"], None)


def backward(lib, p, **over):
    a = {**PLACES, **SIZES, **over}
    return lib.pa_cross_attention_backward(
        a["Nq"], a["Nk"], a["dtype"], None if p is None else ctypes.byref(p), a["q"], a["ldq"],
        a["k"], a["ldk"], a["v"], a["ldv"], a["o"], a["ldo"], a["lse"], a["d_o"], a["lddo"], a["dq"],
        a["lddq"], a["dk"], a["lddk"], a["dv"], a["lddv"], a["ws"], a["bytes"], None)


COMMON = [
    (dict(R=0), {}, INV, "R"),
    (dict(R=2), {}, INV, "q_off"),
    (dict(q_off=FAKE), {}, INV, "together"),
    (dict(k_off=FAKE), {}, INV, "together"),
    (dict(q_off=FAKE + 4, k_off=FAKE), {}, INV, "aligned"),
    (dict(Hq=0), {}, INV, "Hkv"),
    (dict(Hkv=3), {}, INV, "Hkv"),
    (dict(Hkv=0), {}, INV, "Hkv"),
    (dict(D=0), {}, UNS, "D"),
    (dict(D=12), {}, UNS, "D"),
    (dict(D=136), {}, UNS, "D"),
    (dict(Hq=8192, Hkv=1), {}, UNS, "4096"),
    (dict(scale=0.0), {}, INV, "scale"),
    (dict(scale=-1.0), {}, INV, "scale"),
    (dict(scale=float("inf")), {}, INV, "scale"),
    (dict(scale=float("nan")), {}, INV, "scale"),
    (dict(max_k=-1), {}, INV, "max_k"),
    ({}, dict(dtype=2), INV, "dtype"),
    ({}, dict(Nq=-1), INV, "Nq"),
    ({}, dict(Nk=-1), INV, "Nk"),
    ({}, dict(Nk=1 << 31), UNS, "2^31"),
    ({}, dict(Nq=1 << 30), UNS, "2^31"),
    (dict(R=1 << 24, Hq=4096, Hkv=4096, q_off=FAKE, k_off=FAKE), {}, UNS, "launch"),
    ({}, dict(ldq=120), INV, "ld of q"),
    ({}, dict(ldk=68), INV, "ld of k"),
    ({}, dict(ldv=0), INV, "ld of v"),
    ({}, dict(ldo=132), INV, "ld of o"),
    ({}, dict(q=None), INV, "q is NULL"),
    ({}, dict(k=None), INV, "k is NULL"),
    ({}, dict(v=FAKE + 8), INV, "v"),
    ({}, dict(o=None), INV, "o is NULL"),
]


@fake_addresses
@pytest.mark.parametrize("kw,over,expected,word", COMMON + [
    ({}, dict(lse=FAKE + 2), INV, "lse"),
    ({}, dict(o=PLACES["q"]), INV, "o and q overlap"),
    ({}, dict(o=PLACES["v"] + 6144 - 128), INV, "overlap"),
    ({}, dict(lse=PLACES["k"]), INV, "lse and k overlap"),
    ({}, dict(lse=PLACES["o"] + 256), INV, "overlap"),
    # columns of o that reach into q's, in rows of one pitch
    ({}, dict(ldq=256, ldo=256, o=PLACES["q"] + 240), INV, "overlap"),
    (dict(mask=PLACES["o"]), {}, INV, "mask"),
    (dict(q_off=PLACES["o"], k_off=PLACES["off"]), {}, INV, "q_off"),
])
def test_forward_refusals(lib, kw, over, expected, word):
    refused(lib, forward(lib, params(**kw), **over), expected, word)


@fake_addresses
@pytest.mark.parametrize("kw,over,expected,word", COMMON + [
    ({}, dict(lse=None), INV, "lse"),
    ({}, dict(d_o=None), INV, "d_o"),
    ({}, dict(dq=None), INV, "dq"),
    ({}, dict(dk=None), INV, "together"),
    ({}, dict(dv=None), INV, "together"),
    ({}, dict(dk=FAKE + 2), INV, "dk"),
    ({}, dict(lddq=130), INV, "ld of dq"),
    ({}, dict(lddk=56), INV, "ld of dk"),
    ({}, dict(dq=PLACES["q"]), INV, "dq and q overlap"),
    ({}, dict(dq=PLACES["d_o"]), INV, "overlap"),
    ({}, dict(dk=PLACES["dv"] + 64), INV, "dk and dv overlap"),
    # side by side, but closer than they are wide
    ({}, dict(lddk=128, lddv=128, dv=PLACES["dk"] + 112), INV, "dk and dv overlap"),
    ({}, dict(ws=None), WS, "workspace"),
    ({}, dict(bytes=16), WS, "workspace"),
    ({}, dict(ws=FAKE + 4), INV, "ws"),
    ({}, dict(ws=PLACES["dq"]), INV, "overlap"),
])
def test_backward_refusals(lib, kw, over, expected, word):
    refused(lib, backward(lib, params(**kw), **over), expected, word)


@fake_addresses
def test_null_params_and_workspace(lib):
    refused(lib, forward(lib, None), INV, "params")
    refused(lib, backward(lib, None), INV, "params")
    n = ctypes.c_size_t(0)
    p = params()
    refused(lib, lib.pa_cross_attention_workspace(1, 1, 1, None, 0, ctypes.byref(n)), INV, "params")
    refused(lib, lib.pa_cross_attention_workspace(1, 1, 1, ctypes.byref(p), 0, None), INV, "bytes")
    # a few queries over many states are worked on in pieces, which need room
    assert lib.pa_cross_attention_workspace(2, 100000, 1, ctypes.byref(p), 0,
                                            ctypes.byref(n)) == B.PA_OK
    assert n.value > 0
    refused(lib, forward(lib, p, Nq=2, Nk=100000, k=FAKE + 64 * MB, v=FAKE + 128 * MB, ws=None),
            WS, "workspace")
    refused(lib, forward(lib, p, Nq=2, Nk=100000, k=FAKE + 64 * MB, v=FAKE + 128 * MB,
                         bytes=n.value - 1), WS, "workspace")
    # and never more than a few hundred MB beside the tensors' own size
    for Nq, Nk in ((1, 1 << 24), (1 << 20, 64), (1 << 14, 1 << 14), (64, 1 << 20), (5000, 5000)):
        for back in (0, 1):
            assert lib.pa_cross_attention_workspace(Nq, Nk, 1, ctypes.byref(p), back,
                                                    ctypes.byref(n)) == B.PA_OK
            assert n.value <= 16 * (Nq * 4 + Nk * 2) * 32 + (512 << 20), (Nq, Nk, back)


def test_nothing_to_do(lib):
    """No queries (and, for the backward, no states): done without a tensor."""
    p, none = params(), {k: None for k in PLACES}
    assert forward(lib, p, **{**none, "Nq": 0, "Nk": 0}) == B.PA_OK
    assert backward(lib, p, **{**none, "Nq": 0, "Nk": 0}) == B.PA_OK
    assert lib.pa_dropout(0, 1, None, None, None, 0.5, 0, 0, None, None) == B.PA_OK


@fake_addresses
@pytest.mark.parametrize("over,expected,word", [
    (dict(n=-1), INV, "n"),
    (dict(n=1 << 41), INV, "n"),
    (dict(dtype=3), INV, "dtype"),
    (dict(p=-0.1), INV, "p"),
    (dict(p=1.0), INV, "p"),
    (dict(p=65535.5 / 65536), INV, "p"),
    (dict(p=float("nan")), INV, "p"),
    (dict(y=None), INV, "y"),
    (dict(out=None), INV, "out"),
    (dict(y=FAKE + 8), INV, "y"),
    (dict(r=FAKE + MB + 2), INV, "r"),
    (dict(out=FAKE + 16), INV, "out and y overlap"),
    (dict(out=FAKE + MB + 16), INV, "out and r overlap"),
    (dict(offset_dev=FAKE + 4), INV, "offset_dev"),
    (dict(offset_dev=FAKE + 2 * MB + 8), INV, "overlap"),
])
def test_dropout_refusals(lib, over, expected, word):
    a = dict(n=1000, dtype=1, y=FAKE, r=FAKE + MB, out=FAKE + 2 * MB, p=0.1, offset_dev=None)
    a.update(over)
    refused(lib, lib.pa_dropout(a["n"], a["dtype"], a["y"], a["r"], a["out"], a["p"], 1, 2,
                                a["offset_dev"], None), expected, word)


# ---- the binding ----
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
    monkeypatch.setattr(ops, "_current_device", lambda: -1)  # (where CPU tensors are)
    monkeypatch.setattr(B, "_stream", lambda s=None: None)
    return rec


BF, F32, I64 = torch.bfloat16, torch.float32, torch.int64


def tensors(Nq=10, Nk=6, Hq=4, Hkv=2, D=16, dt=BF):
    z = lambda n, h: torch.zeros(n, h, D, dtype=dt)
    return {"q": z(Nq, Hq), "k": z(Nk, Hkv), "v": z(Nk, Hkv), "o": z(Nq, Hq),
            "lse": torch.zeros(Hq, Nq), "d_o": z(Nq, Hq), "dq": z(Nq, Hq), "dk": z(Nk, Hkv),
            "dv": z(Nk, Hkv)}


def test_binding_marshals_one_argument_per_parameter(fake):
    par = ops.make_cross_attention(4, 2, 16, q_off=torch.tensor([0, 3, 10]),
                                   k_off=torch.tensor([0, 2, 6]), mask=torch.ones(6, dtype=torch.bool))
    assert (par.st.R, par.st.Hq, par.st.Hkv, par.st.D) == (2, 4, 2, 16)
    assert abs(par.st.scale - 0.25) < 1e-7
    t = tensors()
    kv = torch.zeros(6, 2, 2, 16, dtype=BF)
    ops.pa_cross_attention(t["q"], kv[:, 0], kv[:, 1], par, t["o"].view(10, 64), t["lse"])
    ops.pa_cross_attention_backward(t["q"], kv[:, 0], kv[:, 1], t["o"], t["lse"], par, t["d_o"],
                                    t["dq"], t["dk"], t["dv"])
    ops.pa_cross_attention_backward(t["q"], t["k"], t["v"], t["o"], t["lse"], par, t["d_o"], t["dq"])
    ops.pa_dropout(t["q"], t["o"], 0.1, -1, r=t["d_o"])
    (n0, a0), (n1, a1), (n2, a2), (n3, a3) = fake.calls
    assert (n0, len(a0)) == ("pa_cross_attention", 16)
    assert a0[:3] == (10, 6, 1) and a0[5] == 64 and a0[7] == a0[9] == 64 and a0[11] == 64
    assert (n1, len(a1)) == ("pa_cross_attention_backward", 24)
    assert a1[18] == a1[20] == 32
    assert a2[17:21] == (None, 0, None, 0)
    assert (n3, len(a3)) == ("pa_dropout", 10) and a3[6] == (1 << 64) - 1


@pytest.mark.parametrize("change,word", [
    (dict(q=torch.zeros(10, 4, 24, dtype=BF)), "q"),
    (dict(q=torch.zeros(10, dtype=BF)), "q"),
    (dict(q=torch.zeros(10, 4, 16, dtype=torch.float16)), "dtype"),
    (dict(k=torch.zeros(6, 2, 16)), "k"),
    (dict(v=torch.zeros(7, 2, 16, dtype=BF)), "v"),
    (dict(v=torch.zeros(2, 6, 16, dtype=BF).transpose(0, 1)), "row"),
    (dict(o=torch.zeros(10, 4, 32, dtype=BF)[:, :, ::2]), "row"),
    (dict(lse=torch.zeros(39)), "lse"),
    (dict(lse=torch.zeros(4, 10, dtype=BF)), "lse"),
])
def test_binding_refuses_tensors_that_do_not_fit(fake, change, word):
    par = ops.make_cross_attention(4, 2, 16)
    t = {**tensors(), **change}
    with pytest.raises(ValueError, match=word):
        ops.pa_cross_attention(t["q"], t["k"], t["v"], par, t["o"], t["lse"])
    assert not fake.calls


@pytest.mark.parametrize("change,word", [
    (dict(lse=None), "lse"),
    (dict(dk=None), "together"),
    (dict(d_o=torch.zeros(10, 4, 16)), "d_o"),
    (dict(dq=torch.zeros(9, 4, 16, dtype=BF)), "dq"),
    (dict(dv=torch.zeros(6, 1, 16, dtype=BF)), "dv"),
])
def test_binding_refuses_gradients_that_do_not_fit(fake, change, word):
    par = ops.make_cross_attention(4, 2, 16)
    t = {**tensors(), **change}
    with pytest.raises(ValueError, match=word):
        ops.pa_cross_attention_backward(t["q"], t["k"], t["v"], t["o"], t["lse"], par, t["d_o"],
                                        t["dq"], t["dk"], t["dv"])
    assert not fake.calls


def test_binding_refuses_parameters_that_do_not_fit(fake):
    off = torch.tensor([0, 5])
    for kw, word in ((dict(q_off=off), "together"), (dict(q_off=off, k_off=off.int()), "k_off"),
                     (dict(q_off=off, k_off=torch.tensor([0, 1, 2])), "k_off"),
                     (dict(mask=torch.ones(6)), "mask")):
        with pytest.raises(ValueError, match=word):
            ops.make_cross_attention(4, 2, 16, **kw)
    par, t = ops.make_cross_attention(4, 2, 16, mask=torch.ones(5, dtype=torch.uint8)), tensors()
    with pytest.raises(ValueError, match="mask"):
        ops.pa_cross_attention(t["q"], t["k"], t["v"], par, t["o"])
    par.device = 3  # made on another device than the current one
    with pytest.raises(ValueError, match="device"):
        ops.pa_cross_attention(t["q"], t["k"], t["v"], par, t["o"])
    y = torch.zeros(8, dtype=BF)
    for kw, word in ((dict(out=torch.zeros(8)), "out"), (dict(out=y, r=torch.zeros(9, dtype=BF)), "r"),
                     (dict(out=y, offset_dev=torch.zeros(1)), "offset_dev"),
                     (dict(out=torch.zeros(16, dtype=BF)[::2]), "contiguous|GPU")):
        with pytest.raises(ValueError, match=word):
            ops.pa_dropout(y, p=0.1, seed=1, **kw)
    assert not fake.calls


def test_published_values_of_the_generator():
    """Philox-4x32-10's known answers: counters and keys of zeros, of ones, and the
    digits of pi."""
    for ctr, key, want in (
            ([0] * 4, [0] * 2, [0x6627E8D5, 0xE169C58D, 0xBC57AC4C, 0x9B00DBD8]),
            ([0xFFFFFFFF] * 4, [0xFFFFFFFF] * 2, [0x408F276D, 0x41C83B0E, 0xA20BC7C6, 0x6D5451FD]),
            ([0x243F6A88, 0x85A308D3, 0x13198A2E, 0x03707344], [0xA4093822, 0x299F31D0],
             [0xD16CFE09, 0x94FDCCEB, 0x5001E420, 0x24126EA1])):
        assert R.philox([ctr], key)[0].tolist() == want


def test_elements_of_one_seed_differ_between_offsets():
    a, scale = R.kept(np.arange(4096), 0.25, 5, 1)
    b, _ = R.kept(np.arange(4096), 0.25, 5, 2)
    c, _ = R.kept(np.arange(4096), 0.25, 6, 1)
    assert scale == 65536 / (65536 - 16384)
    for x in (a, b, c):  # five standard deviations
        assert abs(x.double().mean().item() - 0.75) < 5 * (0.1875 / 4096) ** 0.5
    for x in (b, c):
        assert abs((a == x).double().mean().item() - 0.625) < 5 * (0.234375 / 4096) ** 0.5


@fake_addresses
@pytest.mark.parametrize("call", [forward, backward])
def test_a_scale_that_the_kernels_cannot_hold(lib, call):
    """They work with scale log2 e, which is infinite from 2.36e38 on (and would make a
    score of 0 NaN): refused above 2^127, and nothing else is wrong with 2^127."""
    for scale in (2.0 ** 127 * (1 + 2.0 ** -23), 2.36e38, 3.4e38):
        refused(lib, call(lib, params(scale=scale)), INV, "scale")
    refused(lib, call(lib, params(scale=2.0 ** 127), q=None), INV, "q is NULL")


@pytest.mark.parametrize("C,H,Hkv,word", [
    (100, 5, None, "multiple of 8"), (60, 2, None, "multiple of 8"), (512, 2, None, "128"),
    (64, 3, None, "divide"), (64, 4, 3, "divide"), (64, 0, None, "divide"), (64, 4, 0, "divide")])
def test_a_decoder_of_heads_that_its_attention_does_not_take(C, H, Hkv, word):
    """Refused when it is made, before it allocates anything."""
    from paper_2502_02414_amd.stack import QueryDecoder
    with pytest.raises(ValueError, match=word):
        QueryDecoder(10, C, H, [], BF, Hkv=Hkv, device="nowhere")


@fake_addresses
def test_where_the_records_of_few_states_end(lib):
    """The backward of few states keeps a record of 64 states for a block, up to 2^25 floats:
    2,048 requests of 8 heads of 32, and not one more."""
    n, sizes = ctypes.c_size_t(0), []
    for requests in (2048, 2049):
        p = params(R=requests, Hq=8, Hkv=8, D=32, max_k=64, q_off=FAKE, k_off=FAKE)
        assert lib.pa_cross_attention_workspace(3 * requests, 64 * requests, 1, ctypes.byref(p), 1,
                                                ctypes.byref(n)) == B.PA_OK
        sizes.append(n.value)
    assert sizes[0] == 2 * 4 * (1 << 25)
    # delta alone (and no pieces): a float for each row and head
    assert sizes[1] < 3 * 2049 * 8 * 4 + 256


def test_a_decoder_of_no_layers_gives_its_states_no_gradient():
    """(What was in memory was returned.)"""
    from paper_2502_02414_amd.stack import QueryDecoder
    dec = QueryDecoder(5, 16, 2, [], F32, device="cpu")
    dec._e = lambda *s, dt=None: torch.full(s, float("nan"), dtype=dt or F32)
    x, s, dy = torch.ones(5, 16), torch.ones(3, 24), torch.full((5, 16), 2.0)
    assert torch.equal(dec.forward(x, s), x)
    dx, ds, grads = dec.backward(dy)
    assert torch.equal(dx, dy) and torch.equal(ds, torch.zeros(3, 24)) and grads == []
