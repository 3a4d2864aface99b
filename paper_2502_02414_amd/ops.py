"""Thin Python binding of include/pa_ops.h, beside ``binding`` (same library,
same manner): the operators around the block stack.

  pa_residual_norm(_backward)  norm after a block, its gate and residual scale,
                               the residual add, norm before the next block
  pa_adamw                     one AdamW step over many tensors, moments in 32
                               or in 8 bits; ``AdamW`` keeps a model's moments
  pa_linear_i8                 a linear layer in 8-bit integers (pa_quant_rows,
                               pa_quant_weight, pa_gemm_i8: its parts)

Tensors are contiguous GPU tensors on the current device; outputs are passed
in.  Each wrapper checks device, dtype, size and contiguity against the call,
and raises ValueError, or PAError with the library's message.
"""
from __future__ import annotations

import ctypes

from . import binding as B
from .binding import PA_BF16, PA_F32, PAError  # noqa: F401

SYMBOLS = (
    "pa_ops_version", "pa_residual_norm", "pa_residual_norm_backward",
    "pa_residual_norm_workspace", "pa_adamw", "pa_adamw_table_size", "pa_adamw_table",
    "pa_adamw_run", "pa_adamw_unpack", "pa_quant_rows",
    "pa_quant_weight", "pa_gemm_i8", "pa_linear_i8", "pa_linear_i8_workspace",
)

NORMS = {None: 0, "none": 0, "layer": 1, "rms": 2}
GATES = {"linear": 0, "sigmoid": 1}
ACTS = {None: 0, "none": 0, "gelu": 1}
BLOCK = 256  # elements that share a scale of the 8-bit moments

_P = ctypes.c_void_p


class pa_residual_norm_params(ctypes.Structure):
    _fields_ = [("post", ctypes.c_int32), ("pre", ctypes.c_int32), ("gate", ctypes.c_int32),
                ("post_eps", ctypes.c_float), ("pre_eps", ctypes.c_float),
                ("alpha", ctypes.c_float), ("post_g", _P), ("post_b", _P), ("scale", _P),
                ("pre_g", _P), ("pre_b", _P)]


class pa_residual_norm_grads(ctypes.Structure):
    _fields_ = [(n, _P) for n in ("dpost_g", "dpost_b", "dscale", "dpre_g", "dpre_b")]


class pa_adamw_item(ctypes.Structure):
    _fields_ = [("n", ctypes.c_int64)] + [(k, _P) for k in (
        "p", "copy", "g", "m", "v", "m_scale", "v_scale")] + [
            ("wd", ctypes.c_float), ("g_dtype", ctypes.c_int32)]


class pa_adamw_args(ctypes.Structure):
    _fields_ = [("lr", ctypes.c_double), ("beta1", ctypes.c_double), ("beta2", ctypes.c_double),
                ("eps", ctypes.c_double), ("step", ctypes.c_int64), ("seed", ctypes.c_uint64),
                ("gscale", _P), ("lr_dev", _P), ("step_dev", _P)]


_lib = None


def load():
    """libpa.so with this header's calls declared."""
    global _lib
    if _lib is not None:
        return _lib
    lib = B.load()
    I64, I32, S = ctypes.c_int64, ctypes.c_int, ctypes.c_size_t
    Sp = ctypes.POINTER(S)
    NP, NG = ctypes.POINTER(pa_residual_norm_params), ctypes.POINTER(pa_residual_norm_grads)
    lib.pa_residual_norm.argtypes = [I64, I32, I32, NP, _P, _P, _P, _P, _P, _P, _P, _P]
    lib.pa_residual_norm_backward.argtypes = [I64, I32, I32, NP] + [_P] * 8 + [NG, _P, S, _P]
    lib.pa_residual_norm_workspace.argtypes = [I64, I32, I32, Sp]
    lib.pa_adamw.argtypes = [I32, ctypes.POINTER(pa_adamw_item), ctypes.POINTER(pa_adamw_args), _P]
    lib.pa_adamw_table_size.argtypes = [I32, ctypes.POINTER(pa_adamw_item), Sp,
                                        ctypes.POINTER(I64)]
    lib.pa_adamw_table.argtypes = [I32, ctypes.POINTER(pa_adamw_item), _P, S]
    lib.pa_adamw_run.argtypes = [I32, I64, _P, ctypes.POINTER(pa_adamw_args), _P]
    lib.pa_adamw_unpack.argtypes = [I64, _P, _P, I32, _P, _P]
    lib.pa_quant_rows.argtypes = [I64, I32, I32, _P, _P, _P, _P]
    lib.pa_quant_weight.argtypes = [I32, I32, I32, _P, _P, _P, _P]
    lib.pa_gemm_i8.argtypes = [I64, I32, I32, _P, _P, _P, _P, _P, I32, _P, _P, I32, _P]
    lib.pa_linear_i8.argtypes = [I64, I32, I32, _P, I32, _P, _P, _P, I32, _P, _P, I32, _P, S, _P]
    lib.pa_linear_i8_workspace.argtypes = [I64, I32, I32, Sp]
    for name in SYMBOLS:
        getattr(lib, name).restype = ctypes.c_int
    _lib = lib
    return lib


def _check(status: int):
    if status != B.PA_OK:
        raise PAError(status, load().pa_last_error().decode())


def _code(dtype, name):
    code = B._codes[dtype]
    if code is None:
        raise ValueError(f"{name}: dtype {dtype} is neither float32 nor bfloat16")
    return code


_device = None


def _current_device() -> int:
    global _device
    if _device is None:
        import torch
        torch.cuda.current_device()
        _device = torch._C._cuda_getDevice
    return _device()


# The checks below run for every tensor of every call: one that holds takes a few
# comparisons, and only one that fails goes on to find out what to say.
def _dev(t, name, cur=None):
    """Pointer of a contiguous tensor on the current device (its index, where a
    call has asked before)."""
    if t.get_device() != (_current_device() if cur is None else cur) or not t.is_contiguous():
        B._ptr(t)
        raise ValueError(f"{name}: on {t.device}, not on the current device")
    return t.data_ptr()


def _in(t, n, dtype, name, required=True, cur=None):
    """Pointer of t after checking it against n elements of a torch dtype."""
    if t is None:
        if required:
            raise ValueError(f"{name} is required")
        return None
    if t.get_device() == cur and t.dtype == dtype and t.numel() == n and t.is_contiguous():
        return t.data_ptr()
    if t.dtype != dtype:
        raise ValueError(f"{name}: dtype {t.dtype}, the call needs {dtype}")
    if t.numel() != n:
        raise ValueError(f"{name}: {t.numel()} elements, the call needs {n}")
    return _dev(t, name, cur)


_torch_module = None


def _torch():
    global _torch_module
    if _torch_module is None:
        import torch
        _torch_module = torch
    return _torch_module


_capture = None


def _capturing(stream=None) -> bool:
    """Whether calls on a stream (the current one, if none is given) go into a graph."""
    global _capture
    if _capture is None:
        _capture = _torch().cuda.is_current_stream_capturing
    if stream is None:
        return _capture()
    with _torch().cuda.stream(stream):
        return _capture()


def pa_ops_version() -> int:
    return load().pa_ops_version()


# ---- the joint between two blocks ----
class ResidualNormParams:
    """The host struct of the joint's parameters and the tensors it points at, on
    one device (None: no tensors)."""

    def __init__(self, st, C, tensors):
        self.st, self.C, self.tensors = st, C, tensors
        self.device = None if C is None else _current_device()
        self.ref = ctypes.byref(st)
        self.pre = st.pre
        self.post = st.post


def _vectors(named):
    """Pointers of fp32 vectors of one length, and that length."""
    f32, C, out = _torch().float32, None, {}
    for k, t in named.items():
        if t is not None:
            C = t.numel() if C is None else C
            out[k] = _in(t, C, f32, k)
    return out, C


def make_residual_norm_params(post=None, pre=None, alpha=1.0, scale=None, gate="sigmoid",
                              post_g=None, post_b=None, pre_g=None, pre_b=None, post_eps=1e-5,
                              pre_eps=1e-5) -> ResidualNormParams:
    """post, pre: None, "layer" or "rms"; scale and the gains and biases: fp32
    [C] or None; gate: "linear" or "sigmoid" (of the gate tensor t, where a
    call has one)."""
    for what, v, table in (("post", post, NORMS), ("pre", pre, NORMS), ("gate", gate, GATES)):
        if v not in table:
            raise ValueError(f"{what}: {v!r} is not one of {sorted(map(str, table))}")
    named = dict(post_g=post_g, post_b=post_b, scale=scale, pre_g=pre_g, pre_b=pre_b)
    ptr, C = _vectors(named)
    st = pa_residual_norm_params(NORMS[post], NORMS[pre], GATES[gate], float(post_eps),
                                 float(pre_eps), float(alpha), *(ptr.get(k) for k in named))
    return ResidualNormParams(st, C, named)


class ResidualNormGrads:
    def __init__(self, st, C, tensors):
        self.C, self.tensors, self.ref = C, tensors, ctypes.byref(st)
        self.device = None if C is None else _current_device()


def make_residual_norm_grads(dpost_g=None, dpost_b=None, dscale=None, dpre_g=None,
                             dpre_b=None) -> ResidualNormGrads:
    """fp32 [C] outputs of the backward, each optional."""
    named = dict(dpost_g=dpost_g, dpost_b=dpost_b, dscale=dscale, dpre_g=dpre_g, dpre_b=dpre_b)
    ptr, C = _vectors(named)
    return ResidualNormGrads(pa_residual_norm_grads(*(ptr.get(k) for k in named)), C, named)


def _here(had, name, cur):
    """Refuses a struct whose pointers are another device's than the current one."""
    if had is not None and had != cur:
        raise ValueError(f"{name}: on device {had}, not on the current one")


def _joint(x, name, par, cur, gr=None):
    _here(par.device, "the parameters", cur)
    if gr is not None:
        _here(gr.device, "the gradients", cur)
    if x.dim() != 2:
        raise ValueError(f"{name} must be [N, C]")
    N, C = x.shape
    if par.C is not None and par.C != C:
        raise ValueError(f"{name} has {C} channels, the parameters {par.C}")
    if gr is not None and gr.C is not None and gr.C != C:
        raise ValueError(f"{name} has {C} channels, the gradients {gr.C}")
    return N, C, N * C, _code(x.dtype, name)


def padded(K: int) -> int:
    """Bytes between the rows of an int8 matrix of K columns."""
    return (K + 15) // 16 * 16


def pa_residual_norm(x, y, par, x1, h=None, t=None, hq=None, hs=None, stream=None):
    """x1 = alpha x + scale gate(t) post(y); h = pre(x1), in x's dtype (h) and /
    or as int8 rows hq [N, padded(C)] with scales hs [N]."""
    cur = _current_device()
    N, C, n, code = _joint(x, "x", par, cur)
    dt = x.dtype
    if hq is not None:
        torch = _torch()
        hqp = _in(hq, N * padded(C), torch.int8, "hq")
        hsp = _in(hs, N, torch.float32, "hs")
    else:
        hqp, hsp = None, (None if hs is None else _dev(hs, "hs"))
    _check(load().pa_residual_norm(
        N, C, code, par.ref, _dev(x, "x", cur), _in(y, n, dt, "y", True, cur),
        None if t is None else _in(t, n, dt, "t", True, cur), _in(x1, n, dt, "x1", True, cur),
        None if h is None else _in(h, n, dt, "h", True, cur), hqp, hsp, B._stream(stream)))


def residual_norm_workspace(N, C, dtype, device="cuda"):
    """A uint8 workspace for the backward of [N, C] tensors of a torch dtype."""
    k = ctypes.c_size_t(0)
    _check(load().pa_residual_norm_workspace(N, C, _code(dtype, "dtype"), ctypes.byref(k)))
    return _torch().empty(k.value, dtype=_torch().uint8, device=device)


def pa_residual_norm_backward(x1, y, par, dx1, dh, dx, dy, gr=None, ws=None, t=None, dt=None,
                              stream=None):
    """The chain rule: dx1 and dh (either may be None) to dx, dy, dt and the
    parameters' gradients gr (make_residual_norm_grads)."""
    cur = _current_device()
    N, C, n, code = _joint(x1, "x1", par, cur, gr)
    ty = x1.dtype
    _check(load().pa_residual_norm_backward(
        N, C, code, par.ref, _dev(x1, "x1", cur), _in(y, n, ty, "y", True, cur),
        _in(t, n, ty, "t", False, cur), _in(dx1, n, ty, "dx1", False, cur),
        _in(dh, n, ty, "dh", False, cur), _in(dx, n, ty, "dx", True, cur),
        _in(dy, n, ty, "dy", True, cur), _in(dt, n, ty, "dt", False, cur),
        gr.ref if gr is not None else None, None if ws is None else _dev(ws, "ws", cur),
        B._nbytes(ws), B._stream(stream)))


# ---- AdamW ----
class AdamWItems:
    """The host array of pa_adamw's tensors, which have to stay where they are.
    ``set_grad`` exchanges a gradient; ``table`` lays the tensors out on the
    device for one launch per step, until a gradient moves.  A graph that a step
    was captured into reads its table and its gradients again in every replay: the
    items keep both, and have to live as long as the graph."""

    def __init__(self, n):
        self.n = n
        self.home = None  # the tensors' device (None: no tensors yet)
        self.arr = (pa_adamw_item * max(n, 1))()
        self.tensors = [None] * n
        self.dev, self.blocks, self.moved = None, 0, 0
        self.captured = []  # tables that graphs read
        self.captured_grads = []  # and gradients, a list for every set of them
        self.grads = [None] * n  # (pointer, elements, dtype) of each gradient

    def set_grad(self, i, g):
        it = self.arr[i]
        if g.numel() != it.n:
            raise ValueError(f"g of item {i}: {g.numel()} elements, the item has {it.n}")
        code, ptr = _code(g.dtype, "g"), _dev(g, "g")
        if ptr != it.g or code != it.g_dtype:
            it.g, it.g_dtype = ptr, code
            self.dev = None
            self.moved += 1
        self.tensors[i]["g"] = g
        self.grads[i] = (ptr, it.n, g.dtype)

    def set_grads(self, gs):
        """All gradients, in the items' order."""
        gs = list(gs)
        if len(gs) != self.n:
            raise ValueError(f"{len(gs)} gradients for {self.n} items")
        cur = _current_device()
        for i, (g, had, d) in enumerate(zip(gs, self.grads, self.tensors)):
            # (one that stayed where it was takes its checks alone)
            if had and (g.data_ptr(), g.numel(), g.dtype) == had and g.get_device() == cur \
                    and g.is_contiguous():
                d["g"] = g
            else:
                self.set_grad(i, g)

    def table(self):
        """Makes the device table (a copy from host memory that has arrived when
        this returns, so that every stream may read it)."""
        torch = _torch()
        _here(self.home, "items", _current_device())
        size, blocks = ctypes.c_size_t(0), ctypes.c_int64(0)
        _check(load().pa_adamw_table_size(self.n, self.arr, ctypes.byref(size),
                                          ctypes.byref(blocks)))
        host = torch.empty(-(-max(size.value, 8) // 8), dtype=torch.int64)
        _check(load().pa_adamw_table(self.n, self.arr, host.data_ptr(), 8 * host.numel()))
        dev = host.to("cuda")
        torch.cuda.current_stream().synchronize()
        self.dev, self.blocks, self.stream = dev, blocks.value, B._stream()
        self.ptr = dev.data_ptr()

    def on(self, stream, handle, capturing):
        """The table's pointer for a launch on a stream (its handle given); a
        stream other than the table's keeps its memory from being handed out."""
        if capturing:
            if not any(t is self.dev for t in self.captured):
                self.captured.append(self.dev)
        elif handle != self.stream:
            self.dev.record_stream(stream or _torch().cuda.current_stream())
        return self.ptr

    def hold(self, stream, handle, capturing, scalars):
        """Before a step on a stream (its handle given): of one that is captured, the
        gradients are kept.  On a stream other than the current one the memory of the
        gradients, which the next step lets go of, and of the device scalars is not
        handed out before the step has run."""
        if capturing:
            now = [d.get("g") for d in self.tensors]
            if not any(all(a is b for a, b in zip(now, had)) for had in self.captured_grads):
                self.captured_grads.append(now)
        elif stream is not None and handle != B._stream():
            for t in (*(d.get("g") for d in self.tensors), *scalars):
                if t is not None:
                    t.record_stream(stream)


def make_adamw_items(items, table=True) -> AdamWItems:
    """items: dicts with p (fp32), g (fp32 or bf16), m and v (fp32; or uint8
    with m_scale and v_scale, fp32 [ceil(n / 256)]), optionally copy (bf16)
    and wd.  table: with all gradients given, as a table on the device
    (AdamWItems.table; waits for the current stream)."""
    torch = _torch()
    f32 = torch.float32
    out = AdamWItems(len(items))
    if items:
        out.home = _current_device()
    for i, d in enumerate(items):
        extra = set(d) - {"p", "g", "m", "v", "m_scale", "v_scale", "copy", "wd"}
        if extra:
            raise ValueError(f"item {i}: unknown {sorted(extra)}")
        n, it = d["p"].numel(), out.arr[i]
        q8 = d.get("m_scale") is not None or d.get("v_scale") is not None
        state, blocks = torch.uint8 if q8 else f32, -(-n // BLOCK)
        it.n = n
        it.p = _in(d["p"], n, f32, "p")
        it.copy = _in(d.get("copy"), n, torch.bfloat16, "copy", False)
        it.m, it.v = _in(d["m"], n, state, "m"), _in(d["v"], n, state, "v")
        if q8:
            it.m_scale = _in(d.get("m_scale"), blocks, f32, "m_scale")
            it.v_scale = _in(d.get("v_scale"), blocks, f32, "v_scale")
        it.wd = float(d.get("wd", 0.0))
        out.tensors[i] = dict(d)
        if d.get("g") is not None:
            out.set_grad(i, d["g"])
    if table and items and all(d.get("g") is not None and d["p"].is_cuda for d in items) \
            and not _capturing():
        out.table()
    return out


def pa_adamw(items, lr, step=1, beta1=0.9, beta2=0.999, eps=1e-8, seed=0, gscale=None,
             lr_dev=None, step_dev=None, stream=None):
    """One step over the tensors of make_adamw_items; gscale: a device fp32
    scalar that every gradient is multiplied by; lr_dev (fp32), step_dev
    (int64): device scalars in place of lr and step, for captured graphs."""
    torch = _torch()
    _here(items.home, "items", _current_device())
    a = pa_adamw_args(float(lr), float(beta1), float(beta2), float(eps), int(step),
                      int(seed) & 0xFFFFFFFFFFFFFFFF,
                      _in(gscale, 1, torch.float32, "gscale", False),
                      _in(lr_dev, 1, torch.float32, "lr_dev", False),
                      _in(step_dev, 1, torch.int64, "step_dev", False))
    handle = B._stream(stream)
    capturing = bool(handle) and _capturing(stream)  # (the default stream never is)
    items.hold(stream, handle, capturing, (gscale, lr_dev, step_dev))
    if items.dev is not None:
        _check(load().pa_adamw_run(items.n, items.blocks, items.on(stream, handle, capturing),
                                   ctypes.byref(a), handle))
    else:
        _check(load().pa_adamw(items.n, items.arr, ctypes.byref(a), handle))


def pa_adamw_unpack(codes, scales, out, signed, stream=None):
    """The values of 8-bit moments (signed: m's codes) as fp32."""
    torch = _torch()
    n = codes.numel()
    _check(load().pa_adamw_unpack(
        n, _in(codes, n, torch.uint8, "codes"), _in(scales, -(-n // BLOCK), torch.float32, "scales"),
        int(bool(signed)), _in(out, n, torch.float32, "out"), B._stream(stream)))


def version(t):
    """How often torch has written a tensor (this library's calls do not count)."""
    return None if t.is_inference() else t._version


class AdamW:
    """AdamW over named fp32 tensors, e.g. a block stack's parameters: the
    moments (fp32, or 8 bits where a tensor has at least ``small`` elements)
    and one pa_adamw call per step.

    params: {name: fp32 tensor}; copies: {name: bf16 tensor} that receive the
    parameters rounded (what the stack's products read); decay: names with
    weight decay (default: tensors of more than one dimension); where: {name:
    (dict, key)}, the places that the program reads a parameter, or its copy, from;
    after: called after every step.

    A step refuses what would be lost in it: a copy that torch has written since the
    last one (``refresh`` takes the parameter from it), and another tensor in a
    place of ``where``."""

    def __init__(self, params, lr, betas=(0.9, 0.999), eps=1e-8, wd=0.01, bits=32, copies=None,
                 decay=None, small=4096, seed=0, where=None, after=None):
        torch = _torch()
        if bits not in (8, 32):
            raise ValueError("bits must be 8 or 32")
        self.lr, self.betas, self.eps, self.seed, self.t = lr, betas, eps, seed, 0
        self.names = list(params)
        copies, where = dict(copies or {}), where or {}
        unknown = [k for k in [*copies, *(decay or ()), *where] if k not in params]
        if unknown:
            raise ValueError(f"not among the parameters: {unknown}")
        items = []
        for k, p in params.items():
            d = {"p": p, "copy": copies.get(k)}
            d["wd"] = wd if (k in decay if decay is not None else p.dim() > 1) else 0.0
            if bits == 8 and p.numel() >= small:
                nb = -(-p.numel() // BLOCK)
                for s in "mv":
                    d[s] = torch.zeros(p.numel(), dtype=torch.uint8, device=p.device)
                    d[s + "_scale"] = torch.zeros(nb, dtype=torch.float32, device=p.device)
            else:
                d["m"], d["v"] = torch.zeros_like(p), torch.zeros_like(p)
            items.append(d)
        self.items = make_adamw_items(items)
        self.copies, self.after = copies, after
        self.versions = {k: version(c) for k, c in copies.items()}
        self.where = [(k, *at, copies.get(k, params[k])) for k, at in where.items()]

    def refresh(self):
        """The parameters from their copies, after the program has written those (a
        checkpoint's weights, say); the moments stay."""
        for k, c in self.copies.items():
            self.items.tensors[self.names.index(k)]["p"].copy_(c)
            self.versions[k] = version(c)

    def state(self):
        """What the next steps depend on beside the parameters that the program holds
        itself, in new tensors: the count of the steps, the seed, the moments as they
        are kept (codes and scales of 8 bits) and the parameters that have copies."""
        return {"t": self.t, "seed": self.seed,
                "tensors": {k: {s: t.detach().clone() for s, t in d.items()}
                            for k, d in self._kept().items()}}

    def _kept(self):
        return {k: {s: d[s] for s in ("p", "m", "v", "m_scale", "v_scale")
                    if d.get(s) is not None and (s != "p" or k in self.copies)}
                for k, d in zip(self.names, self.items.tensors)}

    def load_state(self, state):
        """``state`` of an optimizer over the same names and sizes, with moments of
        the same bits, put into this one's tensors (also where graphs read them);
        copies are rounded from their parameters."""
        mine, tensors = self._kept(), state["tensors"]
        if set(tensors) != set(mine):
            raise ValueError(f"names that differ: {sorted(set(tensors) ^ set(mine))}")
        for k, d in mine.items():
            if set(d) != set(tensors[k]):
                raise ValueError(f"{k}: has {sorted(d)}, the state {sorted(tensors[k])}")
            for s, t in d.items():
                o = tensors[k][s]
                if o.shape != t.shape or o.dtype != t.dtype:
                    raise ValueError(f"{k}: {s} is {list(t.shape)} {t.dtype}, the state's "
                                     f"{list(o.shape)} {o.dtype}")
        for k, d in mine.items():
            for s, t in d.items():
                t.copy_(tensors[k][s])
            if k in self.copies:
                self.copies[k].copy_(d["p"])
                self.versions[k] = version(self.copies[k])
        self.t, self.seed = int(state["t"]), int(state["seed"])

    def _unchanged(self):
        for k, d, key, t in self.where:
            if d.get(key) is not t:
                raise ValueError(f"{k}: another tensor has taken its place, and this optimizer "
                                 "holds the one before; it needs an optimizer of its own")
        for k, c in self.copies.items():
            if version(c) != self.versions[k]:
                raise ValueError(f"{k}: its copy was written since the last step, which this one "
                                 "would undo; refresh() takes the parameter from it")

    def step(self, grads, gscale=None, lr=None, stream=None, lr_dev=None, step_dev=None):
        """grads: {name: tensor} for every parameter (fp32 or bf16).  A step that
        is captured into a graph needs its number on the device, step_dev (int64,
        from 1, advanced by the graph or between its replays), since a number from
        here would stand still, and its learning rate there, lr_dev (fp32), where
        that changes; the count of the calls goes on without such steps."""
        capturing = _capturing(stream)
        if step_dev is None and capturing:
            raise ValueError("a step captured into a graph needs step_dev")
        self._unchanged()
        it = self.items
        before = it.moved
        it.set_grads([grads[k] for k in self.names])
        if it.dev is None and it.moved == before and not capturing:
            it.table()  # the gradients stay where they are
        pa_adamw(self.items, self.lr if lr is None else lr, self.t + 1, *self.betas, self.eps,
                 self.seed, gscale, lr_dev, step_dev, stream)
        if step_dev is None:
            self.t += 1
        if self.after is not None:
            self.after()

    def moments(self, name):
        """(m, v) of a parameter as fp32 tensors."""
        torch = _torch()
        d = self.items.tensors[self.names.index(name)]
        if d.get("m_scale") is None:
            return d["m"].clone(), d["v"].clone()
        out = []
        for s in "mv":
            o = torch.empty(d["p"].shape, dtype=torch.float32, device=d["p"].device)
            pa_adamw_unpack(d[s], d[s + "_scale"], o, signed=s == "m")
            out.append(o)
        return tuple(out)


# ---- 8-bit integer products ----
def pa_quant_rows(x, q, s, stream=None):
    """x [N, K] to int8 rows q [N, padded(K)] with scales s [N]."""
    torch = _torch()
    N, K = x.shape
    _check(load().pa_quant_rows(N, K, _code(x.dtype, "x"), _dev(x, "x"),
                                _in(q, N * padded(K), torch.int8, "q"),
                                _in(s, N, torch.float32, "s"), B._stream(stream)))


def pa_quant_weight(W, Wq, sw, stream=None):
    """W [K, F] to Wq [F, padded(K)] int8 with a scale per output channel."""
    torch = _torch()
    K, F = W.shape
    _check(load().pa_quant_weight(K, F, _code(W.dtype, "W"), _dev(W, "W"),
                                  _in(Wq, F * padded(K), torch.int8, "Wq"),
                                  _in(sw, F, torch.float32, "sw"), B._stream(stream)))


def empty_weight(W):
    """(Wq, sw): tensors for the integers and scales of a weight [K, F]."""
    torch = _torch()
    K, F = W.shape
    return (torch.empty(F, padded(K), dtype=torch.int8, device=W.device),
            torch.empty(F, dtype=torch.float32, device=W.device))


def quant_weight(W):
    """(Wq, sw) of a weight [K, F], in new tensors."""
    Wq, sw = empty_weight(W)
    pa_quant_weight(W, Wq, sw)
    return Wq, sw


def _product(K, wq, sw, D, bias, act, C):
    torch = _torch_module or _torch()
    if D.dim() != 2:
        raise ValueError("D must be [N, F]")
    a = ACTS.get(act)
    if a is None:
        raise ValueError(f"act: {act!r} is not one of {sorted(map(str, ACTS))}")
    N, F = D.shape
    f32, cur, dt = torch.float32, _current_device(), D.dtype
    return (N, F, cur, (_in(wq, F * ((K + 15) // 16 * 16), torch.int8, "Wq", True, cur),
                        _in(sw, F, f32, "sw", True, cur),
                        None if bias is None else _in(bias, F, f32, "bias", True, cur), a,
                        None if C is None else _in(C, N * F, dt, "C", True, cur),
                        _dev(D, "D", cur), _code(dt, "D")))


def pa_gemm_i8(q, s, wq, sw, D, K=None, bias=None, act=None, C=None, stream=None):
    """D = act(s sw (q wq^T) + bias) + C from int8 rows q [N, padded(K)] (K:
    q's width when not given) and weights wq [F, padded(K)]."""
    torch = _torch()
    K = q.shape[1] if K is None else K
    N, F, cur, rest = _product(K, wq, sw, D, bias, act, C)
    _check(load().pa_gemm_i8(N, F, K, _in(q, N * padded(K), torch.int8, "q", True, cur),
                             _in(s, N, torch.float32, "s", True, cur), *rest, B._stream(stream)))


def linear_i8_workspace(N, K, F, device="cuda"):
    """A uint8 workspace for pa_linear_i8 at these sizes."""
    k = ctypes.c_size_t(0)
    _check(load().pa_linear_i8_workspace(N, F, K, ctypes.byref(k)))
    return _torch().empty(k.value, dtype=_torch().uint8, device=device)


def pa_linear_i8(x, wq, sw, D, ws, bias=None, act=None, C=None, stream=None):
    """D [N, F] = act(x W + bias) + C with x [N, K] quantised row by row and W
    as pa_quant_weight left it."""
    N, K = x.shape
    Nd, F, cur, rest = _product(K, wq, sw, D, bias, act, C)
    if Nd != N:
        raise ValueError(f"D has {Nd} rows, x {N}")
    _check(load().pa_linear_i8(N, F, K, _dev(x, "x", cur), _code(x.dtype, "x"), *rest,
                               None if ws is None else _dev(ws, "ws", cur), B._nbytes(ws),
                               B._stream(stream)))
