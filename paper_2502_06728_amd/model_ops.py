"""ctypes binding of include/detonation_model.h: the operators that a training step needs around its
library products, next to the optimizer step of binding.py (same library).

Argument checks and marshalling only: device tensors in, raw pointers out; every tensor is given by the
caller, outputs too, and is written by the kernels on `stream` (the current stream if it is None).
Matrices are 2-D tensors whose rows may lie any distance apart; their elements are consecutive.  Written
matrices, 8-bit forms and workspaces that share memory with each other or with an input are refused, except
where an operator works in place.  There is no CPU fallback.  Calls hand their arguments to csrc_model/marshal.c first, which checks and converts
what a program usually passes; what it does not take goes through the checks below, which name what is
wrong, and so does every call where it cannot be used.
"""
from __future__ import annotations

import ctypes
import os
import sysconfig
from dataclasses import dataclass

from . import binding
from .binding import BF16, F16, F32, DetonationError, _handle

NORM_NONE, NORM_RMS, NORM_LAYER = 0, 1, 2
ACT_SILU, ACT_GELU, ACT_GELU_TANH, ACT_RELU = 0, 1, 2, 3
ACT8_GROUP = 32
MAX_TOP = 32
MAX_NORM_WIDTH = 16384

MARSHAL_PATH = os.path.join(os.path.dirname(os.path.abspath(__file__)),
                            "_model_marshal" + (sysconfig.get_config_var("EXT_SUFFIX") or ".so"))

EXPORTS = ("detonation_token_logprobs", "detonation_token_logprobs_backward",
           "detonation_token_logprobs_workspace", "detonation_norm_residual",
           "detonation_norm_residual_backward", "detonation_norm_residual_workspace",
           "detonation_act8_encode", "detonation_act8_decode", "detonation_glu_forward",
           "detonation_glu_backward", "detonation_act8_weight_grad",
           "detonation_act8_weight_grad_workspace")


class deto_rows(ctypes.Structure):
    _fields_ = [("data", ctypes.c_void_p), ("ld", ctypes.c_int64), ("dtype", ctypes.c_int32),
                ("reserved", ctypes.c_int32)]


class deto_act8(ctypes.Structure):
    _fields_ = [("codes", ctypes.c_void_p), ("ld_codes", ctypes.c_int64),
                ("exps", ctypes.c_void_p), ("ld_exps", ctypes.c_int64)]


class deto_norm_residual(ctypes.Structure):
    _fields_ = [("pre", ctypes.c_int32), ("post", ctypes.c_int32), ("eps_pre", ctypes.c_float),
                ("eps_post", ctypes.c_float), ("scale", ctypes.c_float),
                ("param_dtype", ctypes.c_int32), ("rows_per_gate", ctypes.c_int64),
                ("w_pre", ctypes.c_void_p), ("b_pre", ctypes.c_void_p),
                ("w_post", ctypes.c_void_p), ("b_post", ctypes.c_void_p),
                ("gate", ctypes.c_void_p), ("ld_gate", ctypes.c_int64)]


class deto_norm_grads(ctypes.Structure):
    _fields_ = [(n, ctypes.c_void_p) for n in ("w_pre", "b_pre", "w_post", "b_post", "gate")]


@dataclass
class NormResidual:
    """x_out = x + scale * gate (.) post(f);  y = pre(x_out)."""
    pre: int = NORM_RMS
    post: int = NORM_NONE
    eps_pre: float = 1e-6
    eps_post: float = 1e-6
    scale: float = 1.0
    rows_per_gate: int = 0


@dataclass
class Act8:
    """A [T, D] matrix in 8 bits: int8 codes [T, D] and uint8 exponents [T, ceil(D / 32)]."""
    codes: object
    exps: object

    @staticmethod
    def empty(T: int, D: int, device="cuda") -> "Act8":
        import torch
        return Act8(torch.empty((T, D), dtype=torch.int8, device=device),
                    torch.empty((T, -(-D // ACT8_GROUP)), dtype=torch.uint8, device=device))


_lib = None
_codes = None          # torch's types by the library's


def _load():
    global _lib, _codes
    if _lib is None:
        import torch
        lib = binding.load()
        vp, i64, i32, f32 = ctypes.c_void_p, ctypes.c_int64, ctypes.c_int32, ctypes.c_float
        rows, act8 = ctypes.POINTER(deto_rows), ctypes.POINTER(deto_act8)
        norm, grads = ctypes.POINTER(deto_norm_residual), ctypes.POINTER(deto_norm_grads)
        for name, args in {
            "token_logprobs": [i64, i64, rows, f32, vp, i32, vp, vp, vp, i32, vp, vp, vp, vp, vp],
            "token_logprobs_backward": [i64, i64, rows, f32, vp, i32, vp, vp, vp, vp, rows, vp],
            "norm_residual": [norm, i64, i64, rows, rows, rows, rows, act8, vp],
            "norm_residual_backward": [norm, i64, i64, rows, rows, rows, rows, rows, rows, grads, vp,
                                       vp],
            "act8_encode": [i64, i64, rows, act8, vp],
            "act8_decode": [i64, i64, act8, rows, vp],
            "glu_forward": [i32, i64, i64, rows, rows, rows, act8, act8, vp],
            "glu_backward": [i32, i64, i64, rows, act8, act8, rows, rows, act8, vp],
            "act8_weight_grad": [i64, i64, i64, rows, act8, rows, i32, vp, vp],
        }.items():
            f = getattr(lib, "detonation_" + name)
            f.argtypes, f.restype = args, i32
        for name, args in {"token_logprobs": [i64, i64, i32], "norm_residual": [norm, i64, i64],
                           "act8_weight_grad": [i64, i64, i64]}.items():
            f = getattr(lib, f"detonation_{name}_workspace")
            f.argtypes, f.restype = args, i64
        _codes = {torch.float32: F32, torch.bfloat16: BF16, torch.float16: F16}
        _lib = lib
    return _lib


class _NoMarshal:
    """Leaves every call to the checks of this module."""

    @staticmethod
    def logprobs(*args) -> int:
        return -1

    logprobs_backward = norm = norm_backward = encode = decode = logprobs
    glu_forward = glu_backward = weight_grad = logprobs


_marshal = None        # csrc_model/marshal.c, or _NoMarshal; set by the first call


def _marshalling():
    global _marshal
    lib = _load()
    if _marshal is None:
        try:
            _marshal = _load_marshal(lib)
        except (ImportError, OSError, AttributeError):
            _marshal = _NoMarshal
    return _marshal


# in the order of csrc_model/marshal.c
_MARSHALLED = ("token_logprobs", "token_logprobs_backward", "token_logprobs_workspace", "norm_residual",
               "norm_residual_backward", "norm_residual_workspace", "act8_encode", "act8_decode",
               "glu_forward", "glu_backward", "act8_weight_grad", "act8_weight_grad_workspace")


def _marshal_types():
    import torch
    return (torch.float32, torch.bfloat16, torch.float16, torch.int32, torch.int64, torch.int8, torch.uint8)


def _load_marshal(lib):
    import importlib.machinery
    import importlib.util

    import torch
    loader = importlib.machinery.ExtensionFileLoader("_model_marshal", MARSHAL_PATH)
    spec = importlib.util.spec_from_file_location("_model_marshal", MARSHAL_PATH, loader=loader)
    m = importlib.util.module_from_spec(spec)
    loader.exec_module(m)
    m.setup(tuple(ctypes.cast(getattr(lib, "detonation_" + n), ctypes.c_void_p).value for n in _MARSHALLED),
            _marshal_types(), torch._C._cuda_getDevice, torch._C._cuda_getCurrentRawStream,
            torch.cuda.device_count())
    return m


def _taken(rc: int) -> bool:
    """Whether the marshalled call ran; it raises for one that the HIP runtime refused."""
    if rc > 0:
        raise DetonationError(rc)
    return rc == 0


def _status(rc: int) -> None:
    if rc != 0:
        raise DetonationError(rc)


# ------------------------------------------------------------------ checks
# A wrong type, shape or device would become an access out of bounds: refused here, on the host.

class _Call:
    """The tensors of one call: all on one device, which is the current one."""

    __slots__ = ("device",)

    def __init__(self):
        self.device = None

    def on_device(self, t, name):
        if not t.is_cuda:
            raise ValueError(f"{name} must be a device tensor")
        d = t.device
        if self.device is None:
            import torch
            if d.index != torch.cuda.current_device():
                raise ValueError(f"{name} is not on the current device")
            self.device = d
        elif d != self.device:
            raise ValueError(f"{name} is on another device than the other tensors")

    def rows(self, t, name, T, D, dtype=None):
        """A deto_rows of a [T, D] tensor (None stays None: absent)."""
        if t is None:
            return None
        _load()
        if t.dtype not in _codes or (dtype is not None and t.dtype != dtype):
            raise ValueError(f"{name}: dtype {t.dtype}, expected "
                             f"{dtype if dtype is not None else [str(d) for d in _codes]}")
        self._shape(t, name, T, D)
        return deto_rows(t.data_ptr(), self._ld(t, name, T, D), _codes[t.dtype], 0)

    def act8(self, m, name, T, D):
        if m is None:
            return None
        import torch
        G = -(-D // ACT8_GROUP)
        if m.codes.dtype != torch.int8 or m.exps.dtype != torch.uint8:
            raise ValueError(f"{name}: codes are int8 and exponents uint8")
        self._shape(m.codes, name + ".codes", T, D)
        self._shape(m.exps, name + ".exps", T, G)
        return deto_act8(m.codes.data_ptr(), self._ld(m.codes, name + ".codes", T, D),
                         m.exps.data_ptr(), self._ld(m.exps, name + ".exps", T, G))

    def _shape(self, t, name, T, D):
        self.on_device(t, name)
        if t.dim() != 2 or t.shape[0] != T or t.shape[1] != D:
            raise ValueError(f"{name}: shape {tuple(t.shape)}, expected ({T}, {D})")

    @staticmethod
    def _ld(t, name, T, D):
        ld, step = t.stride()
        if (D > 1 and step != 1) or (T > 1 and ld < D):
            raise ValueError(f"{name}: rows of consecutive elements, not overlapping, are needed")
        return ld if T > 1 else max(D, 1)

    def vector(self, t, name, numel, dtypes, optional=True):
        """The address of a contiguous tensor (None: 0)."""
        if t is None:
            if not optional:
                raise ValueError(f"{name} is required")
            return None
        self.on_device(t, name)
        if t.dtype not in dtypes:
            raise ValueError(f"{name}: dtype {t.dtype}, expected one of {[str(d) for d in dtypes]}")
        if not t.is_contiguous() or t.numel() != numel:
            raise ValueError(f"{name}: {numel} consecutive elements are needed")
        return t.data_ptr()

    def scratch(self, t, nbytes):
        if nbytes <= 0:
            return None
        if t is None:
            raise ValueError(f"a workspace of {nbytes} bytes is needed")
        self.on_device(t, "workspace")
        if not t.is_contiguous() or t.numel() * t.element_size() < nbytes:
            raise ValueError(f"the workspace is shorter than {nbytes} bytes")
        return t.data_ptr()


def _stream(stream):
    return binding._stream(stream)


def _by_ref(s):
    return None if s is None else ctypes.byref(s)


def _apart(out, *others):
    """An output is not the memory of something else, except where an operator says so: the same rows."""
    for name, t in others:
        if t is None or out is None:
            continue
        if out.data_ptr() == t.data_ptr() and out.dtype == t.dtype and out.stride() == t.stride():
            continue
        if _meet(_span(out), _span(t)):
            raise ValueError(f"an output overlaps {name} without being the same rows")


def _disjoint(outs: dict, ins: dict, same=()) -> None:
    """Outputs (matrices, Act8 and the workspace, a (tensor, bytes)) share no memory with each other, nor with
    the inputs; the pairs of names in `same` may be the same rows."""
    outs, ins = _matrices(outs), _matrices(ins)
    for i, (name, t, span) in enumerate(outs):
        for other, u, span_u in outs[i + 1:] + ins:
            if (name, other) in same:
                _apart(t, (other, u))
            elif _meet(span, span_u):
                raise ValueError(f"{name} overlaps {other}")


def _matrices(tensors: dict) -> list:
    out = []
    for name, t in tensors.items():
        if isinstance(t, tuple):
            t, nbytes = t
            if t is not None and nbytes > 0:
                out.append((name, t, (t.data_ptr(), 1, 0, nbytes)))
        elif hasattr(t, "codes"):
            out += [(name + ".codes", t.codes, _span(t.codes)), (name + ".exps", t.exps, _span(t.exps))]
        elif t is not None and t.dim() == 2:
            out.append((name, t, _span(t)))
        elif t is not None:
            out.append((name, t, (t.data_ptr(), 1, 0, t.numel() * t.element_size())))
    return out


def _span(t):
    """Rows of memory: address, number, distance and width in bytes."""
    e = t.element_size()
    return t.data_ptr(), t.shape[0], t.stride(0) * e, t.shape[1] * e


def _meet(a, b) -> bool:
    """Whether two of them share memory (columns of one matrix lie side by side; rows a different step
    apart are taken to meet where the memory from the first one to the last does)."""
    (at, rows, step, wide), (at_b, rows_b, step_b, wide_b) = a, b
    if not rows or not rows_b:
        return False
    if at + (rows - 1) * step + wide <= at_b or at_b + (rows_b - 1) * step_b + wide_b <= at:
        return False
    if (rows == 1 and rows_b == 1) or (rows > 1 and rows_b > 1 and step != step_b):
        return True
    d = (at_b - at) % (step if rows > 1 else step_b)
    return d < wide or d + wide_b > (step if rows > 1 else step_b)


# ------------------------------------------------------------------ log probabilities

def token_logprobs_workspace(T: int, V: int, top: int = 0) -> int:
    """Bytes of scratch for detonation_token_logprobs."""
    return _size(_load().detonation_token_logprobs_workspace(T, V, top))


def _size(n: int) -> int:
    if n < 0:
        raise ValueError("sizes that the operator does not take")
    return int(n)


def detonation_token_logprobs(logits, targets, logp, *, lse=None, entropy=None, top_idx=None,
                              top_logp=None, stats=None, logit_scale: float = 1.0, workspace=None,
                              stream=None) -> None:
    """Per row of logits [T, V]: the log probability of targets[t] (int32 or int64; 0 where that is
    outside [0, V)), and where tensors are given for them log sum exp, the entropy, the best tokens
    (top_idx int32 and top_logp float32, both [T, K]), and the [T, 2] `stats` of the backward pass."""
    if _taken((_marshal or _marshalling()).logprobs(logits, targets, logp, lse, entropy, top_idx, top_logp,
                                                    stats, logit_scale, workspace, _handle(stream))):
        return
    import torch
    lib, c = _load(), _Call()
    T, V = logits.shape
    x = c.rows(logits, "logits", T, V)
    f32 = (torch.float32,)
    y = c.vector(targets, "targets", T, (torch.int64, torch.int32), optional=False)
    top = 0
    if top_idx is not None:
        if top_idx.dim() != 2:
            raise ValueError("top_idx is [T, K]")
        top = top_idx.shape[1]
    elif top_logp is not None:
        raise ValueError("top_logp needs top_idx")
    args = (c.vector(logp, "logp", T, f32, optional=False), c.vector(lse, "lse", T, f32),
            c.vector(entropy, "entropy", T, f32), top,
            c.vector(top_idx, "top_idx", T * top, (torch.int32,)),
            c.vector(top_logp, "top_logp", T * top, f32),
            c.vector(stats, "stats", 2 * T, f32))
    need = lib.detonation_token_logprobs_workspace(T, V, top)
    ws = c.scratch(workspace, need)
    _disjoint({"workspace": (workspace, need)}, {"logits": logits})
    _status(lib.detonation_token_logprobs(T, V, ctypes.byref(x), logit_scale, y,
                                          targets.element_size(), *args, ws, _stream(stream)))


def detonation_token_logprobs_backward(logits, targets, stats, dlogits, *, g_logp=None, entropy=None,
                                       g_entropy=None, logit_scale: float = 1.0,
                                       stream=None) -> None:
    """dlogits [T, V] (may be the logits themselves): the gradient of sum(g_logp * logp) +
    sum(g_entropy * entropy); stats and entropy as detonation_token_logprobs wrote them."""
    if _taken((_marshal or _marshalling()).logprobs_backward(logits, targets, stats, dlogits, g_logp, entropy,
                                                             g_entropy, logit_scale, _handle(stream))):
        return
    import torch
    lib, c = _load(), _Call()
    T, V = logits.shape
    x = c.rows(logits, "logits", T, V)
    dx = c.rows(dlogits, "dlogits", T, V, logits.dtype)
    _disjoint({"dlogits": dlogits}, {"logits": logits}, same=(("dlogits", "logits"),))
    f32 = (torch.float32,)
    if g_logp is None and g_entropy is None:
        raise ValueError("g_logp or g_entropy is required")
    _status(lib.detonation_token_logprobs_backward(
        T, V, ctypes.byref(x), logit_scale,
        c.vector(targets, "targets", T, (torch.int64, torch.int32), optional=False),
        targets.element_size(), c.vector(stats, "stats", 2 * T, f32, optional=False),
        c.vector(entropy, "entropy", T, f32, optional=g_entropy is None),
        c.vector(g_logp, "g_logp", T, f32), c.vector(g_entropy, "g_entropy", T, f32),
        ctypes.byref(dx), _stream(stream)))


# ------------------------------------------------------------------ norm, gate, residual

def _norm_struct(c, cfg, T, D, gate, w_post, b_post, w_pre, b_pre):
    _load()
    s = deto_norm_residual(cfg.pre, cfg.post, cfg.eps_pre, cfg.eps_post, cfg.scale, F32,
                           cfg.rows_per_gate)
    dtype = None
    for name, t in (("w_pre", w_pre), ("b_pre", b_pre), ("w_post", w_post), ("b_post", b_post)):
        if t is not None:
            dtype = t.dtype if dtype is None else dtype
            setattr(s, name, c.vector(t, name, D, (dtype,)))
    if gate is not None:
        dtype = gate.dtype if dtype is None else dtype
        rows = gate_rows(cfg, T)
        if gate.dim() == 1 and rows == 1:
            gate = gate[None]
        g = c.rows(gate, "gate", rows, D, dtype)
        s.gate, s.ld_gate = g.data, g.ld
    if dtype is not None:
        if dtype not in _codes:
            raise ValueError(f"weights of dtype {dtype}")
        s.param_dtype = _codes[dtype]
    return s


def gate_rows(cfg: NormResidual, T: int) -> int:
    """Rows of the gate for T rows of the matrices."""
    return -(-T // cfg.rows_per_gate) if cfg.rows_per_gate > 0 else 1


def norm_residual_workspace(cfg: NormResidual, T: int, D: int) -> int:
    """Bytes of scratch for detonation_norm_residual_backward."""
    s = deto_norm_residual(cfg.pre, cfg.post, cfg.eps_pre, cfg.eps_post, cfg.scale, F32,
                           cfg.rows_per_gate)
    return _size(_load().detonation_norm_residual_workspace(ctypes.byref(s), T, D))


def detonation_norm_residual(cfg: NormResidual, x, f, x_out, y, *, y8: Act8 | None = None, gate=None,
                             w_post=None, b_post=None, w_pre=None, b_pre=None, stream=None) -> None:
    """x_out = x + scale * gate (.) post(f), y = pre(x_out), y8 = y in 8 bits; x_out may be x.  f and
    x_out are None for a norm alone, y (and y8) under cfg.pre = NORM_NONE.  gate: [D], or a row for
    every cfg.rows_per_gate rows.  Weights, biases and gate are of one type."""
    if _taken((_marshal or _marshalling()).norm(cfg, x, f, x_out, y, y8, gate, w_post, b_post, w_pre, b_pre,
                                                _handle(stream))):
        return
    lib, c = _load(), _Call()
    T, D = x.shape
    s = _norm_struct(c, cfg, T, D, gate, w_post, b_post, w_pre, b_pre)
    xs, fs = c.rows(x, "x", T, D), c.rows(f, "f", T, D)
    xo = c.rows(x_out, "x_out", T, D, x.dtype)
    ys = c.rows(y, "y", T, D, None if f is None else f.dtype)
    q = c.act8(y8, "y8", T, D)
    _disjoint({"x_out": x_out, "y": y, "y8": y8},
              {"x": x, "f": f, "gate": gate, "w_post": w_post, "b_post": b_post, "w_pre": w_pre, "b_pre": b_pre},
              same=(("x_out", "x"),))
    _status(lib.detonation_norm_residual(ctypes.byref(s), T, D, ctypes.byref(xs), _by_ref(fs),
                                         _by_ref(xo), _by_ref(ys), _by_ref(q), _stream(stream)))


def detonation_norm_residual_backward(cfg: NormResidual, x_out, f, dy, dx_out, dx, df, *,
                                      workspace=None, gate=None, w_post=None, b_post=None,
                                      w_pre=None, dgate=None, dw_post=None, db_post=None, dw_pre=None,
                                      db_pre=None, stream=None) -> None:
    """Gradients of detonation_norm_residual, given those of y (dy; None under NORM_NONE) and of x_out
    (dx_out; None: zeros): dx (may be dx_out), df, and the sums over rows that float32 tensors are
    given for."""
    if _taken((_marshal or _marshalling()).norm_backward(
            cfg, x_out, f, dy, dx_out, dx, df, workspace, gate, w_post, b_post, w_pre, dgate, dw_post,
            db_post, dw_pre, db_pre, _handle(stream))):
        return
    import torch
    lib, c = _load(), _Call()
    T, D = x_out.shape
    s = _norm_struct(c, cfg, T, D, gate, w_post, b_post, w_pre, None)
    xs, fs = c.rows(x_out, "x_out", T, D), c.rows(f, "f", T, D)
    dys = c.rows(dy, "dy", T, D, None if f is None else f.dtype)
    dxo = c.rows(dx_out, "dx_out", T, D, x_out.dtype)
    dxs = c.rows(dx, "dx", T, D, x_out.dtype)
    dfs = c.rows(df, "df", T, D, None if f is None else f.dtype)
    f32 = (torch.float32,)
    g = deto_norm_grads(*(c.vector(t, n, m, f32) for n, t, m in (
        ("dw_pre", dw_pre, D), ("db_pre", db_pre, D), ("dw_post", dw_post, D),
        ("db_post", db_post, D), ("dgate", dgate, gate_rows(cfg, T) * D))))
    need = lib.detonation_norm_residual_workspace(ctypes.byref(s), T, D)
    need = need if any((dw_pre is not None, db_pre is not None, dgate is not None, dw_post is not None,
                        db_post is not None)) else 0
    ws = c.scratch(workspace, need)
    _disjoint({"workspace": (workspace, need), "dx": dx, "df": df},
              {"x_out": x_out, "f": f, "dy": dy, "dx_out": dx_out, "gate": gate, "w_post": w_post,
               "b_post": b_post, "w_pre": w_pre}, same=(("dx", "dx_out"),))
    _status(lib.detonation_norm_residual_backward(
        ctypes.byref(s), T, D, ctypes.byref(xs), _by_ref(fs), _by_ref(dys), _by_ref(dxo),
        _by_ref(dxs), _by_ref(dfs), ctypes.byref(g), ws, _stream(stream)))


# ------------------------------------------------------------------ activations in 8 bits

def detonation_act8_encode(x, x8: Act8, stream=None) -> None:
    """x [T, D] into 8 bits."""
    if _taken((_marshal or _marshalling()).encode(x, x8, _handle(stream))):
        return
    lib, c = _load(), _Call()
    T, D = x.shape
    xs, q = c.rows(x, "x", T, D), c.act8(x8, "x8", T, D)
    _disjoint({"x8": x8}, {"x": x})
    _status(lib.detonation_act8_encode(T, D, ctypes.byref(xs), ctypes.byref(q), _stream(stream)))


def detonation_act8_decode(x8: Act8, x, stream=None) -> None:
    """The values of x8, rounded to x's type."""
    if _taken((_marshal or _marshalling()).decode(x8, x, _handle(stream))):
        return
    lib, c = _load(), _Call()
    T, D = x.shape
    xs, q = c.rows(x, "x", T, D), c.act8(x8, "x8", T, D)
    _disjoint({"x": x}, {"x8": x8})
    _status(lib.detonation_act8_decode(T, D, ctypes.byref(q), ctypes.byref(xs), _stream(stream)))


def detonation_glu_forward(act: int, a, b, h, *, a8: Act8 | None = None, b8: Act8 | None = None,
                           stream=None) -> None:
    """h = act(a) (.) b (b None: act(a)), with a and b left in 8 bits for the backward pass; h may be a
    or b."""
    if _taken((_marshal or _marshalling()).glu_forward(act, a, b, h, a8, b8, _handle(stream))):
        return
    lib, c = _load(), _Call()
    T, D = a.shape
    sa, sb = c.rows(a, "a", T, D), c.rows(b, "b", T, D, a.dtype)
    sh = c.rows(h, "h", T, D, a.dtype)
    qa, qb = c.act8(a8, "a8", T, D), c.act8(b8, "b8", T, D)
    _disjoint({"h": h, "a8": a8, "b8": b8}, {"a": a, "b": b}, same=(("h", "a"), ("h", "b")))
    _status(lib.detonation_glu_forward(act, T, D, ctypes.byref(sa), _by_ref(sb), ctypes.byref(sh),
                                       _by_ref(qa), _by_ref(qb), _stream(stream)))


def detonation_glu_backward(act: int, dh, a8: Act8, b8: Act8 | None, da, db=None, *,
                            h8: Act8 | None = None, stream=None) -> None:
    """da and db (None without b8) from dh and the saved a and b; h8 receives act(a) (.) b of the saved
    values.  da or db may be dh."""
    if _taken((_marshal or _marshalling()).glu_backward(act, dh, a8, b8, da, db, h8, _handle(stream))):
        return
    lib, c = _load(), _Call()
    T, D = dh.shape
    sd, sa = c.rows(dh, "dh", T, D), c.rows(da, "da", T, D, dh.dtype)
    sb = c.rows(db, "db", T, D, dh.dtype)
    qa, qb, qh = c.act8(a8, "a8", T, D), c.act8(b8, "b8", T, D), c.act8(h8, "h8", T, D)
    _disjoint({"da": da, "db": db, "h8": h8}, {"dh": dh, "a8": a8, "b8": b8},
              same=(("da", "dh"), ("db", "dh")))
    _status(lib.detonation_glu_backward(act, T, D, ctypes.byref(sd), _by_ref(qa), _by_ref(qb),
                                        ctypes.byref(sa), _by_ref(sb), _by_ref(qh),
                                        _stream(stream)))


def act8_weight_grad_workspace(T: int, N: int, K: int) -> int:
    """Bytes of scratch for detonation_act8_weight_grad."""
    return _size(_load().detonation_act8_weight_grad_workspace(T, N, K))


def detonation_act8_weight_grad(dy, x8: Act8, dw, *, accumulate: bool = False, workspace=None,
                                stream=None) -> None:
    """dw [N, K] = [dw +] dy^T x with dy [T, N] and x [T, K] in 8 bits."""
    if _taken((_marshal or _marshalling()).weight_grad(dy, x8, dw, accumulate, workspace, _handle(stream))):
        return
    lib, c = _load(), _Call()
    T, N = dy.shape
    K = dw.shape[1]
    sy, q = c.rows(dy, "dy", T, N), c.act8(x8, "x8", T, K)
    sw = c.rows(dw, "dw", N, K)
    need = lib.detonation_act8_weight_grad_workspace(T, N, K)
    ws = c.scratch(workspace, need)
    _disjoint({"dw": dw, "workspace": (workspace, need)}, {"dy": dy, "x8": x8})
    _status(lib.detonation_act8_weight_grad(T, N, K, ctypes.byref(sy), ctypes.byref(q),
                                            ctypes.byref(sw), int(accumulate), ws,
                                            _stream(stream)))
