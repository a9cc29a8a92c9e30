"""The native argument marshalling of model_ops.py (csrc_model/marshal.c) without a GPU: what it hands to the
library for ordinary calls, and that it leaves everything else to the checks in Python."""
import ctypes

import pytest
import torch

from paper_2502_06728_amd import model_ops as ops

vp, i32, i64, f32 = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_float
T, D = 5, 70


class OnDevice:
    """A tensor that says it is on device `at`."""
    is_cuda = True

    def __init__(self, t, at=3):
        self.t, self.dtype, self.shape, self.at = t, t.dtype, t.shape, at

    def __getattr__(self, name):
        return getattr(self.t, name)

    def get_device(self):
        return self.at


def mat(rows, cols, dtype=torch.float32, pad=0, at=3):
    return OnDevice(torch.zeros((rows, cols + pad), dtype=dtype)[:, :cols], at)


def vec(n, dtype=torch.float32):
    return OnDevice(torch.zeros(n, dtype=dtype))


def act8(rows, cols, pad=0):
    return ops.Act8(mat(rows, cols, torch.int8, pad), mat(rows, -(-cols // 32), torch.uint8, pad))


def fields(p, kind):
    if not p:
        return None
    s = ctypes.cast(p, ctypes.POINTER(kind)).contents
    return {n: getattr(s, n) for n, _ in kind._fields_}


def same_rows(p, t):
    got = fields(p, ops.deto_rows)
    if t is None:
        return got is None
    codes = {torch.float32: 0, torch.bfloat16: 1, torch.float16: 2}
    return got == {"data": t.data_ptr(), "ld": t.stride(0) if t.shape[0] > 1 else t.shape[1],
                   "dtype": codes[t.dtype], "reserved": 0}


def same_act8(p, m):
    got = fields(p, ops.deto_act8)
    if m is None:
        return got is None
    return got == {"codes": m.codes.data_ptr(), "ld_codes": m.codes.stride(0), "exps": m.exps.data_ptr(),
                   "ld_exps": m.exps.stride(0)}


def ptr(t):
    return None if t is None else t.data_ptr()


SIGNATURES = {
    "token_logprobs": [i64, i64, vp, f32, vp, i32, vp, vp, vp, i32, vp, vp, vp, vp, vp],
    "token_logprobs_backward": [i64, i64, vp, f32, vp, i32, vp, vp, vp, vp, vp, vp],
    "norm_residual": [vp, i64, i64, vp, vp, vp, vp, vp, vp],
    "norm_residual_backward": [vp, i64, i64, vp, vp, vp, vp, vp, vp, vp, vp, vp],
    "act8_encode": [i64, i64, vp, vp, vp], "act8_decode": [i64, i64, vp, vp, vp],
    "glu_forward": [i32, i64, i64, vp, vp, vp, vp, vp, vp],
    "glu_backward": [i32, i64, i64, vp, vp, vp, vp, vp, vp, vp],
    "act8_weight_grad": [i64, i64, i64, vp, vp, vp, i32, vp, vp],
}


@pytest.fixture
def m():
    """The marshalling with the library's entry points replaced: `m.check` sees the arguments of a call, which
    returns `m.status`; a workspace takes 64 bytes.  Three devices, the current one is number 3."""
    lib = ops._load()
    fast = ops._load_marshal(lib)

    class Replaced:
        status, called, check = 0, "", staticmethod(lambda *a: True)

        def __getattr__(self, name):
            return getattr(fast, name)

    r = Replaced()

    def replace(name):
        if name.endswith("workspace"):
            args = {"token_logprobs_workspace": [i64, i64, i32], "norm_residual_workspace": [vp, i64, i64],
                    "act8_weight_grad_workspace": [i64, i64, i64]}[name]
            return ctypes.CFUNCTYPE(i64, *args)(lambda *a: 64)

        def f(*a):
            r.called, r.ok = name, bool(r.check(*a))
            return r.status
        return ctypes.CFUNCTYPE(i32, *SIGNATURES[name])(f)
    fns = [replace(n) for n in ops._MARSHALLED]
    fast.setup(tuple(ctypes.cast(f, vp).value for f in fns), ops._marshal_types(), lambda: 3, lambda d: 40 + d, 3)
    yield r
    ops._load_marshal(lib)


def ran(m, name, rc):
    return rc == 0 and m.called == name and m.ok


@pytest.mark.parametrize("stream,handle", [(None, 43), (7, 7)])
def test_logprobs(m, stream, handle):
    x, y, out, best = mat(T, D, torch.bfloat16, 3), vec(T, torch.int64), vec(T), mat(T, 4, torch.int32)
    lp, stats, ws = mat(T, 4), mat(T, 2), vec(64, torch.uint8)
    m.check = lambda *a: (a[:2] == (T, D) and same_rows(a[2], x) and a[3] == 0.5 and a[4:] == (
        ptr(y), 8, ptr(out), None, ptr(out), 4, ptr(best), ptr(lp), ptr(stats), ptr(ws), handle))
    assert ran(m, "token_logprobs", m.logprobs(x, y, out, None, out, best, lp, stats, 0.5, ws, stream))
    g = mat(T, D, torch.bfloat16)
    m.check = lambda *a: (a[:2] == (T, D) and same_rows(a[2], x) and a[3:10] == (
        1.0, ptr(y), 8, ptr(stats), None, ptr(out), None) and same_rows(a[10], g) and a[11] == handle)
    assert ran(m, "token_logprobs_backward", m.logprobs_backward(x, y, stats, g, out, None, None, 1.0, stream))


def test_logprobs_left_to_python(m):
    x, y, out, ws = mat(T, D), vec(T, torch.int64), vec(T), vec(64, torch.uint8)
    good = [x, y, out, None, None, None, None, None, 1.0, ws, None]
    assert m.logprobs(*good) == 0
    for i, bad in [(0, mat(T, D, torch.int8)), (0, mat(T, D, at=2)), (0, torch.zeros(T, D)), (0, vec(T)),
                   (0, OnDevice(torch.zeros(D, T).t())), (1, vec(T - 1, torch.int64)), (1, vec(T)),
                   (2, None), (2, vec(T + 1)), (2, OnDevice(torch.zeros(2 * T)[::2])), (3, vec(T, torch.float16)),
                   (5, mat(T, 33, torch.int32)), (5, mat(T, 4, torch.int32, 1)), (5, mat(T, 4, torch.int64)),
                   (6, mat(T, 4)), (7, vec(T)), (8, "1"), (9, vec(63, torch.uint8)), (9, None), (10, "s")]:
        args = list(good)
        args[i] = bad
        assert m.logprobs(*args) == -1, (i, bad)
    assert m.logprobs(*good[:-1]) == -1
    for status, said in ((1, -1), (2, -1), (5, 5)):       # refusals are named in Python
        m.status = status
        assert m.logprobs(*good) == said
    m.status = 0
    over = OnDevice(torch.zeros(T + 1, D))
    a, b = OnDevice(over.t[:T]), OnDevice(over.t[1:])
    assert m.logprobs_backward(a, y, mat(T, 2), b, out, None, None, 1.0, None) == -1
    assert m.logprobs_backward(a, y, mat(T, 2), a, out, None, None, 1.0, None) == 0


def test_norm(m):
    cfg = ops.NormResidual(pre=ops.NORM_RMS, post=ops.NORM_LAYER, eps_pre=0.5, eps_post=0.25, scale=2.0,
                           rows_per_gate=2)
    x, f, xo, y, y8 = mat(T, D, pad=1), mat(T, D, torch.float16), mat(T, D), mat(T, D, torch.float16), act8(T, D, 2)
    w, b, gate, ws = vec(D), vec(D), mat(3, D), vec(64, torch.uint8)
    want = {"pre": 1, "post": 2, "eps_pre": 0.5, "eps_post": 0.25, "scale": 2.0, "param_dtype": 0,
            "rows_per_gate": 2, "w_pre": ptr(w), "b_pre": None, "w_post": None, "b_post": ptr(b),
            "gate": ptr(gate), "ld_gate": D}
    m.check = lambda *a: (fields(a[0], ops.deto_norm_residual) == want and a[1:3] == (T, D) and same_rows(a[3], x)
                          and same_rows(a[4], f) and same_rows(a[5], xo) and same_rows(a[6], y)
                          and same_act8(a[7], y8) and a[8] == 43)
    good = [cfg, x, f, xo, y, y8, gate, None, b, w, None, None]
    assert ran(m, "norm_residual", m.norm(*good))
    dy, df, g = mat(T, D, torch.float16), mat(T, D, torch.float16), vec(D)
    m.check = lambda *a: (fields(a[0], ops.deto_norm_residual) == want and a[1:3] == (T, D) and same_rows(a[3], x)
                          and same_rows(a[4], f) and same_rows(a[5], dy) and same_rows(a[6], None)
                          and same_rows(a[7], xo) and same_rows(a[8], df)
                          and fields(a[9], ops.deto_norm_grads) == {"w_pre": ptr(g), "b_pre": None, "w_post": None,
                                                                    "b_post": None, "gate": ptr(gate)}
                          and a[10:] == (ptr(ws), 43))
    back = [cfg, x, f, dy, None, xo, df, ws, gate, None, b, w, gate, None, None, g, None, None]
    assert ran(m, "norm_residual_backward", m.norm_backward(*back))
    m.check = lambda *a: True
    for i, bad in [(1, mat(T, D, torch.int8)), (2, mat(T, D - 1)), (3, mat(T, D, torch.float16)), (4, mat(T, D)),
                   (5, act8(T, D + 32)), (6, mat(2, D)), (6, mat(3, D, torch.float16)), (8, vec(D - 1)),
                   (9, vec(D, torch.bfloat16)), (0, ops.NormResidual(pre=5)), (0, ops.NormResidual(rows_per_gate=-1))]:
        args = list(good)
        args[i] = bad
        assert m.norm(*args) == -1, (i, bad)
    for i, bad in [(5, None), (5, x), (7, None), (15, vec(D, torch.float16)), (12, mat(2, D)), (6, mat(T, D))]:
        args = list(back)
        args[i] = bad
        assert m.norm_backward(*args) == -1, (i, bad)
    one = [cfg, x, f, xo, y, None, None, None, None, None, None, None]      # a gate of one row: [D] too
    one[0], one[6] = ops.NormResidual(), vec(D)
    assert m.norm(*one) == 0


def test_activations(m):
    x, q = mat(T, D, torch.bfloat16, 2), act8(T, D, 1)
    m.check = lambda *a: a[:2] == (T, D) and same_rows(a[2], x) and same_act8(a[3], q) and a[4] == 43
    assert ran(m, "act8_encode", m.encode(x, q, None))
    m.check = lambda *a: a[:2] == (T, D) and same_act8(a[2], q) and same_rows(a[3], x) and a[4] == 43
    assert ran(m, "act8_decode", m.decode(q, x, None))
    a_, b_, h, q2 = mat(T, D), mat(T, D), mat(T, D), act8(T, D)
    m.check = lambda *a: (a[:3] == (2, T, D) and same_rows(a[3], a_) and same_rows(a[4], b_) and same_rows(a[5], h)
                          and same_act8(a[6], q) and same_act8(a[7], None) and a[8] == 43)
    assert ran(m, "glu_forward", m.glu_forward(2, a_, b_, h, q, None, None))
    m.check = lambda *a: (a[:3] == (3, T, D) and same_rows(a[3], h) and same_act8(a[4], q) and same_act8(a[5], q2)
                          and same_rows(a[6], a_) and same_rows(a[7], b_) and same_act8(a[8], None) and a[9] == 43)
    assert ran(m, "glu_backward", m.glu_backward(3, h, q, q2, a_, b_, None, None))
    m.check = lambda *a: True
    assert m.encode(x, None, None) == -1 and m.encode(x, act8(T, D - 1), None) == -1
    assert m.encode(x, ops.Act8(mat(T, D, torch.uint8), q.exps), None) == -1
    assert m.glu_forward(4, a_, b_, h, None, None, None) == -1 and m.glu_forward(0, a_, x, h, None, None, None) == -1
    assert m.glu_forward(0, a_, b_, None, None, None, None) == -1
    assert m.glu_backward(0, h, None, None, a_, None, None, None) == -1


def test_weight_grad(m):
    dy, q, dw, ws = mat(T, 9, torch.float16), act8(T, D), mat(9, D, torch.bfloat16, 1), vec(64, torch.uint8)
    m.check = lambda *a: (a[:3] == (T, 9, D) and same_rows(a[3], dy) and same_act8(a[4], q) and same_rows(a[5], dw)
                          and a[6:] == (1, ptr(ws), 43))
    assert ran(m, "act8_weight_grad", m.weight_grad(dy, q, dw, True, ws, None))
    assert m.weight_grad(dy, q, dw, 1, ws, None) == -1
    assert m.weight_grad(dy, q, mat(8, D), True, ws, None) == -1
    assert m.weight_grad(dy, act8(T - 1, D), dw, True, ws, None) == -1
    assert m.weight_grad(dy, q, dw, True, None, None) == -1
