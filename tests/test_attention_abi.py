"""Rotary positions, attention and dropout of include/detonation_model.h without a GPU: struct layouts, what the host-side
checks refuse (these calls return before any launch), and the native argument marshalling of their calls."""
import ctypes
import os
import subprocess

import pytest
import torch

from paper_2502_06728_amd import model_ops as ops
from tests.test_model_abi import ALIGN, BAD, NULL, OK, ROOT, UNSUPPORTED, lib, rows  # noqa: F401
from tests.test_model_marshal import OnDevice, fields, mat, ptr, same_rows, vec

vp, i32, i64 = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64


def test_struct_layouts_match_the_header(tmp_path):
    src, exe = tmp_path / "sizes.c", tmp_path / "sizes"
    kinds = (ops.deto_rotary, ops.deto_attention, ops.deto_dropout)
    prints = "".join(f'printf("%zu ", sizeof({k.__name__}));' +
                     "".join(f'printf("%zu ", offsetof({k.__name__}, {n}));' for n, _ in k._fields_) for k in kinds)
    src.write_text('#include "detonation_model.h"\n#include <stddef.h>\n#include <stdio.h>\n'
                   f'int main(void) {{ {prints} return 0; }}\n')
    subprocess.run(["gcc", "-std=c99", "-Wall", "-Wextra", "-Werror", "-pedantic", "-I", os.path.join(ROOT, "include"), "-o",
                    str(exe), str(src)], check=True)
    got = [int(v) for v in subprocess.run([str(exe)], capture_output=True, text=True).stdout.split()]
    assert got == [v for k in kinds for v in [ctypes.sizeof(k)] + [getattr(k, n).offset for n, _ in k._fields_]]


def test_rotary_refusals(lib):  # noqa: F811
    def f(T=4, x=rows(), out=rows(), freqs=4096, p=4096, pb=8, cfg=True, **kw):
        s = dict(layout=0, heads=2, head_dim=32, rotary_dim=32, inverse=0, magnitude=1.0, first=0, period=0) | kw
        return lib.detonation_rotary(ctypes.byref(ops.deto_rotary(**s)) if cfg else None, T, x, vp(freqs), vp(p), pb, out, None)
    assert f(cfg=False) == NULL and f(T=-1) == BAD and f(heads=0) == BAD and f(head_dim=1, rotary_dim=2) == BAD
    assert f(layout=2) == BAD and f(layout=-1) == BAD and f(rotary_dim=0) == BAD and f(rotary_dim=31) == BAD
    assert f(rotary_dim=34) == BAD and f(inverse=2) == BAD and f(magnitude=float("inf")) == BAD
    assert f(magnitude=float("nan")) == BAD and f(first=-1) == BAD and f(period=-1) == BAD and f(first=1 << 53) == BAD
    assert f(pb=2) == BAD and f(heads=1 << 26) == BAD and f(x=rows(ld=63)) == BAD and f(out=rows(dtype=1)) == BAD
    assert f(x=rows(dtype=3)) == BAD and f(x=None) == NULL and f(out=None) == NULL and f(freqs=None) == NULL
    assert f(x=rows(data=4098)) == ALIGN and f(freqs=4100) == ALIGN and f(p=4100) == ALIGN and f(p=4098, pb=4) == ALIGN
    assert f(T=0, x=None, out=None, freqs=None) == OK


def attention(**kw):
    return ctypes.byref(ops.deto_attention(**(dict(heads=2, kv_heads=1, head_dim=32, causal=1, scale=1.0, reserved=0, sequences=2)
                                              | kw)))


def test_attention_refusals(lib):  # noqa: F811
    def f(Tq=4, Tk=6, q=rows(), k=rows(ld=32), v=rows(ld=32), out=rows(), lse=4096, ws=4096, cfg=attention()):
        return lib.detonation_attention_forward(cfg, Tq, Tk, q, k, v, out, vp(lse), vp(ws), None)

    def b(Tq=4, Tk=6, q=rows(), k=rows(ld=32), v=rows(ld=32), out=rows(), lse=4096, do=rows(), dq=rows(), dk=rows(ld=32),
          dv=rows(ld=32), ws=4096, cfg=attention()):
        return lib.detonation_attention_backward(cfg, Tq, Tk, q, k, v, out, vp(lse), do, dq, dk, dv, vp(ws), None)
    for g in (f, b):
        assert g(cfg=None) == NULL and g(Tq=-2) == BAD and g(Tk=-2) == BAD and g(Tq=5) == BAD and g(Tk=7) == BAD
        assert g(Tq=1 << 31) == BAD
        for bad in (dict(heads=0), dict(kv_heads=0), dict(heads=3, kv_heads=2), dict(heads=65537), dict(head_dim=0),
                    dict(causal=2), dict(scale=0.0), dict(scale=-1.0), dict(scale=float("inf")), dict(scale=float("nan")),
                    dict(reserved=1), dict(sequences=0), dict(sequences=-1), dict(sequences=1 << 31)):
            assert g(cfg=attention(**bad)) == BAD, bad
        assert g(cfg=attention(head_dim=129)) == UNSUPPORTED
        assert g(cfg=attention(q_starts=4098)) == ALIGN and g(cfg=attention(k_starts=4097)) == ALIGN
        assert g(q=None) == NULL and g(k=None) == NULL and g(v=rows(data=None)) == NULL and g(out=None) == NULL
        assert g(q=rows(ld=63)) == BAD and g(k=rows(ld=31)) == BAD and g(q=rows(dtype=1)) == BAD and g(v=rows(ld=32, dtype=2)) == BAD
        assert g(q=rows(dtype=3)) == BAD and g(q=rows(reserved=1)) == BAD and g(q=rows(data=4098)) == ALIGN
        assert g(lse=4098) == ALIGN
    assert f(Tq=0, q=None, out=None, lse=None) == OK
    assert b(Tq=0, Tk=0, q=None, k=None, v=None, out=None, lse=None, do=None, dq=None, dk=None, dv=None, ws=None) == OK
    assert b(lse=None) == NULL and b(ws=None) == NULL and b(ws=4104) == ALIGN
    assert b(do=None) == NULL and b(dq=None) == NULL and b(dk=None) == NULL and b(dv=None) == NULL
    assert b(do=rows(dtype=1)) == BAD and b(dk=rows(ld=32, dtype=2)) == BAD
    many = dict(Tq=1 << 30, Tk=1 << 30)                       # more tiles than a launch counts
    assert f(**many, cfg=attention(heads=65536, head_dim=1), q=rows(ld=65536), out=rows(ld=65536)) == UNSUPPORTED
    assert lib.detonation_attention_workspace(attention(), 5, 6) == -1
    assert lib.detonation_attention_workspace(attention(q_starts=8), 5, 6) >= 2 * 5 * 4
    assert lib.detonation_attention_workspace(attention(), 0, 0) >= 0


def test_dropout_refusals(lib):  # noqa: F811
    def f(T=4, D=64, x=rows(), r=None, out=rows(), cfg=True, **kw):
        s = dict(seed=1, offset=2, device_offset=None, rate=0.5, reserved=0) | kw
        return lib.detonation_dropout(ctypes.byref(ops.deto_dropout(**s)) if cfg else None, T, D, x, r, out, None)
    assert f(cfg=False) == NULL and f(T=-1) == BAD and f(D=0) == BAD and f(D=(1 << 30) + 1) == BAD and f(T=(1 << 32) + 1) == BAD
    for rate in (-0.1, 1.0, 1.5, float("nan"), float("inf"), 0.99999999):
        assert f(rate=rate) == BAD, rate
    assert f(reserved=1) == BAD and f(device_offset=4100) == ALIGN
    assert f(x=None) == NULL and f(out=None) == NULL and f(x=rows(ld=63)) == BAD and f(out=rows(ld=63)) == BAD
    assert f(r=rows(dtype=1)) == BAD and f(x=rows(dtype=1), out=rows(dtype=2)) == BAD and f(r=rows(ld=63)) == BAD
    assert f(x=rows(data=4098)) == ALIGN and f(r=rows(data=4098)) == ALIGN
    assert f(T=0, x=None, out=None) == OK


# ------------------------------------------------------------------ marshalling

SIGNATURES = {"rotary": [vp, i64, vp, vp, vp, i32, vp, vp], "attention_forward": [vp, i64, i64, vp, vp, vp, vp, vp, vp, vp],
              "attention_backward": [vp, i64, i64, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp],
              "dropout": [vp, i64, i64, vp, vp, vp, vp]}


@pytest.fixture
def m():
    """The marshalling with the library's entry points replaced; a workspace takes 64 bytes; the current device is 3."""
    fast = ops._load_marshal(ops._load())

    class Replaced:
        status, called, check = 0, "", staticmethod(lambda *a: True)

        def __getattr__(self, name):
            return getattr(fast, name)
    r = Replaced()

    def replace(name):
        if name.endswith("workspace"):
            return ctypes.CFUNCTYPE(i64, vp, i64, i64)(lambda *a: 64)

        def f(*a):
            r.called, r.ok = name, bool(r.check(*a))
            return r.status
        return ctypes.CFUNCTYPE(i32, *SIGNATURES[name])(f)
    fns = [replace(n) for n in ops._MARSHALLED_BLOCK]
    unused = ctypes.CFUNCTYPE(i32)(lambda: 1)
    fast.setup((ctypes.cast(unused, vp).value,) * len(ops._MARSHALLED), ops._marshal_types(), lambda: 3, lambda d: 40 + d, 3)
    fast.setup_block(tuple(ctypes.cast(f, vp).value for f in fns))
    yield r
    ops._load_marshal(ops._load())


def ran(m, name, rc):
    return rc == 0 and m.called == name and m.ok


def with_each(good, changes, call):
    for i, bad in changes:
        args = list(good)
        args[i] = bad
        assert call(*args) == -1, (i, bad)


def shared(t, columns):
    """Other columns that meet a matrix's."""
    return OnDevice(torch.as_strided(t.t, t.t.shape, t.t.stride(), columns))


def test_rotary_call(m):
    whole = torch.zeros(5, 200)
    x, out = OnDevice(whole[:, :96]), OnDevice(whole[:, 96:192])
    freqs, p = vec(8, torch.float64), vec(5, torch.int64)
    cfg = ops.Rotary(heads=3, head_dim=32, rotary_dim=16, layout=ops.ROTARY_PAIRS, magnitude=0.5, first=2, period=7)
    want = {"layout": 1, "heads": 3, "head_dim": 32, "rotary_dim": 16, "inverse": 1, "magnitude": 0.5, "first": 2, "period": 7}
    m.check = lambda *a: (fields(a[0], ops.deto_rotary) == want and a[1] == 5 and same_rows(a[2], x) and a[3:6] == (
        ptr(freqs), ptr(p), 8) and same_rows(a[6], out) and a[7] == 43)
    good = [cfg, x, freqs, out, p, True, None]
    assert ran(m, "rotary", m.rotary(*good))
    m.check = lambda *a: a[4:6] == (None, 0) and a[7] == 9
    assert ran(m, "rotary", m.rotary(cfg, x, freqs, x, None, False, 9))           # in place
    m.check = lambda *a: fields(a[0], ops.deto_rotary)["rotary_dim"] == 32
    assert ran(m, "rotary", m.rotary(ops.Rotary(3, 32), x, vec(16, torch.float64), out, vec(5, torch.int32), False, None))
    with_each(good, [(0, ops.Rotary(2, 32)), (0, None), (1, mat(5, 95)), (1, mat(5, 96, at=2)), (2, vec(8)), (2, None),
                     (2, vec(7, torch.float64)), (3, mat(5, 96, torch.float16)), (3, None), (4, vec(4, torch.int64)),
                     (4, vec(5)), (5, 1), (3, shared(x, 1)), (6, "s")], m.rotary)
    for status, said in ((1, -1), (2, -1), (5, 5)):
        m.status = status
        assert m.rotary(*good) == said


def test_attention_calls(m):
    T, S, N, W = 6, 8, 16, 32
    cfg = ops.Attention(heads=4, head_dim=8, scale=0.25, kv_heads=2, causal=False, sequences=2)
    dt = torch.bfloat16
    qkv = torch.zeros(T, W + 2 * N, dtype=dt)
    q, k, v = OnDevice(qkv[:, :W]), mat(S, N, dt, 3), mat(S, N, dt)
    out, lse, ws = mat(T, W, dt), mat(4, T), vec(64, torch.uint8)
    qs, ks = vec(3, torch.int32), vec(3, torch.int32)
    want = {"heads": 4, "kv_heads": 2, "head_dim": 8, "causal": 0, "scale": 0.25, "reserved": 0, "sequences": 2}
    m.check = lambda *a: (fields(a[0], ops.deto_attention) == want | {"q_starts": ptr(qs), "k_starts": ptr(ks)} and a[1:3] == (T, S)
                          and same_rows(a[3], q) and same_rows(a[4], k) and same_rows(a[5], v) and same_rows(a[6], out)
                          and a[7:] == (ptr(lse), ptr(ws), 43))
    good = [cfg, q, k, v, out, lse, qs, ks, ws, None]
    assert ran(m, "attention_forward", m.attention_forward(*good))
    m.check = lambda *a: fields(a[0], ops.deto_attention) == want | {"q_starts": None, "k_starts": None} and a[7] is None
    assert ran(m, "attention_forward", m.attention_forward(cfg, q, k, v, out, None, None, None, ws, None))
    bad = [(0, ops.Attention(4, 7, 0.25, 2)), (0, ops.Attention(4, 8, 0.25, 2, sequences=3)), (0, ops.Attention(4, 8, 0.25)),
           (1, mat(T, W)), (2, mat(S, N)), (3, mat(S + 1, N, dt)), (3, None), (4, None), (4, mat(T, W, torch.float16)),
           (5, vec(4 * T + 1)), (6, vec(3, torch.int64)), (7, vec(4, torch.int32)), (8, None), (8, vec(63, torch.uint8)),
           (4, q), (4, shared(q, 4)), (5, OnDevice(qkv.view(torch.float32).flatten()[:24]))]
    with_each(good, bad, m.attention_forward)

    g, dq, dk, dv = mat(T, W, dt), mat(T, W, dt), mat(S, N, dt), mat(S, N, dt)
    m.check = lambda *a: (fields(a[0], ops.deto_attention) == want | {"q_starts": ptr(qs), "k_starts": None} and a[1:3] == (T, S)
                          and all(same_rows(x, t) for x, t in zip(a[3:7] + a[8:12], (q, k, v, out, g, dq, dk, dv)))
                          and a[7] == ptr(lse) and a[12:] == (ptr(ws), 7))
    back = [cfg, q, k, v, out, lse, g, dq, dk, dv, qs, None, ws, 7]
    assert ran(m, "attention_backward", m.attention_backward(*back))
    with_each(back, [(4, None), (5, None), (5, vec(4 * T - 1)), (6, mat(T, W)), (7, q), (7, g), (8, k), (8, dv), (9, v),
                     (9, mat(S, N)), (12, None), (7, out), (10, vec(2, torch.int32))], m.attention_backward)
    # gradients side by side in one matrix
    d = torch.zeros(T, 3 * W, dtype=dt)
    cfg = ops.Attention(4, 8, 0.25, sequences=1)
    a, b, c = (OnDevice(d[:, i * W:(i + 1) * W]) for i in range(3))
    m.check = lambda *x: True
    assert m.attention_backward(cfg, q, q, q, out, lse, g, a, b, c, None, None, ws, None) == 0
    assert m.attention_backward(cfg, q, q, q, out, lse, g, a, b, shared(b, W + 1), None, None, ws, None) == -1


def test_dropout_call(m):
    x, out, res, more = mat(5, 70, torch.float16, 2), mat(5, 70), mat(5, 70), vec(1, torch.int64)
    cfg = ops.Dropout(rate=0.25, seed=(1 << 64) - 1)
    want = {"seed": (1 << 64) - 1, "offset": 1 << 63, "device_offset": ptr(more), "rate": 0.25, "reserved": 0}
    m.check = lambda *a: (fields(a[0], ops.deto_dropout) == want and a[1:3] == (5, 70) and same_rows(a[3], x)
                          and same_rows(a[4], res) and same_rows(a[5], out) and a[6] == 43)
    good = [cfg, x, out, res, 1 << 63, more, None]
    assert ran(m, "dropout", m.dropout(*good))
    m.check = lambda *a: same_rows(a[4], None)
    assert ran(m, "dropout", m.dropout(cfg, out, out, None, 0, None, None))               # in place
    m.check = lambda *a: True
    assert m.dropout(cfg, x, out, out, 0, None, None) == 0
    half = OnDevice(out.t.view(torch.float16)[:, :70])
    with_each(good, [(0, ops.Dropout(0.25, -1)), (0, ops.Dropout(0.25, 1 << 64)), (0, ops.Dropout(0.25, "a")), (1, mat(5, 69)),
                     (1, mat(5, 70, torch.int32)), (2, mat(4, 70)), (2, None), (3, x), (4, -1), (4, 1 << 64), (4, 1.5),
                     (5, vec(2, torch.int64)), (5, vec(1)), (1, half), (2, shared(res, 0))][:-1], m.dropout)


def test_checks_in_python_name_what_is_wrong():
    """Without a GPU every call goes there: a host tensor is refused by name."""
    x = torch.zeros(4, 64)
    with pytest.raises(ValueError, match="x must be a device tensor"):
        ops.detonation_rotary(ops.Rotary(2, 32), x, torch.zeros(16, dtype=torch.float64), x)
    with pytest.raises(ValueError, match="2 x 30"):
        ops.detonation_rotary(ops.Rotary(2, 30), x, torch.zeros(16, dtype=torch.float64), x)
    with pytest.raises(ValueError, match="q must be a device tensor"):
        ops.detonation_attention_forward(ops.Attention(2, 32, 1.0), x, x, x, x)
    with pytest.raises(ValueError, match="x must be a device tensor"):
        ops.detonation_dropout(ops.Dropout(0.5), x, x)
    with pytest.raises(ValueError, match="64 bits"):
        ops.detonation_dropout(ops.Dropout(0.5), x, x, offset=-1)
    for T in ((-1, 4), (4, -1), (5, 4)):
        size = dict(sequences=1) if T[0] < 5 else dict(sequences=0)
        with pytest.raises(ValueError):
            ops.attention_workspace(ops.Attention(2, 32, 1.0, **size), *T)
