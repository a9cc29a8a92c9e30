"""Which outputs of model_ops.py may lie where: the native marshalling and the checks in Python against the bytes that
the matrices really cover, without a GPU."""
import itertools

import pytest
import torch

from paper_2502_06728_amd import model_ops as ops
from tests.test_model_marshal import D, T, OnDevice, act8, m, mat, vec  # noqa: F401


def covered(t):
    e = t.element_size()
    return {t.data_ptr() + (r * t.stride(0) + c * t.stride(1)) * e + i
            for r in range(t.shape[0]) for c in range(t.shape[1]) for i in range(e)}


def slices():
    """Matrices of 3 rows in one piece of memory: columns side by side, rows below each other, shifted rows."""
    flat = torch.zeros(400)
    for ld, first in itertools.product((10, 12), (0, 1, 5, 9, 10, 30, 60)):
        for width in (1, 4, 5, 9):
            yield torch.as_strided(flat, (3, width), (ld, 1), first)
    for first in (0, 5, 10, 35):                  # one row
        for width in (1, 5, 30):
            yield torch.as_strided(flat, (1, width), (width, 1), first)


def test_memory_that_meets():
    for a, b in itertools.product(slices(), slices()):
        shared, says = bool(covered(a) & covered(b)), ops._meet(ops._span(a), ops._span(b))
        if a.shape[0] > 1 and b.shape[0] > 1 and a.stride(0) != b.stride(0):
            assert says or not shared
        else:
            assert says == shared, (a.shape, a.stride(), a.storage_offset(), b.shape, b.stride(), b.storage_offset())


def test_columns_of_one_matrix(m):  # noqa: F811
    """Three columns of one matrix take a, b and h of a gated activation; a gradient beside its logits."""
    whole = torch.zeros(T, 3 * D, dtype=torch.bfloat16)
    a, b, h = (OnDevice(whole[:, i * D:(i + 1) * D]) for i in range(3))
    assert m.glu_forward(0, a, b, h, None, None, None) == 0
    assert m.glu_backward(0, a, act8(T, D), act8(T, D), b, h, None, None) == 0
    assert m.glu_forward(0, a, b, OnDevice(whole[:, 2 * D - 1:3 * D - 1]), None, None, None) == -1
    y, out = vec(T, torch.int64), vec(T)
    assert m.logprobs_backward(a, y, mat(T, 2), b, out, None, None, 1.0, None) == 0
    assert m.logprobs_backward(b, y, mat(T, 2), a, out, None, None, 1.0, None) == 0
    for shift in (1, D - 1):
        near = OnDevice(torch.as_strided(whole, (T, D), (3 * D, 1), shift))
        assert m.logprobs_backward(a, y, mat(T, 2), near, out, None, None, 1.0, None) == -1
        assert m.logprobs_backward(near, y, mat(T, 2), a, out, None, None, 1.0, None) == -1
    with pytest.raises(ValueError, match="overlaps"):
        ops._apart(near, ("logits", a))
    ops._apart(a, ("logits", b), ("itself", a))


def test_native_checks_say_the_same(m):  # noqa: F811
    for a, b in itertools.product(slices(), slices()):
        if a.shape == b.shape:
            rows = a.shape[0]
            same = a.data_ptr() == b.data_ptr() and a.stride() == b.stride()
            got = m.logprobs_backward(OnDevice(a), vec(rows, torch.int64), mat(rows, 2), OnDevice(b), vec(rows), None,
                                      None, 1.0, None)
            assert (got == 0) == (same or not ops._meet(ops._span(a), ops._span(b)))


def as_act8(t):
    """8-bit codes and exponents in the memory of a [T, D] matrix."""
    raw = t.t.view(torch.int8)
    return ops.Act8(OnDevice(raw[:, :D]), mat(T, -(-D // 32), torch.uint8)), \
        ops.Act8(mat(T, D, torch.int8), OnDevice(raw.view(torch.uint8)[:, :-(-D // 32)]))


def test_outputs_lie_apart(m):  # noqa: F811
    """Every call is taken with matrices of their own and left to the checks in Python, which name it, with an output
    in the memory of an input or of another output."""
    x, f, xo, y, dy, dxo, df, dx = (mat(T, D) for _ in range(8))
    q, gate, w, g = act8(T, D), mat(1, D), vec(D), vec(D)
    ws = vec(64, torch.uint8)
    inside = lambda t: OnDevice(t.t.view(torch.uint8).flatten()[:64])  # noqa: E731
    cfg = ops.NormResidual(post=ops.NORM_RMS)

    good = [cfg, x, f, xo, y, q, gate, w, None, None, None, None]
    assert m.norm(*good) == 0
    assert m.norm(*good[:3], x, *good[4:]) == 0                       # in place
    for bad in [{4: x}, {4: f}, {4: xo}, {3: f}, {3: y},
                *({5: a} for t in (x, f, xo, y) for a in as_act8(t)), {7: OnDevice(y.t[0])}, {6: OnDevice(xo.t[:1])}]:
        args = [bad.get(i, v) for i, v in enumerate(good)]
        assert m.norm(*args) == -1, bad

    good = [cfg, x, f, dy, dxo, dx, df, ws, gate, w, None, None, None, g, None, None, None, None]
    assert m.norm_backward(*good) == 0
    assert m.norm_backward(*good[:5], dxo, *good[6:]) == 0            # in place
    for bad in [{5: x}, {5: f}, {5: dy}, {5: df}, {6: f}, {6: dy}, {6: x}, {6: dxo}, {7: inside(x)}, {7: inside(dx)},
                {7: inside(f)}, {9: OnDevice(df.t[1])}]:
        args = [bad.get(i, v) for i, v in enumerate(good)]
        assert m.norm_backward(*args) == -1, bad

    for a in as_act8(x):
        assert m.encode(x, a, None) == -1 and m.decode(a, x, None) == -1
    both = torch.zeros(T, D, dtype=torch.int8)
    assert m.encode(x, ops.Act8(OnDevice(both), OnDevice(both.view(torch.uint8)[:, :-(-D // 32)])), None) == -1

    a, b, h, q2 = mat(T, D), mat(T, D), mat(T, D), act8(T, D)
    good = [0, a, b, h, q, q2, None]
    assert m.glu_forward(*good) == 0
    assert m.glu_forward(0, a, b, a, q, q2, None) == 0 and m.glu_forward(0, a, b, b, q, q2, None) == 0
    for bad in [{5: q}, *({4: p} for t in (a, b, h) for p in as_act8(t)), *({5: p} for t in (a, b, h) for p in as_act8(t))]:
        args = [bad.get(i, v) for i, v in enumerate(good)]
        assert m.glu_forward(*args) == -1, bad

    q3 = act8(T, D)
    good = [0, h, q, q2, a, b, q3, None]
    assert m.glu_backward(*good) == 0
    assert m.glu_backward(0, h, q, q2, h, b, q3, None) == 0 and m.glu_backward(0, h, q, q2, a, h, q3, None) == 0
    for bad in [{5: a}, {4: h, 5: h}, {6: q}, {6: q2}, *({6: p} for t in (a, b, h) for p in as_act8(t)),
                *({2: p} for t in (a, b) for p in as_act8(t))]:
        args = [bad.get(i, v) for i, v in enumerate(good)]
        assert m.glu_backward(*args) == -1, bad

    dw, wide = mat(D, D), mat(T, D)
    good = [wide, q, dw, True, ws, None]
    assert m.weight_grad(*good) == 0
    for bad in [{0: OnDevice(dw.t[:T])}, {4: inside(dw)}, {4: inside(wide)},
                {1: ops.Act8(OnDevice(dw.t.view(torch.int8)[:T, :D]), q.exps)},
                {1: ops.Act8(q.codes, OnDevice(dw.t.view(torch.uint8)[:T, :-(-D // 32)]))}]:
        args = [bad.get(i, v) for i, v in enumerate(good)]
        assert m.weight_grad(*args) == -1, bad

    yv, out = vec(T, torch.int64), vec(T)
    assert m.logprobs(x, yv, out, None, None, None, None, None, 1.0, inside(x), None) == -1


def test_the_checks_in_python_name_it():
    (x, y, z), q = (torch.zeros(T, D) for _ in range(3)), act8(T, D)
    ops._disjoint({"a": x, "b": y, "workspace": (torch.zeros(9), 36)}, {"c": z, "q": q, "none": None})
    ops._disjoint({"a": x}, {"c": x}, same=(("a", "c"),))
    for outs, ins, same in [({"a": x, "c": x}, {}, ()), ({"a": x}, {"c": x}, ()), ({"a": x}, {"c": x[:, 1:]}, (("a", "c"),)),
                            ({"a": x}, {"c": x[2]}, ()), ({"workspace": (x, 4)}, {"c": x}, ()),
                            ({"q": ops.Act8(x.view(torch.int8)[:, :D], q.exps)}, {"c": x}, ()),
                            ({"a": x, "b": x}, {"c": x}, (("a", "c"), ("b", "c")))]:
        with pytest.raises(ValueError, match="overlaps"):
            ops._disjoint(outs, ins, same)
    ops._disjoint({"workspace": (x, 0)}, {"c": x})
    ops._disjoint({"a": x[:0]}, {"c": x[:0]})


def test_gates_of_another_shape(m):  # noqa: F811
    """As many elements as the gate's rows have, but not those rows: named in Python."""
    cfg = ops.NormResidual(rows_per_gate=2)
    x, f, xo, y, ws = mat(T, D), mat(T, D), mat(T, D), mat(T, D), vec(64, torch.uint8)
    for gate, taken in [(mat(3, D), True), (mat(D, 3), False), (vec(3 * D), False), (mat(2, D), False)]:
        assert m.norm(cfg, x, f, xo, y, None, gate, None, None, None, None, None) == (0 if taken else -1)
        assert m.norm_backward(cfg, x, f, y, None, xo, mat(T, D), ws, gate, None, None, None, None, None, None, None, None,
                               None) == (0 if taken else -1)
    cfg = ops.NormResidual()
    for gate in (mat(1, D), vec(D)):
        assert m.norm(cfg, x, f, xo, y, None, gate, None, None, None, None, None) == 0
