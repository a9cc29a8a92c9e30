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
