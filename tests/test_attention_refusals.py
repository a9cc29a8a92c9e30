"""What the operators of an attention block refuse, without a GPU, beside tests/test_attention_abi.py: problems that one of two
launches cannot count, lengths at the end of an int, and outputs that meet an input in part."""
import pytest
import torch

from paper_2502_06728_amd import model_ops as ops
from tests.test_attention_abi import attention, m, vp  # noqa: F401
from tests.test_model_abi import BAD, UNSUPPORTED, lib, rows  # noqa: F401
from tests.test_model_marshal import OnDevice, mat


@pytest.mark.parametrize("Tq,Tk,sequences", [(1, 1 << 16, 1 << 16), (1 << 16, 1, 1 << 16), (1 << 12, 1 << 29, 1)])
def test_more_tiles_than_either_launch_counts(lib, Tq, Tk, sequences):  # noqa: F811
    """64 heads: of queries, or of keys alone."""
    starts = dict(q_starts=4096, k_starts=4096) if sequences > 1 else {}
    cfg = attention(heads=64, kv_heads=64, head_dim=1, sequences=sequences, causal=0, **starts)
    r = rows(ld=64)
    assert lib.detonation_attention_backward(cfg, Tq, Tk, r, r, r, r, vp(4096), r, r, r, r, vp(4096), None) == UNSUPPORTED


def test_lengths_that_a_step_would_count_past_an_int(lib):  # noqa: F811
    """The step behind the last whole one of 2^31 - 1 keys begins in an int and ends outside."""
    cfg, r, most = attention(heads=1, kv_heads=1, head_dim=1, sequences=1, causal=0), rows(ld=1), (1 << 31) - 512
    for Tq, Tk in ((1, (1 << 31) - 1), (1, most + 1), ((1 << 31) - 1, 1), (most + 1, 0)):
        assert lib.detonation_attention_workspace(cfg, Tq, Tk) == -1
        assert lib.detonation_attention_forward(cfg, Tq, Tk, r, r, r, r, None, vp(4096), None) == BAD
        assert lib.detonation_attention_backward(cfg, Tq, Tk, r, r, r, r, vp(4096), r, r, r, r, vp(4096), None) == BAD
    assert lib.detonation_attention_workspace(cfg, 1, most) > 0


def test_dropout_onto_other_columns_of_its_inputs(m):  # noqa: F811
    """In place is the same rows; rows that are moved by some columns, or are a part of others, are not."""
    whole = torch.zeros(5, 200)
    x, out = mat(5, 70), OnDevice(whole[:, 20:90])
    cfg = ops.Dropout(0.25, 1)

    def call(x, out, residual):
        return m.dropout(cfg, x, out, residual, 0, None, None)
    assert call(x, out, out) == 0 and call(out, out, None) == 0 and call(x, out, OnDevice(whole[:, 90:160])) == 0
    for columns in (19, 21, 89, 0):
        other = OnDevice(whole[:, columns:columns + 70])
        assert call(x, out, other) == -1, columns
        assert call(other, out, None) == -1, columns
    moved = OnDevice(torch.as_strided(whole, (4, 70), (200, 1), 220))
    assert call(OnDevice(whole[:4, 20:90]), moved, None) == -1                 # each row the next one
    x, out = torch.zeros(5, 70), whole[:, 20:90]
    for columns in (19, 21, 89, 0):
        with pytest.raises(ValueError, match="overlaps residual"):
            ops._disjoint({"out": out}, {"x": x, "residual": whole[:, columns:columns + 70]}, same=(("out", "x"), ("out", "residual")))
