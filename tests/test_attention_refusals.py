"""What the operators of an attention block refuse, without a GPU, beside tests/test_attention_abi.py: problems that one of two
launches cannot count."""
import pytest

from tests.test_attention_abi import attention, vp
from tests.test_model_abi import UNSUPPORTED, lib, rows  # noqa: F401


@pytest.mark.parametrize("Tq,Tk,sequences", [(1, 1 << 16, 1 << 16), (1 << 16, 1, 1 << 16), (1 << 12, 1 << 29, 1)])
def test_more_tiles_than_either_launch_counts(lib, Tq, Tk, sequences):  # noqa: F811
    """64 heads: of queries, or of keys alone."""
    starts = dict(q_starts=4096, k_starts=4096) if sequences > 1 else {}
    cfg = attention(heads=64, kv_heads=64, head_dim=1, sequences=sequences, causal=0, **starts)
    r = rows(ld=64)
    assert lib.detonation_attention_backward(cfg, Tq, Tk, r, r, r, r, vp(4096), r, r, r, r, vp(4096), None) == UNSUPPORTED
