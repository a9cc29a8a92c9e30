"""Attention where few tests go: sequences without queries under grouped heads, infinities that are seen, scores so large that
fp32 does not hold them to a unit, queries with few keys beside long sequences, calls without a workspace."""
import pytest
import torch

from paper_2502_06728_amd import model_ops as ops
from tests import attention_reference as ref
from tests.model_reference import BF16, F16, F32
from tests.test_gpu_attention import Case, even
from tests.test_gpu_model_ops import DEV, INF, NAN, TYPES, say

pytestmark = pytest.mark.gpu


def defined(c):
    """out, lse, dq, dk and dv of a case of one sequence, all heads at once in 64 bits; infinite keys count as zeros in the
    product that gives dq.  And the size of what is added up in dq."""
    H, K, n, m = c.cfg.heads, c.cfg.kv_heads, len(c.q), len(c.k)

    def apart(t, heads):
        t = t.double().reshape(len(t), heads, -1).transpose(0, 1)
        return t.repeat_interleave(H // heads, 0).contiguous()

    def together(t):
        return t.transpose(0, 1).reshape(t.shape[1], -1)
    q, k, v, g = apart(c.q, H), apart(c.k, K), apart(c.v, K), apart(c.dout, H)
    sees = torch.ones((n, m), dtype=torch.bool, device=DEV)
    if c.cfg.causal:
        sees = sees.tril(m - n)
    s = torch.where(sees, q @ k.transpose(1, 2).contiguous() * c.cfg.scale, -INF)
    p = torch.softmax(s, 2)
    out = p @ v
    ds = p * (g @ v.transpose(1, 2).contiguous() - (g * out).sum(2, keepdim=True))
    k = torch.where(torch.isfinite(k), k, 0.0)
    dk, dv = (x.transpose(1, 2).contiguous() @ y for x, y in ((ds * c.cfg.scale, q), (p, g)))
    dk, dv = (t.unflatten(0, (K, H // K)).sum(1) for t in (dk, dv))
    return ({"out": together(out), "lse": torch.logsumexp(s, 2), "dq": together(ds @ k * c.cfg.scale), "dk": together(dk),
             "dv": together(dv)}, together(ds.abs() @ k.abs() * c.cfg.scale))


def unit(dtype):
    """What a row of results may be off by, of its size (the type's own rounding, that of the weights, that of the written out:
    a third of u^2 each; in fp32 those of scores and of sums)."""
    return 64 * ref.FINE if dtype == F32 else ref.UNIT[dtype]


def assert_rows(got, want, u, what):
    """As a whole to u, each row to 4 u of its size or of the rows' mean size."""
    got = got.double()
    assert bool(torch.isfinite(got).all()), what
    off, size = (got - want).norm(dim=1), want.norm(dim=1)
    say(what, float(off.norm() / size.norm()) / u)
    assert float(off.norm()) <= u * float(size.norm()), what
    assert bool((off <= 4 * u * torch.maximum(size, size.norm() / len(size) ** 0.5)).all()), what


# ------------------------------------------------------------------ sequences without queries

@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("heads,kv_heads", [(4, 2), (4, 1)])
@pytest.mark.parametrize("head_dim", [128, 104])
def test_keys_without_queries(gpu, dtype, heads, kv_heads, head_dim):
    """Groups of heads are taken two or four at a time: a sequence of keys alone has no step to wait in, and its gradients
    are zeros all the same."""
    c = Case(dtype, [0, 0, 150, 150, 151], [0, 140, 290, 355, 400], heads, kv_heads, head_dim, True)
    c.forward()
    c.backward()
    c.check()
    assert not bool(c.dk[:140].any()) and not bool(c.dv[:140].any())
    assert not bool(c.dk[290:355].any()) and not bool(c.dv[290:355].any())
