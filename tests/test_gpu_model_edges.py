"""The kernels behind include/detonation_model.h where their arithmetic has few bits to spare: widths that leave
lanes empty, values at the ends of a type's range, sums of many steps.  Plain definitions in 64 bits."""
import math

import pytest
import torch

from paper_2502_06728_amd import model_ops as ops
from tests import model_reference as ref
from tests import test_gpu_model_ops as base
from tests.model_reference import BF16, F16, F32, assert_near
from tests.test_gpu_model_ops import DEV, INF, NAN, TYPES, like, normal, rows, say, scratch

pytestmark = pytest.mark.gpu


# ------------------------------------------------------------------ norm, gate, residual

@pytest.mark.parametrize("xt,ft", [(F32, F32), (F32, BF16), (BF16, BF16)])
@pytest.mark.parametrize("weights,rows_per_gate", [(False, None), (False, 0), (True, None)])
@pytest.mark.parametrize("pre,post", [("layer", "layer"), ("layer", "rms"), ("layer", "none"), ("rms", "layer"),
                                      ("rms", "rms"), ("none", "layer")])
@pytest.mark.parametrize("D", [40, 72, 96, 264, 768, 1152, 1536, 5120, 9000])
def test_norm_gradient_at_widths_that_leave_lanes_empty(gpu, D, pre, post, weights, rows_per_gate, xt, ft):
    """Absent weights and gates are ones, in the lanes past the row's end too: what those hold must not reach the
    row's sums."""
    T = 3
    s = base.norm_inputs(T, D, pre, post, rows_per_gate, weights, xt, ft, 0, 0)
    dy = rows(normal(5, T, D), ft) if pre != "none" else None
    dxo, dx, df = rows(normal(6, T, D), xt), like(T, D, xt), like(T, D, ft)
    grads = {"d" + n: torch.full(v.shape, NAN, device=DEV) for n, v in s["p"].items()}
    ops.detonation_norm_residual_backward(
        s["cfg"], s["x"], s["f"], dy, dxo, dx, df, workspace=scratch(ops.norm_residual_workspace(s["cfg"], T, D)),
        **{n: v for n, v in s["p"].items() if n != "b_pre"}, **grads)
    p = {n: ref.double(v).requires_grad_() for n, v in s["p"].items()}
    f = ref.double(s["f"]).requires_grad_()
    with torch.no_grad():
        branch = base.reference_block(s, "none", post, torch.zeros_like(f), f, p)[0]
    x = (ref.double(s["x"]) - branch).requires_grad_()
    x_out, y = base.reference_block(s, pre, post, x, f, p)
    loss = (x_out * ref.double(dxo)).sum() + ((y * ref.double(dy)).sum() if pre != "none" else 0.0)
    g = torch.autograd.grad(loss, [x, f, *p.values()])
    # gradients, normalised rows and parameters of a few units each: 64 roundings of products of two of them
    assert_near(dx, g[0], 32.0, base.NORM_STEPS, "dx")
    assert_near(df, g[1], 32.0, base.NORM_STEPS, "df")
    for (name, got), want in zip(grads.items(), g[2:]):
        assert_near(got, want, 32.0, base.NORM_STEPS, name)


# ------------------------------------------------------------------ log probabilities

def check_sums(x, y, out, scale=1.0):
    """logp, log s and the entropy by what they are made of, whatever the logits' common offset.

    A thread adds at most V / 256 exponentials one after the other, 64 more roundings are joins, the exponential's own
    (two units) and those of the maximum's; an exponent d is rounded four times, which a sum weighted by the
    probabilities counts at most log V + 1 of.  logp rounds its difference of logits four times; the entropy's second sum is of
    terms d p, each as far off, and d itself adds up to log V + 1."""
    T, V = x.shape
    z = ref.double(x)
    unit, log_v = 2.0 ** -24, math.log(V) + 1
    m = z.max(1).values
    d = (z - m[:, None]) * scale
    log_s = torch.log(torch.exp(d).sum(1))
    sums = unit * (V / 256 + 64 + 4 * log_v + 2 * log_s)
    assert torch.equal(out["stats"][:, 0].cpu().double(), m)
    off = (out["stats"][:, 1].cpu().double() - log_s).abs()
    assert bool((off <= sums).all()), ("log s", off / unit, sums / unit)
    scored = (y >= 0) & (y < V)
    gap = d[torch.arange(T), torch.where(scored, y, 0).cpu()]
    want = torch.where(scored.cpu(), gap - log_s, torch.zeros_like(gap))
    got = out["logp"].cpu().double()
    far = want == -INF
    assert torch.equal(got[far], want[far])
    off = (got - want)[~far].abs()
    assert bool((off <= (sums + unit * (4 * gap.abs() + 2 * want.abs()))[~far]).all()), ("logp", off / unit)
    p = torch.exp(d - log_s[:, None])
    H = -torch.where(p > 0, p * (d - log_s[:, None]), torch.zeros_like(p)).sum(1)
    off = (out["entropy"].cpu().double() - H).abs()
    assert bool((off <= sums * (2 + 2 * log_v)).all()), ("entropy", off / unit)


def run_and_check_sums(x, y, scale=1.0, keep=None):
    keep = torch.arange(x.shape[0]) if keep is None else keep
    for top in (0, 8):
        out = base.run_logprobs(x, y, min(top, x.shape[1]), scale)
        check_sums(x[keep], y[keep], {n: v[keep] for n, v in out.items()}, scale)
    # without the entropy the sums are others
    got = {"logp": torch.full((x.shape[0],), NAN, device=DEV), "stats": torch.full((x.shape[0], 2), NAN, device=DEV)}
    ops.detonation_token_logprobs(x, y, logit_scale=scale, **got,
                                  workspace=scratch(ops.token_logprobs_workspace(*x.shape, 0)))
    check_sums(x[keep], y[keep], {n: v[keep] for n, v in got.items()} | {"entropy": out["entropy"][keep]}, scale)
    return out


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("offset", [0.0, 1e3, -1e3, 1e4, -1e5])
@pytest.mark.parametrize("T,V", [(3, 70001), (3, 200003), (520, 50001)])
def test_sums_of_logits_with_a_common_offset(gpu, dtype, offset, T, V):
    """Rows of many steps a lane, whose maxima a lane has seen long before the row's end."""
    if dtype == F16:
        offset = max(offset, -5e4)               # within its range
    say(dtype, offset, T, V)
    g = torch.Generator(device=DEV).manual_seed(V)
    x = (torch.randn((T, V), generator=g, device=DEV) * 2 + offset).to(dtype)
    y = torch.randint(-1, V, (T,), generator=g, device=DEV)
    run_and_check_sums(x, y, 1.0, torch.arange(0, T, max(1, T // 16)))
