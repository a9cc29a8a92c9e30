"""The kernels behind include/detonation_model.h where their arithmetic has few bits to spare: widths that leave
lanes empty, values at the ends of a type's range, sums of many steps.  Plain definitions in 64 bits."""
import math

import pytest
import torch

from paper_2502_06728_amd import model_ops as ops
from tests import model_reference as ref
from tests import test_gpu_model_ops as base
from tests.model_reference import BF16, F16, F32, assert_near
from tests.test_gpu_model_ops import ACT, DEV, INF, NAN, TYPES, act8_of, empty_act8, like, normal, rows, say, scratch

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
