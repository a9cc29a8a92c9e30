"""The example's training step: its gradient against torch's own differentiation of the same model, and its loss."""
import importlib.util
import os

import pytest
import torch

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def load():
    spec = importlib.util.spec_from_file_location("train_residual_lm",
                                                  os.path.join(ROOT, "examples", "train_residual_lm.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


def plain_loss(ex, p, tokens, targets):
    """The model by elementary operations in 64 bits on the host."""
    def rms(x, w):
        return x / torch.sqrt((x * x).mean(1, keepdim=True) + 1e-6) * w
    x = p["embed"][tokens]
    y = rms(x, p["norm0"])
    for i in range(ex.BLOCKS):
        ab = y @ p[f"up{i}"].t()
        h = torch.nn.functional.silu(ab[:, :ex.HIDDEN]) * ab[:, ex.HIDDEN:]
        x = x + p[f"gate{i}"] * rms(h @ p[f"down{i}"].t(), p[f"post{i}"])
        y = rms(x, p[f"norm{i + 1}"])
    logp = torch.log_softmax(y @ p["out"].t(), 1)
    return -logp[torch.arange(len(targets)), targets].mean()


def test_gradient(gpu):
    ex = load()
    model = ex.Model(gpu)
    tokens, targets = next(ex.batches(gpu, 1))
    loss = model.forward(tokens, targets)
    model.backward(tokens, targets)
    p = {n: v.detach().cpu().double().requires_grad_() for n, v in model.p.items()}
    want = plain_loss(ex, p, tokens.cpu(), targets.cpu())
    want.backward()
    # products of bf16 (2^-8) and activations in 8 bits (2^-8 of a group's largest), over a few layers
    assert abs(float(loss) - float(want)) < 0.02
    for n, v in p.items():
        g, w = model.g[n].detach().cpu().double(), v.grad
        assert float((g - w).norm() / w.norm()) < 0.04, n


def test_loss_falls(gpu):
    losses = load().train(60, report=lambda line: print(line, flush=True))
    assert losses[0] > 5.5 and losses[-1] < 0.5 * losses[0]
