"""A small language model trained with this framework's kernels around the library products: norms, gated
activations and the loss from model_ops, activations kept in 8 bits between the two passes, weight gradients
straight into the flat gradient, and the optimizer step (compress, decompress-and-update) on that.

    python examples/train_residual_lm.py [--steps 60]

Residual blocks without attention, on synthetic text (a noisy map from each token to its successor): enough for
the loss to fall from log(vocabulary) towards the text's entropy.
"""
from __future__ import annotations

import argparse
import math
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

from paper_2502_06728_amd import binding, model_ops as ops  # noqa: E402

VOCAB, WIDTH, HIDDEN, BLOCKS, TOKENS = 512, 256, 640, 2, 1024


class Model:
    """Parameters and gradients are views of two flat fp32 arrays, as a sharded optimizer holds them."""

    def __init__(self, device, seed=0):
        shapes = {"embed": (VOCAB, WIDTH), "norm0": (WIDTH,), "out": (VOCAB, WIDTH)}
        for i in range(BLOCKS):
            shapes |= {f"up{i}": (2 * HIDDEN, WIDTH), f"down{i}": (WIDTH, HIDDEN), f"post{i}": (WIDTH,),
                       f"gate{i}": (1, WIDTH), f"norm{i + 1}": (WIDTH,)}
        n = sum(math.prod(s) for s in shapes.values())
        self.params = torch.empty(n, device=device)
        self.grads = torch.zeros(n, device=device)
        self.p, self.g, at = {}, {}, 0
        gen = torch.Generator(device=device).manual_seed(seed)
        for name, s in shapes.items():
            m = math.prod(s)
            self.p[name] = self.params[at:at + m].view(s)
            self.g[name] = self.grads[at:at + m].view(s)
            at += m
            if name.startswith(("embed", "out", "up", "down")):
                self.p[name].normal_(0, 1 if name == "embed" else s[-1] ** -0.5, generator=gen)
            else:
                self.p[name].fill_(0.5 if name.startswith("gate") else 1.0)
        self.first = ops.NormResidual(pre=ops.NORM_RMS)
        self.block = ops.NormResidual(pre=ops.NORM_RMS, post=ops.NORM_RMS, scale=1.0)
        T, bf16 = TOKENS, torch.bfloat16
        new = lambda *s, dtype=bf16: torch.empty(s, dtype=dtype, device=device)  # noqa: E731
        act8 = lambda d: ops.Act8.empty(T, d, device)  # noqa: E731
        # what a training step keeps from its forward to its backward pass
        self.x = [new(T, WIDTH, dtype=torch.float32) for _ in range(BLOCKS + 1)]
        self.y8 = [act8(WIDTH) for _ in range(BLOCKS + 1)]
        self.a8, self.b8 = [act8(HIDDEN) for _ in range(BLOCKS)], [act8(HIDDEN) for _ in range(BLOCKS)]
        self.f = [None] * BLOCKS
        self.stats = new(T, 2, dtype=torch.float32)
        self.logp = new(T, dtype=torch.float32)
        # scratch
        self.y, self.h, self.h8 = new(T, WIDTH), new(T, HIDDEN), act8(HIDDEN)
        self.dab = new(T, 2 * HIDDEN)
        self.dx, self.df = [new(T, WIDTH, dtype=torch.float32) for _ in range(2)], new(T, WIDTH)
        self.g_logp = torch.full((T,), -1.0 / T, device=device)
        sizes = [ops.act8_weight_grad_workspace(T, *s) for s in
                 ((VOCAB, WIDTH), (2 * HIDDEN, WIDTH), (WIDTH, HIDDEN))]
        sizes += [ops.norm_residual_workspace(self.block, T, WIDTH), ops.norm_residual_workspace(self.first, T, WIDTH),
                  ops.token_logprobs_workspace(T, VOCAB)]
        self.scratch = torch.empty(max(sizes), dtype=torch.uint8, device=device)

    def weight(self, name):
        return self.p[name].to(torch.bfloat16)

    def forward(self, tokens, targets):
        """Mean negative log probability of the targets, on the device."""
        p = self.p
        torch.index_select(p["embed"], 0, tokens, out=self.x[0])
        ops.detonation_norm_residual(self.first, self.x[0], None, None, self.y, y8=self.y8[0], w_pre=p["norm0"])
        for i in range(BLOCKS):
            ab = self.y @ self.weight(f"up{i}").t()
            ops.detonation_glu_forward(ops.ACT_SILU, ab[:, :HIDDEN], ab[:, HIDDEN:], self.h, a8=self.a8[i], b8=self.b8[i])
            self.f[i] = self.h @ self.weight(f"down{i}").t()
            ops.detonation_norm_residual(self.block, self.x[i], self.f[i], self.x[i + 1], self.y, y8=self.y8[i + 1],
                                         gate=p[f"gate{i}"], w_post=p[f"post{i}"], w_pre=p[f"norm{i + 1}"])
        self.logits = self.y @ self.weight("out").t()
        ops.detonation_token_logprobs(self.logits, targets, self.logp, stats=self.stats, workspace=self.scratch)
        return -self.logp.mean()

    def backward(self, tokens, targets):
        """Fills the flat gradient."""
        p, g, ws = self.p, self.g, self.scratch
        dz = self.logits                       # the gradient takes the logits' place
        ops.detonation_token_logprobs_backward(self.logits, targets, self.stats, dz, g_logp=self.g_logp)
        ops.detonation_act8_weight_grad(dz, self.y8[BLOCKS], g["out"], workspace=ws)
        dy, dx_out = dz @ self.weight("out"), None
        for i in reversed(range(BLOCKS)):
            dx = self.dx[i % 2]
            ops.detonation_norm_residual_backward(
                self.block, self.x[i + 1], self.f[i], dy, dx_out, dx, self.df, workspace=ws, gate=p[f"gate{i}"],
                w_post=p[f"post{i}"], w_pre=p[f"norm{i + 1}"], dgate=g[f"gate{i}"], dw_post=g[f"post{i}"],
                dw_pre=g[f"norm{i + 1}"])
            dh = self.df @ self.weight(f"down{i}")
            ops.detonation_glu_backward(ops.ACT_SILU, dh, self.a8[i], self.b8[i], self.dab[:, :HIDDEN],
                                        self.dab[:, HIDDEN:], h8=self.h8)
            ops.detonation_act8_weight_grad(self.df, self.h8, g[f"down{i}"], workspace=ws)
            ops.detonation_act8_weight_grad(self.dab, self.y8[i], g[f"up{i}"], workspace=ws)
            dy, dx_out = self.dab @ self.weight(f"up{i}"), dx
        ops.detonation_norm_residual_backward(self.first, self.x[0], None, dy, dx_out, dx_out, None, workspace=ws,
                                              w_pre=p["norm0"], dw_pre=g["norm0"])
        g["embed"].zero_().index_add_(0, tokens, dx_out)


class Optimizer:
    """One rank's step on the flat gradient: the payload that would be gathered is its own."""

    def __init__(self, model, lr=2e-3, decay=0.9):
        n = model.params.numel()
        self.model = model
        self.cfg = binding.Config(chunk=64, topk=16, sign=True, decay=decay, lr=lr)
        self.momentum = torch.zeros(n, device=model.params.device)
        entries = binding.payload_entries(self.cfg, n)
        self.idx = torch.empty(entries, dtype=torch.int32, device=model.params.device)
        self.val = torch.empty(entries, device=model.params.device)

    def step(self):
        binding.detonation_compress(self.cfg, self.model.grads, self.momentum, self.idx, self.val)
        binding.detonation_decompress_step(self.cfg, 1, self.idx, self.val, self.model.params)


def batches(device, steps, seed=1):
    """Each token is followed by a fixed other one, one time in eight by any."""
    gen = torch.Generator(device=device).manual_seed(seed)
    follows = torch.randperm(VOCAB, generator=gen, device=device)
    for _ in range(steps):
        tokens = torch.randint(0, VOCAB, (TOKENS,), generator=gen, device=device)
        noise = torch.randint(0, VOCAB, (TOKENS,), generator=gen, device=device)
        keep = torch.rand((TOKENS,), generator=gen, device=device) < 7 / 8
        yield tokens, torch.where(keep, follows[tokens], noise)


def train(steps=60, report=print):
    model = Model(torch.device("cuda:0"))
    optimizer, losses = Optimizer(model), []
    for i, (tokens, targets) in enumerate(batches(model.params.device, steps)):
        losses.append(model.forward(tokens, targets))
        model.backward(tokens, targets)
        optimizer.step()
        if i % 10 == 0 or i == steps - 1:
            report(f"step {i:4d}  loss {float(losses[-1]):.4f}")
    return [float(v) for v in losses]


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--steps", type=int, default=60)
    train(ap.parse_args().steps)
