"""Plain definitions, in 64 bits on the host, of the operators in include/detonation_model.h, and how far a
kernel may be from them.  Inputs are torch tensors of any type; results are float64."""
from __future__ import annotations

import math

import numpy as np
import torch

F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16
UNIT = {F32: 2.0 ** -24, BF16: 2.0 ** -8, F16: 2.0 ** -11}      # half a unit in the last place of 1
TINY = {F32: 0.0, BF16: 0.0, F16: 2.0 ** -25}                   # the same below the normal range


def double(t):
    return None if t is None else t.detach().cpu().double()


def assert_near(got, want, mag, steps, what=""):
    """got is `want` computed in fp32 from terms of magnitude `mag` in `steps` roundings, at worst all in
    one direction, and rounded once to its own type."""
    dtype = got.dtype
    got = got.detach().cpu().double()
    assert got.shape == want.shape, (what, got.shape, want.shape)
    # what lies past the type's largest value by half a unit or more is an infinity in it
    top = torch.finfo(dtype).max * (1 + UNIT[dtype] / 2)
    want = torch.where(want.abs() >= top, torch.copysign(torch.full_like(want, math.inf), want), want)
    odd = ~torch.isfinite(want)
    assert torch.equal(torch.isnan(got), torch.isnan(want)), what
    inf = odd & ~torch.isnan(want)
    assert torch.equal(got[inf], want[inf]), what
    mag = torch.as_tensor(mag, dtype=torch.float64).expand(want.shape)
    bound = UNIT[dtype] * (want.abs() + steps * 2.0 ** -24 * mag) + TINY[dtype] \
        + steps * 2.0 ** -24 * mag + 1e-37
    off = ((got - want).abs() - bound)[~odd]
    if off.numel() and float(off.max()) > 0:
        at = int(torch.argmax(off))
        raise AssertionError(f"{what}: {got[~odd].flatten()[at]} is not {want[~odd].flatten()[at]} "
                             f"to {bound[~odd].flatten()[at]}")


# ------------------------------------------------------------------ 8 bits

def act8(x):
    """(codes, exponent bytes, values) of x in 8 bits, by the format's definition."""
    x = double(x)
    T, D = x.shape
    G = -(-D // 32)
    codes = torch.zeros((T, G * 32), dtype=torch.int64)
    exps = torch.zeros((T, G), dtype=torch.int64)
    for t in range(T):
        for g in range(G):
            v = x[t, 32 * g:32 * (g + 1)]
            if not bool(torch.isfinite(v).all()):
                exps[t, g] = 255
                continue
            top = float(v.abs().max()) if v.numel() else 0.0
            e = -126
            if top > 0:
                e = max(-126, math.frexp(top)[1] - 9)       # at most the one that is looked for
                while abs(round(math.ldexp(top, -e))) > 127:    # (round: ties to even)
                    e += 1
            exps[t, g] = e + 127
            codes[t, 32 * g:32 * g + v.numel()] = torch.round(v * 2.0 ** -e).long()
    codes = codes[:, :D]
    return codes, exps, act8_values(codes, exps)


def act8_values(codes, exps):
    D = codes.shape[1]
    e = exps.long().cpu()
    scale = torch.where(e == 255, torch.full(e.shape, float("nan"), dtype=torch.float64),
                        torch.exp2((e - 127).double()))
    scale = torch.where(e == 0, torch.zeros_like(scale), scale)
    return codes.cpu().double() * scale.repeat_interleave(32, 1)[:, :D]


def act(x, kind):
    """act(x) by name"""
    if kind == "relu":
        return torch.where(x > 0, x, torch.zeros_like(x))
    if kind == "silu":
        return x * torch.sigmoid(x)
    if kind == "gelu":
        return x * 0.5 * (1 + torch.erf(x / math.sqrt(2)))
    return 0.5 * x * (1 + torch.tanh(math.sqrt(2 / math.pi) * (x + 0.044715 * x ** 3)))


def act_slope(x, kind):
    if kind == "relu":
        return (x > 0).double()
    if kind == "silu":
        s = torch.sigmoid(x)
        return s * (1 + x * (1 - s))
    if kind == "gelu":
        return 0.5 * (1 + torch.erf(x / math.sqrt(2))) + x * torch.exp(-x * x / 2) / math.sqrt(2 * math.pi)
    c = math.sqrt(2 / math.pi)
    t = torch.tanh(c * (x + 0.044715 * x ** 3))
    return 0.5 * (1 + t) + 0.5 * x * (1 - t * t) * c * (1 + 3 * 0.044715 * x * x)


# ------------------------------------------------------------------ log probabilities

def logprobs(logits, targets, scale=1.0, top=0):
    """logp, lse, entropy, top_idx, top_logp"""
    z = double(logits) * scale
    T, V = z.shape
    none = (double(logits) == -math.inf).all(1)
    m = z.max(1, keepdim=True).values
    m = torch.where(none[:, None], torch.zeros_like(m), m)
    d = z - m
    s = torch.exp(d).sum(1, keepdim=True)
    logs = d - torch.log(s)                 # of all probabilities
    lse = torch.where(none, torch.full((T,), -math.inf, dtype=torch.float64), (m + torch.log(s))[:, 0])
    y = targets.cpu().long()
    scored = (y >= 0) & (y < V)
    picked = logs[torch.arange(T), torch.where(scored, y, 0)]
    picked = torch.where(none, torch.full_like(picked, -math.inf), picked)
    logp = torch.where(scored, picked, torch.zeros_like(picked))
    p = torch.exp(logs)
    terms = torch.where(p == 0, torch.zeros_like(p), p * logs)
    entropy = torch.where(none, torch.zeros_like(lse), -terms.sum(1))
    idx = torch.zeros((T, top), dtype=torch.int64)
    best = torch.zeros((T, top), dtype=torch.float64)
    raw = double(logits)
    for t in range(T if top else 0):
        v, odd = raw[t].numpy(), torch.isnan(raw[t]).numpy()
        order = np.lexsort((np.arange(V), -np.where(odd, 0.0, v), ~odd))[:top].tolist()
        idx[t] = torch.tensor(order, dtype=torch.int64)
        for i, v in enumerate(order):
            best[t, i] = -math.inf if raw[t, v] == -math.inf and not math.isnan(float(s[t])) \
                else logs[t, v]
    return logp, lse, entropy, idx, best


def logprobs_grad(logits, targets, g_logp, g_entropy, scale=1.0):
    z = double(logits) * scale
    T, V = z.shape
    none = (double(logits) == -math.inf).all(1)
    logs = torch.log_softmax(torch.where(none[:, None], torch.zeros_like(z), z), 1)
    p = torch.exp(logs)
    y = targets.cpu().long()
    scored = (y >= 0) & (y < V)
    out = torch.zeros_like(z)
    if g_logp is not None:
        g = torch.where(scored, double(g_logp), torch.zeros(T, dtype=torch.float64))[:, None]
        out = out - g * p
        out[torch.arange(T), torch.where(scored, y, 0)] += g[:, 0]
    if g_entropy is not None:
        l = torch.where(p == 0, torch.zeros_like(p), logs)
        H = -(p * l).sum(1, keepdim=True)
        out = out - double(g_entropy)[:, None] * p * (l + H)
    return torch.where(none[:, None], torch.zeros_like(out), out * scale)


# ------------------------------------------------------------------ norm, gate, residual

def norm(x, kind, w, b, eps):
    if kind == "none":
        return x
    if kind == "layer":
        x = x - x.mean(1, keepdim=True)
    y = x / torch.sqrt((x * x).mean(1, keepdim=True) + eps)
    if w is not None:
        y = y * w
    return y if b is None else y + b


def block(x, f, pre, post, eps_pre, eps_post, scale, rows_per_gate, p):
    """(x_out, y) as float64 functions of float64 tensors; p: parameters by name."""
    if f is not None:
        u = norm(f, post, p.get("w_post"), p.get("b_post"), eps_post)
        if p.get("gate") is not None:
            rows = torch.arange(x.shape[0]) // (rows_per_gate or max(1, x.shape[0]))
            u = u * p["gate"][rows]
        x = x + scale * u
    return x, norm(x, pre, p.get("w_pre"), p.get("b_pre"), eps_pre)
