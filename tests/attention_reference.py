"""Plain definitions, in 64 bits on the host, of rotary positions, attention and dropout in
include/detonation_model.h, and how far a kernel may be from those of attention."""
from __future__ import annotations

import math

import torch

from tests.model_reference import F16, UNIT, double

FINE = 2.0 ** -24               # half a unit of fp32


# ------------------------------------------------------------------ rotary positions

def rotary(x, positions, freqs, heads, head_dim, rotary_dim, layout, inverse=False, magnitude=1.0):
    """A pair at a time, as the header says it."""
    x = double(x).reshape(x.shape[0], heads, head_dim)
    out = x.clone()
    w = double(positions)[:, None] * double(freqs) * (-1 if inverse else 1)
    for i in range(rotary_dim // 2):
        a, b = (i, i + rotary_dim // 2) if layout == "halves" else (2 * i, 2 * i + 1)
        cos, sin = torch.cos(w[:, i, None]), torch.sin(w[:, i, None])
        out[:, :, a] = magnitude * (x[:, :, a] * cos - x[:, :, b] * sin)
        out[:, :, b] = magnitude * (x[:, :, a] * sin + x[:, :, b] * cos)
    return out.reshape(x.shape[0], -1)


# ------------------------------------------------------------------ dropout

def philox(counter, key):
    """Four words of 32 bits, from whole numbers of any size."""
    c, k = list(counter), list(key)
    for _ in range(10):
        p, r = c[0] * 0xD2511F53, c[2] * 0xCD9E8D57
        c = [(r >> 32) ^ c[1] ^ k[0], r % 2 ** 32, (p >> 32) ^ c[3] ^ k[1], p % 2 ** 32]
        k = [(k[0] + 0x9E3779B9) % 2 ** 32, (k[1] + 0xBB67AE85) % 2 ** 32]
    return c


def kept(T, D, rate, seed, offset):
    """Which elements stay, and what they are multiplied with."""
    n = min(65535, round(float(torch.tensor(rate, dtype=torch.float32)) * 65536))
    offset %= 2 ** 64
    keep = torch.zeros((T, -(-D // 8) * 8), dtype=torch.bool)
    for t in range(T):
        for g in range(-(-D // 8)):
            words = philox((g, t, offset % 2 ** 32, offset >> 32), (seed % 2 ** 32, seed >> 32))
            for j in range(8):
                keep[t, 8 * g + j] = (words[j // 2] >> (16 * (j % 2))) % 65536 >= n
    return keep[:, :D], 65536 / (65536 - n)


# ------------------------------------------------------------------ attention

def sequences(starts_q, starts_k):
    return [(slice(a, b), slice(c, d)) for a, b, c, d in zip(starts_q, starts_q[1:], starts_k, starts_k[1:])]


def attention(q, k, v, out, lse, dout, heads, kv_heads, head_dim, scale, causal, starts_q, starts_k):
    """{name: (value, bound)} of out, lse and, where dout is given, dq, dk and dv.  Bounds count each rounding at its
    worst: products of head_dim terms and sums over a row or column in fp32, weights and their gradients rounded to
    the matrices' type (u) before the second product, results rounded to it.  The gradients take `out` and `lse` as
    they were written, which are off by their own bounds."""
    dtype = q.dtype
    u, low = UNIT[dtype], 2.0 ** -25 if dtype == F16 else 0.0        # `low`: what a weight below the normal range loses
    q, k, v, dout = (double(t) for t in (q, k, v, dout))
    D, group = head_dim, heads // kv_heads
    names = ["out", "lse"] + ([] if dout is None else ["dq", "dk", "dv"])
    shape = {"out": q.shape, "lse": (heads, len(q)), "dq": q.shape, "dk": k.shape, "dv": k.shape}
    want = {n: torch.full(shape[n], math.nan, dtype=torch.float64) for n in names}      # NaN: not written
    off = {n: torch.zeros(shape[n], dtype=torch.float64) for n in names}
    for sq, sk in sequences(starts_q, starts_k):
        nq, nk = sq.stop - sq.start, sk.stop - sk.start
        for n in names:
            rows = sk if n in ("dk", "dv") else sq
            if n == "lse":
                want[n][:, sq] = 0
            else:
                want[n][rows] = 0
        sees = torch.ones((nq, nk), dtype=torch.bool)
        if causal:
            sees = torch.arange(nk)[None] <= torch.arange(nq)[:, None] + nk - nq
        for h in range(heads):
            cq, ck = slice(h * D, (h + 1) * D), slice(h // group * D, (h // group + 1) * D)
            x, y, z = q[sq, cq], k[sk, ck], v[sk, ck]
            s = torch.where(sees, scale * (x @ y.t()), -math.inf)
            size = torch.where(sees, scale * (x.abs() @ y.abs().t()), 0.0)
            top = s.amax(1, keepdim=True) if nk else torch.full((nq, 1), -math.inf, dtype=torch.float64)
            empty = top == -math.inf
            e = torch.exp(s - torch.where(empty, 0.0, top))
            total = e.sum(1, keepdim=True)
            p = e / torch.where(empty, 1.0, total)
            log_sum = torch.where(empty, -math.inf, top + torch.log(total))
            # a score's error (its product, the factor, the difference to the maximum), and a row's largest
            ds = (D + 4) * FINE * size + 4 * FINE * torch.where(sees, s.abs(), 0.0)
            worst = ds.amax(1, keepdim=True) + 4 * FINE * torch.where(empty, 0.0, top.abs()) if nk else ds.sum(1, keepdim=True)
            steps = (nk / 32 + 40) * FINE                            # of a row's sums, and of the exponentials
            want["lse"][h, sq] = log_sum[:, 0]
            off["lse"][h, sq] = torch.where(empty, 0.0, worst + steps + 2 * FINE * log_sum.abs())[:, 0]
            o = p @ z
            want["out"][sq, cq] = o
            err = (p @ z.abs()) * (u + 2 * worst + 2 * steps) + low * z.abs().sum(0)
            off["out"][sq, cq] = err + u * o.abs() + low
            if dout is None:
                continue
            g = dout[sq, cq]
            dp, dp_size = g @ z.t(), g.abs() @ z.abs().t()
            delta = (g * o).sum(1, keepdim=True)
            err_delta = (g.abs() * (off["out"][sq, cq] + (D + 4) * FINE * o.abs())).sum(1, keepdim=True)
            # lse's own error, and a weight's beside it
            err_p = 2 * worst + 2 * steps + 4 * FINE * torch.where(empty, 0.0, log_sum).abs()
            d = p * (dp - delta)
            err_d = p * (err_p * (dp - delta).abs() + (D + 4) * FINE * dp_size + err_delta)
            err_d = err_d + u * (d.abs() + err_d) + low * sees
            long = (max(nq, nk) * group / 32 + 40) * FINE
            dq, dk, dv = scale * d @ y, scale * d.t() @ x, p.t() @ g
            want["dq"][sq, cq] = dq
            off["dq"][sq, cq] = scale * (err_d + long * d.abs()) @ y.abs() + u * dq.abs() + low
            want["dk"][sk, ck] += dk
            off["dk"][sk, ck] += scale * (err_d + long * d.abs()).t() @ x.abs()
            want["dv"][sk, ck] += dv
            off["dv"][sk, ck] += (p * (u + err_p + long) + low * sees).t() @ g.abs()
    for n in ("dk", "dv"):
        if n in names:
            off[n] += u * (torch.nan_to_num(want[n]).abs() + off[n]) + low
    return {n: (want[n], 1.001 * off[n] + 1e-30) for n in names}


def assert_within(got, want, bound, what):
    """Elements whose wanted value is a NaN were not to be written: the caller filled them with NaN."""
    got = double(got)
    assert got.shape == want.shape, (what, got.shape, want.shape)
    kept_out = torch.isnan(want)
    assert bool(torch.isnan(got[kept_out]).all()), f"{what}: rows of no sequence were written"
    infinite = torch.isinf(want)
    assert torch.equal(got[infinite], want[infinite]), f"{what}: infinities"
    there = ~kept_out & ~infinite
    off = (got - want)[there].abs() - bound[there]
    assert not bool(torch.isnan(off).any()), f"{what}: NaN"
    if off.numel() and float(off.max()) > 0:
        at = int(torch.argmax(off))
        raise AssertionError(f"{what}: {got[there][at]} is not {want[there][at]} to {bound[there][at]} "
                             f"(element {int(torch.nonzero(there.flatten())[at])} of {tuple(got.shape)})")


def whole(q, k, v, dout, heads, kv_heads, scale, causal, sequences):
    """out, dq, dk and dv of sequences of equal length, all heads at once in 64 bits where the matrices are."""
    def apart(x, n):
        return x.double().reshape(sequences, -1, n, x.shape[1] // n).transpose(1, 2)

    def together(x):
        return x.transpose(1, 2).reshape(sequences * x.shape[2], -1)

    group = heads // kv_heads
    q, dout = apart(q, heads), apart(dout, heads)
    k, v = (apart(t, kv_heads).repeat_interleave(group, 1).contiguous() for t in (k, v))
    s = q @ k.transpose(2, 3).contiguous() * scale
    if causal:
        nq, nk = s.shape[2:]
        s.masked_fill_(torch.ones((nq, nk), dtype=torch.bool, device=s.device).triu(nk - nq + 1), -math.inf)
    p = torch.softmax(s, 3)
    out = p @ v
    ds = p * (dout @ v.transpose(2, 3).contiguous() - (dout * out).sum(3, keepdim=True))
    dk, dv = ds.transpose(2, 3).contiguous() @ q * scale, p.transpose(2, 3).contiguous() @ dout
    dk, dv = (t.unflatten(1, (kv_heads, group)).sum(2) for t in (dk, dv))
    return {"out": together(out), "dq": together(ds @ k * scale), "dk": together(dk), "dv": together(dv)}
