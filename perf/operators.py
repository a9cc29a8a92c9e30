"""The operators around the library products of a training step, as cases that can be timed and checked.

A residual block and its loss, as the models that `synth` lists are made of them, and what a training
step saves in 8 bits between its forward and its backward pass:

    op        logp       log probability of each row's target, entropy and the K best tokens; with
                         `train` also the gradient of the logits
              norm_fwd   residual + scale * gate * norm(block output), and the next block's norm of it
              norm_bwd   its gradients: both inputs, the gate and the norms' weights
              glu        act(a) * b and its backward pass out of a and b held in 8 bits
              wgrad      a linear layer's weight gradient out of its input held in 8 bits
              codec      activations into 8 bits and back
    T         rows (tokens); V, D, N, K: vocabulary, features, output and input features
    dtype     f32, bf16 or f16; xdtype: the residual stream's, where it is another one
    pad       elements between the end of a row and the next row

Where `own` is false, the same is computed by elementary torch operations in 32 bits.
"""
from __future__ import annotations

import math

import torch

own = False

DTYPE = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
SIZE = {"f32": 4, "bf16": 2, "f16": 2}
GROUP = 32                    # features that share an exponent in the 8-bit form
EPS = 1e-6
IGNORED = -100                # a target that is not scored


# ------------------------------------------------------------------ cases

def _logp(name, T, V, dtype, top=0, train=False, pad=0, masked=False):
    return _named(name, dict(op="logp", T=T, V=V, dtype=dtype, top=top, train=train, pad=pad,
                             masked=masked))


def _norm(name, op, T, D, dtype, xdtype, pre="rms", post="rms", rows_per_gate=0, gate=True, pad=0,
          ckpt=False):
    return _named(name, dict(op=op, T=T, D=D, dtype=dtype, xdtype=xdtype, pre=pre, post=post,
                             rows_per_gate=rows_per_gate, gate=gate, pad=pad, ckpt=ckpt))


def _glu(name, T, D, dtype, act="silu", gated=True, pad=0):
    return _named(name, dict(op="glu", T=T, D=D, dtype=dtype, act=act, gated=gated, pad=pad))


def _wgrad(name, T, N, K, dtype, out):
    return _named(name, dict(op="wgrad", T=T, N=N, K=K, dtype=dtype, out=out))


def _codec(name, T, D, dtype, pad=0):
    return _named(name, dict(op="codec", T=T, D=D, dtype=dtype, pad=pad))


def _named(name, c):
    return dict(name=name, **c) if name else c


def listed():
    return [
        # sampling one token of a language model: its probability, the row's entropy, the eight best
        _logp("logp_1x50304", 1, 50304, "bf16", top=8),
        # loss of a training step of the 1B language model, with an entropy bonus
        _logp("logp_train_8192x50304", 8192, 50304, "bf16", train=True),
        # scoring given text: a vocabulary of no round size, its last entries masked, padded rows
        _logp("logp_1021x32101_top20", 1021, 32101, "f16", top=20, pad=27, masked=True),
        # one token through a block's norms
        _norm("norm_fwd_1x2048", "norm_fwd", 1, 2048, "bf16", "bf16"),
        # a training step's tokens: fp32 residual stream, the norm's output also saved in 8 bits
        _norm("norm_fwd_16384x2048", "norm_fwd", 16384, 2048, "bf16", "f32", ckpt=True),
        # and the same tokens backward
        _norm("norm_bwd_16384x2048", "norm_bwd", 16384, 2048, "bf16", "f32"),
        # an image model's layer norm with a gate per image (197 patches), no round width
        _norm("norm_bwd_1379x771", "norm_bwd", 1379, 771, "f16", "f16", pre="layer", post="none",
              rows_per_gate=197, pad=5),
        # the 1B language model's feed-forward activation, forward and backward
        _glu("glu_8192x8192", 8192, 8192, "bf16"),
        # an image model's: GELU without a gate, few rows
        _glu("glu_197x771_gelu", 197, 771, "f32", act="gelu", gated=False),
        # weight gradient of the 1B language model's projection out of the feed-forward layer
        _wgrad("wgrad_8192x2048x8192", 8192, 2048, 8192, "bf16", "f32"),
        # a small layer's, ragged everywhere, in fp32
        _wgrad("wgrad_1021x770x519", 1021, 770, 519, "f32", "f32"),
        # activations of the translation model into 8 bits and back
        _codec("codec_16384x768", 16384, 768, "bf16"),
    ]


def _spread(rng, lo, hi):
    """A whole number between lo and hi, uniform over the logarithm, odd as often as even."""
    n = int(math.exp(rng.uniform(math.log(lo), math.log(hi + 1))))
    return max(lo, min(hi, n ^ rng.randint(0, 1)))


def draw(rng):
    """One more case of the same ranges."""
    op = rng.choice(["logp", "logp", "norm_fwd", "norm_bwd", "glu", "wgrad", "codec"])
    dtype = rng.choice(["bf16", "bf16", "f16", "f32"])
    pad = rng.choice([0, 0, rng.randint(1, 64)])
    if op == "logp":
        V = _spread(rng, 1000, 50304)
        top = rng.choice([0, rng.randint(1, 32)])
        T = _spread(rng, 1, min(8192, int(3e8 / V)) if not top else min(2048, int(6e7 / V)))
        return _logp(None, T, V, dtype, top, rng.random() < 0.5, pad, rng.random() < 0.3)
    if op in ("norm_fwd", "norm_bwd"):
        D = _spread(rng, 64, 8192)
        T = _spread(rng, 1, int(3e7 / D))
        kinds = [rng.choice(["rms", "layer", "none"]) for _ in range(2)]
        if kinds == ["none", "none"]:
            kinds = ["rms", "rms"]
        rows = rng.choice([0, 0, _spread(rng, 1, max(1, T))])
        return _norm(None, op, T, D, dtype, rng.choice([dtype, "f32"]), *kinds, rows,
                     rows > 0 or rng.random() < 0.5, pad,
                     op == "norm_fwd" and kinds[0] != "none" and rng.random() < 0.3)
    if op == "glu":
        D = _spread(rng, 64, 11008)
        return _glu(None, _spread(rng, 1, int(6e7 / D)), D, dtype,
                    rng.choice(["silu", "gelu", "gelu_tanh", "relu"]), rng.random() < 0.6, pad)
    if op == "wgrad":
        N, K = _spread(rng, 64, 8192), _spread(rng, 64, 8192)
        return _wgrad(None, _spread(rng, 16, min(8192, int(1.3e11 / (N * K)))), N, K, dtype,
                      rng.choice(["f32", "f32", "bf16"]))
    D = _spread(rng, 64, 8192)
    return _codec(None, _spread(rng, 1, int(6e7 / D)), D, dtype, pad)


def work(case):
    T, e, op = case["T"], SIZE[case["dtype"]], case["op"]
    if op == "logp":
        n = T * case["V"]
        return {"bytes": n * e * (2 if case["train"] else 1) + T * (20 + 8 * case["top"]),
                "flops": n * (9 if case["train"] else 5)}
    if op == "norm_fwd":
        ex, D = SIZE[case["xdtype"]], case["D"]
        y = 0 if case["pre"] == "none" else e + (33 / 32 if case["ckpt"] else 0)
        gates = _gates(case) * D * 4
        return {"bytes": T * D * (2 * ex + e + y) + gates + 4 * D * 4, "flops": T * D * 12}
    if op == "norm_bwd":
        ex, D = SIZE[case["xdtype"]], case["D"]
        y = 0 if case["pre"] == "none" else e
        return {"bytes": T * D * (3 * ex + 2 * e + y) + 2 * _gates(case) * D * 4 + 8 * D * 4,
                "flops": T * D * 30}
    if op == "glu":
        n, ins = T * case["D"], 2 if case["gated"] else 1
        return {"bytes": n * e * (2 * ins + 2), "flops": n * 30}
    if op == "wgrad":
        N, K = case["N"], case["K"]
        return {"bytes": T * N * e + T * K * 33 / 32 + N * K * SIZE[case["out"]],
                "flops": 2 * T * N * K}
    return {"bytes": 2 * T * case["D"] * e, "flops": 3 * T * case["D"]}


def _gates(case):
    if not case["gate"]:
        return 0
    return -(-case["T"] // case["rows_per_gate"]) if case["rows_per_gate"] else 1


# ------------------------------------------------------------------ inputs

def _rows(T, D, dtype, pad, dev, fill=None):
    """[T, D] whose rows lie `pad` elements further apart than their length."""
    t = torch.empty((T, D + pad), dtype=dtype, device=dev)[:, :D]
    if fill is not None:
        t.copy_(fill)
    return t


def _activations(g, T, D, dev):
    """Normal values, a few features of every row much larger than the others (as activations of
    trained models have them)."""
    x = torch.randn((T, D), generator=g, device=dev)
    big = torch.rand((D,), generator=g, device=dev) < 0.01
    return x * torch.where(big, 20.0, 1.0)


def _inputs(case, seed, dev):
    g = torch.Generator(device=dev).manual_seed(seed)
    T, dt, op = case["T"], DTYPE[case["dtype"]], case["op"]
    s = {"case": case}
    if op == "logp":
        V = case["V"]
        s["targets"] = torch.randint(0, V, (T,), generator=g, device=dev)
        z = _rows(T, V, dt, case["pad"], dev)
        at = torch.arange(T, device=dev)
        for lo in range(0, T, 1024):      # a block of rows at a time: the logits are large
            hi = min(T, lo + 1024)
            z[lo:hi] = torch.randn((hi - lo, V), generator=g, device=dev) * 2.5
        z[at, s["targets"]] += (torch.rand((T,), generator=g, device=dev) * 14).to(dt)
        if case["masked"]:
            z[:, V - V // 16:] = -math.inf
            s["targets"].clamp_(max=V - V // 16 - 1)
        s["targets"][torch.rand((T,), generator=g, device=dev) < 0.05] = IGNORED
        s["logits"] = z
        if case["train"]:
            s["g_logp"] = -torch.rand((T,), generator=g, device=dev)
            s["g_entropy"] = torch.randn((T,), generator=g, device=dev) * 0.01
            s["dlogits"] = _rows(T, V, dt, case["pad"], dev)
        for name in ("logp", "lse", "entropy"):
            s[name] = torch.empty((T,), device=dev)
        s["stats"] = torch.empty((T, 2), device=dev)
        if case["top"]:
            s["top_idx"] = torch.empty((T, case["top"]), dtype=torch.int32, device=dev)
            s["top_logp"] = torch.empty((T, case["top"]), device=dev)
    elif op in ("norm_fwd", "norm_bwd"):
        D, xt, pad = case["D"], DTYPE[case["xdtype"]], case["pad"]
        s["x"] = _rows(T, D, xt, pad, dev, _activations(g, T, D, dev) * 2)
        s["f"] = _rows(T, D, dt, pad, dev, torch.randn((T, D), generator=g, device=dev) * 0.7)
        for name, kind in (("post", case["post"]), ("pre", case["pre"])):
            if kind != "none":
                s["w_" + name] = 1 + 0.2 * torch.randn((D,), generator=g, device=dev)
            if kind == "layer":
                s["b_" + name] = 0.1 * torch.randn((D,), generator=g, device=dev)
        if case["gate"]:
            s["gate"] = 0.5 + 0.3 * torch.randn((_gates(case), D), generator=g, device=dev)
        if op == "norm_fwd":
            s["x_out"] = _rows(T, D, xt, pad, dev)
            if case["pre"] != "none":
                s["y"] = _rows(T, D, dt, pad, dev)
            if case["ckpt"]:
                s.update(_codes(T, D, dev, "y"))
                s["y_back"] = torch.empty((T, D), dtype=torch.bfloat16, device=dev)
        else:
            if case["pre"] != "none":
                s["dy"] = _rows(T, D, dt, pad, dev, torch.randn((T, D), generator=g, device=dev))
            s["dx_out"] = _rows(T, D, xt, pad, dev, torch.randn((T, D), generator=g, device=dev))
            s["dx"], s["df"] = _rows(T, D, xt, pad, dev), _rows(T, D, dt, pad, dev)
            for name in [n for n in s if n in ("gate", "w_post", "b_post", "w_pre", "b_pre")]:
                s["d" + name] = torch.empty(s[name].shape, device=dev)
    elif op == "glu":
        D, pad = case["D"], case["pad"]
        for name, grad in [("a", "da"), ("b", "db")] if case["gated"] else [("a", "da")]:
            s[name] = _rows(T, D, dt, pad, dev, _activations(g, T, D, dev))
            s[grad] = _rows(T, D, dt, pad, dev)
            s.update(_codes(T, D, dev, name))
        s["dh"] = _rows(T, D, dt, pad, dev, torch.randn((T, D), generator=g, device=dev))
        s["h"] = _rows(T, D, dt, pad, dev)
    elif op == "wgrad":
        N, K = case["N"], case["K"]
        s["dy"] = (torch.randn((T, N), generator=g, device=dev) * 0.1).to(dt)
        s["x_codes"], s["x_exps"] = _encode(_activations(g, T, K, dev))
        s["dw"] = torch.empty((N, K), dtype=DTYPE[case["out"]], device=dev)
    else:
        D = case["D"]
        s["x"] = _rows(T, D, dt, case["pad"], dev, _activations(g, T, D, dev))
        s.update(_codes(T, D, dev, "x"))
        s["back"] = _rows(T, D, dt, case["pad"], dev)
    return s


def _codes(T, D, dev, name):
    return {name + "_codes": torch.empty((T, D), dtype=torch.int8, device=dev),
            name + "_exps": torch.empty((T, -(-D // GROUP)), dtype=torch.uint8, device=dev)}


def prepare(case, seed):
    return _inputs(case, seed, torch.device("cuda:0"))


# ------------------------------------------------------------------ plain forms, 32 bits

def _pow2(e):
    """2**e as fp32, e an int32 tensor between -126 and 127."""
    return ((e + 127) << 23).view(torch.float32)


def _grouped(x):
    T, D = x.shape
    short = -D % GROUP
    x = torch.cat([x, x.new_zeros((T, short))], 1) if short else x
    return x.reshape(T, -1, GROUP)


def _exponents(x):
    """Per group of 32 features the smallest exponent at which every code is within 127."""
    m, e = torch.frexp(_grouped(x).abs().amax(2))
    return (e - 7 + (m * 128 >= 127.5)).clamp(min=-126).to(torch.int32)


def _encode(x):
    e = _exponents(x)
    q = torch.round(_grouped(x) * _pow2(-e)[:, :, None]).to(torch.int8)
    return (q.reshape(x.shape[0], -1)[:, :x.shape[1]].contiguous(), (e + 127).to(torch.uint8))


def _decode(codes, exps):
    scale = _pow2(exps.to(torch.int32) - 127).repeat_interleave(GROUP, 1)[:, :codes.shape[1]]
    return codes.float() * scale


def _plain_logp(s):
    z = s["logits"].float()
    m = z.amax(1, keepdim=True)
    d = z - m
    e = torch.exp(d)
    total = e.sum(1, keepdim=True)
    lse = (m + torch.log(total))[:, 0]
    p = e / total
    scored = (s["targets"] >= 0) & (s["targets"] < z.shape[1])
    at = s["targets"].clamp(min=0, max=z.shape[1] - 1)
    logp = torch.where(scored, z.gather(1, at[:, None])[:, 0] - lse, 0.0)
    entropy = torch.log(total[:, 0]) - torch.where(p > 0, p * d, 0.0).sum(1)
    out = {"logp": logp, "lse": lse, "entropy": entropy}
    K = s["case"]["top"]
    if K:
        v, i = torch.sort(z, dim=1, descending=True, stable=True)
        out["top_idx"], out["top_logp"] = i[:, :K].to(torch.int32), v[:, :K] - lse[:, None]
    if s["case"]["train"]:
        g = torch.where(scored, s["g_logp"], 0.0)
        h = torch.where(p > 0, d - torch.log(total) + entropy[:, None], 0.0)
        dz = -p * (g[:, None] + s["g_entropy"][:, None] * h)
        dz.scatter_add_(1, at[:, None], g[:, None])
        out["dlogits"] = dz.to(s["logits"].dtype)
    return out


def _plain_stats(x, kind):
    """What a norm subtracts from a row, and what it multiplies with."""
    mean = x.mean(1, keepdim=True) if kind == "layer" else torch.zeros_like(x[:, :1])
    d = x - mean
    return mean, torch.rsqrt((d * d).mean(1, keepdim=True) + EPS)


def _plain_norm(x, kind, w, b):
    if kind == "none":
        return x
    mean, r = _plain_stats(x, kind)
    y = (x - mean) * r * w
    return y if b is None else y + b


def _gate_rows(s):
    """The gate, a row for each token or one for all."""
    if "gate" not in s:
        return torch.ones((1, 1), device=s["x"].device)
    rows = s["case"]["rows_per_gate"]
    return s["gate"].repeat_interleave(rows, 0)[:s["case"]["T"]] if rows else s["gate"]


SCALE = 0.8                   # of the branch


def _plain_norm_fwd(s):
    c = s["case"]
    u = _plain_norm(s["f"].float(), c["post"], s.get("w_post"), s.get("b_post"))
    x = s["x"].float() + SCALE * _gate_rows(s) * u
    out = {"x_out": x.to(s["x"].dtype)}
    if c["pre"] != "none":
        y = _plain_norm(x, c["pre"], s["w_pre"], s.get("b_pre"))
        out["y"] = y.to(s["f"].dtype)
        if c["ckpt"]:
            out["y_back"] = _decode(*_encode(y)).to(torch.bfloat16)
    return out


def _plain_norm_grad(x, kind, w, dy):
    """(gradient of the norm's input, x normalised)"""
    mean, r = _plain_stats(x, kind)
    n = (x - mean) * r
    a = dy * w
    dx = a - n * (a * n).mean(1, keepdim=True)
    if kind == "layer":
        dx = dx - a.mean(1, keepdim=True)
    return dx * r, n


def _plain_norm_bwd(s):
    c, out = s["case"], {}
    G = s["dx_out"].float()
    if c["pre"] != "none":
        dy = s["dy"].float()
        d, n = _plain_norm_grad(s["x"].float(), c["pre"], s["w_pre"], dy)
        G = G + d
        out["dw_pre"] = (dy * n).sum(0)
        if "b_pre" in s:
            out["db_pre"] = dy.sum(0)
    out["dx"] = G.to(s["x"].dtype)
    f = s["f"].float()
    u = _plain_norm(f, c["post"], s.get("w_post"), s.get("b_post"))
    if "gate" in s:
        dg, rows = SCALE * G * u, c["rows_per_gate"]
        if rows:
            full = dg.new_zeros((_gates(c) * rows, c["D"]))
            full[:c["T"]] = dg
            out["dgate"] = full.reshape(-1, rows, c["D"]).sum(1)
        else:
            out["dgate"] = dg.sum(0, keepdim=True)
    du = SCALE * _gate_rows(s) * G
    if c["post"] != "none":
        df, n = _plain_norm_grad(f, c["post"], s["w_post"], du)
        out["dw_post"] = (du * n).sum(0)
        if "b_post" in s:
            out["db_post"] = du.sum(0)
        du = df
    out["df"] = du.to(s["f"].dtype)
    return out


ROOT_HALF, ROOT_2_PI, CUBIC = math.sqrt(0.5), math.sqrt(2 / math.pi), 0.044715


def _plain_act(x, kind):
    """(act(x), act'(x))"""
    if kind == "relu":
        return x.clamp(min=0), (x > 0).to(x.dtype)
    if kind == "silu":
        g = 1 / (1 + torch.exp(-x))
        return x * g, g * (1 + x * (1 - g))
    if kind == "gelu":
        p = 0.5 * (1 + torch.erf(x * ROOT_HALF))
        return x * p, p + x * torch.exp(-0.5 * x * x) * (1 / math.sqrt(2 * math.pi))
    t = torch.tanh(ROOT_2_PI * (x + CUBIC * x * x * x))
    return (0.5 * x * (1 + t),
            0.5 * (1 + t) + 0.5 * x * (1 - t * t) * ROOT_2_PI * (1 + 3 * CUBIC * x * x))


def _plain_glu(s):
    c, dt = s["case"], s["dh"].dtype
    a, dh = s["a"].float(), s["dh"].float()
    h = _plain_act(a, c["act"])[0]
    b = s["b"].float() if c["gated"] else None
    out = {"h": (h if b is None else h * b).to(dt)}
    h, slope = _plain_act(_decode(*_encode(a)), c["act"])
    if b is None:
        out["da"] = (dh * slope).to(dt)
    else:
        b = _decode(*_encode(b))
        out["da"], out["db"] = (dh * b * slope).to(dt), (dh * h).to(dt)
    return out


def _plain(s):
    op = s["case"]["op"]
    if op == "logp":
        return _plain_logp(s)
    if op == "norm_fwd":
        return _plain_norm_fwd(s)
    if op == "norm_bwd":
        return _plain_norm_bwd(s)
    if op == "glu":
        return _plain_glu(s)
    if op == "wgrad":
        dw = s["dy"].float().t() @ _decode(s["x_codes"], s["x_exps"])
        return {"dw": dw.to(s["dw"].dtype)}
    return {"back": _decode(*_encode(s["x"].float())).to(s["x"].dtype)}


# ------------------------------------------------------------------ the framework's operators

def _kept(s, name, make):
    """What a program keeps from one call to the next: configurations and scratch memory."""
    if name not in s:
        s[name] = make()
    return s[name]


def _norm_config(ops, c):
    kind = {"none": ops.NORM_NONE, "rms": ops.NORM_RMS, "layer": ops.NORM_LAYER}
    return ops.NormResidual(pre=kind[c["pre"]], post=kind[c["post"]], eps_pre=EPS, eps_post=EPS,
                            scale=SCALE, rows_per_gate=c["rows_per_gate"])


def _scratch(nbytes):
    return torch.empty((nbytes,), dtype=torch.uint8, device="cuda:0")


def _run_own(s):
    from paper_2502_06728_amd import model_ops as ops
    c = s["case"]
    op = c["op"]
    if op == "logp":
        ws = _kept(s, "workspace", lambda: _scratch(
            ops.token_logprobs_workspace(c["T"], c["V"], c["top"])))
        ops.detonation_token_logprobs(s["logits"], s["targets"], s["logp"], lse=s["lse"],
                                      entropy=s["entropy"], top_idx=s.get("top_idx"),
                                      top_logp=s.get("top_logp"),
                                      stats=s["stats"] if c["train"] else None, workspace=ws)
        names = ["logp", "lse", "entropy"] + (["top_idx", "top_logp"] if c["top"] else [])
        if c["train"]:
            ops.detonation_token_logprobs_backward(
                s["logits"], s["targets"], s["stats"], s["dlogits"], g_logp=s["g_logp"],
                entropy=s["entropy"], g_entropy=s["g_entropy"])
            names.append("dlogits")
    elif op == "norm_fwd":
        cfg = _kept(s, "config", lambda: _norm_config(ops, c))
        y8 = ops.Act8(s["y_codes"], s["y_exps"]) if c["ckpt"] else None
        ops.detonation_norm_residual(cfg, s["x"], s["f"], s["x_out"], s.get("y"), y8=y8,
                                     gate=s.get("gate"), w_post=s.get("w_post"),
                                     b_post=s.get("b_post"), w_pre=s.get("w_pre"),
                                     b_pre=s.get("b_pre"))
        names = ["x_out"] + (["y"] if c["pre"] != "none" else [])
        if c["ckpt"]:
            ops.detonation_act8_decode(y8, s["y_back"])
            names.append("y_back")
    elif op == "norm_bwd":
        cfg = _kept(s, "config", lambda: _norm_config(ops, c))
        ws = _kept(s, "workspace", lambda: _scratch(
            ops.norm_residual_workspace(cfg, c["T"], c["D"])))
        grads = {"d" + n: s["d" + n] for n in ("gate", "w_post", "b_post", "w_pre", "b_pre")
                 if n in s}
        ops.detonation_norm_residual_backward(
            cfg, s["x"], s["f"], s.get("dy"), s["dx_out"], s["dx"], s["df"], workspace=ws,
            gate=s.get("gate"), w_post=s.get("w_post"), b_post=s.get("b_post"),
            w_pre=s.get("w_pre"), **grads)
        names = ["dx", "df", *grads]
    elif op == "glu":
        act = {"silu": ops.ACT_SILU, "gelu": ops.ACT_GELU, "gelu_tanh": ops.ACT_GELU_TANH,
               "relu": ops.ACT_RELU}[c["act"]]
        a8 = ops.Act8(s["a_codes"], s["a_exps"])
        b8 = ops.Act8(s["b_codes"], s["b_exps"]) if c["gated"] else None
        ops.detonation_glu_forward(act, s["a"], s.get("b"), s["h"], a8=a8, b8=b8)
        ops.detonation_glu_backward(act, s["dh"], a8, b8, s["da"], s.get("db"))
        names = ["h", "da"] + (["db"] if c["gated"] else [])
    elif op == "wgrad":
        ws = _kept(s, "workspace", lambda: _scratch(
            ops.act8_weight_grad_workspace(c["T"], c["N"], c["K"])))
        ops.detonation_act8_weight_grad(s["dy"], ops.Act8(s["x_codes"], s["x_exps"]), s["dw"],
                                        workspace=ws)
        names = ["dw"]
    else:
        x8 = ops.Act8(s["x_codes"], s["x_exps"])
        ops.detonation_act8_encode(s["x"], x8)
        ops.detonation_act8_decode(x8, s["back"])
        names = ["back"]
    return {n: s[n] for n in names}


def run(state):
    return _run_own(state) if own else _plain(state)


# ------------------------------------------------------------------ the definitions in 64 bits

def _exact_act8(x):
    """Values in the 8-bit form, from its definition: the smallest power of two (2**-126 at least) at
    which the group's largest value rounds to 127 or less, every value rounded to a multiple."""
    T, D = x.shape
    x = torch.nn.functional.pad(x, (0, -D % GROUP)).reshape(T, -1, GROUP)
    top = x.abs().amax(2, keepdim=True)
    step = torch.exp2(torch.floor(torch.log2(top / 127)).clamp(min=-126)).double()
    for _ in range(2):                # from below, in case the logarithm was rounded
        step = torch.where(torch.round(top / step) > 127, 2 * step, step)
    return (torch.round(x / step) * step).reshape(T, -1)[:, :D]


def _exact_norm(x, kind, w, b):
    if kind == "none":
        return x
    var, mean = torch.var_mean(x, 1, correction=0, keepdim=True)
    if kind == "rms":
        var, mean = var + mean * mean, 0.0
    y = (x - mean) / torch.sqrt(var + EPS) * w.double()
    return y if b is None else y + b.double()


def _exact_block(c, s, x, f, p):
    """(residual stream after the branch, its norm) as functions of x, f and the parameters p"""
    u = _exact_norm(f, c["post"], p.get("w_post"), p.get("b_post"))
    if "gate" in p:
        T = x.shape[0]
        u = u * p["gate"][torch.arange(T, device=x.device) // (c["rows_per_gate"] or T)]
    x = x + SCALE * u
    return x, _exact_norm(x, c["pre"], p.get("w_pre"), p.get("b_pre"))


def _exact_norm_bwd(c, s):
    """Gradients by torch's own differentiation of the definition.  The residual stream is given after
    the branch was added, so x is what it was before."""
    p = {n: s[n].double().requires_grad_() for n in ("gate", "w_post", "b_post", "w_pre", "b_pre")
         if n in s}
    f = s["f"].double().requires_grad_()
    with torch.no_grad():
        off = _exact_block(dict(c, pre="none"), s, torch.zeros_like(f), f, p)[0]
    x = (s["x"].double() - off).requires_grad_()
    x_out, y = _exact_block(c, s, x, f, p)
    loss = (x_out * s["dx_out"].double()).sum()
    if c["pre"] != "none":
        loss = loss + (y * s["dy"].double()).sum()
    names = list(p)
    g = torch.autograd.grad(loss, [x, f] + [p[n] for n in names])
    return {"dx": g[0], "df": g[1], **{"d" + n: v for n, v in zip(names, g[2:])}}


def _exact_act(x, kind):
    F = torch.nn.functional
    return {"relu": F.relu, "silu": F.silu, "gelu": F.gelu,
            "gelu_tanh": lambda t: F.gelu(t, approximate="tanh")}[kind](x)


def _exact_logp(c, s):
    z, V = s["logits"], c["V"]
    got = {n: [] for n in ("logp", "lse", "entropy", "top_logp", "dlogits")}
    for lo in range(0, c["T"], 512):      # by blocks of rows: 64 bits take room
        rows = slice(lo, lo + 512)
        logs = z[rows].double()
        lse = torch.logsumexp(logs, 1)
        logs = logs - lse[:, None]
        p = torch.exp(logs)
        y = s["targets"][rows]
        scored = (y >= 0) & (y < V)
        y = torch.where(scored, y, 0)
        got["lse"].append(lse)
        got["logp"].append(torch.where(scored, logs[torch.arange(len(y), device=y.device), y], 0.0))
        logs = torch.where(p > 0, logs, 0.0)
        H = -(p * logs).sum(1)
        got["entropy"].append(H)
        if c["top"]:
            best = torch.topk(z[rows].float(), c["top"], 1).values.double()
            got["top_logp"].append(best - lse[:, None])
        if c["train"]:
            g = torch.where(scored, s["g_logp"][rows].double(), 0.0)
            one = torch.zeros_like(p)
            one[torch.arange(len(y), device=y.device), y] = 1.0
            got["dlogits"].append(g[:, None] * (one - p)
                                  - s["g_entropy"][rows].double()[:, None] * p * (logs + H[:, None]))
    out = {n: torch.cat(v) for n, v in got.items() if v}
    if c["top"]:
        out["top_idx"] = None
    return out


def exact(case, seed):
    c, s = case, prepare(case, seed)
    op = c["op"]
    if op == "logp":
        return _exact_logp(c, s)
    if op == "norm_bwd":
        return _exact_norm_bwd(c, s)
    with torch.no_grad():
        if op == "norm_fwd":
            p = {n: s[n].double() for n in ("gate", "w_post", "b_post", "w_pre", "b_pre") if n in s}
            x, y = _exact_block(c, s, s["x"].double(), s["f"].double(), p)
            out = {"x_out": x}
            if c["pre"] != "none":
                out["y"] = y
            if c["ckpt"]:
                out["y_back"] = _exact_act8(y)
            return out
        if op == "wgrad":
            scale = torch.exp2(s["x_exps"].double() - 127).repeat_interleave(GROUP, 1)
            x = s["x_codes"].double() * scale[:, :c["K"]]
            return {"dw": s["dy"].double().t().contiguous() @ x}
        if op == "codec":
            return {"back": _exact_act8(s["x"].double())}
    a = s["a"].double()
    out = {"h": _exact_act(a, c["act"])}
    if c["gated"]:
        out["h"] = out["h"] * s["b"].double()
    a = _exact_act8(a).requires_grad_()
    h = _exact_act(a, c["act"])
    if not c["gated"]:
        return {**out, "da": torch.autograd.grad(h, a, s["dh"].double())[0]}
    b = _exact_act8(s["b"].double()).requires_grad_()
    da, db = torch.autograd.grad(h * b, [a, b], s["dh"].double())
    return {**out, "da": da, "db": db}
