"""The kernels behind include/detonation_model.h against plain definitions in 64 bits.

Bounds: a result is computed in fp32 and rounded once, so it may be off by half a unit of its type plus the
fp32 roundings on the way, each half a unit (2^-24) of the terms it acts on: `steps` counts them, at worst all
in one direction."""
import math

import pytest
import torch

from paper_2502_06728_amd import model_ops as ops
from tests import model_reference as ref
from tests.model_reference import BF16, F16, F32, assert_near

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
TYPES = [F32, BF16, F16]
INF, NAN = math.inf, math.nan
KIND = {"none": ops.NORM_NONE, "rms": ops.NORM_RMS, "layer": ops.NORM_LAYER}
ACT = {"silu": ops.ACT_SILU, "gelu": ops.ACT_GELU, "gelu_tanh": ops.ACT_GELU_TANH, "relu": ops.ACT_RELU}


def say(*what):
    print(*what, flush=True)


def normal(seed, *shape, scale=1.0):
    g = torch.Generator().manual_seed(seed)
    return torch.randn(shape, generator=g, dtype=torch.float64) * scale


def rows(values, dtype, pad=0, offset=0):
    """A device matrix of these values whose rows lie `pad` elements apart, its first one `offset`
    elements into an allocation; the elements around it are NaN."""
    T, D = values.shape
    flat = torch.full((offset + T * (D + pad) + 8,), NAN, dtype=dtype, device=DEV)
    m = flat[offset:offset + T * (D + pad)].view(T, D + pad)[:, :D]
    m.copy_(values.to(dtype))
    return m


def like(T, D, dtype, pad=0, offset=0):
    return rows(torch.full((T, D), NAN, dtype=torch.float64), dtype, pad, offset)


def untouched(m):
    """Nothing was written between the rows of an output."""
    T, D = m.shape
    ld = m.stride(0)
    if ld > D and T > 1:
        gap = torch.as_strided(m, (T - 1, ld - D), (ld, 1), m.storage_offset() + D)
        assert bool(torch.isnan(gap).all())


def scratch(n):
    return torch.full((n,), 0xFF, dtype=torch.uint8, device=DEV)


def empty_act8(T, D, pad=0):
    G = -(-D // 32)
    return ops.Act8(torch.full((T, D + pad), 77, dtype=torch.int8, device=DEV)[:, :D],
                    torch.full((T, G + pad), 77, dtype=torch.uint8, device=DEV)[:, :G])


def check_act8(m, x):
    codes, exps, _ = ref.act8(x)
    assert torch.equal(m.exps.cpu().long(), exps)
    keep = (exps != 255).repeat_interleave(32, 1)[:, :codes.shape[1]]
    assert torch.equal(m.codes.cpu().long()[keep], codes[keep])


def act8_of(x):
    m = empty_act8(*x.shape)
    codes, exps, values = ref.act8(x)
    m.codes.copy_(codes)
    m.exps.copy_(exps)
    return m, values


# ------------------------------------------------------------------ log probabilities

def run_logprobs(x, y, top=0, scale=1.0, stream=None):
    T, V = x.shape
    out = {n: torch.full((T,), NAN, device=DEV) for n in ("logp", "lse", "entropy")}
    out["stats"] = torch.full((T, 2), NAN, device=DEV)
    if top:
        out["top_idx"] = torch.full((T, top), -7, dtype=torch.int32, device=DEV)
        out["top_logp"] = torch.full((T, top), NAN, device=DEV)
    ops.detonation_token_logprobs(x, y, logit_scale=scale, stream=stream,
                                  workspace=scratch(ops.token_logprobs_workspace(T, V, top)), **out)
    return out


def check_logprobs(x, y, out, scale=1.0, top=0):
    T, V = x.shape
    logp, lse, H, idx, best = ref.logprobs(x, y, scale, top)
    # V / 256 additions of a thread and 32 joins of relative 2^-23 each in the sum of exponentials, whose own
    # errors (arguments of up to 2^7 in units of log 2 that matter) are below 2^-16 together
    steps = V / 128 + 64
    finite = torch.where(torch.isfinite(x), x, torch.zeros_like(x)).double().abs().cpu() * scale
    mag = 1 + finite.max(1).values + math.log(V) if V else 1.0
    assert_near(out["logp"], logp, mag, steps + 256, "logp")
    assert_near(out["lse"], lse, mag, steps + 256, "lse")
    spread = torch.clamp(mag, max=104 * math.log(2) + math.log(V))     # of what has a probability
    assert_near(out["entropy"], H, 1 + spread, steps + 256, "entropy")
    if top:
        assert torch.equal(out["top_idx"].cpu().long(), idx)
        assert_near(out["top_logp"], best, mag[:, None], steps + 256, "top_logp")


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("T,V,top,pad,offset,scale", [
    (1, 1, 1, 0, 0, 1.0), (3, 2, 2, 0, 1, 1.0), (1, 7, 7, 0, 3, 0.5), (2, 8, 0, 3, 0, 1.0),
    (5, 33, 32, 1, 1, 2.0), (1, 2047, 5, 0, 0, 1.0), (1, 2049, 5, 0, 1, 1.0), (1, 20011, 32, 0, 0, 1.0),
    (37, 1000, 3, 7, 5, 0.125), (2, 4096, 1, 0, 0, 1.0), (1030, 301, 4, 0, 0, 1.0),
    (1500, 130, 0, 2, 0, 1.0), (1100, 5003, 8, 1, 0, 1.0)])
def test_logprobs(gpu, dtype, T, V, top, pad, offset, scale):
    say(dtype, T, V, top)
    x = rows(normal(V + T, T, V, scale=3.0), dtype, pad, offset)
    y = torch.randint(-1, V + 1, (T,), generator=torch.Generator().manual_seed(1)).to(DEV)
    check_logprobs(x, y, run_logprobs(x, y, top, scale), scale, top)
    y32 = y.to(torch.int32)
    again = run_logprobs(x, y32, top, scale)
    check_logprobs(x, y32, again, scale, top)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("V", [40, 2500, 9000])
def test_logprobs_of_unusual_rows(gpu, dtype, V):
    lowest = torch.finfo(dtype).min
    x = normal(5, 12, V)
    x[0] = -INF                              # nothing left
    x[1] = lowest                            # the type's lowest value throughout
    x[2, 1:] = -INF                          # one left
    x[3, ::2] = -INF
    x[4, 1:] = lowest
    x[5, V // 2] = INF
    x[6, V - 1] = NAN
    x[7] = 0.0                               # equal values: ties by index
    x[8] = torch.round(x[8])                 # many ties
    x[9, 0], x[9, 1:] = -0.0, 0.0            # -0 and 0 are one value
    x[10] = NAN
    x[11, :-3] = -INF                        # fewer left than are asked for
    d = rows(x, dtype)
    y = torch.tensor([0, 3, 0, 0, 1, 2, 0, V - 1, 5, 1, 0, 0], device=DEV)
    for top in (0, 1, 20):
        say(dtype, V, top)
        out = run_logprobs(d, y, top)
        check_logprobs(d, y, out, 1.0, top)
        assert_near(out["logp"][1:2], torch.tensor([-math.log(V)], dtype=torch.float64), 16.0, V / 128 + 64)
        assert_near(out["entropy"][1:2], torch.tensor([math.log(V)], dtype=torch.float64), 16.0, V / 128 + 64)
    for g_entropy in (None, torch.ones(12, device=DEV)):
        want = ref.logprobs_grad(d, y, torch.ones(12), None if g_entropy is None else torch.ones(12))
        got = like(12, V, dtype)
        ops.detonation_token_logprobs_backward(d, y, out["stats"], got, g_logp=torch.ones(12, device=DEV),
                                               entropy=out["entropy"], g_entropy=g_entropy)
        plain = [0, 1, 2, 3, 4, 7, 8, 9, 11]
        assert_near(got[plain], want[plain], 2 + math.log(V) + 20, V / 128 + 320, "dlogits")
        assert bool(torch.isnan(got[[6, 10]]).all()) and bool(torch.isnan(got[5]).any())


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("T,V", [(3, 40000), (2, 65535), (3, 70001), (1, 200003), (530, 9001), (520, 70001)])
def test_logprobs_of_long_rows(gpu, dtype, T, V):
    """Rows that take a workgroup several steps or several workgroups; a lane sees masked values (the type's
    lowest, -infinity) for its first steps and others later, and the other way round."""
    say(dtype, T, V)
    x = normal(V + T, T, V, scale=2.0).float()
    x[0, :V // 2] = torch.finfo(dtype).min
    x[T - 1, V // 2:] = -INF if T > 1 else torch.finfo(dtype).min
    x[T // 2, ::3] = torch.finfo(dtype).min
    d = rows(x, dtype)
    y = torch.randint(0, V, (T,), generator=torch.Generator().manual_seed(1)).to(DEV)
    y[0] = V - 1
    out = run_logprobs(d, y, 6, 2.0)
    keep = torch.arange(0, T, max(1, T // 16))
    part = {n: v[keep] for n, v in out.items()}
    check_logprobs(d[keep], y[keep], part, 2.0, 6)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("T,V,pad,offset,scale", [
    (1, 1, 0, 0, 1.0), (3, 9, 2, 1, 1.0), (2, 8192, 0, 0, 1.0), (5, 8193, 1, 3, 0.5), (700, 515, 0, 0, 2.0)])
def test_logprobs_gradient(gpu, dtype, T, V, pad, offset, scale):
    x = rows(normal(T, T, V, scale=2.0), dtype, pad, offset)
    y = torch.randint(-1, V + 1, (T,), generator=torch.Generator().manual_seed(2)).to(DEV)
    out = run_logprobs(x, y, 0, scale)
    g, ge = normal(3, T).float().to(DEV), normal(4, T).float().to(DEV)
    for a, b in ((g, None), (None, ge), (g, ge)):
        want = ref.logprobs_grad(x, y, a, b, scale)
        got = like(T, V, dtype, pad, offset)
        ops.detonation_token_logprobs_backward(x, y, out["stats"], got, g_logp=a, g_entropy=b,
                                               entropy=out["entropy"], logit_scale=scale)
        size = scale * (g.abs().max() + ge.abs().max()).item() * (2 + math.log(V))
        # relative to a probability: what the forward pass's sum is off by
        mag = size * torch.exp(ref.double(x) * scale - out["lse"].cpu().double()[:, None]).clamp(min=1e-30)
        mag[torch.arange(T)[(y.cpu() >= 0) & (y.cpu() < V)], y.cpu()[(y.cpu() >= 0) & (y.cpu() < V)]] += size
        assert_near(got, want, mag * (1 + ref.double(x).abs() * scale), V / 128 + 320, "dlogits")
        untouched(got)
    twin = x.clone()                            # in place
    twin_rows = like(T, V, dtype, pad, offset)
    twin_rows.copy_(twin)
    ops.detonation_token_logprobs_backward(twin_rows, y, out["stats"], twin_rows, g_logp=g, g_entropy=ge,
                                           entropy=out["entropy"], logit_scale=scale)
    assert torch.equal(twin_rows, got)


@pytest.mark.parametrize("dtype", TYPES)
def test_logprobs_of_large_matrices(gpu, dtype):
    """More logits than the caches hold: the kernels that stream them."""
    T, V = (1400, 50001) if dtype != F32 else (700, 50001)
    say(dtype, T, V)
    g = torch.Generator(device=DEV).manual_seed(1)
    x = (torch.randn((T, V), generator=g, device=DEV) * 2).to(dtype)
    y = torch.randint(0, V, (T,), generator=g, device=DEV)
    out = run_logprobs(x, y)
    gl, ge = torch.randn(T, generator=g, device=DEV), torch.randn(T, generator=g, device=DEV)
    keep = torch.tensor([0, 1, T // 2, T - 1])
    before = x[keep].clone()
    check_logprobs(before, y[keep], {n: v[keep] for n, v in out.items()})
    ops.detonation_token_logprobs_backward(x, y, out["stats"], x, g_logp=gl, entropy=out["entropy"], g_entropy=ge)
    want = ref.logprobs_grad(before, y[keep], gl[keep], ge[keep])
    size = (gl.abs().max() + ge.abs().max()).item() * (2 + math.log(V))
    mag = size * torch.exp(ref.double(before) - out["lse"][keep].cpu().double()[:, None]).clamp(min=1e-30)
    mag[torch.arange(4), y[keep].cpu()] += size
    assert_near(x[keep], want, mag * (1 + ref.double(before).abs()), V / 128 + 320, "dlogits")


def test_logprobs_gradient_by_differences(gpu):
    T, V, h = 4, 3001, 1e-2
    x, v = normal(1, T, V), normal(2, T, V)
    y = torch.tensor([3, 3000, -100, 17], device=DEV)
    g, ge = normal(3, T).float().to(DEV), normal(4, T).float().to(DEV)

    def loss(z):
        o = run_logprobs(rows(z, F32), y)
        return float((g * o["logp"]).double().sum() + (ge * o["entropy"]).double().sum())
    out = run_logprobs(rows(x, F32), y)
    d = like(T, V, F32)
    ops.detonation_token_logprobs_backward(rows(x, F32), y, out["stats"], d, g_logp=g, g_entropy=ge,
                                           entropy=out["entropy"])
    slope = (loss(x + h * v) - loss(x - h * v)) / (2 * h)
    # third-order terms of h^2, and fp32 values of about 30 divided by 2 h
    assert abs(slope - float((ref.double(d) * v).sum())) < 20 * h * h + 30 * 2.0 ** -24 * 50 / (2 * h)


# ------------------------------------------------------------------ norm, gate, residual

CASES = [  # T, D, pre, post, rows_per_gate (None: no gate), weights
    (1, 1, "rms", "rms", 0, True), (1, 2048, "rms", "rms", 0, True), (7, 64, "layer", "none", 0, True),
    (5, 771, "layer", "layer", 2, True), (33, 768, "rms", "none", None, True),
    (9, 513, "none", "rms", 4, True), (3, 1025, "rms", "layer", 1, False), (4, 4099, "layer", "rms", 3, True),
    (2, 8192, "rms", "rms", 0, True), (3, 16384, "layer", "rms", 0, True), (2, 9001, "rms", "layer", 1, True),
    (4500, 40, "rms", "rms", 3, True), (2600, 130, "layer", "layer", 1, True),
    (1300, 100, "rms", "none", 1000, True), (5000, 33, "rms", "rms", 0, False)]


def norm_inputs(T, D, pre, post, rows_per_gate, weights, xt, ft, pad, offset):
    s = dict(x=rows(normal(1, T, D, scale=2.0) + 0.5, xt, pad, offset),
             f=rows(normal(2, T, D), ft, pad, offset), p={})
    if weights:
        for i, (name, kind) in enumerate((("w_pre", pre), ("b_pre", pre), ("w_post", post),
                                          ("b_post", post))):
            if kind != "none" and (name[0] == "w" or kind == "layer"):
                s["p"][name] = (normal(10 + i, D, scale=0.3) + (name[0] == "w")).float().to(DEV)
    if rows_per_gate is not None:
        n = -(-T // rows_per_gate) if rows_per_gate else 1
        s["p"]["gate"] = (normal(20, n, D, scale=0.5) + 0.5).float().to(DEV)
    s["cfg"] = ops.NormResidual(pre=KIND[pre], post=KIND[post], eps_pre=1e-5, eps_post=1e-6, scale=0.7,
                                rows_per_gate=rows_per_gate or 0)
    return s


def reference_block(s, pre, post, x, f, p=None):
    c = s["cfg"]
    return ref.block(x, f, pre, post, c.eps_pre, c.eps_post, c.scale, c.rows_per_gate,
                     {n: ref.double(v) for n, v in s["p"].items()} if p is None else p)


# Sums over a row of D: a lane adds 16 values at most, then 12 joins; norms are a dozen roundings of values of
# the row's spread.
NORM_STEPS = 64


@pytest.mark.parametrize("xt,ft", [(F32, F32), (BF16, BF16), (F16, F16), (F32, BF16), (F32, F16)])
@pytest.mark.parametrize("T,D,pre,post,rows_per_gate,weights", CASES)
def test_norm_residual(gpu, xt, ft, T, D, pre, post, rows_per_gate, weights):
    say(xt, ft, T, D, pre, post, rows_per_gate)
    pad, offset = (3, 1) if D % 2 else (0, 0)
    s = norm_inputs(T, D, pre, post, rows_per_gate, weights, xt, ft, pad, offset)
    x_out, y = like(T, D, xt, pad, offset), like(T, D, ft, pad, offset) if pre != "none" else None
    y8 = empty_act8(T, D, pad) if pre != "none" else None
    ops.detonation_norm_residual(s["cfg"], s["x"], s["f"], x_out, y, y8=y8, **s["p"])
    want_x, want_y = reference_block(s, pre, post, ref.double(s["x"]), ref.double(s["f"]))
    assert_near(x_out, want_x, 12.0, NORM_STEPS, "x_out")
    untouched(x_out)
    if pre == "none":
        return
    assert_near(y, want_y, want_y.abs() + 4.0, NORM_STEPS, "y")
    untouched(y)
    # the codes are those of an fp32 y: off by one only where y is half way between two (an exponent also
    # where the group's largest is at the border of one)
    codes, exps, values = ref.act8(want_y)
    step = 2.0 ** (torch.maximum(exps, y8.exps.cpu().long()) - 127).double().repeat_interleave(32, 1)[:, :D]
    got = ref.act8_values(y8.codes, y8.exps)
    off = NORM_STEPS * 2.0 ** -24 * (want_y.abs() + 4.0)
    assert bool(((got - want_y).abs() <= 0.5 * step + off).all())
    assert int((y8.exps.cpu().long() - exps).abs().max()) <= 1
    inplace = s["x"]
    ops.detonation_norm_residual(s["cfg"], inplace, s["f"], inplace, y, y8=None, **s["p"])
    assert torch.equal(inplace, x_out)


@pytest.mark.parametrize("dtype", TYPES)
def test_norm_alone(gpu, dtype):
    for D in (96, 2048, 3001):
        x = rows(normal(D, 6, D), dtype)
        w = (normal(1, D) + 1).to(dtype).to(DEV)
        y = like(6, D, dtype)
        cfg = ops.NormResidual(pre=ops.NORM_RMS)
        ops.detonation_norm_residual(cfg, x, None, None, y, w_pre=w)
        want = ref.norm(ref.double(x), "rms", ref.double(w), None, 1e-6)
        assert_near(y, want, want.abs() + 1, NORM_STEPS, "y")
        y8 = empty_act8(6, D)
        ops.detonation_norm_residual(cfg, x, None, None, None, y8=y8, w_pre=w)
        if dtype == F32:
            check_act8(y8, y)
        dy, dx, dw = rows(normal(3, 6, D), dtype), like(6, D, dtype), torch.full((D,), NAN, device=DEV)
        ops.detonation_norm_residual_backward(
            cfg, x, None, dy, None, dx, None, w_pre=w, dw_pre=dw,
            workspace=scratch(ops.norm_residual_workspace(cfg, 6, D)))
        xd = ref.double(x).requires_grad_()
        wd = ref.double(w).requires_grad_()
        g = torch.autograd.grad((ref.norm(xd, "rms", wd, None, 1e-6) * ref.double(dy)).sum(), [xd, wd])
        assert_near(dx, g[0], 16.0, NORM_STEPS, "dx")
        assert_near(dw, g[1], 6 * 10.0, NORM_STEPS, "dw")


def test_norm_of_unusual_rows(gpu):
    D = 96
    x = normal(1, 6, D)
    x[0] = 0.0
    x[1] = 1e-30
    x[2, 5] = INF
    x[3, 7] = NAN
    x[4] = 3000.0 + normal(2, D) * 1e-2        # a mean that drowns the spread
    for kind in ("rms", "layer"):
        y, y8 = like(6, D, F32), empty_act8(6, D)
        cfg = ops.NormResidual(pre=KIND[kind], eps_pre=1e-6)
        m = rows(x, F32)
        ops.detonation_norm_residual(cfg, m, None, None, y, y8=y8)
        want = ref.norm(ref.double(m), kind, None, None, 1e-6)
        keep = [0, 1, 4, 5]
        # row 4: a mean of 3000 is off by 3000 * 2^-24 * 16 against a spread of 1e-2
        assert_near(y[keep], want[keep], torch.tensor([1.0, 1.0, 3000 / 1e-2 if kind == "layer" else 1.0, 4.0],
                                                      dtype=torch.float64)[:, None], NORM_STEPS, kind)
        assert bool(torch.isnan(y[3]).all()) and bool(torch.isnan(y[2]).any())
        assert bool((y8.exps[3] == 255).all())


def tolerance(T):
    """Roundings of a sum over T rows: a team adds its own, then teams are added four at a time."""
    return T + 64


@pytest.mark.parametrize("xt,ft", [(F32, F32), (BF16, BF16), (F16, F16), (F32, BF16), (F32, F16)])
@pytest.mark.parametrize("T,D,pre,post,rows_per_gate,weights", CASES)
def test_norm_residual_gradient(gpu, xt, ft, T, D, pre, post, rows_per_gate, weights):
    say(xt, ft, T, D, pre, post, rows_per_gate)
    pad, offset = (5, 3) if D % 2 else (0, 0)
    s = norm_inputs(T, D, pre, post, rows_per_gate, weights, xt, ft, pad, offset)
    dy = rows(normal(5, T, D), ft, pad, offset) if pre != "none" else None
    dxo = rows(normal(6, T, D), xt, pad, offset)
    dx, df = like(T, D, xt, pad, offset), like(T, D, ft, pad, offset)
    grads = {"d" + n: torch.full(v.shape, NAN, device=DEV) for n, v in s["p"].items()}
    params = {n: v for n, v in s["p"].items() if n != "b_pre"}

    def call(dx_out, dx):
        ops.detonation_norm_residual_backward(
            s["cfg"], s["x"], s["f"], dy, dx_out, dx, df,
            workspace=scratch(ops.norm_residual_workspace(s["cfg"], T, D)), **params, **grads)
    call(dxo, dx)
    p = {n: ref.double(v).requires_grad_() for n, v in s["p"].items()}
    f = ref.double(s["f"]).requires_grad_()
    with torch.no_grad():                        # x_out is given: x is what makes it so
        branch = reference_block(s, "none", post, torch.zeros_like(f), f, p)[0]
    x = (ref.double(s["x"]) - branch).requires_grad_()
    x_out, y = reference_block(s, pre, post, x, f, p)
    loss = (x_out * ref.double(dxo)).sum()
    if pre != "none":
        loss = loss + (y * ref.double(dy)).sum()
    g = torch.autograd.grad(loss, [x, f, *p.values()], allow_unused=True)
    def magnitude(kind, v):                      # a row's gradient times the norm's factor
        if kind == "none":
            return 8.0
        v = v.detach()
        v = v - v.mean(1, keepdim=True) if kind == "layer" else v
        eps = min(s["cfg"].eps_pre, s["cfg"].eps_post)
        return 8.0 + 64.0 / torch.sqrt((v * v).mean(1, keepdim=True) + eps)
    mx = magnitude(pre, ref.double(s["x"]))
    mf = mx * magnitude(post, f)
    assert_near(dx, g[0], mx, NORM_STEPS, "dx")
    assert_near(df, g[1], mf, NORM_STEPS, "df")
    untouched(dx)
    untouched(df)
    for (name, got), want in zip(grads.items(), g[2:]):
        assert_near(got, want, 16.0 * torch.as_tensor(mx).max(), tolerance(T), name)
    first = {n: v.clone() for n, v in grads.items()}
    call(dxo, dxo)                               # in place, and the same bits again
    assert torch.equal(dxo, dx)
    for n, v in grads.items():
        assert torch.equal(v, first[n])


def test_norm_gradient_by_differences(gpu):
    T, D, h = 6, 200, 1e-2
    s = norm_inputs(T, D, "layer", "rms", 4, True, F32, F32, 0, 0)
    a, b = normal(30, T, D), normal(31, T, D)    # of y and x_out
    dx, df = like(T, D, F32), like(T, D, F32)
    x0, f0 = ref.double(s["x"]), ref.double(s["f"])

    def forward(x, f):
        x_out, y = like(T, D, F32), like(T, D, F32)
        ops.detonation_norm_residual(s["cfg"], rows(x, F32), rows(f, F32), x_out, y, **s["p"])
        return x_out, float((ref.double(y) * a).sum() + (ref.double(x_out) * b).sum())
    x_out, _ = forward(x0, f0)
    grads = {"d" + n: torch.empty_like(v) for n, v in s["p"].items()}
    ops.detonation_norm_residual_backward(
        s["cfg"], x_out, s["f"], rows(a, F32), rows(b, F32), dx, df, **grads,
        **{n: v for n, v in s["p"].items() if n != "b_pre"},
        workspace=scratch(ops.norm_residual_workspace(s["cfg"], T, D)))
    vx, vf = normal(32, T, D), normal(33, T, D)
    slope = (forward(x0 + h * vx, f0 + h * vf)[1] - forward(x0 - h * vx, f0 - h * vf)[1]) / (2 * h)
    got = float((ref.double(dx) * vx).sum() + (ref.double(df) * vf).sum())
    # third derivatives of order one, 1200 values of fp32 rounding
    assert abs(slope - got) < 0.01 * abs(got) + 100 * h * h + 35 * 4 * 2.0 ** -24 * 64 / (2 * h)


@pytest.mark.parametrize("rows_per_gate", [0, 3])
def test_norm_gradient_without_rows(gpu, rows_per_gate):
    D = 70
    cfg = ops.NormResidual(pre=ops.NORM_LAYER, post=ops.NORM_RMS, rows_per_gate=rows_per_gate)
    none = torch.empty((0, D), device=DEV)
    gate = torch.ones((0 if rows_per_gate else 1, D), device=DEV)
    g = {n: torch.full((D,), NAN, device=DEV) for n in ("dw_pre", "db_pre", "dw_post", "db_post")}
    g["dgate"] = torch.full(gate.shape, NAN, device=DEV)
    w = torch.ones(D, device=DEV)
    ops.detonation_norm_residual(cfg, none, none, none, none, gate=gate, w_pre=w, w_post=w)
    ops.detonation_norm_residual_backward(cfg, none, none, none, none, none, none, gate=gate, w_pre=w,
                                          w_post=w, **g)
    for v in g.values():
        assert bool((v == 0).all())


# ------------------------------------------------------------------ 8 bits

def wide(seed, T, D):
    """Magnitudes over the whole range of the type, zeros, and values half way between codes."""
    x = normal(seed, T, D) * torch.exp2(torch.round(normal(seed + 1, T, 1) * 30).clamp(-100, 100))
    x[:, ::7] = 0.0
    half = torch.round(normal(seed + 2, T, D) * 40) + 0.5
    return torch.where(torch.arange(T)[:, None] % 3 == 0, half, x)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("T,D,pad,offset", [(1, 1, 0, 0), (3, 31, 0, 1), (2, 32, 0, 0), (5, 33, 3, 0),
                                            (300, 96, 0, 0), (7, 1000, 9, 5), (129, 8, 0, 0)])
def test_act8_codec(gpu, dtype, T, D, pad, offset):
    x = wide(D, T, D)
    if dtype == F16:
        x = x.clamp(-60000, 60000)
    m = rows(x, dtype, pad, offset)
    q = empty_act8(T, D, pad)
    ops.detonation_act8_encode(m, q)
    check_act8(q, m)
    for out in TYPES:
        back = like(T, D, out, pad, offset)
        ops.detonation_act8_decode(q, back)
        assert torch.equal(back, ref.act8_values(q.codes, q.exps).to(F32).to(out).to(DEV))
        untouched(back)
    if pad:
        whole = torch.as_strided(q.codes, (T, D + pad), (D + pad, 1))
        assert bool((whole[:, D:] == 77).all())


def test_act8_borders(gpu):
    """Largest magnitudes around those where the exponent changes, the smallest and the largest values, and
    groups that hold an infinity or a NaN."""
    tops = []
    for e in (-149, -140, -127, -126, -120, -119, -20, 0, 1, 63, 126, 127):
        for m in (1.0, 1.5, 1.984375, 1.9921874, 1.9921875, 1.9999999):
            tops.append(min(m * 2.0 ** e, 3.4028234e38))
    tops += [0.0, INF, -INF, NAN]
    x = torch.zeros((len(tops), 64), dtype=torch.float64)
    x[:, 3] = torch.tensor(tops, dtype=torch.float64)
    x[:, 40] = 1.0
    m = rows(x, F32)
    q = empty_act8(*x.shape)
    ops.detonation_act8_encode(m, q)
    check_act8(q, m)
    back = like(*x.shape, F32)
    ops.detonation_act8_decode(q, back)
    assert bool(torch.isnan(back[-3:, :32]).all()) and bool((back[-3:, 40] == 1.0).all())
    assert bool((q.exps[-3:, 0] == 255).all())


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("act", list(ACT))
@pytest.mark.parametrize("gated", [True, False])
@pytest.mark.parametrize("T,D,pad,offset", [(1, 1, 0, 0), (3, 71, 3, 1), (17, 256, 0, 0), (260, 40, 0, 0)])
def test_glu(gpu, dtype, act, gated, T, D, pad, offset):
    say(dtype, act, gated, T, D)
    a = rows(normal(1, T, D, scale=3.0), dtype, pad, offset)
    b = rows(normal(2, T, D), dtype, pad, offset) if gated else None
    h = like(T, D, dtype, pad, offset)
    a8, b8 = empty_act8(T, D), empty_act8(T, D) if gated else None
    ops.detonation_glu_forward(ACT[act], a, b, h, a8=a8, b8=b8)
    check_act8(a8, a)
    ad = ref.double(a)
    bd = ref.double(b) if gated else torch.ones_like(ad)
    # an activation and its slope: 32 roundings of its argument's size
    assert_near(h, ref.act(ad, act) * bd, (1 + ad.abs()) * bd.abs(), 32, "h")
    untouched(h)
    if gated:
        check_act8(b8, b)
    dh = rows(normal(3, T, D), dtype, pad, offset)
    da, db = like(T, D, dtype, pad, offset), like(T, D, dtype, pad, offset) if gated else None
    h8 = empty_act8(T, D)
    ops.detonation_glu_backward(ACT[act], dh, a8, b8, da, db, h8=h8)
    ad = ref.act8(a)[2]
    bd = ref.act8(b)[2] if gated else torch.ones_like(ad)
    dd = ref.double(dh)
    mag = (1 + ad.abs()) ** 3 if act == "gelu_tanh" else 1 + ad.abs()
    assert_near(da, dd * bd * ref.act_slope(ad, act), (dd * bd).abs() * mag, 32, "da")
    untouched(da)
    if gated:
        assert_near(db, dd * ref.act(ad, act), dd.abs() * mag, 32, "db")
    want = ref.act(ad, act) * bd
    _, exps, _ = ref.act8(want)
    got = ref.act8_values(h8.codes, h8.exps)
    step = 2.0 ** (torch.maximum(exps, h8.exps.cpu().long()) - 127).double().repeat_interleave(32, 1)[:, :D]
    assert bool(((got - want).abs() <= 0.5 * step + 32 * 2.0 ** -24 * mag * bd.abs()).all())
    ops.detonation_glu_backward(ACT[act], dh, a8, b8, dh, db)          # in place
    assert torch.equal(dh, da)
    ops.detonation_glu_forward(ACT[act], a, b, a)
    assert torch.equal(a, h)


def test_glu_of_a_fused_projection(gpu):
    """a and b are the two halves of one matrix, their gradients of another."""
    T, D = 9, 160
    both, grad = rows(normal(1, T, 2 * D), BF16), like(T, 2 * D, BF16)
    h, dh = like(T, D, BF16), rows(normal(2, T, D), BF16)
    a8, b8 = empty_act8(T, D), empty_act8(T, D)
    ops.detonation_glu_forward(ops.ACT_SILU, both[:, :D], both[:, D:], h, a8=a8, b8=b8)
    ops.detonation_glu_backward(ops.ACT_SILU, dh, a8, b8, grad[:, :D], grad[:, D:])
    a, b, d = ref.act8(both[:, :D])[2], ref.act8(both[:, D:])[2], ref.double(dh)
    assert_near(grad[:, :D], d * b * ref.act_slope(a, "silu"), (d * b).abs() * (1 + a.abs()), 32, "da")
    assert_near(grad[:, D:], d * ref.act(a, "silu"), d.abs() * (1 + a.abs()), 32, "db")


def test_glu_at_extreme_arguments(gpu):
    a = torch.tensor([[0.0, -0.0, 1e-30, 20.0, -20.0, 90.0, -90.0, 3e4, -3e4, 1e-3, -1e-3, 6.0]],
                     dtype=torch.float64)
    for act in ACT:
        m, h = rows(a, F32), like(1, 12, F32)
        ops.detonation_glu_forward(ACT[act], m, None, h)
        assert_near(h, ref.act(ref.double(m), act), 1e-30 + a.abs(), 64, act)
        codes = torch.zeros((11, 32), dtype=torch.int8, device=DEV)
        exps = torch.full((11, 1), 127, dtype=torch.uint8, device=DEV)
        for i, v in enumerate((0, 1, -1, 20, -20, 90, -90, 5, -5, 127, -127)):
            codes[i, :16] = v
        dh, da = rows(torch.ones(11, 32), F32), like(11, 32, F32)
        ops.detonation_glu_backward(ACT[act], dh, ops.Act8(codes, exps), None, da)
        x = codes.cpu().double()
        assert_near(da, ref.act_slope(x, act), 1 + x.abs(), 64, act)


# ------------------------------------------------------------------ weight gradient

@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("out", TYPES)
@pytest.mark.parametrize("T,N,K", [(1, 1, 1), (5, 3, 33), (64, 128, 128), (65, 129, 127), (1000, 70, 130),
                                   (2049, 65, 40), (130, 300, 520)])
def test_weight_grad(gpu, dtype, out, T, N, K):
    say(dtype, out, T, N, K)
    pad, offset = (3, 1) if N % 2 else (0, 0)
    dy = rows(normal(1, T, N), dtype, pad, offset)
    x8, x = act8_of(normal(2, T, K))
    dw = like(N, K, out, pad, offset)
    ws = scratch(ops.act8_weight_grad_workspace(T, N, K))
    ops.detonation_act8_weight_grad(dy, x8, dw, workspace=ws)
    d = ref.double(dy)
    want, mag = d.t() @ x, d.abs().t() @ x.abs()
    # exact products, of three terms at most, added in any order; then the splits of T
    assert_near(dw, want, mag, 3 * T + 40, "dw")
    untouched(dw)
    again = like(N, K, out, pad, offset)
    ops.detonation_act8_weight_grad(dy, x8, again, workspace=ws)
    assert torch.equal(dw, again)
    old = normal(3, N, K)
    dw.copy_(old)
    start = ref.double(dw)
    ops.detonation_act8_weight_grad(dy, x8, dw, accumulate=True, workspace=ws)
    assert_near(dw, want + start, mag + start.abs(), 3 * T + 41, "dw accumulated")


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("N,K,pad_y,pad_x", [(129, 130, 3, 2), (131, 127, 1, 1), (64, 33, 0, 3), (7, 5, 1, 0)])
def test_weight_grad_of_rows_apart(gpu, dtype, N, K, pad_y, pad_x):
    """Widths that are not whole words, at strides that are, and the other way round; what lies between the
    rows is NaN (and codes under exponents of 255)."""
    T = 130
    dy = rows(normal(1, T, N), dtype, pad_y)
    codes, exps, x = ref.act8(normal(2, T, K))
    x8 = empty_act8(T, K, pad_x)
    torch.as_strided(x8.exps, (T, x8.exps.stride(0)), (x8.exps.stride(0), 1)).fill_(255)
    x8.codes.copy_(codes)
    x8.exps.copy_(exps)
    dw = like(N, K, F32, 1)
    ops.detonation_act8_weight_grad(dy, x8, dw,
                                    workspace=scratch(ops.act8_weight_grad_workspace(T, N, K)))
    d = ref.double(dy)
    assert_near(dw, d.t() @ x, d.abs().t() @ x.abs(), 3 * T + 40, "dw")
    untouched(dw)


def test_weight_grad_of_distant_rows(gpu):
    """Rows of one matrix 2^25 bytes apart: a step of them passes 2^31 bytes."""
    T, N, K = 70, 20, 40
    far = torch.zeros((T, 1 << 24), dtype=BF16, device=DEV)
    dy = far[:, 100:100 + N]
    dy.copy_(normal(1, T, N))
    x8, x = act8_of(normal(2, T, K))
    dw = like(N, K, F32)
    ops.detonation_act8_weight_grad(dy, x8, dw, workspace=scratch(ops.act8_weight_grad_workspace(T, N, K)))
    d = ref.double(dy)
    assert_near(dw, d.t() @ x, d.abs().t() @ x.abs(), 3 * T + 40, "dw")


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("T,N,K", [(500, 1800, 1900), (500, 1801, 1901), (4100, 768, 776), (4100, 769, 777)])
def test_weight_grad_of_many_tiles(gpu, dtype, T, N, K):
    """Sizes at which workgroups share tiles of 128, in one split of T and in several."""
    say(dtype, T, N, K)
    g = torch.Generator(device=DEV).manual_seed(1)
    dy = torch.randn((T, N), generator=g, device=DEV).to(dtype)
    x8 = empty_act8(T, K)
    ops.detonation_act8_encode(torch.randn((T, K), generator=g, device=DEV), x8)
    d, v = ref.double(dy), ref.act8_values(x8.codes, x8.exps)
    for out in (F32, BF16):
        dw = like(N, K, out)
        ops.detonation_act8_weight_grad(dy, x8, dw, workspace=scratch(ops.act8_weight_grad_workspace(T, N, K)))
        assert_near(dw, d.t() @ v, d.abs().t() @ v.abs(), 3 * T + 40, "dw")


def test_weight_grad_large_tiles(gpu):
    T, N, K = 136, 2050, 6100
    say(T, N, K)
    dy = rows(normal(1, T, N), BF16)
    x8 = empty_act8(T, K)
    x = normal(2, T, K)
    ops.detonation_act8_encode(rows(x, F32), x8)
    dw = like(N, K, F32, 4)
    ops.detonation_act8_weight_grad(dy, x8, dw,
                                    workspace=scratch(ops.act8_weight_grad_workspace(T, N, K)))
    d, v = ref.double(dy), ref.act8_values(x8.codes, x8.exps)
    assert_near(dw, d.t() @ v, d.abs().t() @ v.abs(), 3 * T + 40, "dw")
    untouched(dw)


def test_weight_grad_without_rows(gpu):
    dy, x8 = torch.empty((0, 40), device=DEV), empty_act8(0, 50)
    dw = torch.full((40, 50), 3.0, device=DEV)
    ops.detonation_act8_weight_grad(dy, x8, dw, accumulate=True)
    assert bool((dw == 3.0).all())
    ops.detonation_act8_weight_grad(dy, x8, dw)
    assert bool((dw == 0.0).all())


def test_weight_grad_of_unusual_values(gpu):
    """Every fp32 bit of dy counts, its range too; an infinity gives one, a group marked as not finite NaNs."""
    dy = torch.tensor([[3.4028234e38, 1.0 + 2.0 ** -23, 1.2345678 * 2.0 ** -100, INF, 1.0]], dtype=torch.float64)
    m = rows(dy, F32)
    x8, x = act8_of(torch.ones(1, 64, dtype=torch.float64) * 0.5)
    x8.exps[0, 1] = 255
    dw = like(5, 64, F32)
    ws = scratch(ops.act8_weight_grad_workspace(1, 5, 64))
    ops.detonation_act8_weight_grad(m, x8, dw, workspace=ws)
    got = ref.double(dw)
    for n in (0, 1, 2, 4):
        assert bool((got[n, :32] == float(ref.double(m)[0, n]) * 0.5).all())
    assert bool((got[3, :32] == INF).all())
    assert bool(torch.isnan(got[:, 32:]).all())


# ------------------------------------------------------------------ streams, graphs, refusals

def test_another_stream(gpu):
    x = rows(normal(1, 50, 4000), BF16)
    y = torch.randint(0, 4000, (50,), device=DEV)
    want = run_logprobs(x, y, 4)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):              # (the outputs are allocated and filled there)
        out = run_logprobs(x, y, 4, stream=s)
    torch.cuda.synchronize()
    for n in want:
        assert torch.equal(out[n], want[n])


def test_replayed_graph(gpu):
    """One block's norm, its backward and a weight gradient, captured and replayed with new data between."""
    T, D = 300, 260
    s = norm_inputs(T, D, "rms", "rms", 0, True, F32, BF16, 0, 0)
    x_out, y, y8 = like(T, D, F32), like(T, D, BF16), empty_act8(T, D)
    dy, dxo = rows(normal(5, T, D), BF16), rows(normal(6, T, D), F32)
    dx, df, dw = like(T, D, F32), like(T, D, BF16), torch.empty((D, D), device=DEV)
    grads = {"d" + n: torch.empty_like(v) for n, v in s["p"].items()}
    ws = scratch(ops.norm_residual_workspace(s["cfg"], T, D))
    ws2 = scratch(ops.act8_weight_grad_workspace(T, D, D))

    def step():
        ops.detonation_norm_residual(s["cfg"], s["x"], s["f"], x_out, y, y8=y8, **s["p"])
        ops.detonation_norm_residual_backward(s["cfg"], x_out, s["f"], dy, dxo, dx, df, workspace=ws,
                                              **s["p"] | {}, **grads)
        ops.detonation_act8_weight_grad(dy, y8, dw, workspace=ws2)
    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for i in range(4):
        s["f"].copy_(normal(40 + i, T, D).to(DEV))
        outs = (x_out, y, dx, df, dw, *grads.values())
        for t in outs:
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in outs]
        step()
        torch.cuda.synchronize()
        for a, b in zip(got, outs):
            assert torch.equal(a, b)


def test_binding_refusals(gpu):
    x = torch.zeros((4, 64), device=DEV)
    y = torch.zeros(4, dtype=torch.int64, device=DEV)
    o = torch.zeros(4, device=DEV)
    bad = [
        lambda: ops.detonation_token_logprobs(x, y[:3], o),
        lambda: ops.detonation_token_logprobs(x, y.float(), o),
        lambda: ops.detonation_token_logprobs(x, y, o.double()),
        lambda: ops.detonation_token_logprobs(x, y, o, top_logp=torch.zeros((4, 2), device=DEV)),
        lambda: ops.detonation_token_logprobs(x, y, o, stats=o),
        lambda: ops.detonation_token_logprobs(x.double(), y, o),
        lambda: ops.detonation_token_logprobs(x.t(), torch.zeros(64, dtype=torch.int64, device=DEV),
                                              torch.zeros(64, device=DEV)),
        lambda: ops.detonation_token_logprobs(x[:1].expand(4, 64), y, o),
        lambda: ops.detonation_token_logprobs_backward(x, y, torch.zeros((4, 2), device=DEV), x),
        lambda: ops.detonation_token_logprobs_backward(x, y, torch.zeros((4, 2), device=DEV), x,
                                                       g_entropy=o),
        lambda: ops.detonation_token_logprobs_backward(x[:3], y[:3], torch.zeros((3, 2), device=DEV),
                                                       x[1:], g_logp=o[:3]),
        lambda: ops.detonation_norm_residual(ops.NormResidual(), x, None, None, x[:, :32]),
        lambda: ops.detonation_norm_residual(ops.NormResidual(), x, None, None, x.clone(),
                                             w_pre=torch.zeros(63, device=DEV)),
        lambda: ops.detonation_norm_residual(ops.NormResidual(), x, None, None, x.clone(),
                                             w_pre=torch.zeros(64, device=DEV),
                                             b_pre=torch.zeros(64, device=DEV, dtype=BF16)),
        lambda: ops.detonation_norm_residual(ops.NormResidual(rows_per_gate=2), x, x.clone(), x, x.clone(),
                                             gate=torch.zeros((1, 64), device=DEV)),
        lambda: ops.detonation_norm_residual_backward(ops.NormResidual(), x, None, x.clone(), None,
                                                      x.clone(), None, dw_pre=torch.zeros(64, device=DEV)),
        lambda: ops.detonation_act8_encode(x, empty_act8(4, 63)),
        lambda: ops.detonation_act8_encode(x, ops.Act8(x.to(torch.uint8), empty_act8(4, 64).exps)),
        lambda: ops.detonation_glu_forward(0, x, x.clone(), x.to(BF16)),
        lambda: ops.detonation_glu_backward(0, x, empty_act8(4, 64), empty_act8(3, 64), x, x.clone()),
        lambda: ops.detonation_act8_weight_grad(x, empty_act8(4, 32), torch.zeros((63, 32), device=DEV)),
        lambda: ops.detonation_act8_weight_grad(torch.zeros((999, 64), device=DEV), empty_act8(999, 32),
                                                torch.zeros((64, 32), device=DEV)),
    ]
    for i, f in enumerate(bad):
        with pytest.raises((ValueError, ops.DetonationError)):
            f()
            pytest.fail(f"call {i} was taken")
    with pytest.raises(ops.DetonationError):
        ops.detonation_glu_forward(7, x, None, x)
    with pytest.raises(ops.DetonationError):
        wide_rows = torch.zeros((1, 16385), device=DEV)
        ops.detonation_norm_residual(ops.NormResidual(), wide_rows, None, None, wide_rows.clone())
