"""The kernels behind include/detonation_model.h where their arithmetic has few bits to spare: widths that leave
lanes empty, values at the ends of a type's range, sums of many steps.  Plain definitions in 64 bits."""
import math

import pytest
import torch

from paper_2502_06728_amd import model_ops as ops
from tests import model_reference as ref
from tests import test_gpu_model_ops as base
from tests.model_reference import BF16, F16, F32, assert_near
from tests.test_gpu_model_ops import ACT, DEV, INF, NAN, TYPES, empty_act8, like, normal, rows, say, scratch

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


@pytest.mark.parametrize("dtype,far", [(F16, 3e4)] + [
    (dtype, far) for dtype in (F32, BF16) for far in (3e4, 1e5, 7e5, 1e6, 1e9, 1e10, 1e12, 1e20, 1e29, 1e31)])
@pytest.mark.parametrize("V", [2500, 20000, 50001])
@pytest.mark.parametrize("T", [12, 516])
def test_sums_of_rows_with_large_finite_values(gpu, dtype, far, V, T):
    """Masks that are neither a type's lowest value nor an infinity, as a lane sees them first, last, always or
    never, and rows whose largest values are of that size."""
    say(dtype, far, V, T)
    x = normal(V, 12, V, scale=2.0)
    at = torch.arange(V)
    x[0, :V // 2] = -far
    x[1, V // 2:] = -far
    x[2, at // 8 % 256 < 128] = -far                 # whole lanes
    x[3, at // 8 % 2 == 0] = -far
    x[4] = -far                                      # nothing else
    x[5, 1:] = -far
    x[6, [3, V // 2, V - 1]] = far                   # three share the row
    x[7] = far
    x[8, :V // 2], x[8, V // 2:] = -far, -far / 2
    x[9, :V // 3], x[9, V // 3:] = far / 2, far
    x[10] = -far * (1 + torch.rand(V, generator=torch.Generator().manual_seed(1)) * 0.25)
    x[11] += far / 16
    x = rows(x.repeat(-(-T // 12), 1)[:T], dtype)
    y = torch.randint(0, V, (T,), generator=torch.Generator().manual_seed(V)).to(DEV)
    y[6], y[5] = 3, 0
    keep = torch.arange(12)
    out = run_and_check_sums(x, y, 1.0, keep)
    for name in ("lse", "top_logp"):
        assert bool(torch.isfinite(out[name]).all())
    gl, ge = normal(1, T).float().to(DEV), normal(2, T).float().to(DEV)
    got = like(T, V, dtype)
    ops.detonation_token_logprobs_backward(x, y, out["stats"], got, g_logp=gl, entropy=out["entropy"], g_entropy=ge)
    want = ref.logprobs_grad(x[keep], y[keep], gl[keep], ge[keep])
    # probabilities of rows whose log s is known to V / 256 + 64 roundings of log V
    assert_near(got[keep], want, 4 * (2 + math.log(V)), V / 256 + 256, "dlogits")


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_sums_at_the_border_of_the_products_range(gpu, dtype):
    """Values on both sides of powers of two, a few units apart, in the order in which each lane's maximum
    rises."""
    V, T = 40000, 40
    x = torch.zeros((T, V), dtype=torch.float64)
    step = 2.0 ** (-23 if dtype == F32 else -7)
    for t in range(T):
        big = -2.0 ** (t // 2 + 10) if t % 2 else 2.0 ** (t // 2 + 10)
        x[t] = big * (1 + step * 3 * (torch.arange(V).double() / V - 0.5) * (-1 if t % 2 else 1)).float().double()
    x = rows(x, dtype)
    y = torch.randint(0, V, (T,), generator=torch.Generator().manual_seed(3)).to(DEV)
    run_and_check_sums(x, y)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("odd", [NAN, INF])
@pytest.mark.parametrize("T,V", [(6, 300), (6, 70001), (600, 300)])
def test_best_tokens_of_a_row_with_a_nan(gpu, dtype, odd, T, V):
    """logit - lse is NaN for every token of such a row, -infinite ones too."""
    x = normal(1, T, V)
    x[0, 2:] = -INF
    x[0, 1] = odd
    x[1, V - 1] = odd
    x[2, 1:] = -INF
    d = rows(x, dtype)
    y = torch.zeros(T, dtype=torch.int64, device=DEV)
    out = base.run_logprobs(d, y, 5)
    assert out["top_idx"][0].tolist() == [1, 0, 2, 3, 4] and out["top_idx"][2].tolist() == [0, 1, 2, 3, 4]
    assert bool(torch.isnan(out["top_logp"][:2]).all())
    assert out["top_logp"][2].tolist() == [0.0] + [-INF] * 4
    for name in ("logp", "lse", "entropy"):
        assert bool(torch.isnan(out[name][:2]).all()) and bool(torch.isfinite(out[name][2:]).all())


def test_logprobs_of_more_rows_than_a_launch_counts(gpu):
    """2^24 workgroups of 256 threads are one launch too many."""
    T, V = (1 << 24) + 5, 3
    g = torch.Generator(device=DEV).manual_seed(1)
    x = torch.randn((T, V), generator=g, device=DEV).to(BF16)
    y = torch.randint(-1, V, (T,), generator=g, device=DEV, dtype=torch.int32)
    out = {n: torch.full((T,), NAN, device=DEV) for n in ("logp", "entropy")}
    out["stats"] = torch.full((T, 2), NAN, device=DEV)
    best = torch.full((T, 1), -7, dtype=torch.int32, device=DEV)
    ops.detonation_token_logprobs(x, y, top_idx=best, **out)
    gl = torch.randn(T, generator=g, device=DEV)
    dx = torch.full((T, V), NAN, dtype=BF16, device=DEV)
    ops.detonation_token_logprobs_backward(x, y, out["stats"], dx, g_logp=gl, entropy=out["entropy"], g_entropy=gl)
    for n in (*out, "dlogits"):
        assert bool(torch.isfinite(dx if n == "dlogits" else out[n]).all()), n
    keep = torch.tensor([0, 1, (1 << 24) - 258, (1 << 24) - 257, (1 << 24) - 1, 1 << 24, T - 1], device=DEV)
    check_sums(x[keep], y[keep], {n: v[keep] for n, v in out.items()})
    assert torch.equal(best[keep, 0].cpu().long(), ref.logprobs(x[keep], y[keep], 1.0, 1)[3][:, 0])
    assert_near(dx[keep], ref.logprobs_grad(x[keep], y[keep], gl[keep], gl[keep]), 16.0, 256, "dlogits")


# ------------------------------------------------------------------ gated activations

@pytest.mark.parametrize("act", list(ACT))
def test_slopes_over_the_range_of_the_8_bit_form(gpu, act):
    """Every exponent of it: values up to fp32's largest, and down to its smallest."""
    exps = torch.arange(1, 249, dtype=torch.uint8)[:, None]
    codes = torch.zeros((248, 32), dtype=torch.int8)
    codes[:, :7] = torch.tensor([1, -1, 5, -5, 127, -127, 64], dtype=torch.int8)
    x = ref.act8_values(codes, exps)
    a8 = ops.Act8(codes.to(DEV), exps.to(DEV))
    dh, da = rows(torch.ones(248, 32), F32), like(248, 32, F32)
    ops.detonation_glu_backward(ACT[act], dh, a8, None, da)
    # beyond 100 every slope is 0 or 1; below, 64 roundings of a value of the argument's size
    assert_near(da, ref.act_slope(x.clamp(-100, 100), act), 1 + x.abs().clamp(max=100), 64, act)
    b8, db = empty_act8(248, 32), like(248, 32, F32)
    b8.codes.fill_(1)
    b8.exps.fill_(127)
    ops.detonation_glu_backward(ACT[act], dh, a8, b8, da, db)
    assert_near(da, ref.act_slope(x.clamp(-100, 100), act), 1 + x.abs().clamp(max=100), 64, act)
    h = like(248, 32, F32)
    ops.detonation_glu_forward(ACT[act], rows(x, F32), None, h)
    for got in (h, db):
        assert_near(got, ref.act(x, act), x.abs(), 64, act)


def test_silu_keeps_its_bits(gpu):
    """silu(x) of a negative x is x e^x / (1 + e^x): its bits are those of the exponential."""
    x = torch.linspace(-85, 85, 170 * 64 + 1, dtype=torch.float64)[:-1].float().double().view(-1, 64)
    h = like(*x.shape, F32)
    ops.detonation_glu_forward(ops.ACT_SILU, rows(x, F32), None, h)
    want = x * torch.sigmoid(x)
    # an exponential (two units in the last place), a sum, a quotient (two)
    assert bool(((ref.double(h) - want).abs() <= 8 * 2.0 ** -24 * want.abs()).all())
    codes = torch.arange(-127, 128, dtype=torch.int8).view(-1, 1).repeat(1, 32)
    a8 = ops.Act8(codes.to(DEV), torch.full((255, 1), 126, dtype=torch.uint8, device=DEV))
    v = ref.act8_values(a8.codes, a8.exps)
    dh, da = rows(torch.ones(255, 32), F32), like(255, 32, F32)
    ops.detonation_glu_backward(ops.ACT_SILU, dh, a8, None, da)
    # g (1 + x (1 - g)): the bracket is rounded at its terms' size
    g = torch.sigmoid(v)
    assert bool(((ref.double(da) - ref.act_slope(v, "silu")).abs() <= 16 * 2.0 ** -24 * g * (1 + v.abs())).all())


# ------------------------------------------------------------------ weight gradient

@pytest.mark.parametrize("T,N,K,out", [
    (136, 2051, 6101, F32), (136, 2051, 6101, BF16), (136, 2050, 6100, F16),     # one split; odd strides and whole words
    (8192, 2049, 2049, F32), (8192, 2049, 2049, BF16),                           # three splits, odd strides
    (8192, 2048, 2048, F32), (6000, 1537, 1791, F32)])                           # four; five, rows that end inside a step
@pytest.mark.parametrize("accumulate", [False, True])
def test_weight_grad_of_large_tiles(gpu, T, N, K, out, accumulate):
    """bf16 sizes at which tiles are 256 wide: rows at odd strides, T cut into several splits, sums added to what
    is there."""
    say(T, N, K, out, accumulate)
    g = torch.Generator(device=DEV).manual_seed(1)
    dy = torch.randn((T, N), generator=g, device=DEV).to(BF16)
    x8 = empty_act8(T, K)
    ops.detonation_act8_encode(torch.randn((T, K), generator=g, device=DEV), x8)
    start = torch.randn((N, K), generator=g, device=DEV).to(out)
    dw = like(N, K, out, 3)
    dw.copy_(start)
    ops.detonation_act8_weight_grad(dy, x8, dw, accumulate=accumulate,
                                    workspace=scratch(ops.act8_weight_grad_workspace(T, N, K)))
    base.untouched(dw)
    n = torch.cat([torch.arange(0, N, 61), torch.tensor([N - 1])])               # rows of every tile and of every block of 64
    d, v = ref.double(dy[:, n]).t().contiguous(), ref.act8_values(x8.codes, x8.exps)
    want, mag = d @ v, d.abs() @ v.abs()
    if accumulate:
        want, mag = want + ref.double(start[n]), mag + ref.double(start[n]).abs()
    # exact products added in any order, then the splits of T
    assert_near(dw[n], want, mag, T + 40, "dw")
