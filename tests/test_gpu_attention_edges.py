"""Attention where few tests go: sequences without queries under grouped heads, infinities that are seen, scores so large that
fp32 does not hold them to a unit, queries with few keys beside long sequences, calls without a workspace."""
import math

import pytest
import torch

from paper_2502_06728_amd import model_ops as ops
from tests import attention_reference as ref
from tests.model_reference import BF16, F16, F32
from tests.test_gpu_attention import Case, even
from tests.test_gpu_model_ops import DEV, INF, NAN, TYPES, say, untouched

pytestmark = pytest.mark.gpu


def defined(c):
    """out, lse, dq, dk and dv of a case of one sequence, all heads at once in 64 bits; infinite keys count as zeros in the
    product that gives dq.  And the size of what is added up in dq: of its terms, and of those of their differences."""
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
    terms = p * (g.abs() @ v.abs().transpose(1, 2).contiguous())
    k = torch.where(torch.isfinite(k), k, 0.0)
    dk, dv = (x.transpose(1, 2).contiguous() @ y for x, y in ((ds * c.cfg.scale, q), (p, g)))
    dk, dv = (t.unflatten(0, (K, H // K)).sum(1) for t in (dk, dv))
    return ({"out": together(out), "lse": torch.logsumexp(s, 2), "dq": together(ds @ k * c.cfg.scale), "dk": together(dk),
             "dv": together(dv)}, together((8 * ds.abs() + 2 * terms) @ k.abs() * c.cfg.scale))


def unit(dtype):
    """What a row of results may be off by, of its size (the type's own rounding, that of the weights, that of the written out:
    a third of u^2 each; in fp32 those of scores and of sums)."""
    return 64 * ref.FINE if dtype == F32 else ref.UNIT[dtype]


def assert_rows(got, want, u, what, low=0.0):
    """As a whole to u, each row to 4 u of its size or of the rows' mean size, and `low` more."""
    if got.dtype == F16:                                    # half of 2^-24 each is what a result below the normal range loses
        low += 2.0 ** -25 * got.shape[1] ** 0.5
    got = got.double()
    assert bool(torch.isfinite(got).all()), what
    off, size = (got - want).norm(dim=1), want.norm(dim=1)
    say(what, float(off.norm() / size.norm()) / u)
    assert float(off.norm()) <= u * float(size.norm()) + low * len(size) ** 0.5, what
    assert bool((off <= 4 * (u * torch.maximum(size, size.norm() / len(size) ** 0.5) + low)).all()), what


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


# ------------------------------------------------------------------ infinities that are seen

@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n,at,causal,heads,kv_heads,head_dim", [
    (150, 75, True, 2, 1, 64), (150, 140, False, 2, 1, 64), (150, 10, False, 2, 1, 128), (150, 149, False, 2, 2, 128),
    (140, 130, True, 4, 1, 128), (600, 595, True, 2, 2, 128), (150, 64, True, 2, 2, 33), (2100, 2090, True, 32, 8, 128)])
def test_key_of_minus_infinity(gpu, dtype, n, at, causal, heads, kv_heads, head_dim):
    """A key that makes a score -infinity has no weight: only its own feature of a query's gradient is 0 * infinity, the others
    and the other keys' gradients are as if it were not there.  Whether the step is masked or not."""
    feature = 5
    c = Case(dtype, [0, n], [0, n], heads, kv_heads, head_dim, causal, packed=False)
    c.q[:, feature::head_dim] = c.q[:, feature::head_dim].abs() + 0.25
    c.k[at, feature::head_dim] = -INF
    c.forward()
    c.backward()
    want, _ = defined(c)
    u = unit(dtype)
    other = torch.arange(heads * head_dim, device=DEV) % head_dim != feature
    assert_rows(c.out, want["out"], u, "out")
    assert_rows(c.dq[:, other], want["dq"][:, other], u, "dq")
    assert_rows(c.dk, want["dk"], u, "dk")
    assert_rows(c.dv, want["dv"], u, "dv")
    assert not bool(c.dk[at].any()) and not bool(c.dv[at].any())
    seen = torch.arange(n, device=DEV) >= (at if causal else 0)
    assert bool(torch.isnan(c.dq[seen][:, ~other]).all())
    if causal:
        assert_rows(c.dq[:at], want["dq"][:at], u, "dq of those that do not see it")


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("bad", [INF, -INF, NAN])
def test_four_heads_and_infinities(gpu, dtype, bad):
    """Groups of four heads: a row that holds infinities or NaNs changes the gradients of what it sees alone, whichever of
    the four it belongs to."""
    at, n = 75, 150
    fine = Case(dtype, [0, n, 2 * n], [0, n, 2 * n], 4, 1, 128, True)
    fine.forward()
    fine.backward()
    for head in (0, 3):
        for name in ("q", "dout"):
            c = Case(dtype, [0, n, 2 * n], [0, n, 2 * n], 4, 1, 128, True)
            getattr(c, name)[at, 128 * head + 7:128 * (head + 1):9] = bad
            c.forward()
            c.backward()
            assert torch.equal(c.dk[at + 1:], fine.dk[at + 1:]) and torch.equal(c.dv[at + 1:], fine.dv[at + 1:]), (head, name)
            assert not bool(torch.isfinite((c.dk if name == "q" else c.dv)[:at + 1, 7::9]).any()), (head, name)
            same = torch.arange(2 * n, device=DEV) != at
            assert torch.equal(c.dq[same], fine.dq[same]), (head, name)


@pytest.mark.parametrize("dtype", TYPES)
def test_hundreds_of_sequences(gpu, dtype):
    """Tiles are counted 64 sequences at a time: a few hundred, some of none, and a long one at the end."""
    starts = [0]
    for s in range(300):
        starts.append(starts[-1] + s % 5)
    starts.append(starts[-1] + 200)
    c = Case(dtype, starts, starts, 2, 1, 64, True, behind=3)
    c.forward()
    c.backward()
    c.check()


# ------------------------------------------------------------------ scores of any size

def far_case(dtype, n, m, causal, heads, kv_heads, head_dim, q0, k0, k1, scale, **layout):
    """Scores scale * (q0 * k0[j] + k1[j]), whose sums fp32 holds exactly; the other features of the keys do not count, as
    those of the queries are zeros."""
    c = Case(dtype, [0, n], [0, m], heads, kv_heads, head_dim, causal, packed=False, scale=scale, **layout)
    c.q.zero_()
    c.q[:, 0::head_dim] = q0
    c.q[:, 1::head_dim] = 1.0
    j = torch.arange(m)
    c.k[:, 0::head_dim] = k0(j).to(dtype).to(DEV)[:, None]
    c.k[:, 1::head_dim] = k1(j).to(dtype).to(DEV)[:, None]
    c.dout.mul_(2.0 ** -6)
    return c


# name: q0, k0, k1, scale.  63 is no power of two, so a score's product with a factor is rounded, by up to half of
#   a million 2^-4, 8 million 1/2, 2,000 million 2^7, 2^116 2^92     (in powers of two)
SCORES = {"a million": (9 * 2.0 ** 7, lambda j: 7 * 2.0 ** 7 + 0 * j, lambda j: j * 31 % 97 / 8, 1.0),
          "minus a million": (-9 * 2.0 ** 7, lambda j: 7 * 2.0 ** 7 + 0 * j, lambda j: j * 31 % 97 / 8, 1.0),
          "8 million": (9 * 2.0 ** 10, lambda j: 7 * 2.0 ** 7 + 0 * j, lambda j: j * 3 % 4, 1.0),
          "2,000 million": (9 * 2.0 ** 10, lambda j: torch.where(j % 50 == 33, 7, 6) * 2.0 ** 10, lambda j: 0.0 * j, 32.0),
          "minus 2,000 million": (-9 * 2.0 ** 10, lambda j: torch.where(j % 50 == 33, 7, 8) * 2.0 ** 10, lambda j: 0.0 * j, 32.0),
          "2^116": (9 * 2.0 ** 10, lambda j: torch.where(j % 50 == 33, 7, 6) * 2.0 ** 10, lambda j: 0.0 * j, 2.0 ** 90)}
LENGTHS = [(150, 150, True, 2, 1, 64), (40, 700, False, 2, 2, 128), (1, 2111, False, 2, 2, 64), (600, 600, True, 4, 1, 128),
           (33, 1111, True, 2, 2, 80)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("name", SCORES)
@pytest.mark.parametrize("n,m,causal,heads,kv_heads,head_dim", LENGTHS)
def test_far_scores(gpu, dtype, name, n, m, causal, heads, kv_heads, head_dim):
    """Finite scores of any size: weights depend on their differences alone, which are small, or so large that only the
    best keys count, alike."""
    c = far_case(dtype, n, m, causal, heads, kv_heads, head_dim, *SCORES[name])
    c.forward()
    want, size = defined(c)
    u = unit(dtype)
    assert_rows(c.out, want["out"], u, "out")
    # two roundings of a sum as large as lse itself, and its own
    assert bool(((c.lse.double() - want["lse"]).abs() <= 2.0 ** -22 * want["lse"].abs()).all())


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n,m,causal,heads,kv_heads,head_dim", LENGTHS)
def test_scores_above_fp32(gpu, dtype, n, m, causal, heads, kv_heads, head_dim):
    """The product of q and k is a number, that with the scale is not: the best keys are."""
    c = far_case(dtype, n, m, causal, heads, kv_heads, head_dim, *SCORES["2,000 million"][:3], 2.0 ** 110)
    c.forward()
    assert_rows(c.out, defined(c)[0]["out"], unit(dtype), "out")
    assert bool((c.lse == INF).all())


def check_far_gradients(c):
    want, size = defined(c)
    dtype, heads, kv_heads, head_dim = c.dtype, c.cfg.heads, c.cfg.kv_heads, c.cfg.head_dim
    n, m, u = len(c.q), len(c.k), unit(dtype)
    # what fp16 does not hold is infinite; below its normal range p and ds are off by half of 2^-24 each, at random, and their
    # sums by the root of as many times the other operand's size
    low = 2.0 ** -25 if dtype == F16 else 0.0
    group = heads // kv_heads
    gradient = low * c.cfg.scale * (group * n) ** 0.5 * float(c.q.abs().max()) * 2 ** 0.5
    fits = want["dk"].abs().amax(1) < 0.99 * torch.finfo(dtype).max
    assert_rows(c.dv, want["dv"], u, "dv", low * (group * n * head_dim) ** 0.5 * 4 * 2.0 ** -6)
    assert_rows(c.dk[fits], want["dk"][fits], u, "dk", gradient)
    # where all keys are alike, a query's gradients cancel out, to what the terms of dout . v and dout . out are off by (those
    # of a definition in 64 bits to 2^-44)
    first = torch.arange(heads * head_dim, device=DEV) % head_dim == 0
    cancel = low * c.cfg.scale * m ** 0.5 * float(c.k.abs().max())
    assert bool(((c.dq.double() - want["dq"]).abs() <= u * size + 2.0 ** -44 * size.max() + 4 * cancel)[:, first].all())
    few = c.k.clone()
    few[:, 0::head_dim] = 0.0
    assert_rows(c.dq[:, ~first], want["dq"][:, ~first], u, "dq", low * c.cfg.scale * float(few.double().norm()))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("name", SCORES)
@pytest.mark.parametrize("n,m,causal,heads,kv_heads,head_dim", LENGTHS)
def test_gradients_of_far_scores(gpu, dtype, name, n, m, causal, heads, kv_heads, head_dim):
    """The same of the gradients: lse, which they take, is known to a rounding of its size alone."""
    if dtype == F16 and name == "2^116":
        pytest.skip("above fp16's largest value")
    c = far_case(dtype, n, m, causal, heads, kv_heads, head_dim, *SCORES[name])
    c.forward()
    c.backward()
    check_far_gradients(c)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("n,m,causal,heads,kv_heads,head_dim", LENGTHS)
def test_gradient_of_values_where_scores_are_above_fp32(gpu, dtype, n, m, causal, heads, kv_heads, head_dim):
    c = far_case(dtype, n, m, causal, heads, kv_heads, head_dim, *SCORES["2,000 million"][:3], 2.0 ** 110)
    c.forward()
    c.backward()
    assert_rows(c.dv, defined(c)[0]["dv"], unit(dtype), "dv")


@pytest.mark.parametrize("dtype", TYPES)
def test_far_queries_among_others(gpu, dtype):
    """One query of a block has scores of a million: the others' gradients keep their bits."""
    n, at = 200, 77
    c, other = (Case(dtype, [0, n], [0, n], 4, 2, 128, True, packed=False) for _ in range(2))
    other.dout[at] = 0.0
    other.q[at] *= 2.0 ** (10 if dtype == F16 else 17)
    c.dout[at] = 0.0
    for x in (c, other):
        x.forward()
        x.backward()
    assert float(other.lse[:, at].abs().min()) > 1000
    same = torch.arange(n, device=DEV) != at
    for name in ("out", "dq"):
        assert torch.equal(getattr(c, name)[same], getattr(other, name)[same]), name
    # (weights of the query that is different times nothing)
    assert torch.equal(c.dk, other.dk) and torch.equal(c.dv, other.dv)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n,causal,heads,kv_heads,head_dim", [(150, True, 2, 1, 64), (150, False, 4, 1, 128), (70, True, 4, 2, 128)])
def test_far_scores_and_infinities(gpu, dtype, n, causal, heads, kv_heads, head_dim):
    """Both at once: a key without weight, and a row of gradients that is no number."""
    at = 66
    c = far_case(dtype, n, n, causal, heads, kv_heads, head_dim, *SCORES["a million"])
    c.k[at, 0::head_dim] = -INF
    c.forward()
    c.backward()
    want, _ = defined(c)
    u = unit(dtype)
    later = torch.arange(head_dim * heads, device=DEV) % head_dim >= 2
    low = 2.0 ** -25 * n ** 0.5 * 4 if dtype == F16 else 0.0
    assert_rows(c.out, want["out"], u, "out")
    assert_rows(c.dv, want["dv"], u, "dv", low)
    assert_rows(c.dk, want["dk"], u, "dk", low * float(c.q.abs().max()))
    assert_rows(c.dq[:, later], want["dq"][:, later], u, "dq", low * head_dim ** 0.5)
    assert not bool(c.dk[at].any()) and not bool(c.dv[at].any())
    dk, dv, dq = c.dk.clone(), c.dv.clone(), c.dq.clone()
    c.dout[at, 7::9] = NAN
    c.backward()
    same = torch.arange(n, device=DEV) != at
    assert torch.equal(torch.nan_to_num(c.dq[same], 7.0), torch.nan_to_num(dq[same], 7.0))
    if causal:
        assert torch.equal(c.dk[at + 1:], dk[at + 1:]) and torch.equal(c.dv[at + 1:], dv[at + 1:])
    assert bool(torch.isnan(c.dv[:at + 1, 7:head_dim:9]).all()) and bool(torch.isnan(c.dq[at]).all())


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n,m,causal,heads,kv_heads,head_dim,pad,offset", [
    (150, 150, True, 2, 1, 33, 0, 0), (300, 300, True, 4, 2, 128, 3, 1), (1, 1111, False, 2, 2, 65, 0, 5), (40, 700, False, 2, 1, 96, 7, 3)])
def test_far_scores_from_any_address(gpu, dtype, n, m, causal, heads, kv_heads, head_dim, pad, offset):
    """The same where rows start at odd elements, or heads are no whole pieces: both ways, and a replayed graph of them."""
    c = far_case(dtype, n, m, causal, heads, kv_heads, head_dim, *SCORES["2,000 million"], pad=pad, offset=offset)
    c.forward()
    c.backward()
    assert_rows(c.out, defined(c)[0]["out"], unit(dtype), "out")
    check_far_gradients(c)
    for name in ("out", "dq", "dk", "dv"):
        untouched(getattr(c, name))
    want = {name: t.clone() for name, t in c.results().items()}
    stream, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.stream(stream):
        graph.capture_begin()
        c.forward(stream)
        c.backward(stream)
        graph.capture_end()
    for _ in range(3):
        for t in (*c.results().values(), c.ws):
            t.fill_(0)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(t, want[name]) for name, t in c.results().items())


# ------------------------------------------------------------------ few keys

@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("head_dim", [64, 128])
@pytest.mark.parametrize("n", [3, 600])
def test_an_only_key_gets_no_gradient(gpu, dtype, head_dim, n):
    """The first query sees one key, whose weight is 1 whatever its score: alone it brings no gradient to any key."""
    c = Case(dtype, [0, n], [0, n], 2, 1, head_dim, True, packed=False)
    c.dout[1:] = 0.0
    c.forward()
    c.backward()
    assert not bool(c.dk.any()) and not bool(c.dq.any())


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("head_dim", [64, 128])
@pytest.mark.parametrize("n", [3, 600])
@pytest.mark.parametrize("bad", [INF, NAN])
def test_an_only_key_and_a_nan(gpu, dtype, head_dim, n, bad):
    """... but where the gradient of its output is no number, its own is none."""
    c = Case(dtype, [0, n], [0, n], 2, 1, head_dim, True, packed=False)
    c.dout[0, ::7] = bad
    c.forward()
    c.backward()
    assert bool(torch.isnan(c.dq[0]).all())


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("heads,kv_heads,head_dim,causal", [
    (2, 2, 128, False), (4, 2, 104, False), (2, 1, 64, False), (4, 1, 128, True), (2, 1, 127, False)])
def test_short_sequences_beside_long_ones(gpu, dtype, heads, kv_heads, head_dim, causal):
    """The gradients of a short sequence are as exact as without its neighbours."""
    short, n = 30, 2
    starts = [n * i for i in range(short + 1)] + [n * short + 2000 * (i + 1) for i in range(11)]
    c = Case(dtype, starts, starts, heads, kv_heads, head_dim, causal)
    c.q.mul_(2.0)                                           # weights that differ
    c.forward()
    c.backward()
    m = n * short
    want = ref.whole(c.q[:m], c.k[:m], c.v[:m], c.dout[:m], heads, kv_heads, c.cfg.scale, causal, short)
    for name in ("out", "dq", "dk", "dv"):
        assert_rows(getattr(c, name)[:m], want[name], unit(dtype), name)


@pytest.mark.parametrize("dtype,heads,kv_heads,head_dim,L", [
    (BF16, 32, 8, 128, 2100), (F16, 16, 16, 128, 1000), (BF16, 64, 16, 104, 700), (BF16, 2, 2, 128, 2000)])
def test_the_first_queries_of_a_long_sequence(gpu, dtype, heads, kv_heads, head_dim, L):
    """Those that see a few keys, apart from the others."""
    c = Case(dtype, [0, L], [0, L], heads, kv_heads, head_dim, True, packed=False)
    c.q.mul_(2.0)
    c.forward()
    c.backward()
    n = 4
    w = ref.whole(c.q[:n], c.k[:n], c.v[:n], c.dout[:n], heads, kv_heads, c.cfg.scale, True, 1)
    assert_rows(c.dq[1:n], w["dq"][1:], unit(dtype), "dq")


# ------------------------------------------------------------------ refusals

def test_backward_refuses_before_it_writes(gpu):
    """Few queries, more tiles of keys than a launch counts: nothing was written."""
    T, H = 1 << 16, 64
    q, k = (torch.ones((n, H), dtype=BF16, device=DEV) for n in (1, T))
    out, dq, dk, dv = (torch.full_like(t, NAN) for t in (q, q, k, k))
    cfg = ops.Attention(heads=H, head_dim=1, scale=1.0, causal=False, sequences=T)
    qs = torch.zeros(T + 1, dtype=torch.int32, device=DEV)
    qs[1:] = 1
    ks = torch.arange(T + 1, dtype=torch.int32, device=DEV)
    ws = torch.full((ops.attention_workspace(cfg, 1, T),), 0xFF, dtype=torch.uint8, device=DEV)
    lse = torch.zeros((H, 1), device=DEV)
    with pytest.raises(ops.DetonationError):
        ops.detonation_attention_backward(cfg, q, k, k, q, lse, q, dq, dk, dv, q_starts=qs, k_starts=ks, workspace=ws)
    torch.cuda.synchronize()
    assert bool(torch.isnan(dq).all()) and bool((ws == 0xFF).all())


@pytest.mark.parametrize("dtype", TYPES)
def test_forward_without_a_workspace(gpu, dtype):
    """A call that does not cut its walks needs none; one that does is refused."""
    c = Case(dtype, even(3, 40), even(3, 40), 2, 1, 64, True)
    c.forward()
    want = c.out.clone()
    c.clear()
    c.ws = None
    c.forward()
    assert torch.equal(c.out, want)
    c = Case(dtype, [0, 1], [0, 3000], 2, 1, 64, False)
    c.ws = None
    with pytest.raises(ops.DetonationError):
        c.forward()
    torch.cuda.synchronize()
    assert bool(torch.isnan(c.out).all())


# ------------------------------------------------------------------ weights below fp16's range

@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("first,n", [(2, 40), (99, 1), (4090, 200)])
def test_many_light_keys(gpu, dtype, first, n):
    """One key outweighs each of the others by nearly 2^21, and all of them by 2^4 alone: what they add up to is there."""
    m, scale = 1 << 17, 1.0
    c = Case(dtype, [0, n], [0, m], 1, 1, 16, False, packed=False, scale=scale)
    c.q.zero_()
    c.q[:, 0] = 1.0
    c.k.zero_()
    c.k[first, 0] = 14.5                                    # 2^21 = exp(14.56)
    c.v.fill_(1.0)
    c.v[first, ::2] = 0.0                                   # (odd features: the weights' sum)
    c.forward()
    rest = (m - 1) * math.exp(-14.5)
    light = rest / (1 + rest)
    # rounding of the result, and of weights, all alike: half a step each; sums of 4,096 steps of fp32
    u = ref.UNIT[dtype] * 2 + (m / 32 + 64) * ref.FINE
    assert bool(((c.out[:, ::2].double() - light).abs() <= u * light).all()), (float(c.out[0, 0]), light)
    assert bool(((c.out[:, 1::2].double() - 1).abs() <= u).all())
