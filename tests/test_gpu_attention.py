"""Attention behind include/detonation_model.h against its definition in 64 bits: types, head layouts, lengths, masks that
leave nothing, packed sequences, what masked places hold, gradients also against differences."""
import math

import pytest
import torch

from paper_2502_06728_amd import model_ops as ops
from tests import attention_reference as ref
from tests.model_reference import BF16, F16, F32
from tests.test_gpu_model_ops import DEV, NAN, INF, like, normal, rows, say, scratch, untouched

pytestmark = pytest.mark.gpu
TYPES = [F32, BF16, F16]


class Case:
    """Inputs of one call; outputs are filled with NaN."""

    def __init__(self, dtype, starts_q, starts_k, heads, kv_heads, head_dim, causal, pad=0, offset=0, behind=0, seed=0,
                 packed=True, scale=None):
        self.dtype, self.pad, self.offset = dtype, pad, offset
        self.starts_q, self.starts_k = starts_q, starts_k
        n = len(starts_q) - 1
        self.cfg = ops.Attention(heads=heads, kv_heads=kv_heads, head_dim=head_dim, causal=causal, sequences=n,
                                 scale=head_dim ** -0.5 if scale is None else scale)
        Tq, Tk = starts_q[-1] + behind, starts_k[-1] + behind
        W, N = heads * head_dim, kv_heads * head_dim
        self.q, self.dout = (rows(normal(seed + i, Tq, W), dtype, pad, offset) for i in (1, 2))
        self.k, self.v = (rows(normal(seed + i, Tk, N), dtype, pad, offset) for i in (3, 4))
        for t, used in ((self.q, starts_q), (self.dout, starts_q), (self.k, starts_k), (self.v, starts_k)):
            t[used[-1]:] = NAN                      # padding behind the last sequence
            t[:used[0]] = NAN
        self.starts = {}
        if packed:
            self.starts = {"q_starts": torch.tensor(starts_q, dtype=torch.int32, device=DEV),
                           "k_starts": torch.tensor(starts_k, dtype=torch.int32, device=DEV)}
        self.ws = scratch(ops.attention_workspace(self.cfg, Tq, Tk))
        self.clear()

    def clear(self):
        def empty(t):
            return like(*t.shape, self.dtype, self.pad, self.offset)
        self.out, self.dq, self.dk, self.dv = empty(self.q), empty(self.q), empty(self.k), empty(self.k)
        self.lse = torch.full((self.cfg.heads, len(self.q)), NAN, device=DEV)

    def forward(self, stream=None):
        ops.detonation_attention_forward(self.cfg, self.q, self.k, self.v, self.out, lse=self.lse, workspace=self.ws,
                                         stream=stream, **self.starts)

    def backward(self, stream=None):
        ops.detonation_attention_backward(self.cfg, self.q, self.k, self.v, self.out, self.lse, self.dout, self.dq, self.dk,
                                          self.dv, workspace=self.ws, stream=stream, **self.starts)

    def results(self):
        return {n: getattr(self, n) for n in ("out", "lse", "dq", "dk", "dv")}

    def check(self):
        c = self.cfg
        want = ref.attention(self.q, self.k, self.v, self.out, self.lse, self.dout, c.heads, c.kv_heads, c.head_dim, c.scale,
                             c.causal, self.starts_q, self.starts_k)
        for n, got in self.results().items():
            ref.assert_within(got, *want[n], n)
            if n != "lse":
                untouched(got)


def even(sequences, length):
    return [i * length for i in range(sequences + 1)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("sequences,Lq,Lk,heads,kv_heads,head_dim,causal,pad,offset", [
    (1, 1, 1, 1, 1, 64, True, 0, 0), (1, 1, 1, 1, 1, 1, False, 0, 0), (2, 3, 3, 2, 1, 128, True, 0, 0),
    (1, 33, 33, 2, 2, 64, True, 8, 0), (1, 129, 129, 1, 1, 128, True, 0, 0), (3, 65, 65, 2, 2, 64, False, 0, 8),
    (1, 257, 257, 4, 2, 80, True, 1, 3), (2, 128, 128, 2, 2, 128, True, 0, 0), (1, 5, 300, 2, 1, 128, True, 0, 0),
    (2, 1, 200, 3, 3, 96, True, 7, 1), (1, 300, 5, 2, 2, 64, True, 0, 0), (1, 140, 96, 2, 1, 7, False, 0, 5),
    (2, 64, 192, 8, 1, 32, True, 0, 0), (1, 1, 1100, 2, 2, 64, False, 0, 0), (1, 31, 64, 1, 1, 127, True, 2, 0),
    (1, 96, 160, 2, 2, 65, False, 0, 0), (1, 200, 200, 1, 1, 33, True, 3, 1), (2, 3, 700, 4, 2, 128, True, 0, 0),
    (1, 150, 1500, 2, 1, 64, True, 0, 0), (1, 1, 2111, 2, 2, 7, True, 1, 1)])
def test_attention(gpu, dtype, sequences, Lq, Lk, heads, kv_heads, head_dim, causal, pad, offset):
    say(dtype, sequences, Lq, Lk, heads, kv_heads, head_dim, causal)
    c = Case(dtype, even(sequences, Lq), even(sequences, Lk), heads, kv_heads, head_dim, causal, pad, offset, packed=False)
    c.forward()
    c.backward()
    c.check()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("starts_q,starts_k,heads,kv_heads,head_dim,causal", [
    ([0, 40, 40, 41, 170, 170, 300], None, 2, 2, 64, True),           # of none, of one, of more than a tile
    ([3, 60, 200], None, 4, 1, 128, True),                            # rows in front of the first one
    ([0, 10, 150, 150, 160], [0, 0, 130, 190, 333], 2, 1, 64, True),  # without keys; without queries
    ([0, 200, 231], [0, 7, 107], 3, 3, 72, False),
    ([0, 150, 160], [0, 30, 200], 2, 2, 128, True),                   # queries that see nothing
    (list(range(0, 71)) + [200], None, 1, 1, 64, True)])              # more than 64 sequences
def test_packed_sequences(gpu, dtype, starts_q, starts_k, heads, kv_heads, head_dim, causal):
    say(dtype, starts_q, starts_k)
    c = Case(dtype, starts_q, starts_k or starts_q, heads, kv_heads, head_dim, causal, behind=13)
    c.forward()
    c.backward()
    c.check()


@pytest.mark.parametrize("dtype", TYPES)
def test_no_keys_at_all(gpu, dtype):
    c = Case(dtype, [0, 40], [0, 0], 2, 2, 64, False, packed=False)
    c.forward()
    c.backward()
    assert bool((c.out == 0).all()) and bool((c.lse == -INF).all()) and bool((c.dq == 0).all())
    c = Case(dtype, [0, 0], [0, 40], 2, 2, 64, False, packed=False)
    c.forward()
    c.backward()
    assert bool((c.dk == 0).all()) and bool((c.dv == 0).all())


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("head_dim", [64, 128])
@pytest.mark.parametrize("bad", [INF, -INF, NAN])
def test_what_is_not_seen_does_not_reach(gpu, dtype, head_dim, bad):
    """A row that holds infinities or NaNs changes only what sees it (or is seen by it)."""
    at, n = 75, 150
    fine = Case(dtype, [0, n, 2 * n], [0, n, 2 * n], 2, 1, head_dim, True)
    fine.forward()
    fine.backward()
    for name in ("v", "k", "q", "dout"):
        c = Case(dtype, [0, n, 2 * n], [0, n, 2 * n], 2, 1, head_dim, True)
        t = getattr(c, name)
        t[at, ::5] = bad
        c.forward()
        c.backward()
        later, earlier = torch.arange(2 * n, device=DEV) >= at, torch.arange(2 * n, device=DEV) <= at
        later[n:] = False                                   # the other sequence
        earlier[n:] = False
        one = torch.arange(2 * n, device=DEV) == at
        # rows that may change, by what is odd
        may = {"v": {"out": later, "dq": later, "dk": ~(~earlier & ~later), "dv": one & ~one},
               "k": {"out": later, "dq": later, "dk": earlier | later, "dv": earlier | later},
               "q": {"out": one, "dq": one, "dk": earlier, "dv": earlier},
               "dout": {"out": one & ~one, "dq": one, "dk": earlier, "dv": earlier}}[name]
        for o, changed in may.items():
            a, b = getattr(c, o), getattr(fine, o)
            assert torch.equal(a[~changed], b[~changed]), (name, o)
        if name == "v":                                     # and what sees it, is reached
            column = torch.arange(2 * head_dim, device=DEV) % head_dim % 5 == 0       # of either head
            assert not bool(torch.isfinite(c.out[at:n, column]).any())
            assert torch.equal(c.out[at:n, ~column], fine.out[at:n, ~column])
        if name == "dout":
            assert not bool(torch.isfinite(c.dv[:at + 1, ::5]).any())
            assert torch.equal(c.dv[at + 1:], fine.dv[at + 1:])


@pytest.mark.parametrize("dtype", TYPES)
def test_large_scores(gpu, dtype):
    """Scores of hundreds, and rows whose scores are all equal or -infinity."""
    c = Case(dtype, [0, 130], [0, 130], 2, 2, 64, True, packed=False, scale=4.0)
    c.k[:, :64] = 0.0                                       # head 0: all keys alike
    c.forward()
    c.backward()
    c.check()
    c = Case(dtype, [0, 40], [0, 40], 1, 1, 64, False, packed=False)
    c.q[:20] = 1.0
    c.q[20:] = -1.0
    c.k[:] = -INF
    c.forward()
    assert bool((c.out[:20] == 0).all()) and bool((c.lse[:, :20] == -INF).all())
    assert bool(torch.isnan(c.out[20:]).all())


@pytest.mark.parametrize("dtype", TYPES)
def test_rising_scores(gpu, dtype):
    """Every step's keys outweigh those before: the running maximum moves, by little and by much."""
    for step in (0.02, 3.0):
        c = Case(dtype, [0, 40], [0, 700], 1, 1, 64, False, packed=False, scale=1.0)
        c.q.zero_()
        c.q[:, 0] = 1.0
        c.k.zero_()
        c.k[:, 0] = (torch.arange(700) * step / 8).to(dtype).to(DEV)
        c.forward()
        c.backward()
        c.check()


def test_gradient_against_differences(gpu):
    """fp32, directions at random: the derivative of sum(dout * out), which differences give to h^2."""
    c = Case(F32, [0, 37, 90], [0, 50, 131], 2, 1, 24, True)
    c.forward()
    c.backward()

    def value(name, by):
        d = Case(F32, [0, 37, 90], [0, 50, 131], 2, 1, 24, True)
        getattr(d, name).copy_((getattr(c, name).double() + by).float())
        d.forward()
        return float((d.out.double() * d.dout.double()).sum())
    for i, name in enumerate(("q", "k", "v")):
        t = getattr(c, name)
        direction = normal(50 + i, *t.shape).to(DEV)
        h = 2.0 ** -7
        slope = (value(name, h * direction) - value(name, -h * direction)) / (2 * h)
        want = float((getattr(c, "d" + name).double() * direction).sum())
        # sums of some 4,000 fp32 products, off by 2^-20 of their size over 2 h, and h^2 of a third derivative
        size = float((c.out.double().abs() * c.dout.double().abs()).sum())
        assert abs(slope - want) < size * (2.0 ** -20 / h + 30 * h * h), (name, slope, want)


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_long_rows_apart(gpu, dtype):
    """Rows so far apart that their places pass 2^32 bytes."""
    T, pad = 130, 1 << 25
    c = Case(dtype, [0, T], [0, T], 1, 1, 64, True)
    far = {}
    for n in ("q", "k", "v", "dout", "out", "dq", "dk", "dv"):
        flat = torch.empty((T * pad,), dtype=dtype, device=DEV) if n in ("q", "dk") else None
        if flat is not None:
            far[n] = flat.view(T, pad)[:, :64]
            far[n].copy_(getattr(c, n))
    c.forward()
    c.backward()
    want = {n: t.clone() for n, t in c.results().items()}
    c.clear()
    c.q, c.dk = far["q"], far["dk"]
    c.forward()
    c.backward()
    for n, t in c.results().items():
        assert torch.equal(t, want[n]), n


def test_long_sequence(gpu):
    """A few queries of a long sequence, and many keys to a query."""
    L = 20011
    c = Case(BF16, [0, L], [0, L], 1, 1, 64, True, packed=False)
    c.forward()
    for i in (0, 64, 1023, 10007, L - 1):
        q, k, v = c.q[i].double(), c.k[:i + 1].double(), c.v[:i + 1].double()
        s = (k @ q) * c.cfg.scale
        p = torch.softmax(s, 0)
        assert abs(float(c.lse[0, i]) - float(torch.logsumexp(s, 0))) < 1e-5
        bound = 2.0 ** -8 * 1.1 * (p @ v.abs() + (p @ v).abs()) + 1e-6
        assert bool(((c.out[i].double() - p @ v).abs() <= bound).all()), i


@pytest.mark.parametrize("dtype,sequences,L,heads,kv_heads,head_dim,causal", [
    (BF16, 1, 2100, 32, 8, 128, True), (F16, 1, 2100, 32, 32, 128, False), (BF16, 20, 130, 16, 8, 128, True),
    (BF16, 9, 1000, 32, 8, 128, True), (F16, 9, 1000, 16, 8, 96, False), (BF16, 1, 2100, 32, 32, 96, True),
    (BF16, 20, 130, 16, 16, 64, False), (BF16, 9, 1000, 16, 2, 40, True), (F32, 1, 2100, 32, 4, 128, True),
    (F32, 20, 130, 16, 16, 128, False), (BF16, 30, 2, 8, 2, 64, False), (F16, 50, 2, 4, 4, 128, False),
    (BF16, 50, 3, 4, 1, 96, True), (F32, 50, 3, 4, 2, 32, True)])
def test_as_exact_as_the_type(gpu, dtype, sequences, L, heads, kv_heads, head_dim, causal):
    """Results are rounded, and so are the weights (or their gradients) that are multiplied: two errors spread over half a
    step u, u / sqrt(3) each, as is a third that the written `out` may bring into the gradients: u together.  In fp32 a
    score of 64 additions of partial sums around 2 is off by some sqrt(64) half units, its product with a factor and lse
    by up to 16 each, and a sum over 2,100 terms by sqrt(2100) / 4: 64 together.  A row has 4 times as much of its own."""
    check_whole(dtype, sequences, L, heads, kv_heads, head_dim, causal)


@pytest.mark.parametrize("dtype,sequences,L,heads,kv_heads,head_dim,causal,pad", [
    (BF16, 1, 2100, 32, 8, 128, True, 1), (F16, 9, 1000, 16, 8, 96, True, 3), (BF16, 20, 130, 16, 16, 127, False, 0),
    (F32, 1, 2100, 32, 32, 99, False, 0)])
def test_as_exact_from_any_address(gpu, dtype, sequences, L, heads, kv_heads, head_dim, causal, pad):
    """The same where rows start at odd elements, or heads are no whole pieces."""
    check_whole(dtype, sequences, L, heads, kv_heads, head_dim, causal, pad)


def check_whole(dtype, sequences, L, heads, kv_heads, head_dim, causal, pad=0):
    n = sequences * L
    c = Case(dtype, even(sequences, L), even(sequences, L), heads, kv_heads, head_dim, causal, pad, packed=False)
    c.q.mul_(2.0)                                    # scores of a standard deviation of two
    c.forward()
    c.backward()
    want = ref.whole(c.q, c.k, c.v, c.dout, heads, kv_heads, c.cfg.scale, causal, sequences)
    u = 64 * ref.FINE if dtype == F32 else ref.UNIT[dtype]
    for name, w in want.items():
        got = getattr(c, name).double()
        assert got.shape == w.shape == (n, w.shape[1])
        off, size = (got - w).norm(dim=1), w.norm(dim=1)
        say(name, float(off.norm() / size.norm()) / u)
        assert float(off.norm()) <= u * float(size.norm()), name
        assert bool((off <= 4 * u * torch.maximum(size, size.norm() / n ** 0.5)).all()), name


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("head_dim", [64, 128])
@pytest.mark.parametrize("Lq,Lk,causal", [(1, 1, True), (300, 1, False), (7, 7, True), (3, 1, True), (600, 600, True)])
def test_one_key(gpu, dtype, head_dim, Lq, Lk, causal):
    """The weight of a query's only key is 1 whatever its score: no gradient reaches the query."""
    c = Case(dtype, [0, Lq], [0, Lk], 2, 1, head_dim, causal)
    c.forward()
    c.backward()
    sees = torch.arange(Lq) + Lk - Lq + 1 if causal else torch.full((Lq,), Lk)
    assert not bool(c.dq[(sees <= 1).to(DEV)].any())
    if Lk == 1:
        assert not bool(c.dk.any())


def test_same_bits_and_other_stream(gpu):
    for args in ((BF16, [0, 300, 420], [0, 300, 420], 4, 2, 64, True), (F32, [0, 5], [0, 3000], 2, 2, 64, False)):
        c = Case(*args)
        c.forward()
        c.backward()
        want = {n: t.clone() for n, t in c.results().items()}
        torch.cuda.synchronize()
        s = torch.cuda.Stream()
        s.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(s):
            c.clear()
            c.ws.fill_(0xFF)
            c.forward(s)
            c.backward(s)
        torch.cuda.synchronize()
        for n, t in c.results().items():
            assert torch.equal(torch.nan_to_num(t, 7.0), torch.nan_to_num(want[n], 7.0)), n


def test_starts_out_of_order(gpu):
    """Results are undefined, but every access is within the matrices (the guards around them stay NaN)."""
    for starts in ([5, 2, 900, -7, 64], [0, 0, 0, 0, 0], [-3, 1 << 30, -(1 << 31), (1 << 31) - 1, 0], [64, 48, 32, 16, 0]):
        c = Case(BF16, [0, 16, 32, 48, 64], [0, 16, 32, 48, 64], 2, 1, 64, True, pad=8, offset=16)
        for t in c.starts.values():
            t.copy_(torch.tensor(starts, dtype=torch.int32))
        c.forward()
        c.backward()
        torch.cuda.synchronize()
        for t in (c.out, c.dq, c.dk, c.dv):
            untouched(t)
