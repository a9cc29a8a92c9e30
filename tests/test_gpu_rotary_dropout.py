"""Rotary positions and dropout behind include/detonation_model.h against their definitions, and the operators of an
attention block together, as a training step uses them."""
import math

import pytest
import torch

from paper_2502_06728_amd import model_ops as ops
from tests import attention_reference as ref
from tests.model_reference import BF16, F16, F32, assert_near, double
from tests.test_gpu_model_ops import DEV, NAN, INF, like, normal, rows, say, scratch, untouched

pytestmark = pytest.mark.gpu
TYPES = [F32, BF16, F16]
LAYOUT = {"halves": ops.ROTARY_HALVES, "pairs": ops.ROTARY_PAIRS}


# ------------------------------------------------------------------ rotary positions

@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("layout", ["halves", "pairs"])
@pytest.mark.parametrize("T,heads,head_dim,rotary_dim,longest,pad,offset", [
    (1, 1, 2, 2, 1, 0, 0), (1, 1, 8, 6, 50, 0, 0), (3, 2, 7, 4, 100, 1, 3), (5, 3, 64, 64, 2048, 0, 0),
    (2, 5, 80, 40, 1 << 20, 8, 8), (33, 2, 128, 128, 1 << 31, 0, 0), (7, 1, 33, 26, 4096, 3, 1), (300, 70, 18, 18, 9, 0, 0),
    (2, 1, 1030, 514, 77, 0, 0)])
def test_rotary(gpu, dtype, layout, T, heads, head_dim, rotary_dim, longest, pad, offset):
    say(dtype, layout, T, heads, head_dim, rotary_dim)
    x = rows(normal(T + head_dim, T, heads * head_dim), dtype, pad, offset)
    freqs = ops.rotary_frequencies(rotary_dim, device=DEV)
    p = torch.randint(0, longest, (T,), generator=torch.Generator().manual_seed(1))
    p[-1] = longest - 1
    for inverse, magnitude, positions in ((False, 1.0, p.to(DEV)), (True, 0.75, p.clamp(max=2 ** 31 - 1).to(torch.int32).to(DEV))):
        cfg = ops.Rotary(heads=heads, head_dim=head_dim, rotary_dim=rotary_dim, layout=LAYOUT[layout], magnitude=magnitude)
        want = ref.rotary(x, positions, freqs, heads, head_dim, rotary_dim, layout, inverse, magnitude)
        out = like(T, heads * head_dim, dtype, pad, offset)
        ops.detonation_rotary(cfg, x, freqs, out, positions=positions, inverse=inverse)
        # an angle is off by 2^-52 of its turns, twice, and 2^-24 of an eighth of a turn; sine and cosine by a few units;
        # two products and a sum
        turns = longest / (2 * math.pi)
        size = double(x).abs().max(1, keepdim=True).values * magnitude
        assert_near(out, want, size, 12 + 2 * math.pi * turns * 2.0 ** -50 * 2.0 ** 24, "out")
        untouched(out)
        again = rows(double(x), dtype, pad, offset)
        ops.detonation_rotary(cfg, again, freqs, again, positions=positions, inverse=inverse)       # in place
        assert torch.equal(again, out)


@pytest.mark.parametrize("period,first", [(0, 0), (0, 1000), (7, 0), (7, 12345)])
def test_positions_of_rows(gpu, period, first):
    x, freqs = rows(normal(1, 23, 96), F32), ops.rotary_frequencies(32, device=DEV)
    t = torch.arange(23, device=DEV)
    given, implied = like(23, 96, F32), like(23, 96, F32)
    cfg = ops.Rotary(heads=3, head_dim=32, first=first, period=period)
    ops.detonation_rotary(cfg, x, freqs, given, positions=first + (t % period if period else t))
    ops.detonation_rotary(cfg, x, freqs, implied)
    assert torch.equal(given, implied)


def test_rotary_of_many_rows(gpu):
    """Several heads to a lane; columns of a wider matrix; turned back, the rows are what they were."""
    T, heads, head_dim = 9000, 24, 64
    whole = torch.randn((T, 3 * heads * head_dim), device=DEV)
    x = whole[:, heads * head_dim:2 * heads * head_dim]
    freqs = ops.rotary_frequencies(head_dim, factor=8.0, trained=512, device=DEV)
    cfg, there, back = ops.Rotary(heads=heads, head_dim=head_dim), torch.empty_like(x), torch.empty_like(x)
    ops.detonation_rotary(cfg, x, freqs, there)
    ops.detonation_rotary(cfg, there, freqs, back, inverse=True)
    assert float((back - x).abs().max()) < 12 * 2.0 ** -23 * float(x.abs().max())
    at = torch.tensor([0, 1, 4567, T - 1])
    want = ref.rotary(x[at.to(DEV)], at, freqs, heads, head_dim, head_dim, "halves")
    assert_near(there[at.to(DEV)], want, double(x).abs().max(), 12, "out")


def test_frequencies(gpu):
    plain = ops.rotary_frequencies(8, base=100.0, device="cpu")
    assert torch.allclose(plain, torch.tensor([1, 100 ** -0.25, 0.1, 100 ** -0.75], dtype=torch.float64), rtol=1e-14)
    assert torch.allclose(ops.rotary_frequencies(8, base=100.0, factor=4.0, device="cpu"), plain / 4, rtol=1e-14)
    blended = ops.rotary_frequencies(64, factor=4.0, trained=1000, device="cpu") / ops.rotary_frequencies(64, device="cpu")
    held = ops.rotary_frequencies(64, device="cpu") * 1000 / (2 * math.pi)
    assert bool((blended[held >= 32] == 1).all()) and torch.allclose(blended[held <= 1], torch.tensor(0.25, dtype=torch.float64))
    between = (held > 1) & (held < 32)
    assert bool(((blended[between] > 0.25) & (blended[between] < 1)).all()) and int(between.sum()) > 3
    for bad in (dict(rotary_dim=7), dict(rotary_dim=0), dict(rotary_dim=4, base=0.0), dict(rotary_dim=4, factor=0.0)):
        with pytest.raises(ValueError):
            ops.rotary_frequencies(**bad)


# ------------------------------------------------------------------ dropout

@pytest.mark.parametrize("dtype,xdtype", [(F32, F32), (BF16, BF16), (F16, F16), (BF16, F32), (F16, F32)])
@pytest.mark.parametrize("T,D,rate,pad,offset", [(1, 1, 0.5, 0, 0), (3, 8, 0.0, 0, 0), (5, 33, 0.1, 3, 1), (9, 64, 0.9, 0, 8),
                                                 (2, 259, 0.3, 1, 0), (4, 7, 0.99999, 0, 0)])
def test_dropout(gpu, dtype, xdtype, T, D, rate, pad, offset):
    say(dtype, xdtype, T, D, rate)
    seed, at = 0x123456789ABCDEF0, 0xFEDCBA9876543210
    cfg = ops.Dropout(rate=rate, seed=seed)
    keep, scale = ref.kept(T, D, rate, seed, at)
    x, res, g = rows(normal(1, T, D), dtype, pad, offset), rows(normal(2, T, D), xdtype, pad), rows(normal(3, T, D), xdtype, pad, offset)
    out, alone, dx = like(T, D, xdtype, pad), like(T, D, dtype, pad), like(T, D, dtype)
    ops.detonation_dropout(cfg, x, out, residual=res, offset=at)
    want = double(res) + torch.where(keep, double(x) * scale, 0.0)
    assert_near(out, want, double(x).abs() * scale + want.abs(), 3, "out")
    ops.detonation_dropout(cfg, x, alone, offset=at)
    assert_near(alone, torch.where(keep, double(x) * scale, 0.0), double(x).abs() * scale, 2, "alone")
    ops.detonation_dropout(cfg, g, dx, offset=at)
    assert_near(dx, torch.where(keep, double(g) * scale, 0.0), double(g).abs() * scale, 2, "dx")
    untouched(out)
    untouched(alone)
    odd = rows(torch.where(keep, double(x), NAN), dtype, pad)            # what is dropped may be anything
    again = like(T, D, dtype, pad)
    ops.detonation_dropout(cfg, odd, again, offset=at)
    assert torch.equal(again, alone)
    more = torch.tensor([5], dtype=torch.int64, device=DEV)
    ops.detonation_dropout(cfg, x, again, offset=at - 5, device_offset=more)
    assert torch.equal(again, alone)
    in_place = rows(double(res), xdtype, pad)
    ops.detonation_dropout(cfg, x, in_place, residual=in_place, offset=at)
    assert torch.equal(in_place, out)
    if dtype == xdtype:
        ops.detonation_dropout(cfg, x, x, offset=at)
        assert torch.equal(x, alone)


def test_shares_of_dropout(gpu):
    """As many stay as should, in every column and row, and other offsets and seeds drop others."""
    x = torch.ones((4096, 512), device=DEV)
    seen = []
    for seed, at in ((1, 0), (1, 1), (2, 0), (1, 1 << 32)):
        out = torch.empty_like(x)
        ops.detonation_dropout(ops.Dropout(rate=0.25, seed=seed), x, out, offset=at)
        stay = out > 0
        assert abs(float(out[stay].double().mean()) - 4 / 3) < 1e-6
        # five standard deviations and a half
        for share, n in ((stay.double().mean(0), 4096), (stay.double().mean(1), 512), (stay.double().mean()[None], x.numel())):
            assert float((share - 0.75).abs().max()) < 5.5 * math.sqrt(0.1875 / n)
        seen.append(stay)
    for i in range(4):
        for j in range(i):
            assert abs(float((seen[i] == seen[j]).double().mean()) - 0.625) < 0.002


# ------------------------------------------------------------------ together

WIDTH, HEADS, KV_HEADS, HEAD_DIM = 192, 6, 2, 32


class Block:
    """x + dropout(attention(rotary(norm(x) Wq, ...)) Wo), forward and backward, by the operators and library products."""

    def __init__(self, dtype, lengths):
        self.T, self.dtype = sum(lengths), dtype
        self.lengths = lengths
        T, narrow, wide = self.T, KV_HEADS * HEAD_DIM, HEADS * HEAD_DIM
        self.x, self.g = normal(1, T, WIDTH).float().to(DEV), normal(2, T, WIDTH).float().to(DEV)
        self.w_in = (normal(3, wide + 2 * narrow, WIDTH) * WIDTH ** -0.5).to(dtype).to(DEV)
        self.w_out = (normal(4, WIDTH, wide) * wide ** -0.5).to(dtype).to(DEV)
        self.w_norm = (1 + 0.1 * normal(5, WIDTH)).float().to(DEV)
        self.freqs = ops.rotary_frequencies(HEAD_DIM, device=DEV)
        self.positions = torch.cat([torch.arange(n) for n in lengths]).to(DEV)
        self.starts = torch.tensor([0] + lengths, device=DEV).cumsum(0).to(torch.int32)
        self.norm = ops.NormResidual()
        self.turn = ops.Rotary(heads=HEADS + KV_HEADS, head_dim=HEAD_DIM)
        self.attention = ops.Attention(heads=HEADS, kv_heads=KV_HEADS, head_dim=HEAD_DIM, scale=HEAD_DIM ** -0.5,
                                       sequences=len(lengths))
        self.dropout = ops.Dropout(rate=0.2, seed=11)
        self.step = torch.zeros(1, dtype=torch.int64, device=DEV)
        new = lambda *s, dtype=dtype: torch.full(s, NAN, dtype=dtype, device=DEV)  # noqa: E731
        self.y, self.qkv, self.o, self.lse = new(T, WIDTH), new(T, wide + 2 * narrow), new(T, wide), new(HEADS, T, dtype=F32)
        self.out = new(T, WIDTH, dtype=F32)
        self.df, self.dqkv, self.dx = new(T, WIDTH), new(T, wide + 2 * narrow), new(T, WIDTH, dtype=F32)
        self.ws = scratch(max(ops.attention_workspace(self.attention, T, T), ops.norm_residual_workspace(self.norm, T, WIDTH)))

    def parts(self, m):
        wide, narrow = HEADS * HEAD_DIM, KV_HEADS * HEAD_DIM
        return m[:, :wide], m[:, wide:wide + narrow], m[:, wide + narrow:]

    def run(self):
        a = dict(q_starts=self.starts, k_starts=self.starts, workspace=self.ws)
        ops.detonation_norm_residual(self.norm, self.x, None, None, self.y, w_pre=self.w_norm)
        torch.mm(self.y, self.w_in.t(), out=self.qkv)
        q, k, v = self.parts(self.qkv)
        both = self.qkv[:, :(HEADS + KV_HEADS) * HEAD_DIM]
        ops.detonation_rotary(self.turn, both, self.freqs, both, positions=self.positions)
        ops.detonation_attention_forward(self.attention, q, k, v, self.o, lse=self.lse, **a)
        f = self.o @ self.w_out.t()
        ops.detonation_dropout(self.dropout, f, self.out, residual=self.x, offset=3, device_offset=self.step)
        # and back
        ops.detonation_dropout(self.dropout, self.g, self.df, offset=3, device_offset=self.step)
        do = self.df @ self.w_out
        dq, dk, dv = self.parts(self.dqkv)
        ops.detonation_attention_backward(self.attention, q, k, v, self.o, self.lse, do, dq, dk, dv, **a)
        both = self.dqkv[:, :(HEADS + KV_HEADS) * HEAD_DIM]
        ops.detonation_rotary(self.turn, both, self.freqs, both, positions=self.positions, inverse=True)
        dy = self.dqkv @ self.w_in
        ops.detonation_norm_residual_backward(self.norm, self.x, None, dy, self.g, self.dx, None, w_pre=self.w_norm)

    def plain(self):
        """(out, dx) in 64 bits, by torch's differentiation."""
        x = double(self.x).requires_grad_()
        w_in, w_out = double(self.w_in), double(self.w_out)
        y = x / torch.sqrt((x * x).mean(1, keepdim=True) + 1e-6) * double(self.w_norm)
        q, k, v = self.parts(y @ w_in.t())
        angle = torch.polar(torch.ones(self.T, HEAD_DIM // 2, dtype=torch.float64),
                            double(self.positions)[:, None] * double(self.freqs))[:, None]

        def turned(m):
            m = m.reshape(self.T, -1, 2, HEAD_DIM // 2)
            z = torch.complex(m[:, :, 0], m[:, :, 1]) * angle
            return torch.stack([z.real, z.imag], 2).reshape(self.T, -1, HEAD_DIM)
        q, k, v = turned(q), turned(k), v.reshape(self.T, -1, HEAD_DIM)
        rows_, at = [], 0
        for n in self.lengths:
            heads = []
            for h in range(HEADS):
                s = q[at:at + n, h] @ k[at:at + n, h // 3].t() * HEAD_DIM ** -0.5
                p = torch.softmax(s.masked_fill(torch.ones(n, n, dtype=torch.bool).triu(1), -INF), 1)
                heads.append(p @ v[at:at + n, h // 3])
            rows_.append(torch.cat(heads, 1))
            at += n
        keep, scale = ref.kept(self.T, WIDTH, 0.2, 11, 3 + int(self.step))
        out = x + torch.where(keep, torch.cat(rows_) @ w_out.t() * scale, 0.0)
        return out.detach(), torch.autograd.grad((out * double(self.g)).sum(), x)[0]


@pytest.mark.parametrize("dtype,far", [(F32, 2e-5), (BF16, 0.02), (F16, 2.5e-3)])
def test_block(gpu, dtype, far):
    """A block's output and its input's gradient.  About ten roundings of each type on the way, none of which is more than
    half a unit of what it acts on: 10 * 2^-8, 2^-11; in fp32 sums of up to 200 terms."""
    b = Block(dtype, [70, 1, 33, 16])
    b.run()
    for got, want in zip((b.out, b.dx), b.plain()):
        assert float((double(got) - want).norm() / want.norm()) < far


def test_replayed_block(gpu):
    """Captured once, replayed with new data and a new step of its dropout, the same as eager; another block's graph of the
    same shapes, with a workspace of its own, runs in between."""
    blocks = [Block(BF16, [70, 1, 33, 16]), Block(BF16, [100, 20])]
    graphs = []
    for b in blocks:
        b.run()
        torch.cuda.synchronize()
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            b.run()
    for i in range(4):
        for b in blocks:
            b.x.copy_(normal(40 + i, b.T, WIDTH).to(DEV))
            b.step.fill_(i * 1000)
            for t in (b.out, b.dx, b.lse, b.dqkv):
                t.fill_(NAN)
        for g in graphs:
            g.replay()
        torch.cuda.synchronize()
        got = [(b.out.clone(), b.dx.clone(), b.lse.clone()) for b in blocks]
        for b, outs in zip(blocks, got):
            b.run()
            torch.cuda.synchronize()
            for a, c in zip(outs, (b.out, b.dx, b.lse)):
                assert torch.equal(a, c)
