"""Rotary positions on the GPU against the definition in 64 bits (angles in more).

Tolerances.  Cosine and sine are off by 2^-23 at most (test_more_abi.py has their
series), their product with the amplitude is rounded (2^-24); in fp32 a result x c -
y s takes on those errors times |x| and |y|, the rounding of y s and its own, 2^-24
each of |x| + |y| at most: (2^-23 + 3 * 2^-24) of amplitude (|x| + |y|), below 2^-21.
Elements in bf16 are rounded once more, 2^-8 of the value at most."""
import numpy as np
import pytest
import torch

from paper_2608_13524_amd import dartree as D
from tests import more_ref as R
from tests import serve_ref as S
from tests.gpu_util import device, say

pytestmark = pytest.mark.gpu
HALF, INTER = D.ROTARY_HALF, D.ROTARY_INTERLEAVED
BF, FP = torch.bfloat16, torch.float32


def i32(a):
    return None if a is None else torch.from_numpy(np.ascontiguousarray(a, np.int32)).to(device())


class Case:
    def __init__(self, b, rows, hq, hkv, d=128, rot=None, layout=HALF, dtype=BF, inverse=0, first=0, amplitude=1.0, positions=None,
                 start=None, counts=None, fused=False, seed=0, scaling=(0, 1.0, 0.0, 0.0, 0), base=10000.0):
        rng = np.random.default_rng(seed)
        rot = d if rot is None else rot
        self.p = D.RotaryParams(b, rows, hq, hkv, d, rot, layout, D.BF16 if dtype is BF else D.FP32, inverse, first, amplitude)
        x = rng.normal(size=(b, rows, hq + 2 * hkv, d)).astype(np.float32)
        self.x = S.bf16(x) if dtype is BF else x
        wide = torch.from_numpy(self.x).to(device()).to(dtype)
        self.q, self.k = wide[:, :, :hq], wide[:, :, hq:hq + hkv]
        self.wide = wide
        if not fused:
            self.q, self.k = self.q.contiguous(), self.k.contiguous()
        self.positions, self.start, self.counts = positions, start, counts
        self.turns = D.rotary_turns(rot, base, D.RotaryScaling(*scaling))
        self.f = R.frequencies(rot, base, *scaling)

    def run(self, place="apart"):
        """(q, k) turned, into outputs of sevens, in place or into rows of a wider tensor."""
        p = self.p
        some = lambda x: x if x.shape[2] else None
        q, k = self.q, self.k
        if place == "in":
            outs = (q, k)
        elif place == "wide":
            wide = torch.full((p.batch, p.rows, p.heads_q + p.heads_kv + 1, p.head_dim), 7.0, dtype=q.dtype, device=device())
            outs = (wide[:, :, :p.heads_q], wide[:, :, p.heads_q:p.heads_q + p.heads_kv])
        else:
            outs = tuple(torch.full((p.batch, p.rows, x.shape[2], p.head_dim), 7.0, dtype=x.dtype, device=device()) for x in (q, k))
        say(f"rotary b={p.batch} rows={p.rows} heads={p.heads_q}/{p.heads_kv} d={p.head_dim} rot={p.rotary_dim} layout={p.layout} "
            f"type={p.type} inverse={p.inverse} {place}")
        D.rotary(p, self.turns, some(q), some(k), some(outs[0]), some(outs[1]), positions=i32(self.positions), start=i32(self.start),
                 counts=i32(self.counts))
        torch.cuda.synchronize()
        return outs

    def check(self, place="apart"):
        p = self.p
        outs = [x.float().cpu().numpy().astype(np.float64) for x in self.run(place)]
        at = np.broadcast_to(np.arange(p.rows), (p.batch, p.rows)) if self.positions is None else np.asarray(self.positions)
        at = at.astype(np.int64) + p.first + (0 if self.start is None else np.asarray(self.start, np.int64)[:, None])
        amplitude = float(np.float32(p.amplitude))
        for out, x in zip(outs, (self.x[:, :, :p.heads_q], self.x[:, :, p.heads_q:p.heads_q + p.heads_kv])):
            want = R.rotate(x, at, self.f, p.layout == HALF, amplitude, p.inverse)
            size = np.abs(x).astype(np.float64)
            pair = R.rotate(size, at * 0, self.f * 0, p.layout == HALF)   # |x| and |y| of each pair, side by side
            r = p.rotary_dim
            if p.layout == HALF:
                both = pair[..., :r // 2] + pair[..., r // 2:r]
                both = np.concatenate([both, both], axis=-1)
            else:
                both = np.repeat(pair[..., 0:r:2] + pair[..., 1:r:2], 2, axis=-1)
            tol = np.zeros_like(want)
            tol[..., :r] = abs(amplitude) * both * 2.0 ** -21
            if p.type == D.BF16:
                tol[..., :r] += 2.0 ** -8 * np.abs(want[..., :r])
            rest = x if place == "in" else np.full_like(want, 7.0)
            if self.counts is not None:
                there = np.arange(p.rows) < np.asarray(self.counts)[:, None]
                want = np.where(there[:, :, None, None], want, rest)
                tol = np.where(there[:, :, None, None], tol, 0.0)
            assert (np.abs(out - want) <= tol).all(), np.abs(out - want).max()


@pytest.mark.parametrize("dtype", [BF, FP])
@pytest.mark.parametrize("layout", [HALF, INTER])
@pytest.mark.parametrize("b,rows,hq,hkv,d,rot", [
    (1, 1, 1, 1, 128, 128), (1, 1, 32, 8, 128, 128), (3, 7, 4, 2, 64, 64), (2, 5, 3, 1, 128, 64), (2, 3, 2, 2, 128, 2), (1, 9, 5, 1, 80, 20),
    (2, 4, 6, 3, 8, 8), (1, 33, 2, 1, 512, 512), (2, 11, 1, 1, 256, 250), (1, 700, 8, 8, 128, 96), (4, 777, 2, 1, 128, 126), (1, 5, 0, 3, 128, 128),
    (1, 5, 3, 0, 128, 128)])
def test_shapes(b, rows, hq, hkv, d, rot, layout, dtype):
    for place, fused in (("apart", False), ("in", True), ("wide", True)):
        Case(b, rows, hq, hkv, d, rot, layout, dtype, fused=fused, start=np.arange(b) * 1000 - 5, seed=rows).check(place)


@pytest.mark.parametrize("dtype", [BF, FP])
@pytest.mark.parametrize("layout", [HALF, INTER])
def test_positions(layout, dtype):
    """Far ones up to 2^31 either way, negative ones, the same one twice, sums past 32 bits."""
    big = np.iinfo(np.int32).max
    positions = np.array([[0, 1, -1, 5, 5, 1 << 20], [big, -big - 1, 1 << 30, 12345678, 3, 0]])
    for start, first in (([0, 0], 0), ([1 << 20, 7], -1), ([big, -big - 1], big)):
        Case(2, 6, 2, 1, 128, 64, layout, dtype, positions=positions, start=start, first=first, seed=3).check()


@pytest.mark.parametrize("scaling", [(1, 8.0, 0.0, 0.0, 0), (2, 4.0, 0.0, 0.0, 0), (3, 4.0, 1.0, 32.0, 4096), (3, 0.5, 1.0, 4.0, 8192)])
@pytest.mark.parametrize("base", [10000.0, 5e6])
def test_rules_for_long_contexts(scaling, base):
    Case(2, 40, 4, 2, scaling=scaling, base=base, start=[0, 200000], amplitude=1.1386, seed=4).check()


@pytest.mark.parametrize("dtype", [BF, FP])
@pytest.mark.parametrize("counts", [[0, 1, 5, 7, 9], [-3, 7, 100, 0, 2]])
def test_rows_past_the_count_are_left(counts, dtype):
    for rows in (7, 700):   # one row a block, four
        for place in ("apart", "in", "wide"):
            Case(5, rows, 3, 2, 128, 64, dtype=dtype, counts=counts, start=[0, 9, 0, 100, 3], fused=True, seed=5).check(place)


def test_many_rows():
    """More blocks than the chip holds, a last block that is not full."""
    rng = np.random.default_rng(6)
    Case(3, 5461, 4, 1, start=rng.integers(0, 1 << 20, 3), seed=6).check()


def test_amplitudes_and_infinities():
    c = Case(1, 3, 1, 1, dtype=FP, amplitude=0.0, seed=7)
    q, k = c.run()
    assert (q == 0).all() and (k == 0).all()
    c = Case(1, 3, 2, 1, dtype=FP, seed=7)
    c.q[0, 1, 0, 3], c.q[0, 1, 1, 100], c.k[0, 2, 0, 64] = float("inf"), float("nan"), float("-inf")
    bad = Case(1, 3, 2, 1, dtype=FP, seed=7).run()
    got = c.run()
    for g, plain, hit in ((got[0], bad[0], [(1, 0, 3), (1, 0, 67), (1, 1, 100), (1, 1, 36)]), (got[1], bad[1], [(2, 0, 64), (2, 0, 0)])):
        for at in hit:   # both elements of the pair, no other one
            assert not g[(0, *at)].isfinite()
            g[(0, *at)] = plain[(0, *at)]
        assert torch.equal(g, plain)


@pytest.mark.parametrize("layout", [HALF, INTER])
@pytest.mark.parametrize("rot", [128, 36])
def test_gradient(layout, rot):
    """The inverse is the gradient: of the formula (the transposed matrix, by <g, R x> = <R' g, x>), against
    differences of the call itself, and back to where it came from."""
    amplitude = 0.75
    fwd = Case(2, 5, 2, 1, 128, rot, layout, FP, amplitude=amplitude, start=[3, 900], seed=8)
    grad = Case(2, 5, 2, 1, 128, rot, layout, FP, inverse=1, amplitude=amplitude, start=[3, 900], seed=9)   # x: the outputs' gradients
    grad.check()
    y, g = fwd.run(), grad.run()
    for out, x, gy, gx in zip(y, (fwd.q, fwd.k), (grad.q, grad.k), g):
        a, b = (out.double() * gy.double()).sum(), (x.double() * gx.double()).sum()
        # sums of n products: each side's elements are off by 2^-21 of their pair at most
        size = float(out.double().abs().sum() * gy.double().abs().max())
        assert abs(float(a - b)) <= 2.0 ** -20 * size
    rng = np.random.default_rng(10)
    for _ in range(20):   # the loss sum(gy y) is linear in x: a difference of any step is the gradient, but for roundings
        i = tuple(int(rng.integers(0, n)) for n in fwd.q.shape)
        was = fwd.q[i].item()
        fwd.q[i] = was + 1.0
        step = fwd.q[i].item() - was
        up = fwd.run()[0]
        fwd.q[i] = was
        slope = float(((up.double() - y[0].double()) * grad.q.double()).sum()) / step
        assert abs(slope - float(g[0][i])) <= 2.0 ** -18 * float(grad.q.abs().max()) * 8
    back = Case(2, 5, 2, 1, 128, rot, layout, FP, inverse=1, start=[3, 900])
    there = Case(2, 5, 2, 1, 128, rot, layout, FP, start=[3, 900], seed=8)
    back.q, back.k = there.run()
    for r, x in zip(back.run(), (there.q, there.k)):
        assert (r - x).abs().max() <= 2.0 ** -19 * 5


def test_a_key_moves_to_another_position():
    """Turned to position 50, then back by 8 (the inverse with positions of 8): as turned to 42."""
    at = lambda p, inverse=0: Case(1, 1, 1, 1, dtype=FP, positions=[[p]], inverse=inverse, seed=11)
    move = at(8, 1)
    move.q, move.k = at(50).run()
    for a, b in zip(move.run(), at(42).run()):
        assert (a - b).abs().max() <= 2.0 ** -19 * 5


def test_on_another_stream_and_replayed():
    """The stream given by argument and the current one; a captured call on new contents of the same tensors."""
    c = Case(2, 64, 4, 2, start=[10, 2000], seed=12)
    want = [x.clone() for x in c.run()]
    outs = [torch.zeros_like(x) for x in want]
    start, side = i32(c.start), torch.cuda.Stream()
    torch.cuda.synchronize()
    D.rotary(c.p, c.turns, c.q, c.k, *outs, start=start, stream=side)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(outs, want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        D.rotary(c.p, c.turns, c.q, c.k, *outs, start=start)
    for i in range(3):
        c.q.copy_(torch.randn_like(c.q))
        start += 5
        say(f"rotary replay {i}")
        graph.replay()
        torch.cuda.synchronize()
        plain = [torch.zeros_like(x) for x in want]
        D.rotary(c.p, c.turns, c.q, c.k, *plain, start=start)
        assert all(torch.equal(a, b) for a, b in zip(outs, plain))
