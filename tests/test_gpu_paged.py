"""Attention over the paged cache on the GPU against a plain softmax in 64 bits.

Tolerance of an element, from the roundings (bf16: half a step is at most 2^-8 of
the value): the softmax weights are rounded to bf16, which moves the weighted mean
of the values by at most 2^-8 max|v|, and the output is rounded, 2^-8 |out|.  The
rest is 32-bit: scores of up to 30 in magnitude whose 128 products add up with an
error of 128 * 2^-24 relative to their absolute sum (a few hundred at most here),
so weights are off by less than 2^-10, and the sums; 2^-9 max|v| covers them."""
import numpy as np
import pytest
import torch

from paper_2608_13524_amd import dartree as D
from tests import serve_ref as S
from tests.gpu_util import device, say
from tests.test_gpu_cache import BF, E8, normal, tables

pytestmark = pytest.mark.gpu
SCALE = 1.0 / np.sqrt(128.0)


def random_tree(rng, n):
    """Ancestor-or-self visibility of a random tree in which parents precede children."""
    see = np.zeros((n, n), bool)
    for i in range(n):
        p = int(rng.integers(-1, i)) if i else -1
        if p >= 0:
            see[i] = see[p]
        see[i, i] = True
    return see


def words_of(see):
    b, n, _ = see.shape
    w = (n + 63) // 64
    out = np.zeros((b, n, w), np.uint64)
    for j in range(n):
        out[:, :, j // 64] |= see[:, :, j].astype(np.uint64) << np.uint64(j % 64)
    return out.view(np.int64)


class Case:
    """A cache filled through cache_write, whose other memory holds NaN, and a tree over it."""

    def __init__(self, b, n, ctx, hq, hkv, page, kind, seed=0, size=1.0, lens=None, num_nodes=None, chain=False, strided=False,
                 holes=(), see=None, spread=0.5):
        rng = np.random.default_rng(seed * 1000 + b * 100 + n + ctx)
        dev = device()
        self.b, self.n, self.ctx, self.hq, self.hkv, self.kind, self.page = b, n, ctx, hq, hkv, kind, page
        per = max(1, (ctx + page - 1) // page)
        self.p = D.CacheParams(b, hkv, 128, page, b * per + 2, per, kind)
        self.table = tables(rng, b, per, self.p.num_pages)
        self.lens = np.full(b, ctx) if lens is None else np.asarray(lens)
        self.nn = None if num_nodes is None else np.asarray(num_nodes)
        k, v = normal(rng, (b, max(ctx, 1), hkv, 128), spread), normal(rng, (b, max(ctx, 1), hkv, 128), spread)
        self.c = D.DeviceCache.alloc(self.p, dev)
        for t in (self.c.k, self.c.v):
            t.view(torch.uint8).fill_(0xFF)            # NaN in both types
        for t in (self.c.k_exp, self.c.v_exp):
            if t is not None:
                t.fill_(0xFF)
        self.c.table.copy_(torch.from_numpy(self.table))
        counts = np.minimum(np.maximum(self.lens, 0), ctx)
        D.cache_write(self.p, self.c, torch.from_numpy(k).to(dev).bfloat16(), torch.from_numpy(v).to(dev).bfloat16(),
                      max(ctx, 1), counts=torch.from_numpy(counts.astype(np.int32)).to(dev))
        for q, column, entry in holes:
            self.table[q, column] = entry
        self.c.table.copy_(torch.from_numpy(self.table))
        if kind == E8:
            (k, ke), (v, ve) = S.quantise(k), S.quantise(v)
            k, v = k * 2.0 ** ke[..., None], v * 2.0 ** ve[..., None]
        self.k, self.v = k.astype(np.float64), v.astype(np.float64)
        self.q = S.bf16(rng.normal(size=(b, n, hq, 128)) * size)
        self.kt, self.vt = S.bf16(rng.normal(size=(b, n, hkv, 128))), S.bf16(rng.normal(size=(b, n, hkv, 128)))
        if see is None:
            see = np.stack([np.tril(np.ones((n, n), bool)) if chain else random_tree(rng, n) for _ in range(b)])
        self.see = see
        self.mask = None if chain else torch.from_numpy(words_of(see)).to(dev)
        if self.nn is not None:                         # slots without a node hold NaN
            for q in range(b):
                self.kt[q, max(int(self.nn[q]), 0):] = np.nan
                self.vt[q, max(int(self.nn[q]), 0):] = np.nan
        parts = [torch.from_numpy(x).to(dev).bfloat16() for x in (self.q, self.kt, self.vt)]
        if strided:                                     # rows of one projection
            wide = torch.cat(parts, dim=2)
            parts = [wide[:, :, :hq], wide[:, :, hq:hq + hkv], wide[:, :, hq + hkv:]]
        self.dq, self.dk, self.dv = parts
        self.a = D.AttnParams(b, n, ctx, hq, hkv, 128, SCALE)
        i32 = lambda x: torch.from_numpy(np.ascontiguousarray(x, np.int32)).to(dev)
        self.dlens = None if lens is None else i32(self.lens)
        self.dnn = None if num_nodes is None else i32(self.nn)
        need = D.tree_attention_paged_workspace_size(self.a, self.p)
        self.ws = torch.full((need,), 0xFF, dtype=torch.uint8, device=dev) if need else None

    def run(self):
        out = torch.full((self.b, self.n, self.hq, 128), float("nan"), dtype=torch.bfloat16, device=device())
        say(f"tree_attention_paged b={self.b} B={self.n} ctx={self.ctx} heads={self.hq}/{self.hkv} page={self.page} type={self.kind}")
        D.tree_attention_paged(self.a, self.p, self.c, self.dq, self.dk, self.dv, self.mask, self.dlens, out, self.ws,
                               num_nodes=self.dnn)
        torch.cuda.synchronize()
        return out

    def check(self, requests=None, heads=None):
        out = self.run()
        got = out.float().cpu().numpy().astype(np.float64)
        assert np.isfinite(got).all()
        group = self.hq // self.hkv
        for q in range(self.b) if requests is None else requests:
            length = min(max(int(self.lens[q]), 0), self.ctx)
            nn = self.n if self.nn is None else min(max(int(self.nn[q]), 0), self.n)
            there = np.array([S.slot(self.table[q], self.page, self.p.num_pages, t) is not None for t in range(length)], bool)
            there = there.reshape(length)
            nodes = self.see[q].copy()
            nodes[:, nn:] = False
            see = np.concatenate([np.broadcast_to(there, (self.n, length)), nodes], axis=1)
            for h in range(self.hq) if heads is None else heads:
                g = h // group
                keys = np.concatenate([self.k[q, :length, g], np.nan_to_num(self.kt[q, :, g])])
                vals = np.concatenate([self.v[q, :length, g], np.nan_to_num(self.vt[q, :, g])])
                want = S.attention(self.q[q, :, h].astype(np.float64), keys, vals, see, SCALE)
                most = np.abs(np.where(see.any(axis=0)[:, None], vals, 0.0)).max(axis=0) if len(vals) else 0.0
                tol = (2.0 ** -8 + 2.0 ** -9) * most + 2.0 ** -8 * np.abs(want)
                assert (np.abs(got[q, :, h] - want) <= tol).all(), (q, h, np.abs(got[q, :, h] - want).max())
        return out


SHAPES = [  # b, B, ctx, heads_q, heads_kv, page
    (1, 1, 1, 1, 1, 16), (1, 1, 0, 4, 2, 16), (2, 1, 15, 8, 8, 16), (2, 1, 31, 8, 2, 32), (3, 1, 127, 4, 1, 64),
    (2, 1, 128, 8, 1, 128), (2, 1, 129, 32, 8, 64), (1, 3, 1000, 32, 8, 256), (2, 5, 500, 6, 2, 16), (2, 7, 95, 3, 1, 32),
    (1, 16, 333, 8, 4, 64), (1, 17, 64, 2, 2, 16), (2, 33, 200, 4, 1, 32), (1, 64, 2048, 8, 2, 64), (3, 64, 300, 4, 4, 128),
    (2, 100, 777, 8, 2, 16), (1, 130, 257, 4, 2, 256), (2, 200, 31, 2, 1, 64), (1, 300, 1500, 4, 1, 64)]


@pytest.mark.parametrize("kind", [E8, BF])
@pytest.mark.parametrize("b,n,ctx,hq,hkv,page", SHAPES)
def test_trees(kind, b, n, ctx, hq, hkv, page):
    Case(b, n, ctx, hq, hkv, page, kind).check()


@pytest.mark.parametrize("kind", [E8, BF])
@pytest.mark.parametrize("b,n,ctx,hq,hkv,page", [(2, 1, 100, 8, 2, 16), (2, 40, 77, 8, 2, 32), (1, 129, 130, 4, 4, 64),
                                                 (1, 500, 40, 4, 2, 64)])
def test_chains_in_wider_rows(kind, b, n, ctx, hq, hkv, page):
    Case(b, n, ctx, hq, hkv, page, kind, chain=True, strided=True, seed=1).check()


@pytest.mark.parametrize("kind", [E8, BF])
@pytest.mark.parametrize("n,hq,hkv", [(1, 8, 2), (6, 4, 1), (20, 8, 2), (70, 4, 2)])
def test_ragged_lengths_and_nodes(kind, n, hq, hkv):
    """Lengths of 0, 1, past a page's and a step's end, negative and too long; requests without nodes."""
    lens = [0, 1, 16, 17, 128, 129, 500, -4, 1 << 30, 250, 31]
    nn = [n, 0, 1, n, n // 2, n + 5, -1, n, n, 0, n]
    for page in (16, 64):
        Case(11, n, 500, hq, hkv, page, kind, lens=lens, num_nodes=nn, seed=2).check()


@pytest.mark.parametrize("kind", [E8, BF])
@pytest.mark.parametrize("n", [1, 20, 70])
def test_positions_without_a_page(kind, n):
    """Entries outside the pool at the beginning, in the middle and at the end, and a request with none at all."""
    low, high = np.iinfo(np.int32).min, np.iinfo(np.int32).max
    holes = [(0, 0, -1), (1, 1, 10 ** 6), (1, 2, low), (2, 9, high), (3, 4, -1)] + [(4, i, -1) for i in range(10)]
    for page in (16, 32):
        Case(5, n, 10 * page - 3, 4, 2, page, kind, holes=holes, seed=3).check()


def test_rows_that_see_nothing():
    see = np.zeros((3, 20, 20), bool)
    see[1, 5, 3] = see[1, 19, 19] = True
    c = Case(3, 20, 50, 4, 2, 16, BF, lens=[0, 0, 50], see=see, seed=4)
    out = c.check()
    assert (out[0] == 0).all() and (out[1, 0] == 0).all() and (out[1, 5] != 0).any()


@pytest.mark.parametrize("kind", [E8, BF])
@pytest.mark.parametrize("n", [1, 40])
def test_peaked_scores(kind, n):
    """Scores of tens: the running maximum moves, and weights underflow."""
    Case(2, n, 700, 8, 2, 64, kind, size=3.0, seed=5).check()


@pytest.mark.parametrize("kind", [E8, BF])
@pytest.mark.parametrize("b,n,ctx,hq,hkv", [(300, 1, 40, 8, 8), (160, 3, 70, 32, 8), (40, 64, 90, 8, 8), (66, 33, 60, 16, 8)])
def test_many_requests(kind, b, n, ctx, hq, hkv):
    rng = np.random.default_rng(b)
    c = Case(b, n, ctx, hq, hkv, 16, kind, lens=rng.integers(0, ctx + 1, size=b), seed=6)
    c.check(requests=rng.choice(b, 6, replace=False), heads=[0, hq - 1])


@pytest.mark.parametrize("kind", [E8, BF])
@pytest.mark.parametrize("n,hq,chain", [(64, 32, False), (125, 16, True), (70, 32, False)])
def test_many_large_trees(kind, n, hq, chain):
    """256, 250 and 280 query rows a key/value head, enough of them for one block each."""
    rng = np.random.default_rng(n)
    lens = rng.integers(0, 200, size=128)
    lens[5], lens[77] = 0, 199
    c = Case(128, n, 199, hq, 8, 16, kind, lens=lens, chain=chain, num_nodes=rng.integers(1, n + 1, size=128), seed=11,
             holes=[(77, 3, -1), (9, 0, 1 << 30)])
    c.check(requests=[0, 5, 9, 77, 127], heads=[0, hq - 1])


@pytest.mark.parametrize("kind", [E8, BF])
@pytest.mark.parametrize("n,hq,hkv,chain", [(1, 8, 2, True), (4, 8, 2, False), (16, 2, 2, True), (5, 16, 4, False),
                                            (40, 4, 2, False), (33, 8, 2, True)])
def test_keys_shared_out_over_blocks(kind, n, hq, hkv, chain):
    """Contexts long enough that blocks cut items anywhere, over requests of all lengths."""
    lens, nn = [3000, 0, 1, 2049, 700, 2999], [n, 0, n, 1, n, n]
    holes = [(0, 0, -1), (0, 187, 1 << 20), (3, 60, -5), (3, 61, -1), (5, 187, -1)] + [(4, i, -1) for i in range(44)]
    Case(6, n, 3000, hq, hkv, 16, kind, lens=lens, num_nodes=nn, chain=chain, strided=True, holes=holes, seed=12).check(heads=[0, hq - 1])


@pytest.mark.parametrize("kind", [E8, BF])
@pytest.mark.parametrize("b,n,ctx,hq,hkv,chain", [(1, 8, 2048, 16, 4, False), (3, 33, 1500, 4, 2, False), (2, 100, 2500, 2, 1, True),
                                                  (1, 16, 4000, 32, 8, True)])
def test_few_items_over_middle_contexts(kind, b, n, ctx, hq, hkv, chain):
    """More than 16 query rows a head whose 16-row items are cut."""
    Case(b, n, ctx, hq, hkv, 32, kind, lens=[ctx, 1, ctx - 77][:b], num_nodes=[n, n, n - 5][:b], chain=chain, strided=True,
         holes=[(0, 3, -1)], seed=16).check(heads=[0, hq - 1])


@pytest.mark.parametrize("kind", [E8, BF])
@pytest.mark.parametrize("b,n,ctx,hq,hkv,lens", [(3, 500, 2048, 32, 8, [2048, 0, 777]), (1, 512, 4000, 16, 8, [3999])])
def test_few_large_trees_over_long_contexts(kind, b, n, ctx, hq, hkv, lens):
    """Tiles of 128 query rows whose keys are shared out over blocks."""
    Case(b, n, ctx, hq, hkv, 64, kind, lens=lens, num_nodes=[n, n - 370, 1][:b], holes=[(0, 7, -1)], seed=13).check(heads=[0, hq - 1])


@pytest.mark.parametrize("kind", [E8, BF])
@pytest.mark.parametrize("b,n,ctx", [(1, 1, 40000), (2, 16, 20011), (1, 64, 9000)])
def test_long_contexts(kind, b, n, ctx):
    Case(b, n, ctx, 8, 2, 64, kind, seed=7).check(heads=[0, 7])


@pytest.mark.parametrize("b,n,ctx", [(1, 1, 3000), (3, 16, 1000), (1, 64, 2048), (2, 200, 500)])
def test_equal_calls_give_equal_bits(b, n, ctx):
    c = Case(b, n, ctx, 8, 2, 64, E8, seed=8)
    first = c.run()
    if c.ws is not None:
        c.ws.fill_(0x77)
    assert torch.equal(first, c.run())


@pytest.mark.parametrize("kind", [E8, BF])
@pytest.mark.parametrize("b,n,ctx,hq,hkv,chain", [(2, 20, 100, 4, 2, False), (2, 12, 3000, 2, 2, True), (2, 70, 3000, 4, 2, False),
                                                  (1, 512, 3000, 32, 8, False), (128, 64, 40, 32, 8, False)])
def test_nodes_that_are_no_numbers(kind, b, n, ctx, hq, hkv, chain):
    """Infinities and NaN in keys and values of tree nodes: rows that see such a node take them, the others do not."""
    plain, odd = (Case(b, n, ctx, hq, hkv, 16, kind, chain=chain, seed=14) for _ in range(2))
    nan, inf = float("nan"), float("inf")
    bad = {n - 1: (inf, nan), n // 2: (0.0, -inf), n // 3: (0.0, inf), n // 5: (nan, 0.0)}   # node: key's element 3, value's element 77
    for j, (k, v) in bad.items():
        for c, kk, vv in ((odd, k, v), (plain, 0.0, 0.0)):
            c.dk[:, j, :, 3] = kk
            c.dv[:, j, :, 77] = vv
    base, out = plain.run().double().cpu(), odd.run().double().cpu()
    for q in {0, b // 2, b - 1}:
        see = torch.from_numpy(odd.see[q])
        lost = torch.zeros(n, dtype=torch.bool)                # rows that see a key that is no number
        value = torch.zeros(n, dtype=torch.float64)            # what element 77 takes besides
        for j, (k, v) in bad.items():
            lost |= see[:, j] & (k != 0.0)
            value += torch.where(see[:, j] & (v != 0.0), v, 0.0).double()
        want = base[q].clone()
        want[:, :, 77] += value[:, None]
        kept = ~lost
        assert kept.any() and torch.equal(out[q][kept].nan_to_num(), want[kept].nan_to_num())
        assert torch.equal(out[q][kept].isnan(), want[kept].isnan()) and (value != 0).any()
        assert not out[q][lost].isfinite().all(dim=-1).any()


def test_follows_the_dense_layer():
    """The same attention as dartree_tree_attention on the context read back."""
    c = Case(2, 48, 300, 8, 2, 16, E8, lens=[300, 123], seed=9)
    dev = device()
    k = torch.zeros(2, 300, 2, 128, dtype=torch.bfloat16, device=dev)
    v = torch.zeros_like(k)
    D.cache_read(c.p, c.c, k, v, counts=c.dlens)
    need = D.tree_attention_workspace_size(c.a)
    ws = torch.empty(max(need, 1), dtype=torch.uint8, device=dev)
    out = torch.empty(2, 48, 8, 128, device=dev)
    D.tree_attention(c.a, c.dq, k, v, c.dk, c.dv, c.mask, c.dlens, out, ws)
    got = c.run().float()
    most = max(float(v.abs().max()), float(c.dv.abs().max()))
    assert float((got - out).abs().max()) <= 2 * (2.0 ** -8 + 2.0 ** -9) * most + 2.0 ** -8 * float(out.abs().max())


@pytest.mark.parametrize("kind", [E8, BF])
def test_pages_past_4_gib(kind):
    """Pages of which keys, values and exponents lie far into the pool."""
    c = Case(1, 5, 600, 8, 8, 256, kind, seed=10)
    page_bytes = 8 * 256 * 128 * (1 if kind == E8 else 2)
    n = (5 << 30) // page_bytes
    far = D.CacheParams(1, 8, 128, 256, n, c.p.max_pages, kind)
    big = D.DeviceCache.alloc(far, device())
    at = [n - 1 - i for i in range(c.p.max_pages)]
    for to, of in zip(at, c.table[0]):
        for x, y in ((big.k, c.c.k), (big.v, c.c.v), (big.k_exp, c.c.k_exp), (big.v_exp, c.c.v_exp)):
            if x is not None:
                x[to].view(torch.uint8).copy_(y[int(of)].view(torch.uint8))
    want = c.run()
    big.table.copy_(torch.tensor([at], dtype=torch.int32))
    c.p, c.c, c.table = far, big, np.array([at])
    assert torch.equal(c.check(heads=[0, 7]), want)
    del big, c
    torch.cuda.empty_cache()
