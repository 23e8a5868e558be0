"""Attention over a paged cache in 4 bits on the GPU against a plain softmax in 64
bits, over what the cache holds.

Tolerance of an element: that of test_gpu_paged.py, derived there.  The one step
that differs, queries multiplied in two e4m3 parts under a power of two for each 32
of them, leaves at most 2^-21 of the largest of those 32 of an element (the second
part has 4 bits of what the first leaves, down to 2^-13 where the largest is held
above 2^7): 128 such errors in a score of the sizes here, below 2^-12 of its absolute
sum, lie within the 2^-10 that are allowed for weights there.  So does what the matrix
instruction drops of a score's products, 2^-17 of the largest of them each: 2^-17 of
a few units here."""
import numpy as np
import pytest
import torch

from paper_2608_13524_amd import dartree as D
from tests import more_ref as R
from tests import serve_ref as S
from tests.gpu_util import device, say
from tests.test_gpu_cache import make_cache
from tests.test_gpu_cache4 import E4, i32, put
from tests.test_gpu_paged import SHAPES, Case
from tests.test_gpu_serve_range import KERNELS

pytestmark = pytest.mark.gpu


class Case4(Case):
    def __init__(self, b, n, ctx, hq, hkv, page, **kw):
        super().__init__(b, n, ctx, hq, hkv, page, E4, **kw)
        self.k, self.v = R.held(self.k), R.held(self.v)


@pytest.mark.parametrize("b,n,ctx,hq,hkv,page", SHAPES)
def test_trees(b, n, ctx, hq, hkv, page):
    Case4(b, n, ctx, hq, hkv, page).check()


@pytest.mark.parametrize("b,n,ctx,hq,hkv,page", [(2, 1, 100, 8, 2, 16), (2, 40, 77, 8, 2, 32), (1, 129, 130, 4, 4, 64),
                                                 (1, 500, 40, 4, 2, 64)])
def test_chains_in_wider_rows(b, n, ctx, hq, hkv, page):
    Case4(b, n, ctx, hq, hkv, page, chain=True, strided=True, seed=1).check()


@pytest.mark.parametrize("n,hq,hkv", [(1, 8, 2), (6, 4, 1), (20, 8, 2), (70, 4, 2)])
def test_ragged_lengths_and_nodes(n, hq, hkv):
    """Lengths of 0, 1, past a page's and a step's end, negative and too long; requests without nodes."""
    lens = [0, 1, 16, 17, 128, 129, 500, -4, 1 << 30, 250, 31]
    nn = [n, 0, 1, n, n // 2, n + 5, -1, n, n, 0, n]
    for page in (16, 64):
        Case4(11, n, 500, hq, hkv, page, lens=lens, num_nodes=nn, seed=2).check()


@pytest.mark.parametrize("n", [1, 20, 70])
def test_positions_without_a_page(n):
    low, high = np.iinfo(np.int32).min, np.iinfo(np.int32).max
    holes = [(0, 0, -1), (1, 1, 10 ** 6), (1, 2, low), (2, 9, high), (3, 4, -1)] + [(4, i, -1) for i in range(10)]
    for page in (16, 32):
        Case4(5, n, 10 * page - 3, 4, 2, page, holes=holes, seed=3).check()


def test_rows_that_see_nothing():
    see = np.zeros((3, 20, 20), bool)
    see[1, 5, 3] = see[1, 19, 19] = True
    out = Case4(3, 20, 50, 4, 2, 16, lens=[0, 0, 50], see=see, seed=4).check()
    assert (out[0] == 0).all() and (out[1, 0] == 0).all() and (out[1, 5] != 0).any()


@pytest.mark.parametrize("n", [1, 40])
def test_peaked_scores(n):
    Case4(2, n, 700, 8, 2, 64, size=3.0, seed=5).check()


@pytest.mark.parametrize("b,n,ctx,hq,hkv", [(300, 1, 40, 8, 8), (160, 3, 70, 32, 8), (40, 64, 90, 8, 8), (66, 33, 60, 16, 8)])
def test_many_requests(b, n, ctx, hq, hkv):
    rng = np.random.default_rng(b)
    c = Case4(b, n, ctx, hq, hkv, 16, lens=rng.integers(0, ctx + 1, size=b), seed=6)
    c.check(requests=rng.choice(b, 6, replace=False), heads=[0, hq - 1])


@pytest.mark.parametrize("n,hq,chain", [(64, 32, False), (125, 16, True), (70, 32, False)])
def test_many_large_trees(n, hq, chain):
    """256, 250 and 280 query rows a key/value head, enough of them for one block each."""
    rng = np.random.default_rng(n)
    lens = rng.integers(0, 200, size=128)
    lens[5], lens[77] = 0, 199
    c = Case4(128, n, 199, hq, 8, 16, lens=lens, chain=chain, num_nodes=rng.integers(1, n + 1, size=128), seed=11,
              holes=[(77, 3, -1), (9, 0, 1 << 30)])
    c.check(requests=[0, 5, 9, 77, 127], heads=[0, hq - 1])


@pytest.mark.parametrize("n,hq,hkv,chain", [(1, 8, 2, True), (4, 8, 2, False), (16, 2, 2, True), (5, 16, 4, False),
                                            (40, 4, 2, False), (33, 8, 2, True)])
def test_keys_shared_out_over_blocks(n, hq, hkv, chain):
    """Contexts long enough that blocks cut items anywhere, over requests of all lengths."""
    lens, nn = [3000, 0, 1, 2049, 700, 2999], [n, 0, n, 1, n, n]
    holes = [(0, 0, -1), (0, 187, 1 << 20), (3, 60, -5), (3, 61, -1), (5, 187, -1)] + [(4, i, -1) for i in range(44)]
    Case4(6, n, 3000, hq, hkv, 16, lens=lens, num_nodes=nn, chain=chain, strided=True, holes=holes, seed=12).check(heads=[0, hq - 1])


@pytest.mark.parametrize("b,n,ctx,hq,hkv,chain", [(1, 8, 2048, 16, 4, False), (3, 33, 1500, 4, 2, False), (2, 100, 2500, 2, 1, True),
                                                  (1, 16, 4000, 32, 8, True)])
def test_few_items_over_middle_contexts(b, n, ctx, hq, hkv, chain):
    Case4(b, n, ctx, hq, hkv, 32, lens=[ctx, 1, ctx - 77][:b], num_nodes=[n, n, n - 5][:b], chain=chain, strided=True,
          holes=[(0, 3, -1)], seed=16).check(heads=[0, hq - 1])


@pytest.mark.parametrize("b,n,ctx,hq,hkv,lens", [(3, 500, 2048, 32, 8, [2048, 0, 777]), (1, 512, 4000, 16, 8, [3999])])
def test_few_large_trees_over_long_contexts(b, n, ctx, hq, hkv, lens):
    Case4(b, n, ctx, hq, hkv, 64, lens=lens, num_nodes=[n, n - 370, 1][:b], holes=[(0, 7, -1)], seed=13).check(heads=[0, hq - 1])


@pytest.mark.parametrize("b,n,ctx", [(1, 1, 40000), (2, 16, 20011), (1, 64, 9000), (1, 200, 65459)])
def test_long_contexts(b, n, ctx):
    Case4(b, n, ctx, 8, 2, 64, seed=7).check(heads=[0, 7])


@pytest.mark.parametrize("b,n,ctx", [(1, 1, 3000), (3, 16, 1000), (1, 64, 2048), (2, 200, 500)])
def test_equal_calls_give_equal_bits(b, n, ctx):
    c = Case4(b, n, ctx, 8, 2, 64, seed=8)
    first = c.run()
    if c.ws is not None:
        c.ws.fill_(0x77)
    assert torch.equal(first, c.run())


@pytest.mark.parametrize("n,ctx,hq,hkv,b", KERNELS)
def test_queries_of_all_sizes(n, ctx, hq, hkv, b):
    """Elements 2^12 apart under one power of two where the large ones meet keys of zero, blocks of zeros, blocks of
    sizes 2^20 apart.  The largest of the first 32 is below 2^9 and held as up to 448 = 2^9 - 64 of a unit, so an element
    is at most 2^-14 of a unit <= 2^1 off; times keys below 2^5, 16 of them and SCALE that is 2^-7 / 11 < 2^-10."""
    rng = np.random.default_rng(n + 5)
    c = Case4(b, n, ctx, hq, hkv, 16, seed=30)
    size = np.ones(128)
    size[:32] = 2.0 ** np.array([6.0, -6.0] * 16)
    size[32:64] = 0.0
    size[64:96] = 2.0 ** -20
    c.q = S.bf16(c.q * size)
    k = rng.normal(size=(b, max(ctx, 1), hkv, 128))
    k[..., 0:32:2], k[..., 1:32:2], k[..., 64:96] = 0.0, k[..., 1:32:2] * 4.0, k[..., 64:96] * 2.0 ** 19
    k = S.bf16(k)
    c.k = R.held(k)
    dv = put(S.bf16(c.v))
    D.cache_write(c.p, c.c, put(k), dv, ctx)
    c.v = R.held(S.bf16(c.v))
    c.kt = S.bf16(np.where(size == 64.0, 0.0, c.kt))
    c.dq, c.dk = put(c.q), put(c.kt)
    c.check(requests=sorted({0, b - 1}), heads=[0, hq - 1])


@pytest.mark.parametrize("n,ctx,hq,hkv,b", KERNELS)
def test_numbers_that_are_none(n, ctx, hq, hkv, b):
    """A NaN among a position's values: those 32 elements of every row are NaN, all others keep their bits.  An infinity
    in a query: its row is NaN.  A NaN among a position's keys: every row is NaN, and none where no row sees it."""
    rng = np.random.default_rng(n + 1)
    dev, page = device(), 16
    per = (ctx + page - 1) // page
    p = D.CacheParams(b, hkv, 128, page, b * per, per, E4)
    draw = lambda rows, heads: put(S.bf16(rng.normal(size=(b, rows, heads, 128))))
    k, v, q, t = draw(ctx, hkv), draw(ctx, hkv), draw(n, hq), draw(n, hkv)
    c = make_cache(p, rng.permutation(b * per).reshape(b, per))
    a = D.AttnParams(b, n, ctx, hq, hkv, 128, 0.0884)
    need = D.tree_attention_paged_workspace_size(a, p)
    ws = torch.empty(need, dtype=torch.uint8, device=dev) if need else None
    nan = float("nan")

    def run(k, v, q, length=ctx):
        D.cache_write(p, c, k, v, ctx)
        out = torch.zeros(b, n, hq, 128, dtype=torch.bfloat16, device=dev)
        say(f"tree_attention_paged e2m1, no numbers: b={b} B={n} ctx={ctx} heads={hq}/{hkv} length={length}")
        D.tree_attention_paged(a, p, c, q, t, t, None, i32([length] * b), out, ws)
        torch.cuda.synchronize()
        return out.cpu()

    def changed(x, *at, to=nan):
        y = x.clone()
        y[at] = to
        return y

    base = run(k, v, q)
    assert base.isfinite().all()
    out = run(k, changed(v, slice(None), ctx // 2, slice(None), 70), q)
    assert out[..., 64:96].isnan().all()
    out[..., 64:96] = base[..., 64:96]
    assert torch.equal(out.view(torch.int16), base.view(torch.int16))
    last = [b - 1, n - 1, hq - 1]
    for bad in (float("inf"), nan):
        out = run(k, v, changed(q, *last, 40, to=bad))
        assert out[tuple(last)].isnan().all()
        out[tuple(last)] = base[tuple(last)]
        assert torch.equal(out.view(torch.int16), base.view(torch.int16))
    assert run(changed(k, slice(None), ctx // 3, slice(None), 5), v, q).isnan().all()
    short = run(k, v, q, ctx - 1)
    hidden = run(changed(k, slice(None), ctx - 1, slice(None), 5), changed(v, slice(None), ctx - 1, slice(None), 5), q, ctx - 1)
    assert short.isfinite().all() and torch.equal(short.view(torch.int16), hidden.view(torch.int16))


@pytest.mark.parametrize("n,ctx,hq,hkv,b", KERNELS)
def test_largest_numbers(n, ctx, hq, hkv, b):
    """Keys and values up to bf16's largest; such values in few positions, so that the sums stay in range."""
    rng = np.random.default_rng(n)
    page = 16
    per = (ctx + page - 1) // page
    p = D.CacheParams(b, hkv, 128, page, b * per, per, E4)
    k, v = (S.bf16(rng.normal(size=(b, ctx, hkv, 128))) for _ in range(2))
    k[..., :32] = 0.0
    k[:, 5, :, 3], k[:, 21, :, 3] = S.bf16(np.float32(3.38e38)), S.bf16(np.float32(-3.3e38))
    v[:, 37, :, 100], v[:, ctx - 1, :, 64] = S.bf16(np.float32(3.35e38)), S.bf16(np.float32(-3.39e38))
    q = np.zeros((b, n, hq, 128), np.float32)
    q[..., 3] = 2.0 ** -124                            # scores of +-12 from the largest keys, 0 from the others
    kt = vt = np.zeros((b, n, hkv, 128), np.float32)
    c = make_cache(p, np.arange(b * per).reshape(b, per))
    D.cache_write(p, c, put(k), put(v), ctx)
    a = D.AttnParams(b, n, ctx, hq, hkv, 128, 0.125)
    need = D.tree_attention_paged_workspace_size(a, p)
    ws = torch.empty(need, dtype=torch.uint8, device=device()) if need else None
    out = torch.zeros(b, n, hq, 128, dtype=torch.bfloat16, device=device())
    say(f"tree_attention_paged e2m1, largest numbers: b={b} B={n} ctx={ctx} heads={hq}/{hkv}")
    D.tree_attention_paged(a, p, c, put(q), put(kt), put(vt), None, None, out, ws)
    got = out.double().cpu().numpy()
    assert np.isfinite(got).all()
    keys, values = R.held(k), R.held(v)
    assert np.abs(keys).max() == np.abs(values).max() == 6.0 * 2.0 ** 125
    for r in {0, b - 1}:
        for h in {0, hq - 1}:
            g = h // (hq // hkv)
            see = np.concatenate([np.ones((n, ctx), bool), np.tril(np.ones((n, n), bool))], axis=1)
            kk, vv = np.concatenate([keys[r, :, g], kt[r, :, g]]), np.concatenate([values[r, :, g], vt[r, :, g]])
            want = S.attention(q[r, :, h].astype(np.float64), kk, vv, see, float(np.float32(0.125)))
            tol = (2.0 ** -8 + 2.0 ** -9) * np.abs(vv).max(axis=0) + 2.0 ** -8 * np.abs(want)
            assert (np.abs(got[r, :, h] - want) <= tol).all(), (r, h)


def test_pages_past_4_gib():
    """Pages of which keys, values and exponents lie far into the pool."""
    c = Case4(1, 5, 600, 8, 8, 256, seed=10)
    n = (5 << 30) // (8 * 256 * 64)
    far = D.CacheParams(1, 8, 128, 256, n, c.p.max_pages, E4)
    big = D.DeviceCache.alloc(far, device())
    at = [n - 1 - i for i in range(c.p.max_pages)]
    for to, of in zip(at, c.table[0]):
        for x, y in ((big.k, c.c.k), (big.v, c.c.v), (big.k_exp, c.c.k_exp), (big.v_exp, c.c.v_exp)):
            x[to].copy_(y[int(of)])
    want = c.run()
    big.table.copy_(torch.tensor([at], dtype=torch.int32))
    c.p, c.c, c.table = far, big, np.array([at])
    assert torch.equal(c.check(heads=[0, 7]), want)
    del big, c
    torch.cuda.empty_cache()
