"""The paged cache and the attention over it at the ends of the numbers' range."""
import numpy as np
import pytest
import torch

from paper_2608_13524_amd import dartree as D
from tests import serve_ref as S
from tests.gpu_util import device, say
from tests.test_gpu_cache import BF, E8, make_cache, run_write, tables

pytestmark = pytest.mark.gpu
LARGEST = 255.0 * 2.0 ** 120   # bf16 0x7F7F


def held(x):
    """What a row in e4m3 stands for: +-2^128 is not a bf16 number, the largest one stands in its place."""
    q, e = S.quantise(x)
    return np.clip(q * 2.0 ** e[..., None], -LARGEST, LARGEST)


def top_rows():
    """Every finite bf16 number from 2^126 on, of both signs, as the largest of its row and all together."""
    top = (np.arange(0x7E80, 0x7F80, dtype=np.uint32) << 16).view(np.float32)
    rows = np.zeros((2 * len(top), 128), np.float32)
    rows[::2, 5], rows[1::2, 77] = top, -top
    rows[:, 6] = 2.0 ** 100
    return np.concatenate([rows, np.resize(np.concatenate([top, -top]), (4, 128))])


def test_read_back_largest_numbers():
    """The nearest held value is within 2^-4 of a number, and so is the largest bf16 number of those that
    round to 2^128 (248 .. 255 times 2^120: at most 7 / 248)."""
    x = top_rows()
    n = len(x)
    x = S.bf16(x).reshape(1, n, 1, 128)
    per = (n + 15) // 16
    p = D.CacheParams(1, 1, 128, 16, per + 1, per, E8)
    c = run_write(p, tables(np.random.default_rng(1), 1, per, per + 1), x, -x, n)
    k, v = (torch.zeros(1, n, 1, 128, dtype=torch.bfloat16, device=device()) for _ in range(2))
    D.cache_read(p, c, k, v)
    torch.cuda.synchronize()
    for got, src in ((k, x), (v, -x)):
        got = got.double().cpu().numpy()
        assert np.isfinite(got).all()
        assert np.array_equal(got, held(src))
        big = np.abs(src) >= 2.0 ** 126
        assert (np.abs(got - src)[big] <= 2.0 ** -4 * np.abs(src.astype(np.float64))[big]).all()


# budget, context, heads_q, heads_kv, requests: few rows, one block an item, tiles of 64, 128 and 256 rows
KERNELS = [(1, 3000, 2, 1, 1), (40, 60, 4, 2, 1), (40, 3000, 4, 2, 8), (300, 3000, 8, 1, 8), (64, 40, 32, 8, 128)]


@pytest.mark.parametrize("n,ctx,hq,hkv,b", KERNELS)
def test_attention_over_largest_numbers(n, ctx, hq, hkv, b):
    """One position of every 16 of the first 64 holds such a key or such a value, so that the sums stay in range.
    Tolerance: test_gpu_paged.py's, of these keys and values."""
    rng = np.random.default_rng(n)
    dev, page = device(), 16
    per = (ctx + page - 1) // page
    p = D.CacheParams(b, hkv, 128, page, b * per, per, E8)
    k, v = (S.bf16(rng.normal(size=(b, ctx, hkv, 128))) for _ in range(2))
    k[..., 3] = 0.0
    k[:, 5] = 0.0
    k[:, 5, :, 3] = S.bf16(np.float32(3.38e38))
    k[:, 21] = 0.0
    k[:, 21, :, 3] = S.bf16(np.float32(-3.3e38))
    v[:, 37, :, 100] = S.bf16(np.float32(3.35e38))
    v[:, ctx - 1, :, 64] = S.bf16(np.float32(-3.39e38))
    q = np.zeros((b, n, hq, 128), np.float32)
    q[..., 3] = 2.0 ** -124                            # scores of +-16 from the largest keys, 0 from the others
    kt = vt = np.zeros((b, n, hkv, 128), np.float32)
    c = make_cache(p, np.arange(b * per).reshape(b, per))
    put = lambda x: torch.from_numpy(x).to(dev).bfloat16()
    D.cache_write(p, c, put(k), put(v), ctx)
    a = D.AttnParams(b, n, ctx, hq, hkv, 128, 0.125)
    need = D.tree_attention_paged_workspace_size(a, p)
    ws = torch.empty(need, dtype=torch.uint8, device=dev) if need else None
    out = torch.zeros(b, n, hq, 128, dtype=torch.bfloat16, device=dev)
    say(f"tree_attention_paged, largest numbers: b={b} B={n} ctx={ctx} heads={hq}/{hkv}")
    D.tree_attention_paged(a, p, c, put(q), put(kt), put(vt), None, None, out, ws)
    torch.cuda.synchronize()
    got = out.double().cpu().numpy()
    assert np.isfinite(got).all()
    keys, values = held(k), held(v)
    for r in {0, b - 1}:
        for h in {0, hq - 1}:
            g = h // (hq // hkv)
            see = np.concatenate([np.ones((n, ctx), bool), np.tril(np.ones((n, n), bool))], axis=1)
            kk, vv = np.concatenate([keys[r, :, g], kt[r, :, g]]), np.concatenate([values[r, :, g], vt[r, :, g]])
            want = S.attention(q[r, :, h].astype(np.float64), kk, vv, see, float(np.float32(0.125)))
            tol = (2.0 ** -8 + 2.0 ** -9) * np.abs(vv).max(axis=0) + 2.0 ** -8 * np.abs(want)
            assert (np.abs(got[r, :, h] - want) <= tol).all(), (r, h)


def test_large_numbers_beside_an_infinity():
    """An e4m3 row with an infinity holds a NaN in its place and zeros elsewhere, whatever the other numbers."""
    dev = device()
    p = D.CacheParams(1, 1, 128, 16, 1, 1, E8)
    c = make_cache(p, np.zeros((1, 1), int))
    x = np.zeros((4, 128), np.float32)
    x[:, :6] = [1e38, -3.38e38, 2.0 ** 112, -2.0 ** 111, 2.0 ** 109, 1.0]
    x[0, 9], x[1, 9], x[2, 9] = np.inf, -np.inf, np.inf
    x[2, 10], x[3, 9] = np.nan, np.nan
    put = torch.from_numpy(x).to(dev).bfloat16().view(1, 4, 1, 128)
    say("cache_write of large numbers beside an infinity")
    D.cache_write(p, c, put, put, 4)
    out = [torch.ones(1, 4, 1, 128, dtype=torch.bfloat16, device=dev) for _ in range(2)]
    D.cache_read(p, c, *out)
    torch.cuda.synchronize()
    want = np.zeros((4, 128))
    want[:, 9] = want[2, 10] = np.nan
    rest = S.bf16(x[3]).astype(np.float64)
    rest[9] = 0.0
    want[3, :9] = held(rest[None])[0, :9]              # a NaN alone changes nothing else
    for o in out:
        assert np.array_equal(o.double().cpu().numpy()[0, :, 0], want, equal_nan=True)


@pytest.mark.parametrize("kind", [E8, BF])
@pytest.mark.parametrize("n,ctx,hq,hkv,b", KERNELS)
def test_a_nan_in_the_context(kind, n, ctx, hq, hkv, b):
    """A position whose value has a NaN in one element: that element of every row is one, all others keep their bits."""
    rng = np.random.default_rng(n + 1)
    dev, page = device(), 16
    per = (ctx + page - 1) // page
    p = D.CacheParams(b, hkv, 128, page, b * per, per, kind)
    x = torch.from_numpy(S.bf16(rng.normal(size=(b, ctx, hkv, 128)))).to(dev).bfloat16()
    q = torch.from_numpy(S.bf16(rng.normal(size=(b, n, hq, 128)))).to(dev).bfloat16()
    t = torch.from_numpy(S.bf16(rng.normal(size=(b, n, hkv, 128)))).to(dev).bfloat16()
    c = make_cache(p, rng.permutation(b * per).reshape(b, per))
    a = D.AttnParams(b, n, ctx, hq, hkv, 128, 0.0884)
    need = D.tree_attention_paged_workspace_size(a, p)
    ws = torch.empty(need, dtype=torch.uint8, device=dev) if need else None
    outs = []
    for value in (0.0, float("nan")):
        v = x.clone()
        v[:, ctx // 2, :, 70] = value
        D.cache_write(p, c, x, v, ctx)
        out = torch.zeros(b, n, hq, 128, dtype=torch.bfloat16, device=dev)
        say(f"tree_attention_paged, a NaN in the context: b={b} B={n} ctx={ctx} heads={hq}/{hkv} type={kind}")
        D.tree_attention_paged(a, p, c, q, t, t, None, None, out, ws)
        torch.cuda.synchronize()
        outs.append(out.cpu())
    assert outs[0].isfinite().all() and outs[1][..., 70].isnan().all()
    outs[1][..., 70] = outs[0][..., 70]
    assert torch.equal(outs[0].view(torch.int16), outs[1].view(torch.int16))
