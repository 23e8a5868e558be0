"""The paged cache in 4 bits on the GPU: writes and reads against the plain form, bit
for bit (the rounding to e2m1 is defined exactly, everything else is a copy)."""
import numpy as np
import pytest
import torch

from paper_2608_13524_amd import dartree as D
from tests import more_ref as R
from tests import serve_ref as S
from tests.gpu_util import device, say
from tests.test_gpu_cache import make_cache, normal, tables

pytestmark = pytest.mark.gpu
E4 = D.CACHE_E2M1
NAMES = ("k", "v", "k_exp", "v_exp")


def i32(a):
    return None if a is None else torch.from_numpy(np.ascontiguousarray(a, np.int32)).to(device())


def put(x):
    return torch.from_numpy(x).to(device()).bfloat16()


def host(c):
    torch.cuda.synchronize()
    return {n: getattr(c, n).cpu().numpy().copy() for n in NAMES}


def expect(before, p, table, k, v, rows, index, counts, start):
    out = {n: x.copy() for n, x in before.items()}
    for q in range(p.batch):
        for i in range(rows if counts is None else min(max(int(counts[q]), 0), rows)):
            j = i if index is None else int(index[q, i])
            at = S.slot(table[q], p.page, p.num_pages, (0 if start is None else int(start[q])) + i)
            if at is None or not 0 <= j < k.shape[1]:
                continue
            for name, x in (("k", k), ("v", v)):
                out[name][at[0], :, at[1]], out[name + "_exp"][at[0], :, at[1]] = R.quantise(x[q, j])
    return out


def run_write(p, table, k, v, rows, index=None, counts=None, start=None, fused=False, fill=0x55):
    c = make_cache(p, table, fill)
    before = host(c)
    dk, dv = put(k), put(v)
    if fused:   # keys and values in the rows of one wider tensor
        wide = torch.cat([dk, dk, dv, dv], dim=2)
        h = p.heads_kv
        dk, dv = wide[:, :, h:2 * h], wide[:, :, 3 * h:]
    say(f"cache_write e2m1 b={p.batch} src={k.shape[1]} rows={rows} heads={p.heads_kv} page={p.page}")
    D.cache_write(p, c, dk, dv, rows, index=i32(index), counts=i32(counts), start=i32(start))
    want, got = expect(before, p, table, k, v, rows, index, counts, start), host(c)
    for name in NAMES:
        assert np.array_equal(got[name], want[name]), name
    return c


@pytest.mark.parametrize("b,src,heads,page,fused", [(1, 1, 1, 16, False), (3, 1, 8, 64, True), (2, 37, 3, 16, False),
                                                    (2, 130, 2, 32, True), (1, 300, 5, 128, True), (2, 257, 1, 256, False)])
def test_write_prompts_and_tokens(b, src, heads, page, fused):
    rng = np.random.default_rng(src + page)
    start = rng.integers(0, page + 3, size=b)
    per = (int(start.max()) + src + page - 1) // page
    p = D.CacheParams(b, heads, 128, page, b * per + 1, per, E4)
    table = tables(rng, b, per, p.num_pages)
    k, v = normal(rng, (b, src, heads, 128)), normal(rng, (b, src, heads, 128))
    run_write(p, table, k, v, src, start=start, fused=fused)
    run_write(p, table, k, v, src, counts=rng.integers(-1, src + 2, size=b), fused=not fused, fill=0xFF)


def test_write_accepted_nodes():
    """Rows by an acceptance walk's indices; what the walk or the table leave out is not written."""
    rng = np.random.default_rng(8)
    p = D.CacheParams(5, 4, 128, 16, 40, 4, E4)
    table = tables(rng, 5, 4, 40)
    table[1, 1], table[2, 0], table[2, 2], table[3, 3] = -1, 40, np.iinfo(np.int32).min, np.iinfo(np.int32).max
    k, v = normal(rng, (5, 20, 4, 128)), normal(rng, (5, 20, 4, 128))
    index = rng.integers(0, 20, size=(5, 12))
    index[0, 7:], index[1, 3], index[4, 2], index[4, 5] = -1, 20, -7, np.iinfo(np.int32).max
    run_write(p, table, k, v, 12, index=index, counts=np.array([12, 12, 0, -3, 100]), start=np.array([10, 13, 0, 5, 57]))
    run_write(p, table, k, v, 12, index=index, start=np.array([-5, 60, 28, 64, np.iinfo(np.int32).max]))


def border_rows():
    rng = np.random.default_rng(9)
    rows = [np.zeros(128), np.full(128, -0.0), np.full(128, 3.38e38), np.full(128, -1e-38), np.full(128, 1e-30)]
    for e in (-99, -100, -101, -103, 0, 3, 60, 119, 124, 125):
        for top in (6.0, 6.03125, 5.96875, 4.0, 3.984375, 3.0, 3.015625):
            rows.append(rng.normal(size=128) * 2.0 ** e)
            rows[-1][::32] = top * 2.0 ** e
    ties = np.concatenate([[0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 6.0], [0.251, 0.249, 0.751, 0.749, 2.52, 2.48, 5.03, 4.97]])
    rows += [np.resize(ties, 128), -np.resize(ties, 128), np.resize(ties, 128) * 2.0 ** -100, np.resize(ties, 128) * 2.0 ** -101]
    rows.append(np.concatenate([6.0 * 2.0 ** -np.arange(32.0)] * 4) * np.repeat(2.0 ** np.array([0.0, 40.0, -40.0, -95.0]), 32))
    return S.bf16(np.array(rows))


def test_write_borders_of_the_scale():
    """Blocks of zeros, the largest and smallest numbers, maxima at and next to 6 * 2^e, ties between codes."""
    x = border_rows().reshape(1, -1, 1, 128)
    p = D.CacheParams(1, 1, 128, 16, 16, 8, E4)
    c = run_write(p, tables(np.random.default_rng(9), 1, 8, 16), x, x[:, ::-1].copy(), x.shape[1])
    k, v = (torch.zeros(1, x.shape[1], 1, 128, dtype=torch.bfloat16, device=device()) for _ in range(2))
    D.cache_read(p, c, k, v)
    assert np.array_equal(k.double().cpu().numpy(), R.held(x))
    assert np.array_equal(v.double().cpu().numpy(), R.held(x[:, ::-1]))


@pytest.mark.parametrize("b,rows,heads,page", [(1, 1, 1, 16), (3, 40, 2, 16), (2, 100, 8, 64), (2, 300, 3, 256)])
def test_read_back(b, rows, heads, page):
    """What was written, as the values held; rows past the count untouched; no page: zeros."""
    rng = np.random.default_rng(rows + heads)
    start = rng.integers(0, page, size=b)
    per = (int(start.max()) + rows + page - 1) // page
    p = D.CacheParams(b, heads, 128, page, b * per + 3, per, E4)
    table = tables(rng, b, per, p.num_pages)
    k, v = normal(rng, (b, rows, heads, 128)), normal(rng, (b, rows, heads, 128))
    c = run_write(p, table, k, v, rows, start=start)
    hole = None
    if per > 1:
        hole = (b - 1, per - 1)
        c.table[hole] = p.num_pages
    counts = rng.integers(0, rows + 2, size=b)
    counts[-1] = rows
    ok = torch.full((b, rows, heads, 128), 7.0, dtype=torch.bfloat16, device=device())
    ov = torch.full_like(ok, -7.0)
    say(f"cache_read e2m1 b={b} rows={rows} heads={heads} page={page}")
    D.cache_read(p, c, ok, ov, counts=i32(counts), start=i32(start))
    for got, src, rest in ((ok, k, 7.0), (ov, v, -7.0)):
        want = R.held(src)
        for q in range(b):
            want[q, min(int(counts[q]), rows):] = rest
            if hole and q == hole[0]:
                want[q, max(hole[1] * page - int(start[q]), 0):rows] = 0.0
        assert np.array_equal(got.double().cpu().numpy(), want)


def test_values_that_are_not_finite():
    """32 elements with a NaN or an infinity are NaN, the others of the row keep theirs."""
    p = D.CacheParams(1, 1, 128, 16, 2, 1, E4)
    c = make_cache(p, np.array([[1]]))
    x = np.ones((1, 5, 1, 128), np.float32)
    x[0, 0, 0, 3], x[0, 1, 0, 36], x[0, 2, 0, 127], x[0, 3], x[0, 4, 0, 64:66] = np.inf, np.nan, -np.inf, np.nan, (3e38, np.nan)
    say("cache_write e2m1 of infinities and NaN")
    D.cache_write(p, c, put(x), put(-x), 5)
    out = [torch.zeros(1, 5, 1, 128, dtype=torch.bfloat16, device=device()) for _ in range(2)]
    D.cache_read(p, c, *out)
    want = np.ones((5, 128))
    want[0, :32] = want[1, 32:64] = want[2, 96:] = want[3] = want[4, 64:96] = np.nan
    for o, sign in zip(out, (1.0, -1.0)):
        assert np.array_equal(o.double().cpu().numpy()[0, :, 0], sign * want, equal_nan=True)


def test_pages_past_4_gib():
    """Pages whose elements lie past 2^32 bytes of the pool."""
    rng = np.random.default_rng(4)
    n = (5 << 30) // (8 * 256 * 64)
    p = D.CacheParams(1, 8, 128, 256, n, 2, E4)
    c = D.DeviceCache.alloc(p, device())
    c.table.copy_(i32([[n - 1, n - 7]]))
    k, v = normal(rng, (1, 300, 8, 128)), normal(rng, (1, 300, 8, 128))
    say(f"cache e2m1 far pages={n}")
    D.cache_write(p, c, put(k), put(v), 300)
    ok, ov = (torch.empty(1, 300, 8, 128, dtype=torch.bfloat16, device=device()) for _ in range(2))
    D.cache_read(p, c, ok, ov)
    for got, src in ((ok, k), (ov, v)):
        assert np.array_equal(got.double().cpu().numpy(), R.held(src))
    del c
    torch.cuda.empty_cache()
