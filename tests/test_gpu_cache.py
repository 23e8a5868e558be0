"""The paged cache on the GPU: writes and reads against the plain form, bit for
bit (the rounding to e4m3 is defined exactly, everything else is a copy)."""
import numpy as np
import pytest
import torch

from paper_2608_13524_amd import dartree as D
from tests import serve_ref as S
from tests.gpu_util import device, say

pytestmark = pytest.mark.gpu

E8, BF = D.CACHE_E4M3, D.CACHE_BF16


def bits(x):
    """bf16 tensor as uint16 bit patterns on the host."""
    return x.view(torch.int16).cpu().numpy().view(np.uint16)


def make_cache(p, table, fill=0x55):
    """A cache whose memory holds `fill` bytes."""
    c = D.DeviceCache.alloc(p, device())
    for t in (c.k, c.v, c.k_exp, c.v_exp):
        if t is not None:
            t.view(torch.uint8).fill_(fill)
    c.table.copy_(torch.from_numpy(np.ascontiguousarray(table, np.int32)))
    return c


def tables(rng, b, per, num_pages):
    return rng.permutation(num_pages)[: b * per].reshape(b, per).astype(np.int32)


def host(c, p):
    """{k, v, k_exp, v_exp} as arrays: bf16 bits or e4m3 bytes, exponent bytes."""
    get = (lambda t: t.view(torch.uint8).cpu().numpy()) if p.type == E8 else bits
    return {"k": get(c.k).copy(), "v": get(c.v).copy(), **({"k_exp": c.k_exp.cpu().numpy().copy(), "v_exp": c.v_exp.cpu().numpy().copy()}
                                                           if p.type == E8 else {})}


CODES = None


def code_of(values):
    """e4m3 bytes of values on its grid (negative zero keeps its sign)."""
    global CODES
    if CODES is None:
        v = S.e4m3_values()
        CODES = {(abs(x), np.signbit(x)): i for i, x in enumerate(v) if not np.isnan(x)}
    return np.array([CODES[(abs(x), bool(np.signbit(x)))] for x in values.ravel()], np.uint8).reshape(values.shape)


def expect_write(before, p, table, k, v, rows, index, counts, start):
    out = {n: x.copy() for n, x in before.items()}
    src = k.shape[1]
    for q in range(p.batch):
        for i in range(rows if counts is None else min(max(int(counts[q]), 0), rows)):
            j = i if index is None else int(index[q, i])
            at = S.slot(table[q], p.page, p.num_pages, (0 if start is None else int(start[q])) + i)
            if at is None or not 0 <= j < src:
                continue
            for name, x in (("k", k), ("v", v)):
                row = x[q, j]
                if p.type == E8:
                    held, e = S.quantise(row)
                    out[name][at[0], :, at[1]] = code_of(held)
                    out[name + "_exp"][at[0], :, at[1]] = e + 127
                else:
                    out[name][at[0], :, at[1]] = (np.ascontiguousarray(row, np.float32).view(np.uint32) >> 16).astype(np.uint16)
    return out


def run_write(p, table, k, v, rows, index=None, counts=None, start=None, fused=False, fill=0x55):
    dev = device()
    c = make_cache(p, table, fill)
    before = host(c, p)
    dk, dv = (torch.from_numpy(x).to(dev).to(torch.bfloat16) for x in (k, v))
    if fused:   # keys and values in the rows of one wider tensor
        h = p.heads_kv
        wide = torch.zeros(*k.shape[:2], 4 * h, 128, dtype=torch.bfloat16, device=dev)
        wide[:, :, h:2 * h], wide[:, :, 3 * h:] = dk, dv
        dk, dv = wide[:, :, h:2 * h], wide[:, :, 3 * h:]
    i32 = lambda a: None if a is None else torch.from_numpy(np.ascontiguousarray(a, np.int32)).to(dev)
    say(f"cache_write b={p.batch} src={k.shape[1]} rows={rows} heads={p.heads_kv} page={p.page} type={p.type}")
    D.cache_write(p, c, dk, dv, rows, index=i32(index), counts=i32(counts), start=i32(start))
    torch.cuda.synchronize()
    want, got = expect_write(before, p, table, k, v, rows, index, counts, start), host(c, p)
    for name in want:
        assert np.array_equal(got[name], want[name]), name
    return c


def normal(rng, shape, spread=3.0):
    return S.bf16(rng.normal(size=shape) * np.exp(rng.normal(size=shape[:-1] + (1,)) * spread))


@pytest.mark.parametrize("kind", [E8, BF])
@pytest.mark.parametrize("b,src,heads,page,fused", [(1, 1, 1, 16, False), (3, 1, 8, 64, True), (2, 37, 3, 16, False),
                                                    (2, 130, 2, 32, True), (1, 300, 5, 128, True), (2, 257, 1, 256, False)])
def test_write_prompts_and_tokens(kind, b, src, heads, page, fused):
    rng = np.random.default_rng(src + page)
    start = rng.integers(0, page + 3, size=b)
    per = (int(start.max()) + src + page - 1) // page
    p = D.CacheParams(b, heads, 128, page, b * per + 1, per, kind)
    table = tables(rng, b, per, p.num_pages)
    k, v = normal(rng, (b, src, heads, 128)), normal(rng, (b, src, heads, 128))
    run_write(p, table, k, v, src, start=start, fused=fused)
    run_write(p, table, k, v, src, counts=rng.integers(-1, src + 2, size=b), fused=not fused, fill=0xFF)


@pytest.mark.parametrize("kind", [E8, BF])
def test_write_accepted_nodes(kind):
    """Rows by an acceptance walk's indices, -1 after the last; indices outside the source, the same index
    twice, positions before the first and past the last page, entries without a page."""
    rng = np.random.default_rng(8)
    p = D.CacheParams(5, 4, 128, 16, 40, 4, kind)
    table = tables(rng, 5, 4, 40)
    table[1, 1], table[2, 0], table[2, 2], table[3, 3] = -1, 40, np.iinfo(np.int32).min, np.iinfo(np.int32).max
    k, v = normal(rng, (5, 20, 4, 128)), normal(rng, (5, 20, 4, 128))
    index = rng.integers(0, 20, size=(5, 12))
    index[0, 7:], index[1, 3], index[4, 2], index[4, 5] = -1, 20, -7, np.iinfo(np.int32).max
    run_write(p, table, k, v, 12, index=index, counts=np.array([12, 12, 0, -3, 100]), start=np.array([10, 13, 0, 5, 57]))
    run_write(p, table, k, v, 12, index=index, start=np.array([-5, 60, 28, 64, np.iinfo(np.int32).max]))


def test_write_borders_of_the_scale():
    """Rows of zeros, the largest and smallest numbers, maxima at and next to 448 * 2^e, ties between codes."""
    rng = np.random.default_rng(9)
    rows = [np.zeros(128), np.full(128, -0.0), np.full(128, 3.38e38), np.full(128, -1e-38), np.full(128, 1e-30)]
    for e in (-99, -100, -101, -92, 0, 3, 60, 119):
        for top in (448.0, 450.0, 446.0, 256.0, 255.0):
            rows.append(rng.normal(size=128) * 2.0 ** e)
            rows[-1][5] = top * 2.0 ** e
    codes = S.e4m3_values()
    mids = np.array([(codes[i] + codes[i + 1]) / 2 for i in range(126)])   # halfway between neighbours
    rows += [np.concatenate([mids, [448.0, 2.0 ** -10]]), -np.concatenate([mids, [448.0, 1.5 * 2.0 ** -9]])]
    rows.append(np.concatenate([[448.0], 2.0 ** -np.arange(1.0, 128.0)]))
    x = S.bf16(np.array(rows)).reshape(1, len(rows), 1, 128)
    p = D.CacheParams(1, 1, 128, 16, 16, 8, E8)
    run_write(p, tables(rng, 1, 8, 16), x, x[:, ::-1].copy(), len(rows))


@pytest.mark.parametrize("kind", [E8, BF])
@pytest.mark.parametrize("b,rows,heads,page", [(1, 1, 1, 16), (3, 40, 2, 16), (2, 100, 8, 64), (2, 300, 3, 256)])
def test_read_back(kind, b, rows, heads, page):
    """What was written, as the values held; rows past the count untouched; no page: zeros."""
    rng = np.random.default_rng(rows + heads)
    dev = device()
    start = rng.integers(0, page, size=b)
    per = (int(start.max()) + rows + page - 1) // page
    p = D.CacheParams(b, heads, 128, page, b * per + 3, per, kind)
    table = tables(rng, b, per, p.num_pages)
    k, v = normal(rng, (b, rows, heads, 128)), normal(rng, (b, rows, heads, 128))
    c = run_write(p, table, k, v, rows, start=start)
    hole = None
    if per > 1:
        hole = (b - 1, per - 1)
        c.table[hole] = p.num_pages
    counts = rng.integers(0, rows + 2, size=b)
    counts[-1] = rows
    ok = torch.full((b, rows, heads, 128), 7.0, dtype=torch.bfloat16, device=dev)
    ov = torch.full_like(ok, -7.0)
    i32 = lambda a: torch.from_numpy(np.ascontiguousarray(a, np.int32)).to(dev)
    say(f"cache_read b={b} rows={rows} heads={heads} page={page} type={kind}")
    D.cache_read(p, c, ok, ov, counts=i32(counts), start=i32(start))
    torch.cuda.synchronize()
    for got, src, rest in ((ok, k, 7.0), (ov, v, -7.0)):
        held, e = S.quantise(src) if kind == E8 else (src, np.zeros(src.shape[:-1]))
        want = held.astype(np.float64) * 2.0 ** e[..., None]
        for q in range(b):
            want[q, min(int(counts[q]), rows):] = rest
            if hole and q == hole[0]:
                want[q, max(hole[1] * page - int(start[q]), 0):rows] = 0.0
        assert np.array_equal(got.float().cpu().numpy().astype(np.float64), want)


@pytest.mark.parametrize("kind", [E8, BF])
def test_values_that_are_not_finite(kind):
    """bf16 keeps them; e4m3 keeps NaN, an infinity becomes NaN and its row's other values 0."""
    dev = device()
    p = D.CacheParams(1, 1, 128, 16, 2, 1, kind)
    c = make_cache(p, np.array([[1]]))
    x = torch.ones(1, 4, 1, 128, dtype=torch.bfloat16, device=dev)
    x[0, 0, 0, 3], x[0, 1, 0, 4], x[0, 2, 0, 5], x[0, 3] = float("inf"), float("nan"), -float("inf"), float("nan")
    say(f"cache_write of infinities and NaN type={kind}")
    D.cache_write(p, c, x, x, 4)
    out = [torch.zeros_like(x) for _ in range(2)]
    D.cache_read(p, c, *out)
    torch.cuda.synchronize()
    want = x.float().cpu().numpy()[0, :, 0]
    if kind == E8:
        for row, at in ((0, 3), (2, 5)):
            want[row] = 0.0
            want[row, at] = np.nan
    for o in out:
        assert np.array_equal(o.float().cpu().numpy()[0, :, 0], want, equal_nan=True)


def test_read_without_counts_and_past_the_table():
    rng = np.random.default_rng(3)
    p = D.CacheParams(2, 2, 128, 16, 8, 2, BF)
    table = tables(rng, 2, 2, 8)
    k, v = normal(rng, (2, 32, 2, 128)), normal(rng, (2, 32, 2, 128))
    c = run_write(p, table, k, v, 32)
    ok = torch.ones(2, 40, 2, 128, dtype=torch.bfloat16, device=device())
    ov = torch.ones_like(ok)
    D.cache_read(p, c, ok, ov, start=torch.tensor([-3, 0], dtype=torch.int32, device=device()))
    torch.cuda.synchronize()
    want = np.zeros((2, 40, 2, 128), np.float32)
    want[0, 3:35], want[1, :32] = v[0], v[1]
    assert np.array_equal(ov.float().cpu().numpy(), want)


@pytest.mark.parametrize("kind", [E8, BF])
def test_pages_past_4_gib(kind):
    """Pages whose elements lie past 2^32 bytes of the pool."""
    rng = np.random.default_rng(4)
    page_bytes = 8 * 256 * 128 * (1 if kind == E8 else 2)
    n = (5 << 30) // page_bytes
    p = D.CacheParams(1, 8, 128, 256, n, 2, kind)
    c = D.DeviceCache.alloc(p, device())
    table = np.array([[n - 1, n - 7]])
    c.table.copy_(torch.from_numpy(table.astype(np.int32)))
    k, v = normal(rng, (1, 300, 8, 128)), normal(rng, (1, 300, 8, 128))
    dk, dv = (torch.from_numpy(x).to(device()).to(torch.bfloat16) for x in (k, v))
    say(f"cache far pages type={kind} pages={n}")
    D.cache_write(p, c, dk, dv, 300)
    ok, ov = torch.empty_like(dk), torch.empty_like(dv)
    D.cache_read(p, c, ok, ov)
    torch.cuda.synchronize()
    for got, src in ((ok, k), (ov, v)):
        held, e = S.quantise(src) if kind == E8 else (src, np.zeros(src.shape[:-1]))
        assert np.array_equal(got.float().cpu().numpy().astype(np.float64), held.astype(np.float64) * 2.0 ** e[..., None])
    assert int((c.k[n - 1].view(torch.uint8) != c.k[0].view(torch.uint8)).sum()) > 0
    del c
    torch.cuda.empty_cache()
