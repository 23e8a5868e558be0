"""The pages of a cache on the GPU against plain loops over the table: all integers,
so everything has to be equal."""
import numpy as np
import pytest
import torch

from paper_2608_13524_amd import dartree as D
from tests import more_ref as R
from tests.gpu_util import device, say

pytestmark = pytest.mark.gpu
LOW, HIGH = np.iinfo(np.int32).min, np.iinfo(np.int32).max


def i32(a):
    return None if a is None else torch.from_numpy(np.ascontiguousarray(a, np.int32)).to(device())


def params(b, columns, num_pages, page=16, heads=1, kind=D.CACHE_BF16):
    return D.CacheParams(b, heads, 128, page, num_pages, columns, kind)


def random_table(rng, b, columns, num_pages, named=0.5, shared=0.2):
    """A table of which `named` of the entries name a page, `shared` of those one of a few; odd entries name none."""
    order = rng.permutation(num_pages)
    table = np.full((b, columns), -1, np.int64)
    some = np.flatnonzero(rng.random(b * columns) < named)[:num_pages]
    table.ravel()[some] = order[:len(some)]
    again = rng.random(table.shape) < shared
    table[again] = order[rng.integers(0, max(1, min(num_pages, 5)), size=int(again.sum()))]
    odd = rng.random(table.shape) < 0.05
    table[odd] = rng.choice([num_pages, LOW, HIGH, -7], size=int(odd.sum()))
    return table.astype(np.int32)


SHAPES = [(1, 1, 1), (1, 3, 2), (2, 5, 33), (7, 13, 64), (3, 1, 5), (64, 40, 3000), (1, 2000, 2500), (300, 9, 70000), (1500, 3, 100),
          (2, 70000, 300000), (5, 33, 1024), (128, 128, 65536), (128, 128, 65537), (182, 181, 20000), (1024, 1, 2000),
          (1025, 1, 900)]


def run_reserve(p, table, rows, start, counts, place="apart", source=None):
    dev = device()
    columns = min(p.max_pages, (rows + p.page - 2) // p.page + 1)
    t = i32(table)
    out = t if place == "in" else torch.full_like(t, 99)
    pairs = torch.full((p.batch * columns + 3, 2), -9, dtype=torch.int32, device=dev)
    totals, granted = torch.full((2,), -9, dtype=torch.int32, device=dev), torch.full((p.batch,), -9, dtype=torch.int32, device=dev)
    ws = torch.full((D.pages_workspace_size(p),), 0xA5, dtype=torch.uint8, device=dev)
    say(f"pages_reserve b={p.batch} columns={p.max_pages} pages={p.num_pages} page={p.page} rows={rows} {place}")
    D.pages_reserve(p, t, out, rows, i32(start), i32(counts), pairs, totals, granted, ws)
    torch.cuda.synchronize()
    if place != "in":
        assert np.array_equal(t.cpu().numpy(), table)
    return out, pairs, totals, granted


def check_reserve(p, table, rows, start=None, counts=None, place="apart"):
    out, pairs, totals, granted = run_reserve(p, table, rows, start, counts, place)
    want = R.reserve(table, p.page, p.num_pages, rows, start, counts)
    assert totals.tolist() == list(want[2])
    assert np.array_equal(out.cpu().numpy(), want[0]) and np.array_equal(granted.cpu().numpy(), want[3])
    n = len(want[1])
    assert pairs[:n].tolist() == [list(x) for x in want[1]] and (pairs[n:] == -9).all()
    return want


@pytest.mark.parametrize("b,columns,num_pages", SHAPES)
def test_reserve(b, columns, num_pages):
    rng = np.random.default_rng(num_pages + b)
    for page, rows, named in ((16, 1, 0.5), (64, 100, 0.7), (256, 3000, 0.3)):
        p = params(b, columns, num_pages, page)
        table = random_table(rng, b, columns, num_pages, named)
        start = rng.integers(-page, columns * page + page, size=b)
        check_reserve(p, table, rows, start, rng.integers(-1, rows + 2, size=b))
        check_reserve(p, table, rows, start, None, "in")
        check_reserve(p, table, min(rows, 40))


def test_reserve_when_pages_run_out():
    """Requests are served in order as far as pages go; one that needs none is, whatever the others need."""
    table = np.full((6, 8), -1, np.int32)
    table[0, 0], table[3, :2], table[5, 0] = 7, [1, 2], 7
    p = params(6, 8, 12)
    start, counts = [16, 0, 0, 0, 0, 8], [48, 64, 0, 32, 16, 4]
    for num_pages in (3, 4, 7, 8, 9, 10, 11, 12, 13, 14, 40):
        table[0, 0] = table[5, 0] = min(7, num_pages - 1)
        table[3, :2] = [0, 1]
        p.num_pages = num_pages
        for place in ("apart", "in"):
            want = check_reserve(p, table, 64, start, counts, place)
        assert want[3][2] == want[3][3] == 1
    assert want[3].all()


def test_reserve_of_shared_pages():
    """Two that share a page and both write it; one written whole (not copied), from its middle, to its middle; a page that
    one row names twice; the holders that do not write keep it."""
    table = np.array([[3, 4, 5, -1], [3, 4, 5, -1], [3, 9, 9, -1], [8, 8, 1, -1]], np.int32)
    p = params(4, 4, 20)
    for start, counts in (([40, 40, 0, 0], [8, 8, 0, 0]), ([32, 20, 0, 0], [16, 40, 48, 48]), ([16, 15, 17, 31], [16, 18, 15, 1]),
                          ([47, 48, 32, 0], [1, 1, 16, 16]), ([0, 0, 0, 0], [64, 64, 64, 64])):
        for place in ("apart", "in"):
            check_reserve(p, table, 64, start, counts, place)


def test_reserve_at_the_ends_of_the_numbers():
    table = np.full((4, 3), -1, np.int32)
    p = params(4, 3, 10, 64)
    check_reserve(p, table, HIGH, [HIGH, LOW, 0, 191], [HIGH, HIGH, HIGH, LOW])
    check_reserve(p, table, 1 << 30, [-5, 128, 190, -64], [6, 1 << 30, 2, 65])
    check_reserve(p, table, 65, [63, 127, 64, 0])


@pytest.mark.parametrize("b,columns,num_pages", SHAPES)
def test_fork(b, columns, num_pages):
    rng = np.random.default_rng(b + columns)
    table = random_table(rng, b, columns, num_pages)
    p = params(b, columns, num_pages, 32)
    source = rng.integers(-2, b + 2, size=b)
    keep = rng.integers(-40, columns * 32 + 40, size=b)
    for s, k, place in ((source, keep, "apart"), (source, None, "apart"), (None, keep, "in"), (None, keep, "apart"), (None, None, "apart")):
        t = i32(table)
        out = t if place == "in" else torch.full_like(t, 99)
        say(f"pages_fork b={b} columns={columns} {place}")
        D.pages_fork(p, t, out, source=i32(s), keep=i32(k))
        torch.cuda.synchronize()
        assert np.array_equal(out.cpu().numpy(), R.fork(table, 32, s, k))


@pytest.mark.parametrize("b,columns,num_pages", SHAPES)
def test_compact(b, columns, num_pages):
    rng = np.random.default_rng(columns + num_pages)
    p = params(b, columns, num_pages)
    dev = device()
    for named in (0.0, 0.1, 0.5, 1.0):
        table = random_table(rng, b, columns, num_pages, named, shared=min(named, 0.1))
        want = R.compact(table, num_pages)
        for place in ("apart", "in"):
            t = i32(table)
            out = t if place == "in" else torch.full_like(t, 99)
            pairs = torch.full((num_pages // 2 + 2, 2), -9, dtype=torch.int32, device=dev)
            totals = torch.full((2,), -9, dtype=torch.int32, device=dev)
            ws = torch.full((D.pages_workspace_size(p),), 0xA5, dtype=torch.uint8, device=dev)
            say(f"pages_compact b={b} columns={columns} pages={num_pages} named={named} {place}")
            D.pages_compact(p, t, out, pairs, totals, ws)
            torch.cuda.synchronize()
            assert totals.tolist() == list(want[2]) and np.array_equal(out.cpu().numpy(), want[0])
            n = len(want[1])
            assert pairs[:n].tolist() == [list(x) for x in want[1]] and (pairs[n:] == -9).all()


@pytest.mark.parametrize("kind", [D.CACHE_BF16, D.CACHE_E4M3, D.CACHE_E2M1])
@pytest.mark.parametrize("heads,page,num_pages", [(1, 16, 3), (8, 64, 50), (3, 256, 20), (1, 32, 4000)])
def test_copy(kind, heads, page, num_pages):
    """Pages copied by a list; pairs outside the pool and entries past the count are left out, all other pages as they were."""
    rng = np.random.default_rng(num_pages + heads)
    p = params(1, 1, num_pages, page, heads, kind)
    c = D.DeviceCache.alloc(p, device())
    names = [n for n in ("k", "v", "k_exp", "v_exp") if getattr(c, n) is not None]
    for n in names:
        getattr(c, n).view(torch.uint8).random_(0, 256)
    before = {n: getattr(c, n).view(torch.uint8).cpu().clone() for n in names}
    order = rng.permutation(num_pages)
    half = num_pages // 2
    pairs = np.stack([rng.choice(order[:num_pages - half], half), order[num_pages - half:]], axis=1).astype(np.int64)
    odd = np.array([[-1, order[-1]], [order[0], num_pages], [LOW, HIGH], [order[0], order[0]]])
    listed = np.concatenate([pairs[:half // 2], odd, pairs[half // 2:]])
    for count in (0, 1, len(listed) - 1, len(listed), HIGH, LOW):
        for n in names:
            getattr(c, n).view(torch.uint8).copy_(before[n])
        want = {n: x.clone() for n, x in before.items()}
        for src, dst in listed[:max(min(count, len(listed)), 0)]:
            if 0 <= src < num_pages and 0 <= dst < num_pages:
                for n in names:
                    want[n][dst] = before[n][src]
        say(f"cache_copy type={kind} heads={heads} page={page} pages={num_pages} count={count}")
        D.cache_copy(p, c, i32(listed), i32([count, 77]))
        torch.cuda.synchronize()
        for n in names:
            assert torch.equal(getattr(c, n).view(torch.uint8).cpu(), want[n]), n


def test_copy_past_4_gib():
    kind, n = D.CACHE_E4M3, (5 << 30) // (8 * 256 * 128)
    p = params(1, 1, n, 256, 8, kind)
    c = D.DeviceCache.alloc(p, device())
    for x in (c.k, c.v, c.k_exp, c.v_exp):
        x[:2].view(torch.uint8).random_(0, 256)
        x[n - 2:].view(torch.uint8).zero_()
    say(f"cache_copy far pages={n}")
    D.cache_copy(p, c, i32([[0, n - 1], [1, n - 2]]), i32([2]))
    torch.cuda.synchronize()
    for x in (c.k, c.v, c.k_exp, c.v_exp):
        y = x.view(torch.uint8)
        assert torch.equal(y[0], y[n - 1]) and torch.equal(y[1], y[n - 2]) and bool((y[0] != 0).any())
    del c, x, y
    torch.cuda.empty_cache()


def test_replayed_with_a_shared_workspace():
    """Two graphs of reserve and compact over tables of their own, one workspace; eager calls between the replays."""
    rng = np.random.default_rng(5)
    p, dev = params(40, 30, 2000), device()
    ws = torch.empty(D.pages_workspace_size(p), dtype=torch.uint8, device=dev)

    class State:
        def __init__(self):
            self.table, self.mid, self.out = (torch.full((40, 30), -1, dtype=torch.int32, device=dev) for _ in range(3))
            self.start = torch.zeros(40, dtype=torch.int32, device=dev)
            self.pairs, self.moves = (torch.full((n, 2), -1, dtype=torch.int32, device=dev) for n in (80, 1000))
            self.totals, self.moved = (torch.zeros(2, dtype=torch.int32, device=dev) for _ in range(2))
            self.granted = torch.zeros(40, dtype=torch.int32, device=dev)

        def step(self):
            D.pages_reserve(p, self.table, self.mid, 17, self.start, None, self.pairs, self.totals, self.granted, ws)
            D.pages_compact(p, self.mid, self.out, self.moves, self.moved, ws)

        def results(self):
            torch.cuda.synchronize()
            n, m = self.totals[0].item(), self.moved[0].item()
            return [x.clone() for x in (self.mid, self.out, self.pairs[:n], self.moves[:m], self.totals, self.moved, self.granted)]

    states, eager = [State(), State()], State()
    eager.step()
    torch.cuda.synchronize()
    graphs = []
    for s in states:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            s.step()
        graphs.append(g)
    for i in range(4):
        tables = [i32(random_table(rng, 40, 30, 2000, 0.6)) for _ in states]
        starts = [i32(rng.integers(0, 470, size=40)) for _ in states]
        for g, s, t, at in zip(graphs, states, tables, starts):
            s.table.copy_(t)
            s.start.copy_(at)
            say(f"pages replay {i}")
            g.replay()
        got = [s.results() for s in states]
        for r, t, at in zip(got, tables, starts):
            eager.table.copy_(t)
            eager.start.copy_(at)
            eager.step()
            assert all(torch.equal(a, b) for a, b in zip(r, eager.results()))
