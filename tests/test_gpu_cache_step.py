"""Steps of a serving loop over a cache in 4 bits whose pages the library manages:
prompts turned to their positions and written, drafted trees turned to their depths,
their layer, the accepted nodes written into reserved pages, requests forked, ended
and compacted between; eagerly, on other streams and as replayed graphs.  What a
request holds is followed by plain lists."""
import numpy as np
import pytest
import torch

from paper_2608_13524_amd import dartree as D
from tests import more_ref as R
from tests import serve_ref as S
from tests.gpu_util import device, say
from tests.test_gpu_paged import random_tree, words_of

pytestmark = pytest.mark.gpu
B, HQ, HKV, PAGE, COLUMNS, POOL, NODES, DEPTH, PROMPT = 4, 8, 2, 16, 12, 40, 20, 5, 50
SCALE = 128.0 ** -0.5
KINDS = [D.CACHE_E2M1, D.CACHE_E4M3, D.CACHE_BF16]


def i32(x):
    return torch.tensor(np.asarray(x), dtype=torch.int32, device=device())


class Loop:
    """What a serving loop of four requests keeps."""

    def __init__(self, kind, seed):
        dev = device()
        self.p = D.CacheParams(B, HKV, 128, PAGE, POOL, COLUMNS, kind)
        self.cache = D.DeviceCache.alloc(self.p, dev)
        for t in (self.cache.k, self.cache.v, self.cache.k_exp, self.cache.v_exp):
            if t is not None:
                t.view(torch.uint8).fill_(0xFF)
        self.spare = self.cache.table.clone()
        self.length = i32([0] * B)
        self.a = D.AttnParams(B, NODES, COLUMNS * PAGE, HQ, HKV, 128, SCALE)
        need = D.tree_attention_paged_workspace_size(self.a, self.p)
        self.attn_ws = torch.empty(max(need, 256), dtype=torch.uint8, device=dev)
        self.pages_ws = torch.empty(D.pages_workspace_size(self.p), dtype=torch.uint8, device=dev)
        self.turns = D.rotary_turns(128)
        rows = max(PROMPT, DEPTH)
        self.pairs = i32([[-1, -1]] * (B * ((rows + PAGE - 2) // PAGE + 1)))
        self.moves = i32([[-1, -1]] * (POOL // 2))
        self.totals, self.moved, self.granted = i32([0, 0]), i32([0, 0]), i32([0] * B)
        self.qkv = torch.zeros(B, NODES, HQ + 2 * HKV, 128, dtype=torch.bfloat16, device=dev)
        self.out = torch.zeros(B, NODES, HQ, 128, dtype=torch.bfloat16, device=dev)
        self.depths, self.mask = i32([[1] * NODES] * B), torch.zeros(B, NODES, 1, dtype=torch.int64, device=dev)
        self.accepted, self.count = i32([[-1] * DEPTH] * B), i32([0] * B)
        self.source, self.keep = i32(range(B)), i32([0] * B)

    def rotary(self, qkv, rows, first, positions, start, counts, stream=None):
        p = D.RotaryParams(B, rows, HQ, HKV, 128, 128, D.ROTARY_HALF, D.BF16, 0, first, 1.0)
        q, k = qkv[:, :, :HQ], qkv[:, :, HQ:HQ + HKV]
        D.rotary(p, self.turns, q, k, q, k, positions=positions, start=start, counts=counts, stream=stream)

    def reserve(self, rows, counts, stream=None):
        D.pages_reserve(self.p, self.cache.table, self.cache.table, rows, self.length, counts, self.pairs[:B * ((rows + PAGE - 2) // PAGE + 1)],
                        self.totals, self.granted, self.pages_ws, stream=stream)
        D.cache_copy(self.p, self.cache, self.pairs, self.totals, stream=stream)

    def prompt(self, qkv, counts):
        rows = qkv.shape[1]
        self.rotary(qkv, rows, 0, None, self.length, counts)
        self.reserve(rows, counts)
        D.cache_write(self.p, self.cache, qkv[:, :, HQ:HQ + HKV], qkv[:, :, HQ + HKV:], rows, counts=counts, start=self.length)
        self.length += counts

    def step(self, stream=None):
        k, v = self.qkv[:, :, HQ:HQ + HKV], self.qkv[:, :, HQ + HKV:]
        self.rotary(self.qkv, NODES, -1, self.depths, self.length, None, stream)
        D.tree_attention_paged(self.a, self.p, self.cache, self.qkv[:, :, :HQ], k, v, self.mask, self.length, self.out, self.attn_ws,
                               stream=stream)
        self.reserve(DEPTH, self.count, stream)
        D.cache_write(self.p, self.cache, k, v, DEPTH, index=self.accepted, counts=self.count, start=self.length, stream=stream)
        self.length += self.count

    def fork(self, stream=None):
        D.pages_fork(self.p, self.cache.table, self.spare, source=self.source, keep=self.keep, stream=stream)
        self.cache.table.copy_(self.spare)
        self.length.copy_(self.keep)

    def compact(self, stream=None):
        D.pages_compact(self.p, self.cache.table, self.cache.table, self.moves, self.moved, self.pages_ws, stream=stream)
        D.cache_copy(self.p, self.cache, self.moves, self.moved, stream=stream)

    def put(self, rng):
        """A new drafted tree for each request, and which of its nodes will be accepted."""
        see = np.stack([random_tree(rng, NODES) for _ in range(B)])
        paths = [np.flatnonzero(s[rng.integers(NODES)])[:DEPTH] for s in see]
        accepted = np.full((B, DEPTH), -1)
        for q, path in enumerate(paths):
            accepted[q, :len(path)] = path
        x = S.bf16(rng.normal(size=(B, NODES, HQ + 2 * HKV, 128)))
        self.qkv.copy_(torch.from_numpy(x))
        self.depths.copy_(i32(see.sum(axis=2)))
        self.mask.copy_(torch.from_numpy(words_of(see)))
        self.accepted.copy_(i32(accepted))
        self.count.copy_(i32([len(p) for p in paths]))
        return x, see, paths

    def state(self):
        torch.cuda.synchronize()
        return [x.clone().view(torch.uint8) for x in (self.cache.table, self.length, self.out, self.qkv, self.granted, self.totals, self.moved)]

    def holds(self):
        """Keys and values of every request's positions, as the cache gives them back."""
        k, v = (torch.zeros(B, COLUMNS * PAGE, HKV, 128, dtype=torch.bfloat16, device=device()) for _ in range(2))
        D.cache_read(self.p, self.cache, k, v, counts=self.length)
        torch.cuda.synchronize()
        return k.double().cpu().numpy(), v.double().cpu().numpy()


def held(kind, x):
    if kind == D.CACHE_E2M1:
        return R.held(x)
    if kind == D.CACHE_E4M3:
        q, e = S.quantise(np.asarray(x))
        return q * 2.0 ** e[..., None]
    return np.asarray(x, np.float64)


def close(got, want, size):
    """Turned elements in bf16 (test_gpu_rotary.py): half a step, and 2^-21 of both elements of a pair."""
    return (np.abs(got - want) <= 2.0 ** -8 * np.abs(want) + 2.0 ** -20 * size).all()


@pytest.mark.parametrize("kind", KINDS)
def test_steps_follow_the_definitions(kind):
    rng = np.random.default_rng(kind + 1)
    loop, f = Loop(kind, 1), R.frequencies(128)
    rows = [[] for _ in range(B)]      # (k, v) of every position of a request, as held
    counts = np.array([PROMPT, 17, 0, 33])
    x = S.bf16(rng.normal(size=(B, PROMPT, HQ + 2 * HKV, 128)))
    qkv = torch.from_numpy(x).to(device()).bfloat16()
    say(f"prompts, type {kind}")
    loop.prompt(qkv, i32(counts))
    turned = qkv.double().cpu().numpy()
    at = np.arange(PROMPT)
    for q in range(B):
        n = counts[q]
        assert close(turned[q, :n, :HQ + HKV], R.rotate(x[q, :n, :HQ + HKV], at[:n], f, True), 16.0)
        assert np.array_equal(turned[q, n:], x[q, n:]) and np.array_equal(turned[q, :, HQ + HKV:], x[q, :, HQ + HKV:])
        rows[q] = [(held(kind, turned[q, i, HQ:HQ + HKV]), held(kind, turned[q, i, HQ + HKV:])) for i in range(n)]
    for i in range(6):
        if i == 2:     # request 2 continues request 0, request 1 has ended, request 3 goes back by 4
            source, keep = [0, 1, 0, 3], [len(rows[0]), 0, len(rows[0]), len(rows[3]) - 4]
            loop.source.copy_(i32(source))
            loop.keep.copy_(i32(keep))
            loop.fork()
            rows = [list(rows[s][:n]) for s, n in zip(source, keep)]
        if i == 4:
            before = [t.copy() for t in loop.holds()]
            loop.compact()
            table = loop.cache.table.cpu().numpy()
            assert table.max() < loop.moved[1].item() <= POOL and loop.moved[0].item() >= 0
            assert all(np.array_equal(a, b) for a, b in zip(before, loop.holds()))
        x, see, paths = loop.put(rng)
        say(f"step {i}, type {kind}, lengths {[len(r) for r in rows]}")
        loop.step()
        torch.cuda.synchronize()
        assert loop.granted.tolist() == [1] * B
        turned, out = loop.qkv.double().cpu().numpy(), loop.out.double().cpu().numpy()
        for q in range(B):
            ctx = len(rows[q])
            at = ctx + see[q].sum(axis=1) - 1
            assert close(turned[q, :, :HQ + HKV], R.rotate(x[q, :, :HQ + HKV], at, f, True), 16.0)
            full = np.concatenate([np.ones((NODES, ctx), bool), see[q]], axis=1)
            for h in range(HQ):
                g = h // (HQ // HKV)
                kk = np.array([r[0][g] for r in rows[q]] + list(turned[q, :, HQ + g]))
                vv = np.array([r[1][g] for r in rows[q]] + list(turned[q, :, HQ + HKV + g]))
                want = S.attention(turned[q, :, h], kk, vv, full, SCALE)
                tol = (2.0 ** -8 + 2.0 ** -9) * np.abs(vv).max(axis=0) + 2.0 ** -8 * np.abs(want)   # as in test_gpu_paged.py
                assert (np.abs(out[q, :, h] - want) <= tol).all()
            rows[q] += [(held(kind, turned[q, n, HQ:HQ + HKV]), held(kind, turned[q, n, HQ + HKV:])) for n in paths[q]]
        k, v = loop.holds()
        for q in range(B):
            n = len(rows[q])
            assert loop.length[q] == n
            assert np.array_equal(k[q, :n], np.array([r[0] for r in rows[q]]).reshape(n, HKV, 128))
            assert np.array_equal(v[q, :n], np.array([r[1] for r in rows[q]]).reshape(n, HKV, 128))
        # no page of two requests is one that both may write
        table = loop.cache.table.cpu().numpy()
        count = R.holders(table, POOL)
        for q in range(B):
            assert all(count[table[q, c]] == 1 for c in range((len(rows[q]) - len(paths[q])) // PAGE, -(-len(rows[q]) // PAGE)))


def rounds(loops, kind, run, between=lambda i: None):
    """Four rounds of new trees, forks and compactions, run(loop, what) each."""
    rng = np.random.default_rng(9)
    for i in range(4):
        state = rng.bit_generator.state
        for loop in loops:
            rng.bit_generator.state = state
            loop.put(rng)
        if i == 2:
            for loop in loops:
                loop.source.copy_(i32([0, 0, 2, 2]))
                loop.keep.copy_(i32([20, 20, 9, 0]))
        torch.cuda.synchronize()
        for what in (("fork", "step") if i == 2 else ("step", "compact")):
            say(f"round {i} {what}, type {kind}")
            for loop in loops:
                run(loop, what)
        between(i)
        for other in loops[1:]:
            assert all(torch.equal(a, b) for a, b in zip(loops[0].state(), other.state())), i


def started(kind, n):
    loops = [Loop(kind, 2) for _ in range(n)]
    g = torch.Generator(device=device()).manual_seed(3)
    qkv = torch.randn(B, PROMPT, HQ + 2 * HKV, 128, generator=g, device=device()).bfloat16()
    for loop in loops:
        loop.prompt(qkv.clone(), i32([PROMPT, 30, 20, 3]))
    torch.cuda.synchronize()
    return loops


@pytest.mark.parametrize("kind", KINDS)
def test_replayed_steps(kind):
    """Every call captured once and replayed, beside an eager loop."""
    eager, loop = started(kind, 2)
    graphs = {}
    for what in ("step", "fork", "compact"):
        graphs[what] = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graphs[what]):
            getattr(loop, what)()
    rounds([eager, loop], kind, lambda x, what: graphs[what].replay() if x is loop else getattr(x, what)())


def test_steps_on_other_streams():
    """The current stream, and the one given by argument."""
    loops = started(D.CACHE_E2M1, 3)
    side = torch.cuda.Stream()

    def run(loop, what):
        if loop is loops[0]:
            getattr(loop, what)()
        else:
            with torch.cuda.stream(side):
                getattr(loop, what)(*(() if loop is loops[1] else (side,)))
            side.synchronize()

    rounds(loops, D.CACHE_E2M1, run)


def test_a_stream_of_another_device_is_refused():
    class Elsewhere:
        device_index, cuda_stream = 1, 0

    loop = started(D.CACHE_E2M1, 1)[0]
    before = loop.state()
    for call in (loop.step, loop.compact, loop.fork):
        with pytest.raises(ValueError, match="stream"):
            call(Elsewhere())
    assert all(torch.equal(a, b) for a, b in zip(before, loop.state()))
