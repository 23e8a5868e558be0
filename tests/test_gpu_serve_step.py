"""Steps of a serving loop with the operators as they are used together: the last
token's layer over the paged cache, a drafted tree, its layer, its verification and
the accepted nodes' keys and values written back; eagerly, on another stream and as
replayed graphs that share workspaces.  The target is one attention layer with rows
of random tables as its queries, keys, values and logits."""
import numpy as np
import pytest
import torch

from paper_2608_13524_amd import dartree as D
from paper_2608_13524_amd import workloads as W
from tests import serve_ref as S
from tests.gpu_util import device, say
from tests.test_gpu_cache import BF, E8, tables

pytestmark = pytest.mark.gpu
B, V, HQ, HKV, PAGE, PER, BUDGET, DEPTH = 3, 1024, 8, 2, 16, 8, 20, 5
CFG = W.Config(name="serve", batch=B, vocab=V, hidden=256, depth=DEPTH, width=6, branch=4, budget=BUDGET, temperature=0.0,
               precision=W.BF16, seed=51, sigma_w=0.06, n_boost=8)
SCALE = 128.0 ** -0.5


class Shared:
    """Weights, the drafter's inputs and workspaces: one set for any number of loops."""

    def __init__(self, kind):
        dev = device()
        g = torch.Generator(device=dev).manual_seed(5)
        normal = lambda *s: torch.randn(*s, generator=g, device=dev)
        self.q, self.k, self.v = (normal(V, h, 128).bfloat16() for h in (HQ, HKV, HKV))
        self.z = normal(V, V)
        self.dp = D.Params.of(CFG)
        self.inputs = D.DeviceInputs.from_host(W.make_inputs(CFG), dev)
        self.build_ws = D.alloc_workspace(self.dp, dev)
        self.p = D.CacheParams(B, HKV, 128, PAGE, B * PER + 2, PER, kind)
        self.one = D.AttnParams(B, 1, PER * PAGE, HQ, HKV, 128, SCALE)
        self.tree = D.AttnParams(B, BUDGET, PER * PAGE, HQ, HKV, 128, SCALE)
        need = max(D.tree_attention_paged_workspace_size(a, self.p) for a in (self.one, self.tree))
        self.attn_ws = torch.empty(max(need, 256), dtype=torch.uint8, device=dev)
        self.verify_ws = torch.empty(D.verify_tree_workspace_size(B, BUDGET, DEPTH, V), dtype=torch.uint8, device=dev)


class Loop:
    """What a serving loop of three requests keeps; the last request has no pages."""

    def __init__(self, shared, seed):
        dev, rng = device(), np.random.default_rng(seed)
        s = self.s = shared
        table = tables(rng, B, PER, s.p.num_pages)
        table[2] = -1
        self.cache = D.DeviceCache.alloc(s.p, dev)
        for t in (self.cache.k, self.cache.v, self.cache.k_exp, self.cache.v_exp):
            if t is not None:
                t.view(torch.uint8).fill_(0xFF)
        self.cache.table.copy_(torch.from_numpy(table))
        i32 = lambda x: torch.tensor(x, dtype=torch.int32, device=dev)
        self.length, self.last = i32([37, 0, 0]), i32(rng.integers(0, V, B))
        prompt = torch.from_numpy(rng.integers(0, V, (B, 40))).to(dev)
        D.cache_write(s.p, self.cache, s.k[prompt], s.v[prompt], 40, counts=self.length)
        self.u = torch.zeros(B, BUDGET + 1, device=dev)
        self.draft = D.DeviceTree.alloc(B, BUDGET, dev)
        self.accepted, self.count = i32([[-9] * DEPTH] * B), i32([-9] * B)
        self.out1, self.out = (torch.empty(B, n, HQ, 128, dtype=torch.bfloat16, device=dev) for n in (1, BUDGET))
        self.logits = torch.empty(B, BUDGET + 1, V, device=dev)

    def step(self, stream=None):
        s, c, t = self.s, self.cache, self.draft
        at = self.last.long().clamp(min=0)[:, None]
        k, v = s.k[at], s.v[at]
        D.tree_attention_paged(s.one, s.p, c, s.q[at], k, v, None, self.length, self.out1, s.attn_ws, stream=stream)
        D.cache_write(s.p, c, k, v, 1, start=self.length, stream=stream)
        self.length += 1
        D.build_tree(s.dp, s.inputs, s.build_ws, t, stream=stream)
        nodes = t.tokens.long().clamp(0, V - 1)
        k, v = s.k[nodes], s.v[nodes]
        D.tree_attention_paged(s.tree, s.p, c, s.q[nodes], k, v, t.mask, self.length, self.out, s.attn_ws,
                               num_nodes=t.num_nodes, stream=stream)
        self.logits[:, :1] = s.z[at] + self.out1.float().view(B, 1, V)
        self.logits[:, 1:] = s.z[nodes] + self.out.float().view(B, BUDGET, V)
        # drafted tokens are likely ones: + 5 at every node's token in its parent's row
        there = torch.arange(BUDGET, device=nodes.device)[None] < t.num_nodes[:, None]
        self.logits.view(B, -1).scatter_add_(1, (t.parents.long().clamp(-1, BUDGET - 1) + 1) * V + nodes, 5.0 * there)
        D.verify_tree(t.tokens, t.parents, t.num_nodes, self.logits, 0.8, self.u, self.accepted, self.count, self.last,
                      s.verify_ws, stream=stream)
        D.cache_write(s.p, c, k, v, DEPTH, index=self.accepted, counts=self.count, start=self.length, stream=stream)
        self.length += self.count

    def state(self):
        torch.cuda.synchronize()
        t = [self.cache.k, self.cache.v, self.cache.k_exp, self.cache.v_exp, self.length, self.last, self.accepted, self.count,
             self.out1, self.out, self.logits]
        return [x.clone().view(torch.uint8) for x in t if x is not None]

    def same_as(self, other):
        return all(torch.equal(a, b) for a, b in zip(self.state(), other.state()))


def uniforms(rng):
    return torch.from_numpy(rng.random((B, BUDGET + 1)).astype(np.float32)).to(device())


@pytest.mark.parametrize("kind", [E8, BF])
def test_steps_follow_the_definitions(kind):
    """Every step's layers and verification against the plain forms, over what the cache holds."""
    loop, rng = Loop(Shared(kind), 1), np.random.default_rng(2)
    s, total = loop.s, 0
    for i in range(5):
        loop.u.copy_(uniforms(rng))
        length = loop.length.cpu().numpy()
        say(f"serving step {i}, type {kind}, lengths {length}")
        loop.step()
        k, v = (torch.zeros(B, PER * PAGE, HKV, 128, dtype=torch.bfloat16, device=device()) for _ in range(2))
        D.cache_read(s.p, loop.cache, k, v)
        torch.cuda.synchronize()
        keys, values = (x.double().cpu().numpy() for x in (k, v))
        t, z = loop.draft.host(), loop.logits.cpu().numpy()
        count, accepted, last = loop.count.cpu().numpy(), loop.accepted.cpu().numpy(), loop.last.cpu().numpy()
        out = loop.out.double().cpu().numpy()
        for q in range(B):
            path, token = S.verify_tree(t["tokens"][q], t["parents"][q], t["num_nodes"][q], z[q], 0.8, loop.u[q].cpu().numpy(), DEPTH)
            assert accepted[q, :count[q]].tolist() == path and last[q] == token
            assert loop.length[q] == length[q] + 1 + len(path)
            ctx, n = length[q] + 1 if q < 2 else 0, int(t["num_nodes"][q])
            see = np.zeros((BUDGET, ctx + BUDGET), bool)
            see[:, :ctx] = True
            for j in range(n):
                see[:, ctx + j] = (t["mask"][q, :, 0] >> np.uint64(j)) & np.uint64(1)
            nodes = np.clip(t["tokens"][q], 0, V - 1)
            for h in range(HQ):
                kt, vt = (x[nodes, h // 4].double().cpu().numpy() for x in (s.k, s.v))
                query = s.q[nodes, h].double().cpu().numpy()
                kk = np.concatenate([keys[q, :ctx, h // 4], kt])
                vv = np.concatenate([values[q, :ctx, h // 4], vt])
                want = S.attention(query, kk, vv, see, SCALE)
                tol = (2.0 ** -8 + 2.0 ** -9) * np.abs(vv).max() + 2.0 ** -8 * np.abs(want)   # as in test_gpu_paged.py
                assert (np.abs(out[q, :, h] - want) <= tol).all()
            # the accepted nodes' keys and values stand behind the last token's
            for i_, node in enumerate(path):
                if q == 2:
                    break
                for held, table in ((keys, s.k), (values, s.v)):
                    row = table[nodes[node]].float().cpu().numpy()
                    if kind == E8:
                        r, e = S.quantise(row)
                        row = r * 2.0 ** e[..., None]
                    assert np.array_equal(held[q, ctx + i_], row)
        total += int(count.sum())
    assert total > 0


@pytest.mark.parametrize("kind", [E8, BF])
def test_replayed_steps_that_share_workspaces(kind):
    """Two loops captured with the same workspaces and replayed in turn, eager steps of two others between."""
    shared, rng = Shared(kind), np.random.default_rng(3)
    graphs, loops, eager = [], [Loop(shared, 1), Loop(shared, 2)], [Loop(shared, 1), Loop(shared, 2)]
    Loop(shared, 9).step()
    torch.cuda.synchronize()
    for loop in loops:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            loop.step()
        graphs.append(g)
    for i in range(4):
        for g, loop, plain in zip(graphs, loops, eager):
            u = uniforms(rng)
            loop.u.copy_(u)
            plain.u.copy_(u)
            say(f"replay {i}, type {kind}")
            g.replay()
            plain.step()
        for loop, plain in zip(loops, eager):
            assert loop.same_as(plain), i


def test_steps_on_another_stream():
    """The stream given by argument, and the current one; both equal the default stream's results."""
    rng = np.random.default_rng(4)
    loops = [Loop(Shared(E8), 6) for _ in range(3)]
    side = torch.cuda.Stream()
    for i in range(3):
        u = uniforms(rng)
        for loop in loops:
            loop.u.copy_(u)
        say(f"streams, step {i}")
        torch.cuda.synchronize()
        loops[0].step()
        with torch.cuda.stream(side):
            loops[1].step()
            loops[2].step(stream=side)
        assert loops[1].same_as(loops[0]) and loops[2].same_as(loops[0])


def test_two_loops_at_once():
    """Steps of two loops in flight on two streams, each with workspaces of its own."""
    rng = np.random.default_rng(8)
    pair, alone = [Loop(Shared(k), 10 + k) for k in (E8, BF)], [Loop(Shared(k), 10 + k) for k in (E8, BF)]
    streams = [torch.cuda.Stream() for _ in pair]
    us = [[uniforms(rng) for _ in pair] for _ in range(4)]
    say("two loops at once")
    torch.cuda.synchronize()
    for u in us:
        for loop, stream, x in zip(pair, streams, u):
            with torch.cuda.stream(stream):
                loop.u.copy_(x)
                loop.step()
    torch.cuda.synchronize()
    for u in us:
        for loop, x in zip(alone, u):
            loop.u.copy_(x)
            loop.step()
    assert pair[0].same_as(alone[0]) and pair[1].same_as(alone[1])


def test_a_stream_of_another_device_is_refused():
    class Elsewhere:
        device_index, cuda_stream = 1, 0

    s = Shared(E8)
    loop = Loop(s, 7)
    before = loop.state()
    with pytest.raises(ValueError, match="stream"):
        D.cache_read(s.p, loop.cache, loop.cache.k, loop.cache.v, stream=Elsewhere())
    with pytest.raises(ValueError, match="stream"):
        D.verify_tree(loop.draft.tokens, loop.draft.parents, loop.draft.num_nodes, loop.logits, 1.0, loop.u, loop.accepted,
                      loop.count, loop.last, s.verify_ws, stream=Elsewhere())
    assert all(torch.equal(a, b) for a, b in zip(before[:6], loop.state()[:6]))
