"""Performance cases of the serving operators: what a verification step of
speculative decoding does around the draft tree, over the range of sizes that
the library serves.

Kinds of case:

* ``write``: keys and values of prompts, tokens or accepted tree nodes into a
  paged cache (``cache_write``), held in bf16 or in 8 bits (e4m3) with a power
  of two per position and head;
* ``read``: positions of that cache back as dense bf16 (``cache_read``);
* ``attn``: one attention layer of a tree of drafted tokens, a chain or a
  single token over that cache (``tree_attention_paged``);
* ``tree``: the drafted tree verified against the target's probabilities from
  given random numbers (``verify_tree``);
* ``chain``: a drafted chain verified against the target's and the drafter's
  probabilities (``verify_chain``).

``own`` false: the plain form, elementary torch operations; true: the library.

Layout of a cache: pages [num_pages][heads_kv][page][128]; position t of a
request lies in slot t % page of page table[request][t // page]; in 8 bits the
row stands for value * 2^(exp - 127) with exp [num_pages][heads_kv][page].
"""
from __future__ import annotations

import math

import torch

own = False

HEAD = 128            # elements of a head
AGREE = 0.85          # how often the target follows the draft's best child
FAVOURED = 1.75       # log odds of that
E4M3_MAX = 448.0
EXP_LOW, EXP_HIGH = -100, 120
BF16, E4M3 = "bf16", "e4m3"


def listed():
    return [
        # a decoding step's accepted nodes (up to 16 of 64 drafted) into the caches of 16 requests: the smallest call
        _write("write-accepted", batch=16, source=64, rows=16, heads_kv=8, page=64, held=E4M3, indexed=True),
        # the prompts of 8 requests, keys and values in the rows of a fused projection
        _write("write-prompt", batch=8, source=2048, rows=2048, heads_kv=8, page=64, held=E4M3, ragged=True, fused=True),
        # 16 prefixes back as the dense context that `tree_attention` reads
        _read("read-prefix", batch=16, rows=2048, heads_kv=8, page=64, held=E4M3),
        # a few ragged prefixes of a bf16 cache with small pages
        _read("read-odd", batch=3, rows=777, heads_kv=4, page=16, held=BF16, ragged=True),
        # one request's drafted tree of 64 nodes over 2048 positions: latency counts
        _attn("attn-4b", batch=1, nodes=64, ctx=2048, heads_q=32, heads_kv=8, page=64, held=E4M3),
        # single tokens of 64 requests over ragged caches of up to 8192 positions
        _attn("attn-token", batch=64, nodes=1, ctx=8192, heads_q=32, heads_kv=8, page=64, held=E4M3, ragged=True),
        # small trees over two long bf16 caches
        _attn("attn-long", batch=2, nodes=16, ctx=65536, heads_q=32, heads_kv=8, page=256, held=BF16),
        # sixteen requests' trees of 512 nodes: the most products
        _attn("attn-x16", batch=16, nodes=512, ctx=2048, heads_q=32, heads_kv=8, page=64, held=E4M3),
        # the tree of the benchmark's default workload
        _tree("tree-4b", batch=1, nodes=64, depth=16, vocab=151936, temperature=1.0),
        # sixteen requests' trees of 512 nodes: 8208 rows of target logits
        _tree("tree-x16", batch=16, nodes=512, depth=16, vocab=151936, temperature=1.0),
        # eight chains of 16 drafted tokens
        _chain("chain-x8", batch=8, depth=16, vocab=151936, temperature=1.0),
        # an odd vocabulary, bf16 logits, a sharper distribution
        _chain("chain-odd", batch=3, depth=7, vocab=50257, temperature=0.7, held=BF16),
    ]


def draw(rng):
    kind = rng.choice(["write", "read", "attn", "attn", "attn", "tree", "chain"])
    held = rng.choice([BF16, E4M3, E4M3])
    page = rng.choice([16, 32, 64, 128, 256])
    hkv = rng.choice([1, 2, 4, 8])
    while kind == "write":
        b, rows = _log(rng, 1, 64), _log(rng, 1, 4096)
        if b * rows * hkv <= 8 * 2048 * 8:
            indexed = rows <= 64 and rng.random() < 0.5
            return _write(None, batch=b, source=rows + _log(rng, 1, 64) if indexed else rows, rows=rows, heads_kv=hkv,
                          page=page, held=held, indexed=indexed, ragged=rng.random() < 0.5, fused=rng.random() < 0.5)
    while kind == "read":
        b, rows = _log(rng, 1, 64), _log(rng, 16, 8192)
        if b * rows * hkv <= 16 * 2048 * 8:
            return _read(None, batch=b, rows=rows, heads_kv=hkv, page=page, held=held, ragged=rng.random() < 0.5)
    while kind == "attn":
        b, nodes, ctx = _log(rng, 1, 64), _log(rng, 1, 512), _log(rng, 64, 65536)
        group = rng.choice([1, 2, 4, 8])
        if b * ctx <= 64 * 8192 and b * nodes * hkv * group * (ctx + nodes) <= 16 * 512 * 32 * 2560:
            return _attn(None, batch=b, nodes=nodes, ctx=ctx, heads_q=hkv * group, heads_kv=hkv, page=page, held=held,
                         ragged=rng.random() < 0.5)
    temperature = rng.choice([0.0, 0.7, 1.0])
    vocab = _log(rng, 16000, 151936)
    while kind == "tree":
        b, nodes = _log(rng, 1, 32), _log(rng, 8, 512)
        if b * nodes <= 16 * 512:
            return _tree(None, batch=b, nodes=nodes, depth=rng.randint(2, 16), vocab=vocab, temperature=temperature,
                         held=rng.choice([BF16, "fp32"]))
    return _chain(None, batch=_log(rng, 1, 32), depth=rng.randint(1, 16), vocab=vocab, temperature=temperature,
                  held=rng.choice([BF16, "fp32"]))


def _log(rng, lo, hi):
    """A whole number of lo .. hi, uniform over its logarithm."""
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _case(name, **kw):
    return {"name": name, **kw} if name else kw


def _write(name, *, batch, source, rows, heads_kv, page, held, indexed=False, ragged=False, fused=False):
    return _case(name, kind="write", batch=batch, source=source, rows=rows, heads_kv=heads_kv, page=page, held=held,
                 indexed=indexed, ragged=ragged, fused=fused)


def _read(name, *, batch, rows, heads_kv, page, held, ragged=False):
    return _case(name, kind="read", batch=batch, rows=rows, heads_kv=heads_kv, page=page, held=held, ragged=ragged)


def _attn(name, *, batch, nodes, ctx, heads_q, heads_kv, page, held, ragged=False):
    return _case(name, kind="attn", batch=batch, nodes=nodes, ctx=ctx, heads_q=heads_q, heads_kv=heads_kv, page=page,
                 held=held, ragged=ragged)


def _tree(name, *, batch, nodes, depth, vocab, temperature, held="fp32"):
    return _case(name, kind="tree", batch=batch, nodes=nodes, depth=min(depth, nodes), vocab=vocab,
                 temperature=temperature, held=held)


def _chain(name, *, batch, depth, vocab, temperature, held="fp32"):
    return _case(name, kind="chain", batch=batch, depth=depth, vocab=vocab, temperature=temperature, held=held)


# ---------------------------------------------------------------------------
# Inputs
# ---------------------------------------------------------------------------

def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(0x0DE70000 + int(seed))


def _normal(g, shape, sigma=1.0, dtype=torch.bfloat16):
    return torch.randn(shape, generator=g, device="cuda").mul_(sigma).to(dtype)


def _whole(g, lo, hi, shape):
    return torch.randint(lo, hi + 1, shape, generator=g, device="cuda", dtype=torch.int32)


def prepare(case, seed):
    s = {"case": case, **_PREPARE[case["kind"]](case, _gen(seed))}
    if own:   # scalar arguments and the workspace, which a program keeps
        s["handle"] = _handle(case, s)
    return s


def _pool(c, g, positions, filled):
    """An empty or a filled cache of `positions` per request, its pages in no order."""
    b, hkv, page, eight = c["batch"], c["heads_kv"], c["page"], c["held"] == E4M3
    per = -(-positions // page)
    n = b * per + 2
    table = torch.randperm(n, generator=g, device="cuda")[: b * per].view(b, per).to(torch.int32)
    out = {"table": table, "num_pages": n}
    for name in ("k", "v"):
        dtype = torch.float8_e4m3fn if eight else torch.bfloat16
        out[name + "_exp"] = torch.full((n, hkv, page), 127, dtype=torch.uint8, device="cuda") if eight else None
        if not filled:
            out[name] = torch.zeros(n, hkv, page, HEAD, dtype=torch.uint8 if eight else dtype, device="cuda").view(dtype)
            continue
        x = torch.randn((n, hkv, page, HEAD), generator=g, device="cuda")
        if eight:
            x, out[name + "_exp"] = _quantised(x.to(torch.bfloat16))
        out[name] = x.to(dtype)
    return out


def _prepare_write(c, g):
    b, src, rows, hkv = c["batch"], c["source"], c["rows"], c["heads_kv"]
    if c["fused"]:   # q, k and v side by side in a row, four query heads a key/value head
        x = _normal(g, (b, src, 6 * hkv, HEAD))
        k, v = x[:, :, 4 * hkv:5 * hkv], x[:, :, 5 * hkv:]
    else:
        k, v = _normal(g, (b, src, hkv, HEAD)), _normal(g, (b, src, hkv, HEAD))
    start = _whole(g, 0, 2 * c["page"], (b,))
    counts = _whole(g, (rows + 1) // 2, rows, (b,)) if c["ragged"] or c["indexed"] else None
    index = None
    if c["indexed"]:
        index = torch.rand(b, src, generator=g, device="cuda").argsort(dim=1)[:, :rows].sort(dim=1).values.to(torch.int32).contiguous()
    return {"k_new": k, "v_new": v, "start": start, "counts": counts, "index": index,
            **_pool(c, g, 2 * c["page"] + rows, False)}


def _prepare_read(c, g):
    b, rows, hkv = c["batch"], c["rows"], c["heads_kv"]
    return {"start": _whole(g, 0, c["page"], (b,)), "counts": _whole(g, (rows + 1) // 2, rows, (b,)) if c["ragged"] else None,
            "k_out": torch.zeros(b, rows, hkv, HEAD, dtype=torch.bfloat16, device="cuda"),
            "v_out": torch.zeros(b, rows, hkv, HEAD, dtype=torch.bfloat16, device="cuda"),
            **_pool(c, g, c["page"] + rows, True)}


def _levels(nodes, depth):
    return [nodes * i // depth for i in range(depth + 1)]


def _parents(g, b, nodes, depth):
    """Trees in breadth-first order: the parents of a level in order, its first node a child of the first node above."""
    edges = _levels(nodes, depth)
    parents = torch.full((b, nodes), -1, dtype=torch.int64, device="cuda")
    for above, lo, hi in zip(edges[:-2], edges[1:-1], edges[2:]):
        p = torch.randint(above, lo, (b, hi - lo), generator=g, device="cuda")
        p[:, 0] = above
        parents[:, lo:hi] = p.sort(dim=1).values
    return parents


def _prepare_attn(c, g):
    b, n, ctx, hq, hkv = c["batch"], c["nodes"], c["ctx"], c["heads_q"], c["heads_kv"]
    parents = _parents(g, b, n, min(16, n))
    see = torch.zeros(b, n, n, dtype=torch.bool, device="cuda")
    edges = _levels(n, min(16, n))
    for lo, hi in zip(edges[:-1], edges[1:]):
        if lo:
            see[:, lo:hi] = see.gather(1, parents[:, lo:hi, None].expand(b, hi - lo, n))
        see[:, range(lo, hi), range(lo, hi)] = True
    words = (n + 63) // 64
    bits = torch.nn.functional.pad(see, (0, 64 * words - n)).view(b, n, words, 64).to(torch.int64)
    return {"see": see, "mask": (bits << torch.arange(64, device="cuda")).sum(-1),
            "q": _normal(g, (b, n, hq, HEAD)), "k_tree": _normal(g, (b, n, hkv, HEAD)),
            "v_tree": _normal(g, (b, n, hkv, HEAD)),
            "ctx_len": _whole(g, (ctx + 1) // 2, ctx, (b,)) if c["ragged"] else torch.full((b,), ctx, dtype=torch.int32, device="cuda"),
            "out": torch.empty(b, n, hq, HEAD, dtype=torch.bfloat16, device="cuda"), **_pool(c, g, ctx, True)}


def _logit_type(c):
    return torch.bfloat16 if c["held"] == BF16 else torch.float32


def _prepare_tree(c, g):
    """Target logits N(0, 2^2) with a boost on every drafted child, the first child of the first node of a level
    the likeliest, so that the target follows the first path most of the time."""
    b, n, vocab = c["batch"], c["nodes"], c["vocab"]
    parents = _parents(g, b, n, c["depth"])
    tokens = torch.rand(b, vocab, generator=g, device="cuda").argsort(dim=1)[:, :n]
    key = (parents * vocab + tokens).argsort(dim=1)   # siblings by token
    tokens, parents = tokens.gather(1, key), parents.gather(1, key)
    z = torch.empty(b, n + 1, vocab, dtype=_logit_type(c), device="cuda")
    for i in range(b):
        z[i] = torch.randn((n + 1, vocab), generator=g, device="cuda").mul_(2.0)
    t = c["temperature"] or 1.0
    likely = t * (math.log(vocab) + 2.0 / (t * t))     # the logit of as much mass as all of a row's others together
    z = z.view(b, -1)
    at = (parents + 1) * vocab + tokens
    boost = likely + t * (torch.randn(b, n, generator=g, device="cuda") - 3.0)
    edges = _levels(n, c["depth"])
    boost[:, edges[:-1]] = likely + t * FAVOURED
    z.scatter_(1, at, boost.to(z.dtype))
    return {"tokens": tokens.to(torch.int32), "parents": parents.to(torch.int32),
            "num_nodes": torch.full((b,), n, dtype=torch.int32, device="cuda"), "logits": z.view(b, n + 1, vocab),
            "uniforms": torch.rand(b, n + 1, generator=g, device="cuda"),
            "accepted": torch.empty(b, c["depth"], dtype=torch.int32, device="cuda"),
            "num_accepted": torch.empty(b, dtype=torch.int32, device="cuda"),
            "bonus": torch.empty(b, dtype=torch.int32, device="cuda")}


def _prepare_chain(c, g):
    """Draft logits N(0, 2^2) with a boost on a few tokens; the target's are near them; tokens drawn from the draft."""
    b, n, vocab, t = c["batch"], c["depth"], c["vocab"], c["temperature"] or 1.0
    q = torch.randn((b, n, vocab), generator=g, device="cuda").mul_(2.0)
    ids = torch.randint(0, vocab, (b, n, 8), generator=g, device="cuda")
    q.scatter_(2, ids, math.log(vocab) + 2.0 + 2.0 * torch.randn((b, n, 8), generator=g, device="cuda"))
    p = torch.randn((b, n + 1, vocab), generator=g, device="cuda").mul_(2.0)
    p[:, :n] = q + 0.5 * torch.randn((b, n, vocab), generator=g, device="cuda")
    p, q = p.to(_logit_type(c)), q.to(_logit_type(c))
    pr = torch.softmax(q.float() / t, dim=2).view(b * n, vocab)
    tokens = torch.multinomial(pr, 1, generator=g).view(b, n) if c["temperature"] else q.float().argmax(dim=2)
    return {"tokens": tokens.to(torch.int32), "target": p, "draft": q,
            "uniforms": torch.rand(b, n + 1, generator=g, device="cuda"),
            "num_accepted": torch.empty(b, dtype=torch.int32, device="cuda"),
            "bonus": torch.empty(b, dtype=torch.int32, device="cuda")}


_PREPARE = {"write": _prepare_write, "read": _prepare_read, "attn": _prepare_attn, "tree": _prepare_tree,
            "chain": _prepare_chain}


# ---------------------------------------------------------------------------
# One pass
# ---------------------------------------------------------------------------

def run(s):
    kind = s["case"]["kind"]
    return (_RUN_OWN if own else _RUN_PLAIN)[kind](s)


def _handle(c, s):
    from paper_2608_13524_amd import dartree as D
    kind = c["kind"]
    if kind in ("tree", "chain"):
        nbytes = (D.verify_tree_workspace_size(c["batch"], c["nodes"], c["depth"], c["vocab"]) if kind == "tree"
                  else D.verify_chain_workspace_size(c["batch"], c["depth"], c["vocab"]))
        return {"ws": torch.empty(nbytes, dtype=torch.uint8, device="cuda")}
    p = D.CacheParams(c["batch"], c["heads_kv"], HEAD, c["page"], s["num_pages"], s["table"].shape[1],
                      D.CACHE_E4M3 if c["held"] == E4M3 else D.CACHE_BF16)
    h = {"p": p, "cache": D.DeviceCache(s["k"], s["v"], s["k_exp"], s["v_exp"], s["table"])}
    if kind == "attn":
        h["a"] = D.AttnParams(c["batch"], c["nodes"], c["ctx"], c["heads_q"], c["heads_kv"], HEAD, 1.0 / math.sqrt(HEAD))
        nbytes = D.tree_attention_paged_workspace_size(h["a"], p)
        h["ws"] = torch.empty(nbytes, dtype=torch.uint8, device="cuda") if nbytes else None
    return h


def _own_write(s):
    from paper_2608_13524_amd import dartree as D
    h = s["handle"]
    D.cache_write(h["p"], h["cache"], s["k_new"], s["v_new"], s["case"]["rows"], index=s["index"], counts=s["counts"],
                  start=s["start"])
    return {"k": s["k"], "v": s["v"], "k_exp": s["k_exp"], "v_exp": s["v_exp"]}


def _own_read(s):
    from paper_2608_13524_amd import dartree as D
    h = s["handle"]
    D.cache_read(h["p"], h["cache"], s["k_out"], s["v_out"], counts=s["counts"], start=s["start"])
    return {"k": s["k_out"], "v": s["v_out"]}


def _own_attn(s):
    from paper_2608_13524_amd import dartree as D
    h = s["handle"]
    D.tree_attention_paged(h["a"], h["p"], h["cache"], s["q"], s["k_tree"], s["v_tree"], s["mask"], s["ctx_len"],
                           s["out"], h["ws"])
    return s["out"]


def _own_tree(s):
    from paper_2608_13524_amd import dartree as D
    D.verify_tree(s["tokens"], s["parents"], s["num_nodes"], s["logits"], s["case"]["temperature"], s["uniforms"],
                  s["accepted"], s["num_accepted"], s["bonus"], s["handle"]["ws"])
    return {"accepted": s["accepted"], "num_accepted": s["num_accepted"], "bonus": s["bonus"]}


def _own_chain(s):
    from paper_2608_13524_amd import dartree as D
    D.verify_chain(s["tokens"], s["target"], s["draft"], s["case"]["temperature"], s["uniforms"], s["num_accepted"],
                   s["bonus"], s["handle"]["ws"])
    return {"num_accepted": s["num_accepted"], "bonus": s["bonus"]}


_RUN_OWN = {"write": _own_write, "read": _own_read, "attn": _own_attn, "tree": _own_tree, "chain": _own_chain}


# ---------------------------------------------------------------------------
# The plain forms
# ---------------------------------------------------------------------------

def _quantised(x):
    """(e4m3 values, exponents + 127) of rows of 128: the least power of two that brings the row's largest to 448."""
    x = x.float()
    m, e = torch.frexp(x.abs().amax(dim=-1))     # m in [0.5, 1): 448 is 0.875 * 2^9
    e = torch.where(m > 0.875, e - 8, e - 9).clamp(EXP_LOW, EXP_HIGH)
    e = torch.where(m == 0, EXP_LOW, e)
    return torch.ldexp(x, -e[..., None]).to(torch.float8_e4m3fn), (e + 127).to(torch.uint8)


def _values(s, name):
    """A cache's pages as the values they stand for, in 32 bits."""
    x = s[name].float()
    if s[name + "_exp"] is None:
        return x
    return torch.ldexp(x, (s[name + "_exp"].int() - 127)[..., None])


def _slots(s, rows):
    """(page, slot, there) of positions start .. start + rows of every request."""
    c = s["case"]
    at = s["start"][:, None].long() + torch.arange(rows, device="cuda")
    there = torch.arange(rows, device="cuda") < (s["counts"] if s["counts"] is not None else torch.full_like(s["start"], rows))[:, None]
    pages = s["table"].long().gather(1, (at // c["page"]).clamp(max=s["table"].shape[1] - 1))
    return pages, at % c["page"], there


def _plain_write(s):
    c = s["case"]
    pages, slot, there = _slots(s, c["rows"])
    pages, slot = pages[there], slot[there]
    for name in ("k", "v"):
        x = s[name + "_new"]
        if s["index"] is not None:
            x = x.gather(1, s["index"].long()[:, :, None, None].expand(-1, -1, c["heads_kv"], HEAD))
        x = x[there]
        if c["held"] == E4M3:
            x, s[name + "_exp"][pages, :, slot] = _quantised(x)
            s[name].view(torch.uint8)[pages, :, slot] = x.view(torch.uint8)
        else:
            s[name][pages, :, slot] = x
    return {"k": s["k"], "v": s["v"], "k_exp": s["k_exp"], "v_exp": s["v_exp"]}


def _plain_read(s):
    pages, slot, there = _slots(s, s["case"]["rows"])
    for name in ("k", "v"):
        s[name + "_out"][there] = _values(s, name)[pages[there], :, slot[there]].to(torch.bfloat16)
    return {"k": s["k_out"], "v": s["v_out"]}


def _plain_attn(s):
    c = s["case"]
    b, n, ctx, hq, hkv = c["batch"], c["nodes"], c["ctx"], c["heads_q"], c["heads_kv"]
    group = hq // hkv

    def keys(name):   # [b][heads_kv][ctx + nodes][128]
        x = _values(s, name)[s["table"].long()].transpose(1, 2).reshape(b, hkv, -1, HEAD)[:, :, :ctx]
        return torch.cat([x, s[name + "_tree"].float().transpose(1, 2)], dim=2)

    q = s["q"].float().view(b, n, hkv, group, HEAD).permute(0, 2, 1, 3, 4).reshape(b, hkv, n * group, HEAD)
    x = torch.matmul(q, keys("k").transpose(2, 3).contiguous()) / math.sqrt(HEAD)
    seen = torch.arange(ctx, device="cuda") < s["ctx_len"][:, None]
    vis = torch.cat([seen[:, None].expand(b, n, ctx), s["see"]], dim=2).repeat_interleave(group, dim=1)
    x = x.masked_fill_(~vis[:, None], -math.inf)
    x = torch.exp(x - x.amax(dim=3, keepdim=True))
    out = torch.matmul(x / x.sum(dim=3, keepdim=True), keys("v"))
    return out.view(b, hkv, n, group, HEAD).permute(0, 2, 1, 3, 4).reshape(b, n, hq, HEAD).to(torch.bfloat16)


def _weights(z, temperature):
    """Softmax of rows of logits in 64 bits; at temperature 0 all of the mass on the first largest."""
    if temperature == 0:
        return torch.zeros(z.shape, dtype=torch.float64, device="cuda").scatter_(-1, z.float().argmax(dim=-1, keepdim=True), 1.0)
    t = float(torch.tensor(temperature, dtype=torch.float32))
    x = torch.exp((z.double() - z.amax(dim=-1, keepdim=True).double()) / t)
    return x / x.sum(dim=-1, keepdim=True)


def _sampled(w, rest, u):
    """The first token whose cumulated mass of `rest` (of `w` where nothing is left) exceeds u of its whole."""
    w = torch.where(rest.sum(dim=1, keepdim=True) > 0, rest, w)
    cum = w.cumsum(dim=1)
    at = (cum <= u.double()[:, None] * cum[:, -1:]).sum(dim=1)
    last = (w > 0).long().mul_(torch.arange(w.shape[1], device="cuda")).amax(dim=1)
    return torch.minimum(at, last).to(torch.int32)


def _plain_tree(s):
    c = s["case"]
    b, n, z = c["batch"], c["nodes"], s["logits"]
    parents, tokens = s["parents"].long(), s["tokens"].long()
    if c["temperature"] == 0:
        best = z.float().argmax(dim=2)
        p = (best.gather(1, parents + 1) == tokens).double()
    else:
        t = float(torch.tensor(c["temperature"], dtype=torch.float32))
        top = z.amax(dim=2).double()
        total = torch.exp((z.double() - top[:, :, None]) / t).sum(dim=2)
        own_z = z.view(b, -1).gather(1, (parents + 1) * c["vocab"] + tokens).double()
        p = torch.exp((own_z - top.gather(1, parents + 1)) / t) / total.gather(1, parents + 1)
    # what the siblings before a node hold, and the first sibling whose test passes
    before = (parents[:, :, None] == parents[:, None, :]) & torch.ones(n, n, dtype=torch.bool, device="cuda").tril(-1)
    rest = 1.0 - torch.where(before, p[:, None, :], 0.0).sum(dim=2)
    passed = s["uniforms"][:, 1:].double() * rest < p
    first = passed & ~(before & passed[:, None, :]).any(dim=2)
    at = torch.full((b,), -1, dtype=torch.int64, device="cuda")
    accepted = torch.full((b, c["depth"]), -1, dtype=torch.int32, device="cuda")
    for step in range(c["depth"]):   # the path, one node at a time (-9: it has ended)
        child = first & (parents == at[:, None])
        at = torch.where(child.any(dim=1), child.long().argmax(dim=1), -9)
        accepted[:, step] = at.clamp(min=-1).to(torch.int32)
    count = (accepted >= 0).sum(dim=1)
    last = accepted.gather(1, (count - 1).clamp(min=0)[:, None])[:, 0].long()
    last = torch.where(count > 0, last, -1)
    w = _weights(z[torch.arange(b, device="cuda"), last + 1], c["temperature"])
    tested = (parents == last[:, None]) & (count < c["depth"])[:, None]
    gone = torch.zeros_like(w).scatter_add_(1, tokens, tested.double()) > 0
    return {"accepted": accepted, "num_accepted": count.to(torch.int32),
            "bonus": _sampled(w, torch.where(gone, 0.0, w), s["uniforms"][:, 0])}


def _plain_chain(s):
    c = s["case"]
    b, n = c["batch"], c["depth"]
    p = _weights(s["target"], c["temperature"])
    q = torch.nn.functional.pad(_weights(s["draft"], c["temperature"]), (0, 0, 0, 1))   # a row of zeros after the last token
    tokens = s["tokens"].long()[:, :, None]
    px, qx = p[:, :n].gather(2, tokens)[:, :, 0], q[:, :n].gather(2, tokens)[:, :, 0]
    passed = px > 0 if c["temperature"] == 0 else s["uniforms"][:, 1:].double() * qx < px
    count = passed.long().cumprod(dim=1).sum(dim=1)
    rows = torch.arange(b, device="cuda")
    w = p[rows, count]
    rest = w if c["temperature"] == 0 else (w - q[rows, count]).clamp(min=0)
    return {"num_accepted": count.to(torch.int32), "bonus": _sampled(w, rest, s["uniforms"][:, 0])}


_RUN_PLAIN = {"write": _plain_write, "read": _plain_read, "attn": _plain_attn, "tree": _plain_tree, "chain": _plain_chain}


# ---------------------------------------------------------------------------
# What a pass cannot do without
# ---------------------------------------------------------------------------

def work(case):
    c = case
    kind = c["kind"]
    if kind in ("write", "read", "attn"):
        row = 2 * c["heads_kv"] * (HEAD + 1 if c["held"] == E4M3 else 2 * HEAD)   # a position's keys and values in the cache
        dense = 4 * c["heads_kv"] * HEAD                                          # and as bf16
    if kind in ("write", "read"):
        positions = c["batch"] * c["rows"] * (0.75 if c["ragged"] or c.get("indexed") else 1.0)
        return {"bytes": positions * (row + dense), "flops": 0}
    if kind == "attn":
        seen = c["ctx"] * (0.75 if c["ragged"] else 1.0)
        nodes = c["batch"] * c["nodes"]
        return {"bytes": c["batch"] * seen * row + nodes * (dense + 4 * c["heads_q"] * HEAD + 8 * ((c["nodes"] + 63) // 64)),
                "flops": 4.0 * nodes * c["heads_q"] * HEAD * (seen + c["nodes"])}
    # the rows of the accepted positions and of the one after them; a chain's draft rows too
    size = 2 if c["held"] == BF16 else 4
    agree = AGREE if c["temperature"] else 1.0
    rows = 1 + sum(agree ** i for i in range(1, c["depth"] + 1))
    return {"bytes": c["batch"] * rows * c["vocab"] * size * (2 if kind == "chain" else 1), "flops": 0}


# ---------------------------------------------------------------------------
# The same outputs in 64 bits
# ---------------------------------------------------------------------------

def _decoded(byte):
    """e4m3 from its bits: sign, 4 exponent bits (bias 7), 3 of mantissa; no infinities."""
    b = byte.to(torch.int64)
    exp, man = (b >> 3) & 15, (b & 7).double()
    v = torch.where(exp == 0, man * 2.0 ** -9, (1.0 + man / 8.0) * torch.pow(2.0, (exp - 7).double()))
    return torch.where(b >= 128, -v, v)


def _exact_pages(s, name):
    if s[name + "_exp"] is None:
        return s[name].double()
    return _decoded(s[name].view(torch.uint8)) * torch.pow(2.0, s[name + "_exp"].double() - 127.0)[..., None]


def exact(case, seed):
    return _EXACT[case["kind"]](case, prepare(case, seed)) if case["kind"] in _EXACT else None


def _exact_write(c, s):
    out = {}
    for name in ("k", "v"):
        page_of = s["table"].cpu().tolist()
        x = s[name + "_new"].double()
        pool = torch.zeros(s[name].shape, dtype=torch.float64, device="cuda")
        for i in range(c["batch"]):
            n = int(s["counts"][i]) if s["counts"] is not None else c["rows"]
            rows = x[i, s["index"][i, :n].long()] if s["index"] is not None else x[i, :n]
            if c["held"] == E4M3:
                top = rows.abs().amax(dim=-1, keepdim=True)
                e = torch.ceil(torch.log2(top.clamp(min=2.0 ** -80) / E4M3_MAX))
                rows = rows * torch.pow(2.0, -e)
                grid = torch.pow(2.0, torch.floor(torch.log2(rows.abs().clamp(min=2.0 ** -6))) - 3.0)
                rows = torch.round(rows / grid) * grid
            first = int(s["start"][i])
            at = torch.arange(first, first + n)
            pages = torch.tensor(page_of[i], device="cuda")[at.cuda() // c["page"]]
            pool[pages, :, at.cuda() % c["page"]] = rows
        out[name] = pool
    return {"k": out["k"], "v": out["v"], "k_exp": None, "v_exp": None}


def _exact_read(c, s):
    out = {}
    for name in ("k", "v"):
        pages = _exact_pages(s, name)
        dense = torch.zeros(c["batch"], c["rows"], c["heads_kv"], HEAD, dtype=torch.float64, device="cuda")
        for i in range(c["batch"]):
            n = int(s["counts"][i]) if s["counts"] is not None else c["rows"]
            first = int(s["start"][i])
            flat = pages[s["table"][i].long()].permute(0, 2, 1, 3).reshape(-1, c["heads_kv"], HEAD)
            dense[i, :n] = flat[first:first + n]
        out[name] = dense
    return out


def _exact_attn(c, s):
    b, n, ctx, hq, hkv = c["batch"], c["nodes"], c["ctx"], c["heads_q"], c["heads_kv"]
    out = torch.empty(b, n, hq, HEAD, dtype=torch.float64, device="cuda")
    for i in range(b):
        length = int(s["ctx_len"][i])
        own_pages = s["table"][i].long()
        k, v = ({**s, name: s[name][own_pages], name + "_exp": None if s[name + "_exp"] is None else s[name + "_exp"][own_pages]}
                for name in ("k", "v"))
        k, v = (_exact_pages(x, name).permute(1, 0, 2, 3).reshape(hkv, -1, HEAD)[:, :length] for x, name in ((k, "k"), (v, "v")))
        vis = torch.cat([torch.ones(n, length, dtype=torch.bool, device="cuda"), s["see"][i]], dim=1)
        for h in range(hq):
            g = h // (hq // hkv)
            kk = torch.cat([k[g], s["k_tree"][i, :, g].double()])
            vv = torch.cat([v[g], s["v_tree"][i, :, g].double()])
            x = (s["q"][i, :, h].double() @ kk.t()) * HEAD ** -0.5
            out[i, :, h] = torch.softmax(x.masked_fill(~vis, -math.inf), dim=1) @ vv
    return out


_EXACT = {"write": _exact_write, "read": _exact_read, "attn": _exact_attn}
