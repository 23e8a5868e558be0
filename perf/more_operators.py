"""Performance cases of the operators around a paged cache held in 4 bits: rotary
positions of queries and keys, the cache itself (written, read back and attended
to), and its pages (taken, shared, copied, moved together and given back).

Kinds of case:

* ``rope``: queries and keys turned by their positions (``rotary``), in either
  layout, whole heads or a part of each, with frequencies for long contexts;
* ``store``: keys and values of prompts or accepted tree nodes into a cache in
  4 bits (``cache_write``) and the same positions back as dense bf16
  (``cache_read``);
* ``attn``: one attention layer of a tree of drafted tokens, a chain or a single
  token over that cache (``tree_attention_paged``);
* ``step``: a serving step's pages: ended requests give theirs back
  (``pages_fork``), the others' next positions get a page each or a copy of one
  that they share (``pages_reserve``, ``cache_copy``);
* ``fork``: prompts continued several times over (the same three calls);
* ``compact``: the pages in use moved to the front of the pool
  (``pages_compact``, ``cache_copy``).

``own`` false: the plain form, elementary torch operations; true: the library.

Layout of a cache: pages [num_pages][heads_kv][page][128]; position t of a
request lies in slot t % page of page table[request][t // page].  In 4 bits
(e2m1: sign, 2 exponent bits, 1 of mantissa: 0, 0.5, 1, 1.5, 2, 3, 4, 6) a row is
64 bytes, element 2 i in the low half of byte i, and block j of 32 elements stands
for its values times 2^(exp - 127) with exp [num_pages][heads_kv][page][4].
"""
from __future__ import annotations

import math

import torch

own = False

HEAD = 128            # elements of a cached head
BLOCK = 32            # elements under one power of two
E2M1 = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)
EXP_LOW, EXP_HIGH = -100, 125
BF16, E4M3, FP32 = "bf16", "e4m3", "fp32"
HALF, INTERLEAVED = "half", "interleaved"
PLAIN, LINEAR, BASE, TURNS = "plain", "linear", "base", "turns"


def listed():
    return [
        # queries and keys of one request's drafted tree of 64 nodes, positions by depth: the smallest call
        _rope("rope-tree", batch=1, rows=64, heads_q=32, heads_kv=8, tree=True),
        # the prompts of 8 requests in the rows of a fused projection, frequencies for four times the trained length
        _rope("rope-prompt", batch=8, rows=2048, heads_q=32, heads_kv=8, scaling=TURNS, fused=True, ragged=True),
        # part of each head, interleaved, in fp32, a million positions on, turned back (the gradient of the rotation)
        _rope("rope-odd", batch=3, rows=777, heads_q=12, heads_kv=4, rot=80, layout=INTERLEAVED, held=FP32, scaling=LINEAR,
              far=1000000, inverse=True),
        # a decoding step's accepted nodes (up to 16 of 64 drafted) of 16 requests
        _store("store-accepted", batch=16, source=64, rows=16, heads_kv=8, page=64, indexed=True),
        # the prompts of 8 requests, keys and values in the rows of a fused projection
        _store("store-prompt", batch=8, source=2048, rows=2048, heads_kv=8, page=64, ragged=True, fused=True),
        # one request's drafted tree of 64 nodes over 2048 positions: latency counts
        _attn("attn4-tree", batch=1, nodes=64, ctx=2048, heads_q=32, heads_kv=8, page=64),
        # single tokens of 64 requests over ragged caches of up to 8192 positions
        _attn("attn4-token", batch=64, nodes=1, ctx=8192, heads_q=32, heads_kv=8, page=64, ragged=True),
        # small trees over two long caches
        _attn("attn4-long", batch=2, nodes=16, ctx=65536, heads_q=32, heads_kv=8, page=256),
        # sixteen requests' trees of 512 nodes: the most products
        _attn("attn4-x16", batch=16, nodes=512, ctx=2048, heads_q=32, heads_kv=8, page=64),
        # a decoding step of 64 requests, an eighth of them ended, some forked by the step before: latency counts
        _pages("pages-step", "step", batch=64, ctx=4096, rows=16, heads_kv=8, page=64, held=E4M3),
        # eight prompts, each continued eight times: their last pages are copied
        _pages("pages-fork", "fork", batch=64, ctx=2048, rows=1, heads_kv=8, page=256, held=BF16),
        # a pool of which two fifths are in use: the largest copy
        _pages("pages-compact", "compact", batch=64, ctx=8192, rows=1, heads_kv=8, page=64, held=E4M3),
    ]


def draw(rng):
    kind = rng.choice(["rope", "rope", "store", "attn", "attn", "attn", "step", "fork", "compact"])
    page = rng.choice([16, 32, 64, 128, 256])
    hkv = rng.choice([1, 2, 4, 8])
    group = rng.choice([1, 2, 4, 8])
    while kind == "rope":
        b, rows, held = _log(rng, 1, 64), _log(rng, 1, 4096), rng.choice([BF16, BF16, FP32])
        if b * rows * hkv * (group + 1) * (2 if held == FP32 else 1) <= 8 * 2048 * 40:
            return _rope(None, batch=b, rows=rows, heads_q=hkv * group, heads_kv=hkv,
                         rot=rng.choice([HEAD, HEAD, 64, 2 * rng.randint(1, 64)]), layout=rng.choice([HALF, INTERLEAVED]),
                         held=held, scaling=rng.choice([PLAIN, LINEAR, BASE, TURNS]), tree=rows <= 512 and rng.random() < 0.4,
                         fused=rng.random() < 0.5, ragged=rng.random() < 0.5, far=rng.choice([0, _log(rng, 1000, 1 << 24)]),
                         inverse=rng.random() < 0.3)
    while kind == "store":
        b, rows = _log(rng, 1, 64), _log(rng, 1, 4096)
        if b * rows * hkv <= 8 * 2048 * 8:
            indexed = rows <= 64 and rng.random() < 0.5
            return _store(None, batch=b, source=rows + _log(rng, 1, 64) if indexed else rows, rows=rows, heads_kv=hkv,
                          page=page, indexed=indexed, ragged=rng.random() < 0.5, fused=rng.random() < 0.5)
    while kind == "attn":
        b, nodes, ctx = _log(rng, 1, 64), _log(rng, 1, 512), _log(rng, 64, 65536)
        if b * ctx <= 64 * 8192 and b * nodes * hkv * group * (ctx + nodes) <= 16 * 512 * 32 * 2560:
            return _attn(None, batch=b, nodes=nodes, ctx=ctx, heads_q=hkv * group, heads_kv=hkv, page=page,
                         ragged=rng.random() < 0.5)
    while True:
        b, ctx, held = _log(rng, 8, 256), _log(rng, 64, 32768), rng.choice([BF16, E4M3])
        if b * ctx * hkv * (2 if held == BF16 else 1) <= 64 * 8192 * 8 and b * (ctx // page + 1) >= 8:
            return _pages(None, kind, batch=b, ctx=ctx, rows=_log(rng, 1, min(ctx, 512)) if kind == "step" else 1,
                          heads_kv=hkv, page=page, held=held)


def _log(rng, lo, hi):
    """A whole number of lo .. hi, uniform over its logarithm."""
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _case(name, **kw):
    return {"name": name, **kw} if name else kw


def _rope(name, *, batch, rows, heads_q, heads_kv, rot=HEAD, layout=HALF, held=BF16, scaling=PLAIN, tree=False, fused=False,
          ragged=False, far=0, inverse=False):
    return _case(name, kind="rope", batch=batch, rows=rows, heads_q=heads_q, heads_kv=heads_kv, rot=rot, layout=layout,
                 held=held, scaling=scaling, tree=tree, fused=fused, ragged=ragged, far=far, inverse=inverse)


def _store(name, *, batch, source, rows, heads_kv, page, indexed=False, ragged=False, fused=False):
    return _case(name, kind="store", batch=batch, source=source, rows=rows, heads_kv=heads_kv, page=page, indexed=indexed,
                 ragged=ragged, fused=fused)


def _attn(name, *, batch, nodes, ctx, heads_q, heads_kv, page, ragged=False):
    return _case(name, kind="attn", batch=batch, nodes=nodes, ctx=ctx, heads_q=heads_q, heads_kv=heads_kv, page=page,
                 ragged=ragged)


def _pages(name, kind, *, batch, ctx, rows, heads_kv, page, held):
    return _case(name, kind=kind, batch=batch, ctx=ctx, rows=rows, heads_kv=heads_kv, page=page, held=held)


# ---------------------------------------------------------------------------
# Inputs
# ---------------------------------------------------------------------------

ROPE_BASE = 10000.0
SCALING = {   # rule, factor, low, high, length, amplitude
    PLAIN: (PLAIN, 1.0, 0.0, 0.0, 0, 1.0),
    LINEAR: (LINEAR, 8.0, 0.0, 0.0, 0, 1.0),
    BASE: (BASE, 4.0, 0.0, 0.0, 0, 1.0),
    TURNS: (TURNS, 4.0, 1.0, 32.0, 4096, 1.0 + 0.1 * math.log(4.0)),
}


def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(0x0DE90000 + int(seed))


def _normal(g, shape, dtype=torch.bfloat16):
    return torch.randn(shape, generator=g, device="cuda").to(dtype)


def _whole(g, lo, hi, shape):
    return torch.randint(lo, hi + 1, shape, generator=g, device="cuda", dtype=torch.int32)


def prepare(case, seed):
    s = {"case": case, **_PREPARE[case["kind"]](case, _gen(seed))}
    if own:   # scalar arguments, the table of frequencies and the workspaces, which a program keeps
        s["handle"] = _HANDLE[case["kind"]](case, s)
    return s


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


def _prepare_rope(c, g):
    b, rows, hq, hkv = c["batch"], c["rows"], c["heads_q"], c["heads_kv"]
    dtype = torch.bfloat16 if c["held"] == BF16 else torch.float32
    if c["fused"]:   # q, k and v side by side in a row
        x = _normal(g, (b, rows, hq + 2 * hkv, HEAD), dtype)
        q, k = x[:, :, :hq], x[:, :, hq:hq + hkv]
    else:
        q, k = _normal(g, (b, rows, hq, HEAD), dtype), _normal(g, (b, rows, hkv, HEAD), dtype)
    positions = None
    if c["tree"]:   # depths 1 .. of the nodes
        edges = _levels(rows, min(16, rows))
        depth = [i + 1 for i, (lo, hi) in enumerate(zip(edges[:-1], edges[1:])) for _ in range(hi - lo)]
        positions = torch.tensor(depth, dtype=torch.int32, device="cuda").repeat(b, 1)
    return {"q": q, "k": k, "positions": positions, "start": _whole(g, c["far"], c["far"] + 4096, (b,)),
            "counts": _whole(g, (rows + 1) // 2, rows, (b,)) if c["ragged"] else None,
            "q_out": torch.zeros(b, rows, hq, HEAD, dtype=dtype, device="cuda"),
            "k_out": torch.zeros(b, rows, hkv, HEAD, dtype=dtype, device="cuda")}


def _pool(c, g, positions, filled):
    """An empty or a filled cache in 4 bits of `positions` per request, its pages in no order."""
    b, hkv, page = c["batch"], c["heads_kv"], c["page"]
    per = -(-positions // page)
    n = b * per + 2
    table = torch.randperm(n, generator=g, device="cuda")[: b * per].view(b, per).to(torch.int32)
    out = {"table": table, "num_pages": n}
    for name in ("k", "v"):
        if filled:
            out[name], out[name + "_exp"] = _packed(torch.randn((n, hkv, page, HEAD), generator=g, device="cuda").to(torch.bfloat16))
        else:
            out[name] = torch.zeros(n, hkv, page, HEAD // 2, dtype=torch.uint8, device="cuda")
            out[name + "_exp"] = torch.full((n, hkv, page, HEAD // BLOCK), 127, dtype=torch.uint8, device="cuda")
    return out


def _prepare_store(c, g):
    b, src, rows, hkv = c["batch"], c["source"], c["rows"], c["heads_kv"]
    if c["fused"]:   # q, k and v side by side in a row, four query heads a key/value head
        x = _normal(g, (b, src, 6 * hkv, HEAD))
        k, v = x[:, :, 4 * hkv:5 * hkv], x[:, :, 5 * hkv:]
    else:
        k, v = _normal(g, (b, src, hkv, HEAD)), _normal(g, (b, src, hkv, HEAD))
    index = None
    if c["indexed"]:
        index = torch.rand(b, src, generator=g, device="cuda").argsort(dim=1)[:, :rows].sort(dim=1).values.to(torch.int32).contiguous()
    return {"k_new": k, "v_new": v, "start": _whole(g, 0, 2 * c["page"], (b,)), "index": index,
            "counts": _whole(g, (rows + 1) // 2, rows, (b,)) if c["ragged"] or c["indexed"] else None,
            "k_out": torch.zeros(b, rows, hkv, HEAD, dtype=torch.bfloat16, device="cuda"),
            "v_out": torch.zeros(b, rows, hkv, HEAD, dtype=torch.bfloat16, device="cuda"),
            **_pool(c, g, 2 * c["page"] + rows, False)}


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


def _shape_of_pages(c):
    """(columns of the page table, pages of the pool)."""
    columns = -(-(c["ctx"] + c["rows"]) // c["page"]) + 1
    return columns, c["batch"] * columns


def _prepare_pages(c, g):
    b, page, hkv, kind = c["batch"], c["page"], c["heads_kv"], c["kind"]
    columns, n = _shape_of_pages(c)
    at = torch.arange(b, device="cuda")
    length = _whole(g, (c["ctx"] + 1) // 2, c["ctx"], (b,))
    if kind == "fork":      # eight rows a prompt, the first of which holds it
        length, shares = length[at // 8 * 8], torch.zeros(b, dtype=torch.bool, device="cuda")
        used = torch.where(at % 8 == 0, length, 0)
    elif kind == "step":    # of four requests the second shares the pages of the first
        shares = at % 4 == 1
        length = torch.where(shares, length.roll(1), length)
        used = length
    else:                   # the requests that have not ended
        shares = torch.zeros(b, dtype=torch.bool, device="cuda")
        used = length = torch.where(torch.rand(b, generator=g, device="cuda") < 0.5, length, 0)
    need = (used + page - 1) // page
    first = (torch.where(shares, 0, need)).cumsum(0) - need
    first = torch.where(shares, first.roll(1), first)
    column = torch.arange(columns, device="cuda")
    named = torch.randperm(n, generator=g, device="cuda")[(first[:, None] + column).clamp(0, n - 1)]
    table = torch.where(column < need[:, None], named, -1).to(torch.int32)
    keep = torch.where(torch.rand(b, generator=g, device="cuda") < 0.125, 0, length) if kind == "step" else length
    counts = torch.where(keep > 0, _whole(g, 1, c["rows"], (b,)), 0)
    i32 = lambda *shape: torch.full(shape, -1, dtype=torch.int32, device="cuda")
    dtype = torch.float8_e4m3fn if c["held"] == E4M3 else torch.bfloat16
    out = {"table": table, "num_pages": n, "keep": keep.to(torch.int32), "counts": counts.to(torch.int32),
           "source": (at // 8 * 8).to(torch.int32), "forked": i32(b, columns), "out": i32(b, columns),
           "pairs": i32(n // 2 if kind == "compact" else b * _most_columns(c), 2), "totals": i32(2), "granted": i32(b)}
    for name in ("k", "v"):
        out[name] = torch.randn((n, hkv, page, HEAD), generator=g, device="cuda").to(dtype)
        out[name + "_exp"] = _whole(g, 120, 130, (n, hkv, page)).to(torch.uint8) if c["held"] == E4M3 else None
    return out


def _most_columns(c):
    """Pages that `rows` positions can touch."""
    return (c["rows"] + c["page"] - 2) // c["page"] + 1


_PREPARE = {"rope": _prepare_rope, "store": _prepare_store, "attn": _prepare_attn, "step": _prepare_pages,
            "fork": _prepare_pages, "compact": _prepare_pages}


# ---------------------------------------------------------------------------
# One pass
# ---------------------------------------------------------------------------

def run(s):
    kind = s["case"]["kind"]
    return (_RUN_OWN if own else _RUN_PLAIN)[kind](s)


def _handle_rope(c, s):
    from paper_2608_13524_amd import dartree as D
    rule, factor, low, high, length, amplitude = SCALING[c["scaling"]]
    kinds = {PLAIN: D.ROTARY_PLAIN, LINEAR: D.ROTARY_LINEAR, BASE: D.ROTARY_BASE, TURNS: D.ROTARY_TURNS}
    p = D.RotaryParams(c["batch"], c["rows"], c["heads_q"], c["heads_kv"], HEAD, c["rot"],
                       D.ROTARY_HALF if c["layout"] == HALF else D.ROTARY_INTERLEAVED,
                       D.BF16 if c["held"] == BF16 else D.FP32, int(c["inverse"]), -1 if c["tree"] else 0, amplitude)
    return {"p": p, "turns": D.rotary_turns(c["rot"], ROPE_BASE, D.RotaryScaling(kinds[rule], factor, low, high, length))}


def _handle_cache(c, s):
    from paper_2608_13524_amd import dartree as D
    held = {E4M3: D.CACHE_E4M3, BF16: D.CACHE_BF16}[c["held"]] if "held" in c else D.CACHE_E2M1
    p = D.CacheParams(c["batch"], c["heads_kv"], HEAD, c["page"], s["num_pages"], s["table"].shape[1], held)
    h = {"p": p, "cache": D.DeviceCache(s["k"], s["v"], s["k_exp"], s["v_exp"], s["table"])}
    nbytes = 0
    if c["kind"] == "attn":
        h["a"] = D.AttnParams(c["batch"], c["nodes"], c["ctx"], c["heads_q"], c["heads_kv"], HEAD, 1.0 / math.sqrt(HEAD))
        nbytes = D.tree_attention_paged_workspace_size(h["a"], p)
    elif c["kind"] in ("step", "fork", "compact"):
        nbytes = D.pages_workspace_size(p)
    h["ws"] = torch.empty(nbytes, dtype=torch.uint8, device="cuda") if nbytes else None
    return h


_HANDLE = {"rope": _handle_rope, **{kind: _handle_cache for kind in ("store", "attn", "step", "fork", "compact")}}


def _own_rope(s):
    from paper_2608_13524_amd import dartree as D
    D.rotary(s["handle"]["p"], s["handle"]["turns"], s["q"], s["k"], s["q_out"], s["k_out"], positions=s["positions"],
             start=s["start"], counts=s["counts"])
    return {"q": s["q_out"], "k": s["k_out"]}


def _own_store(s):
    from paper_2608_13524_amd import dartree as D
    h = s["handle"]
    D.cache_write(h["p"], h["cache"], s["k_new"], s["v_new"], s["case"]["rows"], index=s["index"], counts=s["counts"],
                  start=s["start"])
    D.cache_read(h["p"], h["cache"], s["k_out"], s["v_out"], counts=s["counts"], start=s["start"])
    return {"k": s["k_out"], "v": s["v_out"]}


def _own_attn(s):
    from paper_2608_13524_amd import dartree as D
    h = s["handle"]
    D.tree_attention_paged(h["a"], h["p"], h["cache"], s["q"], s["k_tree"], s["v_tree"], s["mask"], s["ctx_len"],
                           s["out"], h["ws"])
    return s["out"]


def _own_reserve(s):
    from paper_2608_13524_amd import dartree as D
    h, fork = s["handle"], s["case"]["kind"] == "fork"
    D.pages_fork(h["p"], s["table"], s["forked"], source=s["source"] if fork else None, keep=s["keep"])
    D.pages_reserve(h["p"], s["forked"], s["out"], s["case"]["rows"], s["keep"], s["counts"], s["pairs"], s["totals"],
                    s["granted"], h["ws"])
    D.cache_copy(h["p"], h["cache"], s["pairs"], s["totals"])
    return _pages_out(s)


def _own_compact(s):
    from paper_2608_13524_amd import dartree as D
    h = s["handle"]
    D.pages_compact(h["p"], s["table"], s["out"], s["pairs"], s["totals"], h["ws"])
    D.cache_copy(h["p"], h["cache"], s["pairs"], s["totals"])
    return _pages_out(s)


def _pages_out(s):
    names = ("out", "pairs", "totals", "k", "v", "k_exp", "v_exp")
    return {name: s[name] for name in (names if s["case"]["kind"] == "compact" else names + ("granted",))}


_RUN_OWN = {"rope": _own_rope, "store": _own_store, "attn": _own_attn, "step": _own_reserve, "fork": _own_reserve,
            "compact": _own_compact}


# ---------------------------------------------------------------------------
# The plain forms
# ---------------------------------------------------------------------------

def _frequencies(rot, scaling):
    """Radians a position of every pair, in 64 bits."""
    rule, factor, low, high, length, _ = SCALING[scaling]
    base = ROPE_BASE * factor ** (rot / (rot - 2)) if rule == BASE and rot > 2 else ROPE_BASE
    f = base ** (-torch.arange(0, rot, 2, dtype=torch.float64, device="cuda") / rot)
    if rule == LINEAR:
        return f / factor
    if rule == TURNS:   # pairs that turn often within the trained length stay, slow ones are stretched
        kept = ((length * f / (2 * math.pi) - low) / (high - low)).clamp(0, 1)
        return f * (kept + (1 - kept) / factor)
    return f


def _plain_rope(s):
    c = s["case"]
    rows, rot = c["rows"], c["rot"]
    at = s["start"][:, None].double() + (s["positions"] - 1 if c["tree"] else torch.arange(rows, device="cuda"))
    angle = at[..., None] * _frequencies(rot, c["scaling"])
    amplitude = SCALING[c["scaling"]][5]
    cos, sin = ((amplitude * x(angle)).float()[:, :, None] for x in (torch.cos, torch.sin))
    if c["inverse"]:
        sin = -sin
    out = {}
    for name in ("q", "k"):
        x = s[name].float()
        part = x[..., :rot]
        if c["layout"] == HALF:
            a, b = part[..., :rot // 2], part[..., rot // 2:]
            turned = torch.cat([a * cos - b * sin, b * cos + a * sin], dim=-1)
        else:
            a, b = part[..., 0::2], part[..., 1::2]
            turned = torch.stack([a * cos - b * sin, b * cos + a * sin], dim=-1).flatten(-2)
        x = torch.cat([turned, x[..., rot:]], dim=-1).to(s[name].dtype)
        if s["counts"] is not None:
            there = torch.arange(rows, device="cuda") < s["counts"][:, None]
            x = torch.where(there[:, :, None, None], x, s[name + "_out"])
        s[name + "_out"].copy_(x)
        out[name] = s[name + "_out"]
    return out


def _packed(x):
    """(bytes, exponents + 127) of rows of 128: per 32 elements the least power of two that brings the largest to 6."""
    x = x.float().unflatten(-1, (-1, BLOCK))
    m, e = torch.frexp(x.abs().amax(dim=-1))     # m in [0.5, 1): 6 is 0.75 * 2^3
    e = torch.where(m > 0.75, e - 2, e - 3).clamp(EXP_LOW, EXP_HIGH)
    e = torch.where(m == 0, EXP_LOW, e)
    y = torch.ldexp(x, -e[..., None])
    # nearest, ties to the even code: an odd code takes in what lies strictly between, an even one its borders too
    a, code = y.abs(), torch.zeros(y.shape, dtype=torch.uint8, device=y.device)
    for i, (lo, hi) in enumerate(zip(E2M1[:-1], E2M1[1:])):
        code += (a > (lo + hi) / 2) if i % 2 == 0 else (a >= (lo + hi) / 2)
    code = (code + 8 * torch.signbit(y).to(torch.uint8)).flatten(-2)
    return code[..., 0::2] | (code[..., 1::2] << 4), (e + 127).to(torch.uint8)


def _unpacked(x, exp):
    """Rows in 4 bits as the values they stand for, in 32 bits."""
    values = torch.tensor(E2M1 + tuple(-v for v in E2M1), device=x.device)
    x = torch.stack([values[(x & 15).int()], values[(x >> 4).int()]], dim=-1).flatten(-2)
    return torch.ldexp(x.unflatten(-1, (-1, BLOCK)), (exp.int() - 127)[..., None]).flatten(-2)


def _plain_store(s):
    c = s["case"]
    rows = c["rows"]
    at = s["start"][:, None].long() + torch.arange(rows, device="cuda")
    there = torch.arange(rows, device="cuda") < (s["counts"] if s["counts"] is not None else torch.full_like(s["start"], rows))[:, None]
    pages = s["table"].long().gather(1, (at // c["page"]).clamp(max=s["table"].shape[1] - 1))[there]
    slot = (at % c["page"])[there]
    for name in ("k", "v"):
        x = s[name + "_new"]
        if s["index"] is not None:
            x = x.gather(1, s["index"].long()[:, :, None, None].expand(-1, -1, c["heads_kv"], HEAD))
        s[name][pages, :, slot], s[name + "_exp"][pages, :, slot] = _packed(x[there])
        s[name + "_out"][there] = _unpacked(s[name][pages, :, slot], s[name + "_exp"][pages, :, slot]).to(torch.bfloat16)
    return {"k": s["k_out"], "v": s["v_out"]}


def _plain_attn(s):
    c = s["case"]
    b, n, ctx, hq, hkv = c["batch"], c["nodes"], c["ctx"], c["heads_q"], c["heads_kv"]
    group = hq // hkv

    def keys(name):   # [b][heads_kv][ctx + nodes][128]
        pages = s["table"].long()
        x = _unpacked(s[name][pages], s[name + "_exp"][pages]).transpose(1, 2).reshape(b, hkv, -1, HEAD)[:, :, :ctx]
        return torch.cat([x, s[name + "_tree"].float().transpose(1, 2)], dim=2)

    q = s["q"].float().view(b, n, hkv, group, HEAD).permute(0, 2, 1, 3, 4).reshape(b, hkv, n * group, HEAD)
    x = torch.matmul(q, keys("k").transpose(2, 3).contiguous()) / math.sqrt(HEAD)
    seen = torch.arange(ctx, device="cuda") < s["ctx_len"][:, None]
    vis = torch.cat([seen[:, None].expand(b, n, ctx), s["see"]], dim=2).repeat_interleave(group, dim=1)
    x = x.masked_fill_(~vis[:, None], -math.inf)
    x = torch.exp(x - x.amax(dim=3, keepdim=True))
    out = torch.matmul(x / x.sum(dim=3, keepdim=True), keys("v"))
    return out.view(b, hkv, n, group, HEAD).permute(0, 2, 1, 3, 4).reshape(b, n, hq, HEAD).to(torch.bfloat16)


def _holders(table, n):
    """How many entries of the table name each page (the last count: entries that name none)."""
    at = torch.where((table >= 0) & (table < n), table, n).long().flatten()
    return torch.zeros(n + 1, dtype=torch.int64, device="cuda").scatter_add_(0, at, torch.ones_like(at))


def _copied(s, pairs):
    """Pages `pairs` [n][2] copied from the first to the second."""
    for name in ("k", "v", "k_exp", "v_exp"):
        if s[name] is not None:
            x = s[name].view(torch.uint8)
            x[pairs[:, 1]] = x[pairs[:, 0]]


def _plain_reserve(s):
    c, n = s["case"], s["num_pages"]
    b, page = c["batch"], c["page"]
    column = torch.arange(s["table"].shape[1], device="cuda")
    from_row = s["table"][s["source"].long()] if c["kind"] == "fork" else s["table"]
    table = torch.where(column < ((s["keep"] + page - 1) // page)[:, None], from_row, -1)
    # what the next positions need: a page where there is none, a copy where others name it too
    first, past = s["keep"], s["keep"] + s["counts"]
    touched = (column >= (first // page)[:, None]) & (column < ((past + page - 1) // page)[:, None]) & (s["counts"] > 0)[:, None]
    holders = _holders(table, n)
    there = (table >= 0) & (table < n)
    shared = touched & there & (holders[table.clamp(0, n - 1).long()] > 1)
    need = shared | (touched & ~there)
    free = (holders[:n] == 0).sum()
    granted = need.sum(dim=1).cumsum(0) <= free
    need &= granted[:, None]
    lowest = torch.argsort((holders[:n] > 0).to(torch.int8), stable=True)   # free pages first, ascending
    rank = need.flatten().cumsum(0).view(b, -1) - 1
    out = torch.where(need, lowest[rank.clamp(0, n - 1)].to(torch.int32), table)
    covered = (first[:, None] <= column * page) & (past[:, None] >= (column + 1) * page)   # a page that is written whole
    moved = need & shared & ~covered
    pairs = torch.stack([table[moved], out[moved]], dim=1)
    s["pairs"][:pairs.shape[0]] = pairs
    s["totals"][0], s["totals"][1] = pairs.shape[0], free - need.sum()
    s["out"].copy_(out)
    s["granted"].copy_(granted)
    _copied(s, pairs.long())
    return _pages_out(s)


def _plain_compact(s):
    n, table = s["num_pages"], s["table"]
    used = _holders(table, n)[:n] > 0
    live = used.sum()
    page = torch.arange(n, device="cuda")
    away, to = page[used & (page >= live)], page[~used & (page < live)]
    place = page.clone()
    place[away] = to
    there = (table >= 0) & (table < n)
    s["out"].copy_(torch.where(there, place[table.clamp(0, n - 1).long()].to(torch.int32), -1))
    pairs = torch.stack([away, to], dim=1)
    s["pairs"][:pairs.shape[0]] = pairs.to(torch.int32)
    s["totals"][0], s["totals"][1] = pairs.shape[0], live
    _copied(s, pairs)
    return _pages_out(s)


_RUN_PLAIN = {"rope": _plain_rope, "store": _plain_store, "attn": _plain_attn, "step": _plain_reserve, "fork": _plain_reserve,
              "compact": _plain_compact}


# ---------------------------------------------------------------------------
# What a pass cannot do without
# ---------------------------------------------------------------------------

def work(case):
    c = case
    kind = c["kind"]
    if kind == "rope":
        rows = c["batch"] * c["rows"] * (0.75 if c["ragged"] else 1.0)
        heads, size = c["heads_q"] + c["heads_kv"], 2 if c["held"] == BF16 else 4
        return {"bytes": rows * (2 * heads * HEAD * size + (4 if c["tree"] else 0)), "flops": rows * heads * 3 * c["rot"]}
    if kind in ("store", "attn"):
        row = 2 * c["heads_kv"] * (HEAD // 2 + HEAD // BLOCK)   # a position's keys and values in the cache
        dense = 4 * c["heads_kv"] * HEAD                        # and as bf16
    if kind == "store":
        positions = c["batch"] * c["rows"] * (0.75 if c["ragged"] or c["indexed"] else 1.0)
        return {"bytes": 2 * positions * (row + dense), "flops": 0}
    if kind == "attn":
        seen = c["ctx"] * (0.75 if c["ragged"] else 1.0)
        nodes = c["batch"] * c["nodes"]
        return {"bytes": c["batch"] * seen * row + nodes * (dense + 4 * c["heads_q"] * HEAD + 8 * ((c["nodes"] + 63) // 64)),
                "flops": 4.0 * nodes * c["heads_q"] * HEAD * (seen + c["nodes"])}
    # the page tables, and the pages that are copied
    columns, n = _shape_of_pages(c)
    one = 2 * c["heads_kv"] * c["page"] * (HEAD + 1 if c["held"] == E4M3 else 2 * HEAD)
    pages = -(-3 * c["ctx"] // (4 * c["page"]))
    if kind == "compact":
        used = min(1.0, c["batch"] * pages / 2 / n)
        return {"bytes": 2 * 4 * c["batch"] * columns + 2 * one * n * used * (1 - used), "flops": 0}
    copies = c["batch"] * (7 / 16 if kind == "step" else 1)    # those of the forked that go on
    return {"bytes": 4 * 4 * c["batch"] * columns + 2 * one * copies * (1 - 1 / c["page"]), "flops": 0}


# ---------------------------------------------------------------------------
# The same outputs in 64 bits
# ---------------------------------------------------------------------------

def exact(case, seed):
    return _EXACT[case["kind"]](case, prepare(case, seed)) if case["kind"] in _EXACT else None


def _exact_rope(c, s):
    """Pairs as complex numbers times amplitude e^(i angle)."""
    rule, factor, low, high, length, amplitude = SCALING[c["scaling"]]
    rot, freq = c["rot"], []
    for i in range(rot // 2):
        base = ROPE_BASE
        if rule == BASE and rot > 2:
            base *= math.pow(factor, rot / (rot - 2))
        f = math.pow(base, -2.0 * i / rot)
        if rule == LINEAR:
            f /= factor
        if rule == TURNS:
            turns = f * length / (2 * math.pi)
            f *= 1 / factor if turns <= low else 1.0 if turns >= high else \
                ((turns - low) + (high - turns) / factor) / (high - low)
        freq.append(f)
    freq = torch.tensor(freq, dtype=torch.float64, device="cuda")
    out = {"q": s["q_out"].double(), "k": s["k_out"].double()}
    for q in range(c["batch"]):
        n = c["rows"] if s["counts"] is None else int(s["counts"][q])
        at = torch.arange(n, device="cuda", dtype=torch.float64) if s["positions"] is None else s["positions"][q, :n].double() - 1
        angle = (at + float(s["start"][q]))[:, None] * freq
        z = torch.polar(torch.full_like(angle, amplitude), -angle if c["inverse"] else angle)[:, None]
        for name in ("q", "k"):
            x = s[name][q, :n].double()
            pair = x[..., :rot].unflatten(-1, (2, -1)).transpose(-1, -2) if c["layout"] == HALF else x[..., :rot].unflatten(-1, (-1, 2))
            pair = torch.view_as_real(torch.view_as_complex(pair.contiguous()) * z)
            pair = pair.transpose(-1, -2).flatten(-2) if c["layout"] == HALF else pair.flatten(-2)
            out[name][q, :n] = torch.cat([pair, x[..., rot:]], dim=-1)
    return out


def _nearest(x):
    """Rows of 128 rounded to 4 bits and back: the multiples that the size of each element allows."""
    x = x.double().unflatten(-1, (-1, BLOCK))
    top = x.abs().amax(dim=-1, keepdim=True)
    scale = torch.pow(2.0, torch.ceil(torch.log2(top.clamp(min=2.0 ** -90) / 6.0)))
    x = x / scale
    grid = torch.pow(2.0, torch.floor(torch.log2(x.abs().clamp(min=1.0))) - 1.0)
    return (torch.round(x / grid) * grid * scale).flatten(-2)


def _exact_store(c, s):
    out = {}
    for name in ("k", "v"):
        out[name] = s[name + "_out"].double()
        for q in range(c["batch"]):
            n = int(s["counts"][q]) if s["counts"] is not None else c["rows"]
            out[name][q, :n] = _nearest(s[name + "_new"][q, s["index"][q, :n].long()] if s["index"] is not None else s[name + "_new"][q, :n])
    return out


def _decoded(x, exp):
    """e2m1 from its bits: sign, 2 exponent bits (bias 1), 1 of mantissa."""
    code = torch.stack([x.long() & 15, x.long() >> 4], dim=-1).flatten(-2)
    e, m = (code >> 1) & 3, (code & 1).double()
    v = torch.where(e == 0, m / 2, (1 + m / 2) * torch.pow(2.0, (e - 1).double())) * torch.where(code >= 8, -1.0, 1.0)
    return (v.unflatten(-1, (-1, BLOCK)) * torch.pow(2.0, exp.double() - 127.0)[..., None]).flatten(-2)


def _exact_attn(c, s):
    b, n, ctx, hq, hkv = c["batch"], c["nodes"], c["ctx"], c["heads_q"], c["heads_kv"]
    out = torch.empty(b, n, hq, HEAD, dtype=torch.float64, device="cuda")
    for i in range(b):
        length, pages = int(s["ctx_len"][i]), s["table"][i].long()
        k, v = (_decoded(s[x][pages], s[x + "_exp"][pages]).permute(1, 0, 2, 3).reshape(hkv, -1, HEAD)[:, :length] for x in ("k", "v"))
        vis = torch.cat([torch.ones(n, length, dtype=torch.bool, device="cuda"), s["see"][i]], dim=1)
        for h in range(hq):
            g = h // (hq // hkv)
            kk = torch.cat([k[g], s["k_tree"][i, :, g].double()])
            vv = torch.cat([v[g], s["v_tree"][i, :, g].double()])
            x = (s["q"][i, :, h].double() @ kk.t()) * HEAD ** -0.5
            out[i, :, h] = torch.softmax(x.masked_fill(~vis, -math.inf), dim=1) @ vv
    return out


_EXACT = {"rope": _exact_rope, "store": _exact_store, "attn": _exact_attn}
