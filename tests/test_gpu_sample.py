"""Verification from given random numbers on the GPU: the same tokens as the
plain forms in 64 bits.  Both evaluate the definition in 64 bits, so a result
could differ only where a random number lies within about 1e-11 of a border."""
import numpy as np
import pytest
import torch

from paper_2608_13524_amd import dartree as D
from tests import serve_ref as S
from tests.gpu_util import device, say

pytestmark = pytest.mark.gpu
F32, B16 = "fp32", "bf16"
LAST = np.float32(1.0) - np.float32(2.0 ** -24)   # the largest float below 1


def logits_of(rng, shape, sigma=2.0, held=F32):
    z = (rng.normal(size=shape) * sigma).astype(np.float32)
    return S.bf16(z) if held == B16 else z


def to_dev(z, held, pad=0):
    """Device logits whose rows are `pad` elements further apart than they are long."""
    t = torch.from_numpy(np.ascontiguousarray(z)).to(torch.bfloat16 if held == B16 else torch.float32)
    wide = torch.full((*z.shape[:-1], z.shape[-1] + pad), float("inf"), dtype=t.dtype, device=device())
    wide[..., : z.shape[-1]] = t.to(device())
    return wide[..., : z.shape[-1]]


def i32(x):
    return torch.from_numpy(np.ascontiguousarray(x, np.int32)).to(device())


def random_trees(rng, b, n, vocab, spine=0.6, kids=4):
    """Trees whose parents precede children; siblings hold distinct tokens."""
    parents, tokens = np.full((b, n), -1), np.zeros((b, n), int)
    for q in range(b):
        held = {}
        for j in range(n):
            while True:
                p = j - 1 if rng.random() < spine else int(rng.integers(-1, j)) if j else -1
                if len(held.get(p, ())) < min(kids, vocab):
                    break
            t = int(rng.integers(0, vocab))
            while t in held.setdefault(p, []):
                t = int(rng.integers(0, vocab))
            held[p].append(t)
            parents[q, j], tokens[q, j] = p, t
    return tokens, parents


def boosted(z, tokens, parents, rng, temperature, p_keep=0.8):
    """Raise drafted children so that the target follows the draft most of the time."""
    t = temperature or 1.0
    for q in range(z.shape[0]):
        for j in range(tokens.shape[1]):
            row = z[q, parents[q, j] + 1]
            rest = t * np.log(np.exp((row.astype(np.float64) - row.max()) / t).sum()) + row.max()
            row[tokens[q, j] % z.shape[2]] = rest + t * np.log(p_keep / (1 - p_keep)) + t * rng.normal()
    return z


def run_tree(tokens, parents, num, z, temperature, u, max_len, held=F32, pad=0):
    b, n = tokens.shape
    vocab = z.shape[2]
    dev = device()
    acc = torch.full((b, max_len), -9, dtype=torch.int32, device=dev)
    cnt, bonus = torch.full((b,), -9, dtype=torch.int32, device=dev), torch.full((b,), -9, dtype=torch.int32, device=dev)
    need = D.verify_tree_workspace_size(b, n, max_len, vocab)
    ws = torch.full((need,), 0xFF, dtype=torch.uint8, device=dev)
    say(f"verify_tree b={b} B={n} V={vocab} T={temperature} max_len={max_len} {held} pad={pad}")
    D.verify_tree(i32(tokens), i32(parents), i32(num), to_dev(z, held, pad), temperature,
                  torch.from_numpy(np.ascontiguousarray(u, np.float32)).to(dev), acc, cnt, bonus, ws)
    torch.cuda.synchronize()
    return acc.cpu().numpy(), cnt.cpu().numpy(), bonus.cpu().numpy()


def check_tree(tokens, parents, num, z, temperature, u, max_len, held=F32, pad=0):
    acc, cnt, bonus = run_tree(tokens, parents, num, z, temperature, u, max_len, held, pad)
    for q in range(len(tokens)):
        path, tok = S.verify_tree(tokens[q], parents[q], num[q], z[q], temperature, u[q], max_len)
        assert acc[q, : len(path)].tolist() == path and (acc[q, len(path):] == -1).all(), q
        assert cnt[q] == len(path) and bonus[q] == tok, (q, bonus[q], tok)
    return cnt


@pytest.mark.parametrize("held", [F32, B16])
@pytest.mark.parametrize("temperature", [0.0, 0.7, 1.0])
@pytest.mark.parametrize("b,n,vocab,pad", [(1, 1, 1, 0), (3, 5, 5, 3), (4, 12, 100, 0), (2, 64, 4096, 0), (3, 40, 4097, 1),
                                           (2, 33, 8191, 2), (2, 16, 50257, 0)])
def test_trees(held, temperature, b, n, vocab, pad):
    rng = np.random.default_rng(b * 1000 + n + vocab)
    tokens, parents = random_trees(rng, b, n, vocab, kids=min(4, vocab)) if vocab > 1 else (np.zeros((b, n), int), np.full((b, n), -1))
    z = boosted(logits_of(rng, (b, n + 1, vocab)), tokens, parents, rng, temperature)
    if held == B16:
        z = S.bf16(z)
    seen = 0
    for trial in range(3):
        u = rng.random((b, n + 1)).astype(np.float32)
        num = np.full(b, n) if trial == 0 else rng.integers(0, n + 1, size=b)
        seen += check_tree(tokens, parents, num, z, temperature, u, 16 if trial < 2 else 2, held, pad).sum()
    assert seen > 0 or n < 5


@pytest.mark.parametrize("budget", [1024, 1025, 2000])
def test_large_budgets(budget):
    """On both sides of the largest tree that is walked from all rows at once; many children of one node."""
    rng = np.random.default_rng(budget)
    tokens, parents = random_trees(rng, 2, budget, 1500, spine=0.02, kids=600)
    z = boosted(logits_of(rng, (2, budget + 1, 1500)), tokens, parents, rng, 1.0, p_keep=0.02)
    for trial in range(3):
        u = rng.random((2, budget + 1)).astype(np.float32)
        u[0, 1:] = LAST if trial == 2 else u[0, 1:]     # every test of request 0 fails that can
        check_tree(tokens, parents, np.array([budget, budget - 7]), z, 1.0, u, 12)


def test_largest_budget_with_many_children():
    """4096 nodes, 600 of them children of the root; every child's token is taken or every one fails."""
    rng = np.random.default_rng(4096)
    tokens, parents = random_trees(rng, 2, 4096, 700, spine=0.02, kids=600)
    parents[0, :600], tokens[0, :600] = -1, rng.permutation(700)[:600]
    z = logits_of(rng, (2, 4097, 700))
    for first in (0.3, LAST):
        u = rng.random((2, 4097)).astype(np.float32)
        u[0, 1:601] = first
        check_tree(tokens, parents, np.array([4096, 4089]), z, 1.0, u, 12)


@pytest.mark.parametrize("held", [F32, B16])
@pytest.mark.parametrize("temperature,keep", [(1.0, 0.8), (1.0, 0.3), (0.7, 0.05), (0.0, 0.6)])
def test_long_paths_over_many_rows(held, temperature, keep):
    """Enough logits that only rows on the likeliest paths are read; paths of up to 60 nodes (more than
    a round's rows), and trees whose sampled path leaves the best children again and again."""
    rng = np.random.default_rng(int(1000 * keep))
    b, n, vocab = 6, 900, 9000
    tokens, parents = random_trees(rng, b, n, vocab, spine=0.9 if keep > 0.5 else 0.3, kids=5)
    parents[0, :60] = np.arange(-1, 59)                  # a chain of 60 at the root
    z = boosted(logits_of(rng, (b, n + 1, vocab)), tokens, parents, rng, temperature, keep)
    if keep < 0.5:                                       # children of equal mass: any of them may follow
        for q in range(b):
            for j in range(n):
                z[q, parents[q, j] + 1, tokens[q, j]] = np.log(vocab) + 2.0
    else:
        z[0, np.arange(60), tokens[0, :60]] = 40.0       # sure to be followed
    if held == B16:
        z = S.bf16(z)
    for max_len in (64, 3):
        u = rng.random((b, n + 1)).astype(np.float32)
        cnt = check_tree(tokens, parents, np.array([n, n, 5, 0, n, 700]), z, temperature, u, max_len, held)
        assert keep < 0.5 or cnt[0] >= min(60, max_len) or temperature == 0.7


def test_tree_edges():
    """Ends of the random numbers, rows without mass, infinities and NaN, foreign tokens and counts."""
    rng = np.random.default_rng(11)
    vocab, n = 300, 8
    tokens = np.tile(np.array([7, 9, 250, 3, 0, 299, 5, 6]), (10, 1))
    parents = np.tile(np.array([-1, -1, -1, 0, 0, 3, 5, 6]), (10, 1))
    z = logits_of(rng, (10, n + 1, vocab))
    z[:, 0, 7] += 8.0
    z[:, 1, 3] += 8.0
    u = rng.random((10, n + 1)).astype(np.float32)
    u[0], u[1] = 0.0, LAST
    z[2, 0], z[3, 1] = -np.inf, -np.inf                  # no mass at the root, after the first node
    u[3, 1] = 0.0
    z[4, 0, 5:290] = np.nan                              # NaN counts as no mass
    z[5, 0, 10] = np.inf                                 # as the largest number: all of the mass
    z[6, 0], z[6, 0, [7, 9, 250]] = -np.inf, 0.0         # the children hold everything
    tokens[7, :3] = [-1, vocab, 2 ** 31 - 1]             # not in the vocabulary
    parents[8, 0] = 100                                  # no such parent
    num = np.array([8, 8, 8, 8, 8, 8, 8, 8, 8, 1 << 20])
    check_tree(tokens, parents, num, z, 1.0, u, 8)
    check_tree(tokens, parents, num, z, 0.0, u, 8)
    check_tree(tokens, parents, np.full(10, -5), z, 1.0, u, 8)
    u[:, 0] = [0.0, LAST] * 5
    check_tree(tokens, parents, num, z, 1e-3, u, 8)
    check_tree(tokens, parents, num, z, 1e30, u, 8)


def test_tree_edges_along_paths():
    """The same in a budget whose rows are read along paths; parents in any order, also in circles."""
    rng = np.random.default_rng(14)
    vocab, n, budget = 300, 8, 1025
    tokens, parents = rng.integers(0, vocab, (12, budget)), np.full((12, budget), -1)
    tokens[:, :n], parents[:, :n] = [7, 9, 250, 3, 0, 299, 5, 6], [-1, -1, -1, 0, 0, 3, 5, 6]
    z = logits_of(rng, (12, budget + 1, vocab))
    z[:, 0, 7] += 8.0
    z[:, 1, 3] += 8.0
    u = rng.random((12, budget + 1)).astype(np.float32)
    u[0], u[1] = 0.0, LAST
    z[2, 0], z[3, 1] = -np.inf, -np.inf
    u[3, 1] = 0.0
    z[4, 0, 5:290] = np.nan
    z[5, 0, 10] = np.inf
    z[6, 0], z[6, 0, [7, 9, 250]] = -np.inf, 0.0
    tokens[7, :3] = [-1, vocab, 2 ** 31 - 1]
    parents[8, 0] = 100
    parents[9, :n] = [3, 0, 1, -1, 3, 4, 7, 6]           # later parents, and a circle of 6 and 7
    parents[10] = rng.integers(-3, budget + 3, budget)   # circles that the root may reach or not
    parents[10, :3], z[10, 0, tokens[10, 0]] = -1, 9.0
    num = np.array([8, 8, 8, 8, 8, 8, 8, 8, 8, 8, budget, 1])
    for temperature in (1.0, 0.0, 1e-3, 1e30):
        check_tree(tokens, parents, num, z, temperature, u, 8)
    check_tree(tokens, parents, np.full(12, -5), z, 1.0, u, 8)


@pytest.mark.parametrize("budget", [8, 1025])
@pytest.mark.parametrize("offset,temperature", [(1e5, 1e-2), (-3e7, 4.0), (2e30, 1e30), (-3e38, 1e37), (1e30, 1.0), (-1e12, 1e-3)])
def test_large_logits(budget, offset, temperature):
    """Logits far from 0 and wide apart: what counts is their exact difference over the temperature."""
    rng = np.random.default_rng(15)
    vocab, b = 5000, 6
    tokens, parents = random_trees(rng, b, budget, vocab, spine=0.5, kids=4)
    step = np.spacing(np.float32(abs(offset)))             # whole steps of the type, a few temperatures wide
    spread = max(1.0, temperature / step)
    with np.errstate(over="ignore"):                       # some become -inf
        z = (offset + np.round(rng.normal(size=(b, budget + 1, vocab)) * 2.0 * spread) * float(step)).astype(np.float32)
    for q in range(b):
        for j in range(min(budget, 200)):
            z[q, parents[q, j] + 1, tokens[q, j]] = z[q, parents[q, j] + 1].max()
    check_tree(tokens, parents, np.full(b, budget), z, temperature, rng.random((b, budget + 1)).astype(np.float32), 8)
    d, v, n = z[:, :5], z[:, 1:5], np.full(b, 4)
    check_chain(tokens[:, :4], n, d, v, temperature, rng.random((b, 5)).astype(np.float32))


def test_tree_little_mass_left():
    """Children that hold all but 1e-7 .. 1e-14 of the mass, tested with the largest random number."""
    rng = np.random.default_rng(12)
    vocab, n = 9000, 3
    tokens, parents = np.tile(np.array([17, 18, 8999]), (8, 1)), np.full((8, n), -1)
    z = logits_of(rng, (8, n + 1, vocab), 1.0)
    for q in range(8):
        z[q, 0, 17] += 24.0 + q
        z[q, 0, 8999] += 14.0 + q
    u = np.full((8, n + 1), LAST, np.float32)
    u[:, 0] = rng.random(8)
    check_tree(tokens, parents, np.full(8, n), z, 1.0, u, 4)


def test_random_numbers_outside_the_unit_interval_stay_in_range():
    """u at or past 1 or NaN is outside the contract; the result is still one of the row's tokens."""
    rng = np.random.default_rng(13)
    tokens, parents = random_trees(rng, 4, 6, 5000)
    z = logits_of(rng, (4, 7, 5000))
    for value in (1.0, 7.0, np.nan, -1.0):
        acc, cnt, bonus = run_tree(tokens, parents, np.full(4, 6), z, 1.0, np.full((4, 7), value, np.float32), 4)
        assert ((bonus >= 0) & (bonus < 5000)).all() and ((cnt >= 0) & (cnt <= 4)).all()


def run_chain(tokens, num, p, q, temperature, u, held=F32, pad=0, draft=True):
    b, n = tokens.shape
    dev = device()
    cnt, bonus = torch.full((b,), -9, dtype=torch.int32, device=dev), torch.full((b,), -9, dtype=torch.int32, device=dev)
    need = D.verify_chain_workspace_size(b, n, p.shape[2])
    ws = torch.full((need,), 0xFF, dtype=torch.uint8, device=dev)
    say(f"verify_chain b={b} depth={n} V={p.shape[2]} T={temperature} {held} pad={pad}")
    D.verify_chain(i32(tokens), to_dev(p, held, pad), to_dev(q, held, pad) if draft else None, temperature,
                   torch.from_numpy(np.ascontiguousarray(u, np.float32)).to(dev), cnt, bonus, ws,
                   num_tokens=None if num is None else i32(num))
    torch.cuda.synchronize()
    return cnt.cpu().numpy(), bonus.cpu().numpy()


def check_chain(tokens, num, p, q, temperature, u, held=F32, pad=0, draft=True):
    cnt, bonus = run_chain(tokens, num, p, q, temperature, u, held, pad, draft)
    for i in range(len(tokens)):
        n = tokens.shape[1] if num is None else num[i]
        want = S.verify_chain(tokens[i], n, p[i], q[i], temperature, u[i])
        assert (cnt[i], bonus[i]) == want, (i, cnt[i], bonus[i], want)
    return cnt


@pytest.mark.parametrize("held", [F32, B16])
@pytest.mark.parametrize("temperature", [0.0, 0.7, 1.0])
@pytest.mark.parametrize("b,n,vocab,pad", [(1, 1, 1, 0), (4, 1, 10, 2), (5, 3, 97, 1), (3, 16, 4099, 0), (2, 64, 1000, 3),
                                           (3, 5, 50257, 0), (6, 7, 20000, 0)])
def test_chains(held, temperature, b, n, vocab, pad):
    rng = np.random.default_rng(b * 100 + n + vocab)
    q = logits_of(rng, (b, n, vocab))
    q[..., : max(1, vocab // 500)] += 6.0
    p = logits_of(rng, (b, n + 1, vocab))
    p[:, :n] = q + 0.4 * logits_of(rng, (b, n, vocab), 1.0)
    if held == B16:
        p, q = S.bf16(p), S.bf16(q)
    seen = 0
    for trial in range(4):
        tokens = np.array([[rng.choice(vocab, p=S.law(q[i, j], temperature)) for j in range(n)] for i in range(b)])
        u = rng.random((b, n + 1)).astype(np.float32)
        num = None if trial == 0 else rng.integers(0, n + 1, size=b)
        seen += check_chain(tokens, num, p, q, temperature, u, held, pad, draft=not (temperature == 0 and trial == 1)).sum()
    assert seen > 0


def test_chain_edges():
    rng = np.random.default_rng(21)
    vocab, n = 500, 4
    q = logits_of(rng, (9, n, vocab))
    p = logits_of(rng, (9, n + 1, vocab))
    tokens = rng.integers(0, vocab, size=(9, n))
    u = rng.random((9, n + 1)).astype(np.float32)
    p[0, :n] = q[0]                                       # the same law: every token passes
    u[0, 1:] = LAST
    p[1], u[1, 1:] = -np.inf, 0.0                         # no mass in the target
    q[2] = -np.inf                                        # none in the draft: any token of the target's passes
    u[2, 1:] = LAST
    p[3, :, 10:], q[3, :, :10] = -np.inf, -np.inf         # nothing in common
    tokens[3] = 20
    p[4, 0], q[4, 0] = np.nan, np.nan
    p[5, 0, 3], q[5, 1, 4] = np.inf, np.inf
    tokens[6] = [-1, vocab, 3, 4]
    u[7], u[8] = 0.0, LAST
    for num in (None, np.array([4, 4, 0, 9, -2, 4, 1, 3, 4])):
        check_chain(tokens, num, p, q, 1.0, u)
        check_chain(tokens, num, p, q, 0.0, u)
    check_chain(tokens, None, p, q, 0.05, u)


def test_the_first_token_follows_the_target():
    """4096 requests with the same logits and random numbers of their own: the first token's counts are
    within 5 standard deviations of the target's."""
    rng = np.random.default_rng(31)
    b, vocab = 4096, 12
    z = np.broadcast_to(logits_of(rng, (1, 4, vocab), 1.2), (b, 4, vocab)).copy()
    y = np.broadcast_to(logits_of(rng, (1, 1, vocab), 1.2), (b, 1, vocab)).copy()
    tokens, parents = np.tile(np.array([2, 5, 6]), (b, 1)), np.full((b, 3), -1)
    acc, cnt, bonus = run_tree(tokens, parents, np.full(b, 3), z, 1.0, rng.random((b, 4)).astype(np.float32), 1)
    first = np.where(cnt > 0, tokens[np.arange(b), acc[:, 0].clip(0)], bonus)
    drawn = rng.choice(vocab, size=(b, 1), p=S.law(y[0, 0], 1.0))
    n, tok = run_chain(drawn, None, z[:, :2], y, 1.0, rng.random((b, 2)).astype(np.float32))
    chain = np.where(n > 0, drawn[:, 0], tok)
    p = S.law(z[0, 0], 1.0)
    for got in (first, chain):
        count = np.bincount(got, minlength=vocab)
        assert (np.abs(count - b * p) <= 5 * np.sqrt(b * p * (1 - p))).all()
