"""Plain NumPy forms, in 64 bits, of the serving operators: the paged cache, the
attention over it and the verification from given random numbers.  Written from
the definitions; nothing here is shared with the GPU path."""
from __future__ import annotations

import numpy as np

EXP_LOW = -100


def bf16(x):
    """Nearest bf16 (ties to even) of finite values, as float32."""
    u = np.ascontiguousarray(x, np.float32).view(np.uint32).astype(np.uint64)
    u = (u + 0x7FFF + ((u >> np.uint64(16)) & np.uint64(1))) & np.uint64(0xFFFF0000)
    return u.astype(np.uint32).view(np.float32)


def e4m3_values():
    """The 256 values of OCP e4m3 (NaN at 0x7F and 0xFF)."""
    out = np.zeros(256)
    for b in range(256):
        exp, man = (b >> 3) & 15, b & 7
        v = man * 2.0 ** -9 if exp == 0 else (1 + man / 8) * 2.0 ** (exp - 7)
        out[b] = -v if b & 128 else v
    out[0x7F] = out[0xFF] = np.nan
    return out


def row_exponent(x):
    """Least e >= EXP_LOW with max |x| <= 448 * 2^e, of rows in the last axis."""
    top = np.abs(x.astype(np.float64)).max(axis=-1)
    e = np.full(top.shape, EXP_LOW)
    some = top > 0
    m, k = np.frexp(top[some])            # top = m 2^k, m in [0.5, 1); 448 = 0.875 * 2^9
    e[some] = np.maximum(np.where(m > 0.875, k - 8, k - 9), EXP_LOW)
    return e


def e4m3_round(x):
    """Nearest e4m3 value (ties to even) of |x| <= 448, in float64."""
    x = x.astype(np.float64)
    step = 2.0 ** (np.floor(np.log2(np.maximum(np.abs(x), 2.0 ** -6))) - 3)
    return np.round(x / step) * step


def quantise(x):
    """(values held / 2^e, e) of rows of 128."""
    e = row_exponent(x)
    return e4m3_round(x.astype(np.float64) * 2.0 ** -e[..., None].astype(np.float64)), e


def slot(table_row, page, num_pages, pos):
    """(page, slot) of a position, or None."""
    if pos < 0 or pos // page >= len(table_row):
        return None
    p = int(table_row[pos // page])
    return (p, pos % page) if 0 <= p < num_pages else None


def attention(q, keys, values, see, scale):
    """softmax(scale q k) v over the seen keys; q [n][d], keys [m][d], see [n][m]; rows that see nothing are 0."""
    s = (q @ keys.T) * scale
    s = np.where(see, s, -np.inf)
    top = s.max(axis=1, keepdims=True) if s.shape[1] else np.full((len(q), 1), -np.inf)
    p = np.exp(s - np.where(np.isfinite(top), top, 0.0))
    p = np.where(see, p, 0.0)
    total = p.sum(axis=1, keepdims=True)
    used = np.where(see.any(axis=0)[:, None], values, 0.0)     # a key that no row sees counts for nothing
    return np.where(total > 0, (p @ used) / np.where(total > 0, total, 1.0), 0.0)


def law(z, temperature):
    """Probabilities of a row of logits (None: no mass)."""
    z = np.asarray(z, np.float64)
    z = np.where(np.isnan(z), -np.inf, np.minimum(z, np.float64(np.finfo(np.float32).max)))
    if not np.any(z > -np.inf):
        return None
    if temperature == 0:
        p = np.zeros(len(z))
        p[int(np.argmax(z))] = 1.0
        return p
    w = np.exp((z - z.max()) / np.float64(np.float32(temperature)))
    return w / w.sum()


def sample(rest, p, u):
    """First index whose cumulated mass exceeds u of the whole; of p where rest holds nothing."""
    if p is None:
        return -1
    w = rest if rest.sum() > 0 else p
    cum = np.cumsum(w)
    past = np.nonzero(cum > np.float64(np.float32(u)) * cum[-1])[0]
    past = past[w[past] > 0]
    return int(past[0]) if len(past) else int(np.nonzero(w > 0)[0][-1])


def verify_tree(tokens, parents, n, logits, temperature, uniforms, max_len):
    """(accepted nodes, final token) of one request."""
    vocab = logits.shape[1]
    path, at, tested = [], -1, []
    n = min(max(int(n), 0), len(tokens))
    while True:
        p = law(logits[at + 1], temperature)
        tested = []
        nxt = None
        if len(path) < min(max_len, n):
            taken = 0.0
            for j in range(n):
                if parents[j] != at:
                    continue
                t = int(tokens[j])
                share = p[t] if p is not None and 0 <= t < vocab else 0.0
                tested.append(t)
                if np.float64(uniforms[j + 1]) * (1.0 - taken) < share:
                    nxt = j
                    break
                taken += share
        if nxt is None:
            break
        path.append(nxt)
        at = nxt
    if p is None:
        return path, -1
    rest = p.copy()
    rest[[t for t in tested if 0 <= t < vocab]] = 0.0
    return path, sample(rest, p, uniforms[0])


def verify_chain(tokens, n, target, draft, temperature, uniforms):
    """(accepted tokens, final token) of one request."""
    vocab = target.shape[1]
    n = min(max(int(n), 0), len(tokens))
    for i in range(n):
        p = law(target[i], temperature)
        t = int(tokens[i])
        px = p[t] if p is not None and 0 <= t < vocab else 0.0
        if temperature == 0:
            if px > 0:
                continue
            return i, sample(p if p is not None else None, p, uniforms[0])
        q = law(draft[i], temperature)
        qx = q[t] if q is not None and 0 <= t < vocab else 0.0
        if np.float64(uniforms[i + 1]) * qx < px:
            continue
        if p is None:
            return i, -1
        return i, sample(np.maximum(p - (q if q is not None else 0.0), 0.0), p, uniforms[0])
    p = law(target[n], temperature)
    return n, sample(p, p, uniforms[0])
