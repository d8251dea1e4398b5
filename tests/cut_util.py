"""Sampling under temperature, top-k, top-p and min-p, and acceptance along a tree under the same cuts, in whole numbers on the host, one step
after another as the definition has them."""
import math

import numpy as np

POLY = (1.52527338e-5, 1.54035304e-4, 1.33335581e-3, 9.61812911e-3, 5.55041087e-2, 2.40226507e-1, 6.93147181e-1, 1.0)


def weights(z):
    """Weights of the scores z (float32) of a row.  A fused step p * f + c is formed in 64 bits of significand, where the product of two
    32-bit numbers is exact, and rounded to 32 bits."""
    ok = ~np.isnan(z)
    w = np.zeros(z.shape, dtype=np.int64)
    m = z[ok].max() if ok.any() else np.float32(-np.inf)
    if m == -np.inf:
        return w
    with np.errstate(invalid="ignore", over="ignore"):
        t = (z - m).astype(np.float32) * np.float32(1.44269504088896341)
    t[z == m] = 0
    at = np.nonzero(t >= -64)[0]
    t = t[at]
    n = np.floor(t)
    f = (t - n).astype(np.longdouble)
    p = np.full(t.shape, np.float32(POLY[0]))
    for c in POLY[1:]:
        p = (p.astype(np.longdouble) * f + np.longdouble(np.float32(c))).astype(np.float32)
    w[at] = [int(math.ldexp(float(x), 32 + int(y))) for x, y in zip(p, n)] if len(at) < 2000 else np.ldexp(p.astype(np.float64), 32 + n.astype(np.int32)).astype(np.int64)
    return w


def cut(row, temperature, top_k, top_p, min_p):
    """Weights of what is kept of a row of logits (float32), 0 elsewhere."""
    t = np.float32(temperature)
    if not (t == 0 or 2.0 ** -100 <= t <= 2.0 ** 100) or np.isnan(top_p) or np.isnan(min_p):
        return np.zeros(row.shape, np.int64)
    with np.errstate(over="ignore", invalid="ignore"):
        z = (row if t == 0 else row * (np.float32(1) / t)).astype(np.float32)
    w = weights(z)
    order = sorted(np.nonzero(w)[0].tolist(), key=lambda v: (-float(z[v]), v))
    if t == 0:
        order = order[:1]
    elif top_k > 0:
        order = order[:top_k]
    S = int(w[order].sum())
    P = int(math.floor(min(max(float(np.float32(top_p)), 0.0), 1.0) * 2 ** 30))
    need, run, n = max(1, -(-P * S // 2 ** 30)), 0, 0
    while n < len(order) and run < need:
        run += int(w[order[n]])
        n += 1
    least = math.ceil(min(max(float(np.float32(min_p)), 0.0), 1.0) * 2 ** 32)
    out = np.zeros_like(w)
    for v in order[:n]:
        if w[v] >= least:
            out[v] = w[v]
    return out


def first_beyond(w, target):
    """The first index whose running sum exceeds target; the last one where none does."""
    run = np.cumsum(w)
    return min(int(np.searchsorted(run, target, side="right")), len(w) - 1)


def sample(row, u, *how):
    """(token, logprob, kept)"""
    w = cut(row, *how)
    R = int(w.sum())
    if R == 0:
        return -1, -math.inf, 0
    U = 0 if not u > 0 else 2 ** 48 - 1 if u >= 1 else int(math.floor(u * 2.0 ** 48))
    v = first_beyond(w, U * R >> 48)
    return v, math.log(int(w[v]) / R), int((w > 0).sum())


def _random(seed, step, k):
    full = 2 ** 64 - 1
    z = (seed ^ (step * 0x9E3779B97F4A7C15) ^ (k * 0xBF58476D1CE4E5B9)) & full
    z = ((z ^ (z >> 30)) * 0xBF58476D1CE4E5B9) & full
    z = ((z ^ (z >> 27)) * 0x94D049BB133111EB) & full
    return (z ^ (z >> 31)) >> 40


def accept(logits, how, token, parent, n_ver, seed, step):
    """(result fields, retain)"""
    T, vocab = len(token), logits.shape[1]
    if n_ver == 0:
        return (0, -1, 0, 1, T, 0), list(range(T))
    u, path, draws, n_new = 0, [0], 0, -1
    while True:
        w = cut(logits[u], *how)
        left, tried, nxt = int(w.sum()), set(), -1
        for c in range(T):
            if parent[c] != u or token[c] in tried or not 0 <= token[c] < vocab:
                continue
            r, draws = _random(seed, step, draws), draws + 1
            if r * left < int(w[token[c]]) << 24:
                nxt = c
                break
            tried.add(token[c])
            left -= int(w[token[c]])
            w[token[c]] = 0
        if nxt < 0:
            U = _random(seed, step, draws) << 24 | _random(seed, step, draws + 1)
            x_new = first_beyond(w, U * left >> 48)
            break
        if nxt >= n_ver:
            n_new, x_new = nxt, int(token[nxt])
            break
        u = nxt
        path.append(u)
    below = set()
    for i in range(T):
        if i == n_new or parent[i] in below:
            below.add(i)
    held = sorted(set(path) | below)
    return (len(path), x_new, n_new, int(n_new >= 0), len(held), sum(i < n_ver for i in below)), held
