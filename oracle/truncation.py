"""Truncated distributions of rows of logits, their draws and their verification (test oracle,
float64, a row at a time).

Entries are ordered by logit, largest first, ties to the lowest token; -inf and NaN are masked.
Kept are the first min(n_k, n_p, n_m) of the order: top_k; the fewest whose weights sum to top_p of
the first n_k entries' sum; those with a weight of min_p at least, weights relative to the greatest.
"""
import numpy as np


def order(z):
    """Tokens of a row's unmasked entries in order."""
    z = np.asarray(z, dtype=np.float64)
    live = np.flatnonzero(z > -np.inf)      # False for NaN too
    return live[np.argsort(-z[live], kind="stable")]


def truncate(z, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0):
    """(n, cut_logit, cut_index, lse, p): p is the truncated distribution [V]."""
    z = np.asarray(z, dtype=np.float64)
    T, top_p, min_p = (float(np.float32(x)) for x in (temperature, top_p, min_p))
    o = order(z)
    p = np.zeros(z.shape[0])
    if o.size == 0:
        return 0, -np.inf, -1, -np.inf, p
    if not T > 0:
        n, lse = 1, 0.0
        p[o[0]] = 1.0
    else:
        w = np.exp((z[o] - z[o[0]]) / T)
        n = o.size if top_k <= 0 else min(int(top_k), o.size)
        if top_p < 1:
            cs = np.cumsum(w[:n])
            n = min(n, 1 + int(np.count_nonzero(cs < top_p * cs[-1])))
        if min_p > 0:
            n = min(n, int(np.count_nonzero(w >= min(min_p, 1.0))))
        s = w[:n].sum()
        lse = z[o[0]] / T + np.log(s)
        p[o[:n]] = w[:n] / s
    if n == o.size:
        return n, -np.inf, -1, lse, p
    return n, z[o[n - 1]], int(o[n - 1]), lse, p


def inverse(p, u):
    """Lowest token whose running sum of p, in token order, exceeds u times the whole; the last
    with a weight where rounding leaves none, -1 without any."""
    live = np.flatnonzero(p > 0)
    if live.size == 0:
        return -1
    cs = np.cumsum(p)
    at = int(np.searchsorted(cs, min(max(float(u), 0.0), 1.0) * cs[-1], side="right"))
    return min(at, int(live[-1]))


def accept(draft, q, p, u):
    """Verification of K drafts under draft distributions q [K][V] and target distributions
    p [K+1][V] with uniforms u [K+1]: (accepted, next token, committed tokens)."""
    K = len(draft)
    V = p.shape[1]
    n = 0
    while n < K:
        x = int(draft[n])
        if not (0 <= x < V and float(u[n]) * q[n][x] < p[n][x]):
            break
        n += 1
    w = p[n]
    if n < K:
        r = np.maximum(p[n] - q[n], 0.0)
        w = r if r.sum() > 0 else w
    t = inverse(w, u[K])
    return n, t, [int(x) for x in draft[:n]] + [t]


def top_logits(z, K, temperature=1.0):
    """(ids [K], values [K], rest): -1 and -inf past the unmasked entries."""
    z = np.asarray(z, dtype=np.float64)
    o = order(z)
    ids = np.full(K, -1)
    values = np.full(K, -np.inf)
    n = min(K, o.size)
    ids[:n], values[:n] = o[:n], z[o[:n]]
    left = z[o[n:]] / float(np.float32(temperature))
    rest = -np.inf
    if left.size:
        rest = left[0] + np.log(np.exp(left - left[0]).sum())
    return ids, values, rest
