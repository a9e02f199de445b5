"""Distillation from a teacher's stored top logits (test oracle, float64, a slot at a time).

p is the softmax at temperature T over the teacher's listed tokens and, if given, a bucket of all
others whose log-sum-exp (at T) is `rest`; ids outside the vocabulary or listed before are no
entries.  q = softmax(z / T) of the student.
"""
import numpy as np


def _softmax(x):
    e = np.exp(x - x.max())
    return e / e.sum()


def teacher(ids, values, rest, V, T):
    """(tokens, p over them, p of the bucket); no tokens and None without any finite logit."""
    seen, toks, ls = set(), [], []
    for i, t in zip(ids, values):
        if 0 <= int(i) < V and int(i) not in seen:
            seen.add(int(i))
            toks.append(int(i))
            ls.append(float(t) / T)
    l = np.array(ls + ([] if rest is None else [float(rest)]), dtype=np.float64)
    if l.size == 0 or l.max() == -np.inf:
        return [], None, 0.0
    p = _softmax(l)
    return toks, p[:len(toks)], 0.0 if rest is None else p[-1]


def slot_kl(z, ids, values, rest=None, T=1.0):
    """(kl, dkl/dz)."""
    z = np.asarray(z, dtype=np.float64)
    T = float(np.float32(T))
    toks, p, pr = teacher(ids, values, rest, z.shape[0], T)
    if p is None:
        return 0.0, np.zeros_like(z)
    q = _softmax(z / T)
    lq = (z - z.max()) / T - np.log(np.exp((z - z.max()) / T).sum())
    inside = np.zeros(z.shape[0], dtype=bool)
    inside[toks] = True
    kl = sum(pi * (np.log(pi) - lq[t]) for t, pi in zip(toks, p) if pi > 0)
    g = q.copy()
    if rest is not None and pr > 0:
        out = lq[~inside]
        top = out.max() if out.size else -np.inf
        if top == -np.inf:
            return np.inf, None
        lqr = top + np.log(np.exp(out - top).sum())
        kl += pr * (np.log(pr) - lqr)
        g = np.where(inside, q, q * (1 - pr / np.exp(lqr)))
    for t, pi in zip(toks, p):
        g[t] -= pi
    return kl, g / T


def slot_ce(z, label):
    """(ce, dce/dz); zeros for a label outside the vocabulary."""
    z = np.asarray(z, dtype=np.float64)
    if not 0 <= label < z.shape[0]:
        return 0.0, np.zeros_like(z)
    q = _softmax(z)
    g = q.copy()
    g[label] -= 1
    return float((z.max() - z[label]) + np.log(np.exp(z - z.max()).sum())), g


def distill(student, ids, values, rest, labels, B, T, alpha, g_loss=(0, 0, 0), g_kl=None, g_ce=None):
    """(kl [n, P], ce [n, B-1] or None, loss [3], gradient [n*B, V])."""
    student = np.asarray(student, dtype=np.float64)
    n, P, _ = np.shape(ids)
    V = student.shape[1]
    T = float(np.float32(T))
    alpha = float(np.float32(alpha))
    kl = np.zeros((n, P))
    ce = np.zeros((n, B - 1))
    grad = np.zeros((n * B, V))
    has = 0 if labels is None else int(((np.asarray(labels) >= 0) & (np.asarray(labels) < V)).sum())
    wk = (g_loss[0] + alpha * g_loss[2]) * T * T / (P * n)
    wc = (g_loss[1] + g_loss[2]) / max(has, 1)
    for s in range(n):
        for k in range(1, B):
            z = student[s * B + k]
            if k <= P:
                r = None if rest is None else rest[s][k - 1]
                kl[s, k - 1], g = slot_kl(z, ids[s][k - 1], values[s][k - 1], r, T)
                w = wk + (0 if g_kl is None else g_kl[s][k - 1])
                if g is not None and w != 0:
                    grad[s * B + k] += w * g
            if labels is not None:
                ce[s, k - 1], g = slot_ce(z, int(labels[s][k - 1]))
                grad[s * B + k] += (wc + (0 if g_ce is None else g_ce[s][k - 1])) * g
    l_kl = T * T / P * kl.sum() / n
    l_ce = ce.sum() / max(has, 1)
    return kl, None if labels is None else ce, np.array([l_kl, l_ce, l_ce + alpha * l_kl]), grad
