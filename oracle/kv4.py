"""The 4-bit KV cache and the attention over it (test oracle, float64, element by element from the
definitions).

An element is stood for by level * scale, level one of LEVELS with a sign.  Keys share a power of
two over 32 dims, values a bfloat16 over a head.
"""
import numpy as np

LEVELS = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


def codes(y):
    """Index of the level nearest to |y|, ties to the even index, 7 beyond the last."""
    a = np.abs(np.asarray(y, dtype=np.float64))
    d = np.abs(a[..., None] - LEVELS)
    best = d.min(-1, keepdims=True)
    near = d == best
    even = near & (np.arange(8) % 2 == 0)
    pick = np.where(even.any(-1, keepdims=True), even, near)
    return np.argmax(pick, -1)


def _stood_for(x, scale):
    y = x / scale
    return np.where(np.signbit(y), -1.0, 1.0) * LEVELS[codes(y)] * scale


def key_exponent(amax):
    """Least e with amax <= 7 * 2^e, within [-125, 125]."""
    for e in range(-125, 125):
        if amax <= 7.0 * 2.0 ** e:
            return e
    return 125


def value_scale(amax):
    """Least bfloat16 s >= 2^-126 with amax <= 6 * s."""
    need = max(amax / 6.0, 2.0 ** -126)
    e = int(np.floor(np.log2(need)))
    if 2.0 ** e > need:
        e -= 1
    n = int(np.floor(need / 2.0 ** (e - 7)))
    while 6.0 * n * 2.0 ** (e - 7) < amax:
        n += 1
    return n * 2.0 ** (e - 7)


def quantise_keys(k):
    """What the cache stands for: k [..., hd], blocks of 32 dims."""
    k = np.asarray(k, dtype=np.float64)
    x = k.reshape(-1, 32)
    out = np.empty_like(x)
    for i in range(x.shape[0]):
        if not np.isfinite(x[i]).all():
            out[i] = np.nan
        else:
            out[i] = _stood_for(x[i], 2.0 ** key_exponent(np.abs(x[i]).max()))
    return out.reshape(k.shape)


def quantise_values(v):
    """v [..., hd], one scale for the last axis."""
    v = np.asarray(v, dtype=np.float64)
    x = v.reshape(-1, v.shape[-1])
    out = np.empty_like(x)
    for i in range(x.shape[0]):
        if not np.isfinite(x[i]).all():
            out[i] = np.nan
        else:
            out[i] = _stood_for(x[i], value_scale(np.abs(x[i]).max()))
    return out.reshape(v.shape)


def attend(q, k, v, kb=None, vb=None, *, causal=False, scale=None):
    """One sequence: q [B, H, hd], context keys and values as the cache stands for them
    [T, n, hd], the block's own kb, vb [B, n, hd] or None.  Returns (out [B, H, hd],
    lse [B, H], mass [B, H, hd] = sum p |v|, reach [B, H] = the largest scale * sum |q| |k|)."""
    B, H, hd = q.shape
    q = np.asarray(q, dtype=np.float64)
    scale = hd ** -0.5 if scale is None else scale
    G = H // k.shape[1]
    out, mass = np.zeros((B, H, hd)), np.zeros((B, H, hd))
    lse, reach = np.full((B, H), -np.inf), np.zeros((B, H))
    for b in range(B):
        for h in range(H):
            kk, vv = k[:, h // G], v[:, h // G]
            if kb is not None:
                n = b + 1 if causal else B
                kk = np.concatenate([kk, kb[:n, h // G]])
                vv = np.concatenate([vv, vb[:n, h // G]])
            if kk.shape[0] == 0:
                continue
            x = scale * (kk @ q[b, h])
            m = x.max()
            p = np.exp(x - m)
            lse[b, h] = m + np.log(p.sum())
            p /= p.sum()
            out[b, h], mass[b, h] = p @ vv, p @ np.abs(vv)
            reach[b, h] = (scale * (np.abs(kk) @ np.abs(q[b, h]))).max()
    return out, lse, mass, reach
