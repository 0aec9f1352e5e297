"""numpy restatement of the paged cache, the rotation and the attention over it, in 64 bits; shares no code with the library.

A cache is [pages, heads, page_size, head_dim]; starts[b] .. starts[b + 1] - 1 are the rows of sequence b, whose last one is at
position lengths[b] - 1.
"""
import numpy as np


def positions(lengths, starts):
    """Per row: (sequence, position); rows of nobody have sequence -1."""
    rows = []
    for b, (s, e) in enumerate(zip(starts[:-1], starts[1:])):
        rows += [(t, b, lengths[b] - (e - t)) for t in range(s, e)]
    return rows


def rotate(x, position, inv_freq, interleaved):
    """x [heads, head_dim] in float64 -> rotated."""
    y = x.copy()
    half = len(inv_freq)
    if half == 0:
        return y
    angle = position * np.asarray(inv_freq, np.float64)
    i = 2 * np.arange(half) if interleaved else np.arange(half)
    j = i + 1 if interleaved else i + half
    y[:, i] = x[:, i] * np.cos(angle) - x[:, j] * np.sin(angle)
    y[:, j] = x[:, j] * np.cos(angle) + x[:, i] * np.sin(angle)
    return y


def attention(q, k_cache, v_cache, table, lengths, starts, scale, window=0, k_scale=None, v_scale=None):
    """q [T, q_heads, head_dim] -> (out, spread, small, mass, keys), float64.  `spread` is sum_j w_j |v_j|, `small` sum_j |v_j|,
    `mass` the largest sum_d |q_d k_d| * scale of a row, `keys` how many it sees: what bounds on rounding errors are made of."""
    T, Hq, D = q.shape
    Hkv, P = k_cache.shape[1], k_cache.shape[2]
    out = np.zeros((T, Hq, D))
    spread, small, mass, keys = np.zeros((T, Hq, D)), np.zeros((T, Hq, D)), np.zeros((T, Hq, 1)), np.zeros((T, 1, 1))
    for t, b, p in positions(lengths, starts):
        first = max(0, p - window + 1) if window else 0
        if p < 0:
            continue
        at = np.arange(first, p + 1)
        pages = table[b][at // P]
        keys[t] = len(at)
        for h in range(Hkv):
            k = k_cache[pages, h, at % P].astype(np.float64) * (1.0 if k_scale is None else float(k_scale[h]))
            v = v_cache[pages, h, at % P].astype(np.float64) * (1.0 if v_scale is None else float(v_scale[h]))
            g = Hq // Hkv
            rows = q[t, h * g:(h + 1) * g].astype(np.float64)
            with np.errstate(invalid="ignore", over="ignore"):
                s = rows @ k.T * scale
                w = np.exp(s - s.max(-1, keepdims=True))
                w /= w.sum(-1, keepdims=True)
                out[t, h * g:(h + 1) * g] = w @ v
                spread[t, h * g:(h + 1) * g] = w @ np.abs(v)
                small[t, h * g:(h + 1) * g] = np.abs(v).sum(0)
                mass[t, h * g:(h + 1) * g, 0] = (np.abs(rows) @ np.abs(k).T).max(-1) * abs(scale)
    return out, spread, small, mass, keys
