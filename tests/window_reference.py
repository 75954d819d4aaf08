"""Float64 references of the paged window: rows with their rotary positions, and attention over a window."""
import numpy as np


def rotate(x, positions, frequencies, interleaved):
    """x [n, heads, d] float64 by positions [n]."""
    x, half = x.copy(), len(frequencies)
    angle = np.asarray(positions, dtype=np.float64)[:, None, None] * frequencies
    first = np.arange(half) * 2 if interleaved else np.arange(half)
    second = first + (1 if interleaved else half)
    a, b = x[..., first], x[..., second]
    x[..., first], x[..., second] = a * np.cos(angle) - b * np.sin(angle), b * np.cos(angle) + a * np.sin(angle)
    return x


def rows_of(pool, table, page_tokens, b, n):
    """(K, V) [n, kv heads, d] of the first n tokens of sequence b; pool [page, kv head, 2, token, d]."""
    t = np.arange(n)
    rows = pool[table[b, t // page_tokens], :, :, t % page_tokens]
    return rows[:, :, 0], rows[:, :, 1]


def attention(q, K, V, scale):
    """q [n_q, Hq, d] causal over K, V [n, Hkv, d]: (out, lse [n_q, Hq]); a query that sees nothing gives zeros and -inf."""
    n_q, hq, d = q.shape
    n, hkv = K.shape[:2]
    out, lse = np.zeros_like(q), np.full((n_q, hq), -np.inf)
    for j in range(n_q):
        seen = n - (n_q - 1 - j)
        if seen <= 0:
            continue
        for h in range(hq):
            e = K[:seen, h // (hq // hkv)] @ q[j, h] * scale
            w = np.exp(e - e.max())
            out[j, h] = w @ V[:seen, h // (hq // hkv)] / w.sum()
            lse[j, h] = e.max() + np.log(w.sum())
    return out, lse
