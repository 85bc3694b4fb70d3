"""Rotary positions, a paged cache and attention over it, in float64 numpy, one row and one position at a time.  Test infrastructure only."""
import numpy as np


def frequencies(rotary_dim, theta=10000.0, scaling="none", factor=1.0, low=1.0, high=2.0, original=1.0, factors=None):
    """Radians a position of each pair."""
    f = np.array([float(theta) ** (-2.0 * i / rotary_dim) for i in range(rotary_dim // 2)])
    if factors is not None:
        f = f / np.asarray(factors, np.float64)
    if scaling == "none":
        return f
    if scaling == "linear":
        return f / factor
    t = original * f / (2 * np.pi)
    r = (t - low) / (high - low) if scaling == "ramp" else (np.log(t) - np.log(low)) / (np.log(high) - np.log(low))
    r = np.minimum(1.0, np.maximum(0.0, r))
    return f * (r + (1.0 - r) / factor)


def turned(x, positions, freq, magnitude=1.0, interleaved=False, inverse=False):
    """x [rows, heads, dim] turned by positions [rows]."""
    x = np.asarray(x, np.float64)
    n = len(freq)
    a, b = (slice(0, 2 * n, 2), slice(1, 2 * n, 2)) if interleaved else (slice(0, n), slice(n, 2 * n))
    out = x.copy()
    for r, p in enumerate(positions):
        t = float(p) * freq * (-1.0 if inverse else 1.0)
        c, s = magnitude * np.cos(t), magnitude * np.sin(t)
        for h in range(x.shape[1]):
            u, w = x[r, h, a], x[r, h, b]
            out[r, h, a], out[r, h, b] = u * c - w * s, u * s + w * c
    return out


def place(page_table, n_pages, page_size, seq, position):
    """(page, slot) of a position; None: no place."""
    at = position // page_size
    if position < 0 or at >= page_table.shape[1]:
        return None
    page = int(page_table[seq, at])
    return (page, position % page_size) if 0 <= page < n_pages else None


def key_at(k_pages, page, head, slot):
    """k_pages [n_pages, heads, dim / G, page_size, G]"""
    return k_pages[page, head, :, slot, :].reshape(-1)


def value_at(v_pages, page, head, slot):
    """v_pages [n_pages, heads, page_size / G, dim, G]"""
    G = v_pages.shape[-1]
    return v_pages[page, head, slot // G, :, slot % G]


def attention(q, k_pages, v_pages, page_table, lens, row_start, scale, window=0, seen=None, k_scale=None, v_scale=None):
    """out, lse, and what bounds their roundings: the largest sum |q k| scale of a row's scores, sum p |v| of each element, the scores seen."""
    rows, heads, dim = q.shape
    n_pages, kv_heads, _, page_size, _ = k_pages.shape
    out, lse = np.zeros((rows, heads, dim)), np.full((rows, heads), -np.inf)
    work, spread, count = np.zeros((rows, heads)), np.zeros((rows, heads, dim)), np.zeros(rows, int)
    capacity = page_table.shape[1] * page_size
    for s in range(len(lens)):
        first, last = row_start[s], row_start[s + 1]
        n, old = last - first, min(max(int(lens[s]), 0), capacity)
        places = {p: place(page_table, n_pages, page_size, s, p) for p in range(old + n)}
        for i in range(n):
            if seen is not None:
                sees = list(range(old)) + [old + j for j in range(min(n, 64)) if int(seen[first + i]) >> j & 1]
            else:
                sees = list(range(max(0, old + i - window + 1) if window else 0, old + i + 1))
            sees = [places[p] for p in sees if places[p] is not None]
            count[first + i] = len(sees)
            if not sees:
                continue
            for g in range(kv_heads):
                k = np.stack([key_at(k_pages, p, g, t) for p, t in sees]).astype(np.float64) * (1.0 if k_scale is None else float(k_scale[g]))
                v = np.stack([value_at(v_pages, p, g, t) for p, t in sees]).astype(np.float64) * (1.0 if v_scale is None else float(v_scale[g]))
                for h in range(g * (heads // kv_heads), (g + 1) * (heads // kv_heads)):
                    x = q[first + i, h].astype(np.float64)
                    z = k @ x * scale
                    top = z.max()
                    if top == -np.inf:
                        continue
                    e = np.exp(z - top)
                    out[first + i, h] = e / e.sum() @ v
                    lse[first + i, h] = top + np.log(e.sum())
                    work[first + i, h] = (np.abs(k) @ np.abs(x)).max() * abs(scale)
                    spread[first + i, h] = e / e.sum() @ np.abs(v)
    return out, lse, work, spread, count
