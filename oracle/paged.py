"""Oracle of the paged key-value cache, fp64 numpy: appending rotated keys, and attention over the cached keys."""

import numpy as np


def rotate(x, pos, theta):
    """x [..., heads, D] at positions pos [...]: pairs (d, d + D/2) turned by pos * theta^(-2d/D)."""
    if theta == 0:
        return np.array(x, dtype=np.float64)
    half = x.shape[-1] // 2
    angle = np.asarray(pos, dtype=np.float64)[..., None] * theta ** (-np.arange(half) / half)
    cos, sin = np.cos(angle)[..., None, :], np.sin(angle)[..., None, :]
    a, b = x[..., :half], x[..., half:]
    return np.concatenate([a * cos - b * sin, b * cos + a * sin], -1)


def paged_append(q, k, v, k_pages, v_pages, page_table, start, n_new=None, pos0=None, theta=500000.0, q_out=None):
    """Returns (q_out, k_pages, v_pages) after the call; pools [pages, page_size, Hkv, D].  Tokens that have no
    place in the pool are skipped."""
    B, T = k.shape[:2]
    k_pages, v_pages = k_pages.copy(), v_pages.copy()
    out = None if q is None else np.zeros_like(q) if q_out is None else q_out.copy()
    pages, ps = k_pages.shape[:2]
    for b in range(B):
        n = T if n_new is None else min(max(int(n_new[b]), 0), T)
        for t in range(n):
            pos = int(start[b] if pos0 is None else pos0[b]) + t
            if q is not None:
                out[b, t] = rotate(q[b, t], pos, theta)
            s = int(start[b]) + t
            if not 0 <= s < page_table.shape[1] * ps:
                continue
            page = int(page_table[b, s // ps])
            if 0 <= page < pages:
                k_pages[page, s % ps] = rotate(k[b, t], pos, theta)
                v_pages[page, s % ps] = v[b, t]
    return out, k_pages, v_pages


def paged_attention(q, k_pages, v_pages, page_table, lens, causal=False, scale=None, n_new=None):
    """Returns (out, weight) [B, T, Hq, D]: the attention and the same sums over |v| (what rounding the weights can move)."""
    B, T, Hq, D = q.shape
    pages, ps, Hkv = k_pages.shape[:3]
    scale = D ** -0.5 if scale is None else scale
    out, weight = np.zeros(q.shape), np.zeros(q.shape)
    for b in range(B):
        n = min(max(int(lens[b]), 0), page_table.shape[1] * ps)
        new = T if n_new is None else min(max(int(n_new[b]), 0), T)
        s = np.arange(n)
        page = page_table[b, s // ps]
        good = (page >= 0) & (page < pages)
        s, page = s[good], page[good]
        k, v = k_pages[page, s % ps], v_pages[page, s % ps]
        for t in range(new):
            seen = s < n - new + t + 1 if causal else np.ones(len(s), bool)
            if not seen.any():
                continue
            for h in range(Hq):
                g = h // (Hq // Hkv)
                x = scale * (k[seen, g] @ q[b, t, h])
                w = np.exp(x - x.max())
                w /= w.sum()
                out[b, t, h] = w @ v[seen, g]
                weight[b, t, h] = w @ np.abs(v[seen, g])
    return out, weight
