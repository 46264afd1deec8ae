"""Oracle of caches and weights in 8 bits, fp64 numpy: e4m3 values times a power of two per block."""

import numpy as np

from .paged import rotate

LARGEST, LOWEST, HIGHEST = 448.0, 27, 247  # largest e4m3; scale bytes


def e4m3(x):
    """Nearest e4m3 value: 4 significant bits, multiples of 2^-9 at least, even on ties."""
    x = np.asarray(x, dtype=np.float64)
    step = 2.0 ** (np.maximum(np.frexp(x)[1], -5) - 4)
    return np.where(np.isfinite(x), np.round(x / step) * step, np.nan)


def scale_byte(amax):
    """Biased exponent of the smallest power of two, 2^-100 at least, with amax <= 448 times it."""
    m, e = np.frexp(np.asarray(amax, dtype=np.float64) / LARGEST)
    return np.where(amax > 0, np.clip(e - (m == 0.5) + 127, LOWEST, HIGHEST), LOWEST).astype(np.int64)


def scale_value(byte):
    return 2.0 ** (np.asarray(byte, dtype=np.float64) - 127)


def magnitude(x):
    """What counts for a scale: finite magnitudes."""
    return np.where(np.isfinite(x), np.abs(x), 0.0)


def quantize8(w):
    """w [K, N] as (values [KP, N], bytes [KP / 128, ceil(N / 128)]): scaled e4m3 values, K padded to a multiple of 128."""
    K, N = w.shape
    p = np.pad(w, ((0, -K % 128), (0, -N % 128)))
    b = p.reshape(p.shape[0] // 128, 128, -1, 128)
    byte = scale_byte(magnitude(b).max((1, 3)))
    return e4m3(b / scale_value(byte)[:, None, :, None]).reshape(p.shape)[:, :N], byte


def dequantize8(values, byte):
    s = scale_value(byte).repeat(128, 0).repeat(128, 1)
    return values * s[:, :values.shape[1]]


def quantize_rows8(x):
    """x [M, K] with each row's blocks of 128 taken to 8 bits: the values they stand for."""
    M, K = x.shape
    b = np.pad(x, ((0, 0), (0, -K % 128))).reshape(M, -1, 128)
    s = scale_value(scale_byte(magnitude(b).max(2)))[..., None]
    return (e4m3(b / s) * s).reshape(M, -1)[:, :K]


def linear8(x, values, byte):
    """Returns (y, size): the product and the same sums over magnitudes (what the accumulation's rounding can move)."""
    q, w = quantize_rows8(x), dequantize8(values, byte)[:x.shape[1]]
    return q @ w, np.abs(q) @ np.abs(w)


def paged_append8(q, k, v, pools, page_table, start, n_new=None, pos0=None, theta=500000.0, q_out=None, lens=None):
    """pools: (k values, v values [pages, page_size, Hkv, D], k bytes, v bytes [pages, blocks, Hkv]), scaled e4m3 values.
    Rows of a block before the call's keep their values, with lens also those behind them up to lens[b].
    Returns (q_out, pools, exact): exact are the keys' and values' pools before rounding, NaN where nothing was written."""
    B, T = k.shape[:2]
    pools = [p.copy() for p in pools]
    exact = [np.full(p.shape, np.nan) for p in pools[:2]]
    out = None if q is None else np.zeros_like(q) if q_out is None else q_out.copy()
    pages, ps = pools[0].shape[:2]
    sb = ps // pools[2].shape[1]
    for b in range(B):
        n = T if n_new is None else min(max(int(n_new[b]), 0), T)
        first = int(start[b])
        pos = np.arange(n) + (first if pos0 is None else int(pos0[b]))
        if q is not None:
            out[b, :n] = rotate(q[b, :n], pos, theta)
        rows = rotate(k[b, :n], pos, theta), v[b, :n]
        for block in range(first // sb, -(-(first + n) // sb)) if n else ():
            s = block * sb
            page = int(page_table[b, s // ps]) if 0 <= s < page_table.shape[1] * ps else -1
            if not 0 <= page < pages:
                continue
            lo, hi = max(s, first), min(s + sb, first + n)
            at = slice(lo - s + s % ps, hi - s + s % ps)
            before = slice(s % ps, lo - s + s % ps)
            for i in (0, 1):
                x = rows[i][lo - first:hi - first]
                byte = scale_byte(magnitude(x).max((0, 2)))
                old = np.clip(pools[2 + i][page, s % ps // sb], LOWEST, HIGHEST)
                kept = [before] if lo > s else []
                if lens is not None:
                    end = min(max(int(lens[b]), 0), page_table.shape[1] * ps, s + sb)  # of what the block holds
                    if end > hi:
                        kept.append(slice(at.stop, at.stop + end - hi))
                if kept:
                    byte = np.maximum(byte, old)
                for rows_kept in kept:
                    x8 = pools[i][page, rows_kept]
                    pools[i][page, rows_kept] = np.where((byte > old)[:, None], e4m3(x8 * scale_value(old - byte + 127)[:, None]), x8)
                pools[2 + i][page, s % ps // sb] = byte
                pools[i][page, at] = e4m3(x / scale_value(byte)[:, None])
                exact[i][page, at] = x
    return out, pools, exact


def paged_values(values, byte):
    """What a pool's values stand for."""
    return values * scale_value(byte).repeat(values.shape[1] // byte.shape[1], 1)[..., None]
