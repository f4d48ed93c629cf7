"""Paged caches and draft verification in plain fp64 numpy, one request after another.

Formats: a row x of one KV head in E4M3 pages is a scale s = max|x| / 448 and codes nearest to
x / s on the grid of 1 + 4 + 3 bits (smallest exponent 2^-6, steps of 2^-9 below it).
"""
import numpy as np


def turned(x, turn, theta):
    """Rows x [T, heads, d] turned by turn [T] positions: channel i pairs with i + d/2."""
    h = x.shape[-1] // 2
    a = np.asarray(turn, np.float64)[:, None] * theta ** (-np.arange(h) / h)
    c, s = np.cos(a)[:, None], np.sin(a)[:, None]
    lo, hi = x[..., :h], x[..., h:]
    return np.concatenate([lo * c - hi * s, lo * s + hi * c], -1)


def e4m3(y):
    """The nearest E4M3 value (ties to even), clamped to +-448."""
    y = np.clip(np.asarray(y, np.float64), -448, 448)
    step = 2.0 ** (np.floor(np.log2(np.maximum(np.abs(y), 2.0 ** -6))) - 3)
    return np.round(y / step) * step


def quantised(x):
    """(codes as values, scales) of rows x [..., d]."""
    top = np.abs(x).max(-1)
    with np.errstate(invalid="ignore"):
        scale = np.where(np.isfinite(top), np.where(top < 2.0 ** -100, 0.0, top / 448), np.nan)
        y = np.where(scale[..., None] > 0, x / np.where(scale > 0, scale, 1.0)[..., None], 0.0)
    return e4m3(y), scale


def page_of(table, r, row, size):
    return int(table[r, row // size]), row % size


def rows_of(pages, table, r, lo, hi, size):
    """Rows lo .. hi of request r of pages [n, Hkv, size, d]."""
    return np.stack([pages[table[r, j // size], :, j % size] for j in range(lo, hi)]) if hi > lo else \
        np.zeros((0, pages.shape[1], pages.shape[3]))


def attend(q, keys, values, n_keys, window=0):
    """q [n, Hq, d] (turned): the last n of n_keys rows; keys, values [n_keys, Hkv, d].  out, lse [Hq, n]."""
    n, hq, d = q.shape
    g = hq // keys.shape[1]
    out, lse = np.zeros((n, hq, d)), np.full((hq, n), -np.inf)
    for t in range(n):
        i = n_keys - n + t
        lo = max(0, i + 1 - window) if window else 0
        if i < lo:
            continue
        for h in range(hq):
            s = keys[lo:i + 1, h // g] @ q[t, h] / np.sqrt(d)
            m = s.max()
            w = np.exp(s - m)
            out[t, h] = w @ values[lo:i + 1, h // g] / w.sum()
            lse[h, t] = m + np.log(w.sum())
    return out, lse


def verify(ptr, tokens, p, q, u_accept, u_next):
    """(accepted, next token) of each request; fp32 arrays, the product rounded to fp32, the weights
    whole multiples of 2^-44."""
    got = []
    for r in range(len(ptr) - 1):
        lo, n = ptr[r], ptr[r + 1] - ptr[r]
        a = 0
        while a < n:
            x = int(tokens[lo + a])
            if not 0 <= x < p.shape[1]:
                break
            qx = np.float32(1) if q is None else q[lo + a, x]
            if not np.float32(u_accept[lo + a]) * qx < p[lo + r + a, x]:
                break
            a += 1
        whole = lambda w: (np.clip(np.nan_to_num(w, nan=0.0, posinf=2.0), 0, 1).astype(np.float64) * 2.0 ** 44).astype(np.int64)  # noqa: E731
        base = p[lo + r + a]
        left = base.copy()
        if a < n:
            if q is not None:
                left = base - q[lo + a]
            elif 0 <= tokens[lo + a] < p.shape[1]:
                left[tokens[lo + a]] = 0
        w = whole(left)
        if not w.any():
            w = whole(base)
        total = int(w.sum())
        k = min(max(int(float(u_next[r]) * 2 ** 24), 0), 2 ** 24 - 1)
        goal = total * k >> 24
        got.append((a, int(np.searchsorted(np.cumsum(w), goal, side="right")) if total else -1))
    return got
