"""Generation that branches, in plain numpy, one request after another: attention of trees of tokens, the walk
down a tree, rows moved together, the choice among beams and the reordering of their pages.

A tree is its nodes' parents, before their children, -1 for a root."""
import numpy as np


def way(parent, i, window=0):
    """Node i and those above it that it sees (at most `window`), and its depth."""
    path = [i]
    while parent[path[-1]] >= 0:
        path.append(parent[path[-1]])
    return path[:window] if window else path, len(path) - 1


def sees(parent, n_keys, window=0):
    """[n, n_keys]: which rows each node sees."""
    n = len(parent)
    x = n_keys - n
    got = np.zeros((n, n_keys), bool)
    for i in range(n):
        path, depth = way(parent, i, window)
        got[i, max(0, x + depth - window + 1) if window else 0:x] = True
        got[i, [x + j for j in path]] = True
    return got


def attend_tree(q, keys, values, parent, window=0, there=None):
    """q [n, Hq, d] (turned), the last rows of keys, values [n_keys, Hkv, d]; `there` [n_keys]: rows of a page that
    is one.  out, lse [Hq, n]."""
    n, hq, d = q.shape
    g = hq // keys.shape[1]
    out, lse = np.zeros((n, hq, d)), np.full((hq, n), -np.inf)
    seen = sees(parent, len(keys), window)
    if there is not None:
        seen &= there
    for t in range(n):
        at = seen[t].nonzero()[0]
        if not len(at):
            continue
        for h in range(hq):
            s = keys[at, h // g] @ q[t, h] / np.sqrt(d)
            m = s.max()
            w = np.exp(s - m)
            out[t, h] = w @ values[at, h // g] / w.sum()
            lse[h, t] = m + np.log(w.sum())
    return out, lse


def drawn(p, u):
    """The token of a row of fp32 probabilities by u: weights are whole multiples of 2^-44; -1 without weight."""
    w = (np.clip(np.nan_to_num(p, nan=0.0, posinf=2.0), 0, 1).astype(np.float64) * 2.0 ** 44).astype(np.int64)
    total = int(w.sum())
    k = min(max(int(float(np.nan_to_num(u, nan=0.0)) * 2 ** 24), 0), 2 ** 24 - 1)
    return int(np.searchsorted(np.cumsum(w), total * k >> 24, side="right")) if total else -1


def walk(parent, tokens, p, u):
    """(path from node 0, next token) down a tree; parents that are not before their children are no parents."""
    if not len(parent):
        return [], -1
    path = [0]
    while True:
        x = drawn(p[path[-1]], u[path[-1]])
        child = [i for i in range(path[-1] + 1, len(parent)) if parent[i] == path[-1] and tokens[i] == x]
        if x < 0 or not child:
            return path, x
        path.append(child[0])


def keep(pages, table, start, path, size):
    """Rows start + path[i] of pages [n, Hkv, size, ..] become rows start + i, in place."""
    old = pages.copy()
    for i, j in enumerate(path):
        a, b = start + j, start + i
        pages[table[b // size], :, b % size] = old[table[a // size], :, a % size]


def select(x, norm, score, done, end_token, best):
    """x [W, V], norm [W] or None, score [W], done [W] or None: the best (score, beam, token), the first of equals."""
    got = []
    for w in range(len(score)):
        if done is not None and done[w]:
            rows = [(score[w], w, end_token)]
        else:
            with np.errstate(invalid="ignore", over="ignore"):
                y = x[w].astype(np.float32)
                y = np.float32(score[w]) + (y - np.float32(norm[w]) if norm is not None else y)
            y = np.where(np.isnan(y), np.float32(-np.inf), y)
            rows = [(y[v], w, int(v)) for v in np.argsort(-y, kind="stable")[:best]]
        got += [r for r in rows if r[0] > -np.inf]
    return sorted(got, key=lambda r: (-r[0], r[1], r[2]))[:best]


def reorder(tables, parent, n_rows, size):
    """A request's tables [W, width] after a choice, and the copies (from page, to page, rows) that it takes."""
    width = len(parent)
    of = [p if p >= 0 else w for w, p in enumerate(parent)]
    free = [w for w in range(width) if w not in of]
    full, part = divmod(n_rows, size)
    out, copies = tables.copy(), []
    for w, p in enumerate(of):
        out[w, :full] = tables[p, :full]
        if part:
            to = p if of.index(p) == w else free.pop(0)
            out[w, full] = tables[to, full]
            if to != p:
                copies.append((int(tables[p, full]), int(tables[to, full]), part))
    return out, copies
