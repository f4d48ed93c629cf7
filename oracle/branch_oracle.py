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
