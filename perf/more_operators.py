"""Timed cases of generation that branches: drafted tokens as a tree, and beams, over a paged cache.

A case is a plain dict.  ``op`` names the call that a pass makes:

``attend``   attention of each request's tree of drafted tokens (its last kept token the root) over its
             pages: a token sees the rows before the tree, its ancestors and itself.
``verify``   the walk down a tree: at each node a token is drawn from the target's probabilities, with given
             random numbers, and the walk goes on where a child holds it.
``keep``     rows of the tokens that the walk kept moved together, in the pages of every layer.
``select``   the best continuations of each request's beams over the vocabulary.
``reorder``  the beams' page tables after a selection, and the pages that several beams would write next
             copied, in every layer.

Pages are the caller's memory, [pages][Hkv][page][d], in any order; a request's (or beam's) table names them.
``fmt`` "native" pages hold the context's type, "e4m3" pages 8-bit codes with one fp32 scale for each row of
each KV head.  Trees are in the order of their levels, ``nodes`` of the largest and ``levels`` below the root.
Rows that an attention must not read hold NaN.

``own`` chooses between the plain form (elementary torch operations in 32 bits) and the library.
"""
import math
import random

import numpy as np
import torch

own = False

DEV = "cuda"
E4M3 = torch.float8_e4m3fn


# ------------------------------------------------------------------------------------ cases

def _pages(op, dtype, fmt, hkv, d, page, batch, ragged):
    return {"op": op, "dtype": dtype, "fmt": fmt, "hkv": hkv, "d": d, "page": page, "batch": batch, "ragged": ragged}


def _attend(name, dtype="bf16", fmt="e4m3", hq=32, hkv=8, d=128, page=64, batch=1, nodes=1, levels=1, ctx=0, ragged=False,
            window=0, lse=False, theta=5.0e5):
    c = _pages("attend", dtype, fmt, hkv, d, page, batch, ragged)
    c.update(hq=hq, nodes=nodes, levels=levels, ctx=ctx, window=window, lse=lse, theta=theta)
    return {**c, "name": name} if name else c


def _verify(name, batch, nodes, levels, vocab, ragged=False):
    c = {"op": "verify", "batch": batch, "nodes": nodes, "levels": levels, "vocab": vocab, "ragged": ragged}
    return {**c, "name": name} if name else c


def _keep(name, layers, batch, nodes, levels, ctx, dtype="bf16", fmt="e4m3", hkv=8, d=128, page=64, ragged=False):
    c = _pages("keep", dtype, fmt, hkv, d, page, batch, ragged)
    c.update(layers=layers, nodes=nodes, levels=levels, ctx=ctx)
    return {**c, "name": name} if name else c


def _select(name, batch, width, vocab, best, dtype="f32", done=False):
    c = {"op": "select", "batch": batch, "width": width, "vocab": vocab, "best": best, "dtype": dtype, "done": done}
    return {**c, "name": name} if name else c


def _reorder(name, layers, batch, width, ctx, dtype="bf16", fmt="e4m3", hkv=8, d=128, page=64, ragged=False):
    c = _pages("reorder", dtype, fmt, hkv, d, page, batch, ragged)
    c.update(layers=layers, width=width, ctx=ctx)
    return {**c, "name": name} if name else c


def listed():
    return [
        # one request's small tree over a conversation's rows: latency
        _attend("attend_tree_one", nodes=16, levels=4, ctx=1500),
        # large trees of a batch, pages in the model's own type
        _attend("attend_tree_batch", fmt="native", batch=8, nodes=64, levels=6, ctx=6000, ragged=True),
        # one tree over a very long context
        _attend("attend_tree_long", nodes=32, levels=5, ctx=120000),
        # fp32 throughout: small heads, a sliding window that ends inside the tree's past
        _attend("attend_tree_f32", dtype="f32", fmt="native", hq=16, hkv=4, d=64, page=16, batch=3, nodes=26, levels=5, ctx=700,
                ragged=True, window=300, lse=True, theta=1.0e4),
        # the walk of one small tree over a small vocabulary
        _verify("verify_tree_one", 1, 16, 4, 32000),
        # a batch's trees over a large vocabulary
        _verify("verify_tree_batch", 16, 32, 6, 131072, ragged=True),
        # one request's kept rows, 32 layers
        _keep("keep_one", 32, 1, 16, 4, 1500, fmt="native"),
        # a batch's kept rows
        _keep("keep_batch", 32, 32, 64, 8, 1000, ragged=True),
        # four beams of one request over a small vocabulary
        _select("select_one", 1, 4, 32000, 4),
        # eight beams of 16 requests over a large vocabulary, logits as a model gives them, some beams ended
        _select("select_batch", 16, 8, 131072, 16, dtype="bf16", done=True),
        # four beams of one request, 32 layers
        _reorder("reorder_one", 32, 1, 4, 1000, fmt="native", page=16),
        # eight beams of 16 requests
        _reorder("reorder_batch", 32, 16, 8, 2000, ragged=True),
    ]


_HEADS = {("bf16", 128): [(32, 8), (32, 8), (64, 8), (8, 8), (32, 4), (28, 4)],
          ("bf16", 64): [(32, 8), (16, 16), (32, 4)],
          ("f32", 64): [(4, 2), (16, 4), (8, 8)],
          ("f32", 128): [(16, 4), (32, 8)]}


def draw(rng):
    """A case of the same ranges: any call, type, head layout and page size, sizes over their logarithm."""
    def log(lo, hi):
        return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.49)))))))

    op = rng.choice(["attend", "attend", "attend", "verify", "keep", "select", "reorder"])
    if op == "verify":
        c = _verify(None, log(1, 64), log(1, 128), rng.randint(1, 8), log(1000, 131072), rng.random() < 0.6)
        while c["batch"] * c["nodes"] * c["vocab"] > 1.0e8:
            c["batch" if c["batch"] > 1 else "nodes"] //= 2
        return c
    if op == "select":
        width = rng.randint(1, 16)
        c = _select(None, log(1, 32), width, log(1000, 131072), rng.choice([width, 2 * width]), rng.choice(["f32", "bf16"]), rng.random() < 0.4)
        while c["batch"] * width * c["vocab"] > (1 << 24):
            c["batch" if c["batch"] > 1 else "vocab"] //= 2
        return c
    dtype, d = rng.choice([("bf16", 128)] * 5 + [("bf16", 64), ("bf16", 64), ("f32", 64), ("f32", 128)])
    hq, hkv = rng.choice(_HEADS[dtype, d])
    fmt, page, ragged = rng.choice(["native", "e4m3", "e4m3"]), rng.choice([16, 32, 64, 128]), rng.random() < 0.7
    if op == "keep":
        return _keep(None, log(1, 48), log(1, 32), log(1, 128), rng.randint(1, 8), log(1, 8000), dtype, fmt, hkv, d, min(page, 64), ragged)
    if op == "reorder":
        c = _reorder(None, log(1, 48), log(1, 16), rng.randint(1, 16), log(1, 8000), dtype, fmt, hkv, d, page, ragged)
        while c["layers"] > 1 and work(c)["bytes"] > 1.5e8:
            c["layers"] //= 2
        return c
    c = _attend(None, dtype, fmt, hq, hkv, d, page, log(1, 32), log(1, 256), rng.randint(1, 8), log(1, 131072), ragged,
                log(16, 8192) if rng.random() < 0.2 else 0, dtype == "f32" and rng.random() < 0.5, rng.choice([1.0e4, 5.0e5]))

    # no dearer than the largest listed ones, and small enough for the plain form
    def too_much():
        w = work(c)
        return (w["bytes"] > 3.0e8 or w["flops"] > (2.0e11 if dtype == "bf16" else 4.0e9) or
                c["batch"] * hq * c["nodes"] * (c["nodes"] + c["ctx"]) > 1.0e9 or c["batch"] * (c["nodes"] + c["ctx"]) * hkv * d > 4.0e8)

    for key, least in (("batch", 1), ("ctx", 1), ("nodes", 1)):
        while c[key] > least and too_much():
            c[key] = max(least, c[key] // 2)
    return c


# ---------------------------------------------------------------------------- shape of a case

def _dtype(c):
    return torch.float32 if c["dtype"] == "f32" else torch.bfloat16


def _tree(rng, nodes, levels):
    """Parents of a tree in the order of its levels (the root is node 0), and the nodes' depths."""
    parent, depth, before, at = [-1], [0], [0], 1
    for level in range(1, levels + 1):
        left = nodes - at
        n = left if level == levels else min(left, max(1, left // (levels - level + 1) + rng.randint(-1, 2)))
        if n < 1:
            break
        of = sorted(rng.choice(before) for _ in range(n))
        parent += of
        depth += [level] * n
        before, at = list(range(at, at + n)), at + n
    return parent, depth


def _trees(c):
    """Per request: its tree's parents and depths, and the rows before it.  In a ragged batch of four and more,
    one request has no tree and one nothing before its own."""
    rng = random.Random(977)
    got = []
    for r in range(c["batch"]):
        n, x = c["nodes"], c.get("ctx", 0)
        if c["ragged"] and r:
            n, x = rng.randint(max(1, n // 4), n), rng.randint(x // 4, x)
            if c["batch"] >= 4:
                n, x = (0 if r == 1 else n), (0 if r == 2 else x)
        got.append((*(_tree(rng, n, c["levels"]) if n else ([], [])), x))
    return got


def _paths(c):
    """Per request: the nodes from the root to the last one kept.  A kept node lies where it goes or behind all
    of them, so that a pass can be repeated."""
    rng = random.Random(411)
    got = []
    for parent, depth, _ in _trees(c):
        fit = [[]]
        for i in range(len(parent)):
            path = [i]
            while parent[path[0]] >= 0:
                path.insert(0, parent[path[0]])
            if all(p == k or p >= len(path) for k, p in enumerate(path)):
                fit.append(path)
        deep = max(len(p) for p in fit)
        want = rng.randint(1, deep) if c["ragged"] and deep else deep
        got.append(rng.choice([p for p in fit if len(p) == want] or [p for p in fit if len(p) == deep]))
    return got


def _done(c):
    """Which beams have ended, and which have no score yet (a first step's, all but one of them)."""
    rng = random.Random(53)
    done = [[c["done"] and rng.random() < 0.2 for _ in range(c["width"])] for _ in range(c["batch"])]
    first = [c["done"] and c["batch"] > 2 and r == 1 for r in range(c["batch"])]
    return done, first


def _beams(c):
    """Per request: its rows, and how many beams descend from each."""
    rng = random.Random(733)
    got = []
    for r in range(c["batch"]):
        x = rng.randint(c["ctx"] // 2, c["ctx"]) if c["ragged"] and r else c["ctx"]
        of = [min(int(c["width"] * rng.random() ** 2), c["width"] - 1) for _ in range(c["width"])]
        got.append((x, of))
    return got


def _held(c):
    """Bytes of one row of K or V in its page."""
    return c["hkv"] * (c["d"] + 4 if c["fmt"] == "e4m3" else c["d"] * (4 if c["dtype"] == "f32" else 2))


def work(c):
    if c["op"] == "verify":
        rows = sum(len(p) for p in _paths(c))
        return {"bytes": 4.0 * rows * c["vocab"] + 16.0 * sum(len(t[0]) for t in _trees(c)), "flops": 4.0 * rows * c["vocab"]}
    if c["op"] == "keep":
        moved = sum(i != k for p in _paths(c) for k, i in enumerate(p))
        return {"bytes": 4.0 * moved * c["layers"] * _held(c) + 8.0 * sum(len(t[0]) for t in _trees(c)), "flops": 0.0}
    if c["op"] == "select":
        done, first = _done(c)
        rows = sum(not d and (not f or w == 0) for of, f in zip(done, first) for w, d in enumerate(of))
        return {"bytes": rows * c["vocab"] * (4.0 if c["dtype"] == "f32" else 2.0) + 16.0 * c["batch"] * (c["width"] + c["best"]),
                "flops": 3.0 * rows * c["vocab"]}
    if c["op"] == "reorder":
        rows = sum((c["width"] - len(set(of))) * (x % c["page"]) for x, of in _beams(c))
        return {"bytes": 4.0 * rows * c["layers"] * _held(c) + 8.0 * c["batch"] * c["width"] * (c["ctx"] // c["page"] + 1), "flops": 0.0}
    pairs = keys = nodes = 0
    for parent, depth, x in _trees(c):
        if parent:
            w = c["window"] or 1 << 40
            pairs += sum(min(d + 1, w) + max(0, min(x, w - d - 1)) for d in depth)
            keys += len(parent) + min(x, w - 1)
            nodes += len(parent)
    eb = 4 if c["dtype"] == "f32" else 2
    return {"bytes": 2.0 * nodes * c["hq"] * c["d"] * eb + 2.0 * keys * _held(c) + 4.0 * keys / c["page"] + 8.0 * nodes + 4.0 * nodes * c["hq"] * c["lse"],
            "flops": 4.0 * pairs * c["hq"] * c["d"]}


# ------------------------------------------------------------------------------------- inputs

def _gen(seed, tag):
    return torch.Generator(device=DEV).manual_seed((int(seed) * 1000003 + tag * 7919) % (2 ** 62))


def _normal(c, seed, tag, rows, heads, outliers=False):
    x = torch.randn((rows, heads, c["d"]), generator=_gen(seed, tag), device=DEV, dtype=_dtype(c))
    if outliers:      # a few channels of each head are large, the same ones in every row
        rng = random.Random(int(seed) * 31 + 5)
        at = [(h, rng.randrange(c["d"])) for h in range(heads) for _ in range(max(1, c["d"] // 50))]
        x[:, [h for h, _ in at], [i for _, i in at]] *= 8
    return x


def _codes(x):
    """fp32 rows [..., d] as 8-bit codes and a scale a row: the largest magnitude of a row becomes 448."""
    top = x.abs().amax(-1)
    scale = torch.where(top < 2.0 ** -100, torch.zeros_like(top), top * (1.0 / 448.0))
    inv = torch.where(scale > 0, 1.0 / scale, torch.zeros_like(scale))
    return (x * inv[..., None]).to(E4M3), scale


class _State:
    pass


class _Context:
    """The library's context, as a program keeps it."""

    def __init__(self, c):
        from paper_2607_17715_gb300 import c2kv
        self.lib = c2kv
        hkv = c.get("hkv", 1)
        self.handle = c2kv.c2kv_create(
            1, c.get("hq", hkv), hkv, c.get("d", 64), c.get("theta", 1.0e4),
            c2kv.DTYPE_F32 if c.get("dtype") == "f32" else c2kv.DTYPE_BF16, 1, stream=torch.cuda.current_stream())

    def __del__(self):
        if getattr(self, "handle", None) is not None:
            self.lib.c2kv_destroy(self.handle)


def _of_trees(s, c):
    """What a program knows of its requests' trees: ranges of tokens, parents, and each token's request."""
    s.trees = _trees(c)
    s.ptr = [0]
    for parent, _, _ in s.trees:
        s.ptr.append(s.ptr[-1] + len(parent))
    s.start = [x for _, _, x in s.trees]
    s.parent = torch.tensor(sum((p for p, _, _ in s.trees), []), dtype=torch.int32, device=DEV)
    s.req = torch.tensor(sum(([r] * len(t[0]) for r, t in enumerate(s.trees)), []), dtype=torch.int64, device=DEV)
    s.first = torch.tensor(s.ptr[:-1], device=DEV)
    s.at = torch.arange(s.ptr[-1], device=DEV) - s.first[s.req]
    s.begin = torch.tensor(s.start, device=DEV)
    s.most = max(1, max(len(t[0]) for t in s.trees))
    s.levels = c["levels"] + 1


def _prepare_attend(c, seed):
    s = _State()
    s.case = c
    _of_trees(s, c)
    s.keys = [len(p) + x for p, _, x in s.trees]
    P, T = c["page"], s.ptr[-1]
    count = [-(-k // P) for k in s.keys]
    total = sum(count) + 3
    order = torch.randperm(total, generator=torch.Generator().manual_seed(int(seed) + 17)).tolist()
    table = torch.full((c["batch"], max(1, max(count))), -1, dtype=torch.int32)
    at = 0
    for r, m in enumerate(count):
        table[r, :m] = torch.tensor(order[at:at + m], dtype=torch.int32)
        at += m
    s.table = table.to(DEV)
    shape, eight = (total, c["hkv"], P, c["d"]), c["fmt"] == "e4m3"
    s.k = torch.full(shape, math.nan, device=DEV, dtype=torch.float32 if eight else _dtype(c)).to(E4M3 if eight else _dtype(c))
    s.v = s.k.clone()
    s.ks = torch.full(shape[:3], math.nan, device=DEV) if eight else None
    s.vs = s.ks.clone() if eight else None
    for tag, pages, scales in ((3, s.k, s.ks), (4, s.v, s.vs)):
        for r, k in enumerate(s.keys):
            if k:
                row = torch.arange(k, device=DEV)
                _put(_normal(c, seed, tag + 10 * r, k, c["hkv"], tag == 3).float(), pages, scales, s.table[r, row // P].long(), row % P)
    # compressed chunks come before the tree: a token's position is beyond its place in the cache
    s.turn = torch.tensor(sum(([4 * x + d for d in depth] for _, depth, x in s.trees), []), dtype=torch.int32, device=DEV)
    s.q = _normal(c, seed, 5, T, c["hq"])
    s.out = torch.empty_like(s.q)
    s.lse = torch.empty((c["hq"], T), device=DEV) if c["lse"] else None
    s.nkeys = torch.tensor(s.keys, device=DEV)
    return s


def _prepare_verify(c, seed):
    s = _State()
    s.case = c
    _of_trees(s, c)
    B, V, T = c["batch"], c["vocab"], s.ptr[-1]
    s.p = torch.softmax(torch.randn((T, V), generator=_gen(seed, 21), device=DEV) * 3.0, -1)
    s.u = torch.rand((T,), generator=_gen(seed, 24), device=DEV)
    # drafted tokens: those of the kept path hold what its nodes draw, no other child does
    rng = random.Random(int(seed) * 97 + 3)
    tokens = [rng.randrange(V) for _ in range(T)]
    paths = _paths(c)
    for level in range(s.levels):
        here = [r for r, p in enumerate(paths) if level < len(p)]
        if not here:
            break
        rows = torch.tensor([s.ptr[r] + paths[r][level] for r in here], device=DEV)
        for r, x in zip(here, _drawn(s.p[rows], s.u[rows]).tolist()):
            kept = paths[r][level + 1] if level + 1 < len(paths[r]) else -1
            for i, of in enumerate(s.trees[r][0]):
                if of == paths[r][level]:
                    at = s.ptr[r] + i
                    tokens[at] = x if i == kept else (x + 1 + tokens[at] % (V - 1)) % V
    s.tokens = torch.tensor(tokens, dtype=torch.int32, device=DEV)
    s.n_accepted = torch.empty((B,), dtype=torch.int32, device=DEV)
    s.path = torch.empty((T,), dtype=torch.int32, device=DEV)
    s.next_token = torch.empty((B,), dtype=torch.int32, device=DEV)
    return s


def _layers(s, c, seed, total):
    """Pages of every layer, all rows of them written."""
    eight = c["fmt"] == "e4m3"
    got = []
    for tag in (31, 32):
        x = torch.randn((c["layers"], total, c["hkv"], c["page"], c["d"]), generator=_gen(seed, tag), device=DEV, dtype=_dtype(c))
        if eight:
            codes = torch.empty(x.shape, dtype=E4M3, device=DEV)
            scale = torch.empty(x.shape[:-1], device=DEV)
            for i in range(c["layers"]):
                codes[i], scale[i] = _codes(x[i].float())
            got.append((codes, scale))
        else:
            got.append((x, None))
    (s.k, s.ks), (s.v, s.vs) = got


def _prepare_keep(c, seed):
    s = _State()
    s.case = c
    _of_trees(s, c)
    P = c["page"]
    # the pages that hold the trees; those before take no part, and are not there
    held = [list(range(x // P, -(-(x + len(p)) // P))) if p else [] for p, _, x in s.trees]
    total = sum(len(h) for h in held) + 2
    order = torch.randperm(total, generator=torch.Generator().manual_seed(int(seed) + 17)).tolist()
    table = torch.full((c["batch"], max([1] + [h[-1] + 1 for h in held if h])), -1, dtype=torch.int32)
    for r, h in enumerate(held):
        for j in h:
            table[r, j] = order.pop()
    s.table = table.to(DEV)
    _layers(s, c, seed, total)
    paths = _paths(c)
    s.n_accepted = torch.tensor([max(0, len(p) - 1) for p in paths], dtype=torch.int32, device=DEV)
    s.path = torch.tensor(sum((p + [-1] * (len(t[0]) - len(p)) for p, t in zip(paths, s.trees)), []), dtype=torch.int32, device=DEV)
    return s


def _prepare_select(c, seed):
    s = _State()
    s.case = c
    B, W, V, K = c["batch"], c["width"], c["vocab"], c["best"]
    x = torch.randn((B * W, V), generator=_gen(seed, 41), device=DEV) * 3.0
    s.norm = None
    if c["dtype"] == "bf16":                         # logits as the model gives them, and what normalises them
        s.x = x.bfloat16()
        s.norm = torch.logsumexp(s.x.float(), -1)
    else:
        s.x = torch.log_softmax(x, -1)
    done, first = _done(c)
    s.score = -20.0 * torch.rand((B, W), generator=_gen(seed, 42), device=DEV)
    for r in range(B):
        if first[r]:
            s.score[r, 1:] = -math.inf
    s.done = torch.tensor(done, dtype=torch.int32, device=DEV) if c["done"] else None
    s.parent, s.token, s.done_out = (torch.empty((B, K), dtype=torch.int32, device=DEV) for _ in range(3))
    s.score_out = torch.empty((B, K), device=DEV)
    return s


def _prepare_reorder(c, seed):
    s = _State()
    s.case = c
    beams, W, P = _beams(c), c["width"], c["page"]
    s.rows = [x for x, _ in beams]
    width = c["ctx"] // P + 1
    tails = c["batch"] * W
    total = tails + 7
    # each beam's last page is its own; pages before are shared by beams
    g = torch.Generator().manual_seed(int(seed) + 17)
    order = torch.randperm(total, generator=g)
    table = torch.randint(0, total, (tails, width), generator=g, dtype=torch.int32)
    for b in range(tails):
        table[b, s.rows[b // W] // P] = order[b]
    s.table = table.to(DEV)
    s.table_out = torch.empty_like(s.table)
    rng = random.Random(int(seed) * 13 + 1)
    parent = []
    for _, of in beams:                              # as many descend from one as from another, beams of another order
        name = rng.sample(range(W), W)
        parent.append([name[i] for i in rng.sample(of, W)])
    s.parent = torch.tensor(parent, dtype=torch.int32, device=DEV)
    s.n_rows = torch.tensor(s.rows, device=DEV)
    _layers(s, c, seed, total)
    return s


def prepare(c, seed):
    s = {"attend": _prepare_attend, "verify": _prepare_verify, "keep": _prepare_keep, "select": _prepare_select,
         "reorder": _prepare_reorder}[c["op"]](c, seed)
    if own:
        s.context = _Context(c)
        lib = s.context.lib
        if c["op"] == "attend":
            s.pages = lib.make_pages(s.k, s.v, s.ks, s.vs)
        elif c["op"] in ("keep", "reorder"):
            s.pages = lib.make_layers(s.k, s.v, s.ks, s.vs)
    return s


# -------------------------------------------------------------------------------- plain forms

def _turned(x, turn, theta):
    """fp32 rows x [..., heads, d] turned by turn [...] positions.  The angle's fraction of a turn is
    held in 64-bit whole numbers, whose wrap-around drops the full turns."""
    h = x.shape[-1] // 2
    freq = [theta ** (-2.0 * i / (2 * h)) / (2.0 * math.pi) * 2.0 ** 64 for i in range(h)]
    step = torch.tensor([int(f) - (1 << 64 if int(f) >= 1 << 63 else 0) for f in freq], dtype=torch.int64, device=DEV)
    angle = (turn.long()[..., None] * step).float() * (math.pi * 2.0 ** -63)
    cos, sin = torch.cos(angle)[..., None, :], torch.sin(angle)[..., None, :]
    a, b = x[..., :h], x[..., h:]
    return torch.cat([a * cos - b * sin, a * sin + b * cos], -1)


def _rows_of(pages, scales, pg, off):
    """Rows of the pages as fp32 values."""
    x = pages.view(torch.uint8)[pg, :, off].view(E4M3).float() if scales is not None else pages[pg, :, off].float()
    return x if scales is None else x * scales[pg, :, off][..., None]


def _put(x, pages, scales, pg, off):
    if scales is None:
        pages[pg, :, off] = x.to(pages.dtype)
    else:
        code, scale = _codes(x)
        pages.view(torch.uint8)[pg, :, off] = code.view(torch.uint8)
        scales[pg, :, off] = scale


def _padded(s, x, fill):
    """Values of the trees' tokens as [requests, most tokens]."""
    y = torch.full((len(s.trees), s.most), fill, dtype=torch.int64, device=DEV)
    y[s.req, s.at] = x.long()
    return y


def _plain_attend(s):
    c, P = s.case, s.case["page"]
    B, G, n, S = c["batch"], c["hq"] // c["hkv"], s.most, max(1, max(s.keys))
    row = torch.arange(S, device=DEV)
    pg = s.table[:, row // P].long().clamp_(min=0)                          # [B, S]
    there = (row < s.nkeys[:, None])[..., None, None]
    k = torch.where(there, _rows_of(s.k, s.ks, pg, row % P), 0.0)
    v = torch.where(there, _rows_of(s.v, s.vs, pg, row % P), 0.0)
    # the tokens on the way from each to the root, and its depth
    parent = _padded(s, s.parent, -1)
    on_way = torch.zeros((B, n, n + 1), dtype=torch.bool, device=DEV)
    at = torch.arange(n, device=DEV).expand(B, n)
    depth = torch.full((B, n), -1, device=DEV)
    for step in range(s.levels):
        if not c["window"] or step < c["window"]:
            on_way.scatter_(2, torch.where(at < 0, n, at)[..., None], True)
        depth += at >= 0
        at = torch.where(at < 0, -1, parent.gather(1, at.clamp(min=0)))
    on_way[..., n] = False
    col = (row - s.begin[:, None]).clamp(-1, n)                             # [B, S]: the tree's token in a row
    seen = on_way.gather(2, torch.where(col < 0, n, col)[:, None].expand(B, n, S))
    before = (col < 0)[:, None]
    if c["window"]:
        before = before & (row > (s.begin[:, None] + depth - c["window"])[..., None])
    seen = (seen | before) & (row < s.nkeys[:, None])[:, None]
    q = torch.zeros((B, n, c["hq"], c["d"]), device=DEV)
    q[s.req, s.at] = _turned(s.q.float(), s.turn, c["theta"])
    q = q.view(B, n, c["hkv"], G, c["d"]).permute(0, 2, 3, 1, 4).reshape(B, c["hkv"], G * n, c["d"])
    x = torch.matmul(q, k.permute(0, 2, 3, 1)).view(B, c["hkv"], G, n, S) * (1.0 / math.sqrt(c["d"]))
    x = x.masked_fill_(~seen[:, None, None], -math.inf)
    top = x.amax(-1, keepdim=True).clamp_(min=-1.0e38)
    x = x.sub_(top).exp_()
    total = x.sum(-1, keepdim=True)
    o = torch.matmul(x.view(B, c["hkv"], G * n, S), v.permute(0, 2, 1, 3)).view(B, c["hkv"], G, n, c["d"]) / total
    o = o.permute(0, 3, 1, 2, 4).reshape(B, n, c["hq"], c["d"])
    s.out.copy_(o[s.req, s.at])
    if c["lse"]:
        lse = (top + total.log())[..., 0].permute(0, 3, 1, 2).reshape(B, n, c["hq"])
        s.lse.copy_(lse[s.req, s.at].t())


def _drawn(p, u):
    """A token of each row of probabilities: weights are whole multiples of 2^-44, so that their sums are exact
    in any order.  -1 where there is no weight."""
    w = (torch.nan_to_num(p, nan=0.0).clamp(0.0, 1.0) * 2.0 ** 44).long()
    total = w.sum(-1)
    k = (u * 2.0 ** 24).long().clamp(0, 2 ** 24 - 1)
    goal = (total >> 24) * k + (((total & (2 ** 24 - 1)) * k) >> 24)
    return torch.where(total == 0, -1, (w.cumsum(-1) <= goal[:, None]).sum(-1))


def _plain_verify(s):
    B, n, T = s.case["batch"], s.most, s.ptr[-1]
    node = torch.zeros(B, dtype=torch.int64, device=DEV)
    parent, tokens = _padded(s, s.parent, -2), _padded(s, s.tokens, -2)
    i = torch.arange(n, device=DEV)
    walking = parent[:, 0] != -2
    accepted = torch.zeros_like(node)
    token = torch.full_like(node, -1)
    path = torch.full((B, n + 1), -1, device=DEV)
    path[:, 0] = torch.where(walking, 0, -1)
    r = torch.arange(B, device=DEV)
    for _ in range(s.levels):
        row = (s.first + node).clamp_(max=T - 1)
        x = _drawn(s.p[row], s.u[row])
        fits = (parent == node[:, None]) & (tokens == x[:, None]) & (x >= 0)[:, None] & (i > node[:, None])
        child = torch.where(fits, i, n).amin(-1)
        on = walking & (child < n)
        token = torch.where(walking & ~on, x, token)
        accepted = accepted + on
        path[r, torch.where(on, accepted, n)] = torch.where(on, child, -1)
        node = torch.where(on, child, node)
        walking = on
    s.n_accepted.copy_(accepted)
    s.path.copy_(path[s.req, s.at])
    s.next_token.copy_(token)


def _page_tensors(s):
    return [x for x in (s.k, s.v, s.ks, s.vs) if x is not None]


def _bits(x):
    return x.view(torch.uint8) if x.dtype == E4M3 else x


def _plain_keep(s):
    P = s.case["page"]
    kept = s.at <= s.n_accepted.long()[s.req]
    from_ = torch.where(kept, s.path.long(), s.at) + s.begin[s.req]
    to = s.at + s.begin[s.req]
    pf, of, pt, ot = s.table[s.req, from_ // P].long(), from_ % P, s.table[s.req, to // P].long(), to % P
    for x in _page_tensors(s):
        x = _bits(x)
        x[:, pt, :, ot] = x[:, pf, :, of]


def _plain_select(s):
    c = s.case
    B, W, V, K = c["batch"], c["width"], c["vocab"], c["best"]
    x = s.x.float()
    if s.norm is not None:
        x = x - s.norm[:, None]
    x = (s.score.view(B * W, 1) + x).view(B, W, V)
    if s.done is not None:                           # an ended beam goes on as it is
        alone = torch.where(torch.arange(V, device=DEV) == 2, s.score[..., None], -math.inf)
        x = torch.where((s.done != 0)[..., None], alone, x)
    x = torch.where(torch.isnan(x), -math.inf, x).view(B, W * V) + 0.0
    # the largest first, of equal ones the first: scores as whole numbers of the same order, then the place
    bits = x.view(torch.int32)
    order = torch.where(bits < 0, bits ^ 0x7fffffff, bits).long()
    key = (order << 32) + (0x7fffffff - torch.arange(W * V, device=DEV))
    best = 0x7fffffff - (key.topk(K, -1).values & 0xffffffff)
    score = x.gather(1, best)
    found = score > -math.inf
    parent, token = torch.where(found, best // V, -1), torch.where(found, best % V, -1)
    s.parent.copy_(parent)
    s.token.copy_(token)
    s.score_out.copy_(score)
    ended = torch.zeros_like(found) if s.done is None else found & (s.done.gather(1, parent.clamp(min=0)) != 0)
    s.done_out.copy_(ended | (found & (token == 2)))


def _plain_reorder(s):
    c = s.case
    B, W, P = c["batch"], c["width"], c["page"]
    width = s.table.shape[1]
    table = s.table.view(B, W, width).long()
    of = s.parent.long()
    full, part = s.n_rows // P, s.n_rows % P
    tail = table.gather(2, full[:, None, None].expand(B, W, 1))[..., 0]
    # the first beam of a parent keeps its page; the others take those of beams that none descends from, in order
    eq = of[..., None] == torch.arange(W, device=DEV)                       # [B, beam, parent]
    first = (eq & (eq.cumsum(1) == 1)).any(-1)
    none = ~eq.any(1)
    match = (~first)[..., None] & none[:, None] & (((~first).cumsum(1) - 1)[..., None] == (none.cumsum(1) - 1)[:, None])
    source = tail.gather(1, of)
    target = torch.where(first, source, (match * tail[:, None]).sum(-1))
    col = torch.arange(width, device=DEV)
    inherited = table.gather(1, of[..., None].expand(B, W, width))
    whole, last = (col < full[:, None])[:, None], (col == full[:, None])[:, None] & (part > 0)[:, None, None]
    s.table_out.copy_(torch.where(whole, inherited, torch.where(last, target[..., None], table)).view(B * W, width))
    target = torch.where((part > 0)[:, None], target, tail).view(-1)
    source = torch.where((part > 0)[:, None], source, tail).view(-1)
    rows = torch.arange(P, device=DEV) < part.repeat_interleave(W)[:, None]  # [beams, P]
    for x in _page_tensors(s):
        x = _bits(x)
        m = rows[None, :, None].reshape(1, B * W, 1, P, *([1] * (x.dim() - 4)))
        x[:, target] = torch.where(m, x[:, source], x[:, target])


# --------------------------------------------------------------------------------------- pass

def run(s):
    c, op = s.case, s.case["op"]
    if own:
        lib, ctx = s.context.lib, s.context.handle
        if op == "attend":
            lib.c2kv_paged_attend_tree(ctx, s.pages, s.table, s.ptr, s.keys, s.parent, s.q, s.out, lse=s.lse, turn=s.turn,
                                       window=c["window"])
        elif op == "verify":
            lib.c2kv_verify_tree(ctx, s.ptr, s.tokens, s.parent, s.p, s.u, s.n_accepted, s.path, s.next_token)
        elif op == "keep":
            lib.c2kv_paged_keep(ctx, s.pages, s.table, s.ptr, s.start, s.path, s.n_accepted)
        elif op == "select":
            lib.c2kv_beam_select(ctx, s.x, s.score, s.parent, s.token, s.score_out, norm=s.norm, done=s.done, end_token=2,
                                 done_out=s.done_out)
        else:
            lib.c2kv_paged_reorder(ctx, s.pages, s.table, s.rows, s.parent, s.table_out)
    else:
        {"attend": _plain_attend, "verify": _plain_verify, "keep": _plain_keep, "select": _plain_select, "reorder": _plain_reorder}[op](s)
    if op == "attend":
        return {"out": s.out, "lse": s.lse}
    if op == "verify":
        return {"n_accepted": s.n_accepted, "path": s.path, "next_token": s.next_token}
    if op == "select":
        return {"parent": s.parent, "token": s.token, "score": s.score_out, "done": s.done_out}
    pages = {"k": s.k, "v": s.v, "k_scale": s.ks, "v_scale": s.vs}
    return pages if op == "keep" else {**pages, "table": s.table_out}


# ------------------------------------------------------------------------------- 64-bit results

def _rope64(x, pos, theta):
    h = x.shape[-1] // 2
    a = pos.double()[:, None, None] * theta ** (-torch.arange(h, dtype=torch.float64, device=DEV) / h)
    z = torch.polar(torch.ones_like(a), a) * torch.complex(x[..., :h].contiguous(), x[..., h:].contiguous())
    return torch.cat([z.real, z.imag], -1)


def _exact_attend(c, s):
    G, P = c["hq"] // c["hkv"], c["page"]
    out = torch.zeros((s.ptr[-1], c["hq"], c["d"]), dtype=torch.float64, device=DEV)
    lse = torch.zeros((c["hq"], s.ptr[-1]), dtype=torch.float64, device=DEV)
    for r, (parent, depth, x) in enumerate(s.trees):
        n, m = len(parent), len(parent) + x
        if not n:
            continue
        pg = s.table[r, :-(-m // P)].long()
        k, v = ((y[pg].double() * (1 if ys is None else ys[pg].double()[..., None])).transpose(1, 2).reshape(-1, c["hkv"], c["d"])[:m]
                for y, ys in ((s.k, s.ks), (s.v, s.vs)))
        hidden = torch.ones((n, m), dtype=torch.bool)
        for i in range(n):
            if c["window"]:
                hidden[i, max(0, x + depth[i] - c["window"] + 1):x] = False
            else:
                hidden[i, :x] = False
            j, left = i, c["window"] or n
            while j >= 0 and left > 0:
                hidden[i, x + j] = False
                j, left = parent[j], left - 1
        hidden = hidden.to(DEV)
        at = slice(s.ptr[r], s.ptr[r + 1])
        q = _rope64(s.q[at].double(), s.turn[at], c["theta"])
        for h in range(c["hq"]):
            z = q[:, h] @ k[:, h // G].t() / math.sqrt(c["d"])
            z[hidden] = -math.inf
            out[at, h] = torch.softmax(z, -1) @ v[:, h // G]
            lse[h, at] = torch.logsumexp(z, -1)
    return {"out": out, "lse": lse if c["lse"] else None}


def _exact_verify(c, s):
    """One request after another, in Python's whole numbers and numpy's search."""
    tokens, u = s.tokens.tolist(), s.u.tolist()
    accepted, paths, nexts = [], [], []
    for r, (parent, _, _) in enumerate(s.trees):
        lo, node, path, x = s.ptr[r], 0, [0] if parent else [], -1
        while parent:
            run_up = (s.p[lo + node].double().cpu().numpy().clip(0, 1) * 2.0 ** 44).astype("int64").cumsum()
            x = int(run_up.searchsorted(int(run_up[-1]) * int(u[lo + node] * 2 ** 24) >> 24, side="right")) if run_up[-1] else -1
            child = [i for i, of in enumerate(parent) if of == node and tokens[lo + i] == x and i > 0]
            if not child:
                break
            node = child[0]
            path.append(node)
        accepted.append(max(0, len(path) - 1))
        paths += path + [-1] * (len(parent) - len(path))
        nexts.append(x)
    return {n: torch.tensor(x, dtype=torch.int32) for n, x in (("n_accepted", accepted), ("path", paths), ("next_token", nexts))}


def _exact_pages(s):
    got = {"k": s.k, "v": s.v, "k_scale": s.ks, "v_scale": s.vs}
    return {n: None if x is None else x.float() for n, x in got.items()}     # (copies hold what was there: exact in 32 bits)


def _exact_keep(c, s):
    got, P, table = _exact_pages(s), c["page"], s.table.tolist()
    for r, path in enumerate(_paths(c)):
        for k, i in enumerate(path):
            a, b = s.start[r] + k, s.start[r] + i
            for x in got.values():
                if x is not None:
                    x[:, table[r][a // P], :, a % P] = x[:, table[r][b // P], :, b % P].clone()
    return got


def _exact_select(c, s):
    B, W, V, K = c["batch"], c["width"], c["vocab"], c["best"]
    score = s.score.cpu().numpy()
    done = s.done.tolist() if s.done is not None else [[0] * W] * B
    want = {n: [] for n in ("parent", "token", "score", "done")}
    for r in range(B):
        x = s.x[r * W:(r + 1) * W].float().cpu().numpy()
        if s.norm is not None:
            x = x - s.norm[r * W:(r + 1) * W, None].cpu().numpy()
        x = score[r][:, None] + x                    # (fp32, as the operator is defined)
        got = []
        for w in range(W):
            if done[r][w]:
                got.append((-float(score[r][w]), w, 2))
            else:
                top = np.argsort(-x[w], kind="stable")[:K]
                got += [(-float(x[w][t]), w, int(t)) for t in top]
        got = sorted(g for g in got if g[0] < math.inf)[:K]
        got += [(math.inf, -1, -1)] * (K - len(got))
        want["score"].append([-g[0] for g in got])
        want["parent"].append([g[1] for g in got])
        want["token"].append([g[2] for g in got])
        want["done"].append([int(g[1] >= 0 and (g[2] == 2 or done[r][g[1]] != 0)) for g in got])
    return {n: torch.tensor(x, dtype=torch.float64 if n == "score" else torch.int32) for n, x in want.items()}


def _exact_reorder(c, s):
    got, P, W, table, parent = _exact_pages(s), c["page"], c["width"], s.table.tolist(), s.parent.tolist()
    out = []
    for r, of in enumerate(parent):
        full, part = divmod(s.rows[r], P)
        free = [w for w in range(W) if w not in of]
        for w in range(W):
            mine, theirs = table[r * W + w], table[r * W + of[w]]
            row = theirs[:full] + mine[full:]
            if part:
                row[full] = theirs[full] if of.index(of[w]) == w else table[r * W + free.pop(0)][full]
                for x in got.values():
                    if x is not None:
                        x[:, row[full], :, :part] = x[:, theirs[full], :, :part].clone()
            out.append(row)
    return {**got, "table": torch.tensor(out, dtype=torch.int32)}


def exact(c, seed):
    global own
    was, own = own, False
    try:
        s = prepare(c, seed)
    finally:
        own = was
    return {"attend": _exact_attend, "verify": _exact_verify, "keep": _exact_keep, "select": _exact_select,
            "reorder": _exact_reorder}[c["op"]](c, s)
