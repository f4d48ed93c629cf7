"""Timed cases of generation over a paged cache: what a serving program does after its chunks are
composed, through the library's public calls.

A case is a plain dict.  ``op`` names the call that a pass makes:

``append``   new tokens' keys and values written into their requests' pages: K turned to its
             position, both quantised where the pages hold 8 bits.
``gather``   rows of a paged cache read back into a dense block, K turned back where it is to
             become a stored chunk.
``attend``   attention of each request's new tokens (one, a few drafted ones, a chunk of a prompt)
             over its pages.
``verify``   drafted tokens accepted or refused against the target's probabilities, and the token
             that follows them drawn, from given random numbers.

Pages are the caller's memory, [pages][Hkv][page][d], in any order; a request's table names them.
``fmt`` "native" pages hold the context's type, "e4m3" pages 8-bit codes with one fp32 scale for
each row of each KV head.  Rows that no token was written to hold NaN where a call must not read
them.  Keys and values are standard normal with a few outlier channels, queries standard normal.

``own`` chooses between the plain form (elementary torch operations in 32 bits) and the library.
"""
import math
import random

import torch

own = False

DEV = "cuda"
E4M3 = torch.float8_e4m3fn


# ------------------------------------------------------------------------------------ cases

def _case(name, op, dtype="bf16", fmt="e4m3", hq=32, hkv=8, d=128, page=64, batch=1, new=1, ctx=0, **more):
    c = {"op": op, "dtype": dtype, "fmt": fmt, "hq": hq, "hkv": hkv, "d": d, "theta": 5.0e5, "page": page,
         "batch": batch, "new": new, "ctx": ctx, "ragged": False, "window": 0, "turn": True, "lse": False}
    if name:
        c["name"] = name
    c.update(more)
    return c


def _drafts(name, batch, drafts, vocab, ragged=False, greedy=False):
    c = {"op": "verify", "batch": batch, "drafts": drafts, "vocab": vocab, "ragged": ragged, "greedy": greedy}
    if name:
        c["name"] = name
    return c


def listed():
    return [
        # one generated token of each of 16 requests written to its page: launch and latency
        _case("append_token", "append", batch=16, new=1, ctx=2000, ragged=True),
        # prompts of eight requests, thousands of rows at once, as a prefill writes them
        _case("append_prompts", "append", batch=8, new=4000, ctx=500, ragged=True),
        # an answer of 300 tokens read back, K turned back to before RoPE, to be stored as a chunk
        _case("gather_answer", "gather", page=16, batch=1, new=300, ctx=1111),
        # whole contexts moved out of their pages into one dense block, as they are
        _case("gather_contexts", "gather", batch=16, new=8000, ctx=0, ragged=True, turn=False),
        # a generation step: one token of each of 16 requests over contexts of 500 to 2000 rows
        _case("attend_token_16", "attend", batch=16, new=1, ctx=2000, ragged=True),
        # one request's token over a very long context in the model's own type
        _case("attend_token_long", "attend", fmt="native", page=128, batch=1, new=1, ctx=131000),
        # four drafted tokens and the one before them, larger groups, thousands of rows each
        _case("attend_drafts", "attend", hq=64, batch=8, new=5, ctx=6000, ragged=True, page=32),
        # chunks of four prompts next to one another, 16-bit pages
        _case("attend_prompts", "attend", fmt="native", batch=4, new=500, ctx=4000, ragged=True),
        # a late chunk of one very long prompt: the largest
        _case("attend_chunk_long", "attend", batch=1, new=2048, ctx=30720),
        # fp32 throughout: small heads, short chunks
        _case("attend_f32", "attend", dtype="f32", fmt="native", hq=16, hkv=4, d=64, page=16, batch=3, new=61,
              ctx=700, ragged=True, theta=1.0e4, lse=True),
        # one request, four drafted tokens, a small vocabulary
        _drafts("verify_one", 1, 4, 32000),
        # a batch's drafts over a large vocabulary
        _drafts("verify_batch_64", 64, 8, 131072, ragged=True),
    ]


_HEADS = {("bf16", 128): [(32, 8), (32, 8), (64, 8), (8, 8), (32, 4), (28, 4)],
          ("bf16", 64): [(32, 8), (16, 16), (32, 4)],
          ("f32", 64): [(4, 2), (16, 4), (8, 8)],
          ("f32", 128): [(16, 4), (32, 8)]}


def draw(rng):
    """A case of the same ranges: any call, type, head layout and page size, sizes over their logarithm."""
    def log(lo, hi):
        return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.49)))))))

    op = rng.choice(["append", "append", "gather", "attend", "attend", "attend", "attend", "verify"])
    if op == "verify":
        return _drafts(None, log(1, 64), log(1, 8), log(1000, 131072), rng.random() < 0.6, rng.random() < 0.25)
    dtype, d = rng.choice([("bf16", 128)] * 5 + [("bf16", 64), ("bf16", 64), ("f32", 64), ("f32", 128)])
    hq, hkv = rng.choice(_HEADS[dtype, d])
    c = _case(None, op, dtype=dtype, fmt=rng.choice(["native", "e4m3", "e4m3"]), hq=hq, hkv=hkv, d=d,
              theta=rng.choice([1.0e4, 5.0e5]), page=rng.choice([16, 32, 64, 128]), batch=log(1, 32),
              ragged=rng.random() < 0.7, turn=rng.random() < 0.8)
    if op == "attend":
        c.update(new=rng.choice([1, 1, rng.randint(2, 9), log(10, 2048)]), ctx=log(1, 131072))
        c["window"] = log(16, 8192) if rng.random() < 0.2 else 0
        c["lse"] = dtype == "f32" and rng.random() < 0.5
    else:
        c.update(new=rng.choice([1, log(1, 8000)]), ctx=log(1, 8000))

    # no dearer than the largest listed one, and small enough for the plain form
    tc = dtype == "bf16"

    def too_much():
        w = work(c)
        scores = c["batch"] * c["hq"] * c["new"] * (c["new"] + c["ctx"]) if op == "attend" else 0
        rows = sum(n + x for n, x in _lens(c)) * hkv * d
        return (w["bytes"] > 5.0e8 or w["flops"] > (1.0e12 if tc else 2.0e10) or scores > 2.0e9 or rows > 3.0e8 or
                c["batch"] * (c["new"] + c["ctx"]) * hkv * d > 6.0e8)

    for key, least in (("batch", 1), ("ctx", 1), ("new", 1)):
        while c[key] > least and too_much():
            c[key] = max(least, c[key] // 2)
    return c


# ---------------------------------------------------------------------------- shape of a case

def _dtype(c):
    return torch.float32 if c["dtype"] == "f32" else torch.bfloat16


def _lens(c):
    """Per request: its new tokens and the rows before them.  In a ragged batch of four and more, one
    request has no new token and one nothing before its own."""
    rng = random.Random(977)
    got = []
    for r in range(c["batch"]):
        n, x = c["new"], c["ctx"]
        if c["ragged"] and r:
            n, x = rng.randint(max(1, n // 4), n), rng.randint(x // 4, x)
            if c["batch"] >= 4:
                n, x = (0 if r == 1 else n), (0 if r == 2 else x)
        got.append((n, x))
    return got


def _n_drafts(c):
    rng = random.Random(411)
    return [rng.randint(0, c["drafts"]) if c["ragged"] and r else c["drafts"] for r in range(c["batch"])]


def _visible(c, n, x):
    """(query, key) pairs that are seen, and keys that any query sees, of n tokens after x rows."""
    w = c["window"]
    if not n:
        return 0, 0
    if not w:
        return n * x + n * (n + 1) // 2, n + x
    return sum(min(w, x + i + 1) for i in range(n)), min(n + x, w + n - 1)


def work(c):
    if c["op"] == "verify":
        rows = c["batch"] * (1 if c["greedy"] else 2)
        return {"bytes": 4.0 * rows * c["vocab"] + 12.0 * sum(_n_drafts(c)) + 12.0 * c["batch"], "flops": 4.0 * rows * c["vocab"]}
    eb = 4 if c["dtype"] == "f32" else 2
    row = c["hkv"] * c["d"] * eb
    held = c["hkv"] * (c["d"] + 4) if c["fmt"] == "e4m3" else row       # one row of K or V in its page
    lens = _lens(c)
    if c["op"] != "attend":
        n = sum(n for n, _ in lens)
        return {"bytes": 2.0 * n * (row + held) + 4.0 * n * c["turn"], "flops": n * c["hkv"] * c["d"] * (5.0 + 3.0 * c["turn"])}
    pairs = keys = 0
    for n, x in lens:
        p, k = _visible(c, n, x)
        pairs, keys = pairs + p, keys + k
    n = sum(n for n, _ in lens)
    return {"bytes": 2.0 * n * c["hq"] * c["d"] * eb + 2.0 * keys * held + 4.0 * keys / c["page"] + 4.0 * n * c["hq"] * c["lse"],
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
        self.handle = c2kv.c2kv_create(
            1, c.get("hq", 1), c.get("hkv", 1), c.get("d", 64), c.get("theta", 1.0e4),
            c2kv.DTYPE_F32 if c.get("dtype") == "f32" else c2kv.DTYPE_BF16, 1, stream=torch.cuda.current_stream())

    def __del__(self):
        if getattr(self, "handle", None) is not None:
            self.lib.c2kv_destroy(self.handle)


def _prepare_verify(c, seed):
    s = _State()
    s.case, n = c, _n_drafts(c)
    B, V, T = c["batch"], c["vocab"], sum(n)
    s.ptr = [0]
    for g in n:
        s.ptr.append(s.ptr[-1] + g)
    s.first = torch.tensor(s.ptr[:-1], device=DEV)
    s.count = torch.tensor(n, device=DEV)
    s.q = s.p = None
    # peaked distributions, the target's near the draft's; row i of request r is i + r beyond its first draft
    rows = torch.cat([torch.arange(s.ptr[r], s.ptr[r + 1] + 1, device=DEV) for r in range(B)])
    logits = torch.randn((T + 1, V), generator=_gen(seed, 21), device=DEV) * 3.0
    near = torch.randn((T + B, V), generator=_gen(seed, 22), device=DEV) * 0.5
    s.p = torch.softmax(near.add_(logits[rows]), -1)
    del near
    q = torch.softmax(logits[:T], -1)
    s.tokens = (q.argmax(-1) if c["greedy"] else torch.multinomial(q, 1, generator=_gen(seed, 23))[:, 0] if T else
                torch.zeros(0, device=DEV)).to(torch.int32)
    s.q = None if c["greedy"] else q
    s.u_accept = torch.rand((T,), generator=_gen(seed, 24), device=DEV)
    s.u_next = torch.rand((B,), generator=_gen(seed, 25), device=DEV)
    s.n_accepted = torch.empty((B,), dtype=torch.int32, device=DEV)
    s.next_token = torch.empty((B,), dtype=torch.int32, device=DEV)
    return s


def prepare(c, seed):
    if c["op"] == "verify":
        s = _prepare_verify(c, seed)
        if own:
            s.context = _Context(c)
        return s
    s = _State()
    s.case = c
    lens = _lens(c)
    s.lens = lens
    s.ptr = [0]
    for n, _ in lens:
        s.ptr.append(s.ptr[-1] + n)
    s.start = [x for _, x in lens]
    s.keys = [n + x for n, x in lens]
    T = s.ptr[-1]
    # the pages of the requests, in no order, and the table that names them; -1 where a request has none
    P = c["page"]
    count = [-(-k // P) for k in s.keys]
    total = sum(count) + 3
    order = torch.randperm(total, generator=torch.Generator().manual_seed(int(seed) + 17)).tolist()
    table = torch.full((c["batch"], max(1, max(count))), -1, dtype=torch.int32)
    at = 0
    for r, m in enumerate(count):
        table[r, :m] = torch.tensor(order[at:at + m], dtype=torch.int32)
        at += m
    s.table = table.to(DEV)
    shape = (total, c["hkv"], P, c["d"])
    eight = c["fmt"] == "e4m3"
    fill = 0.0 if c["op"] == "append" else math.nan
    s.k = torch.full(shape, fill, device=DEV, dtype=torch.float32 if eight else _dtype(c)).to(E4M3 if eight else _dtype(c))
    s.v = s.k.clone()
    s.ks = torch.full(shape[:3], fill, device=DEV) if eight else None
    s.vs = s.ks.clone() if eight else None
    # token t of the batch: its request and its row there
    s.req = torch.cat([torch.full((n,), r, dtype=torch.int64) for r, (n, _) in enumerate(lens)]).to(DEV)
    s.row = torch.cat([torch.arange(x, x + n) for n, x in lens]).to(DEV)
    # compressed chunks come before the new tokens: a row's position is beyond its place in the cache
    pos = torch.cat([torch.arange(4 * x, 4 * x + n) for n, x in lens]).to(DEV, torch.int32)
    s.turn = (-pos if c["op"] == "gather" else pos) if c["turn"] else None
    if c["op"] == "append":
        s.new_k, s.new_v = _normal(c, seed, 1, T, c["hkv"], True), _normal(c, seed, 2, T, c["hkv"])
    else:             # what is in the pages already
        for tag, pages, scales in ((3, s.k, s.ks), (4, s.v, s.vs)):
            for r, k in enumerate(s.keys):
                row = torch.arange(k, device=DEV)
                pg, off = s.table[r, row // P].long(), row % P
                _put(_normal(c, seed, tag + 10 * r, k, c["hkv"], tag == 3).float(), pages, scales, pg, off)
    if c["op"] == "gather":
        s.out_k = torch.empty((T, c["hkv"], c["d"]), dtype=_dtype(c), device=DEV)
        s.out_v = torch.empty_like(s.out_k)
    if c["op"] == "attend":
        s.q = _normal(c, seed, 5, T, c["hq"])
        s.out = torch.empty_like(s.q)
        s.lse = torch.empty((c["hq"], T), device=DEV) if c["lse"] else None
        s.nkeys = torch.tensor(s.keys, device=DEV)
    if own:
        s.context = _Context(c)
        s.pages = s.context.lib.make_pages(s.k, s.v, s.ks, s.vs)
    return s


# -------------------------------------------------------------------------------- plain forms

def _turned(x, turn, theta):
    """fp32 rows x [..., heads, d] turned by turn [...] positions.  The angle's fraction of a turn is
    held in 64-bit whole numbers, whose wrap-around drops the full turns."""
    if turn is None:
        return x
    h = x.shape[-1] // 2
    freq = [theta ** (-2.0 * i / (2 * h)) / (2.0 * math.pi) * 2.0 ** 64 for i in range(h)]
    step = torch.tensor([int(f) - (1 << 64 if int(f) >= 1 << 63 else 0) for f in freq], dtype=torch.int64, device=DEV)
    angle = (turn.long()[..., None] * step).float() * (math.pi * 2.0 ** -63)
    cos, sin = torch.cos(angle)[..., None, :], torch.sin(angle)[..., None, :]
    a, b = x[..., :h], x[..., h:]
    return torch.cat([a * cos - b * sin, a * sin + b * cos], -1)


def _held(pages, scales, pg, off):
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


def _plain_append(s):
    c, P = s.case, s.case["page"]
    pg, off = s.table[s.req, s.row // P].long(), s.row % P
    _put(_turned(s.new_k.float(), s.turn, c["theta"]), s.k, s.ks, pg, off)
    _put(s.new_v.float(), s.v, s.vs, pg, off)


def _plain_gather(s):
    c, P = s.case, s.case["page"]
    pg, off = s.table[s.req, s.row // P].long(), s.row % P
    s.out_k.copy_(_turned(_held(s.k, s.ks, pg, off), s.turn, c["theta"]))
    s.out_v.copy_(_held(s.v, s.vs, pg, off))


def _plain_attend(s):
    c, P = s.case, s.case["page"]
    B, G, n, S = c["batch"], c["hq"] // c["hkv"], max(n for n, _ in s.lens), max(s.keys)
    row = torch.arange(S, device=DEV)
    pg = s.table[:, row // P].long().clamp_(min=0)                          # [B, S]
    there = (row < s.nkeys[:, None])[..., None, None]
    k = torch.where(there, _held(s.k, s.ks, pg, row % P), 0.0)
    v = torch.where(there, _held(s.v, s.vs, pg, row % P), 0.0)
    # queries padded to the longest request's
    at = s.row - torch.tensor(s.start, device=DEV)[s.req]
    q = torch.zeros((B, n, c["hq"], c["d"]), device=DEV)
    q[s.req, at] = _turned(s.q.float(), s.turn, c["theta"])
    last = torch.full((B, n), -1, device=DEV)
    last[s.req, at] = s.row
    q = q.view(B, n, c["hkv"], G, c["d"]).permute(0, 2, 3, 1, 4).reshape(B, c["hkv"], G * n, c["d"])
    x = torch.matmul(q, k.permute(0, 2, 3, 1)).view(B, c["hkv"], G, n, S) * (1.0 / math.sqrt(c["d"]))
    seen = row <= last[..., None]
    if c["window"]:
        seen &= row > last[..., None] - c["window"]
    x = x.masked_fill_(~seen[:, None, None], -math.inf)
    top = x.amax(-1, keepdim=True).clamp_(min=-1.0e38)
    x = x.sub_(top).exp_()
    total = x.sum(-1, keepdim=True)
    o = torch.matmul(x.view(B, c["hkv"], G * n, S), v.permute(0, 2, 1, 3)).view(B, c["hkv"], G, n, c["d"]) / total
    o = o.permute(0, 3, 1, 2, 4).reshape(B, n, c["hq"], c["d"])
    s.out.copy_(o[s.req, at])
    if c["lse"]:
        lse = (top + total.log())[..., 0].permute(0, 3, 1, 2).reshape(B, n, c["hq"])
        s.lse.copy_(lse[s.req, at].t())


def _plain_verify(s):
    c = s.case
    B, g, T = c["batch"], c["drafts"], s.ptr[-1]
    r = torch.arange(B, device=DEV)
    i = torch.arange(g, device=DEV)
    there = i < s.count[:, None]
    t = (s.first[:, None] + i).clamp_(max=max(0, T - 1))                     # [B, g]: index of the draft
    x = s.tokens.long()[t] if T else torch.zeros_like(t)
    px = s.p[(s.first + r)[:, None] + torch.minimum(i, s.count[:, None]), x]
    if T:
        qx = s.q[t, x] if s.q is not None else torch.ones_like(px)
        there = there & (s.u_accept[t] * qx < px)
    a = there.long().cumprod(-1).sum(-1)
    p = s.p[s.first + r + a]
    left = p
    if T:
        refused = (a < s.count)[:, None]
        d = (s.first + a).clamp(max=T - 1)
        if s.q is not None:
            left = torch.where(refused, p - s.q[d], p)
        else:
            left = torch.where(refused & (torch.arange(c["vocab"], device=DEV) == s.tokens.long()[d][:, None]), 0.0, p)

    def whole(w):       # multiples of 2^-44: their sums are exact in any order
        return (torch.nan_to_num(w, nan=0.0).clamp(0.0, 1.0) * 2.0 ** 44).long()

    w = whole(left)
    w = torch.where((w.sum(-1) == 0)[:, None], whole(p), w)
    total = w.sum(-1)
    u = (s.u_next * 2.0 ** 24).long().clamp(0, 2 ** 24 - 1)
    goal = (total >> 24) * u + (((total & (2 ** 24 - 1)) * u) >> 24)
    token = (w.cumsum(-1) <= goal[:, None]).sum(-1)
    s.n_accepted.copy_(a)
    s.next_token.copy_(torch.where(total == 0, -1, token))


# --------------------------------------------------------------------------------------- pass

def run(s):
    c, op = s.case, s.case["op"]
    if own:
        lib, ctx = s.context.lib, s.context.handle
        if op == "append":
            lib.c2kv_paged_append(ctx, s.pages, s.table, s.ptr, s.start, s.new_k, s.new_v, turn=s.turn)
        elif op == "gather":
            lib.c2kv_paged_gather(ctx, s.pages, s.table, s.ptr, s.start, s.out_k, s.out_v, turn=s.turn)
        elif op == "attend":
            lib.c2kv_paged_attend(ctx, s.pages, s.table, s.ptr, s.keys, s.q, s.out, lse=s.lse, turn=s.turn,
                                  window=c["window"])
        else:
            lib.c2kv_verify_drafts(ctx, s.ptr, s.tokens, s.p, s.q, s.u_accept, s.u_next, s.n_accepted, s.next_token)
    else:
        {"append": _plain_append, "gather": _plain_gather, "attend": _plain_attend, "verify": _plain_verify}[op](s)
    if op == "append":
        return {"k": s.k, "v": s.v, "k_scale": s.ks, "v_scale": s.vs}
    if op == "gather":
        return {"k": s.out_k, "v": s.out_v}
    if op == "attend":
        return {"out": s.out, "lse": s.lse}
    return {"n_accepted": s.n_accepted, "next_token": s.next_token}


# ------------------------------------------------------------------------------- 64-bit results

def _rope64(x, pos, theta):
    h = x.shape[-1] // 2
    a = pos.double()[:, None, None] * theta ** (-torch.arange(h, dtype=torch.float64, device=DEV) / h)
    z = torch.polar(torch.ones_like(a), a) * torch.complex(x[..., :h].contiguous(), x[..., h:].contiguous())
    return torch.cat([z.real, z.imag], -1)


def _quantise64(x):
    """Scales, and the nearest values of a sign, 4 bits of exponent and 3 of fraction."""
    top = x.abs().amax(-1, keepdim=True)
    scale = torch.where(top < 2.0 ** -100, 0.0, top / 448)
    y = torch.where(scale > 0, x / scale, 0.0)
    step = torch.exp2(torch.floor(torch.log2(y.abs().clamp(min=2.0 ** -6))) - 3)
    return torch.round(y / step) * step, scale[..., 0]


def _exact_rows(s, pages, scales, r, lo, hi):
    """Rows lo .. hi of request r, in 64 bits."""
    P = s.case["page"]
    first, last = lo // P, -(-hi // P)
    pg = s.table[r, first:last].long()
    x = pages[pg].double() * (1 if scales is None else scales[pg].double()[..., None])
    return x.transpose(1, 2).reshape(-1, *x.shape[1:2], x.shape[3])[lo - first * P:hi - first * P]


def _exact_append(c, s):
    got = {"k": s.k.double(), "v": s.v.double()}
    if c["fmt"] == "e4m3":
        got |= {"k_scale": s.ks.double(), "v_scale": s.vs.double()}
    for r, (n, x) in enumerate(s.lens):
        if not n:
            continue
        lo, hi = s.ptr[r], s.ptr[r + 1]
        k, v = s.new_k[lo:hi].double(), s.new_v[lo:hi].double()
        if s.turn is not None:
            k = _rope64(k, s.turn[lo:hi], c["theta"])
        for j in range(x // c["page"], -(-(x + n) // c["page"])):
            a, b = max(x, j * c["page"]), min(x + n, (j + 1) * c["page"])
            pg, o = int(s.table[r, j]), a - j * c["page"]
            for name, y in (("k", k), ("v", v)):
                y = y[a - x:b - x]
                if c["fmt"] == "e4m3":
                    y, scale = _quantise64(y)
                    got[name + "_scale"][pg, :, o:o + b - a] = scale.t()
                got[name][pg, :, o:o + b - a] = y.transpose(0, 1)
    return {**{"k_scale": None, "v_scale": None}, **got}


def _exact_attend(c, s):
    G = c["hq"] // c["hkv"]
    out = torch.zeros((s.ptr[-1], c["hq"], c["d"]), dtype=torch.float64, device=DEV)
    lse = torch.zeros((c["hq"], s.ptr[-1]), dtype=torch.float64, device=DEV)
    for r, (n, x) in enumerate(s.lens):
        if not n:
            continue
        at = slice(s.ptr[r], s.ptr[r + 1])
        q = s.q[at].double()
        if s.turn is not None:
            q = _rope64(q, s.turn[at], c["theta"])
        k, v = _exact_rows(s, s.k, s.ks, r, 0, n + x), _exact_rows(s, s.v, s.vs, r, 0, n + x)
        i, j = torch.arange(x, x + n, device=DEV)[:, None], torch.arange(n + x, device=DEV)
        hidden = (j > i) | ((j <= i - c["window"]) if c["window"] else torch.zeros_like(j > i))
        for h in range(c["hq"]):
            z = q[:, h] @ k[:, h // G].t() / math.sqrt(c["d"])
            z[hidden] = -math.inf
            out[at, h] = torch.softmax(z, -1) @ v[:, h // G]
            if c["lse"]:
                lse[h, at] = torch.logsumexp(z, -1)
    return {"out": out, "lse": lse if c["lse"] else None}


def _exact_verify(c, s):
    """One request after another, in Python's whole numbers and numpy's search."""
    accepted, token = [], []
    for r in range(c["batch"]):
        lo, g = s.ptr[r], s.ptr[r + 1] - s.ptr[r]
        a = 0
        while a < g:
            x = int(s.tokens[lo + a])
            product = s.u_accept[lo + a] * s.q[lo + a, x] if s.q is not None else s.u_accept[lo + a]
            if not bool(product < s.p[lo + r + a, x]):
                break
            a += 1
        p = s.p[lo + r + a].double().cpu().numpy()
        w = p.copy()
        if a < g and s.q is not None:
            w = (s.p[lo + r + a] - s.q[lo + a]).double().cpu().numpy()
        elif a < g:
            w[int(s.tokens[lo + a])] = 0
        w = (w.clip(0, 1) * 2.0 ** 44).astype("int64")
        if not w.any():
            w = (p.clip(0, 1) * 2.0 ** 44).astype("int64")
        run_up = w.cumsum()
        goal = int(run_up[-1]) * int(float(s.u_next[r]) * 2 ** 24) >> 24
        accepted.append(a)
        token.append(int(run_up.searchsorted(goal, side="right")) if run_up[-1] else -1)
    return {name: torch.tensor(x, dtype=torch.int32) for name, x in (("n_accepted", accepted), ("next_token", token))}


def exact(c, seed):
    if c["op"] == "verify":
        return _exact_verify(c, _prepare_verify(c, seed))
    global own
    was, own = own, False
    try:
        s = prepare(c, seed)
    finally:
        own = was
    if c["op"] == "append":
        return _exact_append(c, s)
    if c["op"] == "attend":
        return _exact_attend(c, s)
    k, v = ([_exact_rows(s, x, xs, r, a, a + n) for r, (n, a) in enumerate(s.lens) if n] for x, xs in ((s.k, s.ks), (s.v, s.vs)))
    k, v = torch.cat(k), torch.cat(v)
    return {"k": k if s.turn is None else _rope64(k, s.turn, c["theta"]), "v": v}
