"""Rows moved within the pages of several layers: those that a walk kept (c2kv_paged_keep) and the beams' last pages
(c2kv_paged_reorder), against the oracle.  Copies, so every byte is equal, of what is not moved too."""
import numpy as np
import pytest
import torch

from oracle import branch_oracle as brc
from tests import _paged_helpers as P

pytestmark = pytest.mark.gpu
KINDS = [("bf16", "e4m3", 8, 128), ("bf16", "native", 8, 128), ("bf16", "native", 3, 64), ("bf16", "e4m3", 5, 64), ("f32", "native", 2, 128),
         ("f32", "e4m3", 4, 64), ("bf16", "e4m3", 1, 64)]


class _Layers:
    """Pages of random bytes in every layer, pages with gaps between them where `gap`."""

    def __init__(self, rng, kind, layers, n_pages, size, gap=0):
        dtype, fmt, hkv, d = kind
        self.eb = 1 if fmt == "e4m3" else 2 if dtype == "bf16" else 4
        self.hkv, self.d, self.n = hkv, d, n_pages
        dt = P.E4M3 if fmt == "e4m3" else P.TDT[dtype]
        self.host, self.dev = {}, {}
        for name in ("k", "v") + (("k_scale", "v_scale") if fmt == "e4m3" else ()):
            inner = (hkv, size, d * self.eb) if name in "kv" else (hkv, size, 4)
            self.host[name] = rng.integers(0, 255, (layers, n_pages + gap, *inner), dtype=np.uint8)
            x = torch.from_numpy(self.host[name]).cuda()
            self.dev[name] = x.view(torch.uint8 if name in "kv" and fmt == "e4m3" else dt if name in "kv" else torch.float32)
            if name not in "kv":
                self.dev[name] = self.dev[name].squeeze(-1)
            if name in "kv" and fmt == "e4m3":
                self.dev[name] = self.dev[name].view(dt)
        if gap:                                          # every layer's pages among another's: a longer stride
            self.dev = {k: x.transpose(0, 1).contiguous().transpose(0, 1) for k, x in self.dev.items()}
        self.pages = P.lib().make_layers(*(self.dev.get(n)[:, :n_pages] if n in self.dev else None for n in ("k", "v", "k_scale", "v_scale")))

    def same(self, want):
        for name, x in self.dev.items():
            got = x.contiguous().view(torch.uint8).cpu().numpy().reshape(self.host[name].shape)
            assert np.array_equal(got, want[name]), name


def _ctx(kind):
    return P.context(kind[0], 2 * kind[2], kind[2], kind[3])


def _tables(rng, starts, counts, size, n_spare=2):
    """Tables with pages for rows start .. start + count, -1 before and behind."""
    need = [list(range(s // size, -(-(s + n) // size))) if n else [] for s, n in zip(starts, counts)]
    total = sum(map(len, need)) + n_spare
    order = rng.permutation(total).tolist()
    table = np.full((len(starts), max([1] + [h[-1] + 1 for h in need if h]) + 1), -1, np.int32)
    for r, h in enumerate(need):
        for j in h:
            table[r, j] = order.pop()
    return table, total


class _Keep:
    def __init__(self, kind, layers, size, paths, starts, nodes, gap=0, seed=0):
        rng = np.random.default_rng(seed)
        self.size, self.paths, self.starts, self.nodes = size, paths, starts, nodes
        self.table_np, n = _tables(rng, starts, nodes, size)
        self.pages = _Layers(rng, kind, layers, n, size, gap)
        self.table = torch.from_numpy(self.table_np).cuda()
        self.ptr = np.cumsum([0] + list(nodes)).tolist()
        full = sum((list(p) + [-1] * (m - len(p)) for p, m in zip(paths, nodes)), [])
        self.path = torch.tensor(full or [0], dtype=torch.int32, device="cuda")
        self.n = torch.tensor([max(0, len(p) - 1) for p in paths], dtype=torch.int32, device="cuda")

    def run(self, ctx):
        P.lib().c2kv_paged_keep(ctx, self.pages.pages, self.table, self.ptr, self.starts, self.path, self.n)

    def check(self, paths=None):
        want = {k: x.copy() for k, x in self.pages.host.items()}
        for x in want.values():
            for layer in x:
                for r, p in enumerate(paths or self.paths):
                    if len(p):
                        brc.keep(layer, self.table_np[r], self.starts[r], p, self.size)
        self.pages.same(want)


def _path(rng, nodes, kept):
    return [0] + sorted(rng.choice(np.arange(1, nodes), kept - 1, replace=False).tolist()) if nodes else []


@pytest.mark.parametrize("size", [16, 64, 128])
@pytest.mark.parametrize("kind", KINDS, ids=lambda k: "-".join(map(str, k)))
def test_keep(kind, size):
    """Paths of one node, all nodes, rows that others move into, across pages, beside requests without a tree."""
    rng = np.random.default_rng(size)
    nodes = [20, 1, 0, 16, 70, 33, 40]
    paths = [_path(rng, 20, 5), [0], [], list(range(16)), _path(rng, 70, 30), [0, 1, 2, 30, 31, 32], [0] + list(range(2, 40))]
    starts = [0, 7, 5, 31, size - 3, 2 * size, 111]
    ctx = _ctx(kind)
    try:
        k = _Keep(kind, 3, size, paths, starts, nodes)
        k.run(ctx)
        P.lib().c2kv_sync(ctx)
        k.check()
    finally:
        P.lib().c2kv_destroy(ctx)


@pytest.mark.parametrize("layers,batch,gap", [(1, 1, 0), (4, 2, 0), (5, 40, 0), (100, 3, 0), (50, 300, 0), (6, 5, 3)])
def test_keep_in_many_layers_and_requests(layers, batch, gap):
    rng = np.random.default_rng(layers)
    kind = ("bf16", "e4m3", 2, 64)
    nodes = rng.integers(0, 25, batch).tolist()
    paths = [_path(rng, n, int(rng.integers(1, min(n, 7) + 1))) if n else [] for n in nodes]
    ctx = _ctx(kind)
    try:
        k = _Keep(kind, layers, 16, paths, rng.integers(0, 60, batch).tolist(), nodes, gap)
        k.run(ctx)
        P.lib().c2kv_sync(ctx)
        k.check()
    finally:
        P.lib().c2kv_destroy(ctx)


def test_keep_the_most_nodes():
    rng = np.random.default_rng(5)
    kind = ("bf16", "native", 2, 64)
    ctx = _ctx(kind)
    try:
        k = _Keep(kind, 2, 32, [_path(rng, 512, 200), [0] + list(range(2, 512)), list(range(512))], [3, 64, 10], [512, 512, 512])
        k.run(ctx)
        P.lib().c2kv_sync(ctx)
        k.check()
    finally:
        P.lib().c2kv_destroy(ctx)


def test_keep_far_down_a_long_request():
    """Rows near the most that a request may have: the table's index, not a row's memory, is far."""
    kind = ("bf16", "native", 2, 64)
    start = (1 << 26) - 40
    ctx = _ctx(kind)
    try:
        k = _Keep(kind, 1, 128, [[0, 3, 9, 11]], [start], [40])
        assert k.table_np.shape[1] > 1 << 18
        k.run(ctx)
        P.lib().c2kv_sync(ctx)
        k.check()
    finally:
        P.lib().c2kv_destroy(ctx)


def test_keep_refuses_paths_and_pages():
    """Counts and entries that are none: reported; what is refused stays as it was, and all that follows it."""
    kind = ("bf16", "e4m3", 2, 64)
    bad = [([0, 5, 5, 7], 3, [0, 5]), ([0, 5, 20, 7], 3, [0, 5]), ([0, 5, 4, 9], 3, [0, 5]), ([0, 5, 7, 9], 20, []), ([0, 5, 7, 9], -1, []),
           ([-1, 5, 7, 9], 3, []), ([0, -1, 7, 9], 3, [0]), ([2, 5, 7, 9], 3, [2, 5, 7, 9])]
    for path, n, kept in bad:
        ctx = _ctx(kind)
        try:
            k = _Keep(kind, 2, 16, [[0, 5, 7, 9], [0, 4]], [9, 3], [20, 6])
            k.path[:4] = torch.tensor(path, dtype=torch.int32)
            k.n[0] = n
            k.run(ctx)
            if kept == path:                             # (a path may begin anywhere, as long as it rises)
                P.lib().c2kv_sync(ctx)
            else:
                with pytest.raises(P.lib().C2KVError) as e:
                    P.lib().c2kv_sync(ctx)
                assert e.value.status == P.lib().ERR_DEVICE_BOUNDS
            k.check([kept, [0, 4]])
        finally:
            P.lib().c2kv_destroy(ctx)
    ctx = _ctx(kind)
    try:
        k = _Keep(kind, 2, 16, [[0, 2, 8], [0, 4]], [9, 3], [20, 6])
        k.table[0, 1] = k.pages.n                        # the page of nodes 7 and on
        k.run(ctx)
        with pytest.raises(P.lib().C2KVError) as e:
            P.lib().c2kv_sync(ctx)
        assert e.value.status == P.lib().ERR_DEVICE_BOUNDS
        k.check([[0, 2], [0, 4]])
    finally:
        P.lib().c2kv_destroy(ctx)


class _Beams:
    def __init__(self, kind, layers, size, width, rows, parents, gap=0, seed=0, table_width=None):
        rng = np.random.default_rng(seed)
        self.size, self.rows, self.parents, self.width = size, rows, parents, width
        n = len(rows) * width * 2 + 3
        wide = table_width or max(rows) // size + 2
        order = rng.permutation(n)
        table = rng.integers(0, n, (len(rows) * width, wide)).astype(np.int32)
        for b in range(len(table)):                      # the page that the next rows go to is each beam's own, and the one behind
            at = rows[b // width] // size
            table[b, at:at + 2] = order[2 * b:2 * b + 2][:wide - at]
        self.table_np = table
        self.pages = _Layers(rng, kind, layers, n, size, gap)
        self.table = torch.from_numpy(table).cuda()
        self.out = torch.full_like(self.table, -5)
        self.parent = torch.tensor(parents, dtype=torch.int32, device="cuda").view(len(rows), width)

    def run(self, ctx):
        P.lib().c2kv_paged_reorder(ctx, self.pages.pages, self.table, self.rows, self.parent, self.out)

    def check(self, parents=None):
        want = {k: x.copy() for k, x in self.pages.host.items()}
        for r, of in enumerate(parents or self.parents):
            rows = slice(r * self.width, (r + 1) * self.width)
            table, copies = brc.reorder(self.table_np[rows], of, self.rows[r], self.size)
            assert np.array_equal(self.out[rows].cpu().numpy(), table), r
            for a, b, n in copies:
                for x in want.values():
                    x[:, b, :, :n] = x[:, a, :, :n]
        self.pages.same(want)


def _check_beams(kind, *args, **more):
    ctx = _ctx(kind)
    try:
        b = _Beams(kind, *args, **more)
        b.run(ctx)
        P.lib().c2kv_sync(ctx)
        b.check()
    finally:
        P.lib().c2kv_destroy(ctx)


@pytest.mark.parametrize("size", [16, 64, 128])
@pytest.mark.parametrize("kind", KINDS, ids=lambda k: "-".join(map(str, k)))
def test_reorder(kind, size):
    """All of one, none moved, turned round, one in two; pages that are empty, full, of one row, of all but one."""
    parents = [[0, 0, 0, 0, 0], [0, 1, 2, 3, 4], [4, 3, 2, 1, 0], [1, 1, 3, 3, 3], [4, 4, 4, 4, 4], [-1, 0, -1, 0, 2], [2, -1, 2, 2, -1], [0, 0, 1, 1, 2]]
    _check_beams(kind, 3, size, 5, [size + 5, 3 * size - 1, size + 1, 7, 2 * size, 9, 2 * size + size // 2, 0], parents)


@pytest.mark.parametrize("layers,batch,width,gap", [(1, 1, 1, 0), (4, 1, 64, 0), (5, 40, 3, 0), (100, 2, 4, 0), (49, 260, 2, 0), (3, 2, 6, 4)])
def test_reorder_of_many(layers, batch, width, gap):
    rng = np.random.default_rng(width)
    kind = ("bf16", "e4m3", 2, 64)
    parents = rng.integers(-1, width, (batch, width)).tolist()
    _check_beams(kind, layers, 16, width, rng.integers(0, 70, batch).tolist(), parents, gap=gap)


def test_reorder_at_the_tables_end():
    """Rows that end with the table: no page behind them."""
    _check_beams(("bf16", "native", 2, 64), 2, 16, 3, [48, 47], [[2, 2, 0], [1, 1, 1]], table_width=3)


def test_reorder_refuses_parents_and_pages():
    kind = ("bf16", "e4m3", 2, 64)
    ctx = _ctx(kind)
    try:
        b = _Beams(kind, 2, 16, 3, [20, 9], [[0, 0, 1], [2, 2, 2]])
        b.parent[0] = torch.tensor([3, 0, -2], dtype=torch.int32)
        b.run(ctx)
        with pytest.raises(P.lib().C2KVError) as e:
            P.lib().c2kv_sync(ctx)
        assert e.value.status == P.lib().ERR_DEVICE_BOUNDS
        b.check([[-1, 0, -1], [2, 2, 2]])
    finally:
        P.lib().c2kv_destroy(ctx)
    ctx = _ctx(kind)
    try:
        b = _Beams(kind, 2, 16, 3, [20, 9], [[0, 0, 1], [2, 2, 2]])
        own = b.table_np[2, 1]                           # the page that beam 1 would copy into
        b.table[2, 1] = b.table_np[2, 1] = -1
        b.run(ctx)
        with pytest.raises(P.lib().C2KVError) as e:
            P.lib().c2kv_sync(ctx)
        assert e.value.status == P.lib().ERR_DEVICE_BOUNDS
        want, copies = brc.reorder(b.table_np[:3], [0, 0, 1], 20, 16)
        assert np.array_equal(b.out[:3].cpu().numpy(), want) and copies[0][1] == -1
        # the page itself is as it was
        got = b.pages.dev["k"].view(torch.uint8).cpu().numpy().reshape(b.pages.host["k"].shape)
        assert np.array_equal(got[:, own], b.pages.host["k"][:, own])
    finally:
        P.lib().c2kv_destroy(ctx)


def test_captured_and_beside_other_streams():
    """Graphs of both calls, replayed on two streams with other paths and parents in place."""
    c2kv, kind = P.lib(), ("bf16", "e4m3", 2, 64)
    ctx, side = _ctx(kind), [torch.cuda.Stream(), torch.cuda.Stream()]
    try:
        rng = np.random.default_rng(3)
        k = _Keep(kind, 5, 16, [[0, 5, 7, 9], [0, 4]], [9, 3], [20, 6])
        b = _Beams(kind, 5, 16, 4, [20, 9], [[0, 0, 1, 1], [2, 2, 2, 0]])
        graphs = []
        for call, s in zip((k, b), side):
            torch.cuda.synchronize()
            c2kv.c2kv_set_stream(ctx, s)
            graphs.append(torch.cuda.CUDAGraph())
            with torch.cuda.graph(graphs[-1], stream=s, capture_error_mode="thread_local"):
                call.run(ctx)
        k.paths = [[0, 1, 8, 13], [0, 5]]
        k.path.copy_(torch.tensor(k.paths[0] + [-1] * 16 + k.paths[1] + [-1] * 4, dtype=torch.int32))
        b.parents = rng.integers(0, 4, (2, 4)).tolist()
        b.parent.copy_(torch.tensor(b.parents, dtype=torch.int32))
        torch.cuda.synchronize()
        for g, s in zip(graphs, side):
            with torch.cuda.stream(s):
                g.replay()
        torch.cuda.synchronize()
        k.check()
        b.check()
        c2kv.c2kv_sync(ctx)
        del graphs
    finally:
        c2kv.c2kv_destroy(ctx)
