"""Attention of trees of tokens over pages (c2kv_paged_attend_tree) against fp64 over the rows that the pages
stand for.

Tolerances: those of the attention of tokens that follow one another, which differs in what a row sees only:
atol = rtol = 2e-2 for bf16 (lse 2e-2) and 1e-5 for fp32."""
import numpy as np
import pytest
import torch

from oracle import branch_oracle as brc
from oracle import paged_oracle as orc
from tests import _paged_helpers as P
from tests._tree_helpers import chain, random_tree, ranges, star

pytestmark = pytest.mark.gpu
TOL = {"bf16": 2e-2, "f32": 1e-5}


def _device(parents):
    return torch.tensor(sum(parents, []) or [0], dtype=torch.int32, device="cuda")


_beside = False


@pytest.fixture(autouse=True, params=["alone", "beside_others"])
def _work_beside(request):
    """Calls of little work go another way than those of much: each test runs as it is, and with a large tree as one
    more request, of more rows and keys than the first way takes."""
    global _beside
    _beside = request.param != "alone"
    yield
    _beside = False


class _Call:
    """A call over pages of random rows: trees (parents, rows before them) per request."""

    def __init__(self, dtype, fmt, hq, hkv, d, size, trees, window=0, turn=True, theta=1.0e4, seed=1, edit=None, strided=False):
        rng = np.random.default_rng(seed)
        self.dtype, self.window, self.trees, self.theta = dtype, window, trees, theta
        self.ctx = P.context(dtype, hq, hkv, d, theta)
        self.keys = [x + len(t) for t, x in trees]
        every = list(trees)
        if _beside:                                      # 40 million values of K, counted for eight rows of queries
            every.append((star(512), max(0, 40000000 // (512 * hq // hkv // 8 * hkv * d) - 512)))
        every_keys = [x + len(t) for t, x in every]
        self.pg = P.Paged(rng, dtype, fmt, hkv, d, size, every_keys)
        self.pg.fill_rows(rng)
        if edit:
            edit(self.pg)
        table = torch.from_numpy(self.pg.table_np).cuda()
        self.pages = self.pg.pages()
        every_ptr = ranges([t for t, _ in every])
        T = every_ptr[-1]
        q = torch.from_numpy(rng.standard_normal((T, hq, d)).astype(np.float32)).to(P.TDT[dtype]).cuda()
        if strided:                                      # rows of a fused projection
            wide = torch.full((T, hq + 2 * hkv, d), float("nan"), device="cuda", dtype=P.TDT[dtype])
            wide[:, :hq] = q
            q = wide[:, :hq]
        pos = torch.from_numpy(rng.integers(0, 200000, max(T, 1)).astype(np.int32)).cuda() if turn else None
        parent = _device([t for t, _ in every])
        out = torch.full((T, hq, d), 7.0, device="cuda", dtype=P.TDT[dtype])
        lse = torch.full((hq, T), 7.0, device="cuda")
        self.every = table, every_ptr, every_keys, parent, q, out, lse, pos
        # of the trees alone
        self.table, self.ptr = table[:len(trees)], every_ptr[:len(trees) + 1]
        n = self.ptr[-1]
        self.parent, self.q, self.out, self.lse = parent[:max(n, 1)], q[:n], out[:n], lse[:, :n]
        self.pos = pos[:max(n, 1)] if turn else None

    def run(self):
        table, ptr, keys, parent, q, out, lse, pos = self.every
        P.lib().c2kv_paged_attend_tree(self.ctx, self.pages, table, ptr, keys, parent, q, out, lse=lse, turn=pos, window=self.window)

    def want(self, trees=None):
        q64 = self.q.float().cpu().numpy().astype(np.float64)
        if self.pos is not None:
            q64 = orc.turned(q64, self.pos.cpu().numpy()[:len(q64)], self.theta)
        hk, hv = self.pg.host()
        T, hq, d = q64.shape
        out, lse = np.zeros((T, hq, d)), np.zeros((hq, T))
        n_pages, size, table = self.pg.k.shape[0], self.pg.size, self.table.cpu().numpy()
        for r, (tree, _) in enumerate(trees or self.trees):
            at = slice(self.ptr[r], self.ptr[r + 1])
            pages = np.array([table[r, j // size] for j in range(self.keys[r])], int)
            there = (pages >= 0) & (pages < n_pages)
            use = np.where(there, pages, 0)
            k, v = (x[use, :, np.arange(self.keys[r]) % size] for x in (hk, hv))
            with np.errstate(invalid="ignore"):
                out[at], lse[:, at] = brc.attend_tree(q64[at], k, v, tree, self.window, there)
        return out, lse

    def check(self, trees=None, more=(0.0, 0.0)):
        """`more`: what the outputs and the lse may be off beside TOL."""
        out, lse = self.out.float().cpu().numpy(), self.lse.cpu().numpy()
        want, want_l = self.want(trees)
        tol = TOL[self.dtype]
        for same in (np.isnan, np.isposinf, np.isneginf):
            assert np.array_equal(same(out), same(want)) and np.array_equal(same(lse), same(want_l))
        fine = np.isfinite(want)
        assert np.all((np.abs(out - want) <= more[0] + tol + tol * np.abs(want))[fine])
        fine = np.isfinite(want_l)
        assert np.all(np.abs(lse[fine] - want_l[fine]) <= more[1] + tol * (1 + np.abs(want_l[fine]) * (self.dtype == "f32")))

    def sync(self):
        P.lib().c2kv_sync(self.ctx)

    def close(self):
        P.lib().c2kv_destroy(self.ctx)


def _run(*args, **more):
    call = _Call(*args, **more)
    try:
        call.run()
        call.sync()
        call.check()
    finally:
        call.close()


SHAPES = [  # dtype, fmt, hq, hkv, d
    ("bf16", "e4m3", 32, 8, 128), ("bf16", "native", 32, 8, 128), ("bf16", "e4m3", 8, 8, 128), ("bf16", "e4m3", 16, 2, 128),
    ("bf16", "native", 28, 4, 128), ("bf16", "e4m3", 28, 4, 64), ("bf16", "native", 8, 2, 64), ("bf16", "e4m3", 20, 1, 128),
    ("bf16", "native", 4, 4, 64), ("f32", "native", 16, 4, 64), ("f32", "e4m3", 8, 2, 128), ("f32", "native", 6, 2, 128),
    ("f32", "e4m3", 4, 4, 64),
]
R = np.random.default_rng(11)
TREES = {  # page size, (parents, rows before) per request
    "one": (16, [([-1], 0)]),
    "ragged": (16, [(chain(5), 37), ([], 12), (star(9), 0), (random_tree(R, 16), 130), ([-1], 0), ([], 0), (random_tree(R, 11, roots=0.3), 3)]),
    "few": (64, [(random_tree(R, 3), 700), (star(2), 63), ([-1], 64), (random_tree(R, 4, roots=0.5), 1300)]),
    "levels": (128, [(random_tree(R, 64, near=12), 129), (random_tree(R, 33, near=5), 300), (random_tree(R, 70), 0)]),
    "large": (32, [(random_tree(R, 300, near=40), 40), (random_tree(R, 130), 513), ([-1], 31)]),
}


@pytest.mark.parametrize("trees", TREES)
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "-".join(map(str, s)))
def test_shapes(shape, trees):
    _run(*shape, *TREES[trees])


@pytest.mark.parametrize("shape", [SHAPES[i] for i in (0, 1, 2, 6, 8, 9, 10, 12)], ids=lambda s: "-".join(map(str, s)))
def test_the_most_nodes(shape):
    """512 nodes: one deep, one wide, one of both, at rows that do not end with a page or a key tile."""
    r = np.random.default_rng(3)
    _run(*shape, 64, [(chain(512), 45), (star(512), 1)])
    _run(*shape, 64, [(random_tree(r, 512, near=100), 200), (random_tree(r, 511, roots=0.1), 0)])


@pytest.mark.parametrize("window", [1, 2, 5, 40, 130, 2 ** 31 - 1])
@pytest.mark.parametrize("shape", [SHAPES[i] for i in (0, 1, 2, 6, 8, 9, 10, 11)], ids=lambda s: "-".join(map(str, s)))
def test_window(shape, window):
    """Windows within a path, up to its root, and into the rows before the tree."""
    r = np.random.default_rng(5)
    _run(*shape, 32, [(chain(6), 300), (random_tree(r, 15, near=3), 33), (chain(3), 0), ([-1], 77)], window=window)
    _run(*shape, 32, [(random_tree(r, 90, near=4), 300), (random_tree(r, 140, near=2), 10)], window=window)


@pytest.mark.parametrize("n", [4, 16, 100])
@pytest.mark.parametrize("shape", [SHAPES[0], SHAPES[1], SHAPES[9]], ids=lambda s: "-".join(map(str, s)))
def test_pages_that_a_window_left_behind(shape, n):
    """Pages whose rows no node sees any more may be gone from the table."""
    def edit(pg):
        pg.table_np[0, :(600 - 37 + 1) // 16] = -1
    _run(*shape, 16, [(random_tree(np.random.default_rng(2), n), 600)], window=37, edit=edit)


@pytest.mark.parametrize("n", [1, 3, 13, 60, 200])
@pytest.mark.parametrize("window", [0, 9])
@pytest.mark.parametrize("shape", [SHAPES[i] for i in (0, 1, 5, 6, 9, 10)], ids=lambda s: "-".join(map(str, s)))
def test_a_chain_is_what_follows_one_another(shape, n, window):
    call = _Call(*shape, 32, [(chain(n), 500), (chain(n), 0)], window=window)
    try:
        call.run()
        out, lse = torch.empty_like(call.out), torch.empty_like(call.lse)
        P.lib().c2kv_paged_attend(call.ctx, call.pages, call.table, call.ptr, call.keys, call.q, out, lse=lse, turn=call.pos, window=window)
        call.sync()
        # (not the same kernels everywhere.  Each is within tol + tol |w| of the exact w, so they are within twice that
        # of one another, and |w| is at most (|x| + tol) / (1 - tol) of either; scores' sums alike, of fp32 by lse's own)
        tol = TOL[shape[0]]
        for x, y in ((out.double(), call.out.double()), (lse.double(), call.lse.double())):
            assert torch.equal(x.isinf(), y.isinf())
            x, y = x[x.isfinite()], y[y.isfinite()]
            assert ((x - y).abs() <= 2 * tol * (1 + (x.abs() + tol) / (1 - tol))).all()
    finally:
        call.close()


@pytest.mark.parametrize("shape", [SHAPES[i] for i in (0, 1, 6, 10)], ids=lambda s: "-".join(map(str, s)))
def test_long_rows_are_split_and_joined(shape):
    r = np.random.default_rng(6)
    _run(*shape, 128, [(random_tree(r, 9), 9000), (random_tree(r, 2), 5000)], turn=False)
    _run(*shape, 128, [(random_tree(r, 40), 9000)])


@pytest.mark.parametrize("shape", [SHAPES[0], SHAPES[1], SHAPES[9]], ids=lambda s: "-".join(map(str, s)))
def test_many_requests(shape):
    r = np.random.default_rng(2)
    _run(*shape, 16, [(random_tree(r, int(r.integers(0, 5))), int(r.integers(0, 60))) for _ in range(290)])
    _run(*shape, 16, [(random_tree(r, int(r.integers(20, 40))), int(r.integers(0, 60))) for _ in range(40)])


@pytest.mark.parametrize("n", [7, 90])
@pytest.mark.parametrize("shape", [SHAPES[0], SHAPES[6], SHAPES[9]], ids=lambda s: "-".join(map(str, s)))
def test_rows_of_a_fused_projection(shape, n):
    _run(*shape, 64, [(random_tree(np.random.default_rng(8), n), 100)], strided=True)


BAD = [("bf16", "native", 32, 8, 128), ("bf16", "native", 8, 2, 64), ("bf16", "e4m3", 8, 2, 128), ("f32", "native", 16, 4, 64),
       ("f32", "e4m3", 8, 2, 128), ("f32", "native", 4, 4, 128)]


@pytest.mark.parametrize("window", [0, 4])
@pytest.mark.parametrize("n,x", [(6, 100), (15, 3), (15, 700), (120, 100), (300, 500)])
@pytest.mark.parametrize("shape", BAD, ids=lambda s: "-".join(map(str, s)))
def test_values_that_are_not_finite(shape, n, x, window):
    """Values of V that are not finite, in rows of the tree and before it: they belong to the nodes that see them,
    channel by channel; 8-bit rows with a scale that is NaN to all channels of them."""
    tree = random_tree(np.random.default_rng(n), n, near=6)

    def edit(pg):
        for key, channel, value in ((x + n // 2, 5, float("inf")), (x + n - 1, 6, float("nan")), (x + n // 3, 5, -float("inf")),
                                    (x + 1, 9, float("inf")), (x - 2, 9, float("nan")), (0, 2, -float("inf"))):
            page, at = int(pg.table_np[0, key // 32]), key % 32
            if pg.vs is None:
                pg.v[page, :, at, channel] = value
            elif np.isnan(value):
                pg.vs[page, 1, at] = value
    _run(*shape, 32, [(tree, x), (chain(3), 20)], window=window, edit=edit)


@pytest.mark.parametrize("n,x", [(6, 100), (15, 3), (120, 100)])
@pytest.mark.parametrize("shape", BAD, ids=lambda s: "-".join(map(str, s)))
def test_keys_that_are_not_finite(shape, n, x):
    """A key that is NaN makes NaN of every node that sees it, and leaves its siblings alone."""
    tree = random_tree(np.random.default_rng(n), n, near=6)

    def edit(pg):
        key = x + n // 2
        page, at = int(pg.table_np[0, key // 32]), key % 32
        if pg.ks is None:
            pg.k[page, :, at, 3] = float("nan")
        else:
            pg.ks[page, :, at] = float("nan")
    call = _Call(*shape, 32, [(tree, x)], edit=edit)
    try:
        call.run()
        call.sync()
        out = call.out.float().cpu().numpy()
        want, _ = call.want()
        touched = brc.sees(tree, n + x)[:, x + n // 2]
        assert np.array_equal(np.isnan(out).all((1, 2)), touched) and np.array_equal(np.isnan(out).any((1, 2)), touched)
        tol = TOL[shape[0]]
        assert np.all(np.abs(out[~touched] - want[~touched]) <= tol + tol * np.abs(want[~touched]))
    finally:
        call.close()


@pytest.mark.parametrize("n", [12, 100])
@pytest.mark.parametrize("shape", [SHAPES[i] for i in (0, 1, 9, 12)], ids=lambda s: "-".join(map(str, s)))
def test_refused_pages(shape, n):
    """Page numbers that are none, within the tree and before it: reported, their rows unseen; a node that sees
    no other gives zeros."""
    def edit(pg):
        pg.table_np[0, 1] = pg.k.shape[0]
        pg.table_np[0, 3] = -7
        pg.table_np[1, 0] = -1
    call = _Call(*shape, 16, [(random_tree(np.random.default_rng(n), n, roots=0.2), 40), (star(5), 0)], edit=edit)
    try:
        call.run()
        with pytest.raises(P.lib().C2KVError) as e:
            call.sync()
        assert e.value.status == P.lib().ERR_DEVICE_BOUNDS
        call.check()
        assert not call.out[n:].any() and torch.isneginf(call.lse[:, n:]).all()
    finally:
        call.close()


@pytest.mark.parametrize("n", [9, 100])
@pytest.mark.parametrize("shape", [SHAPES[i] for i in (0, 1, 9, 12)], ids=lambda s: "-".join(map(str, s)))
def test_refused_parents(shape, n):
    """Parents that are not before their children: reported, the node taken for a root."""
    tree = random_tree(np.random.default_rng(n), n, near=5)
    call = _Call(*shape, 16, [(tree, 40)])
    taken = list(tree)
    try:
        for at, value in ((2, 2), (4, 7), (5, -2), (7, 2 ** 31 - 1), (8, -2 ** 31)):
            call.parent[at] = value
            taken[at] = -1
        call.run()
        with pytest.raises(P.lib().C2KVError) as e:
            call.sync()
        assert e.value.status == P.lib().ERR_DEVICE_BOUNDS
        call.check([(taken, 40)])
    finally:
        call.close()


@pytest.mark.parametrize("n", [6, 100])
@pytest.mark.parametrize("shape", [SHAPES[1], SHAPES[9]], ids=lambda s: "-".join(map(str, s)))
def test_nodes_whose_every_score_is_minus_infinity(shape, n):
    """No row before the tree, and a root's key that every query meets at -inf: the root alone is NaN."""
    call = _Call(*shape, 16, [(star(n), 0)], turn=False)
    try:
        call.q[..., 0] = 1.0
        page = int(call.pg.table_np[0, 0])
        call.pg.k[page, :, 0, 0] = -float("inf")
        call.run()
        call.sync()
        out, lse = call.out.float(), call.lse
        assert out[0].isnan().all() and torch.isneginf(lse[:, 0]).all()
        v = call.pg.host()[1]
        for i in range(1, n):                            # the root's weight is nothing: the node's own value
            own = v[int(call.pg.table_np[0, i // 16]), :, i % 16].repeat(shape[2] // shape[3], 0)
            assert np.all(np.abs(out[i].cpu().numpy() - own) <= TOL[shape[0]] * (1 + np.abs(own)))
    finally:
        call.close()


def test_same_result_twice():
    r = np.random.default_rng(8)
    for n in (13, 90):
        call = _Call("bf16", "e4m3", 32, 8, 128, 64, [(random_tree(r, n), 6000), (chain(2), 30)])
        try:
            first = None
            for _ in range(20):
                call.out.zero_()
                call.run()
                call.sync()
                first = call.out.clone() if first is None else first
                assert torch.equal(call.out, first)
        finally:
            call.close()


@pytest.mark.parametrize("shape", [SHAPES[0], SHAPES[1], SHAPES[9], SHAPES[10]], ids=lambda s: "-".join(map(str, s)))
@pytest.mark.parametrize("n", [5, 90])
def test_captured_on_another_stream(shape, n):
    """A graph of the call replayed with other parents, larger calls on the context's stream in between."""
    r = np.random.default_rng(n)
    side, other = torch.cuda.Stream(), torch.cuda.Stream()
    call, large = (_Call(*shape, 32, [(random_tree(r, m), x), (chain(2), 10)]) for m, x in ((n, 3000), (2 * n, 9000)))
    c2kv = P.lib()
    try:
        for c in (call, large):
            c.run()
            c.sync()
        torch.cuda.synchronize()
        c2kv.c2kv_set_stream(call.ctx, side)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side, capture_error_mode="thread_local"):
            call.run()
        tree = random_tree(r, n, near=3)
        call.parent[:n] = torch.tensor(tree, device="cuda", dtype=torch.int32)
        call.out.zero_()
        torch.cuda.synchronize()
        for _ in range(5):
            with torch.cuda.stream(other):
                graph.replay()
            large.run()
        torch.cuda.synchronize()
        call.check([(tree, 3000), (chain(2), 10)])
        large.check()
        del graph
    finally:
        call.close()
        large.close()


@pytest.mark.parametrize("n,x", [(70, 30), (70, 100), (70, 170), (70, 700), (40, 2000)])
@pytest.mark.parametrize("shape", [("bf16", "native", 32, 8, 128), ("bf16", "native", 8, 2, 64)], ids=lambda s: "-".join(map(str, s)))
def test_infinite_keys_and_values_over_any_number_of_tiles(shape, n, x):
    """Infinities of K (scores of -inf and of inf's own sign) and of V, one key tile to seventeen: odd and even numbers."""
    tree = random_tree(np.random.default_rng(n), n, near=8)

    def edit(pg):
        for key in (3, x - 5, x + 2):
            pg.k[int(pg.table_np[0, key // 32]), :, key % 32, 1] = -float("inf")
        for key, value in ((9, float("inf")), (x - 9, float("nan")), (x + 5, -float("inf"))):
            pg.v[int(pg.table_np[0, key // 32]), :, key % 32, 4] = value
    call = _Call(*shape, 32, [(tree, x)], turn=False, edit=edit)
    try:
        call.q[..., 1] = 0.5
        call.run()
        call.sync()
        call.check()
    finally:
        call.close()


@pytest.mark.parametrize("at", [32, 64, 96, 128, 160, 192, 224, 288, 480])
@pytest.mark.parametrize("shape", [("bf16", "native", 32, 8, 128), ("bf16", "native", 8, 2, 64), ("bf16", "e4m3", 32, 8, 128)], ids=lambda s: "-".join(map(str, s)))
def test_scores_that_rise_within_a_tile(shape, at):
    """Keys from `at` on outweigh those before by 2^15, which hold values 2^13 times theirs (16-bit pages): both count, and
    weights formed before the rise keep their share."""
    n, x, d = 20, 500, shape[4]
    rise = 15 * np.log(2) * np.sqrt(d)

    def edit(pg):
        for key in range(x + n):
            page, row = int(pg.table_np[0, key // 32]), key % 32
            if pg.ks is None:
                pg.k[page, :, row, 0] = rise if key >= at else 0.0
                if key < at:
                    pg.v[page, :, row] *= 2.0 ** 13
            elif key >= at:
                pg.k.view(torch.uint8)[page, :, row, 0] = 0x7e                    # (448)
                pg.ks[page, :, row] = rise / 448
    call = _Call(*shape, 32, [(star(n), x)], turn=False, edit=edit)
    try:
        call.q[..., 0] = 1.0
        call.run()
        call.sync()
        # 8-bit rows whose scale is raised have all their channels raised, and scores of a hundred and more.  Operands made
        # of codes and queries have f16's eleven bits, each off by 2^-11 at most, so a score is off by e = 2^-10 of the sum of
        # its products' magnitudes, and so may its row's lse be.  Of weights that are off by factors of exp(-e) .. exp(e),
        # out' - out = sum w_j (exp(e_j) - 1) (v_j - out) / sum w_j exp(e_j), at most (exp(2 e) - exp(e)) sum w_j |v_j - out|.
        more = 0.0, 0.0
        if call.pg.ks is not None:
            k, v = (y[call.pg.table_np[0, :-(-(x + n) // 32)]].swapaxes(1, 2).reshape(-1, shape[3], d)[:x + n] for y in call.pg.host())
            q = call.q.float().cpu().numpy().astype(np.float64).reshape(n, shape[3], -1, d)
            score = np.where(brc.sees(star(n), x + n)[:, None, None], np.einsum("nhgd,khd->nhgk", q, k) / np.sqrt(d), -np.inf)
            e = 2.0 ** -10 * np.einsum("nhgd,khd->nhgk", np.abs(q), np.abs(k)).max(-1) / np.sqrt(d)
            w = np.exp(score - score.max(-1, keepdims=True))
            w /= w.sum(-1, keepdims=True)
            out = np.einsum("nhgk,khd->nhgd", w, v)
            spread = np.stack([np.einsum("nhg,nhgd->nhgd", w[..., j], np.abs(v[j][None, :, None] - out)) for j in range(x + n)]).sum(0)
            more = ((np.exp(2 * e) - np.exp(e))[..., None] * spread).reshape(n, -1, d), e.max()
        call.check(more=more)
    finally:
        call.close()


@pytest.mark.parametrize("window", [0, 1500])
@pytest.mark.parametrize("shape", [("bf16", "native", 8, 2, 64), ("bf16", "e4m3", 8, 2, 128), ("f32", "native", 8, 2, 64)], ids=lambda s: "-".join(map(str, s)))
def test_uneven_requests(shape, window):
    """Requests of a few keys beside ones of thousands, in no order: some are cut into stretches, some are not."""
    r = np.random.default_rng(window)
    rows = [40, 7000, 3, 900, 5200, 0, 2600, 130, 4100, 61, 1700, 3300]
    _run(*shape, 64, [(random_tree(r, int(r.integers(9, 40)), near=9), x) for x in rows], window=window)
