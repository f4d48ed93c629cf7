"""The walk down a tree of drafted tokens (c2kv_verify_tree) against the oracle: whole numbers, so equal."""
import numpy as np
import pytest
import torch

from oracle import branch_oracle as brc
from tests import _paged_helpers as P
from tests._tree_helpers import chain, random_tree, ranges, star

pytestmark = pytest.mark.gpu


class _Walk:
    """Trees whose children hold likely tokens, so that walks go some way."""

    def __init__(self, trees, vocab, seed=0, sure=0.5, stride=None, p=None, u=None):
        rng = np.random.default_rng(seed)
        self.trees, self.ptr, self.vocab = trees, ranges(trees), vocab
        T = self.ptr[-1]
        if p is None:
            p = rng.dirichlet(np.full(min(vocab, 64), 0.1), T) if T else np.zeros((0, min(vocab, 64)))
            wide = np.zeros((T, vocab), np.float32)
            for t in range(T):
                wide[t, rng.permutation(vocab)[:p.shape[1]]] = p[t]
            p = wide
        self.p = p.astype(np.float32)
        self.u = (rng.random(T) if u is None else np.broadcast_to(np.asarray(u), (T,))).astype(np.float32)
        self.tokens = rng.integers(0, vocab, T).astype(np.int32)
        for r, tree in enumerate(trees):                 # many children hold what their parent draws
            lo = self.ptr[r]
            for i, of in enumerate(tree):
                if of >= 0 and rng.random() < sure:
                    self.tokens[lo + i] = brc.drawn(self.p[lo + of], self.u[lo + of])
        rows = torch.full((max(T, 1), stride or vocab), float("nan"))
        rows[:T, :vocab] = torch.from_numpy(self.p)
        self.rows = rows.cuda()[:T, :vocab]
        i32 = lambda x, n: torch.tensor(np.asarray(x), dtype=torch.int32, device="cuda") if n else torch.zeros(0, dtype=torch.int32, device="cuda")  # noqa: E731
        self.parent = i32(sum(trees, []), T)
        self.dev_tokens, self.dev_u = i32(self.tokens, T), torch.from_numpy(self.u).cuda()
        self.n, self.next = (torch.full((len(trees),), 77, dtype=torch.int32, device="cuda") for _ in range(2))
        self.path = torch.full((T,), 77, dtype=torch.int32, device="cuda")

    def run(self, ctx):
        P.lib().c2kv_verify_tree(ctx, self.ptr, self.dev_tokens, self.parent, self.rows, self.dev_u, self.n, self.path, self.next)

    def check(self, trees=None):
        n, nxt, path = self.n.tolist(), self.next.tolist(), self.path.tolist()
        deepest = 0
        for r, tree in enumerate(trees or self.trees):
            at = slice(self.ptr[r], self.ptr[r + 1])
            want, x = brc.walk(tree, self.tokens[at], self.p[at], self.u[at])
            assert path[at] == want + [-1] * (len(tree) - len(want)), r
            assert (n[r], nxt[r]) == (max(0, len(want) - 1), x), r
            deepest = max(deepest, len(want))
        return deepest


@pytest.fixture()
def ctx():
    c = P.context("bf16", 4, 2, 64)
    yield c
    P.lib().c2kv_destroy(c)


def _run(ctx, *args, **more):
    w = _Walk(*args, **more)
    w.run(ctx)
    P.lib().c2kv_sync(ctx)
    return w.check()


@pytest.mark.parametrize("vocab", [1, 2, 31, 33, 1000, 8191, 32000, 32001, 151936])
def test_vocabularies(ctx, vocab):
    r = np.random.default_rng(vocab)
    assert _run(ctx, [random_tree(r, 20, near=6), chain(5), [], star(9), [-1]], vocab, seed=1) > 1


def test_the_largest_vocabulary(ctx):
    assert _run(ctx, [chain(3)], 1 << 19, sure=1.0) == 3


@pytest.mark.parametrize("seed", range(6))
def test_trees(ctx, seed):
    r = np.random.default_rng(100 + seed)
    trees = [random_tree(r, int(r.integers(0, 60)), near=int(r.integers(1, 9)), roots=0.1 * (seed % 2)) for _ in range(12)]
    assert _run(ctx, trees, 997, seed=seed, sure=0.8) > 3


def test_the_most_nodes(ctx):
    r = np.random.default_rng(4)
    assert _run(ctx, [chain(512), random_tree(r, 512, near=30), star(512)], 100, sure=1.0) == 512


@pytest.mark.parametrize("batch", [33, 300])
def test_many_requests(ctx, batch):
    r = np.random.default_rng(batch)
    _run(ctx, [random_tree(r, int(r.integers(0, 12)), near=3) for _ in range(batch)], 131, sure=0.7)


def test_no_nodes_at_all(ctx):
    assert _run(ctx, [[], [], []], 50) == 0


@pytest.mark.parametrize("vocab,stride", [(1000, 1024), (1001, 1003), (40, 1000)])
def test_rows_with_gaps(ctx, vocab, stride):
    _run(ctx, [random_tree(np.random.default_rng(3), 30, near=5), chain(4)], vocab, stride=stride)


@pytest.mark.parametrize("u", [0.0, 1.0 - 2.0 ** -24, 1.0, 2.0, -1.0, float("nan"), 2.0 ** -30])
def test_ends_of_the_random_numbers(ctx, u):
    _run(ctx, [chain(6), star(5)], 300, u=u)


def test_weights_that_are_none(ctx):
    """NaN, negative and infinite probabilities, rows without weight; a walk that meets one of those has no next
    token."""
    rng = np.random.default_rng(9)
    trees = [chain(8), random_tree(rng, 20, near=4), chain(3)]
    p = rng.random((31, 700)).astype(np.float32) * 0.01
    p[rng.random(p.shape) < 0.2] = np.nan
    p[rng.random(p.shape) < 0.2] = -1.0
    p[5, 17] = np.inf
    p[[2, 12, 29]] = 0.0
    p[30] = np.nan
    w = _Walk(trees, 700, p=p, sure=1.0)
    w.run(ctx)
    P.lib().c2kv_sync(ctx)
    w.check()
    assert w.next.tolist()[0] == -1 and w.n.tolist()[0] == 2 and w.next.tolist()[2] == -1


def test_one_hot_rows_are_greedy(ctx):
    """Rows of one weight: the walk takes the children of the largest probability, whatever u is."""
    p = np.zeros((7, 50), np.float32)
    p[np.arange(7), [4, 9, 0, 0, 49, 0, 0]] = 1.0
    w = _Walk([[-1, 0, 0, 1, 1, 4, 4]], 50, p=p, u=0.7)
    w.tokens[:] = [0, 4, 5, 8, 9, 7, 49]
    w.dev_tokens.copy_(torch.from_numpy(w.tokens))
    w.run(ctx)
    P.lib().c2kv_sync(ctx)
    w.check()
    assert w.path.tolist() == [0, 1, 4, 6, -1, -1, -1] and w.next.tolist() == [0]


def test_equal_children_and_tokens_that_are_none(ctx):
    """Of siblings that hold one token the first is taken; tokens outside the vocabulary are never drawn."""
    p = np.zeros((5, 10), np.float32)
    p[:, 3] = 1.0
    w = _Walk([[-1, 0, 0, 0, 2]], 10, p=p, u=0.5)
    w.tokens[:] = [3, -1, 3, 3, 10]
    w.dev_tokens.copy_(torch.from_numpy(w.tokens))
    w.run(ctx)
    P.lib().c2kv_sync(ctx)
    assert w.path.tolist() == [0, 2, -1, -1, -1] and w.n.tolist() == [1] and w.next.tolist() == [3]


def test_refused_parents(ctx):
    w = _Walk([chain(6), chain(4)], 20, sure=1.0)
    bad = [[-1, 0, 2, 2, 3, 9], [-1, -5, 0, 1]]
    w.parent.copy_(torch.tensor(sum(bad, []), dtype=torch.int32))
    w.run(ctx)
    with pytest.raises(P.lib().C2KVError) as e:
        P.lib().c2kv_sync(ctx)
    assert e.value.status == P.lib().ERR_DEVICE_BOUNDS
    w.check(bad)


def test_kept_tokens_are_the_targets_draws(ctx):
    """Over many random numbers the first token after the root, kept or not, is distributed as p: within five
    standard deviations of each count."""
    p = np.tile(np.array([[0.5, 0.3, 0.15, 0.05]], np.float32), (3, 1))
    counts = np.zeros(4)
    rng = np.random.default_rng(1)
    trees = [[-1, 0, 0]] * 200
    for _ in range(20):
        w = _Walk(trees, 4, p=np.tile(p, (200, 1)), u=rng.random(600))
        w.tokens[:] = np.tile([0, 1, 3], 200)            # drafts of the second and the last
        w.dev_tokens.copy_(torch.from_numpy(w.tokens))
        w.run(ctx)
        path, nxt = w.path.view(200, 3).cpu().numpy(), w.next.cpu().numpy()
        np.add.at(counts, np.where(path[:, 1] == 1, 1, np.where(path[:, 1] == 2, 3, nxt)), 1)
    n = counts.sum()
    assert n == 4000 and np.all(np.abs(counts - n * p[0]) <= 5 * np.sqrt(n * p[0] * (1 - p[0])))


def test_captured_and_beside_other_streams(ctx):
    """Two graphs of one context replayed on two streams at once, with new inputs in place."""
    r = np.random.default_rng(2)
    c2kv, side = P.lib(), [torch.cuda.Stream(), torch.cuda.Stream()]
    walks = [_Walk([random_tree(r, 40, near=5) for _ in range(6)], v, seed=i, sure=0.8) for i, v in enumerate((5000, 777))]
    graphs = []
    for w, s in zip(walks, side):
        torch.cuda.synchronize()
        c2kv.c2kv_set_stream(ctx, s)
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1], stream=s, capture_error_mode="thread_local"):
            w.run(ctx)
    for k in range(3):
        for w in walks:
            w.u = r.random(len(w.u)).astype(np.float32)
            w.dev_u.copy_(torch.from_numpy(w.u))
        torch.cuda.synchronize()
        for _ in range(3):
            for g, s in zip(graphs, side):
                with torch.cuda.stream(s):
                    g.replay()
        torch.cuda.synchronize()
        for w in walks:
            w.check()
    del graphs
