"""The oracle of generation that branches, pinned by hand, by torch and by what the operations are for (no GPU)."""
import itertools

import numpy as np
import pytest
import torch

from oracle import branch_oracle as brc
from oracle import paged_oracle as orc
from tests._tree_helpers import chain, random_tree


def test_sight_by_hand():
    #        0
    #      1   2        rows before: 0, 1
    #      3   4 5
    parent = [-1, 0, 0, 1, 2, 2]
    want = ["11100000", "11110000", "11101000", "11110100", "11101010", "11101001"]
    assert [[int(c) for c in w] for w in want] == brc.sees(parent, 8).astype(int).tolist()
    assert brc.sees(parent, 8, 2).astype(int).tolist()[4] == [0, 0, 0, 0, 1, 0, 1, 0]
    assert brc.sees(parent, 8, 4).astype(int).tolist()[4] == [0, 1, 1, 0, 1, 0, 1, 0]
    assert brc.sees([-1, -1, 0], 3).astype(int).tolist() == [[1, 0, 0], [0, 1, 0], [1, 0, 1]]


@pytest.mark.parametrize("window", [0, 1, 3, 100])
def test_attention_by_torch(window):
    rng = np.random.default_rng(window)
    for n, x in ((1, 0), (7, 0), (12, 9)):
        tree = random_tree(rng, n, roots=0.2)
        q, k, v = rng.standard_normal((n, 6, 8)), rng.standard_normal((n + x, 2, 8)), rng.standard_normal((n + x, 2, 8))
        mask = torch.zeros((n, n + x), dtype=torch.bool)
        for i in range(n):                                   # a node's way up, and the rows that its window still reaches
            at, left, depth = i, window or n + x, 0
            while at >= 0:
                mask[i, x + at] = left > 0
                at, left = tree[at], left - 1
            mask[i, max(0, x - max(0, left)):x] = True
        want = torch.nn.functional.scaled_dot_product_attention(
            *(torch.from_numpy(y).transpose(0, 1) for y in (q, k.repeat(3, 1), v.repeat(3, 1))), attn_mask=mask)
        out, lse = brc.attend_tree(q, k, v, tree, window)
        assert np.allclose(out, want.transpose(0, 1).numpy(), atol=1e-12) and np.isfinite(lse).all()


def test_a_chain_is_what_follows_one_another():
    rng = np.random.default_rng(1)
    q, k, v = rng.standard_normal((5, 4, 8)), rng.standard_normal((14, 2, 8)), rng.standard_normal((14, 2, 8))
    for window in (0, 3, 9):
        for got, want in zip(brc.attend_tree(q, k, v, chain(5), window), orc.attend(q, k, v, 14, window)):
            assert np.allclose(got, want, atol=1e-12)


def test_draws_are_those_of_the_verification_without_drafts():
    rng = np.random.default_rng(2)
    for p in (*rng.dirichlet(np.full(50, 0.1), 60).astype(np.float32), np.zeros(9, np.float32), np.array([0, np.nan, 2, -1], np.float32)):
        for u in np.float32([0, 1e-9, rng.random(), 1 - 2.0 ** -24, 1.0]):
            ((_, want),) = orc.verify([0, 0], np.zeros(0, np.int32), p[None], None, np.zeros(0, np.float32), u[None])
            assert brc.drawn(p, u) == want
        assert brc.drawn(p, np.nan) == brc.drawn(p, 0.0)


def test_walk_by_hand():
    eye = np.eye(6, dtype=np.float32)
    parent, tokens = [-1, 0, 0, 1, 2, 2, 5], [9, 1, 2, 3, 3, 4, 5]
    u = np.full(7, 0.5, np.float32)

    def walk(*draws):
        return brc.walk(parent, tokens, eye[list(draws)], u)
    assert walk(2, 0, 4, 0, 0, 5, 0) == ([0, 2, 5, 6], 0)
    assert walk(2, 0, 4, 0, 0, 1, 0) == ([0, 2, 5], 1)
    assert walk(1, 2, 0, 0, 0, 0, 0) == ([0, 1], 2)
    assert walk(5, 0, 0, 0, 0, 0, 0) == ([0], 5)
    assert brc.walk([-1, 0, 0], [0, 3, 3], eye[[3, 4, 5]], u) == ([0, 1], 4)          # of equal children the first
    assert brc.walk([-1, 0], [0, 3], 0 * eye[:2], u) == ([0], -1)
    assert brc.walk([], [], eye[:0], u) == ([], -1)


def test_walks_draw_what_the_model_draws():
    """Whatever is drafted, tokens come as from the rows themselves: over a grid of u as often as their probability."""
    p = np.float32([[0.5, 0.25, 0.25], [0.25, 0.75, 0.0], [0.0, 0.5, 0.5]])
    seen = {}
    for a, b in itertools.product((np.arange(16) + 0.5) / 16, repeat=2):
        path, x = brc.walk([-1, 0, 0], [0, 0, 2], p, np.float32([a, b, b]))
        way = tuple([0, 0, 2][i] for i in path[1:]) + (x,)
        seen[way] = seen.get(way, 0) + 1 / 256
    want = {(1,): 0.25, (0, 0): 0.125, (0, 1): 0.375, (2, 1): 0.125, (2, 2): 0.125}
    assert seen == want


def test_kept_rows():
    rng = np.random.default_rng(3)
    for size, start in ((16, 0), (16, 13), (4, 6)):
        pages = rng.standard_normal((9, 2, size, 3))
        table = rng.permutation(9)
        row = lambda x, j: x[table[j // size], :, j % size]  # noqa: E731
        was, path = pages.copy(), [0, 2, 3, 7, 11]
        brc.keep(pages, table, start, path, size)
        for j in range(9 * size):
            moved = 0 <= j - start < len(path)
            assert np.array_equal(row(pages, j), row(was, start + path[j - start] if moved else j))


@pytest.mark.parametrize("best", [1, 3, 8])
def test_choice_by_torch(best):
    rng = np.random.default_rng(best)
    for case in range(20):
        x = np.round(rng.standard_normal((4, 30)) * 2).astype(np.float32) / 2           # (many are equal)
        norm = np.log(np.exp(x).sum(-1)).astype(np.float32) if case % 2 else None
        score = rng.standard_normal(4).astype(np.float32)
        score[case % 4] = -np.inf
        x[1, case] = np.nan
        y = torch.from_numpy(score)[:, None] + (torch.from_numpy(x) - (torch.from_numpy(norm)[:, None] if norm is not None else 0))
        top = torch.nan_to_num(y, nan=-torch.inf, neginf=-torch.inf).flatten().sort(descending=True, stable=True)
        want = [(float(s), int(i) // 30, int(i) % 30) for s, i in zip(top.values[:best], top.indices[:best])]
        assert [(float(s), w, v) for s, w, v in brc.select(x, norm, score, None, -1, best)] == want
    done = np.array([0, 1, 0, 0])
    got = brc.select(np.zeros((4, 30), np.float32), None, np.float32([-1, 5, -2, -3]), done, 7, 3)
    assert [(float(s), w, v) for s, w, v in got] == [(5, 1, 7), (-1, 0, 0), (-1, 0, 1)]


@pytest.mark.parametrize("n_rows", [0, 1, 4, 7, 8, 11])
def test_beams_go_on_from_their_parents(n_rows):
    """Each beam's rows become its parent's, and no two write the same page next."""
    rng, size, width = np.random.default_rng(n_rows), 4, 5
    for _ in range(50):
        tables = rng.permutation(width * 4).reshape(width, 4)
        tables[:, :n_rows // size] = tables[0, :n_rows // size] if rng.random() < 0.5 else tables[:, :n_rows // size]
        rows = rng.integers(0, 10 ** 6, (width * 4, size))
        before = [[rows[tables[w, j // size], j % size] for j in range(n_rows)] for w in range(width)]
        parent = rng.integers(-1, width, width)
        out, copies = brc.reorder(tables, parent, n_rows, size)
        old = rows.copy()
        for a, b, n in copies:
            assert n == n_rows % size
            rows[b, :n] = old[a, :n]
        for w in range(width):
            got = [rows[out[w, j // size], j % size] for j in range(n_rows)]
            assert got == before[parent[w] if parent[w] >= 0 else w]
        assert len({int(t) for t in out[:, n_rows // size]}) == width
