"""The calls of generation that branches together, as a program uses them (examples/branching_generation.py): against
the same program with the walk, the moves of rows, the choice among beams and their pages done in plain torch and numpy.
What the models compute is then the same to the bit, and so is what comes out."""
import pytest
import torch

from oracle import branch_oracle as brc

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def example():
    import __graft_entry__ as g
    g.build()
    from examples import branching_generation
    return branching_generation


def _same(x, y):
    return all(torch.equal(a, b) if isinstance(a, torch.Tensor) else a == b for a, b in zip(x, y))


class _Caches(list):
    """The caches that an example makes, whose memory the plain forms work on."""

    def __init__(self, example, monkeypatch):
        made = example.Cache

        def cache(*args):
            self.append(made(*args))
            return self[-1]
        monkeypatch.setattr(example, "Cache", cache)

    def held(self):
        """Pages of both sides and all layers, and their scales: [n, layers, pages, ..] of bytes."""
        c = self[-1]
        return [c.store.view(torch.uint8)] + ([] if c.scales[0] is None else [c.scales])


def _plain_walk(ctx, ptr, tokens, parent, p, u, n_accepted, path, next_token):
    way, x = brc.walk(parent.tolist(), tokens.tolist(), p.cpu().numpy(), u.cpu().numpy())
    path.fill_(-1)
    path[:len(way)] = torch.tensor(way, dtype=torch.int32)
    n_accepted.fill_(len(way) - 1)
    next_token.fill_(x)


@pytest.mark.parametrize("branch,levels", [(3, 4), (1, 3), (6, 2), (4, 12)])
@pytest.mark.parametrize("native", [False, True], ids=["e4m3", "native"])
def test_trees(example, monkeypatch, native, branch, levels):
    got = example.generate(tokens=40, branch=branch, levels=levels, native=native)
    caches = _Caches(example, monkeypatch)

    def plain_keep(ctx, layers, table, ptr, start, path, n_accepted):
        size = example.PAGE
        n = int(n_accepted) + 1
        a, b = start[0] + path[:n].long(), start[0] + torch.arange(n, device="cuda")
        for x in caches.held():
            x[:, :, table[0, b // size].long(), :, b % size] = x[:, :, table[0, a // size].long(), :, a % size].clone()
    monkeypatch.setattr(example.c2kv, "c2kv_verify_tree", _plain_walk)
    monkeypatch.setattr(example.c2kv, "c2kv_paged_keep", plain_keep)
    assert _same(got, example.generate(tokens=40, branch=branch, levels=levels, native=native))
    assert len(got[0]) == 40 and all(0 <= t < example.VOCAB for t in got[0]) and got[1] <= 40


@pytest.mark.parametrize("native", [False, True], ids=["e4m3", "native"])
def test_trees_change_nothing_but_the_passes(example, native):
    """The most likely tokens are the same with trees of drafts and without, in fewer passes."""
    one = example.generate(tokens=24, levels=0, native=native, greedy=True)
    many = example.generate(tokens=24, branch=4, levels=3, native=native, greedy=True)
    assert one[0] == many[0]
    assert one[1] == 24 and many[1] < 24


@pytest.mark.parametrize("width,prompt,ends", [(4, 37, False), (1, 5, False), (7, 64, True), (16, 31, True)])
@pytest.mark.parametrize("native", [False, True], ids=["e4m3", "native"])
def test_beams(example, monkeypatch, native, width, prompt, ends):
    """Over two or three page ends, with and without a token that ends a beam (one that the first run chose)."""
    end = -1
    if ends:
        end = int(example.beams(40, width, native, prompt=prompt)[0][-1, 3])
    got = example.beams(40, width, native, prompt=prompt, end_token=end)
    caches = _Caches(example, monkeypatch)

    def plain_select(ctx, x, score, parent, token, score_out, norm=None, done=None, end_token=-1, done_out=None):
        y = score[0, :, None] + (x - norm[:, None])
        if done is not None:                                 # a beam that has ended goes on as itself alone
            y[done[0] != 0] = -torch.inf
            y[done[0] != 0, end_token] = score[0][done[0] != 0]
        top = y.flatten().sort(descending=True, stable=True)
        at = top.indices[:parent.shape[1]]
        parent[0], token[0], score_out[0] = at // x.shape[1], at % x.shape[1], top.values[:parent.shape[1]]
        if done is not None:
            done_out[0] = (token[0] == end_token).int()

    def plain_reorder(ctx, layers, table, n_rows, parent, table_out):
        """Every beam has pages of its own, and copies all of its parent's rows."""
        table_out.copy_(table)
        for x in caches.held():
            x[:, :, table.flatten().long()] = x[:, :, table[parent[0].long()].flatten().long()].clone()
    monkeypatch.setattr(example.c2kv, "c2kv_beam_select", plain_select)
    monkeypatch.setattr(example.c2kv, "c2kv_paged_reorder", plain_reorder)
    assert _same(got, example.beams(40, width, native, prompt=prompt, end_token=end))
    assert got[0].shape == (width, 40) and got[1].isfinite().all() and (got[1][:-1] >= got[1][1:]).all()
