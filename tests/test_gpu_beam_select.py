"""The best continuations of beams (c2kv_beam_select) against the oracle.  Scores are single fp32 operations and
the order is by them and then by place, so everything is equal."""
import numpy as np
import pytest
import torch

from oracle import branch_oracle as brc
from tests import _paged_helpers as P

pytestmark = pytest.mark.gpu
INF, NAN = float("inf"), float("nan")


class _Choice:
    def __init__(self, batch, width, vocab, best, dtype="f32", norm=False, done=None, end_token=-1, seed=0, x=None, score=None, stride=None):
        rng = np.random.default_rng(seed)
        self.shape, self.end_token = (batch, width, vocab, best), end_token
        x = rng.standard_normal((batch * width, vocab)) * 4 - 10 if x is None else x
        wide = torch.full((batch * width, stride or vocab), 1e30, dtype=P.TDT[dtype])
        wide[:, :vocab] = torch.from_numpy(np.asarray(x, np.float32)).to(P.TDT[dtype])
        self.x = wide.cuda()[:, :vocab]
        self.score = torch.from_numpy(np.asarray(-20 * rng.random((batch, width)) if score is None else score, np.float32)).cuda()
        self.norm = torch.from_numpy(rng.standard_normal(batch * width).astype(np.float32) + 8).cuda() if norm else None
        self.done = torch.from_numpy((rng.random((batch, width)) < done).astype(np.int32) * 5).cuda() if done is not None else None
        self.parent, self.token, self.done_out = (torch.full((batch, best), 77, dtype=torch.int32, device="cuda") for _ in range(3))
        self.score_out = torch.full((batch, best), 77.0, device="cuda")

    def run(self, ctx):
        P.lib().c2kv_beam_select(ctx, self.x, self.score, self.parent, self.token, self.score_out, norm=self.norm, done=self.done,
                                 end_token=self.end_token, done_out=self.done_out)

    def check(self):
        B, W, V, K = self.shape
        x, score = self.x.float().cpu().numpy(), self.score.cpu().numpy()
        for r in range(B):
            rows = slice(r * W, (r + 1) * W)
            done = self.done[r].tolist() if self.done is not None else None
            got = brc.select(x[rows], None if self.norm is None else self.norm[rows].cpu().numpy(), score[r], done, self.end_token, K)
            n = K - len(got)
            assert self.score_out[r].tolist() == [float(g[0]) for g in got] + [-INF] * n
            assert self.parent[r].tolist() == [g[1] for g in got] + [-1] * n
            assert self.token[r].tolist() == [g[2] for g in got] + [-1] * n
            assert self.done_out[r].tolist() == [int(g[2] == self.end_token or bool(done and done[g[1]])) for g in got] + [0] * n


@pytest.fixture()
def ctx():
    c = P.context("bf16", 4, 2, 64)
    yield c
    P.lib().c2kv_destroy(c)


def _run(ctx, *args, **more):
    c = _Choice(*args, **more)
    c.run(ctx)
    P.lib().c2kv_sync(ctx)
    c.check()
    return c


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("vocab", [1, 2, 7, 255, 256, 1000, 4095, 4096, 4097, 12345, 32000, 131072])
def test_vocabularies(ctx, vocab, dtype):
    _run(ctx, 2, 4, vocab, 8, dtype)
    _run(ctx, 1, 3, vocab, 6, dtype, norm=True, done=0.3, end_token=vocab // 2)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("width,best", [(1, 1), (1, 64), (2, 3), (5, 10), (8, 8), (16, 32), (33, 63), (64, 64), (64, 1)])
def test_widths(ctx, width, best, dtype):
    _run(ctx, 3, width, 5000, best, dtype, norm=dtype == "bf16")


def test_the_largest_vocabulary(ctx):
    _run(ctx, 1, 2, 1 << 19, 64)
    _run(ctx, 1, 1, 1 << 19, 5, "bf16")


def test_many_requests(ctx):
    _run(ctx, 700, 2, 300, 4, done=0.2, end_token=7)
    _run(ctx, 40, 16, 9000, 16, "bf16", norm=True)


@pytest.mark.parametrize("vocab,stride", [(1000, 1024), (999, 1001), (8200, 8208)])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_rows_with_gaps(ctx, vocab, stride, dtype):
    _run(ctx, 2, 3, vocab, 6, dtype, stride=stride)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("best", [1, 8, 64])
@pytest.mark.parametrize("vocab", [3000, 20000, 70000])
def test_equal_scores(ctx, vocab, best, dtype):
    """All alike; few values; all alike but for a few at the end: the lowest places win."""
    rng = np.random.default_rng(vocab)
    _run(ctx, 1, 2, vocab, best, dtype, x=np.full((2, vocab), -3.0), score=[[0.0, 0.0]])
    _run(ctx, 1, 2, vocab, best, dtype, x=rng.integers(-2, 2, (2, vocab)), score=[[0.0, 1.0]])
    x = np.full((2, vocab), -3.0)
    x[:, -best // 2:] = 5.0
    x[1, 17] = 5.0
    _run(ctx, 1, 2, vocab, best, dtype, x=x, score=[[0.0, 0.0]])


@pytest.mark.parametrize("vocab", [5000, 70000])
def test_orders(ctx, vocab):
    """Rising, falling and one lane's values largest: every chunk brings better ones, or none does."""
    up = np.arange(vocab, dtype=np.float32)[None].repeat(2, 0)
    lane = np.random.default_rng(1).standard_normal((2, vocab))
    lane[:, ::1024] += 100
    blocks = up // 700
    for x in (up, -up, lane, blocks, -blocks, np.abs(up - vocab // 2)):
        _run(ctx, 1, 2, vocab, 48, x=x, score=[[0.0, 0.25]])


def test_signed_zeros_are_equal(ctx):
    x = np.zeros((1, 5000), np.float32)
    x[:, ::2] = -0.0
    c = _run(ctx, 1, 1, 5000, 9, x=x, score=[[-0.0]])
    assert c.token.tolist() == [list(range(9))] and not torch.signbit(c.score_out).any()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("norm", [False, True])
def test_scores_that_are_none(ctx, norm, dtype):
    """NaN and -inf are no candidates; +inf comes first; fewer candidates than places leave -1 and -inf."""
    x = np.random.default_rng(3).standard_normal((8, 6000))
    x[0] = NAN
    x[1] = -INF
    x[2, :5990] = -INF
    x[3, ::3] = NAN
    x[4, 77] = INF
    _run(ctx, 2, 4, 6000, 16, dtype, norm=norm, x=x)
    x[:] = -INF
    x[3, 5] = 1.0
    x[6, 0] = NAN
    _run(ctx, 2, 4, 6000, 16, dtype, norm=norm, x=x)


def test_scores_of_beams(ctx):
    """A first step (all beams but one at -inf), beams without a number, infinite ones, and none left at all."""
    _run(ctx, 2, 4, 9000, 8, score=[[0.0, -INF, -INF, -INF], [-1.0, NAN, INF, -2.0]])
    _run(ctx, 2, 3, 9000, 8, score=[[-INF] * 3, [NAN] * 3], done=0.5, end_token=3)
    _run(ctx, 1, 3, 100, 8, score=[[-1e38, -3e38, 1e-30]], x=np.random.default_rng(1).standard_normal((3, 100)) * 3e38)


@pytest.mark.parametrize("share", [0.5, 1.0])
def test_beams_that_have_ended(ctx, share):
    _run(ctx, 5, 6, 3000, 12, done=share, end_token=2999)
    _run(ctx, 5, 6, 3000, 6, "bf16", norm=True, done=share, end_token=0)


def test_end_without_ended_beams(ctx):
    x = np.random.default_rng(2).standard_normal((4, 500))
    x[:, 9] = 20
    c = _run(ctx, 2, 2, 500, 4, x=x, end_token=9)
    assert c.done_out.sum() == 4


def test_captured_and_beside_other_streams(ctx):
    c2kv, side = P.lib(), [torch.cuda.Stream(), torch.cuda.Stream()]
    calls = [_Choice(3, 8, 40000, 16, "bf16", norm=True, done=0.1, end_token=2), _Choice(2, 4, 9999, 9, seed=4)]
    graphs = []
    for c, s in zip(calls, side):
        torch.cuda.synchronize()
        c2kv.c2kv_set_stream(ctx, s)
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1], stream=s, capture_error_mode="thread_local"):
            c.run(ctx)
    larger = _Choice(8, 16, 50000, 64, seed=6)
    for k in range(3):
        for c in calls:
            c.x.copy_(torch.randn_like(c.x.float()).to(c.x.dtype))
        torch.cuda.synchronize()
        for _ in range(3):
            for g, s in zip(graphs, side):
                with torch.cuda.stream(s):
                    g.replay()
            larger.run(ctx)
        torch.cuda.synchronize()
        for c in calls + [larger]:
            c.check()
    del graphs


def test_a_loop_of_steps_without_the_host(ctx):
    """Two steps in a row, the second's scores and ends the first's outputs."""
    c = _Choice(2, 4, 3000, 4, end_token=5, done=0.0)
    c.run(ctx)
    d = _Choice(2, 4, 3000, 4, end_token=5, seed=1)
    d.score, d.done = c.score_out, c.done_out
    d.run(ctx)
    P.lib().c2kv_sync(ctx)
    c.check()
    d.check()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("batch,width", [(1, 2), (16, 12)])
def test_masks_of_the_lowest_value(ctx, batch, width, dtype):
    """Most of the vocabulary at the type's lowest value, here all of a stretch, there all but a few: the scores
    round to one another's, and the first places win."""
    rng = np.random.default_rng(4)
    lowest = float(torch.finfo(P.TDT[dtype]).min)
    x = np.full((batch * width, 40000), lowest)
    for row in x[::2]:
        at = rng.integers(0, 40000, 9)
        row[at] = rng.standard_normal(9)
    _run(ctx, batch, width, 40000, 8, dtype, x=x)
    _run(ctx, batch, width, 40000, 16, dtype, x=np.where(x == lowest, -1e9, x), norm=True)


def test_values_beside_large_scores(ctx):
    """Scores so large that hundreds of values round to one score: places decide."""
    x = np.random.default_rng(5).standard_normal((40, 50000))
    _run(ctx, 1, 1, 50000, 16, x=x[:1], score=[[-3.0e6]])
    _run(ctx, 20, 2, 50000, 16, x=x, score=-1.0e5 * np.arange(1, 41).reshape(20, 2))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("vocab", [31, 255, 257, 511, 513, 1023, 1025, 1279, 1281, 1500, 1791, 1793, 2047, 2049, 2500, 4099, 5000, 8191, 50000])
def test_stretches_that_leave_lanes_without_values(ctx, vocab, dtype):
    """Vocabularies that give some warps of a stretch no values, or fewer than lanes; from one continuation to 64."""
    for best in (1, 5, 33, 64):
        _run(ctx, 2, 3, vocab, best, dtype, norm=True, seed=best)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_beams_far_apart(ctx, dtype):
    """One beam's candidates all come before the others': the join meets long lists that its bound does not shorten."""
    for width, vocab, best in ((16, 40000, 64), (64, 5000, 64), (32, 32000, 32)):
        score = np.tile(-60.0 * np.arange(width), (2, 1))
        score[1] = score[1][::-1]
        _run(ctx, 2, width, vocab, best, dtype, score=score, seed=width)
