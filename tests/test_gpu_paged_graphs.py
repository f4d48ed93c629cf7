"""Paged attention captured in CUDA graphs: what a captured call works in is the graph's own, so that neither
larger calls nor calls on other streams disturb a replay."""
import numpy as np
import pytest
import torch

from tests import _paged_helpers as P

pytestmark = pytest.mark.gpu

KINDS = [("bf16", "e4m3", 32, 8, 128, 1, 9000), ("bf16", "native", 8, 2, 64, 3, 5000), ("bf16", "e4m3", 32, 8, 128, 64, 9000),
         ("f32", "native", 16, 4, 64, 1, 9000), ("f32", "e4m3", 8, 2, 128, 20, 700)]


class _Step:
    """One request's attention of `new` tokens over `rows` rows."""

    def __init__(self, kind, ctx, new=None, rows=None):
        dtype, fmt, hq, hkv, d, n, k = kind
        self.new, self.rows, self.ctx = new or n, rows or k, ctx
        rng = np.random.default_rng(1)
        self.pg = P.Paged(rng, dtype, fmt, hkv, d, 128, [self.rows])
        # (every row alike in kind; the sums differ from key to key)
        raw = torch.randn(self.pg.k.shape, device="cuda")
        for x, s in ((self.pg.k, self.pg.ks), (self.pg.v, self.pg.vs)):
            x.copy_(raw.to(x.dtype))
            if s is not None:
                s.fill_(0.5)
        self.pages = self.pg.pages()
        self.q = torch.randn((self.new, hq, d), device="cuda").to(P.TDT[dtype])
        self.out, self.lse = torch.zeros_like(self.q), torch.zeros((hq, self.new), device="cuda")

    def run(self):
        P.lib().c2kv_paged_attend(self.ctx, self.pages, self.pg.table, [0, self.new], [self.rows], self.q, self.out, lse=self.lse)

    def result(self):
        return self.out.clone(), self.lse.clone()


def _capture(step, stream):
    graph = torch.cuda.CUDAGraph()
    stream.synchronize()
    with torch.cuda.graph(graph, stream=stream, capture_error_mode="thread_local"):
        step.run()
    return graph


@pytest.mark.parametrize("kind", KINDS, ids=lambda k: "-".join(map(str, k)))
def test_replay_after_larger_calls(kind):
    """A graph of a step, then calls that need more scratch on the same stream, then the graph again."""
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        ctx = P.context(*kind[:1], *kind[2:5], stream=side)
        try:
            step = _Step(kind, ctx)
            step.run()
            P.lib().c2kv_sync(ctx)
            want = step.result()
            graph = _capture(step, side)
            larger = _Step(kind, ctx, new=2 * step.new, rows=4 * step.rows)
            for _ in range(3):
                larger.run()
                first = larger.result()
                step.out.zero_()
                step.lse.zero_()
                graph.replay()
                larger.run()
                assert all(torch.equal(a, b) for a, b in zip(step.result(), want))
                assert all(torch.equal(a, b) for a, b in zip(larger.result(), first))
            P.lib().c2kv_sync(ctx)
            del graph
        finally:
            P.lib().c2kv_destroy(ctx)


@pytest.mark.parametrize("kind", KINDS, ids=lambda k: "-".join(map(str, k)))
def test_replay_beside_calls_on_the_captured_stream(kind):
    """The first call on a stream may be a captured one, and the graph may run on another stream while calls
    go on on the first."""
    side, other = torch.cuda.Stream(), torch.cuda.Stream()
    ctx = P.context(*kind[:1], *kind[2:5], stream=torch.cuda.current_stream())
    try:
        step, direct = _Step(kind, ctx), _Step(kind, ctx, rows=kind[6] + 640)
        wants = []
        for s in (step, direct):
            s.run()
            wants.append(s.result())
        P.lib().c2kv_sync(ctx)
        P.lib().c2kv_set_stream(ctx, side)
        graph = _capture(step, side)
        for s in (step, direct):
            s.out.zero_()
            s.lse.zero_()
        torch.cuda.synchronize()
        for _ in range(20):
            with torch.cuda.stream(other):
                graph.replay()
            direct.run()
        torch.cuda.synchronize()
        for s, want in zip((step, direct), wants):
            assert all(torch.equal(a, b) for a, b in zip(s.result(), want))
        P.lib().c2kv_sync(ctx)
        del graph
    finally:
        P.lib().c2kv_destroy(ctx)
