"""The paged calls together, as a program uses them (examples/paged_generation.py)."""
import numpy as np
import pytest
import torch

from tests import _paged_helpers as P

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def example():
    import __graft_entry__ as g
    g.build()
    from examples import paged_generation
    return paged_generation


@pytest.mark.parametrize("native", [False, True], ids=["e4m3", "native"])
def test_drafts_change_nothing_but_the_passes(example, native):
    """The most likely tokens are the same with drafts and without, in fewer passes."""
    one = example.generate(drafts=0, tokens=24, native=native, greedy=True)
    many = example.generate(drafts=4, tokens=24, native=native, greedy=True)
    assert one[0] == many[0]
    assert one[1] == 24 and many[1] < 24


def test_answer_becomes_a_chunk(example):
    answer, passes, chunk = example.generate(drafts=3, tokens=20)
    assert len(answer) == 20 and all(0 <= t < example.VOCAB for t in answer)
    assert chunk["n_slots"] == -(-chunk["n_tokens"] // example.RATIO) and chunk["n_tokens"] >= 19


def test_a_captured_step_gives_the_same():
    """Append, attend and gather in a CUDA graph, behind and between work that is not a kernel's."""
    c2kv = P.lib()
    rng = np.random.default_rng(3)
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        ctx = P.context("bf16", 8, 2, 128, stream=side)
        pg = P.Paged(rng, "bf16", "e4m3", 2, 128, 32, [400, 700])
        pg.fill_rows(rng)
        k, v = (torch.randn((4, 2, 128), device="cuda", dtype=torch.bfloat16) for _ in "kv")
        q = torch.randn((4, 8, 128), device="cuda", dtype=torch.bfloat16)
        pos = torch.arange(4, device="cuda", dtype=torch.int32)
        out, back_k, back_v, flag = torch.zeros_like(q), torch.zeros_like(k), torch.zeros_like(v), torch.zeros(256, device="cuda")

        def step():
            flag.zero_()
            c2kv.c2kv_paged_append(ctx, pg.pages(), pg.table, [0, 2, 4], [398, 698], k, v, turn=pos)
            flag.zero_()
            c2kv.c2kv_paged_attend(ctx, pg.pages(), pg.table, [0, 2, 4], [400, 700], q, out, turn=pos)
            c2kv.c2kv_paged_gather(ctx, pg.pages(), pg.table, [0, 2, 4], [398, 698], back_k, back_v)
        step()
        c2kv.c2kv_sync(ctx)
        want = [x.clone() for x in (out, back_k, back_v)]
        graph = torch.cuda.CUDAGraph()
        side.synchronize()
        with torch.cuda.graph(graph, stream=side, capture_error_mode="thread_local"):
            step()
        for x in (out, back_k, back_v):
            x.zero_()
        graph.replay()
        side.synchronize()
        assert all(torch.equal(a, b) for a, b in zip((out, back_k, back_v), want))
        c2kv.c2kv_destroy(ctx)
