"""Drafted tokens against the target's probabilities: every accepted count and drawn token equals the
oracle's (the definition is exact in whole numbers), and over many draws they follow the target."""
import numpy as np
import pytest
import torch

from oracle import paged_oracle as orc
from tests import _paged_helpers as P

pytestmark = pytest.mark.gpu


def _draws(rng, counts, vocab, greedy=False, pad=0):
    T, B = sum(counts), len(counts)

    def soft(x):
        e = np.exp(x - x.max(-1, keepdims=True))
        return (e / e.sum(-1, keepdims=True)).astype(np.float32)
    base = rng.standard_normal((T + B, vocab)) * 2
    p = soft(base + 0.5 * rng.standard_normal((T + B, vocab)))
    rows = np.concatenate([np.arange(n) + o + r for r, (n, o) in enumerate(zip(counts, np.cumsum([0] + counts[:-1])))]).astype(int) \
        if T else np.zeros(0, int)
    q = soft(base[rows]) if T else np.zeros((0, vocab), np.float32)
    tokens = np.array([rng.choice(vocab, p=x / x.sum()) for x in q.astype(np.float64)], np.int32)
    return p, (None if greedy else q), tokens, rng.random(T, np.float32), rng.random(B, np.float32)


def _run(counts, p, q, tokens, ua, un, pad=0):
    c2kv, ctx = P.lib(), P.context("bf16", 1, 1, 64)
    try:
        def dev(x):
            x = torch.from_numpy(x).cuda()
            if pad and x.dim() == 2:
                wide = torch.full((x.shape[0], x.shape[1] + pad), float("nan"), device="cuda")
                wide[:, :x.shape[1]] = x
                x = wide[:, :x.shape[1]]
            return x
        ptr = np.cumsum([0] + counts).tolist()
        acc, nxt = (torch.full((len(counts),), -7, dtype=torch.int32, device="cuda") for _ in range(2))
        c2kv.c2kv_verify_drafts(ctx, ptr, dev(tokens), dev(p), None if q is None else dev(q), dev(ua), dev(un), acc, nxt)
        try:
            c2kv.c2kv_sync(ctx)
            bad = False
        except c2kv.C2KVError as e:
            assert e.status == c2kv.ERR_DEVICE_BOUNDS
            bad = True
        return list(zip(acc.tolist(), nxt.tolist())), bad
    finally:
        c2kv.c2kv_destroy(ctx)


@pytest.mark.parametrize("greedy", [False, True], ids=["drawn", "greedy"])
@pytest.mark.parametrize("counts,vocab,pad", [
    ([4], 32000, 0), ([1, 0, 3, 8, 2, 0], 5003, 0), ([0], 1, 0), ([2, 2], 1, 0), ([3, 5, 1], 33, 7), ([40, 70, 0], 257, 0),
    ([2] * 40, 131, 0), ([1] * 300, 64, 1), ([6] * 9, 131072, 0)])
def test_equals_oracle(counts, vocab, pad, greedy):
    rng = np.random.default_rng(len(counts) * 1000 + vocab)
    p, q, tokens, ua, un = _draws(rng, counts, vocab, greedy)
    got, bad = _run(counts, p, q, tokens, ua, un, pad)
    assert not bad
    assert got == orc.verify(np.cumsum([0] + counts).tolist(), tokens, p, q, ua, un)


def test_edges():
    """Nothing left over, no weight at all, NaN and negative weights, numbers at the ends of their range."""
    V = 1000
    rng = np.random.default_rng(1)
    p = np.zeros((8 + 4, V), np.float32)
    q = np.zeros((8, V), np.float32)
    counts, tokens = [2, 2, 2, 2], np.array([3, 4] * 4, np.int32)
    p[0:3] = rng.random((3, V)).astype(np.float32) / V
    q[0:2] = p[0:2]                                       # equal: nothing is left over q
    p[6:9] = np.nan                                       # request 2: no weight
    p[9:12, 5] = 0.25
    p[9:12, 7] = -1
    p[9:12, 8] = np.nan
    p[9:12, V - 1] = 0.75
    q[6:8, 3:5] = 1
    for ua, un in ((0.0, 0.0), (1 - 2.0 ** -24, 1 - 2.0 ** -24), (0.5, 0.25), (0.5, 0.2499999), (2.0 ** -30, 2.0 ** -26)):
        ua_, un_ = np.full(8, ua, np.float32), np.full(4, un, np.float32)
        got, bad = _run(counts, p, q, tokens, ua_, un_)
        assert got == orc.verify([0, 2, 4, 6, 8], tokens, p, q, ua_, un_)
        assert got[2][1] == -1 and got[1] == (0, -1) and not bad


def test_token_outside_the_vocabulary():
    rng = np.random.default_rng(2)
    p, q, tokens, ua, un = _draws(rng, [3, 3], 100)
    ua[:] = 0
    for x in (-1, 100, 2 ** 31 - 1):
        tokens[1] = x
        for qq in (q, None):
            got, bad = _run([3, 3], p, qq, tokens, ua, un)
            assert bad and got == orc.verify([0, 3, 6], tokens, p, qq, ua, un) and got[0][0] == 1


def test_follows_the_target():
    """The first token kept is distributed as p, whatever q drafts: 200 000 requests, a vocabulary of 8.
    A frequency's standard error is at most 0.5 / sqrt(200000) = 0.0011; five of them are allowed."""
    n, V = 200_000, 8
    g = torch.Generator(device="cuda").manual_seed(5)
    p1 = torch.tensor([0.30, 0.05, 0.20, 0.01, 0.14, 0.10, 0.00, 0.20], device="cuda")
    q1 = torch.tensor([0.10, 0.25, 0.20, 0.05, 0.10, 0.10, 0.10, 0.10], device="cuda")
    tokens = torch.multinomial(q1, n, replacement=True, generator=g).int()
    p = p1.expand(2 * n, V).contiguous()
    q = q1.expand(n, V).contiguous()
    ua, un = (torch.rand(n, device="cuda", generator=g) for _ in range(2))
    acc, nxt = (torch.empty(n, dtype=torch.int32, device="cuda") for _ in range(2))
    c2kv, ctx = P.lib(), P.context("bf16", 1, 1, 64)
    try:
        c2kv.c2kv_verify_drafts(ctx, list(range(n + 1)), tokens, p, q, ua, un, acc, nxt)
        c2kv.c2kv_sync(ctx)
    finally:
        c2kv.c2kv_destroy(ctx)
    kept = torch.where(acc > 0, tokens, nxt).long()
    freq = torch.bincount(kept, minlength=V).float() / n
    assert (freq - p1).abs().max() <= 5 * 0.0011
