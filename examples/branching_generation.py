"""Generation that branches, over a paged cache.

    python examples/branching_generation.py [--tokens 64] [--branch 3] [--levels 4] [--native]

The small decoder of paged_generation.py stands in for a model again.  Around it:

1. Trees of drafts.  A cheaper model (the same weights with the last layer left out) drafts several tokens after each
   of the best few nodes of a level; the tree's rows are appended, attended in one pass in which a node sees its own
   path alone, and walked by the model's own draws; the rows that the walk kept move together in every layer.
2. Beams.  The prompt's pages are shared; a beam's last page becomes its own where beams part.  Every step appends and
   attends a token a beam, chooses the best continuations over the vocabulary, and hands the beams their pages on.
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from examples.paged_generation import D, E, HKV, HQ, LAYERS, PAGE, THETA, VOCAB, Decoder  # noqa: E402
from paper_2607_17715_gb300 import c2kv  # noqa: E402


def int32(x):
    return torch.tensor(x, device="cuda", dtype=torch.int32)


class Cache:
    """Pages in every layer, shared by the rows of one table."""

    def __init__(self, sequences, rows, native):
        self.width = -(-rows // PAGE)
        n = sequences * self.width
        dtype = torch.bfloat16 if native else torch.float8_e4m3fn
        shape = (2, LAYERS, n, HKV, PAGE, D)
        self.store = torch.zeros(shape, device="cuda", dtype=torch.bfloat16 if native else torch.uint8).view(dtype)
        self.scales = [None, None] if native else torch.zeros(shape[:-1], device="cuda")
        self.layers = c2kv.make_layers(*self.store, *self.scales)
        self.pages = [c2kv.make_pages(*(None if x is None else x[i] for x in (*self.store, *self.scales))) for i in range(LAYERS)]
        order = torch.randperm(n, generator=torch.Generator().manual_seed(1))
        self.table = order.to("cuda", torch.int32).view(sequences, self.width)
        self.rows = 0                                        # of each sequence


def forward(model, ctx, cache, tokens, depth, parent=None, layers=LAYERS, sequences=1):
    """Logits of `tokens` [n] that come after the cache's rows, `depth` [n] positions after them: a tree of one
    sequence (parent), or as many tokens of each of several that follow one another."""
    n = tokens.shape[0]
    pos = depth + cache.rows
    table, each = cache.table[:sequences], n // sequences
    ptr = [each * i for i in range(sequences + 1)]
    keys = [cache.rows + each] * sequences
    x = model.embed[tokens.long()]
    for i in range(layers):
        rows = (model.norm(x) @ model.qkv[i]).view(n, HQ + 2 * HKV, D)
        q, k, v = rows[:, :HQ], rows[:, HQ:HQ + HKV], rows[:, HQ + HKV:]
        c2kv.c2kv_paged_append(ctx, cache.pages[i], table, ptr, [cache.rows] * sequences, k, v, turn=pos)
        out = torch.empty((n, HQ, D), device="cuda", dtype=torch.bfloat16)
        if parent is None:
            c2kv.c2kv_paged_attend(ctx, cache.pages[i], table, ptr, keys, q, out, turn=pos)
        else:
            c2kv.c2kv_paged_attend_tree(ctx, cache.pages[i], table, ptr, keys, parent, q, out, turn=pos)
        x = x + out.view(n, E) @ model.out[i]
    return (model.norm(x) @ model.head).float()


def prefill(model, ctx, cache, prompt):
    """The logits after a prompt, which the cache's first sequence then holds."""
    n = prompt.shape[0]
    logits = forward(model, ctx, cache, prompt, torch.arange(n, device="cuda", dtype=torch.int32))
    cache.rows = n
    return logits[-1:]


def draft(model, ctx, cache, token, branch, levels):
    """A tree of drafts after `token`: parents, tokens and depths, node 0 being the token itself.  Each level is the
    `branch` likeliest paths of the tree so far, one token longer."""
    parent, tokens, depth, score, leaves = [-1], [token], [0], [0.0], [0]
    for level in range(1, levels + 1):
        logits = forward(model, ctx, cache, int32(tokens), int32(depth), int32(parent), LAYERS - 1)
        best = torch.log_softmax(logits[leaves], -1) + torch.tensor([score[i] for i in leaves], device="cuda")[:, None]
        top = best.flatten().topk(branch)
        at = len(parent)
        for s, i in sorted(zip(top.values.tolist(), top.indices.tolist()), reverse=True):
            parent.append(leaves[i // VOCAB])
            tokens.append(i % VOCAB)
            depth.append(level)
            score.append(s)
        leaves = list(range(at, at + branch))
    return parent, tokens, depth


def generate(tokens=64, branch=3, levels=4, native=False, greedy=False, seed=0, prompt=37):
    """The generated tokens, and how many passes of the model they took."""
    model = Decoder(seed)
    ctx = c2kv.c2kv_create(LAYERS, HQ, HKV, D, THETA, c2kv.DTYPE_BF16, pool_slots=64, stream=torch.cuda.current_stream())
    try:
        cache = Cache(1, prompt + tokens + (levels + 2) * (branch + 1), native)
        g = torch.Generator(device="cuda").manual_seed(seed + 2)
        logits = prefill(model, ctx, cache, torch.randint(VOCAB, (prompt,), generator=g, device="cuda", dtype=torch.int32))
        accepted, following = int32([0]), int32([0])

        def walk(logits, drafted, parent):
            """How many drafts the model's draws follow, and the token after them; the rows kept move together."""
            n = logits.shape[0]
            p = torch.nn.functional.one_hot(logits.argmax(-1), VOCAB).float() if greedy else torch.softmax(logits, -1)
            path = torch.empty(n, device="cuda", dtype=torch.int32)
            u = torch.rand(n, generator=g, device="cuda")
            c2kv.c2kv_verify_tree(ctx, [0, n], int32(drafted), int32(parent), p, u, accepted, path, following)
            return path

        walk(logits, [0], [-1])
        answer, passes = [int(following)], 1
        while len(answer) < tokens:
            parent, drafted, depth = draft(model, ctx, cache, answer[-1], branch, levels) if levels else ([-1], answer[-1:], [0])
            logits = forward(model, ctx, cache, int32(drafted), int32(depth), int32(parent))
            path = walk(logits, drafted, parent)
            c2kv.c2kv_paged_keep(ctx, cache.layers, cache.table, [0, len(parent)], [cache.rows], path, accepted)
            kept = int(accepted)
            answer += [drafted[i] for i in path[1:kept + 1].tolist()] + [int(following)]
            cache.rows += kept + 1
            passes += 1
        c2kv.c2kv_sync(ctx)
        return answer[:tokens], passes
    finally:
        c2kv.c2kv_destroy(ctx)


def beams(tokens=32, width=4, native=False, seed=0, prompt=37, end_token=-1):
    """The beams' tokens [width, tokens], best first, and their scores (sums of log-probabilities)."""
    model = Decoder(seed)
    ctx = c2kv.c2kv_create(LAYERS, HQ, HKV, D, THETA, c2kv.DTYPE_BF16, pool_slots=64, stream=torch.cuda.current_stream())
    try:
        cache = Cache(width, prompt + tokens, native)
        g = torch.Generator(device="cuda").manual_seed(seed + 2)
        logits = prefill(model, ctx, cache, torch.randint(VOCAB, (prompt,), generator=g, device="cuda", dtype=torch.int32))
        logits = logits.repeat(width, 1)
        # all beams start as the first: the others have no chance until they are its children
        score = torch.full((1, width), -torch.inf, device="cuda")
        score[0, 0] = 0.0
        done = torch.zeros((1, width), device="cuda", dtype=torch.int32) if end_token >= 0 else None
        history = torch.zeros((width, 0), device="cuda", dtype=torch.int32)
        depth = torch.zeros(width, device="cuda", dtype=torch.int32)
        for step in range(tokens):
            parent, token, sums = (torch.empty((1, width), device="cuda", dtype=t) for t in (torch.int32, torch.int32, torch.float32))
            ended = None if done is None else torch.empty_like(done)
            c2kv.c2kv_beam_select(ctx, logits, score, parent, token, sums, norm=torch.logsumexp(logits, -1), done=done, end_token=end_token,
                                  done_out=ended)
            score, done = sums, ended
            history = torch.cat([history[parent[0].clamp(min=0).long()], token.t()], 1)
            if step + 1 == tokens:
                break
            table = torch.empty_like(cache.table)
            c2kv.c2kv_paged_reorder(ctx, cache.layers, cache.table, [cache.rows], parent, table)
            cache.table = table
            logits = forward(model, ctx, cache, token[0].clamp(min=0), depth, sequences=width)
            cache.rows += 1
        c2kv.c2kv_sync(ctx)
        return history, score[0]
    finally:
        c2kv.c2kv_destroy(ctx)


def main():
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--tokens", type=int, default=64)
    ap.add_argument("--branch", type=int, default=3)
    ap.add_argument("--levels", type=int, default=4)
    ap.add_argument("--width", type=int, default=4)
    ap.add_argument("--native", action="store_true")
    a = ap.parse_args()
    answer, passes = generate(a.tokens, a.branch, a.levels, a.native)
    print(f"{len(answer)} tokens in {passes} passes: {answer}")
    best, score = beams(a.tokens, a.width, a.native)
    print(f"best of {a.width} beams, {float(score[0]):.3f}: {best[0].tolist()}")


if __name__ == "__main__":
    main()
