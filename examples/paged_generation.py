"""Generation over a paged cache, from reused documents to a stored answer.

    python examples/paged_generation.py [--drafts 4] [--tokens 64] [--native]

A small decoder of random weights stands in for a model.  What a serving program does around it is
real:

1. documents are compressed into the chunk pool, and the request's are composed into one cache;
2. the composed rows move into pages, 8-bit unless --native is given, as they are (turned already);
3. the question is appended and attended as one chunk;
4. tokens are drafted (here: by the same weights with the last layer left out), appended together,
   attended in one pass, and verified against the model's probabilities; the rows of refused drafts
   are simply written over by the next ones;
5. the answer's rows are read back, turned to before RoPE, and stored as a chunk that later requests
   can reuse.
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2607_17715_gb300 import c2kv  # noqa: E402

LAYERS, HQ, HKV, D, VOCAB, PAGE, THETA, RATIO = 3, 16, 4, 128, 4000, 32, 1.0e4, 4
E = HQ * D


class Decoder:
    """Random weights, with the library's attention over pages in every layer."""

    def __init__(self, seed):
        g = torch.Generator(device="cuda").manual_seed(seed)

        def w(*shape):
            return torch.randn(shape, generator=g, device="cuda", dtype=torch.bfloat16) * shape[-2] ** -0.5
        self.embed = torch.randn((VOCAB, E), generator=g, device="cuda", dtype=torch.bfloat16)
        self.qkv = [w(E, (HQ + 2 * HKV) * D) for _ in range(LAYERS)]
        self.out = [w(E, E) for _ in range(LAYERS)]
        self.head = w(E, VOCAB)

    @staticmethod
    def norm(x):
        return torch.nn.functional.rms_norm(x.float(), (E,)).to(x.dtype)

    def forward(self, ctx, cache, tokens, position, layers=LAYERS):
        """Logits of `tokens` [n] that come after the cache's rows, at positions position, .. + n - 1;
        their keys and values are left in the pages after the cache's rows."""
        n = tokens.shape[0]
        pos = torch.arange(position, position + n, device="cuda", dtype=torch.int32)
        x = self.embed[tokens.long()]
        for i in range(layers):
            rows = (self.norm(x) @ self.qkv[i]).view(n, HQ + 2 * HKV, D)
            q, k, v = rows[:, :HQ], rows[:, HQ:HQ + HKV], rows[:, HQ + HKV:]
            c2kv.c2kv_paged_append(ctx, cache.pages[i], cache.table, [0, n], [cache.rows], k, v, turn=pos)
            out = torch.empty((n, HQ, D), device="cuda", dtype=torch.bfloat16)
            c2kv.c2kv_paged_attend(ctx, cache.pages[i], cache.table, [0, n], [cache.rows + n], q, out, turn=pos)
            x = x + out.view(n, E) @ self.out[i]
        return (self.norm(x) @ self.head).float()


class PagedCache:
    """One request's pages in every layer: one table, whose page numbers all layers share."""

    def __init__(self, rows, native):
        n = -(-rows // PAGE) + 2
        dtype = torch.bfloat16 if native else torch.float8_e4m3fn
        shape = (LAYERS, 2, n, HKV, PAGE, D)
        self.store = torch.zeros(shape, device="cuda", dtype=torch.bfloat16 if native else torch.uint8).view(dtype)
        self.scales = None if native else torch.zeros(shape[:-1], device="cuda")
        self.pages = [c2kv.make_pages(self.store[i, 0], self.store[i, 1], *([] if native else self.scales[i])) for i in range(LAYERS)]
        order = torch.randperm(n, generator=torch.Generator().manual_seed(1))
        self.table = order.to("cuda", torch.int32)[None]
        self.rows = 0


def compose(ctx, seed, documents, tokens):
    """Documents of random keys and values, compressed; the request's cache of them in order."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    ids = []
    for _ in range(documents):
        k, v = (torch.randn((LAYERS, tokens, HKV, D), generator=g, device="cuda", dtype=torch.bfloat16) for _ in "kv")
        ids.append(c2kv.c2kv_compress_chunk(ctx, k, v, tokens, RATIO, c2kv.MODE_MEANPOOL))
    return c2kv.c2kv_compose(ctx, [0, documents], ids)


def generate(drafts=4, tokens=64, native=False, greedy=False, seed=0, documents=6, chunk=500, question=37):
    """The generated tokens, how many passes of the model they took, and the stored answer's chunk info."""
    model = Decoder(seed)
    ctx = c2kv.c2kv_create(LAYERS, HQ, HKV, D, THETA, c2kv.DTYPE_BF16, pool_slots=8192, stream=torch.cuda.current_stream())
    try:
        composed = compose(ctx, seed + 1, documents, chunk)
        info = c2kv.c2kv_cache_info(composed)
        slots, span = int(info["n_slots"][0]), int(info["l_req"][0])
        cache = PagedCache(slots + question + tokens + drafts + 1, native)
        shape = (LAYERS, info["rows"], HKV, D)
        k, v = (c2kv.device_view(info[w], shape, torch.bfloat16) for w in "kv")
        for i in range(LAYERS):                              # composed rows are turned already
            c2kv.c2kv_paged_append(ctx, cache.pages[i], cache.table, [0, slots], [0], k[i, :slots], v[i, :slots])
        c2kv.c2kv_cache_release(ctx, composed)
        cache.rows = slots

        g = torch.Generator(device="cuda").manual_seed(seed + 2)
        prompt = torch.randint(VOCAB, (question,), generator=g, device="cuda", dtype=torch.int32)
        position = span                                      # a row's position runs ahead of its place: slots stand for RATIO tokens

        def probabilities(logits):
            if greedy:
                return torch.nn.functional.one_hot(logits.argmax(-1), VOCAB).float()
            return torch.softmax(logits, -1)

        logits = model.forward(ctx, cache, prompt, position)
        cache.rows += question
        position += question
        first = slots + question                             # the answer's first row
        accepted, following = (torch.empty(1, dtype=torch.int32, device="cuda") for _ in range(2))

        def verify(p, q, drafted):
            n = drafted.shape[0]
            u = torch.rand(n + 1, generator=g, device="cuda")
            c2kv.c2kv_verify_drafts(ctx, [0, n], drafted, p, q, u[:n], u[n:], accepted, following)
            return int(accepted), int(following)

        none = torch.empty(0, dtype=torch.int32, device="cuda")
        _, token = verify(probabilities(logits[-1:]), None, none)
        answer, passes = [token], 1
        while len(answer) < tokens:
            # drafts: token by token through the layers but the last, whose rows the full pass writes again
            drafted, q_rows, t, rows = [], [], answer[-1], cache.rows
            for j in range(drafts):
                q = probabilities(model.forward(ctx, cache, torch.tensor([t], device="cuda"), position + j, LAYERS - 1))
                cache.rows += 1
                t = int(torch.multinomial(q[0], 1, generator=g))
                drafted.append(t)
                q_rows.append(q)
            cache.rows = rows
            step = torch.tensor([answer[-1]] + drafted, device="cuda", dtype=torch.int32)
            p = probabilities(model.forward(ctx, cache, step, position))
            kept, token = verify(p, torch.cat(q_rows) if drafts else None, step[1:].contiguous())
            answer += drafted[:kept] + [token]
            cache.rows += kept + 1                           # the rows of refused drafts lie past them, to be written over
            position += kept + 1
            passes += 1

        # the answer as a chunk: its rows turned back by their positions, to before RoPE
        n = cache.rows - first
        back = -torch.arange(span + question, span + question + n, device="cuda", dtype=torch.int32)
        k, v = (torch.empty((LAYERS, n, HKV, D), device="cuda", dtype=torch.bfloat16) for _ in "kv")
        for i in range(LAYERS):
            c2kv.c2kv_paged_gather(ctx, cache.pages[i], cache.table, [0, n], [first], k[i], v[i], turn=back)
        stored = c2kv.c2kv_compress_chunk(ctx, k, v, n, RATIO, c2kv.MODE_MEANPOOL)
        c2kv.c2kv_sync(ctx)
        return answer[:tokens], passes, c2kv.c2kv_chunk_info(ctx, stored)
    finally:
        c2kv.c2kv_destroy(ctx)


def main():
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--drafts", type=int, default=4)
    ap.add_argument("--tokens", type=int, default=64)
    ap.add_argument("--native", action="store_true")
    a = ap.parse_args()
    answer, passes, chunk = generate(a.drafts, a.tokens, a.native)
    print(f"{len(answer)} tokens in {passes} passes; stored as a chunk of {chunk['n_slots']} slots")
    print(answer)


if __name__ == "__main__":
    main()
