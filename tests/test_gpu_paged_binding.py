"""The binding of the paged calls knows the context that it made: rows of another type and pages of other heads are
refused before the call."""
import numpy as np
import pytest
import torch

from tests import _paged_helpers as P

pytestmark = pytest.mark.gpu


def test_rows_and_pages_must_be_the_contexts():
    rng = np.random.default_rng(0)
    c2kv = P.lib()
    bf16, f32, wide = P.context("bf16", 4, 2, 64), P.context("f32", 4, 2, 64), P.context("bf16", 8, 4, 64)
    try:
        codes, native = P.Paged(rng, "bf16", "e4m3", 2, 64, 16, [40], fill=0.0), P.Paged(rng, "bf16", "native", 2, 64, 16, [40], fill=0.0)
        kv, q = torch.zeros((3, 2, 64), device="cuda", dtype=torch.bfloat16), torch.zeros((3, 4, 64), device="cuda", dtype=torch.bfloat16)

        def calls(ctx, pages, kv, q):
            c2kv.c2kv_paged_append(ctx, pages, codes.table, [0, 3], [30], kv, kv)
            c2kv.c2kv_paged_gather(ctx, pages, codes.table, [0, 3], [30], torch.empty_like(kv), torch.empty_like(kv))
            c2kv.c2kv_paged_attend(ctx, pages, codes.table, [0, 3], [33], q, torch.empty_like(q))
        shared = codes.pages()
        calls(bf16, shared, kv, q)
        calls(bf16, native.pages(), kv, q)
        calls(f32, shared, kv.float(), q.float())            # 8-bit pages are either's
        calls(bf16, shared, kv, q)
        for ctx, pages, a, b in ((bf16, shared, kv.float(), q.float()), (f32, shared, kv, q), (f32, native.pages(), kv.float(), q.float()),
                                 (bf16, shared, kv.half(), q.half()), (wide, shared, kv, torch.cat([q, q], 1)),
                                 (wide, codes.pages(), torch.cat([kv, kv], 1), torch.cat([q, q], 1))):
            for name, args in (("append", ([30], a, a)), ("gather", ([30], a, a)), ("attend", ([33], b, b))):
                with pytest.raises(ValueError):
                    getattr(c2kv, "c2kv_paged_" + name)(ctx, pages, codes.table, [0, 3], *args)
        for ctx in (bf16, f32):
            c2kv.c2kv_sync(ctx)
    finally:
        for ctx in (bf16, f32, wide):
            c2kv.c2kv_destroy(ctx)


def test_a_destroyed_contexts_handle_says_nothing_of_the_next():
    """A handle may come back for another context: its heads and type are the new one's."""
    rng = np.random.default_rng(0)
    c2kv = P.lib()
    pg = P.Paged(rng, "bf16", "e4m3", 2, 64, 16, [40], fill=0.0)
    pages = pg.pages()
    for dtype in ("bf16", "f32", "bf16"):
        ctx = P.context(dtype, 4, 2, 64)
        x = torch.zeros((1, 2, 64), device="cuda", dtype=P.TDT[dtype])
        c2kv.c2kv_paged_append(ctx, pages, pg.table, [0, 1], [3], x, x)
        other = x.float() if dtype == "bf16" else x.bfloat16()
        with pytest.raises(ValueError):
            c2kv.c2kv_paged_append(ctx, pages, pg.table, [0, 1], [3], other, other)
        c2kv.c2kv_sync(ctx)
        c2kv.c2kv_destroy(ctx)
