"""Paged attention of a few tokens over values near the largest that 8-bit rows and bf16 outputs have: the output is their
mean, whatever their sum is.  Tolerance: 5e-3 of a row's norm, as over values near one (test_gpu_paged_errors.py)."""
import pytest
import torch

from tests import _dense_pages as D
from tests import _paged_helpers as P
from tests._tree_helpers import chain

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("size", [2.0 ** 60, 2.0 ** 111, 2.0 ** 124])
@pytest.mark.parametrize("n,x", [(1, 300), (1, 20000), (3, 5000), (8, 900)])
@pytest.mark.parametrize("hq,hkv,d", [(32, 8, 128), (28, 4, 64)])
def test_large_values(hq, hkv, d, n, x, size):
    gen = torch.Generator(device="cuda").manual_seed(1)
    k, v = (torch.randn((x + n, hkv, d), generator=gen, device="cuda", dtype=torch.float64) for _ in range(2))
    rows = D.Rows("bf16", "e4m3", [k], [(1 + 0.25 * v).clamp(0.25, 2) * size], 64)
    q = torch.randn((n, hq, d), generator=gen, device="cuda").bfloat16()
    c2kv, ctx = P.lib(), P.context("bf16", hq, hkv, d)
    try:
        out = torch.empty_like(q)
        c2kv.c2kv_paged_attend(ctx, rows.pages(), rows.table, [0, n], [x + n], q, out)
        c2kv.c2kv_sync(ctx)
    finally:
        c2kv.c2kv_destroy(ctx)
    want, _ = D.attend_tree(q.double(), rows.k[0], rows.v[0], chain(n))
    assert torch.isfinite(out).all() and D.relative(out, want) <= 5e-3
