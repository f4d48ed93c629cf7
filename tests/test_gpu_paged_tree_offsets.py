"""Attention of trees over pages that lie far apart (offsets past 32 bits, other layers' pages in between) and over pages that
requests share.  Tolerances as test_gpu_paged_tree_errors.py."""
import numpy as np
import pytest
import torch

from tests import _dense_pages as D
from tests import _paged_helpers as P
from tests._tree_helpers import random_tree

pytestmark = pytest.mark.gpu
TOL = {"bf16": 5e-3, "f32": 1e-5}
SHAPES = [("bf16", "e4m3", 32, 8, 128), ("bf16", "native", 32, 8, 128), ("f32", "e4m3", 8, 2, 64), ("f32", "native", 8, 2, 64)]


def _data(shape, counts, size, trees):
    dtype, fmt, hq, hkv, d = shape
    gen = torch.Generator(device="cuda").manual_seed(4)
    k, v = ([torch.randn((n, hkv, d), generator=gen, device="cuda") for n in counts] for _ in range(2))
    q = torch.randn((sum(len(t) for t in trees), hq, d), generator=gen, device="cuda").to(P.TDT[dtype])
    return D.Rows(dtype, fmt, k, v, size), q


@pytest.mark.parametrize("n", [3, 12, 100, 200])
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "-".join(map(str, s)))
def test_pages_far_apart(shape, n):
    """Elements 2^29 and scales 2^28 from page to page, eight pages: past 2^32 of them, K's and V's in one allocation."""
    dtype, fmt, hq, hkv, d = shape
    tree = random_tree(np.random.default_rng(n), n, near=9)
    rows, q = _data(shape, [700 + n], 128, [tree])
    far = []
    pools = [torch.empty(10 * 2 ** 29, dtype=rows.held[0][0].dtype, device="cuda"),
             torch.empty(10 * 2 ** 28, device="cuda") if fmt == "e4m3" else None]
    for i, (pages, scale, stand) in enumerate(rows.held):
        moved = []
        for x, pool, stride in ((pages, pools[0], 2 ** 29 + 4096), (scale, pools[1], 2 ** 28 + 4096)):
            if x is None:
                moved.append(None)
                continue
            y = torch.as_strided(pool, x.shape, (stride, *x.stride()[1:]), i * 2 ** 21)
            for page in range(len(x)):
                (y[page].view(torch.uint8) if x.element_size() == 1 else y[page]).copy_(x[page].view(torch.uint8) if x.element_size() == 1 else x[page])
            moved.append(y)
        far.append((*moved, stand))
    assert far[0][0].stride(0) * (len(far[0][0]) - 1) > 2 ** 31
    rows.held = far
    call = D.Call(dtype, hq, hkv, d, rows, [tree], q)
    assert D.relative(call.out, call.want()[0]) <= TOL[dtype]


@pytest.mark.parametrize("n", [3, 20, 100])
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "-".join(map(str, s)))
def test_pages_that_requests_share(shape, n):
    """Three requests go on from one prefix of 40 pages, each with a tree in pages of its own."""
    dtype, fmt, hq, hkv, d = shape
    trees = [random_tree(np.random.default_rng(n + i), n + i, near=9) for i in range(3)]
    rows, q = _data(shape, [40 * 32 + 5 + len(t) for t in trees], 32, trees)
    for r in (1, 2):
        rows.table[r, :40] = rows.table[0, :40]
        for x in (rows.k, rows.v):
            x[r][:40 * 32] = x[0][:40 * 32]
    call = D.Call(dtype, hq, hkv, d, rows, trees, q)
    assert D.relative(call.out, call.want()[0]) <= TOL[dtype]
