"""Rows of paged attention whose every seen score is -inf: the softmax of them is not a number, and neither is
the output.  Zeros belong to a row that sees no key at all."""
import numpy as np
import pytest
import torch

from oracle import paged_oracle as orc
from tests import _paged_helpers as P

pytestmark = pytest.mark.gpu

SHAPES = [("bf16", "native", 32, 8, 128), ("bf16", "native", 8, 2, 64), ("f32", "native", 16, 4, 64), ("f32", "native", 6, 2, 128),
          ("f32", "native", 4, 4, 64)]
TOL = {"bf16": 2e-2, "f32": 1e-5}


def _paged(shape, lens, edit, window=0, table=None):
    dtype, fmt, hq, hkv, d = shape
    rng = np.random.default_rng(3)
    c2kv, ctx = P.lib(), P.context(dtype, hq, hkv, d)
    try:
        pg = P.Paged(rng, dtype, fmt, hkv, d, 32, [k for _, k in lens])
        pg.fill_rows(rng)
        edit(pg)
        ptr = np.cumsum([0] + [n for n, _ in lens]).tolist()
        q = torch.from_numpy(rng.standard_normal((ptr[-1], hq, d)).astype(np.float32))
        q[..., 3] = q[..., 3].abs() + 0.1
        q = q.to(P.TDT[dtype]).cuda()
        out, lse = torch.full_like(q, 7.0), torch.full((hq, ptr[-1]), 7.0, device="cuda")
        c2kv.c2kv_paged_attend(ctx, pg.pages(), pg.table, ptr, [k for _, k in lens], q, out, lse=lse, window=window)
        bad = False
        try:
            c2kv.c2kv_sync(ctx)
        except c2kv.C2KVError as e:
            assert e.status == c2kv.ERR_DEVICE_BOUNDS
            bad = True
        hk, hv = pg.host()
        want = []
        for r, (n, keys) in enumerate(lens):
            k, v = (orc.rows_of(x, pg.table_np, r, 0, keys, 32) for x in (hk, hv))
            with np.errstate(invalid="ignore"):
                want.append(orc.attend(q[ptr[r]:ptr[r + 1]].double().cpu().numpy(), k, v, keys, window)[0])
        return out.float().cpu().numpy(), lse.cpu().numpy(), np.concatenate(want), ptr, bad
    finally:
        c2kv.c2kv_destroy(ctx)


def _near(out, want, dtype):
    assert np.array_equal(np.isnan(out), np.isnan(want))
    fine = np.isfinite(want)
    assert np.all(np.abs(out - want)[fine] <= TOL[dtype] + TOL[dtype] * np.abs(want[fine]))


@pytest.mark.parametrize("nq", [1, 3, 140])
@pytest.mark.parametrize("keys", [40, 300, 9000])
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "-".join(map(str, s)))
def test_paged_keys_of_infinity(shape, keys, nq):
    """Every key of one request, beside a request of finite keys and one of no rows (zeros)."""
    nq = min(nq, keys)

    def edit(pg):
        pages = torch.from_numpy(pg.table_np[0][:-(-keys // 32)].astype(np.int64)).cuda()
        pg.k[pages, :, :, 3] = -float("inf")
    out, lse, want, ptr, bad = _paged(shape, [(nq, keys), (nq, 500), (2, 0)], edit)
    assert np.isnan(want[:nq]).all() and not bad
    _near(out, want, shape[0])
    assert np.isneginf(lse[:, :nq]).all() and np.isfinite(lse[:, nq:2 * nq]).all()
    assert not out[2 * nq:].any() and np.isneginf(lse[:, 2 * nq:]).all()


@pytest.mark.parametrize("nq,keys", [(40, 40), (200, 200)])
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "-".join(map(str, s)))
def test_paged_first_and_windowed_rows(shape, nq, keys):
    """The first query sees one key, and under a window of one each does: those of infinity give no number, and
    queries that see others too leave them out."""
    def edit(pg):
        for row in (0, 7, keys - 1):
            pg.k[int(pg.table_np[0, row // 32]), :, row % 32, 3] = -float("inf")
    for window, rows in ((0, [0]), (1, [0, 7, keys - 1])):
        out, lse, want, ptr, bad = _paged(shape, [(nq, keys)], edit, window)
        assert np.isnan(want[rows]).all() and np.isnan(want).all((1, 2)).sum() == len(rows)
        _near(out, want, shape[0])
        assert np.isneginf(lse[:, rows]).all()


@pytest.mark.parametrize("nq", [1, 140])
@pytest.mark.parametrize("keys", [150, 9000])
@pytest.mark.parametrize("shape", [("bf16", "e4m3", 32, 8, 128), *SHAPES], ids=lambda s: "-".join(map(str, s)))
def test_paged_rows_that_see_no_page(shape, keys, nq):
    """All pages refused: no key is seen, whatever the scores would have been."""
    nq = min(nq, keys)

    def edit(pg):
        if pg.ks is None:
            pg.k[..., 3] = -float("inf")
        pg.table.fill_(-1)
    out, lse, want, ptr, bad = _paged(shape, [(nq, keys)], edit)
    assert bad and not out.any() and np.isneginf(lse).all()
