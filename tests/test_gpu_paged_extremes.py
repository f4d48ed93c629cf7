"""Paged attention at the ends of the types' ranges: queries far smaller or larger than one over keys of zero, or
that they do not meet.  All scores are zero, so a row is the mean of the values it sees."""
import numpy as np
import pytest
import torch

from oracle import paged_oracle as orc
from tests import _paged_helpers as P

pytestmark = pytest.mark.gpu

SHAPES = [("bf16", "e4m3", 32, 8, 128), ("bf16", "native", 32, 8, 128), ("bf16", "e4m3", 8, 2, 64), ("bf16", "native", 8, 2, 64),
          ("f32", "native", 16, 4, 64), ("f32", "e4m3", 8, 2, 128)]
TOL = {"bf16": 5e-3, "f32": 1e-5}        # of a row's norm: bf16's rounding is at most 2^-9 of it


@pytest.mark.parametrize("q_size,k_size", [(2.0 ** -40, 0.0), (2.0 ** -90, 0.0), (2.0 ** 100, 0.0), (2.0 ** -60, 2.0 ** -60), (2.0 ** 100, 2.0 ** 60)])
@pytest.mark.parametrize("nq,keys", [(1, 300), (140, 300), (64, 6000)])
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "-".join(map(str, s)))
def test_scores_of_zero(shape, nq, keys, q_size, k_size):
    dtype, fmt, hq, hkv, d = shape
    rng = np.random.default_rng(2)
    c2kv, ctx = P.lib(), P.context(dtype, hq, hkv, d)
    try:
        pg = P.Paged(rng, dtype, fmt, hkv, d, 64, [keys])
        pg.fill_rows(rng)
        raw = torch.uint8 if fmt == "e4m3" else torch.int16 if dtype == "bf16" else torch.int32
        pg.k.view(raw).zero_()
        if fmt == "e4m3":
            pg.ks.fill_(k_size / 448)
            pg.k[..., 1] = 448.0 if k_size else 0.0
        else:
            pg.k[..., 1] = k_size
        q = torch.zeros((nq, hq, d), device="cuda", dtype=P.TDT[dtype])
        q[..., 0] = q_size
        out, lse = torch.empty_like(q), torch.empty((hq, nq), device="cuda")
        c2kv.c2kv_paged_attend(ctx, pg.pages(), pg.table, [0, nq], [keys], q, out, lse=lse)
        c2kv.c2kv_sync(ctx)
        _, v = pg.host()
        v = orc.rows_of(v, pg.table_np, 0, 0, keys, 64)
        want = np.cumsum(v, 0)[keys - nq:] / np.arange(keys - nq + 1, keys + 1)[:, None, None]
        want = np.repeat(want, hq // hkv, 1)
        err = np.linalg.norm(out.double().cpu().numpy() - want, axis=-1) / np.linalg.norm(want, axis=-1)
        assert err.max() <= TOL[dtype]
        assert np.abs(lse.cpu().numpy() - np.log(np.arange(keys - nq + 1, keys + 1))).max() <= 1e-4
    finally:
        c2kv.c2kv_destroy(ctx)
