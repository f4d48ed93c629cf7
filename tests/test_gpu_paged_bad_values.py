"""Values of V that are not finite, in paged attention: they belong to the queries that see them, channel by
channel, and cost the others neither their result nor their time."""
import numpy as np
import pytest
import torch

from oracle import paged_oracle as orc
from tests import _paged_helpers as P

pytestmark = pytest.mark.gpu
INF, NAN = float("inf"), float("nan")
TOL = {"bf16": 2e-2, "f32": 1e-5}
SHAPES = [("bf16", "native", 32, 8, 128), ("bf16", "native", 8, 2, 64), ("bf16", "e4m3", 32, 8, 128), ("bf16", "e4m3", 8, 2, 64)]


def _set(pg, key, channel, value):
    """One value of a row (native pages), or the row's scale or one code (8-bit ones) made not finite."""
    page, at = int(pg.table_np[0, key // 32]), key % 32
    if pg.vs is None:
        pg.v[page, :, at, channel] = value
    elif channel is None:
        pg.vs[page, :, at] = value
    else:
        pg.v.view(torch.uint8)[page, :, at, channel] = 0x7f if value > 0 else 0xff


@pytest.mark.parametrize("window", [0, 90])
@pytest.mark.parametrize("nq,keys", [(140, 200), (300, 300), (70, 9000), (260, 5000)])
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "-".join(map(str, s)))
def test_every_channel_is_its_own(shape, nq, keys, window):
    dtype, fmt, hq, hkv, d = shape
    rng = np.random.default_rng(6)
    c2kv, ctx = P.lib(), P.context(dtype, hq, hkv, d)
    try:
        pg = P.Paged(rng, dtype, fmt, hkv, d, 32, [keys, 77])
        pg.fill_rows(rng)
        spots = [(2, 5, INF), (keys // 2, 6, -INF), (keys - nq, 7, INF), (keys - nq + 1, 7, -INF), (keys - 60, 8, NAN), (keys - 1, 9, INF),
                 (keys - 59, d - 1, INF), (keys - 33, 5, INF)]
        for key, channel, value in spots:
            _set(pg, key, channel, value)
        q = torch.from_numpy(rng.standard_normal((nq + 66, hq, d)).astype(np.float32)).to(P.TDT[dtype]).cuda()
        out, lse = torch.full_like(q, 7.0), torch.empty((hq, nq + 66), device="cuda")
        c2kv.c2kv_paged_attend(ctx, pg.pages(), pg.table, [0, nq, nq + 66], [keys, 77], q, out, lse=lse, window=window)
        c2kv.c2kv_sync(ctx)
        hk, hv = pg.host()
        out = out.float().cpu().numpy()
        for r, (lo, hi, n) in enumerate(((0, nq, keys), (nq, nq + 66, 77))):
            k, v = (orc.rows_of(x, pg.table_np, r, 0, n, 32) for x in (hk, hv))
            with np.errstate(invalid="ignore"):
                want, want_l = orc.attend(q[lo:hi].double().cpu().numpy(), k, v, n, window)
            got = out[lo:hi]
            assert np.array_equal(np.isnan(got), np.isnan(want)) and np.array_equal(np.isposinf(got), np.isposinf(want)) and \
                np.array_equal(np.isneginf(got), np.isneginf(want))
            fine = np.isfinite(want)
            assert (r == 1) == fine.all()
            assert np.all(np.abs(got - want)[fine] <= TOL[dtype] + TOL[dtype] * np.abs(want[fine]))
            assert np.abs(lse[:, lo:hi].cpu().numpy() - want_l).max() <= TOL[dtype]
    finally:
        c2kv.c2kv_destroy(ctx)


@pytest.mark.parametrize("key", [3, 7900])
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "-".join(map(str, s)))
def test_a_chunk_over_one_bad_row_takes_its_usual_time(shape, key):
    """256 tokens over 8192 rows; a row that is not finite may make it twice as long."""
    dtype, fmt, hq, hkv, d = shape
    rng = np.random.default_rng(7)
    c2kv, ctx = P.lib(), P.context(dtype, hq, hkv, d)
    try:
        pg = P.Paged(rng, dtype, fmt, hkv, d, 32, [8192], fill=0.5)
        q = torch.randn((256, hq, d), device="cuda").to(P.TDT[dtype])
        out = torch.empty_like(q)
        pages = pg.pages()

        def time():
            took = []
            for _ in range(6):
                a, b = (torch.cuda.Event(enable_timing=True) for _ in range(2))
                a.record()
                c2kv.c2kv_paged_attend(ctx, pages, pg.table, [0, 256], [8192], q, out)
                b.record()
                torch.cuda.synchronize()
                took.append(a.elapsed_time(b))
            return min(took)
        usual = time()
        _set(pg, key, 3 if fmt == "native" else None, NAN)
        assert time() <= 2 * usual
        assert out[..., 3].isnan().any()
    finally:
        c2kv.c2kv_destroy(ctx)


@pytest.mark.parametrize("window", [0, 90])
@pytest.mark.parametrize("nq,keys", [(1, 300), (3, 300), (10, 2000), (5, 9000)])
@pytest.mark.parametrize("shape", [*SHAPES[:2], ("bf16", "native", 28, 4, 128), ("bf16", "native", 4, 4, 64)], ids=lambda s: "-".join(map(str, s)))
def test_every_channel_is_its_own_of_few_rows(shape, nq, keys, window):
    test_every_channel_is_its_own(shape, nq, keys, window)


@pytest.mark.parametrize("nq,batch", [(1, 64), (4, 64), (1, 1)])
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "-".join(map(str, s)))
def test_few_rows_over_one_bad_row_take_their_usual_time(shape, nq, batch):
    """Requests over the same 8192 rows; a row that is not finite may make them twice as long."""
    dtype, fmt, hq, hkv, d = shape
    rng = np.random.default_rng(7)
    c2kv, ctx = P.lib(), P.context(dtype, hq, hkv, d)
    try:
        pg = P.Paged(rng, dtype, fmt, hkv, d, 32, [8192], fill=0.5)
        q = torch.randn((nq * batch, hq, d), device="cuda").to(P.TDT[dtype])
        out, table, pages = torch.empty_like(q), pg.table.repeat(batch, 1), pg.pages()

        def time():
            took = []
            for _ in range(8):
                a, b = (torch.cuda.Event(enable_timing=True) for _ in range(2))
                a.record()
                c2kv.c2kv_paged_attend(ctx, pages, table, [nq * i for i in range(batch + 1)], [8192] * batch, q, out)
                b.record()
                torch.cuda.synchronize()
                took.append(a.elapsed_time(b))
            return min(took)
        usual = time()
        _set(pg, 5000, 3 if fmt == "native" else None, NAN)
        assert time() <= 2 * usual
        assert out[..., 3].isnan().all()
    finally:
        c2kv.c2kv_destroy(ctx)


@pytest.mark.parametrize("nq,keys", [(1, 300), (3, 300), (5, 9000), (140, 200), (140, 9000)])
@pytest.mark.parametrize("shape", [*SHAPES[:2], ("f32", "native", 16, 4, 64), ("f32", "native", 4, 4, 128)], ids=lambda s: "-".join(map(str, s)))
def test_infinite_values_of_keys_of_no_weight(shape, nq, keys):
    """A key that scores -inf has weight 0, and 0 times an infinity is NaN: for the rows that see it, in the
    channels where its value is one."""
    dtype, fmt, hq, hkv, d = shape
    rng = np.random.default_rng(6)
    c2kv, ctx = P.lib(), P.context(dtype, hq, hkv, d)
    try:
        pg = P.Paged(rng, dtype, fmt, hkv, d, 32, [keys])
        pg.fill_rows(rng)
        for key, channel, value in ((4, 5, INF), (keys // 2, 6, -INF), (keys - 1, 7, INF), (keys - 1, 8, NAN)):
            _set(pg, key, channel, value)
            pg.k[int(pg.table_np[0, key // 32]), :, key % 32, 3] = -INF
        _set(pg, 40, 9, INF)                                  # and one of a key that has its weight
        q = torch.from_numpy(rng.standard_normal((nq, hq, d)).astype(np.float32))
        q[..., 3] = q[..., 3].abs() + 0.1
        q = q.to(P.TDT[dtype]).cuda()
        out = torch.full_like(q, 7.0)
        c2kv.c2kv_paged_attend(ctx, pg.pages(), pg.table, [0, nq], [keys], q, out)
        c2kv.c2kv_sync(ctx)
        k, v = (orc.rows_of(x, pg.table_np, 0, 0, keys, 32) for x in pg.host())
        with np.errstate(invalid="ignore"):
            want, _ = orc.attend(q.double().cpu().numpy(), k, v, keys)
        got = out.float().cpu().numpy()
        assert np.isnan(want[-1][..., [5, 6, 7, 8]]).all() and np.isposinf(want[..., 9]).all()
        assert np.array_equal(np.isnan(got), np.isnan(want)) and np.array_equal(np.isposinf(got), np.isposinf(want))
        fine = np.isfinite(want)
        assert np.all(np.abs(got - want)[fine] <= TOL[dtype] + TOL[dtype] * np.abs(want[fine]))
    finally:
        c2kv.c2kv_destroy(ctx)
