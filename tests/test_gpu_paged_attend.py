"""Attention over pages (c2kv_paged_attend) against fp64 over the rows that the pages stand for.

Tolerances: those of the library's attention over composed caches, atol = rtol = 2e-2 for bf16 and
1e-5 for fp32; lse within 2e-2 (a score of magnitude below 8 whose query was rounded to 8 bits is off
by at most 8 * 2^-8 / sqrt(d) * a few) and 1e-5 of its magnitude plus one."""
import numpy as np
import pytest
import torch

from oracle import paged_oracle as orc
from tests import _paged_helpers as P

pytestmark = pytest.mark.gpu
TOL = {"bf16": 2e-2, "f32": 1e-5}


def _run(dtype, fmt, hq, hkv, d, size, lens, window=0, turn=True, theta=1.0e4, seed=1, edit=None, q_scale=1.0):
    """lens: (queries, rows) per request.  Returns out, lse and the fp64 ones."""
    rng = np.random.default_rng(seed)
    c2kv, ctx = P.lib(), P.context(dtype, hq, hkv, d, theta)
    try:
        pg = P.Paged(rng, dtype, fmt, hkv, d, size, [k for _, k in lens])
        pg.fill_rows(rng)
        if edit:
            edit(pg)
        ptr = np.cumsum([0] + [n for n, _ in lens]).tolist()
        T = ptr[-1]
        q = torch.from_numpy((rng.standard_normal((T, hq, d)) * q_scale).astype(np.float32)).to(P.TDT[dtype]).cuda()
        pos = torch.from_numpy(rng.integers(0, 200000, max(T, 1)).astype(np.int32)).cuda()
        out = torch.full((T, hq, d), 7.0, device="cuda", dtype=P.TDT[dtype])
        lse = torch.full((hq, T), 7.0, device="cuda")
        c2kv.c2kv_paged_attend(ctx, pg.pages(), pg.table, ptr, [k for _, k in lens], q, out, lse=lse,
                               turn=pos if turn else None, window=window)
        c2kv.c2kv_sync(ctx)
        q64 = q.float().cpu().numpy().astype(np.float64)
        if turn:
            q64 = orc.turned(q64, pos.cpu().numpy()[:T], theta)
        hk, hv = pg.host()
        want, want_l = np.zeros((T, hq, d)), np.zeros((hq, T))
        for r, (n, keys) in enumerate(lens):
            k, v = (orc.rows_of(x, pg.table_np, r, 0, keys, size) for x in (hk, hv))
            with np.errstate(invalid="ignore"):
                want[ptr[r]:ptr[r + 1]], want_l[:, ptr[r]:ptr[r + 1]] = orc.attend(q64[ptr[r]:ptr[r + 1]], k, v, keys, window)
        return out.float().cpu().numpy(), lse.cpu().numpy(), want, want_l
    finally:
        c2kv.c2kv_destroy(ctx)


def _check(got, dtype):
    out, lse, want, want_l = got
    tol = TOL[dtype]
    assert np.array_equal(np.isnan(out), np.isnan(want))
    fine = np.isfinite(want)
    assert np.all(np.abs(out - want)[fine] <= tol + tol * np.abs(want[fine]))
    assert np.array_equal(np.isneginf(lse), np.isneginf(want_l)) and np.array_equal(np.isnan(lse), np.isnan(want_l))
    fine = np.isfinite(want_l)
    assert np.all(np.abs(lse - want_l)[fine] <= tol * (1 + np.abs(want_l[fine]) * (dtype == "f32")))


SHAPES = [  # dtype, fmt, hq, hkv, d
    ("bf16", "e4m3", 32, 8, 128), ("bf16", "native", 32, 8, 128), ("bf16", "e4m3", 8, 8, 128), ("bf16", "e4m3", 16, 2, 128),
    ("bf16", "native", 28, 4, 128), ("bf16", "e4m3", 28, 4, 64), ("bf16", "native", 8, 2, 64), ("bf16", "e4m3", 20, 1, 128),
    ("bf16", "native", 4, 4, 64), ("f32", "native", 16, 4, 64), ("f32", "e4m3", 8, 2, 128), ("f32", "native", 6, 2, 128),
]
LENS = [  # page size, (queries, rows) per request
    (16, [(1, 1)]),
    (16, [(1, 37), (0, 12), (5, 5), (3, 130), (1, 0), (0, 0), (4, 2)]),   # no query, no row, rows that see nothing
    (64, [(1, 700), (2, 64), (9, 65), (1, 1300)]),
    (128, [(33, 129), (70, 300)]),
    (32, [(130, 513), (1, 31)]),
]


@pytest.mark.parametrize("lens", LENS, ids=["one", "ragged", "few", "chunks", "chunk"])
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "-".join(map(str, s)))
def test_shapes(shape, lens):
    _check(_run(*shape, lens[0], lens[1]), shape[0])


@pytest.mark.parametrize("window", [1, 7, 64, 100])
@pytest.mark.parametrize("shape", [SHAPES[0], SHAPES[1], SHAPES[8], SHAPES[9]], ids=lambda s: "-".join(map(str, s)))
def test_window(shape, window):
    _check(_run(*shape, 32, [(1, 300), (40, 333), (4, 3), (150, 150)], window=window), shape[0])


@pytest.mark.parametrize("nq", [3, 140])
@pytest.mark.parametrize("size", [16, 64])
@pytest.mark.parametrize("shape", [SHAPES[0], SHAPES[1], SHAPES[9]], ids=lambda s: "-".join(map(str, s)))
def test_pages_that_a_window_left_behind(shape, size, nq):
    """Pages whose rows no query sees any more may be gone from the table."""
    def edit(pg):
        pg.table[0, :(700 - nq - 37 + 1) // size] = -1
    _check(_run(*shape, size, [(nq, 700)], window=37, edit=edit), shape[0])


@pytest.mark.parametrize("shape", [SHAPES[0], SHAPES[1], SHAPES[6], SHAPES[10]], ids=lambda s: "-".join(map(str, s)))
def test_long_rows_are_split_and_joined(shape):
    _check(_run(*shape, 128, [(1, 9001), (3, 5000)], turn=False), shape[0])


@pytest.mark.parametrize("shape", [SHAPES[0], SHAPES[1], SHAPES[2], SHAPES[5]], ids=lambda s: "-".join(map(str, s)))
def test_long_chunks(shape):
    _check(_run(*shape, 64, [(300, 1100), (257, 257)]), shape[0])


@pytest.mark.parametrize("shape", [SHAPES[0], SHAPES[1], SHAPES[9]], ids=lambda s: "-".join(map(str, s)))
def test_many_requests(shape):
    rng = np.random.default_rng(2)
    _check(_run(*shape, 16, [(int(rng.integers(0, 3)), int(rng.integers(0, 60))) for _ in range(290)]), shape[0])


@pytest.mark.parametrize("q_scale", [1e-3, 30.0])
@pytest.mark.parametrize("shape", [SHAPES[0], SHAPES[1]], ids=lambda s: "-".join(map(str, s)))
def test_scales_of_scores(shape, q_scale):
    """Nearly flat and nearly one-hot softmax.  A query rounded to 8 bits moves scores by up to
    30 * 4 * 2^-8, so the one-hot case is checked by its weights' sum alone: values of one."""
    def ones(pg):
        if q_scale > 1:
            pg.v.view(torch.uint8 if pg.fmt == "e4m3" else torch.int16).copy_(
                torch.ones(pg.v.shape, device="cuda").to(pg.v.dtype).view(torch.uint8 if pg.fmt == "e4m3" else torch.int16))
            if pg.vs is not None:
                pg.vs.copy_(torch.where(pg.vs.isnan(), pg.vs, torch.ones_like(pg.vs)))
    out, lse, want, want_l = _run(*shape, 64, [(1, 900), (40, 300)], q_scale=q_scale, edit=ones)
    assert np.all(np.abs(out - want) <= 2e-2)


@pytest.mark.parametrize("value", [float("inf"), float("nan"), -float("inf")])
@pytest.mark.parametrize("nq", [6, 140])
@pytest.mark.parametrize("shape", [SHAPES[1], SHAPES[6], SHAPES[9]], ids=lambda s: "-".join(map(str, s)))
def test_values_that_only_later_queries_see(shape, nq, value):
    """A value that is not finite, in a row of the chunk itself: the queries before it must not feel it."""
    keys = 200

    def edit(pg):
        row = keys - nq // 2
        pg.v[int(pg.table_np[0, row // 32]), 1, row % 32, 3] = value
    out, lse, want, want_l = _run(*shape, 32, [(nq, keys)], edit=edit)
    touched = ~np.isfinite(want)
    assert touched.any() and not touched[:nq // 2 - 1].any()
    assert np.array_equal(np.isnan(out), np.isnan(want))
    fine = np.isfinite(want)
    tol = TOL[shape[0]]
    assert np.all(np.abs(out - want)[fine] <= tol + tol * np.abs(want[fine]))


@pytest.mark.parametrize("nq", [6, 140])
@pytest.mark.parametrize("which", ["k", "v"])
@pytest.mark.parametrize("shape", [SHAPES[0], SHAPES[5], SHAPES[10]], ids=lambda s: "-".join(map(str, s)))
def test_rows_whose_scale_is_nan(shape, which, nq):
    keys = 200

    def edit(pg):
        row = keys - nq // 2
        (pg.ks if which == "k" else pg.vs)[int(pg.table_np[0, row // 32]), 1, row % 32] = float("nan")
    out, lse, want, want_l = _run(*shape, 32, [(nq, keys)], edit=edit)
    g = shape[2] // shape[3]
    first = nq // 2 - 1                                  # the first query that sees the row
    seen = np.zeros(out.shape[:2], bool)
    seen[first + 1 if (keys - nq // 2) > (keys - nq + first) else first:, g:2 * g] = True
    assert np.array_equal(np.isnan(out), np.broadcast_to(seen[..., None], out.shape))
    fine = ~np.isnan(out)
    tol = TOL[shape[0]]
    assert np.all(np.abs(out - want)[fine] <= tol + tol * np.abs(want[fine]))


@pytest.mark.parametrize("shape", [SHAPES[0], SHAPES[5], SHAPES[10]], ids=lambda s: "-".join(map(str, s)))
@pytest.mark.parametrize("nq", [2, 140])
def test_scales_far_apart(shape, nq):
    """Rows whose scales span many powers of two, zero among them, in K and V."""
    rng = np.random.default_rng(9)

    def edit(pg):
        f = torch.from_numpy(2.0 ** rng.integers(-30, 4, pg.ks.shape)).float().cuda()
        f[rng.random(pg.ks.shape) < 0.1] = 0
        pg.ks *= f
        f = torch.from_numpy(2.0 ** rng.integers(-30, 1, pg.ks.shape)).float().cuda()
        f[rng.random(pg.ks.shape) < 0.1] = 0
        pg.vs *= f
    out, lse, want, want_l = _run(*shape, 16, [(nq, 300), (1, 77)], edit=edit, q_scale=0.2)
    tol = TOL[shape[0]]
    assert np.all(np.abs(out - want) <= tol + tol * np.abs(want))


@pytest.mark.parametrize("shape", [SHAPES[0], SHAPES[1], SHAPES[9]], ids=lambda s: "-".join(map(str, s)))
@pytest.mark.parametrize("nq", [1, 140])
def test_refused_page(shape, nq):
    """A page number that is none: reported, its rows unseen."""
    dtype, fmt, hq, hkv, d = shape
    rng = np.random.default_rng(4)
    c2kv, ctx = P.lib(), P.context(dtype, hq, hkv, d)
    try:
        pg = P.Paged(rng, dtype, fmt, hkv, d, 32, [200])
        pg.fill_rows(rng)
        table = pg.table.clone()
        table[0, 1] = pg.k.shape[0]
        q = torch.from_numpy(rng.standard_normal((nq, hq, d)).astype(np.float32)).to(P.TDT[dtype]).cuda()
        out = torch.empty_like(q)
        c2kv.c2kv_paged_attend(ctx, pg.pages(), table, [0, nq], [200], q, out)
        with pytest.raises(c2kv.C2KVError) as ei:
            c2kv.c2kv_sync(ctx)
        assert ei.value.status == c2kv.ERR_DEVICE_BOUNDS
        k, v = pg.dense(0)
        q64 = q.float().cpu().numpy().astype(np.float64)
        keep = np.ones(200, bool)
        keep[32:64] = False
        want = np.zeros(q64.shape)
        for t in range(nq):
            i = 200 - nq + t
            see = keep[:i + 1].nonzero()[0]
            want[t] = orc.attend(q64[t:t + 1], k[see], v[see], len(see))[0][0]
        tol = TOL[dtype]
        assert np.all(np.abs(out.float().cpu().numpy() - want) <= tol + tol * np.abs(want))
    finally:
        c2kv.c2kv_destroy(ctx)


def test_same_result_twice():
    """Splits joined in whatever order give the same bits."""
    rng = np.random.default_rng(8)
    c2kv, ctx = P.lib(), P.context("bf16", 32, 8, 128)
    try:
        pg = P.Paged(rng, "bf16", "e4m3", 8, 128, 64, [6000, 30])
        pg.fill_rows(rng)
        q = torch.randn((2, 32, 128), device="cuda", dtype=torch.bfloat16)
        first = None
        for _ in range(20):
            out = torch.empty_like(q)
            c2kv.c2kv_paged_attend(ctx, pg.pages(), pg.table, [0, 1, 2], [6000, 30], q, out)
            c2kv.c2kv_sync(ctx)
            first = out if first is None else first
            assert torch.equal(out, first)
    finally:
        c2kv.c2kv_destroy(ctx)


@pytest.mark.parametrize("shape", [SHAPES[0], SHAPES[1], SHAPES[9]], ids=lambda s: "-".join(map(str, s)))
def test_window_that_leaves_nothing_out(shape):
    """Any window from the longest request's rows on, to the largest number, is none."""
    lens = [(1, 300), (40, 333), (150, 150), (3, 0)]
    none = _run(*shape, 32, lens)
    for window in (333, 2 ** 31 - 1):
        got = _run(*shape, 32, lens, window=window)
        assert np.array_equal(got[0], none[0]) and np.array_equal(got[1], none[1])


@pytest.mark.parametrize("shape", [SHAPES[0], SHAPES[1]], ids=lambda s: "-".join(map(str, s)))
def test_chunk_over_no_rows_after_other_calls(shape):
    """A chunk whose request has no row: zeros, in its place among the stream's other work."""
    dtype, fmt, hq, hkv, d = shape
    rng = np.random.default_rng(5)
    c2kv, ctx = P.lib(), P.context(dtype, hq, hkv, d)
    try:
        pg = P.Paged(rng, dtype, fmt, hkv, d, 16, [400])
        pg.fill_rows(rng)
        q = torch.randn((200, hq, d), device="cuda", dtype=torch.bfloat16)
        out, lse = torch.empty_like(q), torch.empty((hq, 200), device="cuda")
        for keys in (400, 0, 400, 0):
            c2kv.c2kv_paged_attend(ctx, pg.pages(), pg.table, [0, 200], [keys], q, out, lse=lse)
        c2kv.c2kv_sync(ctx)
        assert not out.any() and torch.isneginf(lse).all()
    finally:
        c2kv.c2kv_destroy(ctx)


FEW_F32 = [("f32", "native", 16, 4, 64), ("f32", "e4m3", 8, 8, 64), ("f32", "native", 4, 4, 128), ("f32", "e4m3", 16, 4, 128),
           ("f32", "native", 6, 2, 128)]


@pytest.mark.parametrize("window", [0, 1, 270, 400])
@pytest.mark.parametrize("lens", [[(1, 300)], [(1, 1200), (0, 400), (1, 0), (1, 1), (2, 40), (3, 257), (1, 32), (1, 999)], [(4, 5003), (1, 700)],
                                  [(1, 260 + 9 * i) for i in range(70)]], ids=["one", "ragged", "long", "many"])
@pytest.mark.parametrize("shape", FEW_F32, ids=lambda s: "-".join(map(str, s)))
def test_few_rows_of_fp32(shape, lens, window):
    """Tokens over more keys than the register-tiled loop is for, next to short and empty requests."""
    _check(_run(*shape, 16, lens, window=window), shape[0])


@pytest.mark.parametrize("shape", FEW_F32, ids=lambda s: "-".join(map(str, s)))
def test_few_rows_of_fp32_beside_values_that_are_not_finite(shape):
    """The last two of 700 rows: the first two of four queries see neither, the last sees both."""
    def edit(pg):
        for key, bad in ((699, float("nan")), (698, float("inf"))):
            page, at = int(pg.table_np[0, key // 32]), key % 32
            if pg.ks is None:
                pg.k[page, :, at, 3] = bad
                pg.v[page, :, at, 5] = bad
            else:
                pg.ks[page, :, at] = float("nan")
                pg.vs[page, :, at] = float("nan")
    out, lse, want, want_l = _run(*shape, 32, [(4, 700)], edit=edit)
    assert np.isfinite(out[:2]).all() and np.isnan(out[3]).all()
    _check((out[:2], lse[:, :2], want[:2], want_l[:, :2]), shape[0])
