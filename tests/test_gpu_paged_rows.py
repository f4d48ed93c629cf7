"""Rows written to pages and read back (c2kv_paged_append, c2kv_paged_gather) against fp64.

Tolerances.  A turned or copied value is one rounding of an fp32 result whose own error is at most
2^-20 of the pair it was turned from: half a unit of the type (2^-8 of the value for bf16, 2^-24 for fp32) and that.
A code is checked as a nearest one: no further from x / s than half the step at its place, with 2^-18 of
x / s for fp32 arithmetic; a scale is within 2^-20 of max|x| / 448."""
import numpy as np
import pytest
import torch

from oracle import paged_oracle as orc
from tests import _paged_helpers as P

pytestmark = pytest.mark.gpu
THETA = 1.0e4


def _rows(rng, dtype, t, hkv, d):
    x = torch.from_numpy(rng.standard_normal((t, hkv, d)).astype(np.float32)).to(P.TDT[dtype]).cuda()
    return x, x.float().cpu().numpy().astype(np.float64)


def _pair(x):
    h = x.shape[-1] // 2
    m = np.hypot(x[..., :h], x[..., h:])
    return np.concatenate([m, m], -1)


def _near(got, want, size, dtype):
    half = 2.0 ** (-8 if dtype == "bf16" else -24)
    assert np.all(np.abs(got - want) <= 1.02 * half * np.maximum(np.abs(want), np.abs(got)) + 2.0 ** -20 * size + 1e-38)


def _check_codes(codes, scale, x, size):
    top = np.abs(x).max(-1)
    assert np.all(np.abs(scale - top / 448) <= 2.0 ** -20 * np.maximum(top, size.max(-1)) / 448 * 4)
    y = x / scale[..., None]
    step = 2.0 ** (np.floor(np.log2(np.maximum(np.abs(codes), 2.0 ** -6))) - 3)
    slack = 2.0 ** -18 * (np.abs(y) + size / scale[..., None])
    assert np.all(np.abs(codes - y) <= 0.5 * step + slack)


CASES = [  # dtype, fmt, hkv, d, page, (start, new) per request
    ("bf16", "e4m3", 8, 128, 64, [(0, 1)]),
    ("bf16", "e4m3", 8, 128, 16, [(15, 2), (0, 0), (3, 129), (64, 1), (0, 16)]),
    ("bf16", "e4m3", 1, 64, 32, [(31, 1), (0, 33), (5, 0)]),
    ("bf16", "native", 4, 128, 128, [(127, 3), (0, 5)]),
    ("bf16", "native", 5, 64, 16, [(1, 31), (200, 1), (0, 0), (16, 16)]),
    ("f32", "e4m3", 3, 128, 16, [(7, 40), (0, 1)]),
    ("f32", "native", 2, 64, 64, [(63, 2), (0, 64), (1, 1)]),
    ("f32", "e4m3", 40, 64, 32, [(0, 3), (9, 1)]),
    ("f32", "native", 70, 128, 16, [(2, 2)]),
    ("bf16", "e4m3", 2, 128, 32, [(i % 40, 1 + i % 3) for i in range(300)]),
]


@pytest.mark.parametrize("turn", [True, False], ids=["turned", "as_is"])
@pytest.mark.parametrize("case", CASES, ids=lambda c: "-".join(map(str, c[:5])))
def test_append_and_gather(case, turn):
    dtype, fmt, hkv, d, size, lens = case
    rng = np.random.default_rng(7)
    c2kv, ctx = P.lib(), P.context(dtype, hkv, hkv, d, THETA)
    try:
        pg = P.Paged(rng, dtype, fmt, hkv, d, size, [s + n for s, n in lens])
        before_k, before_ks = pg.k.clone(), pg.ks.clone() if pg.ks is not None else None
        ptr = np.cumsum([0] + [n for _, n in lens]).tolist()
        start = [s for s, _ in lens]
        T = ptr[-1]
        k, k64 = _rows(rng, dtype, T, hkv, d)
        v, v64 = _rows(rng, dtype, T, hkv, d)
        pos = torch.from_numpy(rng.integers(0, 100000, T).astype(np.int32)).cuda()
        size_k = _pair(k64) if turn else np.zeros_like(k64)
        want_k = orc.turned(k64, pos.cpu().numpy(), THETA) if turn else k64
        c2kv.c2kv_paged_append(ctx, pg.pages(), pg.table, ptr, start, k, v, turn=pos if turn else None)
        c2kv.c2kv_sync(ctx)
        written = np.zeros(pg.k.shape[:3], bool)
        codes = [x.float().cpu().numpy().astype(np.float64) for x in (pg.k, pg.v)]
        scales = [x.cpu().numpy().astype(np.float64) if x is not None else None for x in (pg.ks, pg.vs)]
        for r, (s, n) in enumerate(lens):
            for i in range(n):
                page, off = orc.page_of(pg.table_np, r, s + i, size)
                written[page, :, off] = True
                t = ptr[r] + i
                for w, (x, sz) in enumerate(((want_k[t], size_k[t]), (v64[t], np.zeros_like(v64[t])))):
                    if fmt == "e4m3":
                        _check_codes(codes[w][page, :, off], scales[w][page, :, off], x, sz)
                    else:
                        _near(codes[w][page, :, off], x, sz, dtype)
        # rows of no new token keep their bytes
        keep = ~torch.from_numpy(written).cuda()
        raw = torch.uint8 if fmt == "e4m3" else torch.int16 if dtype == "bf16" else torch.int32
        assert torch.equal(pg.k.view(raw)[keep], before_k.view(raw)[keep])
        if fmt == "e4m3":
            assert torch.equal(pg.ks.view(torch.int32)[keep], before_ks.view(torch.int32)[keep])
        # and back, turned back to before RoPE
        ko, vo = (torch.full((T, hkv, d), 9.0, dtype=P.TDT[dtype], device="cuda") for _ in "kv")
        c2kv.c2kv_paged_gather(ctx, pg.pages(), pg.table, ptr, start, ko, vo, turn=-pos if turn else None)
        c2kv.c2kv_sync(ctx)
        hk, hv = pg.host()
        rows_k = np.concatenate([orc.rows_of(hk, pg.table_np, r, s, s + n, size) for r, (s, n) in enumerate(lens)])
        rows_v = np.concatenate([orc.rows_of(hv, pg.table_np, r, s, s + n, size) for r, (s, n) in enumerate(lens)])
        want = orc.turned(rows_k, -pos.cpu().numpy(), THETA) if turn else rows_k
        _near(ko.float().cpu().numpy(), want, _pair(rows_k) if turn else np.abs(rows_k), dtype)
        _near(vo.float().cpu().numpy(), rows_v, np.abs(rows_v), dtype)
    finally:
        c2kv.c2kv_destroy(ctx)


def test_strided_tokens_and_pages():
    """K and V inside one fused projection, pages inside one allocation that holds two layers."""
    rng = np.random.default_rng(3)
    c2kv, ctx = P.lib(), P.context("bf16", 8, 2, 64, THETA)
    try:
        fused = torch.randn((37, 12, 64), device="cuda", dtype=torch.bfloat16)
        k, v = fused[:, 8:10], fused[:, 10:12]
        pool = torch.zeros((9, 2, 2, 2, 16, 64), device="cuda", dtype=torch.bfloat16)   # page, layer, K/V, head, row
        pages = c2kv.make_pages(pool[:, 1, 0], pool[:, 1, 1])
        table = torch.full((1, 8), -1, dtype=torch.int32, device="cuda")
        order = rng.permutation(9)[:3]
        table[0, :3] = torch.from_numpy(order.astype(np.int32))
        c2kv.c2kv_paged_append(ctx, pages, table[:, :3], [0, 37], [5], k, v)
        out = torch.zeros((37, 12, 64), device="cuda", dtype=torch.bfloat16)
        c2kv.c2kv_paged_gather(ctx, pages, table, [0, 37], [5], out[:, 8:10], out[:, 10:12])
        c2kv.c2kv_sync(ctx)
        assert torch.equal(out[:, 8:], fused[:, 8:]) and not out[:, :8].any()
        assert not pool[:, 0].any()
        got = torch.cat([pool[p, 1, 0] for p in order], 1)
        assert torch.equal(got[:, 5:42].transpose(0, 1), k) and not got[:, :5].any() and not got[:, 42:].any()
    finally:
        c2kv.c2kv_destroy(ctx)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_rows_that_codes_cannot_hold(dtype):
    """Zero rows, rows too small for a scale, infinities and NaN: per KV head, K and V each."""
    rng = np.random.default_rng(5)
    c2kv, ctx = P.lib(), P.context(dtype, 4, 4, 128, THETA)
    try:
        pg = P.Paged(rng, dtype, "e4m3", 4, 128, 16, [5])
        x = torch.randn((5, 4, 128), device="cuda").to(P.TDT[dtype])
        x[0, 0] = 0
        x[1, 1] = 1e-37
        x[2, 2, 7] = float("inf")
        x[3, 3, 127] = float("nan")
        x[4, 0] *= 1e30
        v = x.flip(1).contiguous()
        c2kv.c2kv_paged_append(ctx, pg.pages(), pg.table, [0, 5], [0], x, v)
        ko, vo = torch.empty_like(x), torch.empty_like(x)
        c2kv.c2kv_paged_gather(ctx, pg.pages(), pg.table, [0, 5], [0], ko, vo)
        c2kv.c2kv_sync(ctx)
        held = [torch.from_numpy(y[pg.table_np[0, 0], :, :5]).cuda().transpose(0, 1) for y in pg.host()]   # before the read-back's rounding
        for got, src, val in ((ko, x, held[0]), (vo, v, held[1])):
            top = src.float().abs().amax(-1)
            lost = ~torch.isfinite(top)
            assert lost.sum() == 2 and got[lost].isnan().all()
            small = top < 2.0 ** -100
            assert small.sum() == 2 and not got[small].any()
            fine = ~lost & ~small
            err = (val - src.double()).abs()[fine].amax(-1) / top[fine]
            assert (err <= 16.0 / 448 * 1.01).all()          # half the largest step
    finally:
        c2kv.c2kv_destroy(ctx)


def test_refused_pages():
    rng = np.random.default_rng(6)
    c2kv, ctx = P.lib(), P.context("bf16", 2, 2, 64, THETA)
    try:
        pg = P.Paged(rng, "bf16", "native", 2, 64, 16, [48], fill=0.0)
        x = torch.randn((48, 2, 64), device="cuda", dtype=torch.bfloat16)
        for bad in (-1, pg.k.shape[0], 2 ** 31 - 1):
            table = pg.table.clone()
            table[0, 1] = bad
            pg.k.zero_()
            c2kv.c2kv_paged_append(ctx, pg.pages(), table, [0, 48], [0], x, x)
            with pytest.raises(c2kv.C2KVError) as ei:
                c2kv.c2kv_sync(ctx)
            assert ei.value.status == c2kv.ERR_DEVICE_BOUNDS
            assert not pg.k[int(pg.table_np[0, 1])].any()
            out = torch.full_like(x, 3.0)
            c2kv.c2kv_paged_gather(ctx, pg.pages(), table, [0, 48], [0], out, out.clone())
            with pytest.raises(c2kv.C2KVError):
                c2kv.c2kv_sync(ctx)
            assert torch.equal(out[:16], x[:16]) and not out[16:32].any() and torch.equal(out[32:], x[32:])
        c2kv.c2kv_sync(ctx)
    finally:
        c2kv.c2kv_destroy(ctx)


def test_offsets_past_32_bits():
    """A page more than 2^32 elements into its allocation."""
    c2kv, ctx = P.lib(), P.context("bf16", 2, 2, 64, THETA)
    try:
        stride = 2 ** 30 + 64                                   # elements from page to page
        pool = torch.empty(5 * stride, device="cuda", dtype=torch.bfloat16)
        k = torch.as_strided(pool, (5, 2, 16, 64), (stride, 1024, 64, 1))
        v = torch.as_strided(pool, (5, 2, 16, 64), (stride, 1024, 64, 1), 2048)
        pages = c2kv.make_pages(k, v)
        x = torch.randn((20, 2, 64), device="cuda", dtype=torch.bfloat16)
        table = torch.tensor([[4, 2]], dtype=torch.int32, device="cuda")
        c2kv.c2kv_paged_append(ctx, pages, table, [0, 20], [0], x, x.neg())
        ko, vo = torch.empty_like(x), torch.empty_like(x)
        c2kv.c2kv_paged_gather(ctx, pages, table, [0, 20], [0], ko, vo)
        out = torch.empty((1, 2, 64), device="cuda", dtype=torch.bfloat16)
        c2kv.c2kv_paged_attend(ctx, pages, table, [0, 1], [20], x[19:], out)
        c2kv.c2kv_sync(ctx)
        assert torch.equal(ko, x) and torch.equal(vo, x.neg())
        assert torch.equal(k[4], x[:16].transpose(0, 1))
        x64 = x.double().cpu().numpy()
        want, _ = orc.attend(x64[19:], x64, -x64, 20)
        assert np.abs(out.double().cpu().numpy() - want).max() <= 2e-2 * (1 + np.abs(want).max())
    finally:
        c2kv.c2kv_destroy(ctx)


def test_a_stream_of_ones_own():
    """Work goes to the context's stream, in order, whatever torch's current one is."""
    c2kv = P.lib()
    side = torch.cuda.Stream()
    ctx = P.context("bf16", 2, 2, 64, THETA, stream=side)
    try:
        pg = P.Paged(np.random.default_rng(1), "bf16", "native", 2, 64, 16, [64])
        x = torch.randn((64, 2, 64), device="cuda", dtype=torch.bfloat16)
        k = torch.zeros_like(x)
        ko, vo = torch.empty_like(x), torch.empty_like(x)
        torch.cuda.synchronize()
        with torch.cuda.stream(side):
            torch.cuda._sleep(50_000_000)
            k.copy_(x)
        c2kv.c2kv_paged_append(ctx, pg.pages(), pg.table, [0, 64], [0], k, k)
        c2kv.c2kv_paged_gather(ctx, pg.pages(), pg.table, [0, 64], [0], ko, vo)
        c2kv.c2kv_sync(ctx)
        assert torch.equal(ko, x) and torch.equal(vo, x)
    finally:
        c2kv.c2kv_destroy(ctx)


def test_turned_codes_are_those_of_fp32_angles():
    """A code differs from the nearest one only where the turned value is within fp32's error of the middle
    between two: the angle's argument is rounded to fp32 (pi 2^-24), its sine and cosine to 2 units, and the
    two products and their sum once each, together below 2^-21 of the pair; the scale's inverse and its
    product below 2^-22 of the value."""
    rng = np.random.default_rng(12)
    c2kv, ctx = P.lib(), P.context("bf16", 8, 8, 128, THETA)
    try:
        n = 1000
        pg = P.Paged(rng, "bf16", "e4m3", 8, 128, 64, [n])
        k, k64 = _rows(rng, "bf16", n, 8, 128)
        pos = rng.integers(0, 100000, n).astype(np.int32)
        c2kv.c2kv_paged_append(ctx, pg.pages(), pg.table, [0, n], [0], k, k, turn=torch.from_numpy(pos).cuda())
        c2kv.c2kv_sync(ctx)
        x = orc.turned(k64, pos, THETA)
        codes = orc.rows_of(pg.k.float().cpu().numpy().astype(np.float64), pg.table_np, 0, 0, n, 64)
        scale = np.stack([pg.ks.cpu().numpy().astype(np.float64)[pg.table_np[0, j // 64], :, j % 64] for j in range(n)])[..., None]
        y = x / scale
        step = 2.0 ** (np.floor(np.log2(np.maximum(np.abs(codes), 2.0 ** -6))) - 3)
        assert np.all(np.abs(codes - y) <= 0.5 * step + 2.0 ** -21 * _pair(k64) / scale + 2.0 ** -22 * np.abs(y))
    finally:
        c2kv.c2kv_destroy(ctx)
