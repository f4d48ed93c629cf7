"""Errors of paged attention relative to a row's norm, where outputs are too small for an absolute tolerance (the mean
of thousands of values) or weights too sharp for a loose one.

Over random keys and values a bf16 output's own rounding is at most 2^-9 of a value, 2.0e-3 of the norm.  Weights
of 8 bits (over 16-bit pages) or 11, queries of 11 bits and 8-bit codes taken exactly add errors of either sign,
2^-9 / sqrt(3) of the norm together at most: 5e-3 leaves room for the sum of both.  A log-sum's error is a
score's: queries rounded to 2^-12 of a value move a score by 2^-12 |q k| / sqrt(d), below 5e-4 for normal ones;
2e-3 is allowed.  fp32: 1e-5, as the library's other fp32 attentions; lse 1e-5 of its magnitude and one."""
import numpy as np
import pytest
import torch

from oracle import paged_oracle as orc
from tests import _paged_helpers as P

gpu = pytest.mark.gpu
TOL = {"bf16": 5e-3, "f32": 1e-5}
TOL_LSE = {"bf16": 2e-3, "f32": 2e-5}

SHAPES = [("bf16", "e4m3", 32, 8, 128), ("bf16", "native", 32, 8, 128), ("bf16", "e4m3", 28, 4, 64), ("bf16", "native", 8, 2, 64),
          ("f32", "native", 16, 4, 64), ("f32", "e4m3", 8, 2, 128)]
# (queries, rows) a request: stretches of few and of many rows, chunks cut and whole, next to one another
LENS = {"tokens": [(1, 9001), (3, 5000), (2, 777)], "chunk": [(70, 9001)], "chunks": [(300, 2500), (140, 1111), (1, 4000)],
        "many": [(1, 2000 + 37 * i) for i in range(40)]}


def _relative(out, want):
    return np.linalg.norm(out - want, axis=-1) / np.linalg.norm(want, axis=-1)


def _run(shape, lens, window, q_scale=1.0, theta=1.0e4):
    """out (twice), lse, the fp64 ones, and for each row the largest change of a score by queries of 11 bits."""
    dtype, fmt, hq, hkv, d = shape
    rng = np.random.default_rng(11)
    c2kv, ctx = P.lib(), P.context(dtype, hq, hkv, d, theta)
    try:
        pg = P.Paged(rng, dtype, fmt, hkv, d, 64, [k for _, k in lens])
        pg.fill_rows(rng)
        ptr = np.cumsum([0] + [n for n, _ in lens]).tolist()
        q = torch.from_numpy((rng.standard_normal((ptr[-1], hq, d)) * q_scale).astype(np.float32)).to(P.TDT[dtype]).cuda()
        pos = torch.from_numpy(rng.integers(0, 100000, ptr[-1]).astype(np.int32)).cuda()
        got = []
        for _ in range(2):
            out, lse = torch.empty_like(q), torch.empty((hq, ptr[-1]), device="cuda")
            c2kv.c2kv_paged_attend(ctx, pg.pages(), pg.table, ptr, [k for _, k in lens], q, out, lse=lse, turn=pos, window=window)
            got.append(out)
        c2kv.c2kv_sync(ctx)
        assert torch.equal(*got)
        q64 = orc.turned(q.double().cpu().numpy(), pos.cpu().numpy(), theta)
        hk, hv = pg.host()
        want, want_l, moved, size = [], [], [], []
        for r, (n, keys) in enumerate(lens):
            k, v = (orc.rows_of(x, pg.table_np, r, 0, keys, 64) for x in (hk, hv))
            x = q64[ptr[r]:ptr[r + 1]]
            o, ls = orc.attend(x, k, v, keys, window)
            want.append(o)
            want_l.append(ls)
            if q_scale > 1:
                g = hq // hkv
                moved.append(2.0 ** -12 / np.sqrt(d) * np.stack([np.sqrt((x[:, h] ** 2) @ (k[:, h // g] ** 2).T).max(-1) for h in range(hq)], 1))
                size.append(np.stack([np.broadcast_to(np.linalg.norm(v[:, h // g], axis=-1).max(), n) for h in range(hq)], 1))
        return (out.double().cpu().numpy(), lse.double().cpu().numpy(), np.concatenate(want), np.concatenate(want_l, 1),
                np.concatenate(moved) if moved else None, np.concatenate(size) if size else None)
    finally:
        c2kv.c2kv_destroy(ctx)


@gpu
@pytest.mark.parametrize("window", [0, 700])
@pytest.mark.parametrize("lens", LENS, ids=str)
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "-".join(map(str, s)))
def test_long_rows(shape, lens, window):
    out, lse, want, want_l, _, _ = _run(shape, LENS[lens], window)
    assert _relative(out, want).max() <= TOL[shape[0]]
    assert np.all(np.abs(lse - want_l) <= TOL_LSE[shape[0]] * (1 + (np.abs(want_l) if shape[0] == "f32" else 0)))


@gpu
@pytest.mark.parametrize("lens", [[(1, 900), (40, 300)], [(140, 900)]], ids=["few", "chunk"])
@pytest.mark.parametrize("shape", SHAPES[:4], ids=lambda s: "-".join(map(str, s)))
def test_sharp_weights(shape, lens):
    """Nearly one-hot weights over values that differ: a score moved by e moves an output by at most 2 e |v|, and
    queries of 11 bits move it by 4 / sqrt(3) < 3 deviations of their rounding at most."""
    out, _, want, _, moved, size = _run(shape, lens, 0, q_scale=30.0)
    bound = TOL["bf16"] * np.linalg.norm(want, axis=-1) + 2 * 3 * moved * size
    assert np.all(np.linalg.norm(out - want, axis=-1) <= bound)


@pytest.mark.parametrize("n,keys", [(1, 9001), (3, 5000), (70, 9001)])
def test_a_lost_block_would_show(n, keys):
    """The tolerance notices 32 keys left out of thousands: outputs without them are off by more, in most rows."""
    rng = np.random.default_rng(0)
    q, k, v = (rng.standard_normal((m, 1, 128)) for m in (n, keys, keys))
    want, want_l = orc.attend(q, k, v, keys)
    for lo in (0, 32 * 70, keys - n - 32):
        keep = np.r_[0:lo, lo + 32:keys]
        out, lse = orc.attend(q, k[keep], v[keep], keys - 32)
        assert np.median(_relative(out, want)) > 4 * TOL["bf16"]
