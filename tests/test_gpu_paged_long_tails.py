"""Paged attention where most of the output comes from many keys of small weight, beside one key of large weight and
one whose value is large but whose weight is negligible.

One key has weight 1, one row of V is 2^apart times the others at a weight of 2^-40, and the rest are equal at
2^-tail, together as much as the first or twice as much.  Tolerance: 5e-3 of a row's norm.  The output's
rounding to bf16 is at most 2^-9 of a value, 2.0e-3 of the norm.  Weights, values and queries of 11 bits add
2^-12 each, 0.7e-3; over 16-bit pages weights have 8 bits, all equal ones the same error, 2^-9 of the tail's
share of at most 2 / 3: 1.3e-3.  The queries' angles do not matter (they are not turned)."""
import numpy as np
import pytest
import torch

from tests import _paged_helpers as P

pytestmark = pytest.mark.gpu


def _case(fmt, hq, hkv, d, batch, nq, keys, tail, apart, big):
    """Relative errors of all rows; every request has the same pages.  `big`: where the large value is."""
    c2kv, ctx = P.lib(), P.context("bf16", hq, hkv, d)
    size, g = 128, torch.Generator(device="cuda").manual_seed(tail)
    try:
        n = keys // size
        k = torch.zeros((n, hkv, size, d), device="cuda")
        v = 1 + 0.25 * torch.randn(k.shape, generator=g, device="cuda")
        # scores in log2: q = 16 in channel 0, nothing else
        per = 16.0 / d ** 0.5 / np.log(2.0)
        k[0, :, 0, 0] = tail / per
        k[big // size, :, big % size, 0] = (tail - 40) / per
        v[0, :, 0] = 1 + torch.randn((hkv, d), generator=g, device="cuda")
        v[big // size, :, big % size] *= 2.0 ** apart
        if fmt == "e4m3":
            held = []
            for x in (k, v):
                s = x.abs().amax(-1) / 448
                held.append(((x / s.clamp(min=1e-30)[..., None]).to(P.E4M3), s))
            (k, ks), (v, vs) = held
            k64, v64 = (x.double() * s.double()[..., None] for x, s in held)
        else:
            k, v, ks, vs = k.bfloat16(), v.bfloat16(), None, None
            k64, v64 = k.double(), v.double()
        q = torch.zeros((batch * nq, hq, d), device="cuda", dtype=torch.bfloat16)
        q[..., 0] = 16
        table = torch.arange(n, device="cuda", dtype=torch.int32).repeat(batch, 1)
        out = torch.empty_like(q)
        c2kv.c2kv_paged_attend(ctx, c2kv.make_pages(k, v, ks, vs), table, [nq * i for i in range(batch + 1)], [keys] * batch, q, out)
        c2kv.c2kv_sync(ctx)
        # all queries are alike: row t sees the first keys - nq + t + 1 keys
        w = torch.exp2(k64[..., 0].transpose(0, 1).reshape(hkv, keys) * per - tail)
        sums = (w[..., None] * v64.transpose(0, 1).reshape(hkv, keys, d)).cumsum(1)[:, keys - nq:] / w.cumsum(1)[:, keys - nq:, None]
        want = sums.transpose(0, 1).repeat_interleave(hq // hkv, 1).repeat(batch, 1, 1)
        return ((out.double() - want).norm(dim=-1) / want.norm(dim=-1)).max().item()
    finally:
        c2kv.c2kv_destroy(ctx)


# units enough that no request's keys are cut: a warp meets the large weight, the large value and the tail
@pytest.mark.parametrize("apart", [0, 6, 10, 13])
@pytest.mark.parametrize("fmt,hq,hkv,d,batch,nq,keys,tail", [
    ("e4m3", 32, 8, 128, 64, 1, 16384, 13), ("e4m3", 8, 8, 64, 64, 3, 32768, 14), ("e4m3", 32, 4, 128, 120, 2, 16384, 13),
    ("native", 32, 8, 128, 64, 1, 16384, 13), ("e4m3", 32, 8, 128, 1, 1, 131072, 16)])
def test_few_rows(fmt, hq, hkv, d, batch, nq, keys, tail, apart):
    assert _case(fmt, hq, hkv, d, batch, nq, keys, tail, apart, 5) <= 5e-3


# chunks: the large weight and the large value in one key tile, or tiles apart, and the tail in all the others
@pytest.mark.parametrize("big", [5, 5000])
@pytest.mark.parametrize("apart", [0, 6, 10, 13])
@pytest.mark.parametrize("fmt,hq,hkv,d,batch,nq,keys,tail", [
    ("e4m3", 32, 8, 128, 1, 1024, 32768, 14), ("native", 32, 8, 128, 1, 1024, 32768, 14), ("e4m3", 8, 8, 64, 4, 200, 16384, 13),
    ("native", 8, 2, 64, 40, 64, 16384, 13), ("e4m3", 32, 8, 128, 1, 64, 131072, 16), ("native", 8, 2, 128, 1, 500, 131072, 16)])
def test_chunks(fmt, hq, hkv, d, batch, nq, keys, tail, apart, big):
    assert _case(fmt, hq, hkv, d, batch, nq, keys, tail, apart, big) <= 5e-3
