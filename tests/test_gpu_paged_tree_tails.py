"""Attention of trees where most of an output comes from many keys of small weight, where scales are far apart at random, and
at the ends of the queries' range: the cases of the attention of tokens that follow one another, with trees.

Tolerance: 5e-3 of a row's norm, as there.  Tails: the output's rounding to bf16 is off by 2^-8 / sqrt(3) of the norm in the mean of
squares, 2.3e-3.  Weights, scales and values of 11 bits are off by 2^-11 each, and two of a heavy key's score of 11 by 1.1e-2 of its
weight: at most a fourth of that of an output whose values are one apart, 2.7e-3.  Weights of 8 bits (few rows over 16-bit
pages; a tail 2^-29 of a heavy key and a large value beside it) are all equal ones, with the same error: 2^-8 of the tail's share of
at most 3 / 4, 2.9e-3.  In squares 3.7e-3."""
import numpy as np
import pytest
import torch

from tests import _dense_pages as D
from tests import _paged_helpers as P
from tests._tree_helpers import chain, random_tree, star

pytestmark = pytest.mark.gpu
TOL = 5e-3


@pytest.mark.parametrize("big", [5, 5000])
@pytest.mark.parametrize("apart", [0, 6, 10, 13])
@pytest.mark.parametrize("fmt,hq,hkv,d,batch,n,keys,tail", [
    ("e4m3", 16, 4, 128, 38, 16, 32768, 14), ("native", 16, 4, 128, 38, 16, 32768, 14), ("e4m3", 32, 8, 64, 19, 40, 16384, 13),
    ("e4m3", 4, 4, 128, 38, 100, 131072, 16), ("e4m3", 4, 4, 128, 38, 100, 131072, 17), ("e4m3", 32, 8, 128, 1, 40, 131072, 16),
    ("e4m3", 32, 8, 128, 8, 2, 16384, 13),
    ("native", 8, 2, 64, 1, 64, 131072, 16), ("e4m3", 32, 8, 128, 1, 200, 16384, 13)])
def test_tails(fmt, hq, hkv, d, batch, n, keys, tail, apart, big):
    """One key of weight 2^0.5, one row of V 2^apart times the others at a weight of 2^-40, the rest equal at 1.28 2^-tail, which
    few bits do not have: together as much as the first and more.  Every request has the same pages; of many, none is cut into stretches."""
    gen = torch.Generator(device="cuda").manual_seed(tail)
    per = 16.0 / d ** 0.5 / np.log(2.0)                  # scores in log2: q = 16 in channel 0, nothing else
    k = torch.zeros((keys, hkv, d), device="cuda", dtype=torch.float64)
    v = 1 + 0.25 * torch.randn(k.shape, generator=gen, device="cuda", dtype=torch.float64)
    k[:, :, 0] = np.log2(1.28125) / per
    k[0, :, 0] = (tail + 0.5) / per
    k[big, :, 0] = (tail - 40) / per
    v[0] = 1 + torch.randn((hkv, d), generator=gen, device="cuda", dtype=torch.float64)
    v[big] *= 2.0 ** apart
    rows = D.Rows("bf16", fmt, [k], [v], 128)
    rows.table = rows.table.repeat(batch, 1)
    rows.k, rows.v = rows.k * batch, rows.v * batch
    q = torch.zeros((batch * n, hq, d), device="cuda", dtype=torch.bfloat16)
    q[..., 0] = 16
    call = D.Call("bf16", hq, hkv, d, rows, [star(n)] * batch, q)
    want, _ = D.attend_tree(q[:n].double(), rows.k[0], rows.v[0], star(n))
    assert max(D.relative(call.out[n * r:n * r + n], want) for r in range(batch)) <= TOL


@pytest.mark.parametrize("n,x", [(2, 300), (40, 300), (100, 1500), (40, 9000), (200, 500)])
@pytest.mark.parametrize("hq,hkv,d", [(32, 8, 128), (28, 4, 64)])
def test_scales_far_apart(hq, hkv, d, n, x):
    """Rows whose scales span many powers of two, zero among them, in K and V."""
    rng, gen = np.random.default_rng(9), torch.Generator(device="cuda").manual_seed(9)
    k, v = (torch.randn((x + n, hkv, d), generator=gen, device="cuda", dtype=torch.float64) for _ in range(2))
    for rows, most in ((k, 4), (v, 1)):
        f = 2.0 ** rng.integers(-30, most, (x + n, hkv))
        f[rng.random(f.shape) < 0.1] = 0
        rows *= torch.from_numpy(f).cuda()[..., None]
    q = (0.2 * torch.randn((n, hq, d), generator=gen, device="cuda")).bfloat16()
    call = D.Call("bf16", hq, hkv, d, D.Rows("bf16", "e4m3", [k], [v], 16), [random_tree(rng, n, near=9)], q)
    want, _ = call.want()
    assert D.relative(call.out, want) <= TOL


@pytest.mark.parametrize("q_size,k_size", [(2.0 ** -40, 0.0), (2.0 ** -90, 0.0), (2.0 ** 100, 0.0), (2.0 ** -60, 2.0 ** -60), (2.0 ** 100, 2.0 ** 60)])
@pytest.mark.parametrize("n,x", [(12, 300), (140, 300), (64, 6000), (300, 900)])
@pytest.mark.parametrize("fmt,d", [("e4m3", 128), ("native", 128), ("e4m3", 64), ("native", 64)])
def test_scores_of_zero(fmt, d, n, x, q_size, k_size):
    """Queries far smaller or larger than one over keys of zero, or that they do not meet: a row is the mean of what it sees."""
    hq, hkv = 16, 4
    gen = torch.Generator(device="cuda").manual_seed(2)
    k = torch.zeros((x + n, hkv, d), device="cuda", dtype=torch.float64)
    k[..., 1] = k_size
    v = torch.randn(k.shape, generator=gen, device="cuda", dtype=torch.float64)
    q = torch.zeros((n, hq, d), device="cuda", dtype=torch.bfloat16)
    q[..., 0] = q_size
    call = D.Call("bf16", hq, hkv, d, D.Rows("bf16", fmt, [k], [v], 64), [chain(n)], q)
    seen = torch.arange(x + 1, x + n + 1, device="cuda")
    want = (call.rows.v[0].cumsum(0)[x:] / seen[:, None, None]).repeat_interleave(hq // hkv, 1)
    assert D.relative(call.out, want) <= TOL
    assert (call.lse - seen.log()).abs().max().item() <= 1e-4
