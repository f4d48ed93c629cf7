"""Errors of attention of trees relative to a row's norm: outputs over thousands of rows are too small for an absolute
tolerance (one of 2e-2 does not notice a key tile that is left out).

Tolerances.  A rounding to bf16 is off by at most 2^-8 of a value, evenly either way: over a row's channels by 2^-8 / sqrt(3) of its
norm at most in the mean of squares, 2.3e-3.  The output has one, weights of 8 bits (few rows over 16-bit pages) another, and eleven
bits of queries, weights, codes times scales an eighth of one each: 3.3e-3 together.  A row's mean of squares over 64 channels
lies within a half of that: 5e-3 leaves room for it.  lse: an operand's eleven bits move a score by 2^-11 / sqrt(3) of
(sum q^2 k^2 / d)^(1/2), one for normal rows, two of them by 4e-4: five times that is 2e-3.  fp32: 1e-5, lse 2e-5 of its magnitude and one,
as the library's other fp32 attentions."""
import numpy as np
import pytest
import torch

from oracle import branch_oracle as brc
from tests import _dense_pages as D
from tests import _paged_helpers as P
from tests._tree_helpers import chain, random_tree, star

gpu = pytest.mark.gpu
TOL = {"bf16": 5e-3, "f32": 1e-5}
TOL_LSE = {"bf16": 2e-3, "f32": 2e-5}

SHAPES = [("bf16", "e4m3", 32, 8, 128), ("bf16", "native", 32, 8, 128), ("bf16", "e4m3", 28, 4, 64), ("bf16", "native", 8, 2, 64),
          ("f32", "native", 16, 4, 64), ("f32", "e4m3", 8, 2, 128)]
# (nodes, rows before) a request: each way that a call may go, of one and several row tiles, odd and even numbers of key
# tiles, stretches cut and whole
LENS = {
    "few": [(2, 9001), (3, 5000), (1, 777)], "short": [(16, 1500), (9, 300)], "tile": [(20, 9001)], "deep": [(120, 4000)],
    "tiles": [(60, 5000), (100, 2500), (33, 95)], "whole": [(20 + i % 9, 400 + 37 * i) for i in range(40)], "large": [(200, 2500), (300, 700)],
}


@gpu
@pytest.mark.parametrize("window", [0, 700])
@pytest.mark.parametrize("lens", LENS, ids=str)
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "-".join(map(str, s)))
def test_relative_errors(shape, lens, window):
    dtype, fmt, hq, hkv, d = shape
    r, gen = np.random.default_rng(5), torch.Generator(device="cuda").manual_seed(5)
    trees = [chain(n) if lens == "deep" else random_tree(r, n, near=12) for n, _ in LENS[lens]]
    k, v = ([torch.randn((n + x, hkv, d), generator=gen, device="cuda") for n, x in LENS[lens]] for _ in range(2))
    T = sum(n for n, _ in LENS[lens])
    q = torch.randn((T, hq, d), generator=gen, device="cuda").to(P.TDT[dtype])
    pos = torch.from_numpy(r.integers(0, 100000, T).astype(np.int32)).cuda()
    call = D.Call(dtype, hq, hkv, d, D.Rows(dtype, fmt, k, v, 64), trees, q, pos, window=window, times=3)
    assert torch.equal(call.outs[0], call.outs[1]) and torch.equal(call.outs[0], call.outs[2])
    want, want_l = call.want()
    assert D.relative(call.out, want) <= TOL[dtype]
    assert ((call.lse - want_l).abs() <= TOL_LSE[dtype] * (1 + (want_l.abs() if dtype == "f32" else 0))).all()


@gpu
@pytest.mark.parametrize("lens", ["tile", "deep", "tiles", "whole"])
@pytest.mark.parametrize("shape", [SHAPES[1], ("bf16", "native", 32, 8, 64)], ids=lambda s: "-".join(map(str, s)))
def test_operands_of_16_bits(shape, lens):
    """Trees straight from 16-bit pages: queries and weights have two terms, so an output's own rounding is nearly all of its
    error.  Second terms are off by 2^-8 of what the first, cut off or rounded, lack: 2^-15 of a weight, 2^-16 of a query's
    value and so of its scores' sum |q k| / sqrt(d), at most 16 for normal ones.  That is 2^-12 of the output at most, which adds
    in squares to 1.5e-3 and more of its rounding: 1.3 %."""
    dtype, fmt, hq, hkv, d = shape
    r, gen = np.random.default_rng(6), torch.Generator(device="cuda").manual_seed(6)
    trees = [random_tree(r, n) for n, _ in LENS[lens]]
    k, v = ([torch.randn((n + x, hkv, d), generator=gen, device="cuda") for n, x in LENS[lens]] for _ in range(2))
    T = sum(n for n, _ in LENS[lens])
    q = torch.randn((T, hq, d), generator=gen, device="cuda").to(P.TDT[dtype])
    call = D.Call(dtype, hq, hkv, d, D.Rows(dtype, fmt, k, v, 64), trees, q)
    want, _ = call.want()
    assert (call.out.double() - want).norm() <= 1.02 * (want.bfloat16().double() - want).norm()


@gpu
@pytest.mark.parametrize("lens", ["tile", "tiles", "large"])
@pytest.mark.parametrize("d", [128, 64])
def test_codes_times_scales_are_rounded_once(d, lens):
    """8-bit pages with channels of K eight times the others': outputs are off by what rounding K and V to eleven bits once makes
    of them, and by their own rounding, in squares.  A quarter more than the first is left for the weights' eleven bits,
    2^-11 / sqrt(3) of the output at most where K and V make twice that and more."""
    r, gen = np.random.default_rng(6), torch.Generator(device="cuda").manual_seed(6)
    trees = [random_tree(r, n) for n, _ in LENS[lens]]
    k, v = ([torch.randn((n + x, 8, d), generator=gen, device="cuda") for n, x in LENS[lens]] for _ in range(2))
    for x in k:
        x[..., [5, d // 2 + 9]] *= 8
    q = torch.randn((sum(n for n, _ in LENS[lens]), 32, d), generator=gen, device="cuda").bfloat16()
    rows = D.Rows("bf16", "e4m3", k, v, 64)
    call = D.Call("bf16", 32, 8, d, rows, trees, q)
    want, _ = call.want()
    rows.k, rows.v = ([x.half().double() for x in held] for held in (rows.k, rows.v))
    once = (call.want()[0] - want).norm().item()
    own = (want.bfloat16().double() - want).norm().item()
    assert (call.out.double() - want).norm().item() <= (own ** 2 + (1.25 * once) ** 2) ** 0.5


@pytest.mark.parametrize("tree,x", [(star(20), 9001), (chain(60), 5000)], ids=["star", "chain"])
def test_a_lost_tile_would_show(tree, x):
    """The tolerances notice a tile of 128 keys left out of thousands: outputs and sums without it are off by more, in most
    rows."""
    rng, n = np.random.default_rng(0), len(tree)
    q, k, v = (rng.standard_normal((m, 1, 128)) for m in (n, x + n, x + n))
    want, want_l = brc.attend_tree(q, k, v, tree)
    for lo in (0, 128 * 21, (x - 128) // 128 * 128):
        there = np.ones(x + n, bool)
        there[lo:lo + 128] = False
        out, lse = brc.attend_tree(q, k, v, tree, there=there)
        assert np.median(np.linalg.norm(out - want, axis=-1) / np.linalg.norm(want, axis=-1)) > 4 * TOL["bf16"]
        assert np.median(np.abs(lse - want_l)) > 4 * TOL_LSE["bf16"]
