"""Attention of trees where values of V, and the scales of 8-bit rows, lie far apart or at the ends of their types.

A score is n / 4 q_0 / sqrt(d), exact in every operand: the keys' channel 0 is n / 4, their channel 1 (which no query
has) makes the scale of 8-bit rows 1 / 4 or 1365 / 4096, eleven bits.  Values have a mean, so that outputs are as large as they are.

Tolerance: 5e-3 of a row's norm.  The output's rounding to bf16 is off by at most 2^-8 of a value, evenly either way: 2^-8 / sqrt(3) of the
norm in the mean of squares, 2.3e-3.  Weights, scales and values of 11 bits are off by 2^-11 each, all together 1.5e-3 if they are
all alike; over 16-bit pages weights of 8 bits, where they are all equal ones, by 2^-8 of the output, values of one sign: 3.9e-3, which
adds in squares to its rounding.  4.5e-3."""
import numpy as np
import pytest
import torch

from tests import _dense_pages as D
from tests import _paged_helpers as P
from tests._tree_helpers import star

pytestmark = pytest.mark.gpu
TOL = 5e-3

# (nodes, rows before): rows by eights, few rows over many, straight from the pages (few and many key tiles), key tiles
WAYS = {"eights": (12, 700), "few": (4, 14000), "direct": (100, 1500), "direct_long": (40, 9000), "large": (200, 1500)}
KINDS = [("e4m3", 128), ("native", 128), ("e4m3", 64)]


def _error(kind, way, steps, size, own=None, hidden=None):
    """Relative error of the worst row.  steps [rows]: n of a row's score; size [rows]: of its values.  own: the nodes'
    values times this, and scales of K of eleven bits; hidden: the last node's K and V times these."""
    fmt, d = kind
    n, x = WAYS[way]
    hq, hkv = 32, 8
    gen = torch.Generator(device="cuda").manual_seed(3)
    rows = x + n
    k = torch.zeros((rows, hkv, d), device="cuda", dtype=torch.float64)
    k[..., 0] = torch.as_tensor(steps, device="cuda", dtype=torch.float64)[:, None] / 4
    k[..., 1] = 112.0
    v = (1 + 0.25 * torch.randn((rows, hkv, d), generator=gen, device="cuda", dtype=torch.float64)).clamp(0.25, 2)
    if own is not None:
        v[x:] *= own
        k[x:, :, 1] *= 1365 / 1024
    v *= torch.as_tensor(size, device="cuda", dtype=torch.float64)[:, None, None]
    if hidden is not None:
        k[-1] *= hidden[0]
        v[-1] *= hidden[1]
    q = torch.zeros((n, hq, d), device="cuda", dtype=torch.bfloat16)
    q[..., 0] = 64.0
    call = D.Call("bf16", hq, hkv, d, D.Rows("bf16", fmt, [k], [v], 32), [star(n)], q)
    last = n - 1 if hidden is not None else n
    want, out = call.want()[0][:last], call.out[:last]
    assert torch.isfinite(out).all()
    if own is None or own > 0:
        return D.relative(out, want)
    # (values of both signs cancel, what their terms are off by does not)
    terms, _ = D.attend_tree(call.q.double(), call.rows.k[0], call.rows.v[0].abs(), star(n))
    return ((out.double() - want).norm(dim=-1) / terms[:last].norm(dim=-1)).max().item()


def _rows(way):
    return sum(WAYS[way])


@pytest.mark.parametrize("up", [0, 6])
@pytest.mark.parametrize("size", [1.0, 0.01, 1e-4, 2.0 ** 100])
@pytest.mark.parametrize("way", WAYS)
@pytest.mark.parametrize("kind", KINDS, ids=lambda s: "-".join(map(str, s)))
def test_rows_of_zeros(kind, way, size, up):
    """A run of rows whose values are all zero, from 32 on and from 192 on, scored as the others or above them by up to 8.5 (12
    with 64 channels): the others' values are what the outputs are made of."""
    steps, sizes = np.zeros(_rows(way)), np.full(_rows(way), size)
    for lo, hi in ((32, 64), (192, 320)):
        steps[lo:hi], sizes[lo:hi] = up, 0.0
    assert _error(kind, way, steps, sizes) <= TOL


@pytest.mark.parametrize("way", WAYS)
@pytest.mark.parametrize("kind", KINDS, ids=lambda s: "-".join(map(str, s)))
def test_rows_of_zeros_first_and_alone(kind, way):
    """All rows zeros but the last 40 before the tree and the tree: sums begin without any value."""
    n, x = WAYS[way]
    sizes = np.where(np.arange(n + x) < x - 40, 0.0, 2.0 ** 20)
    assert _error(kind, way, np.zeros(n + x), sizes) <= TOL


@pytest.mark.parametrize("order", ["up", "down", "mixed"])
@pytest.mark.parametrize("way", WAYS)
@pytest.mark.parametrize("kind", KINDS, ids=lambda s: "-".join(map(str, s)))
def test_values_far_apart_that_count_alike(kind, way, order):
    """Groups of 32 rows whose scores rise as their values fall, by up to 2^20: each is as much of the output."""
    rows, most = _rows(way), 10 if kind[1] == 128 else 7
    of = np.arange(rows) // 32
    steps = {"up": of * most // of[-1], "down": most - of * most // of[-1], "mixed": np.random.default_rng(1).integers(0, most + 1, of[-1] + 1)[of]}[order]
    assert _error(kind, way, steps, 2.0 ** -np.round(steps * 64 / 4 / np.sqrt(kind[1]) / np.log(2))) <= TOL


@pytest.mark.parametrize("far", [0, 12, 20, 24])
@pytest.mark.parametrize("way", WAYS)
@pytest.mark.parametrize("kind", KINDS, ids=lambda s: "-".join(map(str, s)))
def test_values_of_a_sibling(kind, way, far):
    """A node's own values are half of its output and more; a sibling next to it that it does not see holds values 2^far
    times as large."""
    n, x = WAYS[way]
    steps = np.where(np.arange(n + x) < x, 0, 6)
    assert _error(kind, way, steps, np.ones(n + x), own=8.0, hidden=(1.0, 2.0 ** far)) <= TOL


@pytest.mark.parametrize("far", [0, 12, 16])
@pytest.mark.parametrize("way", WAYS)
@pytest.mark.parametrize("kind", KINDS, ids=lambda s: "-".join(map(str, s)))
def test_keys_of_a_sibling(kind, way, far):
    """The same of K: a node's own score decides how its value and those before the tree, of the other sign, are mixed.

    Errors are relative to the sum of the terms' magnitudes w_j |v_j|, of which each is off as elsewhere.  The nodes' scores have
    15 bits, 2^-11 of eight where eleven are kept: e = 3.9e-3.  Rows of weight p that are 4 beside ones of 1 of the other sign move
    an output by e p (1 - p) 5, at most 0.56 e of 4 p + 1 - p: 2.2e-3, beside 0.5e-3 of weights and 2.3e-3 of the output's rounding,
    in squares 3.6e-3.  Over 16-bit pages scores are exact, and weights 2^-8: 4.5e-3."""
    n, x = WAYS[way]
    steps = np.where(np.arange(n + x) < x, 0, 5 if kind[1] == 128 else 4)
    assert _error(kind, way, steps, np.ones(n + x), own=-4.0, hidden=(2.0 ** far, 1.0)) <= TOL


@pytest.mark.parametrize("way", ["eights", "few", "direct", "direct_long"])
@pytest.mark.parametrize("kind", KINDS, ids=lambda s: "-".join(map(str, s)))
def test_keys_of_a_sibling_further(kind, way):
    n, x = WAYS[way]
    steps = np.where(np.arange(n + x) < x, 0, 5 if kind[1] == 128 else 4)
    assert _error(kind, way, steps, np.ones(n + x), own=-4.0, hidden=(2.0 ** 24, 1.0)) <= TOL


@pytest.mark.parametrize("size", [2.0 ** 114, 2.0 ** 117])
@pytest.mark.parametrize("way", ["eights", "direct"])
def test_values_near_the_largest(way, size):
    """16-bit pages: outputs are numbers where their values are."""
    steps = np.where(np.arange(_rows(way)) % 500 == 499, 6, 0)       # (scores that rise late, too)
    assert _error(("native", 128), way, steps, np.full(_rows(way), size)) <= TOL
@pytest.mark.parametrize("size", [2.0 ** -98, 2.0 ** -80, 2.0 ** 80, 2.0 ** 111])
@pytest.mark.parametrize("way", WAYS)
@pytest.mark.parametrize("kind", KINDS, ids=lambda s: "-".join(map(str, s)))
def test_all_values_small_or_large(kind, way, size):
    """Values near the smallest that 8-bit rows keep, and large ones that thousands of rows add up to 2^126 of."""
    assert _error(kind, way, np.arange(_rows(way)) % 3, np.full(_rows(way), size)) <= TOL


@pytest.mark.parametrize("way,far", [(w, f) for w in ("eights", "few", "direct", "direct_long") for f in (12, 20, 24)] + [("large", 12)])
@pytest.mark.parametrize("kind", KINDS, ids=lambda s: "-".join(map(str, s)))
def test_small_values_that_count_alone(kind, way, far):
    """The tree's rows outweigh those before it by e^31 (e^44 with 64 channels), whose values, in the same 32 rows as some of the
    tree's, are 2^far times theirs."""
    n, x = WAYS[way]
    assert _error(kind, way, np.where(np.arange(n + x) < x, 0, 22), np.ones(n + x), own=2.0 ** -far) <= TOL
