"""Paged calls without a GPU: the oracle pinned by hand and by torch, and the refusals that are answered
before any CUDA call (made here through the library over a stand-in for the CUDA runtime)."""
import numpy as np
import torch

from oracle import paged_oracle as orc


def test_e4m3_grid_is_torchs():
    y = np.concatenate([np.linspace(-448, 448, 4001), 2.0 ** np.linspace(-12, 8.8, 3001), -2.0 ** np.linspace(-12, 8.8, 999), [0.0]])
    y = y.astype(np.float32).astype(np.float64)
    want = torch.from_numpy(y).float().to(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(orc.e4m3(y), want)


def test_quantised_rows():
    x = np.array([[1.0, -2.0, 0.5, 0.0], [0, 0, 0, 0], [1e-38, 0, 0, 0], [np.inf, 1, 2, 3], [np.nan, 1, 2, 3]])
    codes, scale = orc.quantised(x)
    assert scale[0] == 2 / 448 and np.array_equal(codes[0], [224, -448, 112, 0])
    assert scale[1] == 0 and scale[2] == 0 and not codes[1:].any()
    assert np.isnan(scale[3]) and np.isnan(scale[4])


def test_attend_by_torch():
    rng = np.random.default_rng(0)
    n, keys, hq, hkv, d = 5, 23, 6, 2, 8
    q, k, v = rng.standard_normal((n, hq, d)), rng.standard_normal((keys, hkv, d)), rng.standard_normal((keys, hkv, d))
    mask = np.tril(np.ones((n, keys)), keys - n).astype(bool)
    for window in (0, 4):
        m = mask & (np.arange(keys) > (np.arange(n)[:, None] + keys - n - window)) if window else mask
        want = torch.nn.functional.scaled_dot_product_attention(
            *(torch.from_numpy(x).transpose(0, 1) for x in (q, k.repeat(3, 1), v.repeat(3, 1))), attn_mask=torch.from_numpy(m))
        out, lse = orc.attend(q, k, v, keys, window)
        assert np.allclose(out, want.transpose(0, 1).numpy(), atol=1e-12)
    out, lse = orc.attend(q, k[:3], v[:3], 3)
    assert not out[:2].any() and np.isneginf(lse[:, :2]).all() and np.isfinite(lse[:, 2:]).all()


def test_verify_by_hand():
    p = np.array([[0.5, 0.25, 0.25, 0.0], [0.0, 1.0, 0.0, 0.0], [0.25, 0.25, 0.25, 0.25]], np.float32)
    q = np.array([[0.25, 0.75, 0.0, 0.0], [0.5, 0.5, 0.0, 0.0]], np.float32)
    run = lambda t, ua, un: orc.verify([0, 2], np.array(t), p, q, np.array(ua, np.float32), np.array([un], np.float32))[0]  # noqa: E731
    assert run([0, 1], [0.9, 0.9], 0.6) == (2, 2)            # both kept; the next from p's last row
    assert run([1, 1], [0.4, 0.0], 0.49) == (0, 0)           # 0.4 * 0.75 >= 0.25: left over q are 0.25, 0, 0.25
    assert run([1, 1], [0.4, 0.0], 0.51) == (0, 2)
    assert run([0, 0], [0.9, 0.0], 0.0) == (1, 1)            # p of the second draft is 0, its product 0: refused


def test_no_context_is_refused():
    import __graft_entry__ as g
    g.build()
    from paper_2607_17715_gb300 import c2kv
    for name in ("c2kv_paged_append", "c2kv_paged_gather", "c2kv_paged_attend", "c2kv_verify_drafts"):
        fn = getattr(c2kv._lib, name)
        assert fn(*[None if t is c2kv._VP else 0 for t in fn.argtypes]) == c2kv.ERR_ARG
