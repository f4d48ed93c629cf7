"""Rows of the calls over composed caches whose every seen score is -inf: the softmax of them is not a number,
and neither is the output."""
import pytest
import torch

import synth
from tests import _gpu_helpers as H

pytestmark = pytest.mark.gpu
CUDA_CORES = [("f32", 64, 4, 2), ("f32", 128, 16, 4), ("bf16", 64, 6, 2), ("bf16", 128, 6, 2)]


def _opposed(dtype, *shape):
    """Zeros but for a channel that barely turns, whose product with its like is beyond fp32: -1e30 by 1e30."""
    x = torch.zeros(shape, device="cuda", dtype=dtype)
    x[..., shape[-1] // 2 - 1] = 1e30
    return x


@pytest.mark.parametrize("layers,slots,n", [(1, 200, 90), (24, 100, 200), (1, 300, 1)])
@pytest.mark.parametrize("dtype,d,hq,hkv", CUDA_CORES)
def test_attend(dtype, d, hq, hkv, layers, slots, n):
    c2kv = H.lib()
    wl = synth.scaled(synth.workload("tiny_f32" if dtype == "f32" else "llama8b"), n_q_heads=hq, n_kv_heads=hkv, head_dim=d, layers=layers)
    td = H.tdtype(wl)
    k = -_opposed(td, layers, slots, hkv, d)
    ks, q = -_opposed(td, layers, 1, n, hkv, d), _opposed(td, layers, 1, n, hq, d)
    v, vs = torch.randn_like(k), torch.randn_like(ks)
    ctx = H.make_ctx(wl, pool_slots=slots, attn_split=1)
    try:
        cid = c2kv.c2kv_compress_chunk(ctx, k, v, slots, 1, c2kv.MODE_STORED)
        cache = c2kv.c2kv_compose(ctx, [0, 1], [cid], None, suffix_capacity=n)
        out, lse = torch.full_like(q, 7.0), torch.zeros((layers, 1, hq, n), device="cuda")
        c2kv.c2kv_attend(ctx, cache, -1, q, ks, vs, n, out, lse)
        c2kv.c2kv_sync(ctx)
        assert out.isnan().all() and not lse.isfinite().any()
    finally:
        c2kv.c2kv_destroy(ctx)


@pytest.mark.parametrize("dtype,d,hq,hkv", CUDA_CORES[:2])
def test_extract(dtype, d, hq, hkv):
    c2kv = H.lib()
    wl = synth.scaled(synth.workload("tiny_f32"), n_q_heads=hq, n_kv_heads=hkv, head_dim=d)
    for n, ratio in ((30, 4), (333, 16)):
        rows = n + -(-n // ratio)
        q, k = _opposed(torch.float32, 1, rows, hq, d), -_opposed(torch.float32, 1, rows, hkv, d)
        out, lse = torch.full_like(q, 7.0), torch.zeros((1, hq, rows), device="cuda")
        ctx = H.make_ctx(wl, pool_slots=16)
        try:
            c2kv.c2kv_extract_attention(ctx, 1, q, k, torch.randn_like(k), n, ratio, out, lse)
            c2kv.c2kv_sync(ctx)
        finally:
            c2kv.c2kv_destroy(ctx)
        assert out.isnan().all() and not lse.isfinite().any()
