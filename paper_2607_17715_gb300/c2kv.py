"""Thin Python binding of libc2kv (the C ABI in include/c2kv.h).

Argument marshalling only: every function here has the name of the C entry point it
calls, turns torch tensors / numpy arrays into raw pointers, and raises ``C2KVError``
on a non-OK status.  No computation of the method happens in Python, and there is no
fallback: if the compiled library is missing, importing this module fails.
"""
from __future__ import annotations

import array
import ctypes
import os
import sys

import numpy as np

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "_lib", "libc2kv.so")

if not os.path.exists(LIB_PATH):
    raise ImportError(
        f"libc2kv.so not found at {LIB_PATH}: build it first "
        "(python -c 'import __graft_entry__ as g; g.build()')")

_lib = ctypes.CDLL(LIB_PATH)

# status codes / enums (mirror include/c2kv.h)
OK = 0
ERR_ARG, ERR_DTYPE, ERR_NOMEM, ERR_POOL_FULL, ERR_BAD_CHUNK = -1, -2, -3, -4, -5
ERR_POSITIONS, ERR_CUDA, ERR_DEVICE_BOUNDS, ERR_STATE, ERR_UNSUPPORTED = -6, -7, -8, -9, -10
DTYPE_BF16, DTYPE_F32 = 0, 1
MODE_MEANPOOL, MODE_PROVIDED, MODE_STORED, MODE_HOST = 0, 1, 2, 3
ATTN_AUTO, ATTN_SIMT, ATTN_TC = 0, 1, 2
FUSE_AUTO, FUSE_NEVER, FUSE_ALWAYS = 0, 1, 2
STORAGE_LOCAL_ROPE, STORAGE_PRE_ROPE = 0, 1
PAGES_NATIVE, PAGES_E4M3 = 0, 1
PROF_COMPOSE, PROF_COMPRESS, PROF_SUFFIX, PROF_ATTN, PROF_COMBINE, PROF_DECODE = 0, 1, 2, 3, 4, 5
PROF_EXTRACT, PROF_FUSED = 6, 7
PROF_KINDS = 8
PROF_NAMES = ("compose", "compress", "suffix", "attention", "combine", "decode", "extract",
              "fused")

STATUS_NAMES = {
    0: "OK", -1: "ERR_ARG", -2: "ERR_DTYPE", -3: "ERR_NOMEM", -4: "ERR_POOL_FULL",
    -5: "ERR_BAD_CHUNK", -6: "ERR_POSITIONS", -7: "ERR_CUDA", -8: "ERR_DEVICE_BOUNDS",
    -9: "ERR_STATE", -10: "ERR_UNSUPPORTED",
}


class c2kv_config(ctypes.Structure):
    _fields_ = [("layers", ctypes.c_int32), ("n_q_heads", ctypes.c_int32),
                ("n_kv_heads", ctypes.c_int32), ("head_dim", ctypes.c_int32),
                ("rope_theta", ctypes.c_double), ("dtype", ctypes.c_int32),
                ("pool_slots", ctypes.c_int32), ("fixed_pos", ctypes.c_int32),
                ("attn_impl", ctypes.c_int32), ("attn_split", ctypes.c_int32),
                ("fuse", ctypes.c_int32), ("storage", ctypes.c_int32),
                ("attn_pairs", ctypes.c_int32)]


class c2kv_chunk_desc(ctypes.Structure):
    _fields_ = [("n_tokens", ctypes.c_int32), ("ratio_k", ctypes.c_int32),
                ("n_slots", ctypes.c_int32), ("slot_base", ctypes.c_int32),
                ("k", ctypes.c_void_p), ("v", ctypes.c_void_p),
                ("layer_stride", ctypes.c_int64)]


_P32 = ctypes.POINTER(ctypes.c_int32)


class c2kv_cache_desc(ctypes.Structure):
    _fields_ = [("batch", ctypes.c_int32), ("layers", ctypes.c_int32),
                ("rows", ctypes.c_int64), ("k", ctypes.c_void_p), ("v", ctypes.c_void_p),
                ("pos", ctypes.c_void_p), ("row_base", _P32), ("n_slots", _P32),
                ("l_req", _P32), ("capacity", _P32), ("suffix_capacity", ctypes.c_int32)]


_VP, _I32, _I64 = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64


class c2kv_pages(ctypes.Structure):
    _fields_ = [("k", _VP), ("v", _VP), ("k_scale", _VP), ("v_scale", _VP), ("page_stride", _I64),
                ("scale_stride", _I64), ("n_pages", _I32), ("page_size", _I32), ("format", _I32)]


_SIGS = {
    "c2kv_abi_version": (_I32, []),
    "c2kv_create": (_I32, [ctypes.POINTER(c2kv_config), _VP, ctypes.POINTER(_VP)]),
    "c2kv_destroy": (_I32, [_VP]),
    "c2kv_set_stream": (_I32, [_VP, _VP]),
    "c2kv_compress_chunk": (_I32, [_VP, _VP, _VP, _I32, _I32, _I32, _P32]),
    "c2kv_free_chunk": (_I32, [_VP, _I32]),
    "c2kv_chunk_info": (_I32, [_VP, _I32, ctypes.POINTER(c2kv_chunk_desc)]),
    "c2kv_compose": (_I32, [_VP, _I32, _P32, _P32, _P32, _I32, ctypes.POINTER(_VP)]),
    "c2kv_compose_attend": (_I32, [_VP, _I32, _P32, _P32, _P32, _I32, _VP, _VP, _VP, _I32, _VP,
                                   _VP, ctypes.POINTER(_VP)]),
    "c2kv_cache_info": (_I32, [_VP, ctypes.POINTER(c2kv_cache_desc)]),
    "c2kv_attend": (_I32, [_VP, _VP, _I32, _VP, _VP, _VP, _I32, _VP, _VP]),
    "c2kv_attend_noalloc": (_I32, [_VP, _VP, _I32, _VP, _VP, _VP, _I32, _VP, _VP]),
    "c2kv_decode": (_I32, [_VP, _VP, _I32, _VP, _VP, _VP, _P32, _VP, _VP]),
    "c2kv_extract_attention": (_I32, [_VP, _I32, _VP, _VP, _VP, _I32, _I32, _VP, _VP]),
    "c2kv_paged_append": (_I32, [_VP, _VP, _I32, _VP, _I32, _I64, _VP, _VP, _VP, _VP, _I64, _VP]),
    "c2kv_paged_gather": (_I32, [_VP, _VP, _I32, _VP, _I32, _I64, _VP, _VP, _VP, _VP, _I64, _VP]),
    "c2kv_paged_attend": (_I32, [_VP, _VP, _I32, _VP, _I32, _I64, _VP, _VP, _I32, _VP, _I64, _VP, _VP, _VP]),
    "c2kv_verify_drafts": (_I32, [_VP, _I32, _VP, _I32, _VP, _VP, _I64, _VP, _I64, _VP, _VP, _VP, _VP]),
    "c2kv_cache_release": (_I32, [_VP, _VP]),
    "c2kv_sync": (_I32, [_VP]),
    "c2kv_last_error": (ctypes.c_char_p, [_VP]),
    "c2kv_inject_fault": (_I32, [_VP, _I32]),
    "c2kv_profile_enable": (_I32, [_VP, _I32]),
    "c2kv_profile_read": (_I32, [_VP, ctypes.POINTER(ctypes.c_float), _P32]),
}
for _name, (_res, _args) in _SIGS.items():
    _fn = getattr(_lib, _name)
    _fn.restype = _res
    _fn.argtypes = _args


class C2KVError(RuntimeError):
    def __init__(self, status: int, message: str):
        super().__init__(f"{STATUS_NAMES.get(status, status)}: {message}")
        self.status = status


def _check(status: int, ctx=None):
    if status != OK:
        raise C2KVError(status, c2kv_last_error(ctx))


def _ptr(x):
    """Raw address of a torch tensor, numpy array, int or None."""
    if x is None:
        return None
    if isinstance(x, int):
        return x
    if hasattr(x, "data_ptr"):
        return x.data_ptr()
    if isinstance(x, np.ndarray):
        return x.ctypes.data
    raise TypeError(f"cannot take the address of {type(x)}")


def _i32(arr):
    """The values as int32 memory that the first result keeps, and its pointer."""
    if arr is None:
        return None, None
    if type(arr) in (list, tuple) and arr:
        # a short list costs numpy some 3 us, an int array 0.5; it refuses what does not fit too.
        # Anything but integers (floats, nested lists) is numpy's to convert
        try:
            a = array.array("i", arr)
        except TypeError:
            pass
        else:
            p = (ctypes.c_int32 * len(a)).from_buffer(a)
            return p, p
    a = np.ascontiguousarray(np.asarray(arr, dtype=np.int32))
    return a, a.ctypes.data_as(_P32)


def _i32_at(arr):
    """The values as int32 memory that the first result keeps, its address and how many there are: for
    calls that a generation step makes by the dozen (an address costs half of what a pointer does)."""
    if type(arr) is list:
        try:
            a = array.array("i", arr)
        except TypeError:
            pass
        else:
            return a, a.buffer_info()[0], len(a)
    a = np.ascontiguousarray(np.asarray(arr, dtype=np.int32))
    return a, a.ctypes.data, len(a)


def _stream_handle(stream):
    if stream is None:
        return None
    if isinstance(stream, int):
        return stream
    return stream.cuda_stream


class _Known:
    """What the paged calls' tensors must be like: heads and channels, and the rows' type (torch's)."""
    __slots__ = ("q", "kv", "f32", "dtype")

    def __init__(self, hq, hkv, d, f32):
        self.q, self.kv, self.f32, self.dtype = (hq, d), (hkv, d), f32, None


_contexts = {}                                       # of each context made here


def _torch():
    """torch, which whoever passes a tensor has imported (the binding does not)."""
    return sys.modules["torch"]


def _of_type(x, dtype, what):
    if x.dtype is not dtype:
        raise ValueError(f"{what} must hold {dtype}, not {x.dtype}")


# ---------------------------------------------------------------------------- calls

def c2kv_abi_version() -> int:
    return _lib.c2kv_abi_version()


def c2kv_last_error(ctx=None) -> str:
    msg = _lib.c2kv_last_error(ctx)
    return msg.decode() if msg else ""


def c2kv_create(layers, n_q_heads, n_kv_heads, head_dim, rope_theta, dtype, pool_slots,
                fixed_pos=0, attn_impl=ATTN_AUTO, stream=None, attn_split=0, fuse=0,
                storage=STORAGE_LOCAL_ROPE, attn_pairs=0):
    cfg = c2kv_config(layers, n_q_heads, n_kv_heads, head_dim, float(rope_theta), dtype,
                      pool_slots, int(fixed_pos), attn_impl, attn_split, fuse, storage, attn_pairs)
    out = _VP()
    _check(_lib.c2kv_create(ctypes.byref(cfg), _stream_handle(stream), ctypes.byref(out)))
    _contexts[out.value] = _Known(n_q_heads, n_kv_heads, head_dim, dtype == DTYPE_F32)
    return out.value


def c2kv_destroy(ctx):
    _check(_lib.c2kv_destroy(ctx), None)
    _contexts.pop(ctx, None)


def c2kv_set_stream(ctx, stream):
    _check(_lib.c2kv_set_stream(ctx, _stream_handle(stream)), ctx)


def c2kv_compress_chunk(ctx, k, v, n_tokens, ratio_k, mode) -> int:
    cid = ctypes.c_int32(-1)
    _check(_lib.c2kv_compress_chunk(ctx, _ptr(k), _ptr(v), n_tokens, ratio_k, mode,
                                    ctypes.byref(cid)), ctx)
    return cid.value


def c2kv_free_chunk(ctx, chunk_id):
    _check(_lib.c2kv_free_chunk(ctx, chunk_id), ctx)


def c2kv_chunk_info(ctx, chunk_id) -> dict:
    d = c2kv_chunk_desc()
    _check(_lib.c2kv_chunk_info(ctx, chunk_id, ctypes.byref(d)), ctx)
    return {f: getattr(d, f) for f, _ in c2kv_chunk_desc._fields_}


def c2kv_compose(ctx, req_ptr, chunk_ids, positions=None, suffix_capacity=0):
    rp, rp_p = _i32(req_ptr)
    ids, ids_p = _i32(chunk_ids)
    pos, pos_p = _i32(positions)
    out = _VP()
    _check(_lib.c2kv_compose(ctx, len(rp) - 1, rp_p, ids_p, pos_p, suffix_capacity,
                             ctypes.byref(out)), ctx)
    return out.value


def c2kv_compose_attend(ctx, req_ptr, chunk_ids, positions, suffix_capacity, q, k_suf, v_suf,
                        n_suffix, out, lse=None):
    """Compose the requests' chunks and attend their suffixes over all layers in one call
    (fused on the tensor-core route); returns the composed cache."""
    rp, rp_p = _i32(req_ptr)
    ids, ids_p = _i32(chunk_ids)
    pos, pos_p = _i32(positions)
    cache = _VP()
    _check(_lib.c2kv_compose_attend(ctx, len(rp) - 1, rp_p, ids_p, pos_p, suffix_capacity, _ptr(q),
                                    _ptr(k_suf), _ptr(v_suf), n_suffix, _ptr(out), _ptr(lse),
                                    ctypes.byref(cache)), ctx)
    return cache.value


def c2kv_cache_info(cache) -> dict:
    d = c2kv_cache_desc()
    _check(_lib.c2kv_cache_info(cache, ctypes.byref(d)))
    b = d.batch
    i32_b = ctypes.c_int32 * b
    host = {f: np.frombuffer(i32_b.from_address(ctypes.addressof(getattr(d, f).contents)), np.int32).copy()
            for f in ("row_base", "n_slots", "l_req", "capacity")}
    return dict(batch=b, layers=d.layers, rows=d.rows, k=d.k, v=d.v, pos=d.pos, **host,
                suffix_capacity=d.suffix_capacity)


def c2kv_attend(ctx, cache, layer, q, k_suf, v_suf, n_suffix, out, lse=None):
    _check(_lib.c2kv_attend(ctx, cache, layer, _ptr(q), _ptr(k_suf), _ptr(v_suf), n_suffix,
                            _ptr(out), _ptr(lse)), ctx)


def c2kv_attend_noalloc(ctx, cache, layer, q, k_suf, v_suf, n_suffix, out, lse=None):
    """c2kv_attend without any device allocation (scratch in a fixed 16 MiB device array;
    see include/c2kv.h for the limits)."""
    _check(_lib.c2kv_attend_noalloc(ctx, cache, layer, _ptr(q), _ptr(k_suf), _ptr(v_suf),
                                    n_suffix, _ptr(out), _ptr(lse)), ctx)


def c2kv_decode(ctx, cache, layer, q, k_new, v_new, steps, out, lse=None):
    """One decode step: request r's new token at suffix index steps[r] (host int array)."""
    st, st_p = _i32(steps)
    _check(_lib.c2kv_decode(ctx, cache, layer, _ptr(q), _ptr(k_new), _ptr(v_new), st_p,
                            _ptr(out), _ptr(lse)), ctx)


def c2kv_extract_attention(ctx, n_layers, q, k, v, n_tokens, ratio_k, out, lse=None):
    """SIF-masked extraction attention over [document tokens; C2 tokens] of one chunk."""
    _check(_lib.c2kv_extract_attention(ctx, n_layers, _ptr(q), _ptr(k), _ptr(v), n_tokens,
                                       ratio_k, _ptr(out), _ptr(lse)), ctx)


def make_pages(k, v, k_scale=None, v_scale=None):
    """Describe pages in torch tensors: k, v [n_pages, Hkv, page_size, d] in the context's type, or
    8-bit (torch.float8_e4m3fn or uint8 codes) with fp32 scales [n_pages, Hkv, page_size].  The
    description keeps the tensors."""
    n, _, rows, d = k.shape
    t = _torch()
    eight = k.dtype in (t.float8_e4m3fn, t.uint8)
    if not eight and k.dtype not in (t.bfloat16, t.float32):
        raise ValueError(f"pages hold bfloat16, float32, float8_e4m3fn or its codes as uint8, not {k.dtype}")
    for x, inner in ((k, (rows * d, d, 1)), (v, (rows * d, d, 1)), (k_scale, (rows, 1)), (v_scale, (rows, 1))):
        # (the stride of a single head says nothing)
        if x is not None and (x.stride()[2:] != inner[1:] or (k.shape[1] > 1 and x.stride(1) != inner[0]) or (n > 1 and x.stride(0) == 0)):
            raise ValueError("a page must be one dense block of its heads' rows")
    if v.shape != k.shape or v.dtype != k.dtype or (n > 1 and v.stride(0) != k.stride(0)):
        raise ValueError("k and v pages must have one shape, type and stride")
    if eight and (k_scale is None or v_scale is None or k_scale.shape != k.shape[:3] or v_scale.shape != k.shape[:3] or
                  k_scale.dtype is not t.float32 or v_scale.dtype is not t.float32 or
                  (n > 1 and v_scale.stride(0) != k_scale.stride(0))):
        raise ValueError("8-bit pages need fp32 scales [n_pages, Hkv, page_size], of one stride")
    p = c2kv_pages(_ptr(k), _ptr(v), _ptr(k_scale), _ptr(v_scale), k.stride(0) if n > 1 else 0,
                   k_scale.stride(0) if eight and n > 1 else 0, n, rows, PAGES_E4M3 if eight else PAGES_NATIVE)
    p.keep = (k, v, k_scale, v_scale)
    p.heads = (k.shape[1], d)
    p.dtype = None if eight else k.dtype
    p.fits = None                                    # the context that they were last found to fit
    p.address = ctypes.addressof(p)
    return p


def _table(table, batch, rows):
    """Address, width and row stride of a table of page numbers (a torch int32 tensor [B, width]) for
    the requests that a call's host arrays describe."""
    b, w = table.shape
    if b != batch or rows != batch:
        raise ValueError("the table, the ranges and the rows must describe one batch")
    _of_type(table, _torch().int32, "a table")
    if table.is_contiguous():
        return table.data_ptr(), w, w
    if w > 1 and table.stride(1) != 1:
        raise ValueError("a table's rows must be dense")
    return table.data_ptr(), w, table.stride(0) if b > 1 else w


def _known(ctx, pages, x, heads):
    """What the tensors of a call must be like, by its context (one that was not made here: by the pages and by
    x, whose heads are `heads`).  The pages must be the context's."""
    known = _contexts.get(ctx)
    if known is not None and pages.fits is known:
        return known
    t = _torch()
    if known is None:
        if x.dtype is not t.bfloat16 and x.dtype is not t.float32:
            raise ValueError(f"rows hold bfloat16 or float32, not {x.dtype}")
        known = _Known(heads, *pages.heads, x.dtype is t.float32)
    known.dtype = t.float32 if known.f32 else t.bfloat16
    if pages.heads != known.kv or pages.dtype not in (None, known.dtype):
        raise ValueError(f"pages hold heads {pages.heads} of {pages.dtype}, the context has {known.kv} of {known.dtype}")
    pages.fits = known
    return known


def _token_stride(x, tokens, heads, dtype):
    """Elements between tokens of a torch tensor [at least `tokens`, *heads] whose heads are dense (0: dense too).
    A dense tensor may have its heads in one dimension, or be one run."""
    dense, shape = x.is_contiguous(), x.shape
    if x.dtype is not dtype:
        raise ValueError(f"rows must hold {dtype}, as the context does, not {x.dtype}")
    t, *inner = shape
    if t < tokens or (shape[1:] != heads and not (dense and inner == [heads[0] * heads[1]])):
        if len(shape) != 1 or not dense or t < tokens * heads[0] * heads[1]:
            raise ValueError(f"{tokens} tokens of {heads[0]} heads of {heads[1]} channels are needed, not {tuple(shape)}")
    if dense:
        return 0
    h, d = inner
    if (h > 1 and x.stride(1) != d) or x.stride(2) != 1:
        raise ValueError("a token's heads must be one dense block")
    if t > 1 and x.stride(0) == 0:
        raise ValueError("tokens must not share their memory")
    return x.stride(0) if t > 1 else 0


def _pair_stride(ctx, pages, x, y, tokens):
    """The token stride of two tensors of the pages' heads."""
    known = _known(ctx, pages, x, 0)
    dtype, (h, d) = known.dtype, known.kv
    want = (tokens, h, d)
    if x.dtype is dtype and y.dtype is dtype and x.shape == want and y.shape == want and x.is_contiguous() and y.is_contiguous():
        return 0
    s, t = _token_stride(x, tokens, known.kv, dtype), _token_stride(y, tokens, known.kv, dtype)
    if s != t and tokens > 1 and x.stride(0) != y.stride(0):
        raise ValueError("k and v must have one token stride")
    return s or t


def _vector(x, n, what, dtype):
    """Address of a dense tensor of at least n entries (or of what has an address only)."""
    if x is None:
        return None
    if not hasattr(x, "data_ptr"):
        return _ptr(x)
    if x.dtype is not dtype or x.numel() < n or not x.is_contiguous():
        raise ValueError(f"{what} must be one dense run of {n} entries of {dtype}, not {tuple(x.shape)} of {x.dtype}")
    return x.data_ptr()


def _rows(x, rows, vocab, what, dtype):
    """Address and row stride of probabilities [at least `rows`, vocab] (0: dense)."""
    shape, dense = x.shape, x.is_contiguous()
    if x.dtype is dtype and dense and shape == (rows, vocab):
        return x.data_ptr(), 0
    if x.dtype is not dtype or len(shape) != 2 or shape[0] < rows or shape[1] != vocab or (vocab > 1 and x.stride(1) != 1):
        raise ValueError(f"{what} must be {rows} rows of {vocab} probabilities, each dense, of {dtype}, not {tuple(shape)} of {x.dtype}")
    if shape[0] < 2 or dense:
        return x.data_ptr(), 0
    if x.stride(0) == 0:
        raise ValueError(f"{what}: rows must not share their memory")
    return x.data_ptr(), x.stride(0)


def c2kv_paged_append(ctx, pages, table, new_ptr, start, k, v, turn=None):
    """Write new tokens k, v [T, Hkv, d] into their requests' pages, K turned by turn [T]."""
    ptr, ptr_p, n = _i32_at(new_ptr)
    st, st_p, m = _i32_at(start)
    tb, w, ts = _table(table, n - 1, m)
    t = ptr[m]
    _check(_lib.c2kv_paged_append(ctx, pages.address, m, tb, w, ts, ptr_p, st_p, k.data_ptr(), v.data_ptr(),
                                  _pair_stride(ctx, pages, k, v, t), _vector(turn, t, "turn", _torch().int32)), ctx)


def c2kv_paged_gather(ctx, pages, table, row_ptr, start, k_out, v_out, turn=None):
    """Read rows of the pages back into k_out, v_out [T, Hkv, d], K turned by turn [T]."""
    ptr, ptr_p, n = _i32_at(row_ptr)
    st, st_p, m = _i32_at(start)
    tb, w, ts = _table(table, n - 1, m)
    t = ptr[m]
    _check(_lib.c2kv_paged_gather(ctx, pages.address, m, tb, w, ts, ptr_p, st_p, k_out.data_ptr(), v_out.data_ptr(),
                                  _pair_stride(ctx, pages, k_out, v_out, t), _vector(turn, t, "turn", _torch().int32)), ctx)


def c2kv_paged_attend(ctx, pages, table, q_ptr, n_keys, q, out, lse=None, turn=None, window=0):
    """Attention of each request's newest tokens q [T, Hq, d] over its n_keys rows."""
    ptr, ptr_p, n = _i32_at(q_ptr)
    nk, nk_p, m = _i32_at(n_keys)
    tb, w, ts = _table(table, n - 1, m)
    t, d = ptr[m], pages.heads[1]
    known = _contexts.get(ctx)
    if known is None or pages.fits is not known:
        known = _known(ctx, pages, q, q.shape[1] if q.dim() == 3 else q.shape[-1] // d)
    dtype, hq, tensor, stride = known.dtype, known.q[0], hasattr(out, "data_ptr"), 0
    want = (t, hq, d)
    if not (q.dtype is dtype and q.shape == want and q.is_contiguous()):
        stride = _token_stride(q, t, known.q, dtype)
    if tensor and not (out.dtype is dtype and out.shape == want and out.is_contiguous()) and _token_stride(out, t, known.q, dtype):
        raise ValueError("out must be dense")
    if lse is not None and hasattr(lse, "data_ptr"):
        _of_type(lse, _torch().float32, "lse")
        if not (lse.is_contiguous() and (lse.shape == (hq, t) or lse.dim() == 1 and lse.shape[0] >= hq * t)):
            raise ValueError(f"lse must be dense, [{hq}, {t}]")
    _check(_lib.c2kv_paged_attend(ctx, pages.address, m, tb, w, ts, ptr_p, nk_p, window, q.data_ptr(), stride,
                                  _vector(turn, t, "turn", _torch().int32), out.data_ptr() if tensor else _ptr(out), _ptr(lse)), ctx)


def c2kv_verify_drafts(ctx, draft_ptr, tokens, p, q, u_accept, u_next, n_accepted, next_token):
    """Accept drafted tokens against the target's probabilities p [T + B, V] and the draft's q [T, V]
    (None: drafts without probabilities), and draw the token that follows them."""
    ptr, ptr_p, n = _i32_at(draft_ptr)
    b, vocab, i32, f32 = n - 1, p.shape[1], _torch().int32, _torch().float32
    t = ptr[b] if n > 0 else 0
    pp, ps = _rows(p, t + b, vocab, "p", f32)
    qp, qs = (None, 0) if q is None else _rows(q, t, vocab, "q", f32)
    _check(_lib.c2kv_verify_drafts(ctx, b, ptr_p, vocab, _vector(tokens, t, "tokens", i32), pp, ps, qp, qs,
                                   _vector(u_accept, t, "u_accept", f32), _vector(u_next, b, "u_next", f32),
                                   _vector(n_accepted, b, "n_accepted", i32), _vector(next_token, b, "next_token", i32)), ctx)


def c2kv_cache_release(ctx, cache):
    _check(_lib.c2kv_cache_release(ctx, cache), ctx)


def c2kv_sync(ctx):
    _check(_lib.c2kv_sync(ctx), ctx)


def c2kv_profile_enable(ctx, on=True):
    _check(_lib.c2kv_profile_enable(ctx, int(bool(on))), ctx)


def c2kv_profile_read(ctx) -> dict:
    """{kind name: (mean ms, launches)} for the launches recorded since the last read."""
    ms = (ctypes.c_float * PROF_KINDS)()
    cnt = (ctypes.c_int32 * PROF_KINDS)()
    _check(_lib.c2kv_profile_read(ctx, ms, cnt), ctx)
    return {PROF_NAMES[k]: (ms[k], cnt[k]) for k in range(PROF_KINDS)}


def c2kv_inject_fault(ctx, what):
    _check(_lib.c2kv_inject_fault(ctx, what), ctx)


# ---------------------------------------------------------------- device memory views

class _CudaArray:
    """Minimal __cuda_array_interface__ wrapper so torch can view library-owned memory."""

    def __init__(self, ptr, shape, typestr):
        self.__cuda_array_interface__ = {
            "shape": tuple(int(s) for s in shape), "typestr": typestr,
            "data": (int(ptr), False), "version": 2, "strides": None,
        }


def device_view(ptr, shape, dtype):
    """A torch tensor aliasing library-owned device memory (no copy).  Valid only while
    the owning object (cache, pool) lives."""
    import torch
    if dtype == torch.bfloat16:
        t = torch.as_tensor(_CudaArray(ptr, shape, "<i2"), device="cuda")
        return t.view(torch.bfloat16)
    typestr = {torch.float32: "<f4", torch.int32: "<i4"}[dtype]
    return torch.as_tensor(_CudaArray(ptr, shape, typestr), device="cuda")
