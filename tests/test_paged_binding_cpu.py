"""What the binding of the paged calls refuses to take the address of (no GPU: the refusal comes before the
call, and a call with no context answers ERR_ARG)."""
import numpy as np
import pytest
import torch

import __graft_entry__ as g

g.build()
from paper_2607_17715_gb300 import c2kv  # noqa: E402

HQ, HKV, D, T = 4, 2, 64, 4


@pytest.fixture()
def args():
    """Arguments of each call that it takes."""
    k = torch.zeros((6, HKV, 16, D), dtype=torch.bfloat16)
    pages, table = c2kv.make_pages(k, k.clone()), torch.zeros((2, 3), dtype=torch.int32)
    kv, q = torch.zeros((T, HKV, D), dtype=torch.bfloat16), torch.zeros((T, HQ, D), dtype=torch.bfloat16)
    turn = torch.zeros(T, dtype=torch.int32)
    move = dict(ctx=None, pages=pages, table=table, ptr=[0, 3, 4], rows=[7, 1], k=kv, v=kv.clone(), turn=turn)
    one, two = torch.zeros(3, dtype=torch.int32), torch.zeros(2, dtype=torch.int32)
    return {
        "append": move, "gather": dict(move),
        "attend": dict(ctx=None, pages=pages, table=table, ptr=[0, 3, 4], rows=[7, 3], q=q, out=q.clone(),
                       lse=torch.zeros((HQ, T)), turn=turn),
        "verify": dict(ctx=None, ptr=[0, 2, 3], tokens=one, p=torch.zeros((5, 10)), q=torch.zeros((3, 10)), u_accept=torch.zeros(3),
                       u_next=torch.zeros(2), n_accepted=two, next_token=two.clone())}


CALLS = {"append": "c2kv_paged_append", "gather": "c2kv_paged_gather", "attend": "c2kv_paged_attend", "verify": "c2kv_verify_drafts"}


def _call(name, a):
    getattr(c2kv, CALLS[name])(*a.values())


def _taken(name, a):
    with pytest.raises(c2kv.C2KVError) as e:         # (by the library, for want of a context)
        _call(name, a)
    assert e.value.status == c2kv.ERR_ARG


@pytest.mark.parametrize("name", CALLS)
def test_plain_arguments_are_taken(args, name):
    _taken(name, args[name])


def _wide(x, dim):
    """The same shape with gaps along `dim`."""
    shape = list(x.shape)
    shape[dim] *= 2
    return torch.zeros(shape, dtype=x.dtype)[tuple(slice(None, None, 2) if i == dim else slice(None) for i in range(x.dim()))]


STRIDES = [(n, key, change) for n, key, change in [
    ("append", "k", lambda x: x[:1].expand(T, HKV, D)),           # tokens over one another
    ("append", "v", lambda x: x[:1].expand(T, HKV, D)),
    ("gather", "k", lambda x: x[:1].expand(T, HKV, D)),
    ("attend", "q", lambda x: x[:1].expand(T, HQ, D)),
    ("attend", "out", lambda x: x[:1].expand(T, HQ, D)),
    ("verify", "p", lambda x: x[:1].expand(5, 10)),
    ("verify", "q", lambda x: x[:1].expand(3, 10)),
    ("append", "turn", lambda x: _wide(x, 0)),                    # gaps where a dense run is read or written
    ("gather", "turn", lambda x: x[:1].expand(T)),
    ("attend", "turn", lambda x: _wide(x, 0)),
    ("attend", "out", lambda x: _wide(x, 0)),
    ("attend", "out", lambda x: _wide(x, 2)),
    ("attend", "lse", lambda x: x.t().contiguous().t()),
    ("attend", "lse", lambda x: torch.zeros((HQ, T + 1))[:, :T]),
    ("verify", "p", lambda x: _wide(x, 1)),
    ("verify", "q", lambda x: x.t().contiguous().t()),
    ("verify", "tokens", lambda x: _wide(x, 0)),
    ("verify", "u_accept", lambda x: _wide(x, 0)),
    ("verify", "u_next", lambda x: x[:1].expand(2)),
    ("verify", "n_accepted", lambda x: _wide(x, 0)),
    ("verify", "next_token", lambda x: _wide(x, 0))]]
SHAPES = [
    ("append", "k", lambda x: x[:3]),                             # fewer tokens than the ranges say
    ("append", "v", lambda x: x[:3]),
    ("append", "k", lambda x: torch.zeros((T, HKV + 1, D), dtype=x.dtype)),
    ("append", "v", lambda x: torch.zeros((T, HKV, D // 2), dtype=x.dtype)),
    ("append", "turn", lambda x: x[:3]),
    ("gather", "v", lambda x: x[:3]),
    ("attend", "q", lambda x: x[:3]),
    ("attend", "q", lambda x: torch.zeros((T, HQ, D // 2), dtype=x.dtype)),
    ("attend", "out", lambda x: x[:3]),
    ("attend", "out", lambda x: torch.zeros((T, HQ - 1, D), dtype=x.dtype)),
    ("attend", "lse", lambda x: torch.zeros((HQ, T - 1))),
    ("attend", "lse", lambda x: torch.zeros((T, HQ + 1))),
    ("attend", "turn", lambda x: x[:3]),
    ("verify", "p", lambda x: x[:4]),                             # a row a draft, and one more a request
    ("verify", "q", lambda x: x[:2]),
    ("verify", "q", lambda x: torch.zeros((3, 9))),
    ("verify", "tokens", lambda x: x[:2]),
    ("verify", "u_accept", lambda x: x[:2]),
    ("verify", "u_next", lambda x: x[:1]),
    ("verify", "n_accepted", lambda x: x[:1]),
    ("verify", "next_token", lambda x: x[:1])]


@pytest.mark.parametrize("name,key,change", STRIDES + SHAPES)
def test_memory_that_is_not_what_the_call_reads_or_writes(args, name, key, change):
    a = args[name]
    with pytest.raises(ValueError):
        _call(name, dict(a, **{key: change(a[key])}))


def test_pages_over_one_another():
    k = torch.zeros((1, HKV, 16, D), dtype=torch.bfloat16).expand(6, HKV, 16, D)
    with pytest.raises(ValueError):
        c2kv.make_pages(k, k)
    codes, scales = torch.zeros((6, HKV, 16, D), dtype=torch.uint8), torch.zeros((1, HKV, 16)).expand(6, HKV, 16)
    with pytest.raises(ValueError):
        c2kv.make_pages(codes, codes.clone(), scales, scales)


def test_other_layouts_of_the_same_are_taken(args):
    """Buffers with room for more tokens, rows of a fused projection, dense tensors of fewer dimensions."""
    for name, keys in (("append", "kv"), ("attend", "q")):
        a = args[name]
        for key in keys:
            x = a[key]
            _taken(name, dict(a, **{key: torch.zeros((T + 3, *x.shape[1:]), dtype=x.dtype)}))
    fused = torch.zeros((T, HQ + 2 * HKV, D), dtype=torch.bfloat16)
    _taken("append", dict(args["append"], k=fused[:, HQ:HQ + HKV], v=fused[:, HQ + HKV:]))
    _taken("attend", dict(args["attend"], q=fused[:, :HQ], out=torch.zeros((T + 2, HQ, D), dtype=torch.bfloat16), lse=None, turn=None))
    _taken("verify", dict(args["verify"], p=torch.zeros((5, 16))[:, :10], q=None))
    flat = torch.zeros((T, HKV * D), dtype=torch.bfloat16)
    _taken("append", dict(args["append"], k=flat, v=flat.view(-1)))
    flat = torch.zeros((T, HQ * D), dtype=torch.bfloat16)
    _taken("attend", dict(args["attend"], q=flat, out=flat.view(-1), lse=torch.zeros(HQ * T)))
    _taken("append", dict(args["append"], ptr=np.array([0, 3, 4]), rows=np.array([7, 1]), turn=None))


TYPES = [("append", "turn", "int64"), ("gather", "turn", "int64"), ("attend", "turn", "int64"), ("attend", "turn", "float32"),
         ("append", "table", "float32"), ("append", "k", "float16"), ("append", "v", "float32"), ("gather", "v", "float16"),
         ("attend", "q", "float32"), ("attend", "out", "float32"), ("attend", "lse", "float64"), ("attend", "lse", "bfloat16"),
         ("verify", "tokens", "int64"), ("verify", "p", "bfloat16"), ("verify", "q", "float64"), ("verify", "u_accept", "float64"),
         ("verify", "u_next", "bfloat16"), ("verify", "n_accepted", "int64"), ("verify", "next_token", "float32")]


@pytest.mark.parametrize("name,key,dtype", TYPES)
def test_types_that_the_call_would_misread(args, name, key, dtype):
    a = args[name]
    with pytest.raises(ValueError):
        _call(name, dict(a, **{key: a[key].to(getattr(torch, dtype))}))


@pytest.mark.parametrize("dtype", ["float16", "float64", "float8_e5m2", "int16", "bool"])
def test_pages_of_types_that_are_none(dtype):
    k = torch.zeros((6, HKV, 16, D)).to(getattr(torch, dtype))
    s = torch.zeros((6, HKV, 16))
    with pytest.raises(ValueError):
        c2kv.make_pages(k, k.clone(), s, s.clone())


def test_scales_of_another_type():
    k = torch.zeros((6, HKV, 16, D), dtype=torch.uint8)
    s = torch.zeros((6, HKV, 16), dtype=torch.int32)
    with pytest.raises(ValueError):
        c2kv.make_pages(k, k.clone(), s, s.clone())


def test_pages_of_another_type_than_the_rows(args):
    """fp32 rows over 16-bit pages; over 8-bit pages both types of row are some context's."""
    f32 = torch.zeros((T, HKV, D))
    with pytest.raises(ValueError):
        _call("append", dict(args["append"], k=f32, v=f32))
    codes, scale = torch.zeros((6, HKV, 16, D)).to(torch.float8_e4m3fn), torch.zeros((6, HKV, 16))
    _taken("append", dict(args["append"], pages=c2kv.make_pages(codes, codes.clone(), scale, scale.clone()), k=f32, v=f32))


def test_entries_in_any_shape(args):
    """A dense tensor of the entries, whatever its dimensions."""
    a = args["verify"]
    _taken("verify", dict(a, n_accepted=a["n_accepted"][:, None], u_next=a["u_next"].view(1, 2)))


def test_pages_of_one_head_among_others():
    """One head's pages as a slice of several heads': each is one run, wherever the next head would lie."""
    k = torch.zeros((6, 3, 16, D), dtype=torch.bfloat16)[:, 1:2]
    p = c2kv.make_pages(k, k)
    assert p.page_stride == 3 * 16 * D and p.heads == (1, D)
    codes, scale = torch.zeros((6, 3, 16, D), dtype=torch.uint8)[:, 2:], torch.zeros((6, 3, 16))[:, :1]
    p = c2kv.make_pages(codes, codes, scale, scale)
    assert (p.page_stride, p.scale_stride) == (3 * 16 * D, 3 * 16)
