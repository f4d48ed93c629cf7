"""What the binding of generation that branches refuses to take the address of (no GPU: the refusal comes before
the call, and a call with no context answers ERR_ARG)."""
import os
import re

import pytest
import torch

import __graft_entry__ as g

g.build()
from paper_2607_17715_gb300 import c2kv  # noqa: E402

HQ, HKV, D, T, V = 4, 2, 64, 4, 10
I32 = torch.int32


@pytest.fixture()
def args():
    """Arguments of each call that it takes."""
    k = torch.zeros((3, 6, HKV, 16, D), dtype=torch.bfloat16)
    pages, layers = c2kv.make_pages(k[0], k[1]), c2kv.make_layers(k, k.clone())
    table, q = torch.zeros((2, 3), dtype=I32), torch.zeros((T, HQ, D), dtype=torch.bfloat16)
    node = torch.zeros(T, dtype=I32)
    return {
        "attend": dict(ctx=None, pages=pages, table=table, ptr=[0, 3, 4], keys=[7, 3], parent=node, q=q, out=q.clone(),
                       lse=torch.zeros((HQ, T)), turn=node.clone()),
        "walk": dict(ctx=None, ptr=[0, 3, 4], tokens=node, parent=node.clone(), p=torch.zeros((T, V)), u=torch.zeros(T),
                     n_accepted=torch.zeros(2, dtype=I32), path=node.clone(), next_token=torch.zeros(2, dtype=I32)),
        "keep": dict(ctx=None, layers=layers, table=table, ptr=[0, 3, 4], start=[7, 3], path=node, n_accepted=torch.zeros(2, dtype=I32)),
        "select": dict(ctx=None, x=torch.zeros((6, V)), score=torch.zeros((2, 3)), parent=torch.zeros((2, 5), dtype=I32),
                       token=torch.zeros((2, 5), dtype=I32), score_out=torch.zeros((2, 5)), norm=torch.zeros(6),
                       done=torch.zeros((2, 3), dtype=I32), end_token=1, done_out=torch.zeros((2, 5), dtype=I32)),
        "reorder": dict(ctx=None, layers=layers, table=torch.zeros((6, 3), dtype=I32), rows=[7, 20], parent=torch.zeros((2, 3), dtype=I32),
                        out=torch.zeros((6, 3), dtype=I32))}


CALLS = {"attend": "c2kv_paged_attend_tree", "walk": "c2kv_verify_tree", "keep": "c2kv_paged_keep", "select": "c2kv_beam_select",
         "reorder": "c2kv_paged_reorder"}


def _call(name, a):
    getattr(c2kv, CALLS[name])(*a.values())


def _taken(name, a):
    with pytest.raises(c2kv.C2KVError) as e:         # (by the library, for want of a context)
        _call(name, a)
    assert e.value.status == c2kv.ERR_ARG


@pytest.mark.parametrize("name", CALLS)
def test_plain_arguments_are_taken(args, name):
    _taken(name, args[name])


def _wide(x):
    """The same shape with gaps along the last dimension."""
    return torch.zeros((*x.shape[:-1], 2 * x.shape[-1]), dtype=x.dtype)[..., ::2]


VECTORS = {"attend": ["parent", "turn"], "walk": ["tokens", "parent", "u", "n_accepted", "path", "next_token"], "keep": ["path", "n_accepted"],
           "select": ["score", "parent", "token", "score_out", "norm", "done", "done_out"], "reorder": ["parent"]}


@pytest.mark.parametrize("name,key", [(n, k) for n, ks in VECTORS.items() for k in ks])
def test_entries_of_another_kind(args, name, key):
    """Gaps where a dense run is read or written, memory shared by entries, another type, fewer entries."""
    a = args[name]
    x = a[key]
    for y in (_wide(x), x[:1].expand(x.shape), x.to(torch.float64), x.to(torch.int16), x.flatten()[:-1]):
        with pytest.raises(ValueError):
            _call(name, dict(a, **{key: y}))


ROWS = [("attend", "q", lambda x: x[:3]), ("attend", "q", lambda x: x.float()), ("attend", "out", lambda x: x[:1].expand(x.shape)),
        ("attend", "lse", lambda x: x.double()), ("attend", "table", lambda x: x[:1]), ("attend", "table", lambda x: x.long()),
        ("walk", "p", lambda x: x[:3]), ("walk", "p", lambda x: x.bfloat16()), ("walk", "p", _wide), ("walk", "p", lambda x: x[:1].expand(T, V)),
        ("keep", "table", lambda x: x.long()), ("keep", "table", lambda x: x[:1]), ("select", "x", lambda x: x[:5]),
        ("select", "x", lambda x: x.half()), ("select", "x", lambda x: x[:1].expand(6, V)), ("select", "x", _wide),
        ("reorder", "table", lambda x: x[:5]), ("reorder", "table", lambda x: x.long()), ("reorder", "out", lambda x: x[:, :2]),
        ("reorder", "out", lambda x: x[:1].expand(6, 3)), ("reorder", "out", lambda x: x.long()), ("reorder", "parent", lambda x: x[:1]),
        ("reorder", "parent", lambda x: x.view(-1))]


@pytest.mark.parametrize("name,key,change", ROWS)
def test_memory_that_is_not_what_the_call_reads_or_writes(args, name, key, change):
    a = args[name]
    with pytest.raises(ValueError):
        _call(name, dict(a, **{key: change(a[key])}))


def test_a_layer_alone_and_layers_one_by_one(args):
    a = args["keep"]
    one = a["layers"].keep[0]
    _taken("keep", dict(a, layers=one))
    _taken("keep", dict(a, layers=c2kv.make_layers([one, one])))
    k = torch.zeros((2, 6, HKV, 16, D)).to(torch.float8_e4m3fn)
    s = torch.zeros((2, 6, HKV, 16))
    _taken("reorder", dict(args["reorder"], layers=c2kv.make_layers(k, k.clone(), s, s.clone())))


def test_layers_that_differ():
    k = torch.zeros((6, HKV, 16, D), dtype=torch.bfloat16)
    p = c2kv.make_pages(k, k.clone())
    for other in (k.float(), torch.zeros((6, HKV + 1, 16, D), dtype=torch.bfloat16)):
        with pytest.raises(ValueError):
            c2kv.make_layers([p, c2kv.make_pages(other, other.clone())])
    with pytest.raises(ValueError):
        c2kv.make_layers([])


def test_other_layouts_of_the_same_are_taken(args):
    _taken("walk", dict(args["walk"], p=torch.zeros((T + 2, V + 6))[:, :V]))
    _taken("select", dict(args["select"], x=torch.zeros((6, V), dtype=torch.bfloat16), norm=None, done=None, done_out=None))
    _taken("reorder", dict(args["reorder"], out=torch.zeros((6, 8), dtype=I32)[:, :3]))
    fused = torch.zeros((T, HQ + 2 * HKV, D), dtype=torch.bfloat16)
    _taken("attend", dict(args["attend"], q=fused[:, :HQ], lse=None, turn=None))


@pytest.mark.parametrize("name,kernel", [("verify_tree.cu", "verify_tree_kernel")])
def test_peers_are_written_after_they_have_started(repo_root, name, kernel):
    """A barrier of the cluster before the first store to another CTA's shared memory, and nothing that can return
    ahead of it."""
    with open(os.path.join(repo_root, "paper_2607_17715_gb300", "csrc", name)) as f:
        text = re.sub(r"//[^\n]*", "", f.read())
    body = text[text.index(kernel + "(const __grid_constant__"):]
    arrive, wait, store = (body.find(x) for x in ("cluster_started()", "cluster_started_wait()", "st_peer("))
    assert 0 <= arrive < wait < store and "return" not in body[:wait]


@pytest.mark.parametrize("name", ["verify_tree.cu", "draw.cuh", "beam_select.cu", "paged_rows.cu", "paged.cuh"])
def test_overlapped_kernels_load_no_read_only_memory(repo_root, name):
    """Kernels that are set up while the one before them runs load what that wrote by ordinary loads."""
    with open(os.path.join(repo_root, "paper_2607_17715_gb300", "csrc", name)) as f:
        text = re.sub(r"//[^\n]*", "", f.read())
    assert not re.search(r"__ldg\(|\bld16\(|ld\.global(\.\w+)*\.nc", text)
    if name.endswith(".cu"):
        assert ("launch_overlapped" in text or "ProgrammaticStreamSerialization" in text) and "after_kernels_before()" in text
