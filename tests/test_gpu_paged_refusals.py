"""What the paged calls refuse, before anything is enqueued, and what they take though there is nothing
to do."""
import numpy as np
import pytest
import torch

from tests import _paged_helpers as P

pytestmark = pytest.mark.gpu


@pytest.fixture()
def setup():
    c2kv = P.lib()
    ctx = P.context("bf16", 4, 2, 64)
    pg = P.Paged(np.random.default_rng(0), "bf16", "e4m3", 2, 64, 16, [40, 20], fill=0.0)
    yield c2kv, ctx, pg
    c2kv.c2kv_sync(ctx)
    c2kv.c2kv_destroy(ctx)


def _status(c2kv, ctx, name, *args):
    s = getattr(c2kv._lib, name)(ctx, *args)
    assert s == c2kv.OK or c2kv.c2kv_last_error(ctx)
    return s


def _calls(c2kv, ctx, pg):
    """Arguments of each call that it takes, by name, in order."""
    keep = [np.array([0, 3, 4], np.int32), np.array([37, 6], np.int32), np.array([40, 20], np.int32)]
    kv = torch.zeros((4, 2, 64), device="cuda", dtype=torch.bfloat16)
    q = torch.zeros((4, 4, 64), device="cuda", dtype=torch.bfloat16)
    turn = torch.zeros(4, device="cuda", dtype=torch.int32)
    lse = torch.zeros((4, 4), device="cuda")
    pages = pg.pages()
    keep += [kv, q, turn, lse, pages]
    base = dict(pages=pages.address, batch=2, table=pg.table.data_ptr(), width=3, stride=3)
    move = dict(base, ptr=keep[0].ctypes.data, start=keep[1].ctypes.data, k=kv.data_ptr(), v=kv.data_ptr(), kv_stride=0,
                turn=turn.data_ptr())
    return keep, {
        "c2kv_paged_append": move, "c2kv_paged_gather": dict(move),
        "c2kv_paged_attend": dict(base, ptr=keep[0].ctypes.data, n_keys=keep[2].ctypes.data, window=0, q=q.data_ptr(), q_stride=0,
                                  turn=turn.data_ptr(), out=q.data_ptr(), lse=lse.data_ptr())}


CALLS = ["c2kv_paged_append", "c2kv_paged_gather", "c2kv_paged_attend"]


@pytest.mark.parametrize("name", CALLS)
def test_shared_refusals(setup, name):
    c2kv, ctx, pg = setup
    keep, calls = _calls(c2kv, ctx, pg)
    a = calls[name]
    assert _status(c2kv, ctx, name, *a.values()) == c2kv.OK

    def refused(status=c2kv.ERR_ARG, **change):
        assert _status(c2kv, ctx, name, *dict(a, **change).values()) == status, change
    host = torch.zeros((4, 4, 64), dtype=torch.bfloat16)
    bad_ptr = [np.array(x, np.int32) for x in ([1, 3, 4], [0, 3, 2])]
    for key in ("pages", "table", "ptr"):
        refused(**{key: None})
    for b in bad_ptr:
        refused(ptr=b.ctypes.data)
    refused(batch=0)
    refused(batch=-1)
    refused(width=0)
    refused(stride=2)
    refused(width=2)                                         # rows past the table
    tensor = "q" if "q" in a else "k"
    refused(**{tensor: None})
    refused(**{tensor: a[tensor] + 2})                       # not on 16 bytes
    refused(**{tensor: host.data_ptr()})                     # host memory
    refused(turn=host.data_ptr())
    refused(table=host.data_ptr())
    stride = "q_stride" if "q" in a else "kv_stride"
    refused(**{stride: 64})                                  # shorter than a row
    refused(**{stride: 1028})                                # not whole 16-byte lines
    p = keep[-1]
    for field, value, status in (("page_size", 24, c2kv.ERR_ARG), ("page_size", 256, c2kv.ERR_ARG), ("n_pages", 0, c2kv.ERR_ARG),
                                 ("format", 2, c2kv.ERR_DTYPE), ("page_stride", 100, c2kv.ERR_ARG), ("page_stride", 2052, c2kv.ERR_ARG),
                                 ("scale_stride", 30, c2kv.ERR_ARG), ("k", None, c2kv.ERR_ARG), ("v_scale", None, c2kv.ERR_ARG),
                                 ("k", p.k + 8, c2kv.ERR_ARG), ("k_scale", p.k_scale + 4, c2kv.ERR_ARG)):
        before = getattr(p, field)
        setattr(p, field, value)
        refused(status)
        setattr(p, field, before)
    assert _status(c2kv, ctx, name, *a.values()) == c2kv.OK


def test_own_refusals(setup):
    c2kv, ctx, pg = setup
    keep, calls = _calls(c2kv, ctx, pg)
    negative, long = np.array([-1, 0], np.int32), np.array([46, 6], np.int32)
    for name in CALLS[:2]:
        for start in (None, negative.ctypes.data, long.ctypes.data):
            assert _status(c2kv, ctx, name, *dict(calls[name], start=start).values()) == c2kv.ERR_ARG
    a = calls["c2kv_paged_attend"]
    far = np.array([49, 20], np.int32)
    for change in (dict(n_keys=None), dict(n_keys=negative.ctypes.data), dict(n_keys=far.ctypes.data), dict(window=-1), dict(out=None),
                   dict(lse=a["lse"] + 2)):
        assert _status(c2kv, ctx, "c2kv_paged_attend", *dict(a, **change).values()) == c2kv.ERR_ARG
    for name in CALLS:
        assert getattr(c2kv._lib, name)(None, *calls[name].values()) == c2kv.ERR_ARG


@pytest.mark.parametrize("name", CALLS)
def test_nothing_to_do(setup, name):
    """No token at all: taken, whatever the tensors."""
    c2kv, ctx, pg = setup
    keep, calls = _calls(c2kv, ctx, pg)
    none = np.zeros(3, np.int32)
    a = dict(calls[name], ptr=none.ctypes.data)
    a["q" if "q" in a else "k"] = None
    assert _status(c2kv, ctx, name, *a.values()) == c2kv.OK


def test_verify_refusals(setup):
    c2kv, ctx, _ = setup
    ptr = np.array([0, 2, 3], np.int32)
    t = torch.zeros(3, dtype=torch.int32, device="cuda")
    p, q = torch.rand((5, 100), device="cuda"), torch.rand((3, 100), device="cuda")
    u, un, acc, nxt = torch.rand(3, device="cuda"), torch.rand(2, device="cuda"), t[:2].clone(), t[:2].clone()
    a = dict(batch=2, ptr=ptr.ctypes.data, vocab=100, tokens=t.data_ptr(), p=p.data_ptr(), p_stride=0, q=q.data_ptr(), q_stride=0,
             ua=u.data_ptr(), un=un.data_ptr(), acc=acc.data_ptr(), nxt=nxt.data_ptr())
    run = lambda **c: _status(c2kv, ctx, "c2kv_verify_drafts", *dict(a, **c).values())  # noqa: E731
    assert run() == c2kv.OK and run(q=None) == c2kv.OK
    host = torch.zeros(500)
    bad = np.array([0, 2, 1], np.int32)
    for c in (dict(batch=0), dict(ptr=None), dict(ptr=bad.ctypes.data), dict(vocab=0), dict(vocab=(1 << 19) + 1), dict(p=None),
              dict(tokens=None), dict(ua=None), dict(un=None), dict(acc=None), dict(nxt=None), dict(p_stride=99), dict(q_stride=50),
              dict(p=host.data_ptr()), dict(nxt=host.data_ptr()), dict(ua=u.data_ptr() + 2)):
        assert run(**c) == c2kv.ERR_ARG, c
    none = np.zeros(3, np.int32)
    assert run(ptr=none.ctypes.data, tokens=None, ua=None, q=None) == c2kv.OK


def test_binding_refuses_what_it_cannot_describe(setup):
    c2kv, ctx, pg = setup
    kv = torch.zeros((4, 2, 64), device="cuda", dtype=torch.bfloat16)
    with pytest.raises(ValueError):
        c2kv.c2kv_paged_append(ctx, pg.pages(), pg.table, [0, 3, 4], [5], kv, kv)            # rows of one request
    with pytest.raises(ValueError):
        c2kv.c2kv_paged_append(ctx, pg.pages(), pg.table.long(), [0, 3, 4], [5, 6], kv, kv)
    with pytest.raises(ValueError):
        c2kv.c2kv_paged_append(ctx, pg.pages(), pg.table, [0, 3, 4], [5, 6], kv.transpose(1, 2), kv.transpose(1, 2))
    with pytest.raises(ValueError):
        c2kv.make_pages(pg.k, pg.v)                                                          # 8 bits without scales
    with pytest.raises(ValueError):
        c2kv.make_pages(pg.k.transpose(2, 3), pg.v.transpose(2, 3), pg.ks, pg.vs)
    with pytest.raises(ValueError):
        c2kv.make_pages(pg.k, pg.v[:2], pg.ks, pg.vs)


def test_rows_end_at_2_30(setup):
    """The kernels count rows in 32 bits: a request past 2^30 is refused, whatever its table names."""
    c2kv, ctx, pg = setup
    keep, calls = _calls(c2kv, ctx, pg)
    wide, far = dict(width=1 << 27, stride=1 << 27), np.array([(1 << 30) + 1, 20], np.int32)
    for name in CALLS[:2]:
        assert _status(c2kv, ctx, name, *dict(calls[name], start=far.ctypes.data, **wide).values()) == c2kv.ERR_ARG
    assert _status(c2kv, ctx, CALLS[2], *dict(calls[CALLS[2]], n_keys=far.ctypes.data, **wide).values()) == c2kv.ERR_ARG
