"""What the calls of generation that branches refuse, before anything is enqueued, and what they take though there
is nothing to do."""
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


def _calls(c2kv, pg):
    """Arguments of each call that it takes, by name, in order, and what they lie in."""
    host = [np.array(x, np.int32) for x in ([0, 3, 4], [37, 6], [40, 20])]
    ptr, start, keys = (x.ctypes.data for x in host)
    q = torch.zeros((4, 4, 64), device="cuda", dtype=torch.bfloat16)
    ints = torch.zeros((12, 16), device="cuda", dtype=torch.int32)
    ints[0, :4] = torch.tensor([-1, 0, 0, -1], dtype=torch.int32)
    ints[1, :4] = torch.arange(4)
    f = torch.zeros((9, 1000), device="cuda")
    layers = c2kv.make_layers([pg.pages(), pg.pages()])
    i, x = [ints[k].data_ptr() for k in range(12)], [f[k].data_ptr() for k in range(9)]
    table = dict(table=pg.table.data_ptr(), width=3, stride=3)
    return [host, q, ints, f, layers], {
        "c2kv_paged_attend_tree": dict(pages=layers.address, batch=2, **table, ptr=ptr, n_keys=keys, parent=i[0], window=0, q=q.data_ptr(),
                                       q_stride=0, turn=i[1], out=q.data_ptr(), lse=x[0]),
        "c2kv_verify_tree": dict(batch=2, ptr=ptr, vocab=1000, tokens=i[1], parent=i[0], p=x[0], p_stride=0, u=x[4], n_accepted=i[2], path=i[3],
                                 next_token=i[4]),
        "c2kv_paged_keep": dict(pages=layers.address, layers=2, batch=2, **table, ptr=ptr, start=start, path=i[5], n_accepted=i[6]),
        "c2kv_beam_select": dict(batch=2, width=2, vocab=1000, best=4, dtype=c2kv.DTYPE_F32, x=x[0], x_stride=0, norm=x[4], score=x[5],
                                 done=i[7], end_token=3, parent=i[8], token=i[9], score_out=x[6], done_out=i[10]),
        "c2kv_paged_reorder": dict(pages=layers.address, layers=2, batch=1, beams=2, **table, n_rows=keys, parent=i[1], out=i[11], out_stride=3)}


CALLS = ["c2kv_paged_attend_tree", "c2kv_verify_tree", "c2kv_paged_keep", "c2kv_beam_select", "c2kv_paged_reorder"]


class _Refused:
    def __init__(self, setup, name):
        self.c2kv, self.ctx, pg = setup
        self.keep, calls = _calls(self.c2kv, pg)
        self.name, self.a = name, calls[name]
        assert self.status() == self.c2kv.OK

    def status(self, **change):
        s = getattr(self.c2kv._lib, self.name)(self.ctx, *dict(self.a, **change).values())
        assert s == self.c2kv.OK or self.c2kv.c2kv_last_error(self.ctx)
        return s

    def __call__(self, status=None, **change):
        assert self.status(**change) == (self.c2kv.ERR_ARG if status is None else status), change


OPTIONAL = {"c2kv_paged_attend_tree": ["turn", "lse"], "c2kv_verify_tree": [], "c2kv_paged_keep": [], "c2kv_beam_select": ["norm", "done", "done_out"],
            "c2kv_paged_reorder": []}
HOST = ["pages", "ptr", "n_keys", "start", "n_rows"]


@pytest.mark.parametrize("name", CALLS)
def test_pointers(setup, name):
    """No pointer, one into the middle of a value, host memory where the GPU reads."""
    refused = _Refused(setup, name)
    assert getattr(refused.c2kv._lib, name)(None, *refused.a.values()) == refused.c2kv.ERR_ARG
    memory = torch.zeros(4096)
    for key, value in refused.a.items():
        if not isinstance(value, int) or value < 1 << 20:
            continue
        if key in OPTIONAL[name]:
            assert refused.status(**{key: None}) == refused.c2kv.OK
        else:
            refused(**{key: None})
        if key not in HOST:
            refused(**{key: value + 2})
            refused(**{key: memory.data_ptr()})


@pytest.mark.parametrize("name", CALLS)
def test_sizes(setup, name):
    refused = _Refused(setup, name)
    c2kv = refused.c2kv
    bad = {"batch": [0, -1], "beams": [0, -1, 65], "width": [0, -1] + [65] * (name == "c2kv_beam_select"), "stride": [2], "layers": [0, -1], "vocab": [0, -1, (1 << 19) + 1], "best": [0, 65], "p_stride": [999],
           "x_stride": [999, -1], "q_stride": [64, 1028], "window": [-1], "out_stride": [2], "end_token": [-2, -1, 1000]}
    for key, values in bad.items():
        for value in values if key in refused.a else []:
            refused(**{key: value})
    if "dtype" in refused.a:
        refused(c2kv.ERR_DTYPE, dtype=2)
        assert refused.status(end_token=-1, done=None) == c2kv.OK
    if "ptr" in refused.a:
        for x in ([1, 3, 4], [0, 3, 2]):
            x = np.array(x, np.int32)
            refused(ptr=x.ctypes.data)
        most, rows = np.array([0, 513, 514], np.int32), np.array([2000, 2000], np.int32)
        refused(c2kv.ERR_UNSUPPORTED, **dict(ptr=most.ctypes.data, **({"width": 200, "stride": 200} if "table" in refused.a else {}),
                                             **({"n_keys": rows.ctypes.data} if "n_keys" in refused.a else {})))
    for key in ("n_keys", "start", "n_rows"):
        if key in refused.a:
            for x in ([50, 20], [-1, 20]) if key != "start" else ([46, 6], [-1, 6]):
                x = np.array(x, np.int32)
                refused(**{key: x.ctypes.data})
    if name == "c2kv_paged_attend_tree":
        few = np.array([2, 20], np.int32)                    # fewer rows than nodes
        refused(n_keys=few.ctypes.data)


@pytest.mark.parametrize("name", ["c2kv_paged_keep", "c2kv_paged_reorder"])
def test_layers(setup, name):
    """Every layer's pages are looked at, and have to be alike."""
    refused = _Refused(setup, name)
    c2kv = refused.c2kv
    p = refused.keep[-1].array[1]
    for field, value, status in (("page_size", 24, c2kv.ERR_ARG), ("page_size", 32, c2kv.ERR_ARG), ("n_pages", 0, c2kv.ERR_ARG), ("n_pages", 2, c2kv.ERR_ARG),
                                 ("format", 2, c2kv.ERR_DTYPE), ("format", 0, c2kv.ERR_ARG), ("page_stride", 4096, c2kv.ERR_ARG),
                                 ("scale_stride", 64, c2kv.ERR_ARG), ("k", 0, c2kv.ERR_ARG), ("v", p.v + 8, c2kv.ERR_ARG), ("k_scale", 0, c2kv.ERR_ARG),
                                 ("v", torch.zeros(64).data_ptr(), c2kv.ERR_ARG)):
        old = getattr(p, field)
        setattr(p, field, value)
        refused(status)
        setattr(p, field, old)
    assert refused.status() == c2kv.OK


def test_a_new_table_over_the_old_one(setup):
    refused = _Refused(setup, "c2kv_paged_reorder")
    for off in (0, 4, 20, -20):
        refused(out=refused.a["table"] + off)


def test_nothing_to_do(setup):
    """No node at all: nothing is enqueued and no tensor needed."""
    refused = _Refused(setup, "c2kv_paged_keep")
    none, zero = np.zeros(3, np.int32), np.zeros(2, np.int32)
    assert refused.status(ptr=none.ctypes.data, path=None, n_accepted=None) == refused.c2kv.OK
    refused = _Refused(setup, "c2kv_paged_attend_tree")
    assert refused.status(ptr=none.ctypes.data, n_keys=zero.ctypes.data, q=None, out=None, parent=None, turn=None, lse=None) == refused.c2kv.OK
    refused = _Refused(setup, "c2kv_verify_tree")
    assert refused.status(ptr=none.ctypes.data, tokens=None, parent=None, p=None, u=None, path=None) == refused.c2kv.OK
    assert refused.keep[2][4, :2].tolist() == [-1, -1] and refused.keep[2][2, :2].tolist() == [0, 0]
