"""Paged caches for the tests: pages in random order with NaN wherever no row was written, and the
64-bit rows that they stand for."""
import numpy as np
import torch

from oracle import paged_oracle as orc

E4M3 = torch.float8_e4m3fn
TDT = {"bf16": torch.bfloat16, "f32": torch.float32}


def lib():
    import __graft_entry__ as g
    g.build()
    from paper_2607_17715_gb300 import c2kv
    return c2kv


def context(dtype, hq, hkv, d, theta=1.0e4, stream=None):
    c2kv = lib()
    return c2kv.c2kv_create(1, hq, hkv, d, theta, c2kv.DTYPE_F32 if dtype == "f32" else c2kv.DTYPE_BF16, 1,
                            stream=stream or torch.cuda.current_stream())


class Paged:
    """Pages for requests of the given rows, and a table with -1 past each request's pages."""

    def __init__(self, rng, dtype, fmt, hkv, d, size, rows, spare=3, fill=float("nan"), width=None):
        self.dtype, self.fmt, self.hkv, self.d, self.size, self.rows = dtype, fmt, hkv, d, size, list(rows)
        count = [-(-r // size) for r in rows]
        n = sum(count) + spare
        order = rng.permutation(n)
        self.table_np = np.full((len(rows), width or max(1, max(count))), -1, np.int32)
        at = 0
        for r, m in enumerate(count):
            self.table_np[r, :m] = order[at:at + m]
            at += m
        shape = (n, hkv, size, d)
        dt = E4M3 if fmt == "e4m3" else TDT[dtype]
        self.k = torch.full(shape, fill, device="cuda").to(dt)
        self.v = self.k.clone()
        self.ks = torch.full(shape[:3], fill, device="cuda") if fmt == "e4m3" else None
        self.vs = self.ks.clone() if fmt == "e4m3" else None
        self.table = torch.from_numpy(self.table_np).cuda()

    def pages(self):
        return lib().make_pages(self.k, self.v, self.ks, self.vs)

    def host(self):
        """(K, V) pages as fp64 values."""
        got = []
        for x, s in ((self.k, self.ks), (self.v, self.vs)):
            y = x.float().cpu().numpy().astype(np.float64)
            got.append(y if s is None else y * s.cpu().numpy().astype(np.float64)[..., None])
        return got

    def fill_rows(self, rng, scale=1.0):
        """Random rows in every request's pages, written by torch; returns nothing (see dense)."""
        for r, n in enumerate(self.rows):
            for j0 in range(0, n, self.size):
                m = min(self.size, n - j0)
                pg = int(self.table_np[r, j0 // self.size])
                for x, s in ((self.k, self.ks), (self.v, self.vs)):
                    y = rng.standard_normal((self.hkv, m, self.d)) * scale
                    if s is None:
                        x[pg, :, :m] = torch.from_numpy(y).to(x.dtype).cuda()
                    else:
                        code, sc = orc.quantised(y)
                        x.view(torch.uint8)[pg, :, :m] = torch.from_numpy(code).float().to(E4M3).view(torch.uint8).cuda()
                        s[pg, :, :m] = torch.from_numpy(sc).float().cuda()

    def dense(self, r, n=None):
        """fp64 rows 0 .. n of request r: K, V [n, Hkv, d]."""
        k, v = self.host()
        n = self.rows[r] if n is None else n
        return orc.rows_of(k, self.table_np, r, 0, n, self.size), orc.rows_of(v, self.table_np, r, 0, n, self.size)
