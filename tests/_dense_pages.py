"""Paged caches made on the GPU from dense rows, with the 64-bit rows that they stand for, and attention of trees over
those in 64 bits."""
import numpy as np
import torch

from oracle import branch_oracle as brc
from oracle import paged_oracle as orc
from tests import _paged_helpers as P


class Rows:
    """k, v: [rows, Hkv, d] of each request.  Pages in random order, NaN where no row was written."""

    def __init__(self, dtype, fmt, k, v, size, seed=0):
        hkv, d = k[0].shape[1:]
        count = [-(-len(x) // size) for x in k]
        order = torch.from_numpy(np.random.default_rng(seed).permutation(sum(count) + 2)).cuda()
        self.table = torch.full((len(k), max(count + [1])), -1, dtype=torch.int32, device="cuda")
        at = 0
        for r, m in enumerate(count):
            self.table[r, :m] = order[at:at + m]
            at += m
        self.held = []
        for rows in (k, v):
            scale = torch.full((len(order), hkv, size), float("nan"), device="cuda") if fmt == "e4m3" else None
            pages = torch.full((len(order), hkv, size, d), float("nan"), device="cuda").to(P.E4M3 if fmt == "e4m3" else P.TDT[dtype])
            raw = pages.view(torch.uint8) if fmt == "e4m3" else pages
            stand = []
            for r, x in enumerate(rows):
                j = torch.arange(len(x), device="cuda")
                page, row = self.table[r, j // size].long(), j % size
                if fmt == "e4m3":
                    s = x.abs().amax(-1).float() / 448
                    code = (x / torch.where(s > 0, s, 1.0)[..., None]).float().to(P.E4M3)
                    raw[page, :, row] = code.view(torch.uint8)
                    scale[page, :, row] = s
                    stand.append(code.double() * s.double()[..., None])
                else:
                    y = x.to(P.TDT[dtype])
                    raw[page, :, row] = y
                    stand.append(y.double())
            self.held.append((pages, scale, stand))
        self.k, self.v = (h[2] for h in self.held)

    def pages(self):
        (k, ks, _), (v, vs, _) = self.held
        return P.lib().make_pages(k, v, ks, vs)


def attend_tree(q, k, v, parent, window=0):
    """q [n, Hq, d] (turned), k, v [rows, Hkv, d], all 64-bit: out [n, Hq, d], lse [Hq, n]."""
    n, hq, d = q.shape
    g = hq // k.shape[1]
    seen = torch.from_numpy(brc.sees(parent, len(k), window)).cuda()
    out, lse = torch.empty_like(q), torch.empty((hq, n), dtype=q.dtype, device="cuda")
    for h in range(hq):
        s = (q[:, h] @ k[:, h // g].T / d ** 0.5).masked_fill(~seen, -float("inf"))
        m = s.amax(-1, keepdim=True)
        w = (s - m).exp()
        total = w.sum(-1, keepdim=True)
        out[:, h], lse[h] = w @ v[:, h // g] / total, (m + total.log())[:, 0]
    return out, lse


def relative(out, want):
    return ((out.double() - want).norm(dim=-1) / want.norm(dim=-1)).max().item()


class Call:
    """One call of c2kv_paged_attend_tree over `rows`, trees [r] of request r, made `times` times: out (of each), lse."""

    def __init__(self, dtype, hq, hkv, d, rows, trees, q, pos=None, theta=1.0e4, window=0, times=1):
        self.rows, self.trees, self.q, self.pos, self.theta, self.window = rows, trees, q, pos, theta, window
        c2kv, ctx = P.lib(), P.context(dtype, hq, hkv, d, theta)
        try:
            self.ptr = np.cumsum([0] + [len(t) for t in trees]).tolist()
            parent = torch.tensor(sum(trees, []), dtype=torch.int32, device="cuda")
            self.outs = []
            for _ in range(times):
                out, self.lse = torch.full_like(q, 7.0), torch.full((hq, self.ptr[-1]), 7.0, device="cuda")
                c2kv.c2kv_paged_attend_tree(ctx, rows.pages(), rows.table, self.ptr, [len(k) for k in rows.k], parent, q, out, lse=self.lse,
                                            turn=pos, window=window)
                self.outs.append(out)
            c2kv.c2kv_sync(ctx)
        finally:
            c2kv.c2kv_destroy(ctx)
        self.out = self.outs[0]

    def want(self):
        q = self.q.double()
        if self.pos is not None:
            q = torch.from_numpy(orc.turned(q.cpu().numpy(), self.pos.cpu().numpy(), self.theta)).cuda()
        got = [attend_tree(q[self.ptr[r]:self.ptr[r + 1]], self.rows.k[r], self.rows.v[r], t, self.window) for r, t in enumerate(self.trees)]
        return torch.cat([o for o, _ in got]), torch.cat([ls for _, ls in got], 1)
