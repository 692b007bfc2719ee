"""Paged caches (CPU) whose sequences share their first rows, and the attention of one new
token over them in 64 bits, checked by the element-wise bounds of attention's bf16 outputs or
by the tolerances of fp32 ones."""
from __future__ import annotations

import math

import numpy as np
import torch

from paged_bounds import Expected
from paged_helpers import Paged, attend, close_lse, close_out
from paper_2608_04771_amd import binding as B


class SharedPaged(Paged):
    """first [groups + 1], shared [groups] or [NL][groups]: of a group's units all but the first
    sequence's lose their shared rows, whose whole pages are not listed any more."""

    def __init__(self, lens, first, shared, page, D, dtype, spare=1, seed=0, extra_pages=0):
        super().__init__(lens, page, D, dtype, spare=spare, seed=seed, extra_pages=extra_pages)
        NL, Bs, H = self.lens.shape
        self.first = np.asarray(first)
        self.shared = np.broadcast_to(np.asarray(shared), (NL, len(first) - 1))
        self.group = np.searchsorted(self.first[1:], np.arange(Bs), side="right")
        junk = np.array([-1, self.k.shape[0], 2 ** 31 - 1, -2 ** 31])
        for u in np.ndindex(NL, Bs, H):
            g = self.group[u[1]]
            P, lead = int(self.shared[u[0], g]), int(self.first[g])
            if u[1] == lead or P == 0:
                continue
            kept = P // page                               # whole pages of shared rows
            rows = torch.arange(P)
            at = self.where(u, rows[rows // page == kept])
            if P > kept * page and int(lens[u]) + spare > kept * page:
                self.k[at], self.v[at] = float("nan"), float("nan")
            self.pages[u][:kept] = torch.from_numpy(junk[(np.arange(kept) + u[1]) % 4].astype(np.int32))

    def seen_rows(self, u):
        """K and V rows that unit u sees, its group's first."""
        g = self.group[u[1]]
        P, lead = int(self.shared[u[0], g]), (u[0], int(self.first[g]), u[2])
        n = int(self.lens[u])
        shared, own = self.where(lead, torch.arange(P)), self.where(u, torch.arange(P, n))
        return tuple(torch.cat([x[shared], x[own]]) for x in (self.k, self.v))

    def groups(self):
        s = self.shared if (self.shared != self.shared[:1]).any() else self.shared[0]
        return (torch.tensor(self.first, dtype=torch.int32).cuda(), torch.tensor(np.array(s), dtype=torch.int32).cuda())


def check_attention(c, q, kn, vn, out, lse, sinks=0, window=0, scale=None, units=None, what=""):
    """out, lse of the token of every unit (or of `units`) against the 64-bit form."""
    NL, Bs, H = c.lens.shape
    G = q.shape[2] // H
    scale = 1 / math.sqrt(c.D) if scale is None else scale
    for u in units or np.ndindex(NL, Bs, H):
        k, v = c.seen_rows(u)
        if kn is not None:
            k, v = torch.cat([k, kn[u][None]]), torch.cat([v, vn[u][None]])
        heads = slice(u[2] * G, (u[2] + 1) * G)
        got, z, n = out[u[:2]][heads], lse[u[:2]][heads], k.shape[0]
        name = f"{what} unit {u}"
        if c.dtype_ == torch.bfloat16 and n:
            e = Expected(k, v, q[u[:2]][heads], n - 1, scale, sinks, window)
            e.check(got, name)
            close_lse(z, e.lse, c.dtype_, name)
        else:
            o, ref, _ = attend(k, v, q[u[:2]][heads], n - 1, scale, sinks, window)
            close_out(got, o, v, c.dtype_, name)
            close_lse(z, ref, c.dtype_, name)


def make(lens, first, shared, page, D, dtype, G, append=True, seed=0, spare=None, **kw):
    """A cache, its groups' tensors, and a token's rows."""
    lens = np.asarray(lens)
    c = SharedPaged(lens, first, shared, page, D, dtype, spare=int(append) if spare is None else spare, seed=seed, **kw)
    c.dtype_ = dtype
    NL, Bs, H = lens.shape
    g = torch.Generator().manual_seed(seed + 1)
    q = torch.randn((NL, Bs, H * G, D), generator=g).to(dtype)
    kn, vn = (torch.randn((NL, Bs, H, D), generator=g).to(dtype) if append else None for _ in "kv")
    return c, q, kn, vn


def call(c, cache, q, kn, vn, err=None, **kw):
    first, shared = c.groups()
    out, lse = B.reco_paged_shared_decode_attn(cache, q.cuda(), first, shared, None if kn is None else kn.cuda(),
                                               None if vn is None else vn.cuda(), dev_err=err, **kw)
    return out.cpu(), lse.cpu()


def check_append(c, cache, kn, vn, what=""):
    """Every unit has the new row behind its others, and the others as they were."""
    n = cache.length.cpu()
    k, v = c.k.clone(), c.v.clone()
    for u in np.ndindex(c.lens.shape):
        L = int(c.lens[u])
        assert n[u] == L + (kn is not None), f"{what}: length of {u}"
        if kn is not None:
            at = c.where(u, [L])
            k[at], v[at] = kn[u][None], vn[u][None]
    bits = torch.int16 if k.dtype == torch.bfloat16 else torch.int32
    assert torch.equal(cache.k.cpu().view(bits), k.view(bits)) and torch.equal(cache.v.cpu().view(bits), v.view(bits)), what
