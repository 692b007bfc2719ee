"""Plain 64-bit forms of the operators over a paged KV cache (CPU), and caches
to test them on.

Tolerances.  The kernels hold logits, softmax statistics and outputs in fp32; D
products of a logit and n terms of a sum are each rounded to 2^-24 of their
size, and sums of rows that cancel are measured against the largest value of a
row of V, to which an output is a weighted mean:
* fp32 out: a logit scale <q, k> of D products is off by about sqrt(D) 2^-24 of
  scale |q| |k| (about sqrt(D)), 7.6e-6 at D = 128; weights are off by that
  relatively, in both directions, so their mean of V is within 1e-5 max |V|.
* bf16 out: half a step of bf16 is 2^-8 of the value (8 significant bits).  P is
  rounded once, so every weight p_j is off by 2^-8 p_j and their mean of V by
  sum_j 2^-8 p_j |v_j| <= 2^-8 max |V| (the sum that divides it is not rounded); the
  result is rounded once, by 2^-8 |out| <= 2^-8 max |V|: together 2^-7 max |V|.
* lse: 1e-5 (fp32) and 1e-4 (bf16: the same fp32 arithmetic on products that are
  exact in fp32; the wider bound covers longer sums), as for the dense cache.
* weights: relative to the row's own weight, the logit's error: 4e-5, over a floor
  of 1e-7 of a whole token's weight.
"""
from __future__ import annotations

import math

import numpy as np
import torch

from paper_2608_04771_amd import binding as B

OUT_TOL = {torch.float32: 1e-5, torch.bfloat16: 2.0 ** -7}
LSE_TOL = {torch.float32: 1e-5, torch.bfloat16: 1e-4}


class Paged:
    """A paged cache on the CPU: shuffled pages, NaN in every row that holds none of
    a unit's rows and ids that would be out of the pool where none may be read.
    spare: rows that calls will append (their pages are listed)."""

    def __init__(self, lens, page, D, dtype, spare=0, seed=0, weights=False, extra_pages=0):
        lens = np.asarray(lens, dtype=np.int64)
        self.lens, self.page, self.D = lens, page, D
        NL, Bs, H = lens.shape
        g = torch.Generator().manual_seed(seed)
        rng = np.random.RandomState(seed)
        need = -(-(lens + spare) // page)
        self.max_pages = max(1, int(need.max())) + extra_pages
        n_pages = int(need.sum()) + 3
        order = rng.permutation(n_pages)[:int(need.sum())]
        junk = np.array([-1, n_pages, 2 ** 31 - 1, -2 ** 31])
        table = junk[rng.randint(0, 4, (NL, Bs, H, self.max_pages))]
        at = 0
        for u in np.ndindex(NL, Bs, H):
            table[u][:need[u]] = order[at:at + need[u]]
            at += need[u]
        self.k, self.v = (torch.full((n_pages, page, D), float("nan"), dtype=dtype) for _ in "kv")
        self.pages = torch.from_numpy(table.astype(np.int32))
        self.length = torch.from_numpy(lens.astype(np.int32))
        self.weight = None
        if weights:
            self.weight = torch.full((NL, Bs, H, self.max_pages * page), float("nan"))
        for u in np.ndindex(NL, Bs, H):
            n = int(lens[u])
            self.put(u, 0, torch.randn((n, D), generator=g).to(dtype), torch.randn((n, D), generator=g).to(dtype))
            if weights:
                self.weight[u][:n] = torch.exp(torch.randn(n, generator=g))

    def where(self, u, rows):
        rows = torch.as_tensor(rows, dtype=torch.int64)
        return self.pages[u][rows // self.page].long(), rows % self.page

    def put(self, u, first, k, v):
        at = self.where(u, torch.arange(first, first + k.shape[0]))
        self.k[at], self.v[at] = k, v

    def rows(self, u, n=None):
        """K and V rows of a unit, in the cache's type."""
        at = self.where(u, torch.arange(int(self.lens[u]) if n is None else n))
        return self.k[at], self.v[at]

    def upload(self):
        return B.PagedKVCache(self.k.cuda(), self.v.cuda(), self.pages.cuda(), self.length.cuda(),
                              None if self.weight is None else self.weight.cuda())

    def download(self, cache):
        """This cache with what the GPU one holds now."""
        self.k, self.v, self.length = cache.k.cpu(), cache.v.cpu(), cache.length.cpu()
        self.lens = self.length.numpy().astype(np.int64)
        if self.weight is not None:
            self.weight = cache.weight.cpu()
        return self


def sees(n_rows, pos, sinks, window):
    """Which of n_rows rows the token at row pos sees."""
    j = torch.arange(n_rows)
    ok = j <= pos
    if window:
        ok &= (j < sinks) | (j > pos - window)
    return ok


def attend(k, v, q, pos, scale, sinks=0, window=0):
    """Queries q [G][D] of the token at row pos over rows k, v [n][D], in 64 bits, on
    the seen rows alone: out [G][D], lse [G], probabilities summed over G [n]."""
    ok = sees(k.shape[0], pos, sinks, window)
    k, v, q = k[ok].double(), v[ok].double(), q.double()
    w = torch.zeros(ok.shape[0], dtype=torch.float64)
    if not ok.any():
        return torch.zeros_like(q), torch.full((q.shape[0],), -math.inf, dtype=torch.float64), w
    x = (q @ k.T) * scale
    lse = torch.logsumexp(x, -1)
    p = torch.exp(x - lse[:, None])
    w[ok] = p.sum(0)
    return p @ v, lse, w


def close_out(got, ref, v, dtype, what):
    """out rows within the tolerance of the largest finite |V|."""
    top = v.double().nan_to_num(0.0, 0.0, 0.0).abs().max().item() if v.numel() else 1.0
    err = (got.double() - ref).abs().max().item() if ref.numel() else 0.0
    assert err <= OUT_TOL[dtype] * top, f"{what}: out off by {err:.3e}, allowed {OUT_TOL[dtype] * top:.3e}"


def close_lse(got, ref, dtype, what):
    fin = torch.isfinite(ref)
    assert torch.equal(torch.isfinite(got), fin), f"{what}: lse finiteness differs"
    err = (got.double() - ref)[fin].abs().max().item() if fin.any() else 0.0
    assert err <= LSE_TOL[dtype], f"{what}: lse off by {err:.3e}"


def close_weight(got, ref, what):
    err = ((got.double() - ref).abs() / (ref.abs() + 2.5e-3)).max().item() if ref.numel() else 0.0
    assert err <= 4e-5, f"{what}: weight off by {err:.3e}"
