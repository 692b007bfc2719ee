"""bf16 attention over a paged cache against bounds that follow every output (paged_bounds):
long caches and runs, where each output is a small mean of many rows of V."""
import math

import numpy as np
import pytest
import torch

from paged_bounds import Expected
from paged_helpers import Paged, close_lse
from paper_2608_04771_amd import binding as B

pytestmark = pytest.mark.gpu

BF = torch.bfloat16


def _randn(seed, *shape):
    return torch.randn(shape, generator=torch.Generator().manual_seed(seed)).to(BF)


@pytest.mark.parametrize("D,G", [(128, 7), (64, 16), (128, 1), (64, 5)])
@pytest.mark.parametrize("lens,sinks,window", [
    ([[[1, 2], [33, 1000]]], 0, 0),                       # short ones
    ([[[9677, 20001], [4096, 12000]]], 0, 0),             # few long units: many splits
    ([[[9677, 20001], [4096, 12000]]], 4, 4096),
    ([[[16383]]], 0, 0),
])
@pytest.mark.parametrize("weights", [False, True])
def test_decode(D, G, lens, sinks, window, weights):
    p = Paged(lens, 16, D, BF, spare=1, seed=D + G, weights=weights)
    _decode(p, G, sinks, window)


@pytest.mark.parametrize("D,G", [(128, 7), (64, 4)])
@pytest.mark.parametrize("weights", [False, True])
def test_decode_of_more_units_than_compute_units(D, G, weights):
    lens = np.random.RandomState(3).randint(50, 300, (1, 130, 2))
    lens[0, 0] = [3000, 2999]
    _decode(Paged(lens, 32, D, BF, spare=1, seed=5, weights=weights), G, 0, 0)


def _decode(p, G, sinks, window):
    NL, Bs, H = p.lens.shape
    q, kn, vn = _randn(1, NL, Bs, H * G, p.D), _randn(2, NL, Bs, H, p.D), _randn(3, NL, Bs, H, p.D)
    out, lse = B.reco_paged_decode_attn(p.upload(), q.cuda(), kn.cuda(), vn.cuda(), sinks, window)
    out, lse = out.cpu(), lse.cpu()
    for u in np.ndindex(NL, Bs, H):
        k, v = p.rows(u)
        k, v = torch.cat([k, kn[u][None]]), torch.cat([v, vn[u][None]])
        hs = slice(u[2] * G, (u[2] + 1) * G)
        e = Expected(k, v, q[u[:2]][hs], k.shape[0] - 1, 1 / math.sqrt(p.D), sinks, window)
        e.check(out[u[:2]][hs], f"unit {u}")
        close_lse(lse[u[:2]][hs], e.lse, BF, f"unit {u}")


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("lens,G,T,sinks,window", [
    ([[[0, 5], [40, 1000]]], 4, 100, 0, 0),               # short ones
    ([[[9645, 9645]]], 7, 32, 0, 0),                      # the probe: splits over keys
    ([[[16001, 20000]]], 5, 9, 4, 12000),
    ([[[0, 0]]], 7, 4500, 0, 0),                          # a long prompt
    ([[[3000, 1500], [100, 4097]]], 4, 2100, 0, 0),       # chunks
    ([[[2500, 0, 900, 7]] * 2], 8, 2600, 4, 1500),        # in a window
    ([[[0] * 8] * 8], 4, 1100, 0, 0),                     # many blocks
    ([[[0] * 8] * 4], 4, 2048, 0, 0),                     # of 256 rows
    ([[[500] * 8] * 8], 4, 1600, 4, 1500),                # of 256 rows, in a window
])
def test_prefill(D, lens, G, T, sinks, window):
    p = Paged(lens, 64, D, BF, spare=T, seed=D + T)
    NL, Bs, H = p.lens.shape
    q, kn, vn = _randn(1, NL, Bs, H * G, T, D), _randn(2, NL, Bs, H, T, D), _randn(3, NL, Bs, H, T, D)
    out, lse = B.reco_paged_prefill_attn(p.upload(), q.cuda(), kn.cuda(), vn.cuda(), sinks=sinks, window=window)
    out, lse = out.cpu(), lse.cpu()
    # the first and last tokens, those around tiles' ends, and some between
    near = {t for a in (0, 32, 64, 128, T // 2 // 64 * 64, T) for t in (a - 1, a, a + 1) if 0 <= t < T}
    some = np.random.RandomState(T).randint(0, T, 1 if Bs * H > 8 else 12)
    for u in np.ndindex(NL, Bs, H):
        k, v = p.rows(u)
        L = k.shape[0]
        k, v = torch.cat([k, kn[u]]), torch.cat([v, vn[u]])
        hs = slice(u[2] * G, (u[2] + 1) * G)
        for t in sorted(near | set(some.tolist())):
            n = L + t + 1
            e = Expected(k[:n], v[:n], q[u[:2]][hs][:, t], n - 1, 1 / math.sqrt(D), sinks, window)
            e.check(out[u[:2]][hs][:, t], f"unit {u} token {t}")
            close_lse(lse[u[:2]][hs][:, t], e.lse, BF, f"unit {u} token {t}")
