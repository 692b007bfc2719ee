"""Shared attention where a workgroup's common rows and a wave's own ones are many, so that
page ids of rows further on are looked up on the way: against the 64-bit form."""
import numpy as np
import pytest
import torch

from paper_2608_04771_amd import binding as B
from shared_helpers import check_attention
from shared_long_cases import COMMON, HEADS, LAYERS, OWN

pytestmark = pytest.mark.gpu


class LongPaged:
    """A cache on the GPU of one group: its first sequence's pages hold the shared rows, whose
    whole pages the others do not list."""

    def __init__(self, case, seed):
        dtype, D, G, page, P, own, _ = case
        self.dtype_, self.D, self.page, self.P = (torch.bfloat16 if dtype == "bf16" else torch.float32), D, page, P
        self.lens = np.zeros((LAYERS, len(own), HEADS), dtype=np.int64) + P + np.asarray(own)[None, :, None]
        most = -(-(P + max(own) + 1) // page)
        at = np.arange(most)
        need = -(-(self.lens + 1) // page)[..., None]
        first = np.arange(len(own))[None, :, None, None] == 0
        has = (at < need) & (first | (at >= P // page))
        rng = np.random.RandomState(seed)
        n = int(has.sum())
        pages = np.where(at % 2 == 0, -1, 2 ** 31 - 1) * np.ones(has.shape, dtype=np.int64)
        pages[has] = rng.permutation(n)
        self.pages = torch.from_numpy(pages.astype(np.int32))
        g = torch.Generator(device="cuda").manual_seed(seed)
        self.k, self.v = (torch.randn((n, page, D), generator=g, device="cuda").to(self.dtype_) for _ in "kv")
        self.length = torch.from_numpy(self.lens.astype(np.int32))

    def seen_rows(self, u):
        rows = torch.arange(int(self.lens[u]))
        ids = torch.where(rows < self.P, self.pages[u[0], 0, u[2]][rows // self.page], self.pages[u][rows // self.page]).long().cuda()
        at = (rows % self.page).cuda()
        return self.k[ids, at].cpu(), self.v[ids, at].cpu()


@pytest.mark.parametrize("case", COMMON + OWN, ids=str)
def test_long_parts(case):
    _, D, G, page, P, own, (sinks, window) = case
    c = LongPaged(case, seed=P)
    g = torch.Generator().manual_seed(1)
    q = torch.randn((LAYERS, len(own), HEADS * G, D), generator=g).to(c.dtype_)
    kn, vn = (torch.randn((LAYERS, len(own), HEADS, D), generator=g).to(c.dtype_) for _ in "kv")
    cache = B.PagedKVCache(c.k, c.v, c.pages.cuda(), c.length.cuda())
    err = torch.zeros(1, dtype=torch.int32, device="cuda")
    first, shared = (torch.tensor(x, dtype=torch.int32).cuda() for x in ([0, len(own)], [P]))
    out, lse = B.reco_paged_shared_decode_attn(cache, q.cuda(), first, shared, kn.cuda(), vn.cuda(), sinks, window, dev_err=err)
    assert err.item() == 0 and torch.equal(cache.length.cpu(), c.length + 1)
    rng = np.random.RandomState(2)
    units = {(0, 0, 0), (LAYERS - 1, len(own) - 1, HEADS - 1)} | \
            {(rng.randint(LAYERS), b, rng.randint(HEADS)) for b in range(len(own)) for _ in range(12)}
    check_attention(c, q, kn, vn, out.cpu(), lse.cpu(), sinks, window, units=sorted(units))
    for u in sorted(units):                                # and the new row is where it belongs
        at = int(c.pages[u][int(c.lens[u]) // page]), int(c.lens[u]) % page
        assert torch.equal(c.k[at].cpu(), kn[u]) and torch.equal(c.v[at].cpu(), vn[u]), u
    # again, over the same rows: the same bits
    cache.length.copy_(c.length)
    o2, z2 = B.reco_paged_shared_decode_attn(cache, q.cuda(), first, shared, kn.cuda(), vn.cuda(), sinks, window, dev_err=err)
    assert torch.equal(o2.view(torch.uint8), out.view(torch.uint8)) and torch.equal(z2, lse)
