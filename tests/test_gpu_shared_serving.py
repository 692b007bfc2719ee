"""Samples of one prompt as a serving loop has them: rows rotated and appended, pages forked,
tokens attended over the prompt's rows once for all samples."""
import math

import numpy as np
import pytest
import torch

from paged_bounds import Expected
from paged_helpers import attend, close_lse, close_out
from paper_2608_04771_amd import binding as B
from rope_helpers import close_rows, frequencies, turned

pytestmark = pytest.mark.gpu

F32, BF = torch.float32, torch.bfloat16


@pytest.mark.parametrize("captured", [False, True])
@pytest.mark.parametrize("dtype,D,G,sinks,window", [(BF, 128, 4, 0, 0), (F32, 64, 7, 2, 60), (BF, 64, 2, 4, 33)])
def test_samples_of_prompts(dtype, D, G, sinks, window, captured):
    NL, H, page, steps = 2, 2, 16, 5
    prompts, samples = [75, 64, 9], [4, 1, 3]              # rows, and sequences that go on from them
    Bs, most = sum(samples), 128 // page
    first = np.concatenate([[0], np.cumsum(samples)])
    group = np.repeat(np.arange(3), samples)
    g = torch.Generator().manual_seed(D)
    freq = frequencies(D)
    rope = B.Rope(freq.cuda())
    n_pages = NL * Bs * H * most
    pools = [torch.full((n_pages, page, D), float("nan"), dtype=dtype, device="cuda") for _ in "kv"]
    table = torch.from_numpy(np.random.RandomState(1).permutation(n_pages).astype(np.int32)).view(NL, Bs, H, most).cuda()
    err = torch.zeros(1, dtype=torch.int32, device="cuda")

    # the prompts' rows: each in its group's first sequence, through a cache of those sequences
    leads = torch.from_numpy(first[:-1].copy()).cuda()
    T = max(prompts)
    fused = torch.randn((NL, 3, T, 2 * H, D), generator=g).to(dtype)
    lead = B.PagedKVCache(*pools, table[:, leads].contiguous(), torch.zeros((NL, 3, H), dtype=torch.int32, device="cuda"))
    n = torch.tensor(prompts, dtype=torch.int32).cuda()
    dev = fused.cuda().transpose(2, 3)
    pos = torch.arange(T, dtype=torch.int32).expand(3, T).contiguous()
    B.reco_paged_append(lead, dev[:, :, :H], dev[:, :, H:], rope, pos.cuda(), n_new=n, dev_err=err)
    assert torch.equal(lead.length.cpu(), n.cpu()[None, :, None].expand(NL, 3, H))
    want, off = turned(fused.transpose(2, 3), pos[None], freq)
    K, V = {}, {}
    for u in np.ndindex(NL, Bs, H):
        p = group[u[1]]
        at = table[u[0], first[p], u[2]].cpu()[torch.arange(prompts[p]) // page].long()
        K[u], V[u] = (x.cpu()[at, torch.arange(prompts[p]) % page] for x in pools)
        close_rows(K[u], want[u[0], p, u[2], :prompts[p]], off[u[0], p, u[2], :prompts[p]], f"prompt {p}")
        assert torch.equal(V[u], fused[u[0], p, :prompts[p], H + u[2]])

    # the fork: whole pages are the first sequence's, a page in part is copied
    for b in range(Bs):
        p = group[b]
        kept = prompts[p] // page
        if b != first[p] and prompts[p] % page:
            for pool in pools:
                pool[table[:, b, :, kept].long()] = pool[table[:, first[p], :, kept].long()]
        table[:, b, :, :kept] = table[:, first[p], :, :kept]
    length = torch.tensor([prompts[p] for p in group], dtype=torch.int32).cuda()[None, :, None].expand(NL, Bs, H).contiguous()
    cache = B.PagedKVCache(*pools, table, length)
    at = torch.tensor([prompts[p] for p in group], dtype=torch.int32).cuda()
    x = torch.zeros((NL, Bs, H * (G + 2), D), dtype=dtype, device="cuda")
    q, kn, vn = x[:, :, :H * G], x[:, :, H * G:H * (G + 1)], x[:, :, H * (G + 1):]
    qo = torch.zeros((NL, Bs, H * G, D), dtype=dtype, device="cuda")
    append = B.PreparedPagedAppend(cache, None, rope, at, qo, dev_err=err)
    ws = B.paged_shared_decode_workspace(cache, H * G, 3)
    out, lse = torch.zeros_like(qo), torch.zeros((NL, Bs, H * G), device="cuda")
    decode = B.PreparedPagedSharedDecode(cache, H * G, torch.from_numpy(first.astype(np.int32)).cuda(), n, out, lse, ws, err, sinks, window)

    def token():
        append(kn, vn, q)
        decode(qo)
        at.add_(1)

    graph = None
    if captured:
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            token()
    scale = 1 / math.sqrt(D)
    for i in range(steps):
        x.copy_(torch.randn(x.shape, generator=g).to(dtype))
        graph.replay() if captured else token()
        torch.cuda.synchronize()
        assert err.item() == 0 and torch.equal(length.cpu(), at.cpu()[None, :, None].expand(NL, Bs, H))
        new = x.cpu()
        want, off = turned(new[:, :, :, None], (at - 1).cpu()[None, :, None], freq)
        close_rows(qo.cpu(), want[:, :, :H * G, 0], off[:, :, :H * G, 0], "queries")
        for u in K:
            L = int(length[u]) - 1
            page_of = int(table[u][L // page])
            k, v = (p[page_of, L % page].cpu()[None] for p in pools)
            j = H * G + u[2]
            close_rows(k[0], want[u[0], u[1], j, 0], off[u[0], u[1], j, 0], "key")
            assert torch.equal(v[0], new[u[0], u[1], j + H])
            K[u], V[u] = torch.cat([K[u], k]), torch.cat([V[u], v])
            heads = slice(u[2] * G, (u[2] + 1) * G)
            got, z, query = out[u[:2]][heads].cpu(), lse[u[:2]][heads].cpu(), qo[u[:2]][heads].cpu()
            what = f"token {i} of {u}"
            if dtype == BF:
                e = Expected(K[u], V[u], query, L, scale, sinks, window)
                e.check(got, what)
                close_lse(z, e.lse, dtype, what)
            else:
                o, ref, _ = attend(K[u], V[u], query, L, scale, sinks, window)
                close_out(got, o, V[u], dtype, what)
                close_lse(z, ref, dtype, what)
