"""reco_paged_shared_decode_attn against the plain form in 64 bits."""
import math

import numpy as np
import pytest
import torch

from paper_2608_04771_amd import binding as B
from shared_helpers import call, check_append, check_attention, make

pytestmark = pytest.mark.gpu

F32, BF = torch.float32, torch.bfloat16
KINDS = [(BF, 128, 4, 16), (F32, 64, 7, 16), (BF, 64, 16, 32), (F32, 128, 3, 64), (BF, 128, 7, 64), (BF, 128, 1, 256)]


def _lens(P, own, H, NL=1):
    """[NL][B][H] lengths of one group's sequences, P shared rows and own ones."""
    base = P + np.asarray(own)[None, :, None] + np.zeros((NL, 1, H), dtype=np.int64)
    return base + np.arange(NL)[:, None, None] + np.arange(H)[None, None, :] % 2


@pytest.mark.parametrize("dtype,D,G,page", KINDS)
@pytest.mark.parametrize("P", [0, 1, 15, 16, 17, 33, 64, 100, 130, 700])
def test_one_group(dtype, D, G, page, P):
    own = [0, 1, 5, 31, 64, 200, 17]
    for append in (True, False):
        lens = _lens(P, own, 2)
        lens[:, 0] = P                                     # no row of its own
        c, q, kn, vn = make(lens, [0, 7], [P], page, D, dtype, G, append, seed=P)
        cache = c.upload()
        err = torch.zeros(1, dtype=torch.int32, device="cuda")
        out, lse = call(c, cache, q, kn, vn, err)
        assert err.item() == 0
        check_attention(c, q, kn, vn, out, lse, what=f"append {append}")
        check_append(c, cache, kn, vn)


@pytest.mark.parametrize("dtype,D,G,page", KINDS)
@pytest.mark.parametrize("sinks,window", [(0, 1), (0, 40), (4, 90), (70, 64), (200, 30), (3, 300), (1000, 16), (5, 5000)])
def test_windows(dtype, D, G, page, sinks, window):
    # windows that begin in the shared rows, for some sequences or all, or behind them; sinks past them
    c, q, kn, vn = make(_lens(150, [0, 3, 20, 100, 149, 331], 2, NL=2), [0, 4, 6], [[150, 150], [151, 90]], page, D, dtype, G, True, seed=window)
    cache = c.upload()
    err = torch.zeros(1, dtype=torch.int32, device="cuda")
    out, lse = call(c, cache, q, kn, vn, err, sinks=sinks, window=window)
    assert err.item() == 0
    check_attention(c, q, kn, vn, out, lse, sinks, window)
    check_append(c, cache, kn, vn)


@pytest.mark.parametrize("dtype,D,G", [(BF, 128, 4), (F32, 64, 2)])
def test_odd_values_in_rows_that_are_not_seen(dtype, D, G):
    # infinities and NaN in shared rows reach the sequences that see them alone
    sinks, window = 2, 60
    own = [0, 10, 25, 59, 58, 100]
    c, q, kn, vn = make(_lens(100, own, 1), [0, 6], [100], 16, D, dtype, G, True, seed=3)
    lead = (0, 0, 0)
    for row, x in ((5, float("nan")), (50, float("inf")), (60, float("nan")), (99, float("-inf"))):
        at = c.where(lead, [row])
        c.k[at], c.v[at] = x, x
    cache = c.upload()
    out, lse = call(c, cache, q, kn, vn, sinks=sinks, window=window)
    for b, own_rows in enumerate(own):
        n = 101 + own_rows
        seen = {j for j in (5, 50, 60, 99) if j < sinks or j >= n - window}
        if not seen:
            check_attention(c, q, kn, vn, out, lse, sinks, window, units=[(0, b, 0)], what=f"{b}")
        else:
            assert not torch.isfinite(out[0, b]).all(), f"sequence {b} sees {seen}"


@pytest.mark.parametrize("dtype,D,G", [(BF, 128, 8), (F32, 64, 3)])
def test_many_sequences_and_groups(dtype, D, G):
    # more groups than a wave has lanes, empty ones among them, and groups of many blocks of rows
    rng = np.random.RandomState(5)
    first = np.sort(np.concatenate([[0, 0, 150, 150], rng.choice(60, 75) + 1]))
    shared = rng.randint(0, 90, len(first) - 1)
    group = np.searchsorted(first[1:], np.arange(150), side="right")
    lens = (shared[group] + rng.randint(0, 70, 150))[None, :, None] + np.array([0, 3])[None, None]
    c, q, kn, vn = make(lens, first, shared, 16, D, dtype, G, True)
    cache = c.upload()
    err = torch.zeros(1, dtype=torch.int32, device="cuda")
    out, lse = call(c, cache, q, kn, vn, err)
    assert err.item() == 0
    check_attention(c, q, kn, vn, out, lse)
    check_append(c, cache, kn, vn)


def test_layers_and_scales():
    # a range of layers, shared counts of each; scales of both signs and 0
    lens = np.stack([_lens(p, [5, 40, 9], 2)[0] for p in (20, 64, 130, 33)])
    for scale in (0.05, -0.1, 0.0, None):
        c, q, kn, vn = make(lens, [0, 2, 3], [[20, 7], [64, 64], [130, 0], [33, 40]], 16, 64, BF, 5, True, seed=2)
        cache = c.upload()
        first, shared = c.groups()
        out, lse = B.reco_paged_shared_decode_attn(cache, q[1:3].contiguous().cuda(), first, shared[1:3].contiguous(),
                                                   kn[1:3].contiguous().cuda(), vn[1:3].contiguous().cuda(), scale=scale, layer0=1, n_layers=2)
        n = cache.length.cpu()
        assert torch.equal(n[[0, 3]], c.length[[0, 3]]) and torch.equal(n[1:3], c.length[1:3] + 1)
        full, z = torch.zeros_like(q), torch.zeros(q.shape[:3])
        full[1:3], z[1:3] = out.cpu(), lse.cpu()
        check_attention(c, q, kn, vn, full, z, scale=scale, units=[u for u in np.ndindex(lens.shape) if u[0] in (1, 2)], what=f"scale {scale}")


@pytest.mark.parametrize("dtype,D", [(BF, 128), (F32, 64)])
def test_nothing_to_see(dtype, D):
    c, q, _, _ = make(np.array([[[0, 3], [0, 0], [2, 0]]]), [0, 2, 3], [0, 0], 16, D, dtype, 2, False)
    out, lse = call(c, c.upload(), q, None, None)
    for u in ((0, 0, 0), (0, 1, 0), (0, 1, 1), (0, 2, 1)):
        heads = slice(2 * u[2], 2 * u[2] + 2)
        assert (out[u[:2]][heads] == 0).all() and torch.isneginf(lse[u[:2]][heads]).all()
    check_attention(c, q, None, None, out, lse, units=[(0, 0, 1), (0, 2, 0)])


def test_lists_of_groups_that_do_not_ascend():
    # count as none: every unit's rows are its own, whatever the counts say
    lens = np.array([[[40, 33], [17, 100], [60, 1], [5, 80]]])
    c, q, kn, vn = make(lens, [0, 1, 2, 3, 4], [0, 0, 0, 0], 16, 128, BF, 4, True)
    for first in ([0, 4, 3], [1, 2, 4], [0, 2, 3], [0, 2, 5], [0, -1, 4], [-2 ** 31, 2, 2 ** 31 - 1], [0, 2 ** 31 - 1, 4]):
        for sinks, window in ((0, 0), (3, 20)):
            cache = c.upload()
            err = torch.zeros(1, dtype=torch.int32, device="cuda")
            out, lse = B.reco_paged_shared_decode_attn(cache, q.cuda(), torch.tensor(first, dtype=torch.int32).cuda(),
                                                       torch.tensor([5, 1], dtype=torch.int32).cuda(), kn.cuda(), vn.cuda(), sinks, window, dev_err=err)
            assert err.item() == 10                        # RECO_DEV_BAD_GROUP
            check_attention(c, q, kn, vn, out.cpu(), lse.cpu(), sinks, window, what=str(first))
            check_append(c, cache, kn, vn)


def test_counts_and_pages_that_are_bad():
    lens = np.array([[[40, 41], [32, 60], [55, 70]]])
    err = torch.zeros(1, dtype=torch.int32, device="cuda")
    for given, used in ((33, 32), (2 ** 31 - 1, 32), (-1, 0), (-2 ** 31, 0)):      # clamped to the shortest unit's rows
        c, q, kn, vn = make(lens, [0, 3], [used], 16, 64, F32, 2, True)
        cache = c.upload()
        first, _ = c.groups()
        err.zero_()
        out, lse = B.reco_paged_shared_decode_attn(cache, q.cuda(), first, torch.tensor([given], dtype=torch.int32).cuda(),
                                                   kn.cuda(), vn.cuda(), dev_err=err)
        assert err.item() == 5
        check_attention(c, q, kn, vn, out.cpu(), lse.cpu(), units=[(0, b, 0) for b in range(3)], what=str(given))
    # bad ids: among the shared rows' (the first sequence's) and a unit's own; the others' are not read
    for u, row, code in (((0, 0, 0), 3, 7), ((0, 2, 1), 69, 7), ((0, 1, 0), 3, 0)):
        c, q, kn, vn = make(lens, [0, 3], [32], 16, 64, F32, 2, True)
        c.pages[u][row // 16] = c.k.shape[0]
        cache = c.upload()
        err.zero_()
        out, lse = call(c, cache, q, kn, vn, err)
        assert err.item() == code, (u, row)
        bad = {(0, b, 0) for b in range(3)} if u == (0, 0, 0) else {u}
        if code == 0:
            bad = set()
        check_attention(c, q, kn, vn, out, lse, units=[x for x in np.ndindex(lens.shape) if x not in bad], what=str(u))
    # stored lengths and full units
    c, q, kn, vn = make(np.array([[[48], [10], [5]]]), [0, 1, 2, 3], [0, 4, 0], 16, 64, F32, 2, False)
    kn, vn = (torch.randn((1, 3, 1, 64)) for _ in "kv")
    for L, code in ((48, 1), (-1, 5), (49, 5)):
        c.length[0, 0, 0] = L
        cache = c.upload()
        err.zero_()
        out, lse = call(c, cache, q, kn, vn, err)
        assert err.item() == code and cache.length.cpu().flatten().tolist() == [L, 11, 6]
        check_attention(c, q, kn, vn, out, lse, units=[(0, 1, 0), (0, 2, 0)])


def test_agrees_with_the_decode_of_each():
    # the same rows in lists of their own; the new token's K and V, and calls twice in a row
    lens = _lens(300, [2, 70, 33, 1], 2, NL=2)
    c, q, kn, vn = make(lens, [0, 4], [300], 32, 128, BF, 7, True)
    pages = c.pages.clone()
    pages[:, 1:, :, :300 // 32] = pages[:, :1, :, :300 // 32]
    k, v = c.k.clone(), c.v.clone()
    for u in np.ndindex(lens.shape):                       # the page that shared rows fill in part
        rows = torch.arange(300 // 32 * 32, 300)
        to, of = c.where(u, rows), c.where((u[0], 0, u[2]), rows)
        k[to], v[to] = c.k[of], c.v[of]
    alone = B.PagedKVCache(k.cuda(), v.cuda(), pages.cuda(), c.length.cuda())
    shared = c.upload()
    first, counts = c.groups()
    for i in range(3):
        a, za = B.reco_paged_decode_attn(alone, q.cuda(), kn.cuda(), vn.cuda()) if i == 0 else B.reco_paged_decode_attn(alone, q.cuda())
        b, zb = B.reco_paged_shared_decode_attn(shared, q.cuda(), first, counts, *((kn.cuda(), vn.cuda()) if i == 0 else ()))
        assert torch.equal(alone.length, shared.length)
        top = max(v.float().nan_to_num(0).abs().max().item(), vn.float().abs().max().item())
        assert (a.float() - b.float()).abs().max().item() <= 2 * 2.0 ** -7 * top      # each is within 2^-7 of it
        assert (za - zb).abs().max().item() <= 2e-4


@pytest.mark.parametrize("dtype,D,G,page", [(BF, 128, 7, 64), (F32, 128, 2, 128), (BF, 64, 4, 4096)])
def test_long_prefixes(dtype, D, G, page):
    lens = np.array([[[9000], [9100], [12000], [9001], [4500]]])
    c, q, kn, vn = make(lens, [0, 4, 5], [8999, 4000], page, D, dtype, G, True, seed=7)
    for sinks, window in ((0, 0), (4, 4096)):
        cache = c.upload()
        out, lse = call(c, cache, q, kn, vn, sinks=sinks, window=window)
        check_attention(c, q, kn, vn, out, lse, sinks, window)


def test_bits_repeat_and_graphs_follow_their_inputs():
    lens = _lens(200, [5, 90, 33, 64, 12, 7], 2, NL=2)
    c, q, kn, vn = make(lens, [0, 2, 6], [200, 180], 16, 128, BF, 4, True, spare=4)
    c.k, c.v = (torch.nan_to_num(x, nan=0.5) for x in (c.k, c.v))      # groups change below: all rows may be seen
    caches = [c.upload() for _ in "ab"]
    first, counts = c.groups()
    dev = [x.cuda() for x in (q, kn, vn)]
    outs = [(torch.zeros_like(dev[0]), torch.zeros(q.shape[:3], device="cuda")) for _ in "ab"]
    wss = [B.paged_shared_decode_workspace(x, 8, 2) for x in caches]
    calls = [B.PreparedPagedSharedDecode(x, 8, first, counts, *o, w) for x, o, w in zip(caches, outs, wss)]
    s1, s2 = torch.cuda.Stream(), torch.cuda.Stream()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s1):
        calls[0](*dev)
    g = torch.Generator().manual_seed(4)
    for i, (groups, rows) in enumerate((([0, 2, 6], [200, 180]), ([0, 5, 6], [201, 10]), ([0, 0, 6], [0, 200]), ([0, 6, 6], [64, 0]))):
        # sequences of these rows whatever the groups: sequence 0's pages are listed whole in each
        for x in caches:
            x.pages[:, :, :, :200 // 16] = x.pages[:, :1, :, :200 // 16]
        first.copy_(torch.tensor(groups, dtype=torch.int32))
        counts.copy_(torch.tensor(rows, dtype=torch.int32))
        for x in dev:
            x.copy_(torch.randn(x.shape, generator=g).to(BF))
        torch.cuda.synchronize()
        with torch.cuda.stream(s1):
            graph.replay()
        with torch.cuda.stream(s2):                        # beside it, the eager call
            calls[1](*dev)
        torch.cuda.synchronize()
        assert torch.equal(caches[0].length, caches[1].length)
        assert caches[0].length.eq(torch.from_numpy(lens).cuda() + i + 1).all()
        for a, b in zip(outs[0], outs[1]):
            assert torch.equal(a.view(torch.int8), b.view(torch.int8)), f"replay {i}"
        assert torch.equal(caches[0].k.view(torch.int16), caches[1].k.view(torch.int16))
        assert torch.isfinite(outs[0][1]).all()


def _big(B_, groups, seed, most=40):
    """first and shared of `groups` groups over B_ sequences, and lengths, some of them of nothing."""
    rng = np.random.RandomState(seed)
    first = np.sort(np.concatenate([[0, B_], rng.randint(0, B_ + 1, groups - 1)]))
    shared = rng.randint(0, 50, groups)
    group = np.searchsorted(first[1:], np.arange(B_), side="right")
    return first, shared, (shared[group] + rng.randint(0, most, B_))[None, :, None], rng


@pytest.mark.parametrize("sinks,window", [(0, 0), (3, 20)])
@pytest.mark.parametrize("batch,groups", [(65, 2), (200, 16), (200, 17), (512, 1), (512, 16), (512, 64), (512, 65), (512, 400),
                                          (513, 3), (700, 16), (1100, 2), (1100, 65), (1100, 1000)])
def test_large_batches(batch, groups, sinks, window):
    # cells of whole batches and of parts of one, groups that cross their borders, lists past a wave's lanes
    first, shared, lens, rng = _big(batch, groups, batch + groups)
    c, q, kn, vn = make(lens, first, shared, 16, 64, BF, 2, True, seed=groups)
    cache = c.upload()
    err = torch.zeros(1, dtype=torch.int32, device="cuda")
    out, lse = call(c, cache, q, kn, vn, err, sinks=sinks, window=window)
    assert err.item() == 0
    some = sorted({0, 63, 64, batch - 1} | {b for b in (511, 512, 1023, 1024) if b < batch} | set(rng.choice(batch, 60).tolist()))
    check_attention(c, q, kn, vn, out, lse, sinks, window, units=[(0, b, 0) for b in some])
    # the others' as a call of another split of work has them: sequences in groups of one
    ones = torch.arange(batch + 1, dtype=torch.int32).cuda()
    if window == 0:
        check_append(c, cache, kn, vn)
    else:
        for u in np.ndindex(lens.shape):                   # shared rows in every list
            lead, P = (0, int(c.first[c.group[u[1]]]), 0), int(c.shared[0, c.group[u[1]]])
            rows = torch.arange(P)
            if u != lead and P:
                kept = P // 16
                c.pages[u][:kept] = c.pages[lead][:kept]
                at, of = c.where(u, rows[kept * 16:]), c.where(lead, rows[kept * 16:])
                c.k[at], c.v[at] = c.k[of], c.v[of]
        alone = c.upload()
        a, za = B.reco_paged_shared_decode_attn(alone, q.cuda(), ones, torch.zeros(batch, dtype=torch.int32).cuda(), kn.cuda(), vn.cuda(),
                                                sinks, window, dev_err=err)
        top = max(c.v.float().nan_to_num(0).abs().max().item(), vn.float().abs().max().item())
        assert err.item() == 0 and (a.cpu().float() - out.float()).abs().max().item() <= 2 * 2.0 ** -7 * top   # each within 2^-7
        assert (za.cpu() - lse).abs().max().item() <= 2e-4


def test_lists_of_many_groups_that_do_not_ascend():
    first, shared, lens, _ = _big(600, 300, 1)
    shared[:] = 0
    for at, x in ((70, -1), (299, 601), (300, 599), (150, 2 ** 31 - 1), (0, 1)):
        c, q, kn, vn = make(lens, first, shared, 16, 64, F32, 1, True)
        cache = c.upload()
        bad = torch.from_numpy(first.astype(np.int64).copy())
        bad[at] = x
        err = torch.zeros(1, dtype=torch.int32, device="cuda")
        out, lse = B.reco_paged_shared_decode_attn(cache, q.cuda(), bad.int().cuda(), torch.ones(300, dtype=torch.int32).cuda(), kn.cuda(),
                                                   vn.cuda(), dev_err=err)
        assert err.item() == 10
        check_attention(c, q, kn, vn, out.cpu(), lse.cpu(), units=[(0, b, 0) for b in range(0, 600, 13)], what=str(at))
        check_append(c, cache, kn, vn)


def test_pages_past_four_gibibytes():
    # 4,200 pages of 1 MiB in each pool; those in use are the last ones
    page, n_pages = 4096, 4200
    c, q, kn, vn = make(np.array([[[5000], [5040], [4999]]]), [0, 3], [4990], page, 128, BF, 4, True, seed=9)
    have = c.k.shape[0]
    pools = [torch.empty((n_pages, page, 128), dtype=BF, device="cuda") for _ in "kv"]
    for pool, x in zip(pools, (c.k, c.v)):
        pool[n_pages - have:] = x.cuda()
    table = torch.where((c.pages >= 0) & (c.pages < have), c.pages + (n_pages - have), c.pages)
    cache = B.PagedKVCache(*pools, table.cuda(), c.length.cuda())
    for sinks, window in ((0, 0), (4, 700)):
        out, lse = call(c, cache, q, kn, vn, sinks=sinks, window=window)
        check_attention(c, q, kn, vn, out, lse, sinks, window)
        cache.length.copy_(c.length)
    for pool, x in zip(pools, (kn, vn)):
        for u in np.ndindex(c.lens.shape):
            L = int(c.lens[u])
            at = table[u][L // page].item()
            assert at >= 4190 and torch.equal(pool[at, L % page].cpu(), x[u])


def test_graphs_that_share_a_workspace():
    # two calls of other sizes, captured with one workspace and replayed in turn
    made = [make(_lens(100, [3, 40, 9, 70], 2), [0, 4], [100], 16, 128, BF, 4, False, seed=1),
            make(_lens(300, [80, 2], 1, NL=3), [0, 1, 2], [300, 290], 16, 128, BF, 7, False, seed=2)]
    caches = [m[0].upload() for m in made]
    sizes = [B.paged_shared_decode_attn_workspace_size(x, m[1].shape[2], len(m[0].first) - 1) for x, m in zip(caches, made)]
    ws = torch.empty(max(sizes), dtype=torch.uint8, device="cuda")
    calls, graphs, s = [], [], torch.cuda.Stream()
    for x, (c, q, _, _) in zip(caches, made):
        out = torch.zeros(q.shape, dtype=BF, device="cuda")
        calls.append((B.PreparedPagedSharedDecode(x, q.shape[2], *c.groups(), out, torch.zeros(q.shape[:3], device="cuda"), ws), q.cuda()))
    torch.cuda.synchronize()
    for f, q in calls:
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1], stream=s):
            f(q)
    for i in range(3):
        for f, q in calls:
            f.out.zero_()
            q.mul_(-1 if i else 1)
        torch.cuda.synchronize()
        with torch.cuda.stream(s):
            for _ in range(2):
                for g in graphs:
                    g.replay()
        torch.cuda.synchronize()
        for (f, q), (c, _, _, _) in zip(calls, made):
            check_attention(c, q.cpu(), None, None, f.out.cpu(), f.lse.cpu(), what=f"turn {i}")


@pytest.mark.parametrize("dtype", [F32, BF])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("sequences", [1, 4, 5, 8, 9, 17, 20, 21])
def test_blocks_of_few_rows(dtype, D, sequences):
    # 8 query heads: blocks of up to 32 rows, up to 64 and more, alone and behind whole ones
    own = [i * 7 % 50 for i in range(sequences)]
    for P, sinks, window in ((0, 0, 0), (31, 0, 0), (300, 0, 0), (1000, 3, 700)):
        c, q, kn, vn = make(_lens(P, own, 2), [0, sequences], [P], 16, D, dtype, 8, True, seed=P)
        cache = c.upload()
        err = torch.zeros(1, dtype=torch.int32, device="cuda")
        out, lse = call(c, cache, q, kn, vn, err, sinks=sinks, window=window)
        assert err.item() == 0
        check_attention(c, q, kn, vn, out, lse, sinks, window, what=f"{P} rows")
        again = c.upload()
        o2, z2 = call(c, again, q, kn, vn, err, sinks=sinks, window=window)
        assert torch.equal(o2.view(torch.uint8), out.view(torch.uint8)) and torch.equal(z2, lse)


def test_short_own_rows_beside_odd_ones():
    # ranges of few rows in their tiles, pages that are full of infinities around them
    for dtype, D, G in ((BF, 128, 4), (BF, 64, 1), (F32, 128, 7)):
        for P, sinks, window in ((47, 0, 0), (64, 0, 0), (64, 2, 21), (100, 5, 33)):
            c, q, kn, vn = make(_lens(P, [0, 1, 2, 15, 16, 17], 2), [0, 6], [P], 64, D, dtype, G, True, seed=P)
            for x in (c.k, c.v):
                x[torch.isnan(x)] = float("inf")
            cache = c.upload()
            out, lse = call(c, cache, q, kn, vn, sinks=sinks, window=window)
            check_attention(c, q, kn, vn, out, lse, sinks, window, what=f"{dtype} {P}")


def test_without_lse_and_on_another_stream():
    c, q, kn, vn = make(_lens(90, [3, 40, 9], 2), [0, 3], [90], 16, 128, BF, 4, True, seed=6)
    cache, (first, shared), s = c.upload(), c.groups(), torch.cuda.Stream()
    dev = [x.cuda() for x in (q, kn, vn)]
    torch.cuda.synchronize()
    with torch.cuda.stream(s):
        out, none = B.reco_paged_shared_decode_attn(cache, dev[0], first, shared, *dev[1:], want_lse=False)
    s.synchronize()
    assert none is None
    again = c.upload()
    o2, z2 = B.reco_paged_shared_decode_attn(again, dev[0], first, shared, *dev[1:])
    assert torch.equal(o2.view(torch.int16), out.view(torch.int16))
    check_attention(c, q, kn, vn, out.cpu(), z2.cpu())
    check_append(c, cache, kn, vn)
