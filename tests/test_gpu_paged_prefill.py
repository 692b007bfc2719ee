"""reco_paged_prefill_attn against the plain 64-bit form: types, head layouts, page
sizes, runs of one token to long ones over empty and long caches, padded batches,
windows and sinks at tile and block borders, and what is left untouched."""
import math

import numpy as np
import pytest
import torch

from paged_helpers import Paged, attend, close_lse, close_out
from paper_2608_04771_amd import binding as B

pytestmark = pytest.mark.gpu

F32, BF = torch.float32, torch.bfloat16


def _inputs(p, G, T, seed):
    NL, Bs, H = p.lens.shape
    g = torch.Generator().manual_seed(seed)
    q = torch.randn((NL, Bs, H * G, T, p.D), generator=g).to(p.k.dtype)
    kn, vn = (torch.randn((NL, Bs, H, T, p.D), generator=g).to(p.k.dtype) for _ in "kv")
    return q, kn, vn


def _ref(p, u, G, q, kn, vn, n, sinks, window, scale, poison=()):
    """64-bit outputs [G][n][D] and lse [G][n] of one unit."""
    k, v = p.rows(u)
    L = k.shape[0]
    k, v = torch.cat([k, kn[u][:n]]).double(), torch.cat([v, vn[u][:n]]).double()
    j, pos = torch.arange(L + n), L + torch.arange(n)[:, None]
    ok = j <= pos
    if window:
        ok &= (j < sinks) | (j > pos - window)
    x = torch.einsum("gtd,jd->gtj", q[u[:2]][u[2] * G:(u[2] + 1) * G, :n].double(), k) * scale
    x = x.masked_fill(~ok, -math.inf)
    lse = torch.logsumexp(x, -1)
    return torch.einsum("gtj,jd->gtd", torch.exp(x - lse[..., None]), v), lse, v


def _check(p, G, T, news=None, sinks=0, window=0, seed=1, expect_err=0, scale=None, every=1):
    NL, Bs, H = p.lens.shape
    dtype = p.k.dtype
    s = 1 / math.sqrt(p.D) if scale is None else scale
    q, kn, vn = _inputs(p, G, T, seed)
    n_new = [T] * Bs if news is None else news
    for b, n in enumerate(n_new):                         # padding places hold what may not be read
        for x in (q, kn, vn):
            x[:, b, :, n:] = float("nan")
    cache = p.upload()
    err = torch.zeros(1, dtype=torch.int32, device="cuda")
    out, lse = torch.full_like(q, 7.0).cuda(), torch.full(q.shape[:4], 7.0).cuda()
    B.reco_paged_prefill_attn(cache, q.cuda(), kn.cuda(), vn.cuda(),
                              None if news is None else torch.tensor(news, dtype=torch.int32).cuda(), sinks, window,
                              scale, out=out, lse=lse, dev_err=err)
    torch.cuda.synchronize()
    assert err.item() == expect_err
    out, lse = out.cpu(), lse.cpu()
    k0, v0, n0 = p.k.clone(), p.v.clone(), p.length.clone()
    w0 = None if p.weight is None else p.weight.clone()
    for u in np.ndindex(NL, Bs, H):
        n, L = n_new[u[1]], int(p.lens[u])
        o, z = out[u[:2]][u[2] * G:(u[2] + 1) * G], lse[u[:2]][u[2] * G:(u[2] + 1) * G]
        what = f"unit {u} L={L} n={n} sinks={sinks} window={window}"
        if np.ravel_multi_index(u, (NL, Bs, H)) % every == 0:
            ref, rl, v = _ref(p, u, G, q, kn, vn, n, sinks, window, s)
            close_out(o[:, :n], ref, v, dtype, what)
            close_lse(z[:, :n], rl, dtype, what)
        assert (o[:, n:] == 7).all() and (z[:, n:] == 7).all(), f"{what}: padding places"
        at = p.where(u, torch.arange(L, L + n))
        k0[at], v0[at] = kn[u][:n], vn[u][:n]
        n0[u] = L + n
        if w0 is not None:
            w0[u][L:L + n] = 0.0
    assert torch.equal(cache.k.cpu().view(torch.int8), k0.view(torch.int8)), "K rows"
    assert torch.equal(cache.v.cpu().view(torch.int8), v0.view(torch.int8)), "V rows"
    assert torch.equal(cache.length.cpu(), n0)
    if w0 is not None:
        assert torch.equal(cache.weight.cpu().view(torch.int32), w0.view(torch.int32)), "weights"
    return cache


TYPES = [(F32, 64, 4, 16), (F32, 128, 7, 32), (BF, 128, 7, 16), (BF, 64, 4, 64), (BF, 128, 1, 256), (BF, 64, 16, 16),
         (F32, 128, 16, 1024), (BF, 128, 5, 4096)]


@pytest.mark.parametrize("dtype,D,G,page", TYPES)
@pytest.mark.parametrize("T", [1, 2, 31, 64, 130])
def test_runs_over_ragged_units(dtype, D, G, page, T):
    lens = np.array([0, 1, 15, 16, 17, 63, 64, 65, 500, 127, 128, 129]).reshape(2, 3, 2)
    _check(Paged(lens, page, D, dtype, spare=T, seed=D + G + T), G, T)


@pytest.mark.parametrize("dtype,D,G,page", TYPES[:4])
def test_padded_batch(dtype, D, G, page):
    lens = np.array([[[0, 40], [64, 3], [100, 100], [7, 0], [30, 31]]])
    _check(Paged(lens, page, D, dtype, spare=70, seed=5, weights=True), G, 70, [70, 1, 0, 33, 64])


@pytest.mark.parametrize("sinks,window", [(0, 1), (1, 1), (4, 64), (33, 32), (16, 31), (64, 500), (5, 16), (1000, 7),
                                          (2 ** 31 - 1, 3), (3, 2 ** 31 - 1), (70, 100), (200, 40)])
@pytest.mark.parametrize("dtype,D,G", [(F32, 64, 4), (BF, 128, 7)])
def test_window_and_sinks(dtype, D, G, sinks, window):
    lens = np.array([[[0, 150], [64, 333]]])
    _check(Paged(lens, 16, D, dtype, spare=200, seed=3), G, 200, [200, 177], sinks, window)


@pytest.mark.parametrize("dtype,D,G,L,T", [(BF, 128, 7, 9645, 32), (BF, 64, 8, 16385, 3), (F32, 64, 4, 5000, 1),
                                           (F32, 128, 2, 3001, 40), (BF, 128, 4, 0, 1500), (BF, 128, 16, 20000, 1)])
def test_long(dtype, D, G, L, T):
    """Few query rows over long caches (split), and a longer prompt."""
    _check(Paged([[[L, L // 3]]], 64, D, dtype, spare=T, seed=L + T), G, T)


@pytest.mark.parametrize("D,sinks,window", [(128, 0, 0), (128, 5, 90), (64, 0, 33), (64, 0, 0), (128, 130, 1)])
@pytest.mark.parametrize("page", [16, 128])
def test_runs_for_the_whole_chip(D, sinks, window, page):
    """Enough query rows for blocks of 256 on every compute unit, over empty, short and
    longer caches, some sequences padded (one to nothing)."""
    rng = np.random.RandomState(D + window)
    lens = rng.randint(0, 400, (1, 40, 2))
    lens[0, :6, 0] = [0, 1, 64, 63, 128, 65]
    news = rng.randint(1, 241, 40)
    news[:5] = [240, 0, 1, 64, 129]
    _check(Paged(lens, page, D, BF, spare=240, seed=D, weights=window == 90), 12, 240, [int(x) for x in news], sinks, window, every=7)


def test_long_prompt_for_the_whole_chip():
    """One long prompt from an empty cache, and one behind a cache, through a window and without."""
    for lens, T, window in (([[[0] * 8]], 2400, 0), ([[[700] * 8]], 2400, 800)):
        _check(Paged(lens, 64, 64, BF, spare=T, seed=T), 8, T, None, 4, window, every=5)


def test_many_units_at_once():
    lens = np.random.RandomState(3).randint(0, 200, (3, 30, 4))
    _check(Paged(lens, 16, 64, BF, spare=5, seed=3), 3, 5, list(np.random.RandomState(4).randint(0, 6, 30)))


@pytest.mark.parametrize("scale", [-0.2, 0.0, 1e-3])
def test_scales(scale):
    _check(Paged([[[100, 30]]], 16, 64, F32, spare=20, seed=2), 4, 20, scale=scale)


def test_layer_range():
    p = Paged(np.array([[[20]], [[33]], [[47]]]), 16, 64, F32, spare=10, seed=8)
    q, kn, vn = _inputs(p, 3, 10, 1)
    cache = p.upload()
    out, lse = B.reco_paged_prefill_attn(cache, q[1:2].contiguous().cuda(), kn[1:2].contiguous().cuda(),
                                         vn[1:2].contiguous().cuda(), layer0=1, n_layers=1)
    ref, rl, v = _ref(p, (1, 0, 0), 3, q, kn, vn, 10, 0, 0, 1 / 8)
    close_out(out[0, 0].cpu(), ref, v, F32, "layer 1")
    close_lse(lse[0, 0].cpu(), rl, F32, "layer 1")
    assert cache.length.cpu().flatten().tolist() == [20, 43, 47]


def test_what_does_not_fit_is_attended_but_not_stored():
    for what, code in (("capacity", 1), ("page", 7), ("length", 5)):
        p = Paged([[[40, 20]]], 16, 64, F32, spare=30, seed=3, weights=True)
        p.k.nan_to_num_(0.0)
        p.v.nan_to_num_(0.0)
        q, kn, vn = _inputs(p, 4, 30, 2)
        if what == "capacity":
            p = Paged([[[80, 50]]], 16, 64, F32, seed=3, weights=True)             # unit 0 is full
            p.lens[0, 0, 1] = p.length[0, 0, 1] = 20
        elif what == "page":
            p.pages[0, 0, 0, 4] = -1
        else:
            p.length[0, 0, 0] = -1
        cache = p.upload()
        k0, w0, n0 = cache.k.clone(), cache.weight.clone(), int(p.length[0, 0, 0])
        err = torch.zeros(1, dtype=torch.int32, device="cuda")
        out, lse = B.reco_paged_prefill_attn(cache, q.cuda(), kn.cuda(), vn.cuda(), dev_err=err)
        torch.cuda.synchronize()
        assert err.item() == code, what
        assert cache.length.cpu().flatten().tolist() == [n0, 50], what
        if what == "length":
            p.lens[0, 0, 0] = 0
        for h in range(2):
            ref, rl, v = _ref(p, (0, 0, h), 4, q, kn, vn, 30, 0, 0, 1 / 8)
            close_out(out[0, 0, 4 * h:4 * h + 4].cpu(), ref, v, F32, what)
            close_lse(lse[0, 0, 4 * h:4 * h + 4].cpu(), rl, F32, what)
        at = p.where((0, 0, 1), torch.arange(20, 50))
        k0[tuple(x.cuda() for x in at)] = kn[0, 0, 1].cuda()
        assert torch.equal(cache.k.view(torch.int32), k0.view(torch.int32)), what
        assert torch.equal(cache.weight[0, 0, 0].view(torch.int32), w0[0, 0, 0].view(torch.int32)), what


def test_bad_counts_and_pages():
    """A count outside [0, T] is reported and its sequence skipped; a cached row's bad page is reported."""
    p = Paged([[[40], [20], [30]]], 16, 64, F32, spare=8, seed=3)
    q, kn, vn = _inputs(p, 4, 8, 2)
    cache = p.upload()
    err = torch.zeros(1, dtype=torch.int32, device="cuda")
    out = torch.full_like(q, 7.0).cuda()
    B.reco_paged_prefill_attn(cache, q.cuda(), kn.cuda(), vn.cuda(), torch.tensor([9, 8, -1], dtype=torch.int32).cuda(),
                              out=out, dev_err=err)
    torch.cuda.synchronize()
    assert err.item() == 5 and cache.length.cpu().flatten().tolist() == [40, 28, 30]
    assert (out[:, 0] == 7).all() and (out[:, 2] == 7).all()
    ref, _, v = _ref(p, (0, 1, 0), 4, q, kn, vn, 8, 0, 0, 1 / 8)
    close_out(out[0, 1].cpu(), ref, v, F32, "good sequence")
    p.pages[0, 0, 0, 1] = p.k.shape[0]
    cache = p.upload()
    err.zero_()
    out, _ = B.reco_paged_prefill_attn(cache, q.cuda(), kn.cuda(), vn.cuda(), dev_err=err)
    torch.cuda.synchronize()
    assert err.item() == 7
    close_out(out[0, 1].cpu(), ref, v, F32, "good sequence")


def test_graph_replays_match_eager():
    p = Paged(np.array([[[700, 90], [33, 1500]]]), 32, 128, BF, spare=40, seed=21, weights=True)
    q, kn, vn = (x.cuda() for x in _inputs(p, 7, 40, 3))
    news = torch.tensor([40, 17], dtype=torch.int32).cuda()
    ref, cap = p.upload(), p.upload()
    n0 = cap.length.clone()
    out, lse = torch.zeros_like(q), torch.zeros(q.shape[:4], device="cuda")
    o, z = torch.zeros_like(q), torch.zeros(q.shape[:4], device="cuda")
    ws = torch.empty(B.paged_prefill_attn_workspace_size(cap, 14, 40), dtype=torch.uint8, device="cuda")

    def step():
        B.reco_paged_prefill_attn(cap, q, kn, vn, news, 4, 600, out=out, lse=lse, ws=ws)
        cap.length.copy_(n0)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for rep in range(4):
        B.reco_paged_prefill_attn(ref, q, kn, vn, news, 4, 600, out=o, lse=z)
        ref.length.copy_(n0)
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, o) and torch.equal(lse, z), rep
        assert torch.equal(cap.k.view(torch.int16), ref.k.view(torch.int16)), rep


@pytest.mark.parametrize("dtype,D,G,L,T,sinks,window", [
    (BF, 128, 4, 0, 100, 0, 0), (BF, 128, 7, 70, 100, 3, 40), (F32, 64, 1, 33, 70, 0, 0), (F32, 128, 3, 64, 40, 2, 16),
    (BF, 64, 1, 200, 90, 0, 33), (BF, 64, 16, 5, 20, 0, 0)])
def test_values_that_only_some_tokens_see(dtype, D, G, L, T, sinks, window):
    # infinities and NaN in V reach the tokens that see them, and their columns, alone
    p = Paged(np.full((1, 1, 2), L), 16, D, dtype, spare=T, seed=D + T)
    q, kn, vn = _inputs(p, G, T, 11)
    inf, nan = float("inf"), float("nan")
    for u in np.ndindex(1, 1, 2):
        for r, c, x in ((1, 0, nan), (L + T // 2, 3, inf), (L + T // 2, 5, nan), (L + T // 3, 40, -inf), (L + T - 1, 17, nan),
                        (L + T // 2 + 1, 3, -inf), (L // 2, 60, inf), (L + 2, D - 1, inf)):
            if r >= L:
                vn[u][r - L, c] = x
            else:
                page, row = p.where(u, [r])
                p.v[page, row, c] = x
    cache = p.upload()
    out, lse = B.reco_paged_prefill_attn(cache, q.cuda(), kn.cuda(), vn.cuda(), None, sinks, window)
    out, lse = out.cpu().double(), lse.cpu()
    s = 1 / math.sqrt(D)
    for u in np.ndindex(1, 1, 2):
        k, v = p.rows(u)
        k, v = torch.cat([k, kn[u]]), torch.cat([v, vn[u]])
        for t in range(T):
            ref, rl, _ = attend(k, v, q[u[:2]][u[2] * G:(u[2] + 1) * G, t], L + t, s, sinks, window)
            got, fin = out[u[:2]][u[2] * G:(u[2] + 1) * G, t], torch.isfinite(ref)
            what = f"unit {u} token {t}"
            for same in (torch.isnan, torch.isposinf, torch.isneginf):
                assert torch.equal(same(got), same(ref)), what
            close_out(got[fin], ref[fin], v, dtype, what)
            close_lse(lse[u[:2]][u[2] * G:(u[2] + 1) * G, t], rl, dtype, what)


@pytest.mark.parametrize("dtype,D,G", [(BF, 128, 4), (F32, 64, 2)])
def test_earlier_tokens_do_not_depend_on_later_rows(dtype, D, G):
    # the run's last rows hold NaN in K and V: all tokens before them get the bits they
    # would get if they were ordinary
    T = 90
    p = Paged(np.full((1, 1, 2), 50), 16, D, dtype, spare=T, seed=4)
    q, kn, vn = _inputs(p, G, T, 12)
    a = B.reco_paged_prefill_attn(p.upload(), q.cuda(), kn.cuda(), vn.cuda())
    for x in (kn, vn):
        x[..., T - 20:, :] = float("nan")
    b = B.reco_paged_prefill_attn(p.upload(), q.cuda(), kn.cuda(), vn.cuda())
    for x, y in zip(a, b):
        assert torch.equal(x[:, :, :, :T - 20], y[:, :, :, :T - 20])
        assert torch.isnan(y[:, :, :, T - 20:]).all()


@pytest.mark.parametrize("D,sinks,window", [(128, 0, 0), (128, 5, 1090), (64, 0, 0), (64, 70, 1024)])
@pytest.mark.parametrize("page", [16, 128])
def test_blocks_of_256_rows(D, sinks, window, page):
    # runs that fill two rounds of such blocks, over caches with room for many keys
    rng = np.random.RandomState(D + window)
    lens = rng.randint(0, 400, (1, 40, 2))
    lens[0, :8, 0] = [0, 1, 64, 63, 128, 65, 1000, 1300]
    news = rng.randint(1, 241, 40)
    news[:7] = [240, 0, 1, 64, 129, 240, 200]
    p = Paged(lens, page, D, BF, spare=240, seed=D, weights=window == 1090, extra_pages=1024 // page)
    _check(p, 12, 240, [int(x) for x in news], sinks, window, every=7)


@pytest.mark.parametrize("window", [0, 1100])
def test_long_prompts_in_blocks_of_256_rows(window):
    _check(Paged([[[0, 700] * 4]], 64, 64, BF, spare=2400, seed=9), 12, 2400, None, 4, window, every=3)


def test_values_that_only_some_tokens_see_in_blocks_of_256_rows():
    # the run's second half holds NaN in K and V: the first half gets the bits it gets
    # from ordinary rows
    p = Paged(np.full((1, 40, 2), 30), 16, 128, BF, spare=240, seed=8, extra_pages=64)
    q, kn, vn = (x.cuda() for x in _inputs(p, 12, 240, 13))
    a = B.reco_paged_prefill_attn(p.upload(), q, kn, vn)
    for x in (kn, vn):
        x[..., 117:, :] = float("nan")
    b = B.reco_paged_prefill_attn(p.upload(), q, kn, vn)
    for x, y in zip(a, b):
        assert torch.equal(x[:, :, :, :117], y[:, :, :, :117])
        assert torch.isnan(y[:, :, :, 117:]).all()


@pytest.mark.parametrize("batch,code", [(300, 1), (300, 7), (300, 5), (700, 1), (700, 7), (700, 5)])
def test_units_that_do_not_fit_among_many(batch, code):
    # enough units that none is split: rows are stored beside the attention, and those
    # of units 3 (bad) and 7 (a bad count) are not
    T, page, D = 150, 16, 64
    lens = np.random.RandomState(batch + code).randint(0, 40, (1, batch, 1))
    lens[0, 3, 0] = 37
    p = Paged(lens, page, D, BF, spare=T, seed=code, weights=True)
    q, kn, vn = _inputs(p, 2, T, 5)
    news = np.random.RandomState(1).randint(0, T + 1, batch)
    news[[3, 7]] = T, T + 1
    if code == 1:
        p.length[0, 3, 0] = p.max_pages * page - T + 1
        p.pages[0, 3, 0] = p.pages[0, 3, 0, 0]              # rows past the 37 are whatever lies there
    elif code == 7:
        p.pages[0, 3, 0, 37 // page + 3] = -5
    else:
        p.length[0, 3, 0] = p.max_pages * page + 1
        p.pages[0, 3, 0] = p.pages[0, 3, 0, 0]
    news[7] = T + 1 if code == 5 else 0
    cache = p.upload()
    err = torch.zeros(1, dtype=torch.int32, device="cuda")
    B.reco_paged_prefill_attn(cache, q.cuda(), kn.cuda(), vn.cuda(), torch.tensor(news, dtype=torch.int32).cuda(),
                              dev_err=err)
    assert err.item() == code
    k0, v0, n0, w0 = p.k.clone(), p.v.clone(), p.length.clone(), p.weight.clone()
    for b in range(batch):
        if b in (3, 7):
            continue
        L, n = int(lens[0, b, 0]), int(news[b])
        at = p.where((0, b, 0), torch.arange(L, L + n))
        k0[at], v0[at] = kn[0, b, 0, :n], vn[0, b, 0, :n]
        n0[0, b, 0] += n
        w0[0, b, 0, L:L + n] = 0.0
    assert torch.equal(cache.k.cpu().view(torch.int16), k0.view(torch.int16))
    assert torch.equal(cache.v.cpu().view(torch.int16), v0.view(torch.int16))
    assert torch.equal(cache.length.cpu(), n0)
    assert torch.equal(cache.weight.cpu().view(torch.int32), w0.view(torch.int32))
