"""reco_paged_decode_attn against the plain 64-bit form: types, head layouts, page
sizes, lengths from nothing to long ones, windows and sinks at tile and page
borders, weights, appends, and what is left untouched."""
import math

import numpy as np
import pytest
import torch

from paged_helpers import Paged, attend, close_lse, close_out, close_weight
from paper_2608_04771_amd import binding as B

pytestmark = pytest.mark.gpu

F32, BF = torch.float32, torch.bfloat16


def _inputs(p, G, append, seed):
    NL, Bs, H = p.lens.shape
    g = torch.Generator().manual_seed(seed)
    q = torch.randn((NL, Bs, H * G, p.D), generator=g).to(p.k.dtype)
    kn = vn = None
    if append:
        kn, vn = (torch.randn((NL, Bs, H, p.D), generator=g).to(p.k.dtype) for _ in "kv")
    return q, kn, vn


def _up(t):
    return None if t is None else t.cuda()


def _check(p, G, append, sinks=0, window=0, seed=1, expect_err=0, prepared=False):
    """One call against the plain form, with everything it may not touch."""
    NL, Bs, H = p.lens.shape
    dtype, scale = p.k.dtype, 1 / math.sqrt(p.D)
    q, kn, vn = _inputs(p, G, append, seed)
    cache = p.upload()
    err = torch.zeros(1, dtype=torch.int32, device="cuda")
    if prepared:
        out, lse = torch.empty_like(q.cuda()), torch.empty(q.shape[:3], device="cuda")
        call = B.PreparedPagedDecode(cache, H * G, out, lse, B.paged_decode_workspace(cache, H * G), err, sinks, window)
        call(q.cuda(), _up(kn), _up(vn))
    else:
        out, lse = B.reco_paged_decode_attn(cache, q.cuda(), _up(kn), _up(vn), sinks, window, dev_err=err)
    torch.cuda.synchronize()
    assert err.item() == expect_err
    out, lse = out.cpu(), lse.cpu()
    k0, v0, w0 = p.k.clone(), p.v.clone(), None if p.weight is None else p.weight.clone()
    for u in np.ndindex(NL, Bs, H):
        n = int(p.lens[u])
        k, v = p.rows(u)
        if append:
            k, v = torch.cat([k, kn[u][None]]), torch.cat([v, vn[u][None]])
        hs = slice(u[2] * G, (u[2] + 1) * G)
        ref, rl, w = attend(k, v, q[u[:2]][hs], k.shape[0] - 1, scale, sinks, window)
        what = f"unit {u} n={n} sinks={sinks} window={window}"
        close_out(out[u[:2]][hs], ref, v, dtype, what)
        close_lse(lse[u[:2]][hs], rl, dtype, what)
        if w0 is not None:
            mine = cache.weight[u].cpu()
            before = p.weight[u][:k.shape[0]].double().clone()
            if append:
                before[n] = 0.0
            close_weight(mine[:k.shape[0]], before + w, what)
            assert torch.equal(mine[k.shape[0]:], w0[u][k.shape[0]:]) or torch.isnan(mine[k.shape[0]:]).all()
        if append:
            at = p.where(u, [n])
            k0[at], v0[at] = kn[u], vn[u]
    assert torch.equal(cache.k.cpu().view(torch.int8), k0.view(torch.int8)), "K rows"
    assert torch.equal(cache.v.cpu().view(torch.int8), v0.view(torch.int8)), "V rows"
    assert (cache.length.cpu().numpy() == p.lens + (1 if append else 0)).all()
    return cache


RAGGED = [0, 1, 15, 16, 17, 31, 32, 33, 63, 64, 65, 1000, 1040, 517, 250, 7]


@pytest.mark.parametrize("append", [False, True])
@pytest.mark.parametrize("dtype,D,G,page", [(F32, 64, 4, 16), (F32, 128, 7, 32), (BF, 128, 7, 16), (BF, 64, 4, 64),
                                            (BF, 128, 1, 256), (BF, 64, 16, 16), (F32, 128, 16, 1024),
                                            (BF, 128, 8, 4096), (F32, 64, 5, 128)])
def test_ragged_units(dtype, D, G, page, append):
    lens = np.array(RAGGED).reshape(2, 2, 4)
    _check(Paged(lens, page, D, dtype, spare=1, seed=D + G), G, append)


@pytest.mark.parametrize("sinks,window", [(0, 1), (1, 1), (4, 64), (33, 32), (16, 31), (64, 500), (5, 16), (1000, 7),
                                          (2 ** 31 - 1, 3), (3, 2 ** 31 - 1), (40, 100)])
@pytest.mark.parametrize("dtype,D", [(F32, 64), (BF, 128)])
def test_window_and_sinks(dtype, D, sinks, window):
    lens = np.array(RAGGED).reshape(1, 4, 4)
    _check(Paged(lens, 16, D, dtype, spare=1, seed=3, weights=True), 4, True, sinks, window)


@pytest.mark.parametrize("append", [False, True])
@pytest.mark.parametrize("dtype,D,G", [(F32, 64, 4), (BF, 128, 7), (BF, 64, 16), (F32, 128, 1)])
@pytest.mark.parametrize("batch,hi", [(1, 5000), (300, 90)])
def test_weights(dtype, D, G, append, batch, hi):
    """Few units (several splits) and more units than compute units (one split each)."""
    lens = np.random.RandomState(5).randint(0, hi + 1, (1, batch, 2))
    lens[0, 0, 0] = hi
    _check(Paged(lens, 32, D, dtype, spare=1, seed=9, weights=True), G, append)


@pytest.mark.parametrize("n", [1, 31, 32, 33, 4095, 4096, 16385])
def test_one_unit(n):
    """One unit takes the most splits; the append opens a page where n is a multiple of 16."""
    _check(Paged([[[n]]], 16, 128, BF, spare=1, seed=n), 7, True, prepared=True)


def test_many_long_units():
    """More units than compute units, long at capacity: two splits each."""
    lens = np.random.RandomState(2).randint(0, 300, (2, 40, 4))
    lens[0, 0, 0] = 8300
    _check(Paged(lens, 16, 64, BF, spare=1, seed=2), 2, True)


def test_layer_range():
    lens = np.array([[[20, 50]], [[33, 64]], [[47, 1]], [[80, 16]]])
    p = Paged(lens, 16, 64, F32, spare=1, seed=8)
    q, kn, vn = _inputs(p, 3, True, 1)
    cache = p.upload()
    out, lse = B.reco_paged_decode_attn(cache, q[1:3].contiguous().cuda(), kn[1:3].contiguous().cuda(),
                                        vn[1:3].contiguous().cuda(), layer0=1, n_layers=2)
    torch.cuda.synchronize()
    assert cache.length.cpu().flatten().tolist() == [20, 50, 34, 65, 48, 2, 80, 16]
    for l in (1, 2):
        for h in range(2):
            k, v = p.rows((l, 0, h))
            k, v = torch.cat([k, kn[l, 0, h][None]]), torch.cat([v, vn[l, 0, h][None]])
            ref, rl, _ = attend(k, v, q[l, 0, 3 * h:3 * h + 3], k.shape[0] - 1, 1 / 8)
            close_out(out[l - 1, 0, 3 * h:3 * h + 3].cpu(), ref, v, F32, f"layer {l}")
            close_lse(lse[l - 1, 0, 3 * h:3 * h + 3].cpu(), rl, F32, f"layer {l}")


def test_shared_pages():
    """Two sequences whose first pages are the same ones: both read them, each appends to its own."""
    p = Paged([[[40], [40]]], 16, 64, F32, spare=1, seed=4)
    p.pages[0, 1, 0, :2] = p.pages[0, 0, 0, :2]
    _check(p, 4, True)


@pytest.mark.parametrize("weights", [False, True])
def test_full_unit_refuses_the_append(weights):
    """At capacity the token takes part in the attention, but nothing is stored."""
    p = Paged([[[64, 10]]], 16, 128, BF, spare=0, seed=3, weights=weights)
    q, kn, vn = _inputs(p, 4, True, 2)
    cache = p.upload()
    k0, v0 = cache.k.clone(), cache.v.clone()
    err = torch.zeros(1, dtype=torch.int32, device="cuda")
    out, _ = B.reco_paged_decode_attn(cache, q.cuda(), kn.cuda(), vn.cuda(), dev_err=err)
    torch.cuda.synchronize()
    assert err.item() == 1 and cache.length.cpu().flatten().tolist() == [64, 11]
    k, v = p.rows((0, 0, 0))
    k, v = torch.cat([k, kn[0, 0, 0][None]]), torch.cat([v, vn[0, 0, 0][None]])
    ref, _, w = attend(k, v, q[0, 0, :4], 64, 1 / math.sqrt(128))
    close_out(out[0, 0, :4].cpu(), ref, v, BF, "full unit")
    if weights:
        close_weight(cache.weight[0, 0, 0].cpu(), p.weight[0, 0, 0].double() + w[:64], "full unit")
    own = p.where((0, 0, 1), [10])
    k0[own], v0[own] = kn[0, 0, 1].cuda(), vn[0, 0, 1].cuda()
    assert torch.equal(cache.k.view(torch.int16), k0.view(torch.int16))
    assert torch.equal(cache.v.view(torch.int16), v0.view(torch.int16))


@pytest.mark.parametrize("n", [40, 3000])
def test_bad_pages_and_lengths_are_reported(n):
    """A cached row's page outside the pool, a page to append to outside it, and lengths
    outside [0, capacity]: reported, in bounds, other units as usual."""
    for what in ("row", "append", "length"):
        p = Paged([[[n, n, n + 1]]], 16, 64, F32, spare=1, seed=6, weights=True)
        if what == "row":
            p.pages[0, 0, 0, 1] = p.k.shape[0]
        elif what == "append":
            # row n of unit 0 would open a page (n is no multiple of 16 here, so cut it there)
            p.lens[0, 0, 0] = n // 16 * 16
            p.length[0, 0, 0] = n // 16 * 16
            p.pages[0, 0, 0, n // 16] = -5
        else:
            p.length[0, 0, 0] = -2
        p.k.nan_to_num_(0.0)
        p.v.nan_to_num_(0.0)
        q, kn, vn = _inputs(p, 4, True, 2)
        cache = p.upload()
        err = torch.zeros(1, dtype=torch.int32, device="cuda")
        out, _ = B.reco_paged_decode_attn(cache, q.cuda(), kn.cuda(), vn.cuda(), dev_err=err)
        torch.cuda.synchronize()
        assert err.item() == (5 if what == "length" else 7), what
        got = cache.length.cpu().flatten().tolist()
        assert got == [{"row": n + 1, "append": n // 16 * 16, "length": -2}[what], n + 1, n + 2], what
        for h in (1, 2):
            k, v = p.rows((0, 0, h))
            k, v = torch.cat([k, kn[0, 0, h][None]]), torch.cat([v, vn[0, 0, h][None]])
            ref, _, _ = attend(k, v, q[0, 0, 4 * h:4 * h + 4], k.shape[0] - 1, 1 / 8)
            close_out(out[0, 0, 4 * h:4 * h + 4].cpu(), ref, v, F32, what)
        if what == "length":
            assert torch.equal(out[0, 0, :4].cpu(), vn[0, 0, 0].expand(4, -1))


def test_infinite_and_nan_values_stay_where_they_are_seen():
    """Infinities and NaN in rows outside the window change nothing."""
    p = Paged([[[300]]], 16, 64, BF, spare=1, seed=12)
    for j, x in ((40, math.inf), (201, math.nan), (7, -math.inf)):
        at = p.where((0, 0, 0), [j])
        p.k[at], p.v[at] = x, x
    _check(p, 4, True, sinks=7, window=98)            # sees rows 0..6 and 203..300


def test_lowest_logits():
    """Keys that give logits of -inf have no weight, beside rows and alone in a tile."""
    p = Paged([[[100]]], 16, 64, F32, spare=0, seed=13)
    q = torch.ones((1, 1, 2, 64))
    for j in list(range(0, 40)) + [64]:
        p.k[p.where((0, 0, 0), [j])] = -math.inf
    cache = p.upload()
    out, lse = B.reco_paged_decode_attn(cache, q.cuda())
    k, v = p.rows((0, 0, 0))
    x = torch.where(torch.isinf(k[:, 0].double()), -math.inf, k.double().sum(-1) / 8)
    pr = torch.softmax(x, 0)
    close_out(out[0, 0, 0].cpu(), pr @ v.double(), v, F32, "out")
    close_lse(lse[0, 0, 0].cpu(), torch.logsumexp(x, 0), F32, "lse")


def test_graph_replays_match_eager():
    """Captured calls, replayed with eager work between, against eager ones; two graphs
    with workspaces of their own."""
    lens = np.array([[[700, 90], [33, 1500]]])
    p = Paged(lens, 32, 128, BF, spare=4, seed=21, weights=True)
    q, kn, vn = (x.cuda() for x in _inputs(p, 7, True, 3))
    ref, cap = p.upload(), p.upload()
    start = cap.weight.clone()
    out, lse = torch.empty_like(q), torch.empty(q.shape[:3], device="cuda")
    ws = B.paged_decode_workspace(cap, 14)

    def step():
        B.reco_paged_decode_attn(cap, q, kn, vn, 4, 600, out=out, lse=lse, ws=ws)
        cap.length.sub_(1)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    cap.weight.copy_(start)
    for rep in range(4):
        o, z = B.reco_paged_decode_attn(ref, q, kn, vn, 4, 600)
        ref.length.sub_(1)
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, o) and torch.equal(lse, z), rep
        assert torch.equal(cap.weight.view(torch.int32), ref.weight.view(torch.int32)), rep


def test_same_call_same_bits():
    lens = np.random.RandomState(1).randint(1, 6000, (1, 3, 4))
    p = Paged(lens, 64, 128, BF, spare=1, seed=5, weights=True)
    q, kn, vn = (x.cuda() for x in _inputs(p, 5, True, 3))
    got = []
    for _ in range(3):
        c = p.upload()
        o, z = B.reco_paged_decode_attn(c, q, kn, vn)
        got.append((o, z, c.weight.nan_to_num()))
    for x in got[1:]:
        assert all(torch.equal(a, b) for a, b in zip(x, got[0]))


@pytest.mark.parametrize("batch,G,cap", [(128, 16, 1904), (128, 16, 2096), (130, 16, 640), (130, 16, 800), (128, 4, 7600)])
def test_weights_at_capacities_on_both_sides_of_what_a_workgroup_holds(batch, G, cap):
    lens = np.random.RandomState(cap).randint(0, 150, (1, batch, 2))
    lens[0, 3] = [cap - 1, 0]
    p = Paged(lens, 16, 128, BF, spare=1, seed=cap, weights=True)
    assert p.max_pages * 16 == cap
    _check(p, G, True)
    _check(Paged(lens, 16, 128, BF, spare=1, seed=cap, weights=True), G, True, 3, 70)
