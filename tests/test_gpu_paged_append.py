"""reco_paged_append: rows put into their pages, keys rotated as the 64-bit form has it."""
import math

import numpy as np
import pytest
import torch

from paged_helpers import Paged, attend, close_lse, close_out
from paper_2608_04771_amd import binding as B
from rope_helpers import close_rows, frequencies, memory_orders, turned

pytestmark = pytest.mark.gpu

F32, BF = torch.float32, torch.bfloat16
KINDS = [(BF, 128, 128, False, 1, 16), (F32, 64, 64, True, 1, 32), (BF, 64, 32, False, 3, 64), (F32, 128, 64, False, 2, 16),
         (BF, 128, 64, True, 1, 4096)]


def _rope(rot, pairs, n_axes):
    freq = frequencies(rot)
    axes = None if n_axes == 1 else [i * n_axes // (rot // 2) for i in range(rot // 2)]
    return freq, axes, B.Rope(freq.cuda(), axes, pairs)


def _up(x):
    return torch.empty_strided(x.shape, x.stride(), dtype=x.dtype, device="cuda").copy_(x)


def _check(c, cache, k, v, koff, news, what):
    """The cache holds what c held and behind it news[b] rows of k (64 bits, off by koff) and v."""
    before = c.lens.copy()
    old = {u: c.rows(u) for u in np.ndindex(before.shape)}
    after = Paged.__new__(Paged)
    after.__dict__.update(c.__dict__)
    after.download(cache)
    for u in np.ndindex(before.shape):
        L, n = int(before[u]), int(news[u[1]])
        assert after.lens[u] == L + n, f"{what}: length of {u}"
        gk, gv = after.rows(u)
        assert torch.equal(gk[:L], old[u][0]) and torch.equal(gv[:L], old[u][1]), f"{what}: rows that {u} had"
        close_rows(gk[L:], k[u][:n], koff[u][:n], f"{what}: keys of {u}") if n else None
        assert torch.equal(gv[L:], v[u][:n]), f"{what}: values of {u}"
        if c.weight is not None:
            assert torch.equal(after.weight[u][:L], c.weight[u][:L]) and (after.weight[u][L:L + n] == 0).all()
    return after


@pytest.mark.parametrize("dtype,D,rot,pairs,n_axes,page", KINDS)
@pytest.mark.parametrize("T", [1, 2, 8, 9, 75])
def test_rows_go_to_their_pages(dtype, D, rot, pairs, n_axes, page, T):
    lens = np.array([[[0, 1], [15, 16], [31, 300]], [[17, 64], [5, 200], [63, 2]]])
    NL, Bs, H = lens.shape
    G = 3
    g = torch.Generator().manual_seed(T + D)
    freq, axes, rope = _rope(rot, pairs, n_axes)
    pos = torch.randint(0, 100000, (n_axes, Bs, T), generator=g, dtype=torch.int32)
    orders = zip(memory_orders((NL, Bs, H, T, D), dtype, g), memory_orders((NL, Bs, H, T, D), dtype, g),
                 memory_orders((NL, Bs, H * G, T, D), dtype, g))
    for i, ((what, kn), (_, vn), (_, q)) in enumerate(orders):
        news = [T, max(0, T - 1 - 3 * i), min(T, 7)]
        c = Paged(lens, page, D, dtype, spare=T, seed=T + i, weights=i % 2 == 0)
        cache = c.upload()
        err = torch.zeros(1, dtype=torch.int32, device="cuda")
        qo = torch.full((NL, Bs, H * G, T, D), 9.0, dtype=dtype, device="cuda")
        got = B.reco_paged_append(cache, _up(kn), _up(vn), rope, pos.cuda(), _up(q),
                                  torch.tensor(news, dtype=torch.int32).cuda(), qo, dev_err=err)
        assert got is qo and err.item() == 0
        want, off = turned(kn, pos, freq, axes, pairs)
        _check(c, cache, want, vn, off, news, what)
        want, off = turned(q, pos, freq, axes, pairs)
        for b in range(Bs):
            close_rows(qo[:, b, :, :news[b]].cpu(), want[:, b, :, :news[b]], off[:, b, :, :news[b]], f"{what}: queries")
            assert (qo[:, b, :, news[b]:] == 9).all()


@pytest.mark.parametrize("dtype,D", [(BF, 128), (F32, 64)])
@pytest.mark.parametrize("T", [None, 1, 20])
def test_without_a_rotation_rows_are_copied(dtype, D, T):
    # bit for bit, infinities and NaN with their payloads
    lens = np.array([[[3, 40]], [[0, 17]]])
    run = () if T is None else (T,)
    g = torch.Generator().manual_seed(2)
    bits = torch.int16 if dtype == BF else torch.int32
    shape = (2, 1, 2, *run, D)
    kn, vn, q = (torch.randint(torch.iinfo(bits).min, torch.iinfo(bits).max, shape, generator=g, dtype=bits) for _ in "kvq")
    c = Paged(lens, 16, D, dtype, spare=T or 1)
    cache = c.upload()
    out = B.reco_paged_append(cache, kn.view(dtype).cuda(), vn.view(dtype).cuda(), q=q.view(dtype).cuda())
    assert torch.equal(out.cpu().view(bits), q)
    after = c.download(cache)
    for u in np.ndindex(lens.shape):
        L = int(lens[u])
        for rows, new in zip(after.rows(u), (kn, vn)):
            assert torch.equal(rows[L:].reshape(-1).view(bits), new[u].reshape(-1)), u


def test_a_range_of_layers():
    lens = np.array([[[4, 9]], [[20, 1]], [[0, 33]]])
    g = torch.Generator().manual_seed(8)
    c = Paged(lens, 16, 64, F32, spare=3)
    kn, vn = (torch.randn((1, 1, 2, 3, 64), generator=g) for _ in "kv")
    freq, axes, rope = _rope(64, False, 1)
    pos = torch.tensor([[7, 8, 9]], dtype=torch.int32)
    cache = c.upload()
    B.reco_paged_append(cache, kn.cuda(), vn.cuda(), rope, pos.cuda(), layer0=1, n_layers=1)
    n = cache.length.cpu()
    assert torch.equal(n[[0, 2]], c.length[[0, 2]]) and torch.equal(n[1], c.length[1] + 3)
    want, off = turned(kn, pos[None], freq)
    c.download(cache)
    for h in range(2):
        L = int(lens[1, 0, h])
        close_rows(c.rows((1, 0, h))[0][L:], want[0, 0, h], off[0, 0, h], "keys")


@pytest.mark.parametrize("T", [2, 40])
def test_what_cannot_be_appended_is_not(T):
    # each unit's trouble is its own: the others are appended, the queries written
    H, D, page = 6, 64, 16
    lens = np.array([[[10, 96 - T + 1, 5, 17, 8, 96 - T]]])
    c = Paged(lens, page, D, F32, spare=T, weights=True)
    assert c.max_pages == 96 // page + 1
    c.max_pages = 96 // page                               # a run of unit 1 ends past its capacity
    c.pages = c.pages[..., :c.max_pages].contiguous()
    c.weight = c.weight[..., :96].contiguous()
    c.pages[0, 0, 2, (5 + T - 1) // page] = c.k.shape[0]   # unit 2: the last new row's page is bad
    c.length[0, 0, 3], c.length[0, 0, 4] = -1, 97
    g = torch.Generator().manual_seed(9)
    kn, vn, q = (torch.randn((1, 1, H, T, D), generator=g) for _ in "kvq")
    freq, axes, rope = _rope(64, False, 1)
    pos = torch.arange(T, dtype=torch.int32)[None]
    for unit, code in ((1, 1), (2, 7), (3, 5), (4, 5)):
        one = B.PagedKVCache(c.k.cuda(), c.v.cuda(), c.pages[:, :, unit:unit + 1].contiguous().cuda(),
                             c.length[:, :, unit:unit + 1].contiguous().cuda(), c.weight[:, :, unit:unit + 1].contiguous().cuda())
        err = torch.zeros(1, dtype=torch.int32, device="cuda")
        B.reco_paged_append(one, kn[:, :, :1].contiguous().cuda(), vn[:, :, :1].contiguous().cuda(), rope, pos.cuda(), dev_err=err)
        assert err.item() == code and one.length.item() == c.length[0, 0, unit]
    cache = c.upload()
    err = torch.zeros(1, dtype=torch.int32, device="cuda")
    qo = B.reco_paged_append(cache, kn.cuda(), vn.cuda(), rope, pos.cuda(), q.cuda(), dev_err=err)
    assert err.item() in (1, 5, 7)
    want, off = turned(q, pos[None], freq)
    close_rows(qo.cpu(), want, off, "queries")
    n, k, v = cache.length.cpu(), cache.k.cpu(), cache.v.cpu()
    assert torch.equal(n[0, 0, 1:5], c.length[0, 0, 1:5]) and n[0, 0, 0] == 10 + T and n[0, 0, 5] == 96
    want, off = turned(kn, pos[None], freq)
    for h in (0, 5):
        L = int(lens[0, 0, h])
        at = c.where((0, 0, h), torch.arange(L, L + T))
        close_rows(k[at], want[0, 0, h], off[0, 0, h], f"keys of {h}")
        assert torch.equal(v[at], vn[0, 0, h])
    # a bad count appends nothing and says so
    cache = c.upload()
    err.zero_()
    B.reco_paged_append(cache, kn.cuda(), vn.cuda(), rope, pos.cuda(), n_new=torch.tensor([T + 1], dtype=torch.int32).cuda(), dev_err=err)
    assert err.item() == 5 and torch.equal(cache.length.cpu(), c.length)


@pytest.mark.parametrize("dtype,D,G", [(BF, 128, 4), (F32, 64, 7)])
def test_a_prompt_and_tokens_through_them(dtype, D, G):
    """As a model's layer calls them: a prompt's queries and keys rotated, attended and appended by the
    prefill, then tokens appended with their rotation and attended."""
    NL, Bs, H, page = 1, 2, 2, 16
    g = torch.Generator().manual_seed(D)
    freq, axes, rope = _rope(D, False, 1)
    c = Paged(np.zeros((NL, Bs, H), dtype=np.int64), page, D, dtype, spare=80, seed=1)
    cache = c.upload()
    news = [50, 33]
    fused = torch.randn((NL, Bs, 50, H * (G + 2), D), generator=g).to(dtype)
    dev = fused.cuda().transpose(2, 3)
    pos = torch.arange(50, dtype=torch.int32).expand(Bs, 50).contiguous()
    n = torch.tensor(news, dtype=torch.int32).cuda()
    err = torch.zeros(1, dtype=torch.int32, device="cuda")
    both = B.reco_rope(rope, dev[:, :, :H * (G + 1)], pos.cuda(), n)
    q, kn = both[:, :, :H * G].contiguous(), both[:, :, H * G:].contiguous()
    vn = dev[:, :, H * (G + 1):].contiguous()
    scale = 1 / math.sqrt(D)
    out, lse = B.reco_paged_prefill_attn(cache, q, kn, vn, n, dev_err=err)
    K = {u: kn[u].cpu()[:news[u[1]]] for u in np.ndindex(NL, Bs, H)}
    V = {u: vn[u].cpu()[:news[u[1]]] for u in np.ndindex(NL, Bs, H)}
    want, off = turned(fused.transpose(2, 3), pos[None], freq)
    for u in K:
        close_rows(K[u], want[u[0], u[1], H * G + u[2], :news[u[1]]], off[u[0], u[1], H * G + u[2], :news[u[1]]], "prompt")
    call = None
    at = torch.zeros((Bs,), dtype=torch.int32, device="cuda")
    qo = torch.empty((NL, Bs, H * G, D), dtype=dtype, device="cuda")
    for i in range(4):
        fused = torch.randn((NL, Bs, H * (G + 2), D), generator=g).to(dtype)
        dev = fused.cuda()
        at.copy_(torch.tensor(news, dtype=torch.int32) + i)
        if call is None:
            call = B.PreparedPagedAppend(cache, None, rope, at, qo, dev_err=err)
        call(dev[:, :, H * G:H * (G + 1)], dev[:, :, H * (G + 1):], dev[:, :, :H * G])
        o, z = B.reco_paged_decode_attn(cache, qo, dev_err=err)
        want, off = turned(fused[:, :, :, None], at.cpu()[None, :, None], freq)
        after = c.download(cache)
        for u in K:
            k, v = after.rows(u)
            assert torch.equal(k[:-1], K[u]) and torch.equal(v[:-1], V[u])
            j = H * G + u[2]
            close_rows(k[-1], want[u[0], u[1], j, 0], off[u[0], u[1], j, 0], "key")
            assert torch.equal(v[-1], fused[u[0], u[1], j + H])
            K[u], V[u] = k, v
            heads = slice(u[2] * G, (u[2] + 1) * G)
            ro, rz, _ = attend(k, v, qo[u[:2]][heads].cpu(), k.shape[0] - 1, scale)
            close_out(o[u[:2]][heads].cpu(), ro, v, dtype, f"token {i}")
            close_lse(z[u[:2]][heads].cpu(), rz, dtype, f"token {i}")
    assert err.item() == 0


def test_captured_beside_eager():
    g = torch.Generator().manual_seed(6)
    NL, Bs, H, G, D, page = 2, 3, 2, 2, 128, 16
    lens = np.full((NL, Bs, H), 20)
    freq, axes, rope = _rope(D, False, 2)
    a, b = (Paged(lens, page, D, BF, spare=60, seed=4).upload() for _ in "ab")
    pos = torch.zeros((2, Bs, 10), dtype=torch.int32, device="cuda")
    x = torch.zeros((NL, Bs, 10, H * (G + 2), D), dtype=BF, device="cuda").transpose(2, 3)
    parts = (x[:, :, H * G:H * (G + 1)], x[:, :, H * (G + 1):], x[:, :, :H * G])
    qa, qb = (torch.zeros((NL, Bs, H * G, 10, D), dtype=BF, device="cuda") for _ in "ab")
    call = B.PreparedPagedAppend(a, 10, rope, pos, qa)
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        call(*parts)
    for i in range(4):
        pos.copy_(torch.randint(0, 9000, pos.shape, generator=g, dtype=torch.int32))
        x.copy_(torch.randn(x.shape, generator=g).to(BF))
        torch.cuda.synchronize()
        with torch.cuda.stream(s):
            graph.replay()
        B.reco_paged_append(b, *parts[:2], rope, pos, parts[2], q_out=qb)
        torch.cuda.synchronize()
        assert torch.equal(a.length, b.length) and a.length.eq(20 + 10 * (i + 1)).all()
        for y, z in ((a.k, b.k), (a.v, b.v), (qa, qb)):
            assert torch.equal(y.view(torch.int16), z.view(torch.int16)), f"replay {i}"


@pytest.mark.parametrize("T", [1, 8, 9])
def test_the_most_heads(T):
    H, D = 1024, 64
    g = torch.Generator().manual_seed(T)
    c = Paged(np.arange(H)[None, None] % 40, 16, D, F32, spare=T, seed=T)
    kn, vn = (torch.randn((1, 1, H, T, D), generator=g) for _ in "kv")
    freq, axes, rope = _rope(D, False, 1)
    pos = torch.arange(100, 100 + T, dtype=torch.int32)[None]
    cache = c.upload()
    err = torch.zeros(1, dtype=torch.int32, device="cuda")
    B.reco_paged_append(cache, kn.cuda(), vn.cuda(), rope, pos.cuda(), dev_err=err)
    assert err.item() == 0
    want, off = turned(kn, pos[None], freq)
    _check(c, cache, want, vn, off, [T], "heads")


def test_pages_past_four_gibibytes():
    # 4,200 pages of 1 MiB in each pool, of which the last are in use
    page, n_pages, T = 4096, 4200, 30
    c = Paged(np.array([[[4090, 0]]]), page, 128, BF, spare=T, seed=3)
    have = c.k.shape[0]
    pools = [torch.empty((n_pages, page, 128), dtype=BF, device="cuda") for _ in "kv"]
    for pool, x in zip(pools, (c.k, c.v)):
        pool[n_pages - have:] = x.cuda()
    table = torch.where((c.pages >= 0) & (c.pages < have), c.pages + (n_pages - have), c.pages)
    g = torch.Generator().manual_seed(1)
    kn, vn = (torch.randn((1, 1, 2, T, 128), generator=g).to(BF) for _ in "kv")
    freq, axes, rope = _rope(128, False, 1)
    pos = torch.arange(T, dtype=torch.int32)[None]
    for some in (slice(0, T), slice(0, 1)):                # a long run, and one that is a workgroup's
        cache = B.PagedKVCache(*pools, table.cuda(), c.length.cuda())
        k, v, p = kn[:, :, :, some].contiguous(), vn[:, :, :, some].contiguous(), pos[:, some].contiguous()
        B.reco_paged_append(cache, k.cuda(), v.cuda(), rope, p.cuda())
        want, off = turned(k, p[None], freq)
        after = B.PagedKVCache(pools[0][n_pages - have:].clone(), pools[1][n_pages - have:].clone(), c.pages.cuda(), cache.length)
        _check(c, after, want, v, off, [k.shape[3]], str(some))


@pytest.mark.parametrize("dtype,D", [(BF, 128), (F32, 64)])
@pytest.mark.parametrize("T", [None, 1, 8, 21])
def test_a_projection_rotated_where_it_lies(dtype, D, T):
    # queries in place, keys and values from the heads beside them, which stay as they are
    NL, Bs, H, G = 2, 3, 2, 3
    g = torch.Generator().manual_seed(5)
    n = T or 1
    fused = torch.randn((NL, Bs, n, H * (G + 2), D), generator=g).to(dtype)
    dev = fused.cuda().transpose(2, 3)
    x = dev if T else dev[:, :, :, 0]
    c = Paged(np.array([[[3, 15], [0, 40], [16, 1]]] * NL), 16, D, dtype, spare=n, seed=2)
    cache = c.upload()
    freq, axes, rope = _rope(D, True, 1)
    pos = torch.randint(-50, 5000, (Bs, n), generator=g, dtype=torch.int32)
    q, kn, vn = x[:, :, :H * G], x[:, :, H * G:H * (G + 1)], x[:, :, H * (G + 1):]
    for bad in (kn, x[:, :, 1:1 + H * G], x[:, :, 2 * H:2 * H + H * G]):
        if bad.shape == q.shape:
            with pytest.raises(ValueError, match="q_out"):
                B.reco_paged_append(cache, kn, vn, rope, pos.cuda(), q, q_out=bad)
    got = B.reco_paged_append(cache, kn, vn, rope, pos.cuda(), q, q_out=q)
    assert got.data_ptr() == q.data_ptr()
    want, off = turned(fused.transpose(2, 3), pos[None], freq, pairs=True)
    close_rows(dev[:, :, :H * G].cpu(), want[:, :, :H * G], off[:, :, :H * G], "queries")
    assert torch.equal(dev[:, :, H * G:].cpu(), fused.transpose(2, 3)[:, :, H * G:])
    _check(c, cache, want[:, :, H * G:H * (G + 1)], fused.transpose(2, 3)[:, :, H * (G + 1):], off[:, :, H * G:H * (G + 1)], [n] * Bs, "fused")
