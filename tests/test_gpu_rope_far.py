"""Rotation and append of so many rows that they are read past the caches (64 MiB and more):
against the 64-bit form on tokens of every block's kind, in place and into another tensor."""
import numpy as np
import pytest
import torch

from paged_helpers import Paged
from paper_2608_04771_amd import binding as B
from rope_helpers import close_rows, frequencies, turned

pytestmark = pytest.mark.gpu

F32, BF = torch.float32, torch.bfloat16
FAR = 64 << 20                                             # bytes of rows


def _axes(rot, n):
    return None if n == 1 else [i * n // (rot // 2) for i in range(rot // 2)]


def _some(T, g):
    """The first and last tokens, and others."""
    return sorted({0, 1, 3, 4, T - 6, T - 2, T - 1} | set(torch.randint(0, T, (60,), generator=g).tolist()))


@pytest.mark.parametrize("dtype,D,rot,heads,T,n_axes,pairs", [(BF, 128, 128, 36, 9001, 1, False), (BF, 128, 64, 40, 7003, 3, True),
                                                              (BF, 64, 32, 10, 60001, 2, False), (F32, 128, 128, 10, 14001, 1, True),
                                                              (F32, 64, 64, 36, 8003, 3, False)])
def test_rotations(dtype, D, rot, heads, T, n_axes, pairs):
    assert heads * T * D * (4 if dtype == F32 else 2) > FAR
    g = torch.Generator().manual_seed(T)
    freq = frequencies(rot)
    rope = B.Rope(freq.cuda(), _axes(rot, n_axes), pairs)
    pos = torch.randint(-1000, 900000, (n_axes, 1, T), generator=g, dtype=torch.int32)
    # a projection's rows, the heads of a token beside each other and two more behind them
    x = torch.randn((1, 1, T, heads + 2, D), generator=torch.Generator(device="cuda").manual_seed(T), device="cuda").to(dtype)
    mine, rest = x.transpose(2, 3)[:, :, :heads], x[:, :, :, heads:].clone()
    some = _some(T, g)
    before = mine[:, :, :, some].cpu()
    for n_new in (None, T - 5):
        out = torch.full((1, 1, heads, T, D), 9.0, dtype=dtype, device="cuda")
        n = None if n_new is None else torch.tensor([n_new], dtype=torch.int32).cuda()
        B.reco_rope(rope, mine, pos.cuda(), n, out)
        real = [i for i, t in enumerate(some) if n_new is None or t < n_new]
        want, off = turned(before, pos[:, :, some], freq, _axes(rot, n_axes), pairs)
        close_rows(out[:, :, :, some].cpu()[:, :, :, real], want[:, :, :, real], off[:, :, :, real], f"{n_new} tokens")
        if n_new is not None:
            assert (out[:, :, :, n_new:] == 9).all()
    whole = B.reco_rope(rope, mine, pos.cuda())
    B.reco_rope(rope, mine, pos.cuda(), out=mine)          # in place: the same, and the heads beside them stay
    assert torch.equal(mine, whole) and torch.equal(x[:, :, :, heads:], rest)


@pytest.mark.parametrize("dtype,D,H,G,T,pairs", [(BF, 128, 4, 7, 9001, False), (BF, 64, 2, 4, 45003, True), (F32, 128, 2, 3, 14001, False),
                                                 (F32, 64, 8, 1, 11003, True)])
def test_appends(dtype, D, H, G, T, pairs):
    assert H * (G + 2) * T * D * (4 if dtype == F32 else 2) > FAR
    g = torch.Generator().manual_seed(T)
    lens = np.array([[[19 + 17 * h for h in range(H)]]])
    page = 64
    c = Paged(lens, page, D, dtype, spare=T, seed=1)
    cache = c.upload()
    freq = frequencies(D)
    rope = B.Rope(freq.cuda(), None, pairs)
    pos = torch.randint(0, 900000, (1, T), generator=g, dtype=torch.int32)
    x = torch.randn((1, 1, T, H * (G + 2), D), generator=torch.Generator(device="cuda").manual_seed(T), device="cuda").to(dtype).transpose(2, 3)
    q, kn, vn = x[:, :, :H * G], x[:, :, H * G:H * (G + 1)], x[:, :, H * (G + 1):]
    some = _some(T, g)
    before = x[:, :, :, some].cpu()
    err = torch.zeros(1, dtype=torch.int32, device="cuda")
    qo = B.reco_paged_append(cache, kn, vn, rope, pos.cuda(), q, dev_err=err)
    assert err.item() == 0 and torch.equal(cache.length.cpu(), c.length + T)
    want, off = turned(before, pos[None][:, :, some], freq, pairs=pairs)
    close_rows(qo[:, :, :, some].cpu(), want[:, :, :H * G], off[:, :, :H * G], "queries")
    for h in range(H):
        L = int(lens[0, 0, h])
        at = [y.cuda() for y in c.where((0, 0, h), L + torch.tensor(some))]
        j = H * G + h
        close_rows(cache.k[at[0], at[1]].cpu(), want[0, 0, j], off[0, 0, j], f"keys of {h}")
        every = [y.cuda() for y in c.where((0, 0, h), torch.arange(L + T))]
        v = cache.v[every[0], every[1]]
        assert torch.equal(v[L:], vn[0, 0, h]) and torch.equal(v[:L].cpu(), c.rows((0, 0, h), L)[1])
        assert torch.equal(cache.k[every[0], every[1]][:L].cpu(), c.rows((0, 0, h), L)[0])
    # queries in place: the same ones
    again = c.upload()
    B.reco_paged_append(again, kn, vn, rope, pos.cuda(), q, q_out=q, dev_err=err)
    assert err.item() == 0 and torch.equal(q, qo)
    for h in range(H):
        rows = [y.cuda() for y in c.where((0, 0, h), torch.arange(int(lens[0, 0, h]) + T))]
        assert torch.equal(cache.k[rows[0], rows[1]], again.k[rows[0], rows[1]])
