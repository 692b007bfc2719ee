"""reco_rope against the rotation in 64 bits."""
import numpy as np
import pytest
import torch

from paper_2608_04771_amd import binding as B
from rope_helpers import close_rows, frequencies, memory_orders, turned

pytestmark = pytest.mark.gpu

F32, BF = torch.float32, torch.bfloat16
# dtype, D, rot, pairs, axes
KINDS = [(BF, 128, 128, False, 1), (BF, 128, 64, True, 1), (F32, 64, 64, False, 1), (F32, 128, 32, False, 3), (BF, 64, 16, False, 2),
         (F32, 64, 48, True, 2), (BF, 128, 96, False, 4), (BF, 64, 64, True, 3), (F32, 128, 128, True, 1)]


def _rope(rot, pairs, n_axes, base=1e4):
    freq = frequencies(rot, base)
    axes = None if n_axes == 1 else [i % n_axes for i in range(rot // 2)]
    return freq, axes, B.Rope(freq.cuda(), axes, pairs)


@pytest.mark.parametrize("dtype,D,rot,pairs,n_axes", KINDS)
@pytest.mark.parametrize("NL,Bs,H,T", [(1, 1, 1, 1), (2, 3, 5, 7), (1, 2, 36, 9), (1, 1, 3, 130)])
def test_rotates_every_order_of_memory(dtype, D, rot, pairs, n_axes, NL, Bs, H, T):
    g = torch.Generator().manual_seed(D + rot + T)
    freq, axes, rope = _rope(rot, pairs, n_axes)
    pos = torch.randint(-5000, 200000, (n_axes, Bs, T), generator=g, dtype=torch.int32)
    for what, x in memory_orders((NL, Bs, H, T, D), dtype, g):
        want, off = turned(x, pos, freq, axes, pairs)
        dev = torch.empty_strided(x.shape, x.stride(), dtype=dtype, device="cuda").copy_(x)
        got = B.reco_rope(rope, dev, pos.cuda())
        assert torch.equal(dev.cpu(), x), what             # the input stays
        close_rows(got.cpu(), want, off, what)
        assert torch.equal(got.cpu()[..., rot:], x[..., rot:]), f"{what}: the rest of a row passes"
        assert B.reco_rope(rope, dev, pos.cuda(), out=dev) is dev
        assert torch.equal(dev, got), f"{what}: in place"


@pytest.mark.parametrize("dtype,D,rot,pairs,n_axes", KINDS[:4])
def test_places_past_a_sequences_tokens(dtype, D, rot, pairs, n_axes):
    NL, Bs, H, T = 2, 5, 3, 11
    g = torch.Generator().manual_seed(1)
    freq, axes, rope = _rope(rot, pairs, n_axes)
    x = torch.randn((NL, Bs, H, T, D), generator=g).to(dtype)
    pos = torch.randint(0, 4000, (n_axes, Bs, T), generator=g, dtype=torch.int32)
    n = [11, 0, 1, 8, 9]
    want, off = turned(x, pos, freq, axes, pairs)
    for b in range(Bs):
        x[:, b, :, n[b]:] = float("nan")
        pos[:, b, n[b]:] = -2 ** 31
    out = torch.full(x.shape, 7.0, dtype=dtype, device="cuda")
    err = torch.zeros(1, dtype=torch.int32, device="cuda")
    B.reco_rope(rope, x.cuda(), pos.cuda(), torch.tensor(n, dtype=torch.int32).cuda(), out, err)
    assert err.item() == 0
    for b in range(Bs):
        close_rows(out[:, b, :, :n[b]].cpu(), want[:, b, :, :n[b]], off[:, b, :, :n[b]], f"sequence {b}")
        assert (out[:, b, :, n[b]:] == 7).all()
    # bad counts are none
    out.fill_(7.0)
    B.reco_rope(rope, x.cuda(), pos.cuda(), torch.tensor([12, -1, 1, 0, 2 ** 31 - 1], dtype=torch.int32).cuda(), out, err)
    assert err.item() == 5                                 # RECO_DEV_BAD_LENGTH
    assert (out[:, [0, 1, 3, 4]] == 7).all() and (out[:, 2, :, 0] != 7).any() and (out[:, 2, :, 1:] == 7).all()


@pytest.mark.parametrize("dtype", [F32, BF])
def test_far_positions_and_odd_values(dtype):
    # the largest positions, frequencies above one and zero; infinities and NaN stay in their pairs
    g = torch.Generator().manual_seed(3)
    D = rot = 64
    freq = torch.cat([torch.tensor([0.0, 1.0, 3.7, 6.2831855]), frequencies(56, 1e7)])
    rope = B.Rope(freq.cuda())
    at = [0, 1, -1, 10 ** 6, 2 ** 24 + 1, -(2 ** 24) - 1, 2 ** 31 - 1, -2 ** 31]
    pos = torch.tensor(at, dtype=torch.int32).reshape(1, 1, -1)
    x = torch.randn((1, 1, 2, len(at), D), generator=g).to(dtype)
    want, off = turned(x, pos, freq)
    got = B.reco_rope(rope, x.cuda(), pos[0].cuda()).cpu()
    close_rows(got, want, off, "far positions")
    assert torch.equal(got[..., 0, :], x[..., 0, :])       # position 0 turns nothing
    odd = x.clone()
    odd[..., 5], odd[..., 7 + rot // 2] = float("inf"), float("nan")
    bad = B.reco_rope(rope, odd.cuda(), pos[0].cuda()).cpu()
    keep = torch.ones(D, dtype=torch.bool)
    keep[[5, 5 + rot // 2, 7, 7 + rot // 2]] = False
    assert torch.equal(bad[..., keep], got[..., keep])


def test_the_rotation_back_is_its_gradient():
    # <R x, y> = <x, R^T y>, and R^T is the rotation by -p; differences of R x agree with it
    g = torch.Generator().manual_seed(4)
    freq, axes, rope = _rope(64, False, 2)
    x, y = (torch.randn((1, 2, 3, 6, 64), generator=g) for _ in "xy")
    pos = torch.randint(0, 3000, (2, 2, 6), generator=g, dtype=torch.int32)
    back = B.reco_rope(rope, y.cuda(), -pos.cuda()).cpu()
    want, off = turned(y, -pos, freq, axes)
    close_rows(back, want, off, "back")
    there = B.reco_rope(rope, B.reco_rope(rope, x.cuda(), pos.cuda()), -pos.cuda()).cpu()
    # twice the rotation's error, of elements within |x| + |y| of their pair
    assert (there - x).abs().max() <= 2 * (2.2e-7 + 2.0 ** -23) * 2 * x.abs().max() * 2
    step = 2.0 ** -4                                       # exact in fp32: the rotation is linear
    for e in (0, 17, 33, 63):
        dx = torch.zeros_like(x)
        dx[..., e] = step
        up, down = (B.reco_rope(rope, (x + k * dx).cuda(), pos.cuda()).double().cpu() for k in (1, -1))
        slope = ((up - down) * y.double()).sum(-1) / (2 * step)
        # each of the row's elements is off by the rotation's error of |x| + |y| + step, and |y| weighs it
        most = (2 * off.amax() + 1e-6) * y.abs().sum(-1).double() / step
        assert ((slope - want[..., e]).abs() <= most).all()


def test_graphs_streams_and_prepared_calls():
    g = torch.Generator().manual_seed(5)
    freq, axes, rope = _rope(128, False, 3)
    x = torch.randn((1, 4, 6, 20, 128), generator=g).to(BF).cuda()
    pos = torch.zeros((3, 4, 20), dtype=torch.int32, device="cuda")
    n = torch.full((4,), 20, dtype=torch.int32, device="cuda")
    out = torch.zeros_like(x)
    call = B.PreparedRope(rope, pos, out, n)
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        call(x)
    for i in range(3):                                     # replays see new positions, counts and rows
        at = torch.randint(0, 9000, pos.shape, generator=g, dtype=torch.int32)
        k = torch.tensor([20, 3 + i, 0, 19], dtype=torch.int32)
        y = torch.randn(x.shape, generator=g).to(BF)
        pos.copy_(at), n.copy_(k), x.copy_(y), out.fill_(3.0)
        torch.cuda.synchronize()
        with torch.cuda.stream(s):
            graph.replay()
        torch.cuda.synchronize()
        want, off = turned(y, at, freq, axes)
        for b in range(4):
            close_rows(out[:, b, :, :k[b]].cpu(), want[:, b, :, :k[b]], off[:, b, :, :k[b]], f"replay {i}")
            assert (out[:, b, :, k[b]:] == 3).all()
        eager = torch.full_like(out, 3.0)
        assert torch.equal(B.reco_rope(rope, x, pos, n, eager), out)


def test_heads_past_4_gib():
    # rows whose offsets pass 32 bits give what the same rows give alone
    freq, axes, rope = _rope(128, False, 1)
    far = 2 ** 31 + 4096                                   # elements of bf16: 4 GiB
    pool = torch.empty(far + 8 * 128, dtype=BF, device="cuda")
    x = torch.randn((2, 4, 128)).to(BF).cuda()
    pool[:4 * 128] = x[0].reshape(-1)
    pool[far:far + 4 * 128] = x[1].reshape(-1)
    rows = pool.as_strided((1, 1, 2, 4, 128), (far, far, far, 128, 1))
    pos = torch.tensor([[0, 3, 70, 9000]], dtype=torch.int32).cuda()
    alone = B.reco_rope(rope, x.reshape(1, 1, 2, 4, 128), pos)
    assert torch.equal(B.reco_rope(rope, rows, pos), alone)
    assert torch.equal(B.reco_rope(rope, rows, pos, out=rows), alone)
