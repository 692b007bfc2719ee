"""reco_paged_evict against a plain form: which rows are kept, where they go, what
is left untouched.  Everything is whole numbers and copied bits: all exact."""
import numpy as np
import pytest
import torch

from paged_helpers import Paged
from paper_2608_04771_amd import binding as B

pytestmark = pytest.mark.gpu

F32, BF = torch.float32, torch.bfloat16


def _kept(w, L, m, sinks, recent):
    """The kept rows of a unit of L rows with weights w, ascending."""
    if L <= m:
        return np.arange(L)
    mid = np.arange(sinks, L - recent)
    order = np.lexsort((mid, -w[mid].astype(np.float64)))         # largest first, then the lower row
    best = mid[order[:m - sinks - recent]]
    return np.concatenate([np.arange(sinks), np.sort(best), np.arange(L - recent, L)])


def _check(p, budget, sinks=0, recent=0, give_idx=True, bad=(), expect_err=0, layer0=0, n_layers=None):
    NL, Bs, H = p.lens.shape
    nl = NL - layer0 if n_layers is None else n_layers
    budget = torch.as_tensor(budget, dtype=torch.int32)
    cache = p.upload()
    cap = p.max_pages * p.page
    kept = torch.full((nl, Bs, H, cap), -7, dtype=torch.int32, device="cuda") if give_idx else None
    err = torch.zeros(1, dtype=torch.int32, device="cuda")
    B.reco_paged_evict(cache, budget.cuda(), sinks, recent, kept_idx=kept, layer0=layer0, n_layers=n_layers, dev_err=err)
    torch.cuda.synchronize()
    assert err.item() == expect_err
    k0, v0, w0, n0 = p.k.clone(), p.v.clone(), p.weight.clone(), p.length.clone()
    for u in np.ndindex(NL, Bs, H):
        L = int(p.lens[u])
        if not layer0 <= u[0] < layer0 + nl or u in bad:
            continue
        m = int(budget[u[1]] if budget.dim() == 1 else budget[u[0] - layer0, u[1]])
        idx = _kept(p.weight[u].numpy(), L, m, sinks, recent)
        if kept is not None:
            got = kept[(u[0] - layer0,) + u[1:]].cpu().numpy()
            assert (got[:len(idx)] == idx).all(), f"unit {u}"
            assert (got[len(idx):] == -7).all(), f"unit {u}: entries past the kept rows"
        src, dst = p.where(u, idx), p.where(u, np.arange(len(idx)))
        k0[dst], v0[dst] = p.k[src], p.v[src]
        w0[u][:len(idx)] = p.weight[u][torch.from_numpy(idx)]
        n0[u] = len(idx)
    assert torch.equal(cache.length.cpu(), n0)
    for name, a, b in (("K", cache.k, k0), ("V", cache.v, v0), ("weight", cache.weight, w0)):
        assert torch.equal(a.cpu().view(torch.int8), b.view(torch.int8)), name
    return cache


LENS = np.array([0, 1, 15, 16, 17, 100, 128, 129, 500, 1000, 63, 64, 65, 300, 999, 1040]).reshape(2, 2, 4)


@pytest.mark.parametrize("dtype,D,page", [(F32, 64, 16), (F32, 128, 64), (BF, 64, 256), (BF, 128, 16), (BF, 128, 4096)])
@pytest.mark.parametrize("budget,sinks,recent", [(64, 0, 0), (100, 4, 32), (20, 4, 16), (1, 1, 0), (1, 0, 1), (999, 3, 7),
                                                 (5000, 4, 4), (128, 0, 64), (128, 128, 0)])
def test_ragged_units(dtype, D, page, budget, sinks, recent):
    p = Paged(LENS, page, D, dtype, seed=budget + D, weights=True)
    _check(p, [budget, budget + 1], sinks, recent)


@pytest.mark.parametrize("L,m", [(16384, 9516), (16385, 16384), (20000, 300), (40001, 39000), (16383, 1)])
def test_long_units(L, m):
    """Around what a workgroup holds in registers, and far past it."""
    p = Paged([[[L, L // 2]]], 64, 64, BF, seed=L, weights=True)
    _check(p, [m], 0, 1)


def test_few_to_evict_in_many_units():
    lens = np.random.RandomState(4).randint(500, 560, (3, 25, 8))
    p = Paged(lens, 16, 64, BF, seed=3, weights=True)
    _check(p, np.random.RandomState(5).randint(490, 560, (3, 25)), 4, 30, give_idx=False)


def test_ties_and_extremes():
    """Equal weights go by the lower row; zeros of either sign are equal; +inf is the largest."""
    p = Paged([[[400, 400, 400]]], 16, 64, F32, seed=1, weights=True)
    p.weight[0, 0, 0][:400] = 1.0
    p.weight[0, 0, 1][:400] = torch.randint(0, 3, (400,)).float()
    z = p.weight[0, 0, 2][:400]
    z[:] = 0.0
    z[::3] = -0.0
    z[250], z[251] = float("inf"), 1e-45
    _check(p, [150], 2, 10)


def test_weights_outside_the_choice_are_not_read():
    """NaN and negative weights of sinks, recent rows and of units that keep everything."""
    p = Paged([[[100, 40]]], 16, 64, F32, seed=1, weights=True)
    p.weight[0, 0, 0][:4] = float("nan")
    p.weight[0, 0, 0][90:100] = -1.0
    p.weight[0, 0, 1][:40] = -float("inf")
    _check(p, [50], 4, 10)


def test_layers_and_budgets_per_layer():
    p = Paged(np.full((4, 2, 3), 90), 16, 64, BF, seed=2, weights=True)
    _check(p, [[50, 60], [70, 33]], 1, 8, layer0=1, n_layers=2)


@pytest.mark.parametrize("what,code", [("budget", 8), ("zero", 8), ("length", 5), ("weight", 3), ("negative", 3), ("page", 7)])
def test_bad_units_are_left_unchanged(what, code):
    p = Paged([[[120, 120]], [[120, 120]]], 16, 64, F32, seed=6, weights=True)
    budget = [[50], [50]]
    bad = ((1, 0, 0), (1, 0, 1)) if what in ("budget", "zero") else ((0, 0, 1),)
    if what == "budget":
        budget[1] = [11]
    elif what == "zero":
        budget[1] = [0]
    elif what == "length":
        p.length[0, 0, 1] = p.max_pages * p.page + 1
    elif what == "weight":
        p.weight[0, 0, 1, 60] = float("nan")
    elif what == "negative":
        p.weight[0, 0, 1, 60] = -1e-30
    else:
        p.pages[0, 0, 1, 6] = -1
    _check(p, budget, 4, 8, bad=bad, expect_err=code)


def test_graph_replays_match_eager():
    p = Paged(np.array([[[700, 90], [333, 1500]]]), 32, 128, BF, seed=21, weights=True)
    a, b = p.upload(), p.upload()
    w0, n0 = b.weight.clone(), b.length.clone()
    budget = torch.tensor([80, 300], dtype=torch.int32, device="cuda")
    ws = torch.empty(B.paged_evict_workspace_size(b), dtype=torch.uint8, device="cuda")

    def step(c):
        c.weight.copy_(w0)
        c.length.copy_(n0)
        B.reco_paged_evict(c, budget, 4, 16, ws=ws if c is b else None)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step(b)
    torch.cuda.current_stream().wait_stream(side)
    step(a)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(b)
    for rep in range(4):
        graph.replay()
        torch.cuda.synchronize()
        step(a)
        torch.cuda.synchronize()
        for x, y in ((a.k, b.k), (a.v, b.v), (a.weight, b.weight), (a.length, b.length)):
            assert torch.equal(x.view(torch.int8), y.view(torch.int8)), rep
