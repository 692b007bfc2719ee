"""The paged operators as a program uses them together: a prompt is run, tokens are
decoded with their attention weights kept, rows are evicted, freed pages serve another
sequence, decoding goes on and a probe is run.  Every step is checked against the plain
64-bit form on rows that this file keeps itself."""
import math

import numpy as np
import pytest
import torch

from paged_helpers import attend, close_lse, close_out, close_weight
from paper_2608_04771_amd import binding as B

pytestmark = pytest.mark.gpu

F32, BF = torch.float32, torch.bfloat16


class Run:
    """A GPU cache with a page allocator, and every unit's rows on the CPU."""

    def __init__(self, NL, Bs, H, G, D, page, cap, dtype, n_pages, sinks=0, window=0, seed=0):
        self.G, self.D, self.page, self.dtype, self.sinks, self.window = G, D, page, dtype, sinks, window
        self.shape = (NL, Bs, H)
        self.g = torch.Generator().manual_seed(seed)
        self.free = np.random.RandomState(seed).permutation(n_pages).tolist()
        self.table = torch.full((NL, Bs, H, cap // page), -1, dtype=torch.int32)
        pool = [torch.full((n_pages, page, D), float("nan"), dtype=dtype, device="cuda") for _ in "kv"]
        self.cache = B.PagedKVCache(*pool, self.table.cuda(), torch.zeros(self.shape, dtype=torch.int32, device="cuda"),
                                    torch.full((NL, Bs, H, cap), float("nan"), device="cuda"))
        self.k = {u: torch.zeros((0, D), dtype=dtype) for u in np.ndindex(self.shape)}
        self.v = dict(self.k)
        self.w = {u: torch.zeros(0, dtype=torch.float64) for u in self.k}
        self.err = torch.zeros(1, dtype=torch.int32, device="cuda")
        self.scale = 1 / math.sqrt(D)

    def lists(self, more):
        """Gives every unit of sequence b pages for its rows and more[b], takes the others back."""
        for u in self.k:
            rows = self.k[u].shape[0] + more[u[1]]
            for i in range(self.table.shape[3]):
                if i * self.page < rows and self.table[u][i] < 0:
                    self.table[u][i] = self.free.pop()
                elif i * self.page >= rows and self.table[u][i] >= 0:
                    self.free.append(int(self.table[u][i]))
                    self.table[u][i] = -1
        self.cache.pages.copy_(self.table)

    def randn(self, *shape):
        return torch.randn(shape, generator=self.g).to(self.dtype)

    def _compare(self, what, u, t, q, got, lse):
        """Token t of the unit's newest rows; its probabilities."""
        o, z, p = attend(self.k[u], self.v[u], q, t, self.scale, self.sinks, self.window)
        close_out(got, o, self.v[u], self.dtype, f"{what} unit {u} row {t}")
        close_lse(lse, z, self.dtype, f"{what} unit {u} row {t}")
        return p

    def prefill(self, news, what):
        NL, Bs, H = self.shape
        T = max(news)
        self.lists(news)
        q, kn, vn = self.randn(NL, Bs, H * self.G, T, self.D), self.randn(NL, Bs, H, T, self.D), self.randn(NL, Bs, H, T, self.D)
        out, lse = B.reco_paged_prefill_attn(self.cache, q.cuda(), kn.cuda(), vn.cuda(),
                                             torch.tensor(news, dtype=torch.int32).cuda(), self.sinks, self.window,
                                             dev_err=self.err)
        out, lse = out.cpu(), lse.cpu()
        for u in self.k:
            n, L = news[u[1]], self.k[u].shape[0]
            self.k[u], self.v[u] = torch.cat([self.k[u], kn[u][:n]]), torch.cat([self.v[u], vn[u][:n]])
            self.w[u] = torch.cat([self.w[u], torch.zeros(n, dtype=torch.float64)])
            heads = slice(u[2] * self.G, (u[2] + 1) * self.G)
            for t in range(0, n, 7):
                self._compare(what, u, L + t, q[u[:2]][heads, t], out[u[:2]][heads, t], lse[u[:2]][heads, t])
        self.same(what)

    def decode(self, what):
        NL, Bs, H = self.shape
        self.lists([1] * Bs)
        q, kn, vn = self.randn(NL, Bs, H * self.G, self.D), self.randn(NL, Bs, H, self.D), self.randn(NL, Bs, H, self.D)
        out, lse = B.reco_paged_decode_attn(self.cache, q.cuda(), kn.cuda(), vn.cuda(), self.sinks, self.window,
                                            dev_err=self.err)
        out, lse = out.cpu(), lse.cpu()
        for u in self.k:
            self.k[u], self.v[u] = torch.cat([self.k[u], kn[u][None]]), torch.cat([self.v[u], vn[u][None]])
            heads = slice(u[2] * self.G, (u[2] + 1) * self.G)
            p = self._compare(what, u, self.k[u].shape[0] - 1, q[u[:2]][heads], out[u[:2]][heads], lse[u[:2]][heads])
            self.w[u] = torch.cat([self.w[u], torch.zeros(1, dtype=torch.float64)]) + p
        self.same(what)

    def evict(self, budget, sinks, recent, what):
        before = self.cache.weight.cpu()
        idx = torch.full(self.cache.weight.shape, -7, dtype=torch.int32, device="cuda")
        B.reco_paged_evict(self.cache, torch.tensor(budget, dtype=torch.int32).cuda(), sinks, recent, kept_idx=idx,
                           dev_err=self.err)
        idx = idx.cpu()
        for u in self.k:
            L, m = self.k[u].shape[0], budget[u[1]]
            keep = np.arange(L)
            if L > m:                                      # by the weights the GPU had, ties to the lower row
                mid = np.arange(sinks, L - recent)
                best = mid[np.argsort(-before[u][:L].numpy()[mid], kind="stable")[:m - sinks - recent]]
                keep = np.sort(np.concatenate([np.arange(sinks), best, np.arange(L - recent, L)]))
            assert idx[u][:len(keep)].tolist() == keep.tolist(), f"{what} unit {u}"
            keep = torch.from_numpy(keep)
            self.k[u], self.v[u], self.w[u] = self.k[u][keep], self.v[u][keep], self.w[u][keep]
        self.lists([0] * self.shape[1])
        self.same(what)

    def forget(self, b):
        """Sequence b is over."""
        for u in self.k:
            if u[1] == b:
                self.k[u], self.v[u], self.w[u] = self.k[u][:0], self.v[u][:0], self.w[u][:0]
        self.cache.length[:, b] = 0
        self.lists([0] * self.shape[1])

    def same(self, what):
        """The GPU's rows, weights and lengths are the ones kept here."""
        assert self.err.item() == 0, what
        k, v, w, n = self.cache.k.cpu(), self.cache.v.cpu(), self.cache.weight.cpu(), self.cache.length.cpu()
        for u in self.k:
            L = self.k[u].shape[0]
            assert n[u] == L, f"{what} unit {u}"
            r = torch.arange(L)
            at = self.table[u][r // self.page].long(), r % self.page
            assert torch.equal(k[at], self.k[u]) and torch.equal(v[at], self.v[u]), f"{what} unit {u}: rows"
            close_weight(w[u][:L], self.w[u], f"{what} unit {u}")


@pytest.mark.parametrize("dtype,D,G,page,sinks,window", [(BF, 128, 4, 16, 0, 0), (F32, 64, 3, 32, 0, 0), (BF, 64, 7, 64, 2, 90)])
def test_a_program_of_them(dtype, D, G, page, sinks, window):
    r = Run(2, 3, 2, G, D, page, 512, dtype, n_pages=12 * (512 // page) * 2 // 3, sinks=sinks, window=window, seed=D + G)
    r.prefill([130, 1, 77], "prompt")
    for i in range(4):
        r.decode(f"token {i}")
    r.evict([64, 64, 50], 2, 8, "eviction")
    for i in range(3):
        r.decode(f"token {i} after the eviction")
    r.forget(0)                                            # its pages go to a longer prompt
    r.prefill([300, 40, 1], "second prompt beside a chunk")
    for i in range(2):
        r.decode(f"late token {i}")
    r.evict([1, 4000, 30], 0, 1, "second eviction")
    r.decode("token on what is left")
    r.prefill([5, 5, 5], "probe")


@pytest.mark.parametrize("dtype,D,G", [(BF, 128, 7), (F32, 64, 2)])
def test_paged_dense_and_one_token_runs_agree(dtype, D, G):
    # the same rows in a dense cache, and the token as a run of one
    NL, Bs, H, cap, page = 2, 2, 2, 512, 32
    g = torch.Generator().manual_seed(2)
    lens = torch.tensor([[[0, 1], [33, 500]], [[511, 64], [200, 7]]], dtype=torch.int32)
    k, v = (torch.randn((NL, Bs, H, cap, D), generator=g).to(dtype).cuda() for _ in "kv")
    q = torch.randn((NL, Bs, H * G, D), generator=g).to(dtype).cuda()
    kn, vn = (torch.randn((NL, Bs, H, D), generator=g).to(dtype).cuda() for _ in "kv")
    pages = torch.arange(NL * Bs * H * cap // page, dtype=torch.int32).reshape(NL, Bs, H, -1).cuda()

    def paged():
        return B.PagedKVCache(k.reshape(-1, page, D).clone(), v.reshape(-1, page, D).clone(), pages, lens.cuda())
    dense, one, run = B.KVCache(k.clone(), v.clone(), lens.cuda()), paged(), paged()
    o0, z0 = B.reco_decode_attn(dense, q, kn, vn)
    o1, z1 = B.reco_paged_decode_attn(one, q, kn, vn)
    o2, z2 = B.reco_paged_prefill_attn(run, q[:, :, :, None], kn[:, :, :, None], vn[:, :, :, None])
    for what, o, z in (("paged", o1, z1), ("run", o2[:, :, :, 0], z2[..., 0])):
        # each is within its tolerance of the exact result
        close_out(o.cpu() / 2, o0.cpu().double() / 2, torch.cat([v.flatten(), vn.flatten()]).cpu(), dtype, what)
        close_lse(z.cpu() / 2, z0.cpu().double() / 2, dtype, what)
    for c in (one, run):
        assert torch.equal(c.k.reshape(k.shape), dense.k) and torch.equal(c.v.reshape(v.shape), dense.v)
        assert torch.equal(c.length, dense.length)


def test_streams_and_graphs_of_a_step():
    # A captured step (decode, evict) on one stream beside the same eager calls on
    # another, each with its own cache and workspaces; replays match eager steps.
    def make(seed):
        r = Run(2, 2, 2, 4, 128, 16, 256, BF, n_pages=8 * 16 + 1, seed=seed)
        r.lists([256, 256])
        g = torch.Generator().manual_seed(seed)
        kv = [torch.randn(r.cache.k.shape, generator=g).to(BF).cuda() for _ in "kv"]
        r.cache.k.copy_(kv[0])
        r.cache.v.copy_(kv[1])
        r.cache.length.fill_(100)
        r.cache.weight.copy_(torch.rand(r.cache.weight.shape, generator=g))
        return r.cache

    a, b = make(1), make(1)
    q = torch.randn((2, 2, 8, 128)).to(BF).cuda()
    kn, vn = (torch.randn((2, 2, 2, 128)).to(BF).cuda() for _ in "kv")
    budget = torch.tensor([98, 90], dtype=torch.int32).cuda()

    def step(cache, out, lse, ws):
        B.reco_paged_decode_attn(cache, q, kn, vn, out=out, lse=lse, ws=ws[0])
        B.reco_paged_evict(cache, budget, 1, 4, ws=ws[1])

    bufs = [(torch.empty_like(q), torch.empty(q.shape[:3], device="cuda"),
             (torch.empty(B.paged_decode_attn_workspace_size(c, 8), dtype=torch.uint8, device="cuda"),
              torch.empty(B.paged_evict_workspace_size(c), dtype=torch.uint8, device="cuda"))) for c in (a, b)]
    start = [x.clone() for x in (a.k, a.v, a.weight, a.length)]
    s1, s2 = torch.cuda.Stream(), torch.cuda.Stream()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s1):
        step(a, *bufs[0])
    for x, y in zip((a.k, a.v, a.weight, a.length), start):
        x.copy_(y)
    torch.cuda.synchronize()
    for i in range(3):
        with torch.cuda.stream(s1):
            graph.replay()
        with torch.cuda.stream(s2):
            step(b, *bufs[1])
        if i != 1:
            torch.cuda.synchronize()
            for x, y in zip((a.k, a.v, a.weight, a.length) + bufs[0][:2], (b.k, b.v, b.weight, b.length) + bufs[1][:2]):
                assert torch.equal(x.view(torch.int8), y.view(torch.int8)), f"replay {i}"
    torch.cuda.synchronize()


def test_rows_past_4_gib_of_a_pool():
    # the same rows at a large pool's end and in a small one give the same bits
    D, page, far, cap = 128, 4096, 4150, 8192
    g = torch.Generator().manual_seed(6)
    kv = [torch.randn((4, page, D), generator=g).to(BF).cuda() for _ in "kv"]
    length = torch.tensor([[[5000, 4095]]], dtype=torch.int32)
    weight = torch.rand((1, 1, 2, cap), generator=g)
    small = B.PagedKVCache(*(x.clone() for x in kv), torch.tensor([[[[2, 0], [3, 1]]]], dtype=torch.int32).cuda(),
                           length.cuda(), weight.cuda())
    pool = [torch.empty((far + 4, page, D), dtype=BF, device="cuda") for _ in "kv"]      # 4.05 GiB each
    for x, y in zip(pool, kv):
        x[far:] = y
    large = B.PagedKVCache(*pool, small.pages + far, length.cuda(), weight.cuda())
    q, kn, vn = (torch.randn((1, 1, n, 70, D), generator=g).to(BF).cuda() for n in (8, 2, 2))
    budget = torch.tensor([3000], dtype=torch.int32).cuda()
    got = []
    for c in (small, large):
        r = list(B.reco_paged_prefill_attn(c, q, kn, vn))
        r += B.reco_paged_decode_attn(c, *(x[:, :, :, 0].contiguous() for x in (q, kn, vn)))
        B.reco_paged_evict(c, budget, 4, 32)
        r += B.reco_paged_decode_attn(c, *(x[:, :, :, 1].contiguous() for x in (q, kn, vn)))
        got.append(r + [c.k[-4:], c.v[-4:], c.weight, c.length])
    for i, (x, y) in enumerate(zip(*got)):
        assert torch.equal(x.contiguous().view(torch.int8), y.contiguous().view(torch.int8)), i
