"""The eviction's compaction alone, on state set by the test: what it does where a wait
for earlier chunks of a unit ends in vain (the state says that a chunk was taken which no
one takes), and where the state lets it pass.  Every wait is bounded by the limit that the
test gives, so each kernel ends by itself."""
import ctypes
import os

import numpy as np
import pytest
import torch

from paged_helpers import Paged
from paper_2608_04771_amd import binding as B

pytestmark = pytest.mark.gpu

SPINS = 1 << 14                              # some ten milliseconds: units that do move need far fewer
TAKEN, PASSED, STORED = 0, 1, 2


def _client():
    path = os.path.join(os.path.dirname(os.path.abspath(__file__)), "c_abi", "libcompact_client.so")
    if not os.path.exists(path):
        pytest.fail("tests/c_abi/libcompact_client.so is not built: run __graft_entry__.build()")
    B.load_library()
    lib = ctypes.CDLL(path)
    lib.compact_alone.argtypes = [ctypes.POINTER(B.RecoPagedCache)] + [ctypes.c_void_p] * 3 + [ctypes.c_int] + \
        [ctypes.c_void_p] * 2
    return lib


def _run(p, kept_rows, prepare, spins):
    """The compaction of p's units, each keeping kept_rows[unit], from the state that prepare
    leaves of a cleared one [units][ints]; returns the cache, the error and the state."""
    lib = _client()
    cache = p.upload()
    NL, Bs, H = p.lens.shape
    units, cap = NL * Bs * H, p.max_pages * p.page
    rows = lib.compact_chunk_rows(p.D * p.k.element_size())
    first = lib.compact_state()
    state = torch.zeros((units, first + -(-cap // rows)), dtype=torch.int32)
    prepare(state, first)
    idx = torch.full((units, cap), -1, dtype=torch.int32)
    for u, k in enumerate(kept_rows):
        idx[u, :len(k)] = torch.from_numpy(k.astype(np.int32))
    kept = torch.tensor([len(k) for k in kept_rows], dtype=torch.int32, device="cuda")
    idx, state = idx.cuda(), state.cuda()
    err = torch.zeros(1, dtype=torch.int32, device="cuda")
    torch.cuda.synchronize()
    st = lib.compact_alone(cache.ref(), idx.data_ptr(), kept.data_ptr(), state.data_ptr(), spins, err.data_ptr(),
                           torch.cuda.current_stream().cuda_stream)
    assert st == 0
    torch.cuda.synchronize()
    return cache, err.item(), state.cpu(), rows, first


def _cache(lens, D=128, dtype=torch.bfloat16):
    return Paged([[lens]], 64, D, dtype, seed=7, weights=True)


def _choice(L, m, seed):
    """m of L rows, ascending, that leave few in place."""
    return np.sort(np.random.RandomState(seed).permutation(np.arange(1, L))[:m])


def _same(a, b):
    return torch.equal(a.cpu().contiguous().view(torch.int8), b.contiguous().view(torch.int8))


def _moved(p, u, idx, upto=None, start=0):
    """p's tensors with rows [start, upto) of unit u put in their places."""
    k, v, w = p.k.clone(), p.v.clone(), p.weight.clone()
    at = np.arange(start, len(idx) if upto is None else upto)
    src, dst = p.where(u, idx[at]), p.where(u, at)
    k[dst], v[dst] = p.k[src], p.v[src]
    w[u][torch.from_numpy(at)] = p.weight[u][torch.from_numpy(idx[at])]
    return k, v, w


@pytest.mark.parametrize("dtype,D", [(torch.bfloat16, 64), (torch.bfloat16, 128), (torch.float32, 128)])
def test_cleared_state_moves_everything(dtype, D):
    p = _cache([3000], D, dtype)
    idx = _choice(3000, 2001, 1)
    cache, err, state, rows, first = _run(p, [idx], lambda s, f: None, 0)
    k, v, w = _moved(p, (0, 0, 0), idx)
    assert err == 0 and cache.length.item() == 2001
    assert _same(cache.k, k) and _same(cache.v, v) and _same(cache.weight, w)
    chunks = -(-2001 // rows)
    assert state[0, STORED].item() == chunks and state[0, first:first + chunks].all()


def test_a_chunk_that_no_one_loads_stops_the_unit():
    """Chunk 0 counts as taken, but no workgroup has it: no later chunk of that unit may be
    stored and its length stays; the unit beside it is moved as usual."""
    p = _cache([3000, 2500])
    idx = [_choice(3000, 2001, 1), _choice(2500, 1900, 2)]

    def prepare(state, first):
        state[0, TAKEN] = 1
    cache, err, state, rows, first = _run(p, idx, prepare, SPINS)
    assert err == 9 and B.DEV_ERRORS[9] == "stalled eviction"
    assert cache.length.cpu().flatten().tolist() == [3000, 1900]
    k, v, w = _moved(p, (0, 0, 1), idx[1])
    assert _same(cache.k, k) and _same(cache.v, v) and _same(cache.weight, w)
    assert state[0, STORED].item() == 0 and state[0, PASSED].item() == 0


def test_a_chunk_missing_among_many():
    """100 chunks are taken and all but the 70th loaded: none of the rest may be stored."""
    L, m = 20000, 14000
    p = _cache([L])
    idx = _choice(L, m, 3)

    def prepare(state, first):
        state[0, TAKEN] = 100
        state[0, first:first + 100] = 1
        state[0, first + 70] = 0
    cache, err, state, rows, first = _run(p, [idx], prepare, SPINS)
    assert m > 101 * rows
    assert err == 9 and cache.length.item() == L
    assert _same(cache.k, p.k) and _same(cache.v, p.v) and _same(cache.weight, p.weight)


def test_chunks_loaded_before_are_not_waited_for():
    """100 chunks taken, loaded and stored by others: the rest is moved and the length set."""
    L, m = 20000, 14000
    p = _cache([L])
    idx = _choice(L, m, 3)

    def prepare(state, first):
        state[0, TAKEN] = 100
        state[0, PASSED] = 40
        state[0, STORED] = 100
        state[0, first + 40:first + 100] = 1
    cache, err, state, rows, first = _run(p, [idx], prepare, SPINS)
    k, v, w = _moved(p, (0, 0, 0), idx, start=100 * rows)
    assert err == 0 and cache.length.item() == m
    assert _same(cache.k, k) and _same(cache.v, v) and _same(cache.weight, w)
    assert state[0, STORED].item() == -(-m // rows)
