"""Shared attention over large batches: the outputs of every sequence against the 64-bit form,
with and without a window, and one long sequence among many short ones."""
import numpy as np
import pytest
import torch

from shared_helpers import call, check_append, check_attention, make

pytestmark = pytest.mark.gpu

F32, BF = torch.float32, torch.bfloat16


@pytest.mark.parametrize("sinks,window", [(0, 0), (3, 20)])
@pytest.mark.parametrize("batch,groups,dtype", [(65, 2, BF), (200, 8, F32), (200, 9, BF), (512, 1, F32), (512, 8, BF), (512, 64, BF),
                                                (512, 65, F32), (512, 400, BF), (513, 3, F32), (700, 16, BF), (1100, 2, BF), (1100, 65, F32),
                                                (1100, 1000, BF)])
def test_every_sequence(batch, groups, dtype, sinks, window):
    rng = np.random.RandomState(batch * groups)
    first = np.sort(np.concatenate([[0, batch], rng.randint(0, batch + 1, groups - 1)]))
    shared = rng.randint(0, 50, groups)
    of = np.searchsorted(first[1:], np.arange(batch), side="right")
    lens = (shared[of] + rng.randint(0, 40, batch))[None, :, None]
    c, q, kn, vn = make(lens, first, shared, 16, 64, dtype, 2, True, seed=groups)
    cache = c.upload()
    err = torch.zeros(1, dtype=torch.int32, device="cuda")
    out, lse = call(c, cache, q, kn, vn, err, sinks=sinks, window=window)
    assert err.item() == 0
    check_attention(c, q, kn, vn, out, lse, sinks, window)
    check_append(c, cache, kn, vn)


def test_one_long_sequence_among_many_short_ones():
    # it has more rows than a wave's even share of all of them many times over
    for dtype, D in ((BF, 128), (F32, 64)):
        lens = np.full((1, 128, 2), 40) + np.arange(128)[None, :, None] % 9
        lens[0, 77] = 2300
        lens[0, 127] = 900
        c, q, kn, vn = make(lens, [0, 60, 128], [33, 40], 16, D, dtype, 2, True, seed=2)
        cache = c.upload()
        err = torch.zeros(1, dtype=torch.int32, device="cuda")
        out, lse = call(c, cache, q, kn, vn, err)
        assert err.item() == 0
        check_attention(c, q, kn, vn, out, lse)
        check_append(c, cache, kn, vn)
