"""What a bad stored length of one sequence does to shared attention: its group of that layer
and head is not specified, everything else is as without it."""
import numpy as np
import pytest
import torch

from shared_helpers import call, check_attention, make

pytestmark = pytest.mark.gpu

F32, BF = torch.float32, torch.bfloat16


@pytest.mark.parametrize("dtype,D,G", [(BF, 128, 4), (F32, 64, 3)])
@pytest.mark.parametrize("bad", [-1, -2 ** 31, 2 ** 31 - 1])
@pytest.mark.parametrize("groups,shared", [([0, 3, 5, 7], [40, 33, 64]), ([0, 3, 5, 5, 5, 5, 5, 6, 7, 8, 12], [40, 33, 0, 0, 0, 0, 5, 7, 9, 64])])
def test_others_are_as_they_were(dtype, D, G, bad, groups, shared):
    # (the second list has more groups than the cells that each wave fills for itself)
    of = np.arange(groups[-1])
    lens = np.asarray(shared)[np.searchsorted(groups[1:], of, side="right")][None, :, None] + \
        of[None, :, None] * 9 + np.array([[[0, 2]], [[1, 5]]])
    for at in ((0, 1, 0), (1, 0, 1), (1, 4, 0)):           # a group's first sequence among them
        for sinks, window in ((0, 0), (2, 50)):
            c, q, kn, vn = make(lens, groups, shared, 16, D, dtype, G, True, seed=3)
            c.length[at] = bad
            cache = c.upload()
            err = torch.zeros(1, dtype=torch.int32, device="cuda")
            out, lse = call(c, cache, q, kn, vn, err, sinks=sinks, window=window)
            assert err.item() in (5, 7)                    # the first one found: rows that its clamped length adds have bad ids
            mine = [u for u in np.ndindex(lens.shape) if (u[0], c.group[u[1]], u[2]) == (at[0], c.group[at[1]], at[2])]
            check_attention(c, q, kn, vn, out, lse, sinks, window, units=[u for u in np.ndindex(lens.shape) if u not in mine], what=f"{at}")
            n = cache.length.cpu()
            for u in np.ndindex(lens.shape):
                if u == at:
                    assert n[u] == bad
                    continue
                assert n[u] == int(lens[u]) + 1
                new = c.where(u, [int(lens[u])])
                assert torch.equal(cache.k.cpu()[new][0], kn[u]) and torch.equal(cache.v.cpu()[new][0], vn[u])
