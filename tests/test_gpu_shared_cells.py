"""reco_paged_shared_decode_attn over more sequences than one cell of the own rows' work takes
(512): groups that reach from one cell into the next, against the 64-bit form, unit by unit."""
import numpy as np
import pytest
import torch

from paper_2608_04771_amd import binding as B
from shared_helpers import call, check_append, check_attention, make

pytestmark = pytest.mark.gpu

F32, BF = torch.float32, torch.bfloat16


def _case(first, shared, own, dtype, D, seed):
    """One layer and KV head; group g's sequences have shared[g] rows and own[g] to own[g] + 6."""
    group = np.searchsorted(np.asarray(first[1:]), np.arange(first[-1]), side="right")
    lens = np.asarray(shared)[group] + np.asarray(own)[group] + np.arange(first[-1]) * 5 % 7
    return make(lens[None, :, None], first, shared, 16, D, dtype, 2, True, seed=seed)


@pytest.mark.parametrize("dtype,D", [(BF, 128), (F32, 64)])
@pytest.mark.parametrize("first,shared,own", [
    ([0, 5, 600], [10, 200], [30, 1]),                     # shorter sequences in front of a group that goes on past 512
    ([0, 5, 600], [10, 200], [900, 1]),                    # longer ones
    ([0, 63, 530], [3, 100], [0, 8]), ([0, 63, 530], [3, 100], [400, 8]),
    ([0, 1, 2, 40, 1030], [0, 9, 5, 70], [2, 300, 0, 3]),  # into a third cell
])
def test_groups_that_reach_past_a_cell(first, shared, own, dtype, D):
    for sinks, window in ((0, 0), (0, 90), (4, 30)):
        c, q, kn, vn = _case(first, shared, own, dtype, D, seed=window)
        cache = c.upload()
        err = torch.zeros(1, dtype=torch.int32, device="cuda")
        out, lse = call(c, cache, q, kn, vn, err, sinks=sinks, window=window)
        assert err.item() == 0
        check_attention(c, q, kn, vn, out, lse, sinks, window, what=f"window {window}")
        check_append(c, cache, kn, vn)


@pytest.mark.parametrize("short", [59, 60, 63, 64, 511, 512, 599])
def test_counts_past_the_shortest_of_a_group_past_a_cell(short):
    # the group's shortest sequence is one of the first cell's or of the next; its rows are all that are shared
    first, used = [0, 5, 600], 40
    lens = np.full((1, 600, 1), 70)
    lens[0, :5] = 90
    lens[0, short] = used
    c, q, kn, vn = make(lens, first, [10, used], 16, 64, F32, 2, True, seed=short)
    cache = c.upload()
    err = torch.zeros(1, dtype=torch.int32, device="cuda")
    given = torch.tensor([10, 65], dtype=torch.int32).cuda()
    out, lse = B.reco_paged_shared_decode_attn(cache, q.cuda(), torch.tensor(first, dtype=torch.int32).cuda(), given, kn.cuda(), vn.cuda(),
                                               dev_err=err)
    assert err.item() == 5
    check_attention(c, q, kn, vn, out.cpu(), lse.cpu(), what=f"shortest {short}")
