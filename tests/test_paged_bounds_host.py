"""The bounds of bf16 outputs over a paged cache, without a GPU: a form that rounds where the
kernels do is within them at every length, and rows of V in the wrong place are not."""
import math

import pytest
import torch

from paged_bounds import Expected

BF = torch.bfloat16


def _rows(n, D, G, seed):
    g = torch.Generator().manual_seed(seed)
    k, v = (torch.randn((n, D), generator=g).to(BF) for _ in "kv")
    return k, v, torch.randn((G, D), generator=g).to(BF)


def _rounded(k, v, q, scale, lag=0.0):
    """P rounded to bf16 (its reference a few log2 units behind the maximum), the sum not, and
    the result rounded."""
    x = (q.float() @ k.float().T) * (scale * math.log2(math.e))
    e = torch.exp2(x - x.amax(-1, keepdim=True) + lag)
    return ((e.to(BF).float() @ v.float()) / e.sum(-1, keepdim=True)).to(BF)


@pytest.mark.parametrize("lag", [0.0, 5.3])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("n", [1, 2, 33, 1000, 9677, 20001])
def test_a_form_that_rounds_alike_is_within(n, D, lag):
    k, v, q = _rows(n, D, 7, n + D)
    e = Expected(k, v, q, n - 1, 1 / math.sqrt(D))
    assert (e.rms is not None) == (n > 1000) or n == 1000
    e.check(_rounded(k, v, q, 1 / math.sqrt(D), lag), f"{n} rows")


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("n", [2000, 9677, 20001])
def test_rows_of_v_in_the_wrong_place_are_not(n, D):
    k, v, q = _rows(n, D, 7, n + D)
    e = Expected(k, v, q, n - 1, 1 / math.sqrt(D))
    for rows in (32, 16):
        w = v.clone()
        w[n // 2:n // 2 + rows] = v[n // 2:n // 2 + rows].flip(0)
        with pytest.raises(AssertionError):
            e.check(_rounded(k, w, q, 1 / math.sqrt(D)), "reversed")
    w = v.clone()
    w[64:96] = v[96:128]                                    # a tile taken for the one before it
    with pytest.raises(AssertionError):
        e.check(_rounded(k, w, q, 1 / math.sqrt(D)), "a tile twice")
    with pytest.raises(AssertionError):
        e.check(torch.zeros_like(q), "nothing")
