"""Outputs that are their input's own rows, seen by another view of the same memory: taken as
in place, without a GPU."""
import pytest
import torch

from paper_2608_04771_amd import binding as B


def test_strides_of_one_do_not_count():
    # one token, one layer or one sequence: the stride of such a dimension is never used
    buf = torch.zeros(2, 6, 64)
    as_tokens = buf.view(1, 2, 1, 6, 64).transpose(2, 3)   # [NL][B][H][T][D], a token's heads beside each other
    as_heads = buf.view(1, 2, 6, 1, 64)
    assert as_tokens.shape == as_heads.shape and as_tokens.stride() != as_heads.stride()
    B._no_partial_overlap(as_tokens, as_heads, "out")
    B._no_partial_overlap(as_heads, as_tokens, "out")
    one = torch.zeros(3, 5, 64)
    B._no_partial_overlap(one.view(1, 1, 3, 5, 64), one.as_strided((1, 1, 3, 5, 64), (7, 11, 320, 64, 1)), "out")
    # rows that are other ones stay refused
    for x, out in ((as_heads, buf.view(1, 6, 2, 1, 64).transpose(1, 2)), (as_tokens[:, :, :5], as_heads[:, :, 1:]),
                   (one[None, None, :, 1:], one[None, None, :, :4])):
        with pytest.raises(ValueError, match="out"):
            B._no_partial_overlap(x, out, "out")
    # and rows that may be rotated in place may not be another call's keys
    with pytest.raises(ValueError, match="q_out"):
        B._no_partial_overlap(as_tokens, as_heads, "q_out", same=False)
