"""Refusals of the rotation and of the append, without a GPU: the C entry points refuse bad
arguments before any launch, the binding tensors that they would index wrongly."""
import ctypes

import pytest
import torch

from paper_2608_04771_amd import binding as B
from test_paged_host import _cache

P = ctypes.c_void_p
INVALID, UNSUPPORTED = B.RECO_ERR_INVALID_ARG, B.RECO_ERR_UNSUPPORTED


def _turn(inv_freq=0x100, pos=0x200, axis=None, n_axes=1, rot=128, pairs=0):
    return B.RecoRope(inv_freq, pos, None if axis is None else (ctypes.c_int32 * len(axis))(*axis), n_axes, rot, pairs)


def _rows(data=0x1000, layer=4096, seq=2048, head=128, token=256):
    return B.RecoRows(data, layer, seq, head, token)


def _ref(x):
    return None if x is None else ctypes.byref(x)


def _rope(rope=_turn(), x=_rows(), out=_rows(), nl=1, b=2, h=3, t=4, d=128, dtype=B.RECO_BF16):
    return B.load_library().reco_rope(_ref(rope), _ref(x), _ref(out), nl, b, h, t, d, dtype, None, None, None)


def _append(cache=_cache(), layer0=0, nl=2, rope=_turn(), t=3, k=_rows(), v=_rows(), q=_rows(), qo=_rows(), hq=4):
    return B.load_library().reco_paged_append(_ref(cache), layer0, nl, _ref(rope), t, None, _ref(k), _ref(v), _ref(q),
                                              _ref(qo), hq, None, None)


@pytest.mark.parametrize("call", [_rope, _append])
def test_rotations_are_refused(call):
    for bad in (dict(inv_freq=0), dict(pos=0), dict(n_axes=0), dict(n_axes=-1), dict(rot=0), dict(rot=-16), dict(rot=127),
                dict(rot=144), dict(pairs=2), dict(axis=[0] * 63 + [1]), dict(axis=[-1] + [0] * 63)):
        assert call(rope=_turn(**bad)) == INVALID, bad
    for bad in (dict(n_axes=5, axis=[4] * 64), dict(rot=24), dict(rot=2)):
        assert call(rope=_turn(**bad)) == UNSUPPORTED, bad


def test_rows_are_refused():
    for bad in (None, _rows(data=0), _rows(data=0x1008), _rows(layer=4), _rows(seq=1), _rows(head=130), _rows(token=-3)):
        assert _rope(x=bad) == INVALID and _rope(out=bad) == INVALID
        assert _append(k=bad) == INVALID and _append(v=bad) == INVALID and _append(q=bad) == INVALID and _append(qo=bad) == INVALID
    assert _rope(x=_rows(head=68), dtype=B.RECO_BF16) == INVALID
    assert _rope(rope=None) == INVALID
    for bad in (dict(nl=0), dict(b=0), dict(h=0), dict(t=0), dict(t=-1)):
        assert _rope(**bad) == INVALID, bad
    for bad in (dict(d=96, rope=_turn(rot=96)), dict(d=256), dict(dtype=2), dict(h=1025), dict(t=2 ** 24 + 1), dict(b=65536), dict(nl=65536)):
        assert _rope(**bad) == UNSUPPORTED, bad


def test_appends_are_refused():
    for bad in (dict(cache=None), dict(cache=_cache(k=0)), dict(cache=_cache(len=0)), dict(cache=_cache(v=0x1004)), dict(t=0),
                dict(layer0=1), dict(layer0=-1), dict(nl=0), dict(hq=0), dict(q=None), dict(qo=None)):
        assert _append(**bad) == INVALID, bad
    for bad in (dict(cache=_cache(head_dim=96)), dict(cache=_cache(dtype=3)), dict(cache=_cache(page_rows=24)), dict(hq=1025),
                dict(t=2 ** 24 + 1)):
        assert _append(**bad) == UNSUPPORTED, bad


def test_binding_refuses_handles():
    with pytest.raises(ValueError, match="GPU"):
        B.Rope(torch.ones(64))
    with pytest.raises(ValueError, match="inv_freq"):
        B.Rope(torch.ones(64, dtype=torch.float64))
    with pytest.raises(ValueError, match="inv_freq"):
        B.Rope(torch.ones(2, 32))


def test_binding_refuses_rows():
    r = B._Rows("x", (1, 2, 3, 4, 64), torch.float32, torch.device("cpu"))
    x = torch.zeros(1, 2, 4, 3, 64).transpose(2, 3)
    r.take(x)
    assert (r.struct.layer, r.struct.seq, r.struct.head, r.struct.token) == (0, 768, 64, 192)
    for bad in (x.double(), x[..., :32], x[:, :1], torch.zeros(1, 2, 3, 64), torch.zeros(1, 2, 3, 4, 128)[..., ::2],
                torch.zeros(1, 2, 3, 4, 65)[..., :64], torch.zeros(1 + 64 * 24)[1:].view(1, 2, 3, 4, 64)):
        with pytest.raises(ValueError, match="x"):
            r.take(bad)
    w = B._Rows("out", (1, 2, 3, 4, 64), torch.float32, torch.device("cpu"), write=True)
    w.take(x)
    w.take(torch.zeros(1, 2, 4, 5, 64)[:, :, :, 1:4].transpose(2, 3))
    for bad in (torch.zeros(1, 1, 3, 4, 64).expand(1, 2, 3, 4, 64), torch.zeros(3000).as_strided((1, 2, 3, 4, 64), (0, 768, 64, 64, 1)),
                torch.zeros(3000).as_strided((1, 2, 3, 4, 64), (0, 64, 384, 96, 1))):
        with pytest.raises(ValueError, match="overlap"):
            w.take(bad)
    one = B._Rows("x", (1, 2, 3, 64), torch.bfloat16, torch.device("cpu"))
    one.take(torch.zeros(1, 2, 3, 64, dtype=torch.bfloat16))
    assert (one.struct.seq, one.struct.head, one.struct.token) == (192, 64, 0)


def test_binding_refuses_outputs_over_inputs():
    x = torch.zeros(1, 2, 4, 10, 64).transpose(2, 3)       # ten heads beside each other
    B._no_partial_overlap(x, x, "out")
    B._no_partial_overlap(x, torch.zeros(1, 2, 10, 4, 64), "out")
    B._no_partial_overlap(x[:, :, :4], x[:, :, 4:8], "out")
    B._no_partial_overlap(x[:, :, 6:], x[:, :, :4], "out")
    flat = x.transpose(2, 3).reshape(-1)
    for a, b in ((x[:, :, :4], x[:, :, 3:7]), (x[:, :, :4], flat[:2 * 4 * 4 * 64].view(1, 2, 4, 4, 64)),
                 (x[:, :, :, :3], x[:, :, :, 1:]), (x[:, :1], x[:, :1].transpose(2, 3)[:, :, :, :4])):
        with pytest.raises(ValueError, match="out"):
            B._no_partial_overlap(a, b, "out")


def test_rotated_queries_meet_no_keys_or_values():
    x = torch.zeros(1, 2, 4, 10, 64).transpose(2, 3)       # six heads of queries, two of keys, two of values
    q, k, v = x[:, :, :6], x[:, :, 6:8], x[:, :, 8:]
    for t in (k, v):
        B._no_partial_overlap(t, q, "q_out", same=False)
        B._no_partial_overlap(t, torch.zeros(1, 2, 6, 4, 64), "q_out", same=False)
    one = torch.zeros(1, 2, 2, 1, 64)                      # one token: a stride of its dimension is not one
    B._no_partial_overlap(one[:, :, :1], one[:, :, 1:], "q_out", same=False)
    flat = x.transpose(2, 3).reshape(-1)
    skew = torch.zeros(2000).as_strided((1, 2, 1, 2, 64), (0, 200, 64, 192, 1))      # rows 0, 192, 200, 392
    for t, out in ((k, x[:, :, 1:7]), (k, k), (v, x[:, :, 4:]), (k, flat[:2 * 6 * 4 * 64].view(1, 2, 6, 4, 64)),
                   (k, x[:, :, 6:8].transpose(2, 3)), (x[:, :, 6:8, 1:], x[:, :, :6, :3]),
                   (skew, torch.as_strided(skew, skew.shape, skew.stride(), 64))):
        with pytest.raises(ValueError, match="q_out must not meet"):
            B._no_partial_overlap(t, out, "q_out", same=False)
    buf = torch.zeros(4096)
    r, span = B._Rows("x", (1, 1, 1, 2, 64), torch.float32, torch.device("cpu")), B._span(buf[1024:2048])
    for at, met in ((0, False), (1024 - 128, False), (1024 - 124, True), (1024, True), (2044, True), (2048, False)):
        r.take(buf[at:at + 128].view(1, 1, 1, 2, 64))
        assert r.meets(span) == met, at
