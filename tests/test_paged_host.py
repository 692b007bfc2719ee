"""Refusals of the operators over a paged cache, and their work split, without a GPU:
the C entry points refuse bad arguments before any launch, the binding refuses
tensors that the entry points would index wrongly."""
import ctypes

import pytest
import torch

from paper_2608_04771_amd import binding as B

P = ctypes.c_void_p
OK = dict(k=0x1000, v=0x2000, pages=0x3000, len=0x4000, weight=0x5000, n_layers=2, batch=1, n_kv_heads=2, n_pages=9,
          page_rows=16, max_pages=4, head_dim=128, dtype=B.RECO_BF16)


def _cache(**kw):
    d = dict(OK, **kw)
    return B.RecoPagedCache(*[d[n] for n, _ in B.RecoPagedCache._fields_])


def _decode(c, layer0=0, nl=2, q=0x100, hq=4, scale=0.1, sinks=0, window=0, kn=0x200, vn=0x300, out=0x400, ws=0x1000,
            wsb=1 << 40):
    return B.load_library().reco_paged_decode_attn(ctypes.byref(c), layer0, nl, P(q), hq, scale, sinks, window, P(kn),
                                                   P(vn), P(out), None, P(ws), wsb, None, None)


def _prefill(c, layer0=0, nl=2, q=0x100, hq=4, T=5, scale=0.1, sinks=0, window=0, kn=0x200, vn=0x300, out=0x400,
             ws=0x1000, wsb=1 << 40):
    return B.load_library().reco_paged_prefill_attn(ctypes.byref(c), layer0, nl, P(q), hq, T, None, scale, sinks, window,
                                                    P(kn), P(vn), P(out), None, P(ws), wsb, None, None)


def _evict(c, layer0=0, nl=2, budget=0x100, stride=0, sinks=0, recent=0, ws=0x1000, wsb=1 << 40):
    return B.load_library().reco_paged_evict(ctypes.byref(c), layer0, nl, P(budget), stride, sinks, recent, None, P(ws),
                                             wsb, None, None)


@pytest.mark.parametrize("call", [_decode, _prefill, _evict])
def test_caches_and_workspaces_are_refused(call):
    for bad in (dict(k=0), dict(v=0), dict(pages=0), dict(len=0), dict(n_layers=0), dict(batch=0), dict(n_kv_heads=0),
                dict(n_pages=0), dict(page_rows=0), dict(max_pages=0), dict(k=0x1008), dict(v=0x2004),
                dict(weight=0x5004)):
        assert call(_cache(**bad)) == B.RECO_ERR_INVALID_ARG, bad
    for bad in (dict(head_dim=96), dict(dtype=5), dict(page_rows=8), dict(page_rows=24), dict(page_rows=8192),
                dict(max_pages=(1 << 25) + 1)):
        assert call(_cache(**bad)) == B.RECO_ERR_UNSUPPORTED, bad
    c = _cache()
    assert call(c, layer0=-1) == call(c, layer0=1) == call(c, nl=0) == B.RECO_ERR_INVALID_ARG
    assert call(_cache(batch=40000)) == B.RECO_ERR_INVALID_ARG                     # 160,000 units
    assert call(c, ws=0) == call(c, wsb=0) == call(c, ws=0x1010) == B.RECO_ERR_WORKSPACE


@pytest.mark.parametrize("call", [_decode, _prefill])
def test_attention_arguments_are_refused(call):
    c = _cache()
    for bad in (dict(q=0), dict(out=0), dict(kn=0), dict(vn=0), dict(q=0x108), dict(out=0x404), dict(kn=0x202),
                dict(vn=0x301), dict(hq=3), dict(hq=0), dict(scale=float("nan")), dict(scale=float("inf")),
                dict(sinks=-1), dict(window=-1)):
        assert call(c, **bad) == B.RECO_ERR_INVALID_ARG, bad
    assert call(c, hq=2 * 17) == B.RECO_ERR_UNSUPPORTED


def test_more_refusals():
    c = _cache()
    assert _prefill(c, T=0) == B.RECO_ERR_INVALID_ARG
    assert _prefill(c, T=1 << 28) == B.RECO_ERR_UNSUPPORTED
    assert _evict(_cache(weight=0)) == _evict(c, budget=0) == _evict(c, stride=-1) == B.RECO_ERR_INVALID_ARG
    assert _evict(c, sinks=-1) == _evict(c, recent=-1) == B.RECO_ERR_INVALID_ARG
    lib, ref = B.load_library(), ctypes.byref
    for size, args in ((lib.reco_paged_decode_attn_workspace_size, (2, 4)),
                       (lib.reco_paged_prefill_attn_workspace_size, (2, 4, 5)),
                       (lib.reco_paged_evict_workspace_size, (2,))):
        need = size(ref(c), *args)
        assert 0 < need <= size(ref(_cache(max_pages=4096)), *args)
        assert size(ref(_cache(batch=40000)), *args) == size(ref(_cache(page_rows=24)), *args) == 0
        call = {(2, 4): _decode, (2, 4, 5): _prefill, (2,): _evict}[args]
        assert call(c, wsb=need - 1) == B.RECO_ERR_WORKSPACE
    assert lib.reco_paged_prefill_attn_workspace_size(ref(c), 2, 4, 1 << 29) == 0
    assert lib.reco_paged_decode_attn_workspace_size(ref(c), 2, 34) == 0
    # a grid of 2^32 threads and more (rows that no device holds) is refused
    huge = _cache(page_rows=4096, max_pages=1 << 17, batch=32000, n_layers=1)
    assert _decode(huge, nl=1, wsb=(1 << 64) - 1) == B.RECO_ERR_UNSUPPORTED
    assert _prefill(huge, nl=1, T=1 << 26, wsb=(1 << 64) - 1) == B.RECO_ERR_UNSUPPORTED


NL, BS, H, NP, PR, MP, D, HQ = 2, 3, 2, 12, 16, 4, 64, 8
BF, F32, I32 = torch.bfloat16, torch.float32, torch.int32


def _z(*shape, dtype=F32):
    return torch.zeros(shape, dtype=dtype)


def _host_cache(weight=True):
    """A PagedKVCache over host tensors: calls with right shapes stop at the device check."""
    c = B.PagedKVCache.__new__(B.PagedKVCache)
    c.k, c.v = _z(NP, PR, D, dtype=BF), _z(NP, PR, D, dtype=BF)
    c.pages, c.length = _z(NL, BS, H, MP, dtype=I32), _z(NL, BS, H, dtype=I32)
    c.weight = _z(NL, BS, H, MP * PR) if weight else None
    return c


def _raises(match, fn, *a, **kw):
    with pytest.raises(ValueError, match=match):
        fn(*a, **kw)


def test_binding_checks_the_cache():
    k, pages, ln = _z(NP, PR, D, dtype=BF), _z(NL, BS, H, MP, dtype=I32), _z(NL, BS, H, dtype=I32)
    _raises("k and v", B.PagedKVCache, k, _z(NP, PR, 128, dtype=BF), pages, ln)
    _raises("k and v", B.PagedKVCache, k[None], k[None], pages, ln)
    _raises("dtype", B.PagedKVCache, k.half(), k.half(), pages, ln)
    _raises("pages", B.PagedKVCache, k, k, pages.long(), ln)
    _raises("length", B.PagedKVCache, k, k, pages, _z(NL, BS, H + 1, dtype=I32))
    _raises("weight", B.PagedKVCache, k, k, pages, ln, _z(NL, BS, H, MP * PR - 1))
    _raises("weight", B.PagedKVCache, k, k, pages, ln, _z(NL, BS, H, MP * PR, dtype=BF))
    _raises("GPU", B.PagedKVCache, k, k, pages, ln)


def test_binding_checks_calls():
    c = _host_cache()
    assert c.shape == (NL, BS, H, MP * PR, D)
    q, kn = _z(NL, BS, HQ, D, dtype=BF), _z(NL, BS, H, D, dtype=BF)
    dec = B.reco_paged_decode_attn
    _raises("q must", dec, c, q.float())
    _raises("q must", dec, c, q[:, :2])
    _raises("together", dec, c, q, kn)
    _raises("k_new", dec, c, q, kn[:, :, :1], kn)
    _raises("v_new", dec, c, q, kn, kn.float())
    _raises("out", dec, c, q, out=_z(NL, BS, HQ, D))
    _raises("lse", dec, c, q, lse=_z(NL, BS, HQ + 1))
    _raises("layers", dec, c, q, layer0=1, n_layers=2)
    _raises("dev_err", dec, c, q, dev_err=_z(1))
    _raises("GPU", dec, c, q, kn, kn)
    qt, kt = _z(NL, BS, HQ, 5, D, dtype=BF), _z(NL, BS, H, 5, D, dtype=BF)
    pre = B.reco_paged_prefill_attn
    _raises("q must", pre, c, q, kn, kn)
    _raises("must be given", pre, c, qt, None, kt)
    _raises("k_new", pre, c, qt, kt[:, :, :, :4], kt)
    _raises("v_new", pre, c, qt, kt, kt.float())
    _raises("n_new", pre, c, qt, kt, kt, _z(BS + 1, dtype=I32))
    _raises("n_new", pre, c, qt, kt, kt, _z(BS, dtype=torch.int64))
    _raises("lse", pre, c, qt, kt, kt, lse=_z(NL, BS, HQ))
    _raises("GPU", pre, c, qt, kt, kt, _z(BS, dtype=I32))
    ev = B.reco_paged_evict
    _raises("weights", ev, _host_cache(False), _z(BS, dtype=I32))
    _raises("budget", ev, c, _z(BS))
    _raises("budget", ev, c, _z(BS + 1, dtype=I32))
    _raises("kept_idx", ev, c, _z(BS, dtype=I32), kept_idx=_z(NL, BS, H, MP, dtype=I32))
    _raises("GPU", ev, c, _z(NL, BS, dtype=I32))
