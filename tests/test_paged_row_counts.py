"""Windows, sinks and recent rows that do not fit the 32 bits of the C ABI are refused by
the binding, without a GPU: cut to 32 bits they would be other counts."""
import pytest

from paper_2608_04771_amd import binding as B
from test_paged_host import BF, BS, D, F32, H, HQ, I32, NL, _host_cache, _raises, _z

BIG = [2 ** 31, 2 ** 32 + 5, 10 ** 12, -2 ** 31 - 1, -2 ** 32 + 5]


def test_what_a_count_cut_to_32_bits_would_be():
    assert B.ctypes.c_int32(2 ** 32 + 5).value == 5 and B.ctypes.c_int32(-2 ** 32 + 5).value == 5


@pytest.mark.parametrize("n", BIG)
def test_counts_past_32_bits_are_refused(n):
    c = _host_cache()
    q, kn = _z(NL, BS, HQ, D, dtype=BF), _z(NL, BS, H, D, dtype=BF)
    qt, kt = _z(NL, BS, HQ, 5, D, dtype=BF), _z(NL, BS, H, 5, D, dtype=BF)
    out, lse, ws = _z(NL, BS, HQ, D, dtype=BF), _z(NL, BS, HQ, dtype=F32), _z(8)
    for what in ("sinks", "window"):
        _raises(what, B.reco_paged_decode_attn, c, q, kn, kn, **{what: n})
        _raises(what, B.reco_paged_prefill_attn, c, qt, kt, kt, **{what: n})
        _raises(what, B.PreparedPagedDecode, c, HQ, out, lse, ws, **{what: n})
    for what in ("sinks", "recent"):
        _raises(what, B.reco_paged_evict, c, _z(BS, dtype=I32), **{what: n})


@pytest.mark.parametrize("n", [0, 2 ** 31 - 1])
def test_counts_of_32_bits_get_to_the_device_check(n):
    c = _host_cache()
    q, kn = _z(NL, BS, HQ, D, dtype=BF), _z(NL, BS, H, D, dtype=BF)
    _raises("GPU", B.reco_paged_decode_attn, c, q, kn, kn, sinks=n, window=n)
    _raises("GPU", B.reco_paged_evict, c, _z(BS, dtype=I32), sinks=n, recent=n)
