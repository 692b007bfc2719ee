"""Refusals and work split of the attention over shared prefixes, without a GPU."""
import ctypes
import os
import subprocess

import pytest
import torch

from paper_2608_04771_amd import binding as B
from test_paged_host import _cache

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2608_04771_amd", "csrc")
P = ctypes.c_void_p


def _shared(c=_cache(weight=0, batch=4), layer0=0, nl=2, q=0x100, hq=4, scale=0.1, sinks=0, window=0, first=0x500, groups=2,
            shared=0x600, stride=0, kn=0x200, vn=0x300, out=0x400, ws=0x1000, wsb=1 << 40):
    return B.load_library().reco_paged_shared_decode_attn(ctypes.byref(c), layer0, nl, P(q), hq, scale, sinks, window, P(first),
                                                          groups, P(shared), stride, P(kn), P(vn), P(out), None, P(ws), wsb, None, None)


def test_calls_are_refused():
    ok = dict(weight=0, batch=4)
    for bad in (dict(c=_cache(**dict(ok, k=0))), dict(c=_cache(**dict(ok, pages=0))), dict(c=_cache(**dict(ok, batch=0))),
                dict(c=_cache(**dict(ok, v=0x2004))), dict(q=0), dict(out=0), dict(first=0), dict(shared=0), dict(sinks=-1), dict(window=-1),
                dict(scale=float("nan")), dict(scale=float("inf")), dict(kn=0), dict(vn=0), dict(q=0x108), dict(out=0x404), dict(kn=0x202),
                dict(stride=-1), dict(groups=0), dict(groups=5), dict(groups=-1), dict(layer0=1), dict(nl=0), dict(hq=0), dict(hq=3)):
        assert _shared(**bad) == B.RECO_ERR_INVALID_ARG, bad
    for bad in (dict(c=_cache(batch=4)), dict(hq=34), dict(c=_cache(**dict(ok, head_dim=96))), dict(c=_cache(**dict(ok, dtype=2))),
                dict(c=_cache(**dict(ok, page_rows=24))), dict(c=_cache(**dict(ok, page_rows=8)))):
        assert _shared(**bad) == B.RECO_ERR_UNSUPPORTED, bad
    size = B.load_library().reco_paged_shared_decode_attn_workspace_size(ctypes.byref(_cache(**ok)), 2, 4, 2)
    assert size > 0
    for bad in (dict(ws=0), dict(wsb=size - 1), dict(ws=0x1010)):
        assert _shared(**bad) == B.RECO_ERR_WORKSPACE, bad
    for args in ((2, 4, 0), (2, 4, 5), (0, 4, 2), (2, 34, 2), (2, 3, 2)):
        assert B.load_library().reco_paged_shared_decode_attn_workspace_size(ctypes.byref(_cache(**ok)), *args) == 0, args


SHIM = r'''
#include "paged.hpp"
extern "C" {
int blocks(int b, int g, int n) { return reco::shared_blocks(b, g, n); }
int splits(int jobs, int blocks, int span, int dt, int cus) { return reco::shared_splits(jobs, blocks, span, dt, cus); }
int own(int jobs, int b, int cus) { return reco::shared_own_parts(b, reco::shared_cell_wgs(jobs * ((b + reco::kSharedCell - 1) / reco::kSharedCell), cus)); }
int span(int cap, int sinks, int window) { return reco::shared_span_rows(cap, sinks, window); }
size_t bytes(int jobs, int b, int g, int n, int cap, int d, int dt, int cus) { return reco::paged_shared_workspace_bytes(jobs, b, g, n, cap, d, dt, cus); }
int rows() { return reco::kSharedRows; }
int most() { return reco::kSharedMaxSplits; }
}
'''


@pytest.fixture(scope="module")
def plan(tmp_path_factory):
    d = tmp_path_factory.mktemp("shared")
    (d / "shim.cpp").write_text(SHIM)
    lib = str(d / "plan.so")
    subprocess.run(["g++", "-std=c++17", "-O1", "-shared", "-fPIC", "-D__HIP_PLATFORM_AMD__", f"-I{CSRC}", f"-I{ROOT}/include",
                    "-I/opt/rocm/include", str(d / "shim.cpp"), os.path.join(CSRC, "paged_plan.cpp"),
                    os.path.join(CSRC, "decode_plan.cpp"), "-o", lib], check=True)
    p = ctypes.CDLL(lib)
    p.bytes.restype = ctypes.c_size_t
    return p


def test_blocks_hold_every_split_of_a_batch(plan):
    R = plan.rows()
    for G in (1, 3, 7, 16):
        for sizes in ([1], [5], [40], [128], [1, 1, 1], [0, 9, 0], [17, 64, 3], [1] * 70, [100, 1, 250, 8]):
            need = sum(-(-n * G // R) for n in sizes)
            assert plan.blocks(sum(sizes), G, len(sizes)) >= need
        assert plan.blocks(33, G, 1) == -(-33 * G // R)


def test_splits_fit_the_workspace(plan):
    for cus in (256, 32, 304):
        for jobs in (1, 4, 8, 112, 512):
            for batch in (1, 2, 8, 32, 200):
                for G in (1, 7, 16):
                    for cap in (16, 300, 4096, 70000):
                        for groups in {1, max(1, batch // 3), batch}:
                            blocks, units = plan.blocks(batch, G, groups), jobs * batch
                            for dt in (0, 1):
                                whole = plan.splits(jobs, blocks, cap, dt, cus) + plan.own(jobs, batch, cus)
                                assert plan.bytes(jobs, batch, G, groups, cap, 128, dt, cus) == whole * units * G * 130 * 4
                                for sinks, window in ((0, 0), (4, 1), (4, 64), (2 ** 31 - 1, 2 ** 31 - 1), (100, 5000)):
                                    span = plan.span(cap, sinks, window)
                                    a, b = plan.splits(jobs, blocks, span, dt, cus), plan.own(jobs, batch, cus)
                                    assert 1 <= a <= plan.most() and 2 <= b <= plan.most() and a + b <= whole
                                    assert a == 1 or a * jobs * blocks < 3 * cus
