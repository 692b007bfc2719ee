"""How blocks of query rows are dealt to the XCDs in pieces, by the device's compute units
(a partition has fewer than the whole device): from four rounds of blocks on, in pieces of
at most one round's share, every block exactly once.  The rules' source is compiled here
with a C interface of its own, without the kernels."""
import ctypes
import os
import random
import shutil
import subprocess

import pytest

from paper_2608_04771_amd.build import CSRC

SHIM = """
#include "paged.hpp"
using namespace reco;
extern "C" void pieces(int units, int blocks, int splits, int tokens, int window, int cus, int *got) {
  PagedPrefillParams p{};
  p.blocks = blocks, p.splits = splits, p.tokens = tokens, p.window = window;
  prefill_pieces(p, units, cus);
  got[0] = p.pieces, got[1] = p.near, got[2] = p.spread, got[3] = p.by_near.d;
}
extern "C" void whole_device(int units, int blocks, int *got) {
  PagedPrefillParams p{};
  p.blocks = blocks, p.splits = 1, p.tokens = 1 << 20;
  prefill_pieces(p, units);
  got[0] = p.pieces, got[1] = p.near, got[2] = p.spread, got[3] = p.by_near.d;
}
"""
CUS = [4, 32, 64, 128, 256, 304]


@pytest.fixture(scope="module")
def plan(tmp_path_factory):
    cxx = shutil.which("g++") or shutil.which("c++")
    if cxx is None:
        pytest.skip("no C++ compiler")
    d = tmp_path_factory.mktemp("pieces")
    (d / "shim.cpp").write_text(SHIM)
    so = str(d / "pieces.so")
    subprocess.run([cxx, "-std=c++17", "-O1", "-w", "-shared", "-fPIC", "-D__HIP_PLATFORM_AMD__", f"-I{CSRC}",
                    "-I/opt/rocm/include", str(d / "shim.cpp"), os.path.join(CSRC, "paged_plan.cpp"),
                    os.path.join(CSRC, "decode_plan.cpp"), "-o", so], check=True)
    return ctypes.CDLL(so)


def _pieces(plan, *args, whole=False):
    got = (ctypes.c_int * 4)()
    (plan.whole_device if whole else plan.pieces)(*args, got)
    return list(got)


@pytest.mark.parametrize("cus", CUS)
def test_dealt_from_four_rounds_on(plan, cus):
    for units in (1, 3, 8, 40):
        for blocks in (1, 2, 7, 33, 100, 500):
            pieces, near, _, by = _pieces(plan, units, blocks, 1, 1 << 20, 0, cus)
            assert (pieces > 0) == (units * blocks >= 4 * cus), (units, blocks)
            assert near <= max(1, cus // 8) and by == max(near, 1)
            assert _pieces(plan, units, blocks, 2, 1 << 20, 0, cus)[0] == 0     # splits are not dealt


@pytest.mark.parametrize("cus", CUS)
def test_every_block_is_dealt_once(plan, cus):
    r = random.Random(cus)
    dealt = 0
    for _ in range(150):
        units, blocks = int(2 ** r.uniform(0, 9)), int(2 ** r.uniform(0, 9))
        pieces, near, spread, _ = _pieces(plan, units, blocks, 1, 1 << 20, r.choice([0, 100]), cus)
        if not pieces:
            continue
        dealt += 1
        seen = set()
        for wg in range(-(-units * pieces // 8) * 8 * near):
            turn, pos = divmod(wg // 8, near)
            unit, j = divmod(turn * 8 + wg % 8, pieces)
            block = j + pieces * pos if spread else j * near + pos
            if unit < units and block < blocks:
                assert (unit, block) not in seen, (units, blocks)
                seen.add((unit, block))
        assert len(seen) == units * blocks, (units, blocks)
    assert dealt > 20


def test_whole_device_by_itself(plan):
    for units, blocks in ((16, 64), (4, 448), (40, 112), (3, 342), (1024, 1), (7, 146)):
        assert _pieces(plan, units, blocks, whole=True) == _pieces(plan, units, blocks, 1, 1 << 20, 0, 256)
