"""That the calls of shared_long_cases.py are long ones: tiles of a workgroup's common rows
and of a wave's own ones, by the functions that split a call's work, on 256 compute units."""
import ctypes
import os
import subprocess

import pytest

from shared_long_cases import COMMON, HEADS, LAYERS, OWN

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2608_04771_amd", "csrc")
SHIM = r'''
#include "paged.hpp"
extern "C" {
int splits(int jobs, int batch, int g, int span, int dt, int cus) { return reco::shared_splits(jobs, reco::shared_blocks(batch, g, 1), span, dt, cus); }
int span(int cap, int sinks, int window) { return reco::shared_span_rows(cap, sinks, window); }
int cell_wgs(int cells, int cus) { return reco::shared_cell_wgs(cells, cus); }
int parts(int batch, int cell_wgs) { return reco::shared_own_parts(batch, cell_wgs); }
}
'''
CUS = 256
WAVES = 4                                                  # of a workgroup
PLACES = 64 * 16                                           # rows that a wave has looked up at a time: 16 a lane


@pytest.fixture(scope="module")
def plan(tmp_path_factory):
    d = tmp_path_factory.mktemp("long")
    (d / "shim.cpp").write_text(SHIM)
    lib = str(d / "plan.so")
    subprocess.run(["g++", "-std=c++17", "-O1", "-shared", "-fPIC", "-D__HIP_PLATFORM_AMD__", f"-I{CSRC}", f"-I{ROOT}/include",
                    "-I/opt/rocm/include", str(d / "shim.cpp"), os.path.join(CSRC, "paged_plan.cpp"),
                    os.path.join(CSRC, "decode_plan.cpp"), "-o", lib], check=True)
    return ctypes.CDLL(lib)


def _seen(rows, sinks, window):
    """Rows of a sequence that its new token, behind them, sees."""
    return rows if window == 0 or rows <= window + sinks else sinks + window - 1


@pytest.mark.parametrize("case", COMMON, ids=str)
def test_common_rows_are_looked_up_again(plan, case):
    dtype, D, G, page, P, own, (sinks, window) = case
    cap = -(-(P + max(own) + 1) // page) * page
    splits = plan.splits(LAYERS * HEADS, len(own), G, plan.span(cap, sinks, window), int(dtype == "bf16"), CUS)
    start = max(0, P + max(own) + 1 - window) if window else 0
    assert splits == 1 and min(sinks, start) + P - start > 2 * PLACES


@pytest.mark.parametrize("case", OWN, ids=str)
def test_own_rows_are_looked_up_again(plan, case):
    dtype, D, G, page, P, own, (sinks, window) = case
    wgs = plan.cell_wgs(LAYERS * HEADS, CUS)
    tiles = [_seen(n, sinks, window) // 32 for n in own]
    share = max(-(-sum(tiles) // (WAVES * wgs)), -(-max(tiles) // (plan.parts(len(own), wgs) - 1)))
    assert wgs == 1 and 32 * share > PLACES * (1 if window else 2)
