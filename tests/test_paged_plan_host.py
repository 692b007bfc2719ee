"""The work split of the paged operators on the host: every block of query rows is done
exactly once wherever its workgroup runs, and no call takes more partials than the
workspace sized for it holds.  The rules' source is compiled here with a C interface of
its own, without the kernels."""
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
extern "C" void prefill(int units, int tokens, int group, int cap, int sinks, int window, int dtype, int cus, int *got) {
  PagedPrefillParams p{};
  p.c.n_layers = 1, p.c.batch = 1, p.c.hkv = units, p.c.cap = cap;
  p.tokens = tokens, p.group = group, p.sinks = sinks, p.window = window;
  p.rows = prefill_rows(units, tokens, group, cap, window, dtype, cus);
  p.blocks = prefill_blocks(tokens, group, p.rows);
  p.splits = p.rows == kPrefillRows ? prefill_splits(units, p.blocks, cap, sinks, window, prefill_tile_rows(dtype), cus) : 1;
  prefill_pieces(p, units);
  const int all[] = {p.rows, p.blocks, p.splits, p.pieces, p.near, p.spread, prefill_fits_grid(p)};
  for (int i = 0; i < 7; ++i) got[i] = all[i];
}
extern "C" size_t prefill_ws(int units, int tokens, int cap, int group, int dim, int dtype, int cus) {
  return prefill_workspace_bytes(units, tokens, cap, group, dim, prefill_tile_rows(dtype), cus);
}
extern "C" int decode(int units, int cap, int sinks, int window, int cus) {
  return paged_decode_splits(units, paged_span_tiles(cap, sinks, window), cus);
}
extern "C" size_t decode_ws(int units, int cap, int group, int dim, int weights, int cus) {
  return paged_decode_workspace_bytes(units, cap, group, dim, weights, cus);
}
extern "C" int divides(int d, int n) { return FastDiv(d).of(n) == n / d && FastDiv(d).rest(n) == n % d; }
"""


@pytest.fixture(scope="module")
def plan(tmp_path_factory):
    cxx = shutil.which("g++") or shutil.which("c++")
    if cxx is None:
        pytest.skip("no C++ compiler")
    d = tmp_path_factory.mktemp("plan")
    (d / "shim.cpp").write_text(SHIM)
    so = str(d / "plan.so")
    subprocess.run([cxx, "-std=c++17", "-O1", "-w", "-shared", "-fPIC", "-D__HIP_PLATFORM_AMD__", f"-I{CSRC}",
                    "-I/opt/rocm/include", str(d / "shim.cpp"), os.path.join(CSRC, "paged_plan.cpp"),
                    os.path.join(CSRC, "decode_plan.cpp"), "-o", so], check=True)
    lib = ctypes.CDLL(so)
    lib.prefill_ws.restype = lib.decode_ws.restype = ctypes.c_size_t
    return lib


def _prefill(plan, units, tokens, group, cap, sinks, window, dtype, cus):
    got = (ctypes.c_int * 7)()
    plan.prefill(units, tokens, group, cap, sinks, window, dtype, cus, got)
    return list(got)


def _cases(n):
    r = random.Random(2)
    for _ in range(n):
        units = r.choice([1, 2, 3, 4, 7, 8, 16, 33, 64, 80, 112, 255, 256, 257, 1024, 1500, 4000])
        tokens = int(2 ** r.uniform(0, 14))
        cap = max(16, (tokens + int(2 ** r.uniform(0, 16))) // 16 * 16)
        window = r.choice([0, 0, 1, 100, 1024, 4096, 2 ** 31 - 1])
        yield (units, tokens, r.choice([1, 2, 4, 5, 7, 8, 16]), cap, r.choice([0, 4, 2 ** 31 - 1]), window,
               r.choice([0, 1]), r.choice([32, 256, 304]))


def test_every_block_is_done_once(plan):
    dealt = 0
    for case in _cases(600):
        units, tokens, group = case[:3]
        rows, blocks, splits, pieces, near, spread, fits = _prefill(plan, *case)
        if units * blocks > 200000:
            continue
        assert fits and 1 <= splits <= 64 and rows in (128, 256) and blocks == -(-tokens * group // rows), case
        if not pieces:                                     # a grid of units, blocks and splits
            assert blocks <= 65535 and units * splits < 2 ** 31
            assert splits == 1 or units * blocks * splits <= 2 * case[7], case
            continue
        dealt += 1
        assert splits == 1 and near <= 32
        size = -(-units * pieces // 8) * 8 * near
        assert size * 2 * rows < 2 ** 32
        seen = set()
        for wg in range(size):
            turn, pos = divmod(wg // 8, near)
            unit, j = divmod(turn * 8 + wg % 8, pieces)
            block = j + pieces * pos if spread else j * near + pos
            if unit < units and block < blocks:
                assert (unit, block) not in seen, case
                seen.add((unit, block))
        assert len(seen) == units * blocks, case
    assert dealt > 50


def test_partials_fit_their_workspace(plan):
    for case in _cases(2000):
        units, tokens, group, cap, sinks, window, dtype, cus = case
        rows, blocks, splits = _prefill(plan, *case)[:3]
        for dim in (64, 128):
            partials = units * blocks * splits * 128 * (dim + 2) * 4 if splits > 1 else 0
            assert plan.prefill_ws(units, tokens, cap, group, dim, dtype, cus) >= partials + 4 * units, case
            s = plan.decode(units, cap, sinks, window, cus)
            assert 1 <= s <= 128 and s <= plan.decode(units, cap, 0, 0, cus), case
            need = units * s * group * (dim + 2) * 4 + 4 * units
            assert plan.decode_ws(units, cap, group, dim, 0, cus) >= need, case
            assert plan.decode_ws(units, cap, group, dim, 1, cus) >= need + units * group * (cap + 1) * 4, case


def test_divisions(plan):
    r = random.Random(1)
    for d in list(range(1, 130)) + [1000, 65535, 1 << 20]:
        for n in [0, 1, d - 1, d, d + 1] + [r.randrange(min(1 << 28, (1 << 36) // d)) for _ in range(50)] + [min((1 << 28), (1 << 36) // d) - 1]:
            assert plan.divides(d, n), (d, n)
