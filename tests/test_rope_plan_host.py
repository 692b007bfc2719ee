"""Which rotations and appends are one workgroup's run, and which read past the caches, by the
function that plans them, without a GPU."""
import ctypes
import os
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2608_04771_amd", "csrc")
SHIM = r'''
#include "rope.hpp"
extern "C" int plan(int append, int layers, int batch, int tokens, int heads, int hkv, int row_bytes, int *block) {
  reco::RopeParams p{};
  p.layers = layers;
  p.batch = batch;
  p.tokens = tokens;
  p.heads = heads;
  p.c.hkv = hkv;
  p.c.k = append ? &p : nullptr;
  reco::rope_plan(p, row_bytes);
  *block = p.block;
  return p.far;
}
'''


@pytest.fixture(scope="module")
def plan(tmp_path_factory):
    d = tmp_path_factory.mktemp("rope")
    (d / "shim.cpp").write_text(SHIM)
    lib = str(d / "plan.so")
    subprocess.run(["g++", "-std=c++17", "-O1", "-shared", "-fPIC", "-D__HIP_PLATFORM_AMD__", f"-I{CSRC}", f"-I{ROOT}/include",
                    "-I/opt/rocm/include", str(d / "shim.cpp"), os.path.join(CSRC, "paged_plan.cpp"),
                    os.path.join(CSRC, "decode_plan.cpp"), "-o", lib], check=True)
    f = ctypes.CDLL(lib).plan

    def call(append, layers, batch, tokens, heads, hkv, row_bytes):
        block = ctypes.c_int()
        far = f(append, layers, batch, tokens, heads, hkv, row_bytes, ctypes.byref(block))
        return bool(far), block.value
    return call


def test_rows_past_the_caches(plan):
    # 64 MiB of rows: those of q, and of K and V where they are appended
    most = 64 << 20
    for append, layers, batch, heads, hkv, row_bytes in ((0, 1, 1, 32, 0, 256), (0, 3, 2, 36, 0, 128), (0, 1, 1, 10, 0, 512),
                                                         (1, 1, 1, 28, 4, 256), (1, 2, 5, 0, 8, 512), (1, 1, 1, 1024, 2, 128)):
        a_token = layers * batch * (heads + 2 * hkv) * row_bytes
        n = most // a_token
        assert not plan(append, layers, batch, n, heads, hkv, row_bytes)[0]
        assert plan(append, layers, batch, n + 1, heads, hkv, row_bytes)[0]
    assert plan(1, 65535, 1, 1 << 24, 1024, 1, 512)[0]     # past 32 bits, too


def test_tokens_of_a_workgroup(plan):
    for tokens, rotation, append in ((1, 1, 1), (2, 2, 2), (3, 4, 4), (4, 4, 4), (5, 4, 8), (8, 4, 8), (9, 4, 4), (1 << 24, 4, 4)):
        assert plan(0, 1, 1, tokens, 4, 0, 256)[1] == rotation
        assert plan(1, 1, 1, tokens, 4, 2, 256)[1] == append
