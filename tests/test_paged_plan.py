"""How the attention over pages is cut (the library's own source, built for the host): the workspace holds the partials of the call and of every
smaller one."""
import ctypes as C
import os
import shutil
import subprocess

import pytest

from paper_2604_16498_amd import build

SHIM = """
#include <stdint.h>
namespace forge {
inline int ceil_div(int a, int b) { return (a + b - 1) / b; }
inline int64_t ceil_div64(int64_t a, int64_t b) { return (a + b - 1) / b; }
}
#include "%s"
using namespace forge;
extern "C" size_t room(int B, int Hq, int Hkv, int dh, int len, int cus) { return paged_room(B, Hq, Hkv, dh, len, cus); }
// bytes of the partials that a call writes (0: none), by the launcher's layout: the outputs' rows, then their statistics
extern "C" size_t written(int B, int Hq, int Hkv, int dh, int len, int bytes, int cus) {
  const TreePlan p = plan_paged(B, Hq, Hkv, dh, len, bytes, cus);
  const size_t rows = (size_t)p.shares * p.row_blocks * 2 * 16;
  return p.block_rows != 16 || p.row_blocks * 16 < Hq / Hkv ? ~(size_t)0 : p.dealt ? (rows * dh + rows * 2) * sizeof(float) : 0;
}
"""


@pytest.fixture(scope="module")
def host(tmp_path_factory):
    if shutil.which("g++") is None:
        pytest.skip("no host compiler")
    d = tmp_path_factory.mktemp("plan")
    (d / "shim.cpp").write_text(SHIM % os.path.join(build.CSRC, "paged_plan.hpp"))
    subprocess.run(["g++", "-O2", "-shared", "-fPIC", str(d / "shim.cpp"), "-o", str(d / "shim.so")], check=True)
    lib = C.CDLL(str(d / "shim.so"))
    lib.room.restype = lib.written.restype = C.c_size_t
    return lib


@pytest.mark.parametrize("cus", [1, 64, 256, 304])
@pytest.mark.parametrize("Hq,Hkv", [(1, 1), (12, 12), (32, 8), (17, 1), (40, 1), (33, 3), (1000, 2), (300, 300), (4096, 4096)])
def test_a_workspace_holds_the_partials_of_every_smaller_call(host, Hq, Hkv, cus):
    lens, batches = [1, 100, 512, 513, 640, 2049, 5000, 30011, 1 << 20], [1, 2, 7, 16, 64, 255, 256, 257, 5000]
    dealt = 0
    for dh in (64, 128):
        for bytes_ in (1, 2, 4):
            writes = {(b, n): host.written(b, Hq, Hkv, dh, n, bytes_, cus) for b in batches for n in lens}
            for B in batches:
                for top in lens:
                    room = host.room(B, Hq, Hkv, dh, top, cus)
                    assert all(w <= room for (b, n), w in writes.items() if b <= B and n <= top), (dh, bytes_, B, top)
            dealt += sum(w > 0 for w in writes.values())
    assert dealt > 0 or cus == 1 or Hkv >= 300          # (the cut that writes them is among these)
