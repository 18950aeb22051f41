"""Which kernel and which cut the attention of drafted trees takes (the library's own source, built for the host): that the calls of
tree_plan_cases.py are cut as listed there, and that they leave out none of the kernels for any type of cache and head size."""
import ctypes as C
import os
import shutil
import subprocess

import pytest

from paper_2604_16498_amd import build
from tree_plan_cases import CASES

SHIM = """
#include <stdint.h>
namespace forge {
inline int ceil_div(int a, int b) { return (a + b - 1) / b; }
inline int64_t ceil_div64(int64_t a, int64_t b) { return (a + b - 1) / b; }
}
#include "%s"
extern "C" void plan(const int* a, int* o) {
  const forge::TreePlan p = forge::plan_tree(a[0], a[1], a[2], a[3], a[4], a[5], a[6], a[7], a[8] != 0, a[9]);
  o[0] = p.block_rows; o[1] = p.row_blocks; o[2] = p.shares; o[3] = p.dealt; o[4] = p.each;
}
extern "C" size_t room(const int* a) {
  return forge::tree_workspace_bytes(a[0], a[1], a[2], a[3], a[4], a[5], a[6], a[7] == 4, a[9]);
}
"""
BYTES = {"8 bits": 1, "bf16": 2, "fp32": 4}


@pytest.fixture(scope="module")
def host(tmp_path_factory):
    if shutil.which("g++") is None:
        pytest.skip("no host compiler")
    d = tmp_path_factory.mktemp("plan")
    (d / "shim.cpp").write_text(SHIM % os.path.join(build.CSRC, "tree_plan.hpp"))
    subprocess.run(["g++", "-O1", "-shared", "-fPIC", str(d / "shim.cpp"), "-o", str(d / "shim.so")], check=True)
    lib = C.CDLL(str(d / "shim.so"))
    lib.room.restype = C.c_size_t
    return lib


def ask(host, store, B, n, Hq, Hkv, dh, length, cap, ragged=True):
    """((rows a block, blocks of rows, cut), shares, bytes of workspace), on 256 compute units"""
    a, o = (C.c_int * 10)(B, Hq, Hkv, dh, n, length, cap, BYTES[store], ragged, 256), (C.c_int * 5)()
    host.plan(a, o)
    return (o[0], o[1], "each" if o[4] else "dealt" if o[3] else "whole"), o[2], host.room(a)


@pytest.mark.parametrize("store", list(CASES))
def test_cases_are_cut_as_listed(host, store):
    for (B, n, Hq, Hkv, dh, top), want in CASES[store]:
        assert ask(host, store, B, n, Hq, Hkv, dh, top + n, top + n + 3)[0] == want, (B, n, Hq, Hkv, dh, top)


@pytest.mark.parametrize("store", list(CASES))
def test_cases_leave_nothing_out(store):
    blocks = [16] if store == "fp32" else [16, 32, 128, 256]
    want = {(dh, r, cut) for dh in (64, 128) for r in blocks for cut in ("whole", "dealt", "each") if cut != "each" or r == 16}
    assert {(c[4], p[0], p[2]) for c, p in CASES[store]} == want


@pytest.mark.parametrize("store", list(CASES))
def test_a_workspace_holds_the_partials_of_every_shorter_cache(host, store):
    """2 slots of a block's rows for each share and block of rows, an output row and two statistics each"""
    for (B, n, Hq, Hkv, dh, top), _ in CASES[store]:
        room = ask(host, store, B, n, Hq, Hkv, dh, top + n, top + n)[2]
        for length in [n, top + n] + list(range(n, top + n, max(1, top // 40))):
            for ragged in (False, True):
                (rows, blocks, cut), shares, _ = ask(host, store, B, n, Hq, Hkv, dh, length, top + n, ragged)
                assert cut != "dealt" or shares * blocks * 2 * rows * (dh + 2) * 4 <= room
                assert blocks * rows >= Hq // Hkv * n > (blocks - 1) * rows
