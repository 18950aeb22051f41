"""Which kernels and which cut the adapters take (the library's own source, built for the host): that the calls of adapter_plan_cases.py take what is
listed there and leave out nothing, and that the workspace holds what the first launch writes."""
import ctypes as C
import os
import shutil
import subprocess

import pytest

from adapter_plan_cases import CASES
from paper_2604_16498_amd import build

SHIM = """
#include <stdint.h>
namespace forge {
inline int ceil_div(int a, int b) { return (a + b - 1) / b; }
inline int64_t ceil_div64(int64_t a, int64_t b) { return (a + b - 1) / b; }
}
#include "%s"
using namespace forge;
extern "C" void plan(int M, int K, int parts, const int* ends, int rank, int ldy, int f32, int cus, int* o) {
  const int N = ends[parts - 1], inner = parts * rank;
  const bool many = adapters_many(M, N, inner, f32);
  const Cut c = adapters_cut(M, K, inner, many, f32, cus);
  o[0] = many ? 64 : 16; o[1] = many && adapters_whole(ldy, parts, ends) ? 64 : 16; o[2] = adapters_steps(rank, f32);
  o[3] = c.splits; o[4] = c.tiles; o[5] = c.chunks; o[6] = c.lanes;
}
extern "C" size_t room(int M, int K, int inner, int f32, int cus) { return adapters_room(M, K, inner, f32, cus); }
// the first of m = 1 .. M rows whose t of all ranges has no room in the workspace of M rows, 0 where there is none
extern "C" int first_without_room(int M, int K, int N, int parts, int rank, int f32, int cus) {
  const int inner = parts * rank;
  const size_t have = adapters_room(M, K, inner, f32, cus);
  for (int m = 1; m <= M; ++m) {
    const Cut c = adapters_cut(m, K, inner, adapters_many(m, N, inner, f32), f32, cus);
    if ((size_t)c.splits * m * inner * sizeof(float) > have) return m;
  }
  return 0;
}
"""


@pytest.fixture(scope="module")
def host(tmp_path_factory):
    if shutil.which("g++") is None:
        pytest.skip("no host compiler")
    d = tmp_path_factory.mktemp("plan")
    (d / "shim.cpp").write_text(SHIM % os.path.join(build.CSRC, "adapters_plan.hpp"))
    subprocess.run(["g++", "-O2", "-shared", "-fPIC", str(d / "shim.cpp"), "-o", str(d / "shim.so")], check=True)
    lib = C.CDLL(str(d / "shim.so"))
    lib.room.restype = C.c_size_t
    return lib


def ask(host, dt, M, K, ends, rank, ldy, cus=256):
    """(rows a block of the two launches, steps), splits, tiles, chunks, lanes"""
    o = (C.c_int * 7)()
    host.plan(M, K, len(ends), (C.c_int * 4)(*ends), rank, ldy or ends[-1], dt == "fp32", cus, o)
    return tuple(o[:3]), o[3], o[4], o[5], o[6]


@pytest.mark.parametrize("dt", list(CASES))
def test_cases_take_what_is_listed(host, dt):
    for call, want in CASES[dt]:
        assert ask(host, dt, *call)[0] == want, call


@pytest.mark.parametrize("dt", list(CASES))
def test_cases_leave_nothing_out(host, dt):
    steps = (1, 2, 4) if dt == "bf16" else (1, 2, 4, 8)
    assert {w for _, w in CASES[dt]} == {(a, b, s) for a, b in ((64, 64), (64, 16), (16, 16)) for s in steps}


# ends of the range of every argument that the sizes depend on; few and many compute units
@pytest.mark.parametrize("cus", [1, 64, 256, 304])
@pytest.mark.parametrize("dt", list(CASES))
def test_a_workspace_holds_what_is_written_for_it_and_every_smaller_call(host, dt, cus):
    for K in (8, 768, 4096, 14336):
        for N in (16, 768, 4096, 28672):
            for rank, parts in ((8, 1), (16, 3), (64, 1), (128, 4)):
                for M in (1, 7, 16, 100, 511, 512, 513, 1500, 4100):
                    m = host.first_without_room(M, K, N, parts, rank, dt == "fp32", cus)
                    assert m == 0, (K, N, rank, parts, M, m)


@pytest.mark.parametrize("dt", list(CASES))
def test_every_range_of_k_has_a_unit_and_every_lane_an_adapter(host, dt):
    for call, _ in CASES[dt] + [((m, k, [4096], r, None), None) for m in (1, 3, 17, 300, 2000) for k in (8, 264, 4096, 14336) for r in (8, 128)]:
        (rows, _, _), splits, tiles, chunks, lanes = ask(host, dt, *call)
        M, K, ends, rank = call[:4]
        assert 1 <= splits <= -(-K // (128 if dt == "fp32" else 256)) and tiles == -(-M // rows) and chunks == -(-len(ends) * rank // 64)
        assert 1 <= lanes <= min(M, 16)
