"""kv_tables on memory that its lists share (no GPU): by how many launches it goes, the rule of kv_common.h compiled for the host, and what is refused."""
import ctypes
import os
import shutil
import subprocess

import pytest

from paper_2603_05232_amd import binding, build

SOURCE = """
#include "kv_common.h"
#include <stdio.h>
int main()
{
    long long lens, want, B, left, N, new_lens, new_left;
    auto at = [](long long x) { return reinterpret_cast<const int32_t*>((1 << 30) + 4 * x); };      // never read
    while (scanf("%lld %lld %lld %lld %lld %lld %lld", &lens, &want, &B, &left, &N, &new_lens, &new_left) == 7)
        printf("%d\\n", ss::kt_route(at(lens), at(want), B, at(left), N, at(new_lens), at(new_left)));
}
"""
WHOLE, EVERY, PLAN = range(3)


@pytest.fixture(scope="module")
def route(tmp_path_factory):
    hipcc = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
    if shutil.which(hipcc) is None:
        pytest.skip("no hipcc")
    d = tmp_path_factory.mktemp("route")
    (d / "route.cpp").write_text(SOURCE)
    subprocess.run([hipcc, "-x", "hip", "--offload-host-only", "--offload-arch=gfx950", "-std=c++17", "-I" + os.path.join(build.ROOT, "include"), "-I" + build.CSRC,
                    "-c", str(d / "route.cpp"), "-o", str(d / "route.o")], check=True)
    subprocess.run([hipcc, str(d / "route.o"), "-o", str(d / "route")], check=True)

    def ask(lens=0, want=10000, B=100, left=20000, N=5000, new_lens=30000, new_left=40000):
        """Lists by the number that they begin with."""
        out = subprocess.run([str(d / "route")], input=f"{lens} {want} {B} {left} {N} {new_lens} {new_left}\n", stdout=subprocess.PIPE, text=True, check=True).stdout
        return int(out)
    return ask


def test_every_workgroup_plans_only_from_memory_that_none_writes(route):
    assert route() == route(B=1024) == route(N=2049) == EVERY and route(N=2048) == WHOLE and route(B=1025) == PLAN
    assert route(new_lens=0) == route(new_left=20000) == PLAN                                          # in place
    assert route(new_lens=10000) == PLAN                                                               # lengths wanted
    assert route(new_lens=99) == route(new_lens=-99) == route(new_lens=10099) == route(new_lens=9901) == PLAN
    assert route(new_lens=100) == route(new_lens=-100) == route(new_lens=10100) == route(new_lens=9900) == EVERY      # side by side
    assert route(new_lens=20000) == route(new_lens=19901) == PLAN and route(new_lens=20001) == route(new_lens=19900) == EVERY
    assert route(new_left=99) == route(new_left=10050) == PLAN and route(new_left=100) == route(new_left=9999) == EVERY
    assert route(B=0, new_lens=0, want=0) == EVERY and route(B=0, new_left=20000) == PLAN              # lists of nothing share nothing
    assert route(N=2048, new_lens=10000) == WHOLE                                                      # one workgroup reads all before it writes


def test_results_that_share_memory_are_refused():
    lib = binding.load()
    assert lib.kv_tables.argtypes

    def call(B=4, N=16, lens=1 << 20, want=2 << 20, table=3 << 20, pool=4 << 20, left=5 << 20, new_lens=6 << 20, new_left=7 << 20, slots=8 << 20, offsets=9 << 20):
        p = ctypes.c_void_p
        return lib.kv_tables(p(lens), p(want), B, p(table), 8, 8, 64, p(pool), 100, p(left), N, p(new_lens), p(new_left), p(slots), p(offsets), None, 0, None)
    for given in ("lens", "want", "left", "new_lens", "new_left"):
        start = {"lens": 1, "want": 2, "left": 5, "new_lens": 6, "new_left": 7}[given] << 20
        assert call(slots=start) == call(offsets=start) == call(slots=start - 15 * 4) == call(offsets=start - 4 * 4) == 3
    assert call(slots=9 << 20) == call(offsets=(8 << 20) + 15 * 4) == call(new_left=(6 << 20) + 12) == 3
