"""Memory that lists and rows share (no GPU): by how many launches kv_tables goes, the rule of kv_common.h compiled for the host, and what is refused."""
import ctypes
import os
import random
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
    if (scanf("%lld %lld %lld %lld %lld", &lens, &want, &B, &left, &N) != 5) return 1;
    if (lens >= 0) { printf("%d\\n", ss::kv_rows_apart(lens, want, B, left, N)); return 0; }
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
        out = subprocess.run([str(d / "route")], input=f"-1 0 0 0 0 {lens} {want} {B} {left} {N} {new_lens} {new_left}\n", stdout=subprocess.PIPE, text=True, check=True).stdout
        return int(out)
    ask.program = str(d / "route")
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


def test_result_rows_that_overlap_are_refused():
    lib = binding.load()
    assert lib.kv_read.argtypes
    p = ctypes.c_void_p

    def read(N=4, H=8, D=64, K=(512, 64), V=(512, 64)):
        return lib.kv_read(p(1 << 20), 10, 64, 2, p(2 << 20), N, H, D, 1, p(3 << 20), *K, p(4 << 20), *V, None)

    def attend(B=4, Hq=8, D=64, out=(512, 64)):
        return lib.kv_attention(p(1 << 20), 1, 512, 64, p(2 << 20), 10, 64, 2, p(3 << 20), 4, 4, p(4 << 20), B, Hq, 4, D, 1.0, 0, p(5 << 20), *out, None, 0, None)
    assert read(K=(512, 64), N=1, V=(0, 32)) == 3
    for rows in ((0, 64), (512, 0), (63, 64), (512, 63), (63, 4096), (4096, 32), (256, 64), (64, 128), (100, 90)):
        assert read(K=rows) == read(V=rows) == attend(out=rows) == 3, rows


def test_rows_apart_is_what_counting_finds(route):
    rng = random.Random(1)
    shapes = [(rng.randint(1, 5), rng.randint(0, 40), rng.randint(1, 5), rng.randint(0, 40), rng.randint(1, 9)) for _ in range(150)] + [(2, 5, 3, 2, 1), (3, 2, 2, 5, 2), (2, 1 << 40, 1024, 1 << 40, 256)]
    answers = []
    for N, ld, H, hs, D in shapes:
        out = subprocess.run([route.program], input=f"{N} {ld} {H} {hs} {D}\n", stdout=subprocess.PIPE, text=True, check=True).stdout
        places = [n * ld + h * hs + d for n in range(N) for h in range(H) for d in range(D)]
        answers.append(int(out))
        assert int(out) == (len(set(places)) == len(places)), (N, ld, H, hs, D)
    assert 30 < sum(answers) < 120
