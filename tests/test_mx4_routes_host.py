"""Which kernel of the microscaled products the shapes of the GPU tests go to (on 256 compute units): the choice of mx4_choice.h, compiled for the host.  All kernels
together, dense and grouped, on rows split and whole, have a test."""
import os
import shutil
import subprocess

import pytest

import test_gpu_mx4
import test_gpu_mx4_kernels
from paper_2603_05232_amd import binding, build

SOURCE = """
#include "mx4_choice.h"
#include <stdio.h>
int main()
{
    long long R, E, U, frags; unsigned long long ws;
    while (scanf("%lld %lld %lld %lld %llu", &R, &E, &U, &frags, &ws) == 5) {
        const ss::mx4_plan p = ss::mx4_choose(R, E, U, frags, 256, (size_t)ws);
        printf("%d %d %d %d\\n", p.kernel, p.ranges, ss::MX_MID, ss::MX_SHORT);
    }
}
"""
ALL = 1 << 62                                                # a workspace for anything
STREAM, SHORT, MID, TILE = "stream", "short rows", "128 channels", "256 channels"


@pytest.fixture(scope="module")
def plans(tmp_path_factory):
    hipcc = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
    if shutil.which(hipcc) is None:
        pytest.skip("no hipcc")
    binding.load()
    d = tmp_path_factory.mktemp("plan")
    (d / "plan.cpp").write_text(SOURCE)
    subprocess.run([hipcc, "-x", "hip", "--offload-host-only", "--offload-arch=gfx950", "-std=c++17", "-I" + os.path.join(build.ROOT, "include"), "-I" + build.CSRC,
                    "-c", str(d / "plan.cpp"), "-o", str(d / "plan.o")], check=True)
    subprocess.run([hipcc, str(d / "plan.o"), "-o", str(d / "plan")], check=True)

    def ask(shapes, ws):
        """(kernel, its rows, ranges, units of a row) of shapes (R, E, K, O, gated)."""
        lines = [f"{R} {E} {-(-K // 256)} {-(-(O << gated) // 32)} {ws}\n" for R, E, K, O, gated in shapes]
        out = subprocess.run([str(d / "plan")], input="".join(lines), stdout=subprocess.PIPE, text=True, check=True).stdout
        answers = []
        for (R, E, K, O, gated), line in zip(shapes, out.splitlines(), strict=True):
            kernel, ranges, mid, short = map(int, line.split())
            family, rows = (SHORT, kernel - short) if kernel >= short else (MID, kernel - mid) if kernel >= mid else (TILE, 256) if kernel == 256 else (STREAM, kernel)
            answers.append((family, rows, ranges, -(-K // 256)))
        return answers
    return ask


def _dense(shapes):
    return [(M, 1, K, O, gated) for M, K, O, gated in shapes]


def test_shapes_that_name_their_kernel(plans):
    dense = [s[:4] for s in test_gpu_mx4_kernels.DENSE]
    for s, p in zip(test_gpu_mx4_kernels.DENSE, plans(_dense(dense), ALL), strict=True):
        assert p[:3] == (MID, *s[4:]), (s, p)
    for s, p in zip(test_gpu_mx4_kernels.GROUPED, plans([s[:5] for s in test_gpu_mx4_kernels.GROUPED], ALL), strict=True):
        assert p[:3] == (MID, *s[6:]), (s, p)


def test_short_rows(plans):
    shapes = [(R, E, K, O, gated) for R, K, O, E in test_gpu_mx4.SHORT for gated in (False, True)]
    taken = {(p[1], p[3], s[1] > 1) for s, p in zip(shapes, plans(shapes, 0), strict=True) if p[0] == SHORT}
    assert taken == {(rows, units, grouped) for rows in (16, 32) for units in (1, 2, 3, 4) for grouped in (False, True)}


def test_every_kernel_has_a_shape(plans):
    both = (False, True)
    dense = _dense([(M, K, O, g) for M, K, O in test_gpu_mx4.SHAPES for g in both] + test_gpu_mx4.FULL + [s[:4] for s in test_gpu_mx4_kernels.DENSE])
    grouped = [(R, E, K, O, g) for R, E, K, O, _ in test_gpu_mx4.GROUPED for g in both] + test_gpu_mx4.GROUPED_FULL + [s[:5] for s in test_gpu_mx4_kernels.GROUPED]
    for shapes in (dense, grouped):
        seen = set()
        for ws in (0, ALL):
            for family, rows, ranges, units in plans(shapes, ws):
                if family != SHORT:
                    seen.add((family, rows, "split" if ranges > 1 else "short" if units < {(STREAM, 16): 16, (TILE, 256): 3}.get((family, rows), 0) else ""))
        assert seen == {(STREAM, 16, "short"), (STREAM, 16, ""), (STREAM, 32, ""), (TILE, 256, "short"), (TILE, 256, "")} | {
            (MID, rows, kind) for rows in (32, 64, 128) for kind in ("", "split")}
