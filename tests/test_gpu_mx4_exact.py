"""Microscaled products on operands whose sums are exact: every result has to be bf16 of the exact sum.  Long rows and rows split into ranges above all."""
import numpy as np
import pytest
import torch

import mx4_exact as ex
from paper_2603_05232_amd import binding
from test_gpu_mx4 import FULL, GROUPED_FULL, groups

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def check(Y, x, w, gated):
    sums = x @ w.t()
    bad = ex.wrong_gated(Y, *sums.chunk(2, dim=1)) if gated else ex.wrong(Y, sums)
    assert not bool(bad.any()), (int(bad.sum()), bad.nonzero()[:4].tolist())


def run_dense(M, K, O, gated):
    g = torch.Generator(device=DEV).manual_seed(M + K + O)
    middle = 123 if gated else 127                              # gates of some units
    xc, wc = ex.operand(g, M, K, middle), ex.operand(g, O << gated, K, middle)
    x, w = ex.values(*xc), ex.values(*wc)
    assert ex.sums_are_exact(x, w, middle, middle)
    packed = binding.mx4_pack(*wc, K, gated=gated)
    n = binding.mx4_gemm_workspace_bytes(M, O, K, gated=gated)
    for ws in [None] + ([torch.full((n,), 0x5A, dtype=torch.uint8, device=DEV)] if n else []):
        check(binding.mx4_gemm(*xc, *packed, O, K, gated=gated, workspace=ws), x, w, gated)


def run_grouped(R, E, K, O, gated, kind="skewed"):
    g = torch.Generator(device=DEV).manual_seed(R + E + K + O)
    middle, rows_e = 123 if gated else 127, O << gated
    off = groups(kind, R, E, np.random.default_rng(R + K))
    xc, wc = ex.operand(g, R, K, middle), ex.operand(g, E * rows_e, K, middle)
    x = ex.values(*xc)
    packed = binding.mx4_pack(*wc, K, experts=E, gated=gated)
    offsets = torch.from_numpy(off.astype(np.int32)).to(DEV)
    n = binding.mx4_gemm_workspace_bytes(R, O, K, experts=E, gated=gated)
    for ws in [None] + ([torch.full((n,), 0x5A, dtype=torch.uint8, device=DEV)] if n else []):
        whole = torch.full((R + 2, O + 3), 7.0, dtype=torch.bfloat16, device=DEV)
        Y = binding.mx4_grouped_gemm(*xc, offsets, *packed, O, K, gated=gated, out=whole[1:R + 1, 1:O + 1], workspace=ws)
        for e in range(E):
            if off[e + 1] > off[e]:
                w = ex.values(wc[0][e * rows_e:(e + 1) * rows_e], wc[1][:, e * rows_e:(e + 1) * rows_e])
                assert ex.sums_are_exact(x, w, middle, middle)
                check(Y[off[e]:off[e + 1]], x[off[e]:off[e + 1]], w, gated)
        assert not bool(Y[off[-1]:].any())
        assert bool((whole[0] == 7).all()) and bool((whole[R + 1] == 7).all()) and bool((whole[:, :1] == 7).all()) and bool((whole[:, O + 1:] == 7).all())


@pytest.mark.parametrize("M,K,O,gated", FULL)
def test_dense(M, K, O, gated):
    run_dense(M, K, O, gated)


@pytest.mark.parametrize("R,E,K,O,gated", GROUPED_FULL)
def test_grouped(R, E, K, O, gated):
    run_grouped(R, E, K, O, gated)


@pytest.mark.parametrize("shift", [0, -40, 40, -100, 100])
@pytest.mark.parametrize("M,K,O", [(1, 512, 64), (40, 2304, 256), (300, 1024, 1000), (200, 2304, 2000), (3200, 2304, 4096), (4000, 256, 4096)])
def test_scales_over_their_whole_range(M, K, O, shift):
    """Scale bytes 0 .. 254 on either side, in blocks whose products come to about the same size, 2^shift."""
    g = torch.Generator(device=DEV).manual_seed(M + K + O + shift)
    xc, wc = ex.operand(g, M, K, 1), ex.operand(g, O, K, 1)
    blocks = K // 32
    b = torch.arange(blocks, device=DEV) * 252 // (blocks - 1)                 # 0 .. 252 below the smallest byte
    there = (252 + shift - b >= 0) & (252 + shift - b <= 252)                  # blocks that have a partner
    xs = xc[1] + b.view(-1, 1, 8).to(torch.uint8)
    ws = wc[1] + (252 + shift - b).clamp(0, 252).view(-1, 1, 8).to(torch.uint8)
    codes = xc[0] * there.repeat_interleave(16).to(torch.uint8)
    x, w = ex.values(codes, xs), ex.values(wc[0], ws)
    check(binding.mx4_gemm(codes, xs, *binding.mx4_pack(wc[0], ws, K), O, K), x, w, False)


@pytest.mark.parametrize("M,K,O", [(1, 512, 64), (40, 2304, 256), (200, 2304, 2000), (3200, 2304, 4096), (4000, 256, 4096)])
def test_results_below_the_normal_range(M, K, O):
    """Sums and results that are subnormal in 32 bits and in bf16."""
    g = torch.Generator(device=DEV).manual_seed(M + K + O)
    for middle in (111, 121):                                                   # products of 2^-146, 32 bits' smallest being 2^-149, and more
        xc, wc = ex.operand(g, M, K, 1), ex.operand(g, O, K, middle)
        check(binding.mx4_gemm(*xc, *binding.mx4_pack(*wc, K), O, K), ex.values(*xc), ex.values(*wc), False)
