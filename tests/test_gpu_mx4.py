"""Microscaled 4-bit quantisation and products against the oracle (64 bits).  Codes, scales and read-back values are equal bit for bit.  Products: bf16's
rounding (2^-8 of the result, twice what it can be) and K 2^-23 of the sum of magnitudes for 32-bit sums of exact products."""
import numpy as np
import pytest
import torch

from oracle import mx4_oracle as mo
from paper_2603_05232_amd import binding

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
DTYPES = {"fp32": torch.float32, "bf16": torch.bfloat16}


def inputs(R, K, dtype, seed):
    """Rows with outliers, zeros of both signs, blocks of zeros, values at the ties and far-apart magnitudes."""
    rng = np.random.default_rng(seed)
    x = rng.standard_normal((R, K)) * np.exp2(rng.integers(-8, 9, (R, 1)))
    x[:, rng.integers(0, K, max(1, K // 50))] *= 20
    x[rng.random((R, K)) < 0.05] = -0.0
    x[0, :32] = 0
    ties = rng.random((R, K)) < 0.1
    x[ties] = (rng.choice([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5, 7], (R, K)) * rng.choice([-1, 1], (R, K)))[ties]
    return torch.from_numpy(x).to(DTYPES[dtype]).to(DEV)


def as_codes(code, b, dev=DEV):
    return torch.from_numpy(mo.pack_codes(code)).to(dev), torch.from_numpy(np.ascontiguousarray(b.transpose(1, 0, 2))).to(dev)


def random_operand(rng, R, K, spread=3):
    """Codes and scales that need not come from a quantiser, zeros beyond K."""
    U = -(-K // 256)
    code = rng.integers(0, 16, (R, U * 256))
    code[:, K:] = 0
    return code.reshape(R, U, 256).astype(np.uint8), (127 + rng.integers(-spread, spread + 1, (R, U, 8))).astype(np.uint8)


def check_product(Y, ref, off):
    got = Y.double().cpu().numpy()
    assert got.shape == ref.shape
    bad = ~(np.abs(got - ref) <= 2.0 ** -8 * np.abs(ref) + off)
    assert not bad.any(), (int(bad.sum()), np.argwhere(bad)[:4].tolist())


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("R,K", [(1, 1), (1, 31), (3, 32), (2, 33), (5, 255), (7, 256), (4, 513), (130, 1000), (1, 18944), (33, 5003)])
def test_quant_and_back(R, K, dtype):
    X = inputs(R, K, dtype, seed=R + K)
    codes, scales = binding.mx4_quant(X)
    code, b = mo.quant(X.double().cpu().numpy())
    want_codes, want_scales = as_codes(code, b, "cpu")
    assert torch.equal(scales.cpu(), want_scales)
    assert torch.equal(codes.cpu(), want_codes)
    want = torch.from_numpy(mo.values(code, b)[:, :K].copy())
    for out in DTYPES.values():
        back = binding.mx4_dequant(codes, scales, K, out)
        assert back.dtype == out and torch.equal(back.cpu().double(), want) and torch.equal(torch.signbit(back.cpu()), torch.signbit(want))


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_quant_of_every_exponent_and_of_what_is_no_number(dtype):
    X = torch.ones((256, 96), dtype=torch.float64)
    X *= torch.exp2(torch.arange(256, dtype=torch.float64) - 127).clamp(max=2.0 ** 127)[:, None] * torch.linspace(0.01, 1.99, 96, dtype=torch.float64)
    X = X.to(DTYPES[dtype]).clamp(-3e38, 3e38)
    X[3, 40], X[5, 0], X[6, 95] = float("inf"), float("nan"), float("-inf")
    codes, scales = binding.mx4_quant(X.to(DEV))
    code, b = mo.quant(X.double().numpy())
    want_codes, want_scales = as_codes(code, b, "cpu")
    assert torch.equal(scales.cpu(), want_scales) and torch.equal(codes.cpu(), want_codes)
    back = binding.mx4_dequant(codes, scales, 96, torch.float32).cpu().double().numpy()
    want = mo.values(code, b)[:, :96]
    assert np.array_equal(back, want, equal_nan=True) and np.isnan(want).sum() == 96


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("K", [64, 300])
def test_quant_of_strided_and_gathered_rows(K, dtype):
    whole = inputs(50, K + 7, dtype, seed=K)
    X = whole[:, 3:3 + K]                                       # rows off every line
    rows = torch.tensor([4, 4, 49, 0, -1, 50, 2 ** 30, -2 ** 31, 7], dtype=torch.int32, device=DEV)
    codes, scales = binding.mx4_quant(X, rows=rows)
    x = X.double().cpu().numpy()
    there = [4, 4, 49, 0, None, None, None, None, 7]
    code, b = mo.quant(np.stack([np.zeros(K) if r is None else x[r] for r in there]))
    want_codes, want_scales = as_codes(code, b, "cpu")
    assert torch.equal(codes.cpu(), want_codes) and torch.equal(scales.cpu(), want_scales)
    out = torch.full((9, K + 5), 7.0, dtype=DTYPES[dtype], device=DEV)
    binding.mx4_dequant(codes, scales, K, out=out[:, 1:K + 1])
    assert torch.equal(out[:, 1:K + 1].cpu().double(), torch.from_numpy(mo.values(code, b)[:, :K].copy()))
    assert bool((out[:, :1] == 7).all()) and bool((out[:, K + 1:] == 7).all())


def test_empty():
    X = torch.zeros((0, 64), device=DEV)
    codes, scales = binding.mx4_quant(X)
    assert codes.shape == (0, 128) and scales.shape == (1, 0, 8) and binding.mx4_dequant(codes, scales, 64).shape == (0, 64)
    w = binding.mx4_pack(*binding.mx4_quant(torch.ones((40, 64), device=DEV)), 64)
    assert binding.mx4_gemm(codes, scales, *w, 40, 64).shape == (0, 40)


SHAPES = [(1, 1, 1), (1, 32, 33), (2, 256, 32), (31, 257, 31), (32, 512, 64), (33, 1000, 129), (64, 768, 96), (65, 2048, 100), (100, 300, 1000),
          (128, 1280, 256), (200, 4099, 77), (257, 512, 513), (300, 1024, 640), (520, 256, 300), (1, 18944, 256), (16, 8192, 160), (700, 2304, 1030)]


@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("M,K,O", SHAPES)
def test_gemm(M, K, O, gated):
    rng = np.random.default_rng(M * 7 + K * 3 + O)
    xc, wc = random_operand(rng, M, K), random_operand(rng, O << gated, K)
    w = binding.mx4_pack(*as_codes(*wc), K, gated=gated)
    n = binding.mx4_gemm_workspace_bytes(M, O, K, gated=gated)
    ref, off = mo.product(mo.values(*xc) * 2.0 ** -4, mo.values(*wc), gated)
    xc = (xc[0], xc[1] - 4)
    for ws in [None] + ([torch.full((n,), 0x5A, dtype=torch.uint8, device=DEV)] if n else []):
        whole = torch.full((M + 2, O + 3), 7.0, dtype=torch.bfloat16, device=DEV)
        Y = binding.mx4_gemm(*as_codes(*xc), *w, O, K, gated=gated, out=whole[1:M + 1, 2:O + 2], workspace=ws)
        check_product(Y, ref, off)
        assert bool((whole[0] == 7).all()) and bool((whole[M + 1] == 7).all()) and bool((whole[:, :2] == 7).all()) and bool((whole[:, O + 2:] == 7).all())
        again = binding.mx4_gemm(*as_codes(*xc), *w, O, K, gated=gated, workspace=ws)
        assert torch.equal(again.view(torch.int16), Y.contiguous().view(torch.int16))


def test_gemm_carries_what_is_no_number():
    X = torch.randn((70, 600), device=DEV)
    X[3, 599], X[66, 0] = float("nan"), float("inf")
    W = torch.randn((90, 600), device=DEV)
    W[5, 300] = float("nan")
    Y = binding.mx4_gemm(*binding.mx4_quant(X), *binding.mx4_pack(*binding.mx4_quant(W), 600), 90, 600)
    want = torch.zeros((70, 90), dtype=torch.bool)
    want[[3, 66]] = True
    want[:, 5] = True
    assert torch.equal(Y.isnan().cpu(), want)


def test_sums_keep_32_bits():
    # 2^20 + 1 - 2^20 over blocks of one unit, over units, and within a block beside +-36 2^10
    K = 1024
    for places in [(0, 40, 80), (0, 200, 255), (0, 300, 900)]:
        x, w = torch.zeros((1, K), device=DEV), torch.zeros((32, K), device=DEV)
        for p, v in zip(places, (2.0 ** 20, 1.0, -2.0 ** 20)):
            x[0, p], w[:, p] = v, 1.0
        assert bool((binding.mx4_gemm(*binding.mx4_quant(x), *binding.mx4_pack(*binding.mx4_quant(w), K), 32, K) == 1).all())


def groups(kind, R, E, rng):
    if kind == "even":
        sizes = np.full(E, R // E)
        sizes[: R - sizes.sum()] += 1
    elif kind == "one":
        sizes = np.zeros(E, int)
        sizes[E // 2] = R
    else:                                                       # skewed, some empty, some rows of no expert
        p = rng.dirichlet(np.full(E, 0.3))
        sizes = rng.multinomial(max(0, R - R // 9), p)
    return np.concatenate([[0], np.cumsum(sizes)])


GROUPED = [(1, 2, 256, 32, "one"), (5, 64, 300, 40, "skewed"), (16, 8, 1024, 96, "even"), (70, 3, 513, 100, "skewed"), (130, 130, 256, 33, "skewed"),
           (300, 5, 800, 200, "skewed"), (400, 1, 512, 256, "even"), (1000, 4, 640, 300, "skewed"), (600, 1024, 64, 32, "skewed"), (900, 7, 1536, 520, "even"),
           (1500, 3, 512, 640, "one")]


@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("R,E,K,O,kind", GROUPED)
def test_grouped(R, E, K, O, kind, gated):
    rng = np.random.default_rng(R * 5 + E + K + O)
    off = groups(kind, R, E, rng)
    xc, wc = random_operand(rng, R, K), random_operand(rng, E * (O << gated), K)
    ref, tol = np.zeros((R, O)), np.zeros((R, O))
    xc = (xc[0], xc[1] - 4)
    xv, wv = mo.values(*xc), mo.values(*wc).reshape(E, O << gated, -1)
    for e in range(E):
        if off[e + 1] > off[e]:
            ref[off[e]:off[e + 1]], tol[off[e]:off[e + 1]] = mo.product(xv[off[e]:off[e + 1]], wv[e], gated)
    w = binding.mx4_pack(*as_codes(*wc), K, experts=E, gated=gated)
    offsets = torch.from_numpy(off.astype(np.int32)).to(DEV)
    n = binding.mx4_gemm_workspace_bytes(R, O, K, experts=E, gated=gated)
    for ws in [None] + ([torch.full((n,), 0x5A, dtype=torch.uint8, device=DEV)] if n else []):
        whole = torch.full((R + 2, O + 3), 7.0, dtype=torch.bfloat16, device=DEV)
        Y = binding.mx4_grouped_gemm(*as_codes(*xc), offsets, *w, O, K, gated=gated, out=whole[1:R + 1, 1:O + 1], workspace=ws)
        check_product(Y, ref, tol)
        assert bool((whole[0] == 7).all()) and bool((whole[R + 1] == 7).all()) and bool((whole[:, :1] == 7).all()) and bool((whole[:, O + 1:] == 7).all())


@pytest.mark.parametrize("off,means", [([0, 9, 4, 30], [0, 9, 9, 30]), ([5, -7, 20, 99], [0, 0, 20, 40]), ([0, 0, 0, 0], [0, 0, 0, 0])])
def test_offsets_out_of_order_stay_in_bounds(off, means):
    rng = np.random.default_rng(1)
    K, O, E, R = 256, 40, 3, 40
    xc, wc = random_operand(rng, R, K), random_operand(rng, E * O, K)
    xv, wv = mo.values(*xc), mo.values(*wc).reshape(E, O, K)
    ref, tol = np.zeros((R, O)), np.zeros((R, O))
    for e in range(E):
        ref[means[e]:means[e + 1]], tol[means[e]:means[e + 1]] = mo.product(xv[means[e]:means[e + 1]], wv[e])
    Y = binding.mx4_grouped_gemm(*as_codes(*xc), torch.tensor(off, dtype=torch.int32, device=DEV), *binding.mx4_pack(*as_codes(*wc), K, experts=E), O, K)
    check_product(Y, ref, tol)


def test_refused_tensors():
    X = torch.randn((4, 300), device=DEV)
    with pytest.raises(TypeError):
        binding.mx4_quant(X.half())
    with pytest.raises(TypeError):
        binding.mx4_quant(X, rows=torch.zeros(4, dtype=torch.int64, device=DEV))
    with pytest.raises(AssertionError):
        binding.mx4_quant(X.t())
    codes, scales = binding.mx4_quant(X)
    w = binding.mx4_pack(*binding.mx4_quant(torch.randn((64, 300), device=DEV)), 300)
    with pytest.raises(AssertionError):
        binding.mx4_gemm(codes, scales, *w, 64, 600)
    with pytest.raises(AssertionError):
        binding.mx4_gemm(codes, scales, *w, 65, 300)
    with pytest.raises(AssertionError):
        binding.mx4_gemm(codes, scales, *w, 64, 300, out=torch.empty((4, 64), device=DEV))
    with pytest.raises(TypeError):
        binding.mx4_grouped_gemm(codes, scales, torch.tensor([0, 4], device=DEV), *w, 64, 300)


def _sampled(rows, cols, codes, scales, w_codes, w_scales, gated, dev=DEV):
    """The products of some rows and columns of Y in 64 bits, from codes on the GPU, and the bound of 32-bit sums."""
    def values(c, s):
        c = c.cpu().numpy()
        code = np.stack([c & 15, c >> 4], axis=-1).reshape(c.shape[0], -1, 256)
        return mo.values(code, s.cpu().numpy().transpose(1, 0, 2))

    xv = values(codes[rows], scales[:, rows].contiguous())
    n = w_codes.shape[0] // 2
    wi = torch.cat([cols, cols + n]) if gated else cols
    return mo.product(xv, values(w_codes[wi], w_scales[:, wi].contiguous()), gated)


SHORT = [(3, 436, 8870, 1), (7, 256, 4100, 1), (64, 512, 8192, 1), (476, 303, 1000, 1), (256, 768, 4096, 1), (100, 1000, 8200, 1), (33, 640, 16384, 1), (500, 512, 2048, 64), (300, 256, 1000, 128),
         (256, 768, 2048, 32), (1016, 278, 1408, 69), (41, 412, 4224, 126), (300, 1024, 1408, 60), (5000, 250, 1030, 40), (2000, 900, 700, 100),
         (100, 250, 16384, 1), (3000, 256, 1025, 1), (1500, 512, 360, 1), (300, 768, 1024, 1), (1500, 700, 361, 1), (300, 1024, 1000, 1), (1500, 1000, 360, 1), (1500, 768, 512, 8), (1500, 1024, 511, 8),
         (1500, 1024, 1024, 64), (3000, 500, 130, 16)]


@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("R,K,O,E", SHORT)
def test_short_rows(R, K, O, E, gated):
    """Rows of one to four units, by tiles of 16 and 32 rows whose operands are in registers at once."""
    g = torch.Generator(device=DEV).manual_seed(R + K)
    off = groups("skewed", R, E, np.random.default_rng(R)) if E > 1 else np.array([0, R])
    codes, scales = binding.mx4_quant(torch.randn((R, K), generator=g, device=DEV))
    rows_e = O << gated
    wc, ws_ = binding.mx4_quant(0.1 * torch.randn((E * rows_e, K), generator=g, device=DEV))
    w = binding.mx4_pack(wc, ws_, K, experts=E, gated=gated)
    whole = torch.full((R + 2, O + 3), 7.0, dtype=torch.bfloat16, device=DEV)
    Y = whole[1:R + 1, 1:O + 1]
    if E > 1:
        binding.mx4_grouped_gemm(codes, scales, torch.from_numpy(off.astype(np.int32)).to(DEV), *w, O, K, gated=gated, out=Y)
    else:
        binding.mx4_gemm(codes, scales, *w, O, K, gated=gated, out=Y)
    assert bool((whole[0] == 7).all()) and bool((whole[R + 1] == 7).all()) and bool((whole[:, :1] == 7).all()) and bool((whole[:, O + 1:] == 7).all())
    rng = np.random.default_rng(E)
    cols = torch.from_numpy(np.unique(np.concatenate([rng.integers(0, O, 20), [0, O - 1]]))).to(DEV)
    for e in range(E):
        if off[e + 1] > off[e]:
            rows = torch.from_numpy(np.unique(np.concatenate([rng.integers(off[e], off[e + 1], 8), [off[e], off[e + 1] - 1]]))).to(DEV)
            part = slice(e * rows_e, (e + 1) * rows_e)
            ref, tol = _sampled(rows, cols, codes, scales, wc[part], ws_[:, part], gated)
            check_product(Y[rows][:, cols], ref, tol)
    assert not bool(Y[off[-1]:].any()) and not bool(Y.isnan().any())


# every kernel and several rounds of each: tiles of 256 x 256 (more of them than compute units, an odd last tile, rows of three units and of many), of 128 channels
# with 32, 64 and 128 rows, ranges of units, few tokens on long rows, rows of one and two units by enough tiles that those of 256 x 256 take them
FULL = [(4099, 800, 9001, False), (2100, 5120, 4224, False), (1500, 3584, 8200, True), (2304, 768, 16384, False), (777, 5003, 4099, False), (600, 4096, 4096, True),
        (200, 4096, 14336, False), (100, 4096, 14336, False), (256, 18944, 3584, False), (100, 14336, 4096, True), (777, 18944, 512, False), (48, 3584, 37888, False),
        (1, 18944, 3584, False), (17, 3584, 18944, True), (40, 600, 600, False),
        (4000, 256, 4096, False), (1000, 512, 16384, True), (1030, 31, 16450, False), (8200, 300, 4100, True), (2500, 512, 33, False)]


@pytest.mark.parametrize("M,K,O,gated", FULL)
def test_gemm_of_full_size(M, K, O, gated):
    g = torch.Generator(device=DEV).manual_seed(M + K + O)
    codes, scales = binding.mx4_quant(torch.randn((M, K), generator=g, device=DEV))
    wc, ws_ = binding.mx4_quant(0.02 * torch.randn((O << gated, K), generator=g, device=DEV))
    w = binding.mx4_pack(wc, ws_, K, gated=gated)
    rng = np.random.default_rng(M)
    rows = torch.from_numpy(np.unique(np.concatenate([rng.integers(0, M, 40), [0, M - 1]]))).to(DEV)
    cols = torch.from_numpy(np.unique(np.concatenate([rng.integers(0, O, 60), [0, O - 1]]))).to(DEV)
    ref, off = _sampled(rows, cols, codes, scales, wc, ws_, gated)
    n = binding.mx4_gemm_workspace_bytes(M, O, K, gated=gated)
    for ws in [None] + ([torch.full((n,), 0x5A, dtype=torch.uint8, device=DEV)] if n else []):
        Y = binding.mx4_gemm(codes, scales, *w, O, K, gated=gated, workspace=ws)
        check_product(Y[rows][:, cols], ref, off)
        if ws is not None:
            assert bool((ws != 0x5A).any())
    assert not bool(Y.isnan().any())


def test_long_rows_ask_for_a_workspace():
    assert binding.mx4_gemm_workspace_bytes(256, 3584, 18944) > 0 and binding.mx4_gemm_workspace_bytes(8192, 37888, 3584) == 0
    assert binding.mx4_gemm_workspace_bytes(0, 64, 64) == binding.mx4_gemm_workspace_bytes(4, 64, 64, experts=1025) == 0


GROUPED_FULL = [(8192, 8, 4096, 2048, False), (3000, 5, 2304, 1500, True), (2000, 64, 2048, 1408, False), (500, 8, 4096, 4096, False), (32, 8, 4096, 1024, True), (1200, 4, 8192, 512, False),
                (256, 1, 18944, 512, False), (8000, 16, 512, 2048, False), (16000, 5, 256, 1030, True), (3000, 128, 200, 400, False)]


@pytest.mark.parametrize("R,E,K,O,gated", GROUPED_FULL)
def test_grouped_of_full_size(R, E, K, O, gated):
    g = torch.Generator(device=DEV).manual_seed(R + E)
    off = groups("skewed", R, E, np.random.default_rng(R))
    codes, scales = binding.mx4_quant(torch.randn((R, K), generator=g, device=DEV))
    rows_e = O << gated
    wc, ws_ = binding.mx4_quant(0.02 * torch.randn((E * rows_e, K), generator=g, device=DEV))
    w = binding.mx4_pack(wc, ws_, K, experts=E, gated=gated)
    n = binding.mx4_gemm_workspace_bytes(R, O, K, experts=E, gated=gated)
    offsets = torch.from_numpy(off.astype(np.int32)).to(DEV)
    rng = np.random.default_rng(E)
    cols = torch.from_numpy(np.unique(np.concatenate([rng.integers(0, O, 40), [0, O - 1]]))).to(DEV)
    for ws in [None] + ([torch.full((n,), 0x5A, dtype=torch.uint8, device=DEV)] if n else []):
        Y = binding.mx4_grouped_gemm(codes, scales, offsets, *w, O, K, gated=gated, workspace=ws)
        for e in range(E):
            if off[e + 1] > off[e]:
                rows = torch.from_numpy(np.unique(np.concatenate([rng.integers(off[e], off[e + 1], 8), [off[e], off[e + 1] - 1]]))).to(DEV)
                part = slice(e * rows_e, (e + 1) * rows_e)
                ref, tol = _sampled(rows, cols, codes, scales, wc[part], ws_[:, part], gated)
                check_product(Y[rows][:, cols], ref, tol)
        assert not bool(Y[off[-1]:].any())


def test_replayed_graph():
    """Captured calls, replayed several times with eager work between: the results of eager calls each time."""
    K, O, E = 1024, 256, 4
    X = torch.randn((300, K), device=DEV).to(torch.bfloat16)
    logits = torch.randn((300, E), device=DEV)
    w = binding.mx4_pack(*binding.mx4_quant(torch.randn((E * 2 * O, K), device=DEV)), K, experts=E, gated=True)
    ws = torch.empty((max(16, binding.mx4_gemm_workspace_bytes(600, O, K, experts=E, gated=True)),), dtype=torch.uint8, device=DEV)

    def step():
        ids, weights, slots, rows, offsets = binding.expert_route(logits, 2)
        codes, scales = binding.mx4_quant(X, rows=rows)
        return binding.expert_combine(binding.mx4_grouped_gemm(codes, scales, offsets, *w, O, K, gated=True, workspace=ws), slots, weights)

    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step()
    for i in range(4):
        X.copy_(torch.randn((300, K), device=DEV))
        logits.copy_(torch.randn((300, E), device=DEV))
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, step())


def test_another_stream():
    X, W = torch.randn((40, 512), device=DEV), torch.randn((64, 512), device=DEV)
    want = binding.mx4_gemm(*binding.mx4_quant(X), *binding.mx4_pack(*binding.mx4_quant(W), 512), 64, 512)
    torch.cuda.synchronize()
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        got = binding.mx4_gemm(*binding.mx4_quant(X), *binding.mx4_pack(*binding.mx4_quant(W), 512), 64, 512)
    stream.synchronize()
    assert torch.equal(got, want)


def test_more_tiles_than_a_grid_is_high():
    M, K, O = 1100000, 64, 16
    g = torch.Generator(device=DEV).manual_seed(1)
    codes, scales = binding.mx4_quant(torch.randn((M, K), generator=g, device=DEV))
    wc, ws_ = binding.mx4_quant(torch.randn((O, K), generator=g, device=DEV))
    Y = binding.mx4_gemm(codes, scales, *binding.mx4_pack(wc, ws_, K), O, K)
    rows = torch.cat([torch.arange(0, M, 9999), torch.tensor([M - 1, 65535 * 16, 65535 * 16 + 1, 65535 * 16 - 1])]).to(DEV)
    ref, off = _sampled(rows, torch.arange(O, device=DEV), codes, scales, wc, ws_, False)
    check_product(Y[rows], ref, off)
