"""The choice of experts and the weighted sum against the oracle (64 bits).  Choices and order are equal; weights may be off by the 32-bit exponential's
argument and the sums: 2^-23 (|largest difference of scores| + summands + 8) of the weight."""
import types

import numpy as np
import pytest
import torch

from oracle import mx4_oracle as mo
from paper_2603_05232_amd import binding

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def check_route(x, k, renormalise=True):
    got = [t.cpu().numpy() for t in binding.expert_route(x, k, renormalise)]
    xs = x.double().cpu().numpy()
    want = mo.route(xs, k, renormalise)
    for i, name in ((0, "ids"), (2, "slots"), (3, "rows"), (4, "offsets")):
        assert np.array_equal(got[i], want[i]), name
    finite = np.where(np.isfinite(xs), xs, 0)
    off = 2.0 ** -23 * (np.ptp(finite, axis=1, keepdims=True) + (k if renormalise else x.shape[1]) + 8) * want[1]
    assert np.array_equal(np.isnan(got[1]), np.isnan(want[1]))
    assert (np.abs(got[1] - want[1])[~np.isnan(want[1])] <= (off + 1e-37)[~np.isnan(want[1])]).all()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("M,E,k", [(1, 1, 1), (1, 64, 8), (4, 8, 2), (63, 65, 1), (64, 128, 64), (65, 3, 3), (200, 100, 6), (129, 256, 8), (70, 257, 4), (90, 1000, 9),
                                   (1100, 16, 4), (17000, 5, 2)])
def test_route(M, E, k, dtype):
    g = torch.Generator().manual_seed(M + E + k)
    x = (3 * torch.randn((M, E), generator=g)).to(dtype)
    check_route(x.to(DEV), k)
    check_route(x.to(DEV), k, renormalise=False)


def test_route_of_equal_masked_and_missing_scores():
    x = torch.zeros((130, 70))
    x[0, ::2] = -0.0                                            # equal to 0: the lower index
    x[1, :] = float("-inf")                                     # no expert has a weight
    x[2, :69] = float("-inf")
    x[3, :] = torch.finfo(torch.float32).min
    x[4, :68] = float("nan")                                    # below every number
    x[5, 7] = float("nan")
    x[6, :] = 1e-40 * torch.arange(70)
    x[100, 60:] = 5.0
    check_route(x.to(DEV), 2)
    check_route(x.to(DEV).to(torch.bfloat16), 3, renormalise=False)
    check_route(x[:40].to(DEV), 5)


def test_route_of_rows_with_a_stride():
    x = torch.randn((80, 50), device=DEV)[:, 7:40]
    check_route(x, 4)
    check_route(x.to(torch.bfloat16)[:1], 4)


def test_route_without_tokens():
    ids, weights, slots, rows, offsets = binding.expert_route(torch.zeros((0, 9), device=DEV), 2)
    assert ids.shape == weights.shape == slots.shape == (0, 2) and rows.shape == (0,) and offsets.cpu().tolist() == [0] * 10


@pytest.mark.parametrize("base", [False, True])
@pytest.mark.parametrize("M,k,O", [(1, 1, 1), (3, 2, 8), (7, 2, 4096), (5, 3, 1001), (100, 8, 264), (33, 64, 7)])
def test_combine(M, k, O, base):
    rng = np.random.default_rng(M + k + O)
    R = M * k
    Y = torch.from_numpy(rng.standard_normal((R, O + 3))).to(DEV).to(torch.bfloat16)[:, 1:O + 1]
    slots = rng.permutation(R).reshape(M, k).astype(np.int32)
    slots[0, 0] = (-1, R, 2 ** 31 - 1, 0)[M % 4]                # most of these add nothing
    weights = rng.random((M, k)).astype(np.float32)
    add = torch.from_numpy(rng.standard_normal((M, O + 1))).to(DEV).to(torch.bfloat16)[:, 1:] if base else None
    ref, off = mo.combine(Y.double().cpu().numpy(), slots, weights.astype(np.float64), add.double().cpu().numpy() if base else None)
    whole = torch.full((M + 1, O + 2), 7.0, dtype=torch.bfloat16, device=DEV)
    got = binding.expert_combine(Y, torch.from_numpy(slots).to(DEV), torch.from_numpy(weights).to(DEV), base=add, out=whole[:M, 1:O + 1])
    bad = ~(np.abs(got.double().cpu().numpy() - ref) <= 2.0 ** -8 * np.abs(ref) + off)
    assert not bad.any(), int(bad.sum())
    assert bool((whole[M] == 7).all()) and bool((whole[:, 0] == 7).all()) and bool((whole[:, O + 1] == 7).all())


def test_combine_refuses():
    Y, s, w = torch.zeros((4, 8), dtype=torch.bfloat16, device=DEV), torch.zeros((2, 2), dtype=torch.int32, device=DEV), torch.ones((2, 2), device=DEV)
    with pytest.raises(AssertionError):
        binding.expert_combine(Y, s, w.double())
    with pytest.raises(TypeError):
        binding.expert_combine(Y, s.long(), w)
    with pytest.raises(AssertionError):
        binding.expert_combine(Y, s, w, base=Y)
    with pytest.raises(binding.SlideSparseError):
        binding.expert_route(torch.zeros((2, 3), device=DEV), 4)


def test_calls_through_the_module_and_without_it(monkeypatch):
    """The extension module takes plain calls, the general path gives the same."""
    binding.load()
    X = torch.randn((70, 600), device=DEV).to(torch.bfloat16)
    w = binding.mx4_pack(*binding.mx4_quant(torch.randn((4 * 96, 600), device=DEV)), 600, experts=4)
    w1 = binding.mx4_pack(*binding.mx4_quant(torch.randn((96, 600), device=DEV)), 600)
    logits = torch.randn((70, 4), device=DEV)

    def calls():
        ids, weights, slots, rows, offsets = binding.expert_route(logits, 2)
        codes, scales = binding.mx4_quant(X, rows=rows)
        Y = binding.mx4_grouped_gemm(codes, scales, offsets, *w, 96, 600)
        Z = binding.mx4_gemm(codes, scales, *w1, 96, 600, out=torch.zeros((140, 100), dtype=torch.bfloat16, device=DEV)[:, :96])
        return [ids, weights, slots, rows, offsets, codes, scales, Y, Z, binding.mx4_dequant(codes, scales, 600), binding.mx4_dequant(codes, scales, 600, torch.bfloat16),
                binding.expert_combine(Y, slots, weights), binding.expert_combine(Y, slots, weights, base=Z[:70])]

    taken = []
    names = ("mx4_quant", "mx4_dequant", "mx4_product", "expert_route", "expert_combine")
    real = binding._mx4_calls

    def spy(name):
        def call(*args):
            r = getattr(real, name)(*args)
            taken.append(r is not None)
            return r
        return call

    monkeypatch.setattr(binding, "_mx4_calls", types.SimpleNamespace(**{n: spy(n) for n in names}))
    a = calls()
    assert taken and all(taken)
    monkeypatch.setattr(binding, "_mx4_calls", types.SimpleNamespace(**dict.fromkeys(names, lambda *args: None)))
    for x, y in zip(a, calls()):
        assert x.shape == y.shape and x.dtype == y.dtype and x.device == y.device and torch.equal(x, y)
