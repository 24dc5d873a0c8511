"""A layer of 4-bit experts, step by step: every step of the chained run against the oracle on the inputs that it received."""
import numpy as np
import pytest
import torch

from oracle import mx4_oracle as mo
from paper_2603_05232_amd.experts import ExpertLayer
from test_gpu_mx4 import _sampled, as_codes, check_product

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.mark.parametrize("M,hidden,inner,experts,top,shared", [(1, 512, 96, 8, 2, True), (50, 600, 200, 16, 4, True), (300, 1024, 352, 5, 2, False)])
def test_every_step(M, hidden, inner, experts, top, shared):
    layer = ExpertLayer(DEV, hidden, inner, experts, top, shared, seed=M)
    x = torch.randn((M, hidden), generator=torch.Generator(device=DEV).manual_seed(M), device=DEV).to(torch.bfloat16)
    r = {}
    out = layer.forward(x, record=r)
    assert out.shape == x.shape and out.dtype == torch.bfloat16
    ids, weights, slots, rows, offsets = mo.route(r["logits"].double().cpu().numpy(), top)
    assert np.array_equal(r["slots"].cpu().numpy(), slots) and np.array_equal(r["rows"].cpu().numpy(), rows) and np.array_equal(r["offsets"].cpu().numpy(), offsets)
    assert np.allclose(r["weights"].cpu().numpy(), weights, rtol=2.0 ** -18, atol=0)
    for src, codes, scales in ((x[r["rows"].long()], r["codes"], r["scales"]), (r["h"], r["h_codes"], r["h_scales"])):
        want_codes, want_scales = as_codes(*mo.quant(src.double().cpu().numpy()))
        assert torch.equal(codes, want_codes) and torch.equal(scales, want_scales)
    for packed, codes, scales, got in ((layer.gate_up, r["codes"], r["scales"], r["h"]), (layer.down, r["h_codes"], r["h_scales"], r["y"])):
        per = packed.codes.shape[0] // experts
        cols = torch.arange(packed.O, device=DEV)
        for e in range(experts):
            if offsets[e + 1] > offsets[e]:
                at = torch.arange(offsets[e], offsets[e + 1], device=DEV)
                ref, off = _sampled(at, cols, codes, scales, packed.codes[e * per:(e + 1) * per], packed.scales[:, e * per:(e + 1) * per], packed.gated)
                check_product(got[at], ref, off)
    ref, off = mo.combine(r["y"].double().cpu().numpy(), slots, r["weights"].double().cpu().numpy(), r["base"].double().cpu().numpy() if shared else None)
    assert (np.abs(out.double().cpu().numpy() - ref) <= 2.0 ** -8 * np.abs(ref) + off).all()
