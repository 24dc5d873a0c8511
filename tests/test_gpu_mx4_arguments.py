"""Tensors in host memory among operands on the GPU: every operator refuses them before it launches anything."""
import pytest
import torch

from paper_2603_05232_amd import binding

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.fixture(scope="module")
def t():
    K, O, E = 300, 40, 3
    X = torch.randn((70, K), device=DEV).to(torch.bfloat16)
    ids, weights, slots, rows, offsets = binding.expert_route(torch.randn((70, E), device=DEV), 2)
    codes, scales = binding.mx4_quant(X, rows=rows)
    wc, ws = binding.mx4_quant(torch.randn((E * O, K), device=DEV))
    return dict(K=K, O=O, E=E, X=X, rows=rows, offsets=offsets, slots=slots, weights=weights, codes=codes, scales=scales, wc=wc, ws=ws, w=binding.mx4_pack(wc, ws, K, experts=E),
                w1=binding.mx4_pack(wc[:O].contiguous(), ws[:, :O].contiguous(), K), Y=torch.zeros((140, O), dtype=torch.bfloat16, device=DEV), logits=torch.zeros((70, E), device=DEV),
                scratch=torch.zeros((4096,), dtype=torch.uint8, device=DEV))


CALLS = {
    "quant X": lambda t: binding.mx4_quant(t["X"].cpu()),
    "quant rows": lambda t: binding.mx4_quant(t["X"], rows=t["rows"].cpu()),
    "quant codes": lambda t: binding.mx4_quant(t["X"], rows=t["rows"], codes=t["codes"].cpu(), scales=t["scales"]),
    "quant scales": lambda t: binding.mx4_quant(t["X"], rows=t["rows"], codes=t["codes"], scales=t["scales"].cpu()),
    "dequant scales": lambda t: binding.mx4_dequant(t["codes"], t["scales"].cpu(), t["K"]),
    "dequant out": lambda t: binding.mx4_dequant(t["codes"], t["scales"], t["K"], out=torch.zeros((140, t["K"]))),
    "pack scales": lambda t: binding.mx4_pack(t["wc"], t["ws"].cpu(), t["K"], experts=t["E"]),
    "gemm scales": lambda t: binding.mx4_gemm(t["codes"], t["scales"].cpu(), *t["w1"], t["O"], t["K"]),
    "gemm w_vals": lambda t: binding.mx4_gemm(t["codes"], t["scales"], t["w1"][0].cpu(), t["w1"][1], t["O"], t["K"]),
    "gemm w_meta": lambda t: binding.mx4_gemm(t["codes"], t["scales"], t["w1"][0], t["w1"][1].cpu(), t["O"], t["K"]),
    "gemm out": lambda t: binding.mx4_gemm(t["codes"], t["scales"], *t["w1"], t["O"], t["K"], out=t["Y"].cpu()),
    "gemm workspace": lambda t: binding.mx4_gemm(t["codes"], t["scales"], *t["w1"], t["O"], t["K"], workspace=t["scratch"].cpu()),
    "grouped offsets": lambda t: binding.mx4_grouped_gemm(t["codes"], t["scales"], t["offsets"].cpu(), *t["w"], t["O"], t["K"]),
    "grouped w_vals": lambda t: binding.mx4_grouped_gemm(t["codes"], t["scales"], t["offsets"], t["w"][0].cpu(), t["w"][1], t["O"], t["K"]),
    "grouped workspace": lambda t: binding.mx4_grouped_gemm(t["codes"], t["scales"], t["offsets"], *t["w"], t["O"], t["K"], workspace=t["scratch"].cpu()),
    "route logits": lambda t: binding.expert_route(t["logits"].cpu(), 2),
    "route workspace": lambda t: binding.expert_route(t["logits"], 2, workspace=t["scratch"].cpu()),
    "combine slots": lambda t: binding.expert_combine(t["Y"], t["slots"].cpu(), t["weights"]),
    "combine weights": lambda t: binding.expert_combine(t["Y"], t["slots"], t["weights"].cpu()),
    "combine base": lambda t: binding.expert_combine(t["Y"], t["slots"], t["weights"], base=t["Y"][:70].cpu()),
    "combine out": lambda t: binding.expert_combine(t["Y"], t["slots"], t["weights"], out=t["Y"][:70].cpu()),
}


@pytest.mark.parametrize("name", CALLS)
def test_host_memory_is_refused(t, name):
    with pytest.raises(AssertionError):
        CALLS[name](t)
