"""What a layer of 4-bit experts holds on the GPU: its packed weights and its router, from which the codes can be read back."""
import pytest
import torch

from paper_2603_05232_amd import binding
from paper_2603_05232_amd.experts import ExpertLayer, Packed

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def test_no_more_than_the_packed_weights():
    hidden, inner, experts = 2048, 1408, 8
    binding.load()
    torch.cuda.synchronize()
    # what was asked for: what is allocated also counts the unused ends of blocks that the allocator has cached
    requested = lambda: torch.cuda.memory_stats()["requested_bytes.all.current"]  # noqa: E731
    before = requested()
    layer = ExpertLayer(DEV, hidden, inner, experts, top=2, shared=True)
    held = requested() - before
    parts = [n for K, O, E, gated in ((hidden, inner, experts, True), (inner, hidden, experts, False), (hidden, inner, 1, True), (inner, hidden, 1, False))
             for n in binding.mx4_packed_sizes(O, K, E, gated)] + [4 * experts * hidden]
    assert held <= sum(parts)
    assert layer.router.shape == (experts, hidden)


@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("O,K,experts", [(32, 256, 1), (40, 300, 3), (1, 1, 2), (97, 1000, 1), (64, 513, 5)])
def test_codes_read_back(O, K, experts, gated):
    W = torch.randn((experts * (O << gated), K), generator=torch.Generator(device=DEV).manual_seed(O + K), device=DEV)
    packed = Packed(W, experts, gated)
    codes, scales = binding.mx4_quant(W)
    assert torch.equal(packed.codes, codes) and torch.equal(packed.scales, scales)
    assert packed.codes.is_contiguous() and packed.scales.is_contiguous()
