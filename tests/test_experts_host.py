"""The layer of 4-bit experts on the host: what it hands to the operators (which are replaced here; no GPU)."""
import types

import pytest
import torch

from paper_2603_05232_amd import experts


@pytest.mark.parametrize("grouped", [False, True])
def test_every_call_has_a_workspace_of_its_own(monkeypatch, grouped):
    """Calls that are under way at once, on streams, in threads or in a captured graph, share no memory: whoever holds one call's workspace finds no other call in it."""
    given = []

    def product(*args, workspace=None, **kwargs):
        given.append(workspace)

    monkeypatch.setattr(experts, "binding", types.SimpleNamespace(mx4_gemm_workspace_bytes=lambda R, O, K, experts, gated: 1024 * (R - 1), mx4_gemm=product, mx4_grouped_gemm=product))
    layer = experts.Packed.__new__(experts.Packed)
    layer.O, layer.K, layer.experts, layer.gated, layer.w_vals, layer.w_meta, layer.scratch = 64, 256, 1, False, None, None, None
    for rows in (3, 3, 9, 2, 1):
        codes = torch.empty((rows, 128), dtype=torch.uint8)
        layer(codes, None, torch.tensor([0, rows]) if grouped else None)
    assert given[4] is None and all(ws.dtype == torch.uint8 and ws.numel() >= 1024 * (rows - 1) for ws, rows in zip(given, (3, 3, 9, 2)))
    spans = [(ws.data_ptr(), ws.data_ptr() + ws.numel()) for ws in given[:4]]
    assert all(a[1] <= b[0] or b[1] <= a[0] for i, a in enumerate(spans) for b in spans[:i])
    assert not any(ws is v for ws in given[:4] for v in vars(layer).values())
