"""A layer of experts on 4-bit weights and activations: the feed-forward part of a transformer block whose tokens go to k of E gated MLPs each, with
one more that every token goes to, all products on microscaled 4-bit operands.

    logits = x . Wr^T                        plain torch (E columns)
    expert_route                             which experts, with what weight, in what order of rows
    mx4_quant(x, rows)                       codes of every token, once for each of its experts
    mx4_grouped_gemm(gated)                  silu(x Wg^T) * (x Wu^T), each row with its expert's weights
    mx4_quant, mx4_grouped_gemm              the way back
    mx4_quant, mx4_gemm (gated), mx4_gemm    the shared expert
    expert_combine                           the weighted sum of a token's experts and the shared one

Weights are random-init, quantised and packed by the library.  `python -m paper_2603_05232_amd.experts` runs and times a layer."""
from __future__ import annotations

import torch

from . import binding

HIDDEN, INNER, EXPERTS, TOP = 4096, 1408, 64, 4


class Packed:
    """Weights of `experts` matrices [out, in] (gated: [2 out, in]) as the products take them."""

    def __init__(self, W: torch.Tensor, experts: int = 1, gated: bool = False):
        self.O, self.K, self.experts, self.gated = W.shape[0] // experts // (2 if gated else 1), W.shape[1], experts, gated
        self.w_vals, self.w_meta = binding.mx4_pack(*binding.mx4_quant(W), self.K, experts=experts, gated=gated)

    def _rows(self, packed: torch.Tensor, order) -> torch.Tensor:
        """What was packed, [rows, units, bytes], from the operand order of csrc/mx4_common.h: its dimensions in `order` are those of a fragment's rows, the unit, the bytes."""
        t = packed.permute(order).reshape(self.experts, packed.shape[1] * 32, packed.shape[2], -1)
        if not self.gated:
            return t[:, :self.O].flatten(0, 1)
        return t[:, :2 * self.O].unflatten(1, (self.O, 2)).transpose(1, 2).flatten(0, 2)

    # The codes and scales of the weights, read back from the packed ones: a layer does not need them, and kept beside those they would double its memory.
    @property
    def codes(self) -> torch.Tensor:
        """[rows, 128 units], as mx4_quant wrote them."""
        units = binding.mx4_row_bytes(self.K) // 128
        return self._rows(self.w_vals.view(self.experts, -1, units, 2, 2, 4, 4, 4, 16), (0, 1, 6, 4, 7, 2, 5, 3, 8)).flatten(1).contiguous()

    @property
    def scales(self) -> torch.Tensor:
        """[units, rows, 8], as mx4_quant wrote them."""
        units = binding.mx4_row_bytes(self.K) // 128
        return self._rows(self.w_meta.view(self.experts, -1, units, 4, 4, 4, 2, 2), (0, 1, 4, 6, 5, 2, 3, 7)).transpose(0, 1).contiguous()

    def __call__(self, codes, scales, offsets=None):
        # A workspace for each call, so that the allocator keeps it to this call's stream, or to the graph that is being captured: one that calls share would be
        # written by two streams at once, and a graph would go on writing to one that has been replaced since.
        n = binding.mx4_gemm_workspace_bytes(codes.shape[0], self.O, self.K, experts=self.experts, gated=self.gated)
        ws = torch.empty((n,), dtype=torch.uint8, device=codes.device) if n else None
        if offsets is None:
            return binding.mx4_gemm(codes, scales, self.w_vals, self.w_meta, self.O, self.K, gated=self.gated, workspace=ws)
        return binding.mx4_grouped_gemm(codes, scales, offsets, self.w_vals, self.w_meta, self.O, self.K, gated=self.gated, workspace=ws)


class ExpertLayer:
    def __init__(self, dev, hidden: int = HIDDEN, inner: int = INNER, experts: int = EXPERTS, top: int = TOP, shared: bool = True, seed: int = 0):
        g = torch.Generator(device=dev).manual_seed(seed)

        def weights(rows, K):
            return 0.02 * torch.randn((rows, K), generator=g, device=dev)

        self.top = top
        self.router = weights(experts, hidden)
        self.gate_up, self.down = Packed(weights(experts * 2 * inner, hidden), experts, gated=True), Packed(weights(experts * hidden, inner), experts)
        self.shared = (Packed(weights(2 * inner, hidden), gated=True), Packed(weights(hidden, inner))) if shared else None

    def forward(self, x: torch.Tensor, record=None):
        """x[M, hidden] bf16 -> [M, hidden] bf16.  record: dict that receives what the steps in between gave."""
        logits = x.float() @ self.router.t()
        ids, weights, slots, rows, offsets = binding.expert_route(logits, self.top)
        codes, scales = binding.mx4_quant(x, rows=rows)
        h = self.gate_up(codes, scales, offsets)
        h_codes, h_scales = binding.mx4_quant(h)
        y = self.down(h_codes, h_scales, offsets)
        base = None
        if self.shared is not None:
            base = self.shared[1](*binding.mx4_quant(self.shared[0](*binding.mx4_quant(x))))
        out = binding.expert_combine(y, slots, weights, base=base)
        if record is not None:
            record.update(logits=logits, weights=weights, slots=slots, rows=rows, offsets=offsets, codes=codes, scales=scales, h=h, h_codes=h_codes, h_scales=h_scales, y=y, base=base)
        return out


def main():
    import argparse
    ap = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    for name, value in (("tokens", 4096), ("hidden", HIDDEN), ("inner", INNER), ("experts", EXPERTS), ("top", TOP), ("steps", 20)):
        ap.add_argument("--" + name, type=int, default=value)
    a = ap.parse_args()
    dev = torch.device("cuda")
    layer = ExpertLayer(dev, a.hidden, a.inner, a.experts, a.top)
    x = torch.randn((a.tokens, a.hidden), device=dev).to(torch.bfloat16)
    for _ in range(3):
        layer.forward(x)
    begin, end = (torch.cuda.Event(enable_timing=True) for _ in range(2))
    begin.record()
    for _ in range(a.steps):
        layer.forward(x)
    end.record()
    torch.cuda.synchronize()
    ms = begin.elapsed_time(end) / a.steps
    flops = 2 * a.tokens * (a.top + 1) * 3 * a.hidden * a.inner
    print(f"{a.tokens} tokens, {a.top} of {a.experts} experts {a.hidden} -> {a.inner} -> {a.hidden} and a shared one: {ms:.3f} ms, {flops / ms / 1e9:.0f} TFLOP/s")


if __name__ == "__main__":
    main()
