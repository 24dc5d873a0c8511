"""A paged cache of keys and values for decoding: the state that the operators kv_tables, kv_write, kv_read and kv_attention work on, all of it on the device.

    step / resize      kv_tables: requests get longer, shorter or empty; pages and the slots of the new tokens
    write              kv_write: keys and values into those slots
    attend             kv_attention: one new token of each request over its cached ones
    read               kv_read: what the pages hold

No call waits for the GPU or reads from it, so that a decoding step can be captured into a graph: lengths, tables and free pages live in the same tensors throughout.
`python -m paper_2603_05232_amd.kv_cache` runs and times the decoding of a block (block.py)."""
from __future__ import annotations

import torch

from . import binding


class PagedCache:
    def __init__(self, dev, requests: int, pages: int, width: int, heads: int, head_dim: int, page: int = 64, dtype: str = "bf16"):
        """Room for `pages` pages of `page` tokens; at most `width` of them for each of `requests` requests, all empty."""
        n = binding.kv_page_bytes(heads, page, head_dim, dtype)
        if n < 0:
            raise binding.SlideSparseError(3, "kv_page_bytes")
        self.page, self.heads, self.head_dim, self.dtype = page, heads, head_dim, dtype
        self.pages = torch.empty((pages, n), dtype=torch.uint8, device=dev)
        self.lens = torch.zeros((requests,), dtype=torch.int32, device=dev)
        self.table = torch.zeros((requests, width), dtype=torch.int32, device=dev)
        self.pool = torch.arange(pages - 1, -1, -1, dtype=torch.int32, device=dev)      # page 0 on top
        self.left = torch.full((1,), pages, dtype=torch.int32, device=dev)

    def resize(self, want: torch.Tensor, rows: int):
        """Requests to want[requests] (int32) tokens -> (slots[rows], offsets[requests + 1]): the new tokens' slots, request by request; -1 behind the last and for
        requests that found no room, whose lengths stay."""
        _, _, slots, offsets = binding.kv_tables(self.lens, want, self.table, self.pool, self.left, self.page, rows, new_lens=self.lens, new_left=self.left)
        return slots, offsets

    def step(self, active=None) -> torch.Tensor:
        """One token more for every request, or for those of active[requests] (bool) -> slots[requests], -1 for the others."""
        B = self.lens.shape[0]
        if active is None:
            return self.resize(self.lens + 1, B)[0]
        slots, offsets = self.resize(self.lens + active.int(), B)
        return torch.where(active, slots[offsets[:-1].long().clamp(max=B - 1)], -1)

    def write(self, k: torch.Tensor, v: torch.Tensor, slots: torch.Tensor) -> None:
        """k, v [rows, heads, head_dim]."""
        binding.kv_write(k, v, slots, self.pages, self.page, self.dtype)

    def read(self, slots: torch.Tensor, dtype: torch.dtype = torch.bfloat16):
        return binding.kv_read(self.pages, slots, self.heads, self.head_dim, self.page, self.dtype, dtype)

    def attend(self, q: torch.Tensor, window: int = 0, scale=None) -> torch.Tensor:
        """q[requests, query heads, head_dim] -> the same in bf16; a request without tokens gives zeros."""
        # A workspace for each call, as experts.Packed has it: calls on several streams or in captured graphs share none.
        n = binding.kv_attention_workspace_bytes(q.shape[0], q.shape[1], self.heads, self.head_dim)
        ws = torch.empty((n,), dtype=torch.uint8, device=q.device) if n else None
        return binding.kv_attention(q, self.pages, self.table, self.lens, self.heads, self.page, self.dtype, scale=scale, window=window, workspace=ws)


def main():
    import argparse

    from . import block
    ap = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    for name, value in (("requests", 64), ("context", 4096), ("page", 64), ("steps", 50)):
        ap.add_argument("--" + name, type=int, default=value)
    ap.add_argument("--dtype", default="bf16", choices=sorted(binding.DTYPE_CODE))
    a = ap.parse_args()
    dev = torch.device("cuda")
    llama = block.LlamaBlock(dev)
    width = -(-(a.context + a.steps + 8) // a.page)
    cache = PagedCache(dev, a.requests, a.requests * width, width, block.N_KV_HEADS, block.HEAD_DIM, a.page, a.dtype)
    # contexts as they may have come in, request by request
    one = torch.arange(a.requests, device=dev)
    for b in range(a.requests):
        slots, _ = cache.resize(torch.where(one == b, a.context, cache.lens).int(), a.context)
        k, v = (torch.randn((a.context, block.N_KV_HEADS, block.HEAD_DIM), device=dev).to(torch.bfloat16) for _ in "kv")
        cache.write(k, v, slots)
    x = torch.randn((a.requests, block.HIDDEN), device=dev).to(torch.bfloat16)

    def step():
        return llama.decode(x, cache, cache.step())

    for _ in range(3):
        step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    begin, end = (torch.cuda.Event(enable_timing=True) for _ in range(2))
    begin.record()
    for _ in range(a.steps):
        graph.replay()
    end.record()
    torch.cuda.synchronize()
    ms = begin.elapsed_time(end) / a.steps
    print(f"{a.requests} requests of {a.context} tokens, {a.dtype} cache: {ms:.3f} ms a step of one block, {a.requests / ms * 1000:.0f} tokens/s")


if __name__ == "__main__":
    main()
