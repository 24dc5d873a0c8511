"""Captured calls on a cache whose lengths change between the replays so far that requests are divided otherwise."""
import numpy as np
import pytest
import torch

from paper_2603_05232_amd import binding
from test_gpu_kv import DEV, Cache, i32, queries
from test_gpu_kv_decode import block, fill, hidden, steps  # noqa: F401

pytestmark = pytest.mark.gpu


def plan(workspace, B):
    """(first item, parts) of each request, which the attention leaves at the head of its workspace."""
    return workspace[:8 * B].view(torch.int32).view(B, 2).tolist()


def parts(lens, groups):
    """Into how many parts requests are divided: blocks of 32 tokens over workgroups, whole rounds of four wavefronts while these are few."""
    blocks = [-(-n // 32) for n in lens]
    n = sum(blocks) / groups
    per = 4 * max(1, int(n / 4 + 0.999)) if n < 32 else int(n) + 1
    return [max(1, -(-b // per)) for b in blocks]


@pytest.mark.parametrize("dtype", ["bf16", "fp8"])
def test_a_captured_attention_follows_its_lengths(dtype):
    """From requests of one part each to many and back, as lengths are written between replays."""
    lens, B, H, D = [9000, 400, 129, 2100, 0], 5, 2, 64
    cache = Cache(np.random.default_rng(31), [9000, 400, 129, 2100, 1], H, D, 64, dtype)
    q = queries(B, 8, D, "bf16")
    table, now = i32(cache.table), i32(lens)
    n = binding.kv_attention_workspace_bytes(B, 8, H, D)
    ws, out = torch.zeros((n,), dtype=torch.uint8, device=DEV), torch.zeros((B, 8, D), dtype=torch.bfloat16, device=DEV)
    groups = 2 * torch.cuda.get_device_properties(0).multi_processor_count // H

    def call(lens, out, ws):
        return binding.kv_attention(q, cache.pages, table, lens, H, 64, dtype, out=out, workspace=ws)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        call(now, out, ws)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call(now, out, ws)
    seen = []
    for lens in ([9000, 400, 129, 2100, 0], [1, 1, 0, 0, 1], [100, 128, 129, 127, 1], [9000, 0, 0, 0, 0], [128, 400, 33, 2100, 1], [129, 400, 128, 2048, 0], [8999, 399, 129, 2099, 1]):
        now.copy_(i32(lens))
        out.fill_(7.0)
        graph.replay()
        given, want = out.clone(), torch.zeros_like(out)
        call(i32(lens), want, torch.full((n,), 0x55, dtype=torch.uint8, device=DEV))      # the same on its own
        torch.cuda.synchronize()
        assert torch.equal(given, want), lens
        kept, cache.lens = cache.lens, lens
        cache.check(given, q)
        cache.lens = kept
        assert [p for _, p in plan(ws, B)] == parts(lens, groups), lens
        seen.append(tuple(p for _, p in plan(ws, B)))
    assert len(set(seen)) >= 6 and max(max(p) for p in seen) > 20 and (1,) * B in seen


def test_captured_steps_that_pass_into_another_part(block):  # noqa: F811
    """Decoding steps in which one request grows from one part to two and another by a part, replayed from one capture."""
    lens = [126, 3, 766]
    groups = 2 * torch.cuda.get_device_properties(0).multi_processor_count // 8
    divisions = [parts([n + i for n in lens], groups) for i in range(1, 7)]
    assert len({tuple(d) for d in divisions}) > 1 and divisions[0][0] == 1 and divisions[-1][0] == 2 and divisions[-1][2] == divisions[0][2] + 1
    x = hidden(3, 17)
    want = steps(block, fill(block, lens, width=14), x, 6)
    cache, other = fill(block, lens, width=14), fill(block, [700, 65, 300])
    state = [t.clone() for t in (cache.lens, cache.table, cache.pool, cache.left)]
    inp = x.clone()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        block.decode(inp, cache, cache.step())
    torch.cuda.current_stream().wait_stream(side)
    for t, s in zip((cache.lens, cache.table, cache.pool, cache.left), state):
        t.copy_(s)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = block.decode(inp, cache, cache.step())
    for i, y in enumerate(want):
        inp.copy_(x + i / 8)
        graph.replay()
        assert torch.equal(out, y), i
        steps(block, other, x, 1)
        torch.cuda.synchronize()
    assert cache.lens.tolist() == [n + 6 for n in lens]
