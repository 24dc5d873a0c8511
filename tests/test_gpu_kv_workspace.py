"""kv_attention in a workspace of just the size that it asks for."""
import numpy as np
import pytest
import torch

from paper_2603_05232_amd import binding
from test_gpu_kv import DEV, Cache, i32, queries
from test_gpu_kv_replay import parts, plan

pytestmark = pytest.mark.gpu


def attend(cache, q, n):
    """Through n bytes among others that stay as they are -> (result, the workspace)."""
    ws = torch.full((n + 4096,), 0x35, dtype=torch.uint8, device=DEV)
    got = binding.kv_attention(q, cache.pages, i32(cache.table), i32(cache.lens), cache.H, cache.page, cache.dtype, workspace=ws[:n])
    assert bool((ws[n:] == 0x35).all())
    return got, ws


@pytest.mark.parametrize("dtype", ["bf16", "i8"])
@pytest.mark.parametrize("B,each", [(51, 160), (40, 160), (28, 290), (1, 30000)])
def test_as_many_parts_as_there_can_be(B, each, dtype):
    """Every request just above a workgroup's share, so that each is in two parts, and more requests without tokens between them."""
    H, D = 8, 64
    groups = 2 * torch.cuda.get_device_properties(0).multi_processor_count // H
    lens = [each if i % 3 == 1 else 0 for i in range(3 * B)]
    cache = Cache(np.random.default_rng(B), lens, H, D, 64, dtype, W=max(40, -(-each // 64)))      # a table that is wide enough for a division
    q = queries(3 * B, 16, D, "bf16")
    divided = parts(lens, groups)
    got, ws = attend(cache, q, binding.kv_attention_workspace_bytes(3 * B, 16, H, D))
    assert [p for _, p in plan(ws, 3 * B)] == divided and min(divided[1::3]) >= 2
    cache.check(got, q)


def test_of_4096_requests():
    """Divided ones first, last and in between; a part's place does not follow from the number of its request."""
    lens = [3 if i % 5 == 0 else 0 for i in range(4096)]
    for i, n in ((0, 9000), (63, 700), (64, 701), (2000, 3000), (4095, 5000)):
        lens[i] = n
    cache = Cache(np.random.default_rng(41), lens, 2, 32, 32, "bf16")
    q = queries(4096, 4, 32, "bf16")
    n = binding.kv_attention_workspace_bytes(4096, 4, 2, 32)
    got, ws = attend(cache, q, n)
    cache.check(got, q)
    assert [p for _, p in plan(ws, 4096)] == parts(lens, torch.cuda.get_device_properties(0).multi_processor_count)
    again, _ = attend(cache, q, n)
    assert torch.equal(got, again)
    for less in (n - 1, n // 2, n // 4, n // 16):                  # fewer parts
        cache.check(attend(cache, q, less)[0], q)
