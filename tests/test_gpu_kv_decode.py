"""The cache's operators together, as a block decodes with them: pages for requests that come and go, keys and values written, attention over them."""
import numpy as np
import pytest
import torch

from oracle import kv_oracle as ko
from paper_2603_05232_amd import synth
from paper_2603_05232_amd.block import HEAD_DIM, HIDDEN, N_KV_HEADS, N_Q_HEADS, LlamaBlock
from paper_2603_05232_amd.kv_cache import PagedCache

pytestmark = pytest.mark.gpu
DEV = torch.device("cuda:0")


@pytest.fixture(scope="module")
def block():
    return LlamaBlock(DEV)


def hidden(M, seed):
    return torch.from_numpy(synth.activations(M, HIDDEN, seed=seed)).to(DEV).to(torch.bfloat16)


def i32(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


def keys_and_values(record):
    qkv = record["qkv"][1].unflatten(1, (-1, HEAD_DIM))
    return qkv[:, N_Q_HEADS:N_Q_HEADS + N_KV_HEADS], qkv[:, N_Q_HEADS + N_KV_HEADS:]


@pytest.mark.parametrize("dtype", ["bf16", "i8"])
def test_prompts_then_tokens(block, dtype):
    """Prompts of several lengths, then steps across a page's end; every step's attention against the oracle on the keys and values that the block's layer gave."""
    prompts = [60, 1, 130]
    cache = PagedCache(DEV, 3, 12, 4, N_KV_HEADS, HEAD_DIM, 64, dtype)
    held = []
    for b, n in enumerate(prompts):
        want = cache.lens.clone()
        want[b] = n
        slots, offsets = cache.resize(want, n + 2)
        assert offsets.tolist() == [0] * (b + 1) + [n] * (3 - b) and slots[n:].tolist() == [-1, -1]
        record = {}
        block.forward(hidden(n, b), record=record, cache=cache, slots=slots[:n])
        held.append([keys_and_values(record)])
    for step in range(7):
        x, record = hidden(3, 50 + step), {}
        y = block.decode(x, cache, cache.step(), record=record)
        assert y.shape == (3, HIDDEN) and bool(torch.isfinite(y.float()).all())
        k, v = keys_and_values(record)
        q, a = record["attention"]
        assert cache.lens.tolist() == [n + step + 1 for n in prompts]
        for b in range(3):
            held[b].append((k[b:b + 1], v[b:b + 1]))
            ks, vs = (ko.held(torch.cat([p[i] for p in held[b]]).float().cpu().numpy(), dtype) for i in (0, 1))
            ref = ko.attention(q[b].double().cpu().numpy(), ks, vs, HEAD_DIM ** -0.5, np.ones(ks.shape[0], bool))
            assert (np.abs(a[b].double().cpu().numpy() - ref[0]) <= ko.bound(*ref, HEAD_DIM, ks.shape[0], dtype, False)).all()
    t = torch.arange(67, device=DEV)                               # and all of it lies where the table says
    k, v = cache.read((cache.table[0].long()[t // 64] * 64 + t % 64).int(), torch.float32)
    assert np.array_equal(k.cpu().numpy(), ko.held(torch.cat([p[0] for p in held[0]]).float().cpu().numpy(), dtype))
    assert np.array_equal(v.cpu().numpy(), ko.held(torch.cat([p[1] for p in held[0]]).float().cpu().numpy(), dtype))


def steps(block, cache, x, n):
    out = []
    for i in range(n):
        out.append(block.decode(x + i / 8, cache, cache.step()))
    return out


def fill(block, lens, pages=40, width=12, dtype="bf16"):
    cache = PagedCache(DEV, len(lens), pages, width, N_KV_HEADS, HEAD_DIM, 64, dtype)
    slots, _ = cache.resize(i32(lens), sum(lens))
    g = torch.Generator(device=DEV).manual_seed(1)
    k, v = (torch.randn((sum(lens), N_KV_HEADS, HEAD_DIM), generator=g, device=DEV).to(torch.bfloat16) for _ in "kv")
    cache.write(k, v, slots)
    return cache


def test_a_captured_step(block):
    """One step in a graph, replayed over a page's end and past the length at which requests are divided, with eager steps of another cache in between."""
    lens = [62, 3, 700]
    x = hidden(3, 7)
    want = steps(block, fill(block, lens), x, 6)
    cache, other = fill(block, lens), fill(block, [100, 650, 9])
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
        torch.empty((1 << 20,), dtype=torch.uint8, device=DEV).fill_(0xA5)
        torch.cuda.synchronize()
    assert cache.lens.tolist() == [n + 6 for n in lens]


def test_two_streams(block):
    a, b = [500, 64, 640], [63, 700, 1]
    x = hidden(3, 8)
    want = [steps(block, fill(block, lens), x, 4) for lens in (a, b)]
    caches = [fill(block, lens) for lens in (a, b)]
    torch.cuda.synchronize()
    streams, got = [torch.cuda.Stream() for _ in range(2)], [[], []]
    for i in range(4):
        for s in range(2):
            with torch.cuda.stream(streams[s]):
                got[s].append(block.decode(x + i / 8, caches[s], caches[s].step()))
    torch.cuda.synchronize()
    for s in range(2):
        for y, z in zip(got[s], want[s]):
            assert torch.equal(y, z)


def test_requests_that_wait_end_and_find_no_room(block):
    cache = fill(block, [64, 10, 64], pages=4, width=3)
    assert cache.left.tolist() == [1]
    x = hidden(3, 9)
    slots = cache.step(torch.tensor([False, True, False], device=DEV))
    assert slots.tolist()[::2] == [-1, -1] and cache.lens.tolist() == [64, 11, 64]
    y = block.decode(x, cache, slots)
    assert bool(torch.isfinite(y.float()).all())
    slots = cache.step()                                           # one page for the two that need one
    assert slots.tolist()[2] == -1 and slots.tolist()[0] >= 0 and cache.lens.tolist() == [65, 12, 64] and cache.left.tolist() == [0]
    before = cache.pages.clone()
    ids = cache.table[2, :1].tolist()
    block.decode(x, cache, slots)
    assert torch.equal(before[ids], cache.pages[ids])              # the request that was left out is as it was
    cache.resize(i32([0, 12, 64]), 0)
    assert cache.left.tolist() == [2] and cache.lens.tolist() == [0, 12, 64]
    slots = cache.step(torch.tensor([False, True, True], device=DEV))
    assert cache.lens.tolist() == [0, 13, 65] and slots.tolist()[2] >= 0
    record = {}
    block.decode(x, cache, slots, record=record)
    assert bool((record["attention"][1][0] == 0).all())            # a request without tokens


def test_command(monkeypatch, capsys):
    from paper_2603_05232_amd import kv_cache
    monkeypatch.setattr("sys.argv", ["kv_cache", "--requests", "3", "--context", "100", "--steps", "2", "--dtype", "fp8"])
    kv_cache.main()
    assert "3 requests of 100 tokens" in capsys.readouterr().out
