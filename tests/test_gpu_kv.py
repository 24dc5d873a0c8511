"""The operators on a paged cache of keys and values against the oracle: pages and slots and what the cache holds bit for bit, attention within the bound that oracle.kv_oracle.bound derives."""
import types

import numpy as np
import pytest
import torch

from oracle import kv_oracle as ko
from paper_2603_05232_amd import binding

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
SOURCE = {"bf16": torch.bfloat16, "fp32": torch.float32}


def i32(x):
    return torch.as_tensor(np.asarray(x, np.int32), device=DEV)


# ---- pages and slots ----

def step_of(rng, B, W, page, kind):
    """Lengths before and after; the pages in use; free ones."""
    most = W * page
    lens = [0 if rng.random() < 0.2 else int(rng.integers(1, most + 1)) for _ in range(B)]
    if kind == "decode":
        want = [n + 1 for n in lens]                    # one over, where a request is at its end
    elif kind == "odd":
        want = [int(rng.choice([0, n, max(n - 1, 0), n + 1, n + page, most, most + 1, -3])) for n in lens]
    else:
        want = [int(rng.integers(0, most + 1)) for _ in range(B)]
    counts = [-(-n // page) for n in lens]
    free = int(rng.integers(0, B * W + 2)) if kind != "decode" else B
    P = sum(counts) + free + 2
    order = rng.permutation(P)
    table, at = rng.integers(-5, P + 5, (B, W)), 0
    for b, n in enumerate(counts):
        table[b, :n] = order[at:at + n]
        at += n
    pool = np.concatenate([order[at:at + free], rng.integers(0, P, P - free)])
    return lens, want, table, pool, free


def check_tables(lens, want, table, pool, left, page, N, **given):
    ref = ko.tables(lens, want, table, page, pool, left, N)
    wide = torch.full((table.shape[0], table.shape[1] + 3), 77, dtype=torch.int32, device=DEV)      # rows of a larger table
    t = wide[:, 1:1 + table.shape[1]]
    t.copy_(i32(table))
    p = i32(pool)
    got = binding.kv_tables(i32(lens), i32(want), t, p, i32([left]), page, N, **given)
    for name, a, b in zip(("lens", "left", "slots", "offsets", "table", "pool"), (*got, t, p), (ref[0], [ref[1]], ref[2], ref[3], ref[4], ref[5])):
        assert a.cpu().numpy().tolist() == np.asarray(b).tolist(), name
    assert bool((wide[:, 0] == 77).all()) and bool((wide[:, 1 + table.shape[1]:] == 77).all())


@pytest.mark.parametrize("kind", ["decode", "any", "odd"])
@pytest.mark.parametrize("B,W,page", [(1, 1, 32), (3, 5, 64), (64, 7, 32), (65, 3, 96), (1000, 4, 32), (1025, 2, 32), (4096, 2, 32)])
def test_tables(B, W, page, kind):
    rng = np.random.default_rng(B + W)
    lens, want, table, pool, left = step_of(rng, B, W, page, kind)
    total = sum(max(0, max(w, 0) - n) for w, n in zip(want, lens))
    check_tables(lens, want, table, pool, left, page, total + 5)
    check_tables(lens, want, table, pool, left, page, total // 2)                                     # rows for half of them


def test_tables_whose_new_pages_were_just_given_back():
    """No free page but those of requests that end or shrink, in the same call, with more rows than one workgroup fills in."""
    rng = np.random.default_rng(21)
    B, W, page = 200, 12, 64
    lens = [int(n) for n in rng.integers(1, W * page + 1, B)]
    want = [int(rng.choice([0, n // 2, n])) if b % 2 else min(n + int(rng.integers(0, 200)), W * page) for b, n in enumerate(lens)]
    counts = [-(-n // page) for n in lens]
    order, table, at = rng.permutation(sum(counts)), np.full((B, W), -1), 0
    for b, n in enumerate(counts):
        table[b, :n] = order[at:at + n]
        at += n
    N = sum(max(0, w - n) for w, n in zip(want, lens))
    assert N > 4096 and sum(-(-w // page) for w in want) <= sum(counts)
    check_tables(lens, want, table, np.zeros(sum(counts)), 0, page, N)


def test_tables_of_one_launch_and_of_two():
    rng = np.random.default_rng(9)
    lens, want, table, pool, left = step_of(rng, 40, 16, 64, "any")
    total = sum(max(0, w - n) for w, n in zip(want, lens))
    assert 4096 < total < 30000
    for N in (2048, 2049, total, 1 << 20):
        check_tables(lens, want, table, pool, left, 64, N)


def test_tables_of_one_long_request_and_of_lists_that_mean_nothing():
    W, page = 2049, 64
    pool = np.arange(W + 3)
    check_tables([0], [131072], np.zeros((1, W)), pool, W + 3, page, 131072)
    check_tables([131072], [0], np.arange(W)[None], np.arange(W + 3), 0, page, 4)                     # all pages back at once
    check_tables([-5, 70, 1 << 30], [3, 1 << 30, -(1 << 31)], np.array([[-7, 900], [1, 2], [3, 4]]), np.array([5, -1, 1 << 30, 8, 2, 1]), 1 << 20, 32, 50)
    check_tables([0, 0], [1, 40], np.zeros((2, 2)), np.array([5, -1, 1 << 30, 0]), 4, 32, 50)         # pages that there are not: slots -1


def test_tables_of_sums_beyond_32_bits():
    """Every request wants as many rows as a call can have, so that their sum is 2^31 and more: all but one, which wants none, are left out, and that one keeps its page."""
    B, W, page, N = 3000, 32769, 32, 1 << 20
    table = torch.arange(B, dtype=torch.int32, device=DEV)[:, None].repeat(1, W)
    before = table.clone()
    lens, want = torch.ones((B,), dtype=torch.int32, device=DEV), torch.full((B,), W * page, dtype=torch.int32, device=DEV)
    want[B - 1] = 1
    pool = torch.arange(1 << 22, dtype=torch.int32, device=DEV)
    got = binding.kv_tables(lens, want, table, pool, i32([1 << 22]), page, N)
    assert torch.equal(got[0], lens) and got[1].tolist() == [1 << 22] and bool((got[2] == -1).all()) and got[3].tolist() == [0] + [N] * B
    assert torch.equal(table, before)
    want[1], want[B - 1] = 3, 0                                    # one that gives a page back; one that is small, but behind a row too many
    got = binding.kv_tables(lens, want, table, pool, i32([1000]), page, N)
    assert got[0].tolist() == [1] * (B - 1) + [0] and got[1].tolist() == [1001] and pool[1000].item() == B - 1 and bool((got[2] == -1).all())


@pytest.mark.parametrize("B,W", [(30, 6), (30, 40), (1024, 9)])
def test_tables_in_place_and_again(B, W):
    """new_lens and new_left may be lens and left; the same call on the same lengths gives the same."""
    rng = np.random.default_rng(4)
    lens, want, table, pool, left = step_of(rng, B, W, 32, "any")
    N = sum(max(0, w - n) for w, n in zip(want, lens)) + 1
    ref = ko.tables(lens, want, table, 32, pool, left, N)
    a = dict(lens=i32(lens), left=i32([left]), table=i32(table), pool=i32(pool))
    for _ in range(2):
        got = binding.kv_tables(a["lens"], i32(want), a["table"], a["pool"], a["left"], 32, N)
        assert got[2].tolist() == ref[2] and a["table"].cpu().numpy().tolist() == ref[4].tolist() and a["pool"].tolist() == ref[5]
    got = binding.kv_tables(a["lens"], i32(want), a["table"], a["pool"], a["left"], 32, N, new_lens=a["lens"], new_left=a["left"])
    assert got[0] is a["lens"] and got[1] is a["left"] and a["lens"].tolist() == ref[0] and a["left"].tolist() == [ref[1]] and got[2].tolist() == ref[2]


def test_tables_without_requests():
    lens, left, slots, offsets = binding.kv_tables(i32([]), i32([]), torch.zeros((0, 3), dtype=torch.int32, device=DEV), i32([1, 2]), i32([2]), 32, 4)
    assert lens.shape == (0,) and left.tolist() == [2] and slots.tolist() == [-1] * 4 and offsets.tolist() == [0]
    assert binding.kv_tables(i32([3]), i32([3]), i32([[0]]), i32([1]), i32([1]), 32, 0)[2].shape == (0,)


# ---- keys and values ----

def empty_pages(P, H, page, D, dtype, fill=0):
    return torch.full((P, binding.kv_page_bytes(H, page, D, dtype)), fill, dtype=torch.uint8, device=DEV)


def rows_of(seed, N, H, D, source, spread=True):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn((N, H, D), generator=g)
    if spread:
        x = x * torch.logspace(-2, 2, max(N, 1))[:N, None, None]
    return x.to(SOURCE[source]).to(DEV)


def runs(rng, P, page, N, kind):
    """Slots of N tokens, all different: one run from anywhere, requests of some tokens each, or single tokens."""
    if kind == "run":
        at = int(rng.integers(0, P * page - N + 1))
        return np.arange(at, at + N)
    if kind == "single":
        return rng.permutation(P * page)[:N]
    pieces = np.split(np.arange(P * page), np.sort(rng.choice(np.arange(1, P * page), size=P * page // 13, replace=False)))
    rng.shuffle(pieces)
    return np.concatenate(pieces)[:N]


def as_out(x, source):
    return ko.bf16(x) if source == "bf16" else x


@pytest.mark.parametrize("dtype", ["bf16", "fp16", "i8", "fp8"])
@pytest.mark.parametrize("N,H,D,page,kind,source", [(1, 1, 1, 32, "single", "fp32"), (1, 8, 128, 64, "single", "bf16"), (100, 2, 64, 32, "run", "bf16"), (300, 3, 80, 96, "pieces", "fp32"),
                                                    (77, 5, 33, 64, "single", "bf16"), (500, 1, 256, 128, "run", "bf16"), (250, 2, 130, 32, "pieces", "bf16"), (41, 4, 100, 32, "run", "fp32"),
                                                    (3001, 2, 96, 64, "pieces", "bf16"), (2500, 1, 16, 4096, "run", "fp32")])
def test_write_and_read(N, H, D, page, kind, source, dtype):
    rng = np.random.default_rng(N + D)
    P = -(-N // page) + 3
    slots = runs(rng, P, page, N, kind)
    all_slots = i32(np.arange(P * page))
    K0, V0 = rows_of(1, P * page, H, D, source), rows_of(2, P * page, H, D, source)
    pages = empty_pages(P, H, page, D, dtype, 0xFF)
    binding.kv_write(K0, V0, all_slots, pages, page, dtype)
    K, V = rows_of(3, N, H, D, source), rows_of(4, N, H, D, source)
    given = slots.copy()
    if N > 3:
        given[[1, N // 2, N - 1]] = (-1, P * page, -(1 << 31))         # passed over
    binding.kv_write(K, V, i32(given), pages, page, dtype)
    for x0, x, got in zip((K0, V0), (K, V), binding.kv_read(pages, all_slots, H, D, page, dtype, SOURCE[source])):
        want = ko.held(x0.float().cpu().numpy(), dtype)
        mine = ko.held(x.float().cpu().numpy(), dtype)
        ok = (given >= 0) & (given < P * page)
        want[given[ok]] = mine[ok]
        assert np.array_equal(got.float().cpu().numpy(), as_out(want, source))
    # slots of reading in any order, and outside
    some = np.concatenate([rng.integers(0, P * page, 9), [-1, P * page, 2 ** 31 - 1]])
    k, v = binding.kv_read(pages, i32(some), H, D, page, dtype, torch.float32)
    assert bool((k[9:] == 0).all()) and bool((v[9:] == 0).all())
    whole = binding.kv_read(pages, all_slots, H, D, page, dtype, torch.float32)
    assert torch.equal(k[:9], whole[0][torch.as_tensor(some[:9], device=DEV)]) and torch.equal(v[:9], whole[1][torch.as_tensor(some[:9], device=DEV)])


@pytest.mark.parametrize("dtype", ["bf16", "fp16", "i8", "fp8"])
def test_write_and_read_with_strides(dtype):
    """Keys and values as columns of a projection's result, values in another order of heads; results into columns of a larger tensor."""
    N, H, D, page = 70, 3, 80, 32
    qkv = rows_of(5, N, 1, 11 * D + 3, "bf16", spread=False)[:, 0]
    K = qkv[:, 1:1 + H * D].unflatten(1, (H, D))
    V = qkv[:, 4 * D:4 * D + 2 * H * D].unflatten(1, (H, 2 * D))[:, :, 1:1 + D]
    slots = i32(np.random.default_rng(1).permutation(96)[:N])
    pages = empty_pages(3, H, page, D, dtype)
    binding.kv_write(K, V, slots, pages, page, dtype)
    out = torch.full((N, 2, H, D + 1), 7.0, device=DEV)
    k, v = binding.kv_read(pages, slots, H, D, page, dtype, K=out[:, 0, :, :D], V=out[:, 1, :, 1:])
    for got, x in ((k, K), (v, V)):
        assert np.array_equal(got.cpu().numpy(), ko.held(x.float().cpu().numpy(), dtype))
    assert bool((out[:, 0, :, D] == 7).all()) and bool((out[:, 1, :, 0] == 7).all())


@pytest.mark.parametrize("dtype", ["i8", "fp8"])
def test_values_that_are_no_numbers_and_tiny_ones(dtype):
    x = torch.randn((16, 2, 64), device=DEV)
    x[0, 0, 5], x[1, 0, 63], x[2, 1], x[3, 0], x[9, 1, 0] = float("inf"), float("nan"), 0.0, 1e-38, float("-inf")
    pages = empty_pages(1, 2, 32, 64, dtype)
    binding.kv_write(x, x.flip(0), i32(range(16)), pages, 32, dtype)
    k, v = binding.kv_read(pages, i32(range(16)), 2, 64, 32, dtype, torch.float32)
    assert np.array_equal(k.cpu().numpy(), ko.held(x.cpu().numpy(), dtype), equal_nan=True) and np.array_equal(v.cpu().numpy(), ko.held(x.flip(0).cpu().numpy(), dtype), equal_nan=True)


def test_no_tokens_and_no_requests():
    pages = empty_pages(2, 3, 32, 40, "i8")
    none = torch.zeros((0, 3, 40), device=DEV)
    binding.kv_write(none, none, i32([]), pages, 32, "i8")
    for given in ({}, dict(K=none.clone()), dict(V=none.clone())):
        k, v = binding.kv_read(pages, i32([]), 3, 40, 32, "i8", torch.float32, **given)
        assert k.shape == v.shape == (0, 3, 40) and k.dtype == v.dtype == torch.float32
    out = binding.kv_attention(torch.zeros((0, 6, 40), device=DEV), pages, torch.zeros((0, 2), dtype=torch.int32, device=DEV), i32([]), 3, 32, "i8")
    assert out.shape == (0, 6, 40) and bool((pages == 0).all())


# ---- attention ----

class Cache:
    """Requests of `lens` tokens in pages of any order; every slot that holds no token is filled with bytes 0xFF: NaNs in bf16, fp16, fp8 and the scales."""

    def __init__(self, rng, lens, H, D, page, dtype, W=None, source="bf16", size=1.0):
        self.lens, self.H, self.D, self.page, self.dtype = list(lens), H, D, page, dtype
        counts = [-(-n // page) for n in lens]
        P = sum(counts) + 2
        W = W or max(1, max(counts, default=1))
        order = rng.permutation(P)
        self.table = rng.choice([-1, P, 1 << 30], (len(lens), W))                       # columns that no token reaches
        at = 0
        for b, n in enumerate(counts):
            self.table[b, :n] = order[at:at + n]
            at += n
        self.pages = empty_pages(P, H, page, D, dtype, 0xFF)
        total = sum(lens)
        self.K, self.V = (size * torch.randn((total, H, D), generator=torch.Generator().manual_seed(int(rng.integers(1 << 30)))) for _ in "KV")
        self.K[:, :, ::17] *= 5
        self.K, self.V = self.K.to(SOURCE[source]), self.V.to(SOURCE[source])
        t = np.concatenate([np.arange(n) for n in lens]).astype(np.int64) if total else np.zeros(0, np.int64)
        b = np.repeat(np.arange(len(lens)), lens)
        slots = self.table[b, t // page] * page + t % page if total else t
        if total:
            binding.kv_write(self.K.to(DEV), self.V.to(DEV), i32(slots), self.pages, page, dtype)
        self.k, self.v = ko.held(self.K.float().numpy(), dtype), ko.held(self.V.float().numpy(), dtype)
        self.starts = np.concatenate([[0], np.cumsum(lens)]).astype(int)

    def __call__(self, q, ws=True, **kw):
        B, Hq, D = q.shape
        n = binding.kv_attention_workspace_bytes(B, Hq, self.H, D)
        self.scratch = scratch = torch.full((n,), 0x7F, dtype=torch.uint8, device=DEV) if ws else None
        return binding.kv_attention(q, self.pages, i32(self.table), i32(self.lens), self.H, self.page, self.dtype, workspace=scratch, **kw)

    def check(self, got, q, scale=None, window=0, seen=None):
        for b, n in enumerate(self.lens):
            t = np.arange(n)
            visible = (t >= n - window if window else t >= 0) & (True if seen is None else seen(b, t))
            rows = slice(self.starts[b], self.starts[b] + n)
            ref = ko.attention(q[b].double().cpu().numpy(), self.k[rows], self.v[rows], self.D ** -0.5 if scale is None else scale, visible)
            off = np.abs(got[b].double().cpu().numpy() - ref[0])
            most = ko.bound(*ref, self.D, n, self.dtype, q.dtype == torch.float32)
            assert (off <= most).all(), (b, n, float((off / most).max()))


def queries(B, Hq, D, source, seed=11, size=1.0):
    return (size * torch.randn((B, Hq, D), generator=torch.Generator().manual_seed(seed))).to(SOURCE[source]).to(DEV)


LENS = [0, 1, 31, 32, 33, 63, 64, 65, 200, 127, 128, 500]


@pytest.mark.parametrize("dtype", ["bf16", "fp16", "i8", "fp8"])
@pytest.mark.parametrize("Hq,H,D,page,source", [(4, 4, 64, 32, "bf16"), (8, 2, 128, 64, "bf16"), (8, 2, 128, 32, "fp32"), (15, 3, 80, 32, "fp32"), (17, 1, 96, 96, "bf16"), (40, 1, 32, 64, "bf16"),
                                               (3, 3, 1, 32, "bf16"), (6, 2, 17, 32, "fp32"), (2, 1, 160, 64, "bf16"), (2, 2, 192, 32, "fp32"), (16, 1, 256, 128, "bf16"), (5, 1, 255, 64, "fp32"),
                                               (32, 1, 100, 4096, "bf16")])
def test_attention(Hq, H, D, page, source, dtype):
    cache = Cache(np.random.default_rng(Hq + D), LENS, H, D, page, dtype)
    q = queries(len(LENS), Hq, D, source)
    got = cache(q)
    cache.check(got, q)
    cache.check(cache(q, ws=False), q)
    assert bool((got[0] == 0).all())
    for window in (1, 33, 100):
        cache.check(cache(q, window=window), q, window=window)


@pytest.mark.parametrize("dtype", ["bf16", "fp16", "i8", "fp8"])
@pytest.mark.parametrize("lens,Hq,H,D,window", [([20000], 4, 1, 128, 0), ([5000, 0, 9, 7001, 513], 8, 2, 64, 0), ([3000] * 9, 20, 1, 96, 0), ([20000, 600], 2, 2, 80, 7000), ([2049] * 3, 6, 3, 256, 0)])
def test_attention_over_long_caches(lens, Hq, H, D, window, dtype):
    cache = Cache(np.random.default_rng(len(lens) + D), lens, H, D, 64, dtype)
    q = queries(len(lens), Hq, D, "bf16", size=2.0)
    divided = cache(q, window=window)
    assert bool((cache.scratch != 0x7F).any())                     # it was
    cache.check(divided, q, window=window)
    cache.check(cache(q, window=window, ws=False), q, window=window)
    for _ in range(3):
        assert torch.equal(divided, cache(q, window=window))


def test_attention_of_many_requests():
    rng = np.random.default_rng(0)
    lens = [int(n) for n in rng.integers(0, 90, 300)] + [4000]
    cache = Cache(rng, lens, 2, 64, 32, "bf16")
    q = queries(301, 6, 64, "bf16")
    cache.check(cache(q), q)


def test_attention_of_4096_requests():
    """As many as there can be, most of them in the last of the pieces in which lengths are read; some are long enough to be divided."""
    rng = np.random.default_rng(12)
    lens = [0 if i % 7 else int(n) for i, n in enumerate(rng.integers(1, 70, 4096))]
    lens[4095], lens[1000], lens[63] = 3000, 2500, 1
    cache = Cache(rng, lens, 1, 16, 32, "bf16")
    q = queries(4096, 3, 16, "bf16")
    got = cache(q)
    cache.check(got, q)
    assert bool((got[[i for i, n in enumerate(lens) if n == 0]] == 0).all())


@pytest.mark.parametrize("Hq,H", [(96, 1), (200, 4), (1024, 1024), (1024, 2)])
def test_attention_of_many_heads(Hq, H):
    cache = Cache(np.random.default_rng(13), [700, 33], H, 16, 32, "fp8")
    q = queries(2, Hq, 16, "bf16")
    cache.check(cache(q), q)


def test_requests_that_share_pages():
    """Two requests whose rows of the table begin with the same pages, as after a common prompt."""
    cache = Cache(np.random.default_rng(14), [1000, 900], 2, 64, 32, "bf16")
    cache.table[1, :20] = cache.table[0, :20]
    cache.k, cache.v = (x.copy() for x in (cache.k, cache.v))
    cache.k[1000:1640], cache.v[1000:1640] = cache.k[:640], cache.v[:640]
    q = queries(2, 4, 64, "bf16")
    cache.check(cache(q), q)


@pytest.mark.parametrize("room", [0, 1, 2, 5])
def test_attention_with_less_room(room):
    """A workspace with room for few parts, or for none."""
    cache = Cache(np.random.default_rng(1), [6000, 700], 2, 64, 64, "bf16")
    q = queries(2, 4, 64, "bf16")
    per = 2 * 16 * (8 + 4 * 64)                                    # a part: two heads of keys, sixteen columns
    n = 16 + (4 + room) * per                                      # behind the division of two requests
    ws = torch.zeros((n + 64,), dtype=torch.uint8, device=DEV)
    got = binding.kv_attention(q, cache.pages, i32(cache.table), i32(cache.lens), 2, 64, "bf16", workspace=ws[:n])
    cache.check(got, q)
    assert bool((ws[n:] == 0).all()) and bool((ws != 0).any()) == (room > 1)


@pytest.mark.parametrize("dtype", ["bf16", "fp16", "i8", "fp8"])
def test_attention_with_strides_and_a_scale(dtype):
    lens, H, D = [70, 0, 33], 2, 72
    cache = Cache(np.random.default_rng(2), lens, H, D, 32, dtype)
    wide = queries(3, 1, 9 * D + 5, "bf16")[:, 0]
    q = wide[:, 3:3 + 8 * D].unflatten(1, (4, 2 * D))[:, :, :D]
    out = torch.full((3, 4, D + 3), 7.0, dtype=torch.bfloat16, device=DEV)
    table = torch.full((3, 20), 1 << 30, dtype=torch.int32, device=DEV)
    table[:, 5:5 + cache.table.shape[1]] = i32(cache.table)
    got = binding.kv_attention(q, cache.pages, table[:, 5:5 + cache.table.shape[1]], i32(lens), H, 32, dtype, scale=0.7, out=out[:, :, 1:1 + D])
    cache.check(got, q, scale=0.7)
    assert bool((out[:, :, 0] == 7).all()) and bool((out[:, :, 1 + D:] == 7).all())
    assert torch.equal(got, cache(q.contiguous(), scale=0.7))


@pytest.mark.parametrize("scale", [-0.3, 0.0])
@pytest.mark.parametrize("dtype", ["bf16", "fp16", "i8"])
def test_attention_of_a_scale_below_and_at_zero(dtype, scale):
    cache = Cache(np.random.default_rng(15), [600, 40], 2, 64, 32, dtype)
    q = queries(2, 4, 64, "bf16")
    cache.check(cache(q, scale=scale), q, scale=float(np.float32(scale)))


@pytest.mark.parametrize("dtype", ["bf16", "fp16", "i8", "fp8"])
def test_attention_passes_over_pages_that_there_are_not(dtype):
    lens = [300, 5000, 64]
    cache = Cache(np.random.default_rng(3), lens, 2, 64, 64, dtype)
    P = cache.pages.shape[0]
    cache.table[0, 1], cache.table[0, 4], cache.table[1, 10], cache.table[1, 60], cache.table[2, 0] = -1, P, 1 << 30, -(1 << 31), P + 7
    missing = [(0, 1), (0, 4), (1, 10), (1, 60), (2, 0)]
    q = queries(3, 4, 64, "bf16")
    got = cache(q)
    cache.check(got, q, seen=lambda b, t: ~np.isin(t // 64, [c for r, c in missing if r == b]))
    assert bool((got[2] == 0).all())


def test_attention_of_lengths_that_mean_nothing():
    """Below 0 counts as 0, beyond the table as its width."""
    cache = Cache(np.random.default_rng(4), [128, 128], 1, 64, 32, "bf16")
    q = queries(2, 2, 64, "bf16")
    got = binding.kv_attention(q, cache.pages, i32(cache.table), i32([-9, 2 ** 31 - 1]), 1, 32, "bf16")
    assert bool((got[0] == 0).all()) and torch.equal(got[1], cache(q)[1])


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
def test_attention_of_scores_that_are_no_numbers(dtype):
    inf, nan = float("inf"), float("nan")
    cache = Cache(np.random.default_rng(5), [40, 40, 40, 40, 700], 1, 64, 32, dtype, source="fp32")
    K, V = cache.K.clone(), cache.V.clone()
    K[:, :, 0] = 1.0
    K[0:40, 0, 0] = -inf                                 # request 0: every score minus infinity
    K[41, 0, 0] = -inf                                   # request 1: one
    K[85, 0, 0] = nan                                    # request 2
    V[130, 0, 7] = nan                                   # request 3: one channel
    K[300, 0, 0] = -inf
    t = np.concatenate([np.arange(n) for n in cache.lens])
    b = np.repeat(np.arange(5), cache.lens)
    binding.kv_write(K.to(DEV), V.to(DEV), i32(cache.table[b, t // 32] * 32 + t % 32), cache.pages, 32, dtype)
    cache.k, cache.v = ko.held(K.numpy(), dtype), ko.held(V.numpy(), dtype)
    q = queries(5, 2, 64, "bf16")
    q[:, :, 0] = 1.0
    got = cache(q)
    assert bool((got[0] == 0).all()) and bool(got[2].isnan().all())
    assert bool(got[3, :, 7].isnan().all()) and int(got[3].isnan().sum()) == 2
    for r in (1, 4):
        n = cache.lens[r]
        rows = slice(cache.starts[r], cache.starts[r] + n)
        keep = np.isfinite(cache.k[rows]).all((1, 2))
        ref = ko.attention(q[r].double().cpu().numpy(), cache.k[rows], cache.v[rows], 0.125, keep)
        assert (np.abs(got[r].double().cpu().numpy() - ref[0]) <= ko.bound(*ref, 64, n, dtype, False)).all()


@pytest.mark.parametrize("dtype", ["i8", "fp8"])
def test_attention_over_keys_that_are_no_numbers(dtype):
    cache = Cache(np.random.default_rng(6), [40, 40, 40], 2, 64, 32, dtype)
    K, V = cache.K.clone(), cache.V.clone()
    K[5, 0, 3] = float("inf")
    V[45, 1, 3] = float("nan")
    t, b = np.tile(np.arange(40), 3), np.repeat(np.arange(3), 40)
    binding.kv_write(K.to(DEV), V.to(DEV), i32(cache.table[b, t // 32] * 32 + t % 32), cache.pages, 32, dtype)
    got = cache(queries(3, 4, 64, "bf16")).isnan()
    assert bool(got[0, :2].all()) and not bool(got[0, 2:].any()) and bool(got[1, 2:].all()) and not bool(got[1, :2].any()) and not bool(got[2].any())


@pytest.mark.parametrize("source", ["bf16", "fp32"])
@pytest.mark.parametrize("dtype", ["bf16", "fp16", "i8", "fp8"])
@pytest.mark.parametrize("size", [1e-30, 1e-4, 3e4, 1e30])
def test_attention_of_queries_of_any_size(size, dtype, source):
    """The scores are brought back by the scale."""
    cache = Cache(np.random.default_rng(7), [100, 3], 1, 64, 32, dtype, size=0.1)
    q = queries(2, 3, 64, source, size=size)
    cache.check(cache(q, scale=0.5 / size), q, scale=float(np.float32(0.5 / size)))


def test_attention_over_a_cache_of_more_than_4_gib():
    """Pages and offsets beyond 32 bits."""
    H, D, page, dtype = 8, 128, 1024, "bf16"
    size = binding.kv_page_bytes(H, page, D, dtype)
    P = (9 << 30) // size
    pages = torch.empty((P, size), dtype=torch.uint8, device=DEV)
    ids = [P - 1, 1, P // 2 + 3]
    K, V = rows_of(1, 3 * page, H, D, "bf16", spread=False), rows_of(2, 3 * page, H, D, "bf16", spread=False)
    slots = i32(np.concatenate([np.arange(page) + i * page for i in ids]))
    binding.kv_write(K, V, slots, pages, page, dtype)
    k, v = binding.kv_read(pages, slots, H, D, page, dtype)
    assert torch.equal(k, K) and torch.equal(v, V)
    q = queries(1, 16, D, "bf16")
    ws = torch.empty((binding.kv_attention_workspace_bytes(1, 16, H, D),), dtype=torch.uint8, device=DEV)
    got = binding.kv_attention(q, pages, i32([ids]), i32([3 * page]), H, page, dtype, workspace=ws)
    ref = ko.attention(q[0].double().cpu().numpy(), K.double().cpu().numpy(), V.double().cpu().numpy(), D ** -0.5, np.ones(3 * page, bool))
    assert (np.abs(got[0].double().cpu().numpy() - ref[0]) <= ko.bound(*ref, D, 3 * page, dtype, False)).all()


# ---- as programs call them ----

def test_calls_through_the_module_and_without_it(monkeypatch):
    """The extension module takes plain calls, the general path gives the same."""
    binding.load()
    lens, want = i32([40, 0, 64, 3000]), i32([41, 90, 10, 3001])
    x = rows_of(1, 92, 2, 64, "bf16", spread=False)
    q = queries(4, 4, 64, "bf16")

    def calls():
        table = torch.zeros((4, 64), dtype=torch.int32, device=DEV)
        table[0, :2], table[2, :2], table[3, :47] = i32([1, 2]), i32([3, 4]), i32(range(5, 52))
        pool, left = torch.arange(52, 152, dtype=torch.int32, device=DEV), i32([60])
        pages = torch.zeros((200, binding.kv_page_bytes(2, 64, 64, "i8")), dtype=torch.uint8, device=DEV)
        a = binding.kv_tables(lens, want, table, pool, left, 64, 100)
        b = binding.kv_tables(lens.clone(), want, table.clone(), pool.clone(), left.clone(), 64, 9000, new_left=left.clone())
        binding.kv_write(x, x.flip(0), a[2][:92], pages, 64, "i8")
        ws = torch.empty((binding.kv_attention_workspace_bytes(4, 4, 2, 64),), dtype=torch.uint8, device=DEV)
        return [*a, *b, table, pool, left, pages, *binding.kv_read(pages, a[2], 2, 64, 64, "i8"), *binding.kv_read(pages, a[2], 2, 64, 64, "i8", torch.float32),
                binding.kv_attention(q, pages, table, a[0], 2, 64, "i8", workspace=ws), binding.kv_attention(q, pages, table, a[0], 2, 64, "i8", scale=0.3, window=9)]

    taken = []
    names = ("kv_tables", "kv_write", "kv_read", "kv_attention")
    real = binding._kv_calls

    def spy(name):
        def call(*args):
            r = getattr(real, name)(*args)
            taken.append(r is not None)
            return r
        return call

    monkeypatch.setattr(binding, "_kv_calls", types.SimpleNamespace(**{n: spy(n) for n in names}))
    a = calls()
    assert taken and all(taken)
    monkeypatch.setattr(binding, "_kv_calls", types.SimpleNamespace(**dict.fromkeys(names, lambda *args: None)))
    for x, y in zip(a, calls()):
        assert x.shape == y.shape and x.dtype == y.dtype and x.device == y.device and torch.equal(x, y)


def test_refusals():
    pages = empty_pages(3, 2, 32, 64, "bf16")
    x, q, table, lens = rows_of(1, 4, 2, 64, "bf16"), queries(2, 4, 64, "bf16"), i32([[0], [1]]), i32([3, 4])
    with pytest.raises(AssertionError):
        binding.kv_write(x, x.float(), i32(range(4)), pages, 32, "bf16")
    with pytest.raises(AssertionError):
        binding.kv_write(x, x, i32(range(4)), pages, 32, "i8")                       # pages of another type
    with pytest.raises(TypeError):
        binding.kv_write(x, x, torch.arange(4, device=DEV), pages, 32, "bf16")
    with pytest.raises(TypeError):
        binding.kv_write(x.half(), x.half(), i32(range(4)), pages, 32, "bf16")
    with pytest.raises(binding.SlideSparseError):
        binding.kv_write(x, x, i32(range(4)), pages, 16, "bf16")
    with pytest.raises(AssertionError):
        binding.kv_attention(q, pages, table[:1], lens, 2, 32, "bf16")
    with pytest.raises(TypeError):
        binding.kv_attention(q, pages, table.long(), lens, 2, 32, "bf16")
    with pytest.raises(binding.SlideSparseError):
        binding.kv_attention(q, pages, table, lens, 2, 32, "bf16", window=-1)
    with pytest.raises(binding.SlideSparseError):
        binding.kv_attention(q[:, :3], pages, table, lens, 2, 32, "bf16")
    with pytest.raises(AssertionError):
        binding.kv_attention(q, pages, table, lens, 2, 32, "bf16", out=torch.zeros((2, 4, 64), device=DEV))
    with pytest.raises(AssertionError):
        binding.kv_tables(lens, lens[:1], table, lens, lens[:1], 32, 4)
    with pytest.raises(TypeError):
        binding.kv_tables(lens, lens, table.float(), lens, lens[:1], 32, 4)
