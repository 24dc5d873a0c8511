"""kv_attention over values at the ends of their ranges, against closed forms and the oracle."""
import numpy as np
import pytest
import torch

from oracle import kv_oracle as ko
from paper_2603_05232_amd import binding
from test_gpu_kv import DEV, Cache, i32, queries

pytestmark = pytest.mark.gpu


def rewrite(cache, K, V):
    """Other keys and values into the slots of a cache's tokens."""
    t = np.concatenate([np.arange(n) for n in cache.lens])
    b = np.repeat(np.arange(len(cache.lens)), cache.lens)
    binding.kv_write(K.to(DEV), V.to(DEV), i32(cache.table[b, t // cache.page] * cache.page + t % cache.page), cache.pages, cache.page, cache.dtype)


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("D", [64, 200])
def test_scores_of_minus_infinity_over_values_that_are_no_numbers(dtype, D):
    """Every score of a request minus infinity: zeros, whatever its values are; of requests that are divided and that are not."""
    inf, nan = float("inf"), float("nan")
    lens = [40, 1, 5000, 300]
    cache = Cache(np.random.default_rng(5), lens, 1, D, 32, dtype)
    K, V = cache.K.clone(), cache.V.clone()
    K[:, 0, 0] = -inf
    K[-300:, 0, 0] = 1.0                                 # but for the last one's
    for at, x in ((3, inf), (40, nan), (41, -inf), (2000, nan), (5040, inf)):
        V[at, 0, 5], V[at, 0, D - 1] = x, x
    rewrite(cache, K, V)
    q = queries(4, 3, D, "bf16")
    q[:, :, 0] = 1.0
    for ws in (True, False):
        got = cache(q, ws=ws)
        assert bool((got[:3] == 0).all())
        assert bool(got[3].isfinite().all()) and bool((got[3] != 0).any())


@pytest.mark.parametrize("source", ["bf16", "fp32"])
@pytest.mark.parametrize("D", [64, 200])
@pytest.mark.parametrize("size", [1e-40, 1e-36, 1e-31, 1e36])
def test_queries_of_any_size_over_a_cache_in_half(size, D, source):
    """The scores are brought back by the scale, as far as there is one."""
    cache = Cache(np.random.default_rng(7), [100, 3], 1, D, 32, "fp16", size=0.1)
    q = queries(2, 3, D, source, size=size)
    scale = min(0.5 / size, 1e38)
    cache.check(cache(q, scale=scale), q, scale=float(np.float32(scale)))


@pytest.mark.parametrize("dtype", ["bf16", "fp16", "i8", "fp8"])
@pytest.mark.parametrize("size,scale", [(2.0 ** 100, 2.0 ** 28), (2.0 ** 120, -2.0 ** 126), (1.0, 2.0 ** 127)])
def test_keys_of_zeros_under_large_queries_and_scales(size, scale, dtype):
    """Every score is zero, however large what multiplies it: the mean of the values."""
    cache = Cache(np.random.default_rng(8), [100, 3, 700], 2, 64, 32, dtype)
    rewrite(cache, torch.zeros_like(cache.K), cache.V)
    cache.k = np.zeros_like(cache.k)
    q = queries(3, 4, 64, "bf16", size=size)
    cache.check(cache(q, scale=scale), q, scale=scale)


@pytest.mark.parametrize("D", [64, 200])
@pytest.mark.parametrize("dtype", ["bf16", "fp16", "i8", "fp8"])
def test_queries_of_32_bits_that_bf16_would_round_to_infinity(dtype, D):
    """Nearest to the largest numbers of 32 bits is no number of bf16: over keys of zeros, and over small ones."""
    cache = Cache(np.random.default_rng(9), [100, 3], 1, D, 32, dtype)
    K = torch.zeros_like(cache.K)
    if dtype == "bf16":                                            # products with codes of 8 bits are infinite, and half has no numbers as small
        K[:, :, 5] = 1e-30 * torch.randn(K.shape[:2], generator=torch.Generator().manual_seed(1))
    rewrite(cache, K, cache.V)
    cache.k = K.double().numpy()
    q = queries(2, 3, D, "fp32")
    q[:, 0, 5], q[:, 1, 5] = 3.4e38, -3.4028234e38
    cache.check(cache(q, scale=1e-8), q, scale=float(np.float32(1e-8)))
    q[0, 2, 7], q[1, 2, 7] = float("inf"), float("nan")            # these are not
    got = cache(q, scale=1e-8)
    assert bool(got[:, 2].isnan().all()) and bool(got[:, :2].isfinite().all())


@pytest.mark.parametrize("D", [64, 200])
@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
def test_keys_of_minus_infinity_under_queries_of_32_bits(dtype, D):
    """Scores of minus infinity, whatever pieces a query is multiplied in: one that a piece holds whole, one whose first piece is above it, one below."""
    lens = [40, 700, 33]
    cache = Cache(np.random.default_rng(10), lens, 1, D, 32, dtype, source="fp32")
    K = cache.K.clone()
    gone = torch.zeros(sum(lens), dtype=torch.bool)
    gone[[0, 7, 39, 41, 300, 739]] = True
    gone[740:] = True                                              # all of the last one's
    K[gone, 0, 0] = float("-inf")
    rewrite(cache, K, cache.V)
    q = queries(3, 3, D, "fp32")
    q[:, :, 0] = torch.tensor([1.0, 1.0 + 2.0 ** -7 - 2.0 ** -12, 1.0 + 2.0 ** -12], device=DEV)
    cache.k[gone.numpy(), 0, 0] = 0.0                              # not seen by the oracle
    starts = cache.starts
    cache.check(cache(q), q, seen=lambda b, t: ~gone.numpy()[starts[b] + t])


@pytest.mark.parametrize("D", [64, 200])
@pytest.mark.parametrize("source", ["bf16", "fp32"])
@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
def test_values_of_infinity(dtype, source, D):
    """An infinity among the values that are seen makes its channel that infinity, two of them a NaN, and no other channel anything."""
    lens = [1, 40, 3000]
    cache = Cache(np.random.default_rng(11), lens, 1, D, 32, dtype)
    inf = float("inf")
    V = cache.V.clone()
    V[0, 0, 3], V[5, 0, 9], V[30, 0, D - 1], V[100, 0, 20], V[101, 0, 20], V[2900, 0, 21], V[2901, 0, 21] = inf, -inf, inf, inf, -inf, inf, inf
    rewrite(cache, cache.K, V)
    q = queries(3, 3, D, source, size=0.3)
    for ws in (True, False):
        got = cache(q, ws=ws)
        assert bool((got[0, :, 3] == inf).all()) and bool((got[1, :, 9] == -inf).all()) and bool((got[1, :, D - 1] == inf).all())
        assert bool(got[2, :, 20].isnan().all()) and bool((got[2, :, 21] == inf).all())
        odd = torch.zeros((3, D), dtype=torch.bool, device=DEV)
        odd[0, 3] = odd[1, 9] = odd[1, D - 1] = odd[2, 20] = odd[2, 21] = True
        assert bool(got.isfinite().eq(~odd[:, None]).all())
        plain = Cache.__new__(Cache)
        vars(plain).update(vars(cache))
        rewrite(plain, cache.K, cache.V)
        cache.check(torch.where(odd[:, None], plain(q, ws=ws), got), q)
        rewrite(cache, cache.K, V)


@pytest.mark.parametrize("source", ["bf16", "fp32"])
@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
def test_probabilities_where_values_cancel(dtype, source):
    """Two groups of tokens, of one probability each, whose values nearly cancel: a probability that is rounded stands out.  Two pieces of a probability are within
    2^-16 of it (bf16: 2^-9 of a unit of 2^-7) or 2^-22 (half: 2^-12 of 2^-10); of the rest as oracle.kv_oracle.bound counts it."""
    rng = np.random.default_rng(12)
    few = rng.integers(2, 8, 40)
    many = few + rng.integers(1, 8, 40)
    lens = [int(n) for n in few + many]
    cache = Cache(rng, lens, 1, 32, 32, dtype)
    K, V = torch.zeros_like(cache.K), torch.ones_like(cache.V)
    for b, (n, m) in enumerate(zip(few, many)):
        rows = slice(cache.starts[b] + int(n), cache.starts[b + 1])
        K[rows, 0, 0] = float(np.log(n / m))                       # their probability, about n / m of the others'
        V[rows] = -1.0
    rewrite(cache, K, V)
    q = torch.zeros((40, 3, 32), device=DEV)
    q[:, :, 0] = torch.tensor([1.0, 1.0078125, 0.9921875])
    got = cache(q.bfloat16() if source == "bf16" else q, scale=1.0).double().cpu().numpy()
    k, v = ko.held(K.float().numpy(), dtype), ko.held(V.float().numpy(), dtype)
    for b in range(40):
        rows = slice(cache.starts[b], cache.starts[b + 1])
        out, share, sums, spread, floor = ko.attention(q[b].double().cpu().numpy(), k[rows], v[rows], 1.0, np.ones(lens[b], bool))
        delta = sums * (32 + 8) * 2.0 ** -24 + 4 * spread * 1.4427 * 2.0 ** -24
        rel = 2 * np.expm1(delta) + 2.0 ** (-16 if dtype == "bf16" else -22) + 2.0 ** -20 + (lens[b] + 64) * 2.0 ** -24
        assert (np.abs(got[b] - out) <= 2.0 ** -8 * np.abs(out) + share * rel[:, None]).all(), b


@pytest.mark.parametrize("source", ["bf16", "fp32"])
@pytest.mark.parametrize("dtype", ["i8", "fp8"])
def test_rows_of_the_largest_numbers(dtype, source):
    """Scales whose inverses are below the normal numbers of 32 bits, or nearly."""
    g = torch.Generator().manual_seed(2)
    x = torch.rand((64, 2, 48), generator=g) * 2 - 1
    x[:, :, 7] = 1.0
    x *= torch.tensor([3.3e38, 8.6e37, 8.4e37, 4.3e37, 2e36, 1e-29, 1.6e-30, 8e-31])[torch.arange(64) % 8][:, None, None]
    x = x.to(torch.bfloat16 if source == "bf16" else torch.float32)
    pages = torch.zeros((2, binding.kv_page_bytes(2, 32, 48, dtype)), dtype=torch.uint8, device=DEV)
    slots = i32(range(64))
    binding.kv_write(x.to(DEV), x.flip(0).to(DEV), slots, pages, 32, dtype)
    k, v = binding.kv_read(pages, slots, 2, 48, 32, dtype, torch.float32)
    assert np.array_equal(k.cpu().numpy(), ko.held(x.float().numpy(), dtype)) and np.array_equal(v.cpu().numpy(), ko.held(x.flip(0).float().numpy(), dtype))


@pytest.mark.parametrize("source", ["bf16", "fp32"])
@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
def test_values_of_infinity_under_any_probability(dtype, source):
    """Two tokens to a request, the second one less likely by anything down to 2^-36 and of infinite values."""
    B = 2000
    cache = Cache(np.random.default_rng(13), [2] * B, 1, 32, 32, dtype)
    K, V = torch.zeros_like(cache.K), torch.ones_like(cache.V)
    K[1::2, 0, 0] = -torch.rand((B,), generator=torch.Generator().manual_seed(3)).to(K.dtype) * 25
    V[1::2, 0, 4], V[1::2, 0, 5] = float("inf"), float("-inf")
    rewrite(cache, K, V)
    q = torch.zeros((B, 2, 32), device=DEV)
    q[:, :, 0] = torch.rand((B, 2), generator=torch.Generator().manual_seed(4)).to(DEV) * 0.1 + 0.9
    got = cache(q.bfloat16() if source == "bf16" else q, scale=1.0)
    assert bool((got[:, :, 4] == float("inf")).all()) and bool((got[:, :, 5] == float("-inf")).all()) and bool((got[:, :, :4] == 1).all())


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
def test_keys_of_minus_infinity_under_any_query_of_32_bits(dtype):
    """One of two tokens is not seen for its score, whatever the query's value there, down to 2^-35 of the largest."""
    B = 2000
    cache = Cache(np.random.default_rng(14), [2] * B, 1, 32, 32, dtype)
    K, V = torch.zeros_like(cache.K), torch.ones_like(cache.V)
    K[1::2, 0, 0], V[1::2] = float("-inf"), 3.0
    rewrite(cache, K, V)
    g = torch.Generator().manual_seed(5)
    q = torch.rand((B, 2, 32), generator=g)
    q[:, :, 0] = torch.exp2(-torch.randint(0, 35, (B, 2), generator=g).float()) * (1 + torch.randint(0, 3, (B, 2), generator=g) * 2.0 ** -23)
    q[:, :, 1] = 1.0
    assert bool((cache(q.to(DEV)) == 1).all())
