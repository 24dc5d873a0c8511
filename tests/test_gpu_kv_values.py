"""kv_attention over values at the ends of their ranges, against closed forms and the oracle."""
import numpy as np
import pytest
import torch

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
