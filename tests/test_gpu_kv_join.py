"""kv_attention of requests in so many parts that their join takes several rounds."""
import numpy as np
import pytest
import torch

from oracle import kv_oracle as ko
from test_gpu_kv import Cache, queries
from test_gpu_kv_replay import parts, plan
from test_gpu_kv_values import rewrite

pytestmark = pytest.mark.gpu


def round_of(D, rows):
    """Parts that a workgroup takes at once: 8 to a row of its threads, 8 lanes to 32 values; few rows of results are cut into slices of 32 values."""
    cus = torch.cuda.get_device_properties(0).multi_processor_count
    steps = -(-D // 32)
    threads, slices = (512, 1) if rows * steps <= cus else (512, steps) if rows <= 2 * cus else (128, steps)
    return threads // (8 * slices) * 8


@pytest.mark.parametrize("where", ["first round", "a round in the middle", "last round"])
@pytest.mark.parametrize("D,Hq,H,B,long_one,dtype", [(256, 32, 8, 64, 30000, "bf16"), (128, 8, 4, 65, 24000, "fp8"), (128, 9, 1, 60, 24000, "fp16"), (192, 10, 2, 60, 20000, "i8"),
                                                     (96, 12, 2, 50, 24000, "bf16"), (64, 20, 1, 30, 24000, "bf16"), (128, 16, 1, 8, 40000, "bf16"), (96, 6, 1, 50, 50000, "fp8"),
                                                     (256, 8, 1, 2, 95000, "fp16")])
def test_many_parts_of_one_request(D, Hq, H, B, long_one, dtype, where):
    """One long request among short ones.  Its largest scores lie in one round, and the tokens of another are not seen at all: their pages are none."""
    rng = np.random.default_rng(D + B)
    groups = (3 if D > 192 else 2) * torch.cuda.get_device_properties(0).multi_processor_count // (H * -(-Hq // H // 16))
    lens = [int(n) for n in rng.integers(0, 40, B)]
    long, room = B // 2, round_of(D, B * Hq)
    lens[long] = long_one
    divided = parts(lens, groups)
    n = divided[long]
    assert n > room, (n, room)
    cache = Cache(rng, lens, H, D, 64, dtype)
    each = -(-(-(-lens[long] // 32)) // n) * 32                    # tokens of a part
    rounds = -(-n // room)
    at = {"first round": 0, "a round in the middle": rounds // 2, "last round": rounds - 1}[where]
    q = queries(B, Hq, D, "bf16", size=0.3)
    # keys along one query of each head, so that the scores there stand out
    K, first = cache.K.clone(), cache.starts[long]
    G = Hq // H
    special = first + min(at * room * each + each // 2, lens[long] - 1)
    for h in range(H):
        K[special, h] = (2.0 * q[long, h * G].cpu().float()).to(K.dtype)
    rewrite(cache, K, cache.V)
    cache.k = ko.held(K.float().numpy(), dtype)
    hidden = (at + 1) % rounds                                     # a round without a token to see
    lo, hi = hidden * room * each // 64, min((hidden + 1) * room * each, lens[long]) // 64
    columns = [c for c in range(lo, max(hi, lo + 1)) if c != (special - first) // 64]
    cache.table[long, columns] = -1
    got = cache(q)
    assert [p for _, p in plan(cache.scratch, B)] == divided
    cache.check(got, q, seen=lambda b, t: ~np.isin(t // 64, columns) if b == long else np.ones(t.shape, bool))
    assert torch.equal(got, cache(q))
