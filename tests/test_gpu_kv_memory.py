"""kv_tables where its results lie in the memory of its inputs."""
import numpy as np
import pytest
import torch

from oracle import kv_oracle as ko
from paper_2603_05232_amd import binding
from test_gpu_kv import DEV, i32, step_of

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("B", [40, 1024, 1500])
@pytest.mark.parametrize("rows", ["few", "many"])
@pytest.mark.parametrize("where", ["want", "behind lens", "before lens", "behind want", "left in lens"])
def test_results_in_the_memory_of_inputs(where, rows, B):
    """Requests that find no room keep their lengths, so that what is wanted and what comes to be differ; any number of rows, which decides by how many launches they are filled in."""
    rng = np.random.default_rng(B)
    W, page = 16, 64
    lens, want, table, pool, left = step_of(rng, B, W, page, "any")
    left = min(left, B)                                            # too few pages
    total = sum(max(0, w - n) for w, n in zip(want, lens))
    N = 1500 if rows == "few" else total - total // 8              # and too few rows
    assert rows == "few" or N > 2048
    ref = ko.tables(lens, want, table, page, pool, left, N)
    assert ref[0] != want
    both = torch.zeros((2 * B + 14,), dtype=torch.int32, device=DEV)
    l, w = both[7:7 + B], both[7 + B:7 + 2 * B]
    l.copy_(i32(lens))
    w.copy_(i32(want))
    f = i32([left])
    if where == "left in lens":                                    # the free pages' number in the memory of a length
        new = dict(new_left=both[7 + B // 2:8 + B // 2])
    else:
        at = {"want": 7 + B, "behind lens": 12, "before lens": 2, "behind want": 14 + B}[where]
        new = dict(new_lens=both[at:at + B])
    t, p = i32(table), i32(pool)
    got = binding.kv_tables(l, w, t, p, f, page, N, **new)
    for name, a, b in zip(("lens", "left", "slots", "offsets", "table", "pool"), (*got, t, p), (ref[0], [ref[1]], ref[2], ref[3], ref[4], ref[5])):
        assert a.cpu().numpy().tolist() == np.asarray(b).tolist(), name
