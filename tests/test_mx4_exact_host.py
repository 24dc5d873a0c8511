"""What the exactly summable operands tell apart on the longest rows, by the oracle on the CPU."""
import pytest
import torch

import mx4_exact as ex

K = 18944


@pytest.mark.parametrize("fault", ["block", "unit", "scale"])
def test_a_fault_in_a_row_shows(fault):
    """A mistake of one block of 32 values, a unit of 256 or a scale byte of one block shows in most results of the row; in none without one."""
    g = torch.Generator().manual_seed(1)
    (xc, xs), wc = ex.operand(g, 16, K), ex.operand(g, 64, K)
    x, w = ex.values(xc, xs), ex.values(*wc)
    assert ex.sums_are_exact(x, w)
    assert torch.equal((x.float() @ w.float().t()).double(), x @ w.t())          # in 32 bits as well
    Y = (x @ w.t()).float().to(torch.bfloat16)
    assert not bool(ex.wrong(Y, x @ w.t()).any())
    for row in range(16):
        bc, bs = xc.clone(), xs.clone()
        if fault == "block":
            bc[row, 16 * 36 * (row + 1):][:16] = 0
        elif fault == "unit":
            bc[row, 128 * 4 * (row + 1):][:128] = 0
        else:
            bs[4 * (row + 1), row, 3] += 1
        bad = ex.wrong((ex.values(bc, bs) @ w.t()).float().to(torch.bfloat16), x @ w.t())
        assert float(bad[row].double().mean()) > 0.75 and not bool(bad[torch.arange(16) != row].any()), (row, float(bad[row].double().mean()))


def test_a_fault_in_a_gated_row_shows():
    g = torch.Generator().manual_seed(2)
    (xc, xs), wc = ex.operand(g, 16, K, 123), ex.operand(g, 128, K, 123)
    x, w = ex.values(xc, xs), ex.values(*wc)
    assert ex.sums_are_exact(x, w, 123, 123)
    gate, up = (x @ w.t()).chunk(2, dim=1)

    def answer(x):
        a, b = (x @ w.t()).float().chunk(2, dim=1)
        return (a / (1 + torch.exp(-a)) * b).to(torch.bfloat16)

    assert not bool(ex.wrong_gated(answer(x), gate, up).any())
    xc[:, 16 * 37:][:, :16] = 0
    assert float(ex.wrong_gated(answer(ex.values(xc, xs)), gate, up).double().mean()) > 0.75
