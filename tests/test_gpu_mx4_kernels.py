"""Every kernel of the microscaled products by shapes that go there (tests/test_mx4_routes_host.py holds them to it), with and without a workspace, dense and grouped,
on operands whose sums are exact."""
import pytest

from test_gpu_mx4_exact import run_dense, run_grouped

pytestmark = pytest.mark.gpu

# rows of no multiple of a tile, channels of no multiple of a panel, rows of odd and even numbers of units, groups without a row; (rows, ..., kernel, ranges)
DENSE = [(117, 36798, 503, False, 32, 16), (94, 13944, 978, True, 32, 5), (82, 9776, 5766, False, 32, 2), (42, 16226, 6623, False, 32, 2),
         (182, 16037, 2337, False, 64, 4), (76, 15682, 3427, True, 64, 2), (3808, 7359, 107, False, 64, 4),
         (230, 13095, 4239, False, 128, 3), (1941, 22080, 130, True, 128, 5), (3653, 37267, 122, False, 128, 8)]
GROUPED = [(252, 3, 1920, 1578, True, "skewed", 32, 1), (508, 5, 4710, 1619, False, "even", 32, 1), (525, 1, 6666, 1797, False, "one", 32, 1), (1850, 16, 641, 202, True, "skewed", 32, 1),
           (73, 2, 38248, 1744, False, "even", 32, 6), (145, 4, 38056, 433, True, "skewed", 32, 6), (291, 8, 35269, 509, False, "skewed", 32, 5), (67, 1, 39507, 862, False, "one", 32, 12),
           (273, 4, 16691, 808, True, "even", 64, 3), (223, 1, 19014, 2513, False, "one", 64, 3),
           (990, 3, 6784, 3136, False, "skewed", 128, 1), (2046, 8, 1445, 666, True, "skewed", 128, 1), (600, 2, 537, 4699, False, "even", 128, 1), (2254, 1, 7345, 1721, False, "one", 128, 1),
           (2270, 3, 11098, 493, False, "skewed", 128, 3), (205, 2, 10856, 3901, False, "one", 128, 3), (846, 4, 20435, 591, True, "even", 128, 2), (1488, 1, 32801, 715, False, "one", 128, 3)]


@pytest.mark.parametrize("M,K,O,gated,rows,ranges", DENSE)
def test_dense(M, K, O, gated, rows, ranges):
    run_dense(M, K, O, gated)


@pytest.mark.parametrize("R,E,K,O,gated,kind,rows,ranges", GROUPED)
def test_grouped(R, E, K, O, gated, kind, rows, ranges):
    run_grouped(R, E, K, O, gated, kind)
