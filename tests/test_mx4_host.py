"""The 4-bit operators' sizes and refusals (no GPU), and the oracle against closed forms."""
import ctypes

import numpy as np
import pytest

from oracle import mx4_oracle as mo
from paper_2603_05232_amd import binding

ONE, ODD = ctypes.c_void_p(16), ctypes.c_void_p(17)          # never dereferenced: validation fails first


@pytest.fixture(scope="module")
def lib():
    return binding.load()


def test_sizes():
    assert [binding.mx4_row_bytes(k) for k in (1, 256, 257, 3584)] == [128, 128, 256, 14 * 128]
    assert binding.mx4_row_bytes(0) == binding.mx4_row_scales((1 << 24) + 1) == -1
    assert binding.mx4_row_scales(5003) == 20 * 8
    assert binding.mx4_packed_sizes(33, 300) == (2 * 2 * 4096, 2 * 2 * 256)                      # fragments of 32 channels, units of 256 values
    assert binding.mx4_packed_sizes(33, 300, experts=5, gated=True) == (5 * 3 * 2 * 4096, 5 * 3 * 2 * 256)
    assert binding.expert_route_workspace_bytes(64, 8, 2) == 0 and binding.expert_route_workspace_bytes(65, 8, 2) > 0
    assert binding.expert_route_workspace_bytes(65, 8, 9) == 0


def test_refusals(lib):
    q = lambda *a: lib.mx4_quant(*a, None)  # noqa: E731
    assert q(ONE, 2, 4, 64, 64, None, 4, ONE, ONE) == 4                                           # type
    assert q(ONE, 0, 4, 64, 63, None, 4, ONE, ONE) == 3 and q(ONE, 0, 4, 0, 64, None, 4, ONE, ONE) == 3
    assert q(ONE, 0, 4, 64, 64, None, 5, ONE, ONE) == 3                                           # other rows without a list of them
    assert q(ODD, 1, 4, 64, 64, None, 4, ONE, ONE) == 3 and q(ONE, 1, 4, 64, 64, None, 4, ONE, ctypes.c_void_p(8)) == 3
    assert q(None, 1, 4, 64, 64, None, 4, ONE, ONE) == 1 and q(ONE, 1, 4, 64, 64, None, 4, None, ONE) == 1
    assert q(None, 1, 0, 64, 64, None, 0, None, None) == 0                                        # nothing to do
    d = lambda *a: lib.mx4_dequant(*a, None)  # noqa: E731
    assert d(ONE, ONE, 4, 64, 3, ONE, 64) == 4 and d(ONE, ONE, 4, 64, 0, ONE, 63) == 3 and d(ONE, ONE, 4, 64, 0, None, 64) == 1
    p = lambda *a: lib.mx4_pack(*a, None)  # noqa: E731
    assert p(ONE, ONE, 0, 64, 64, 0, ONE, ONE) == 3 and p(ONE, ONE, 1025, 64, 64, 0, ONE, ONE) == 3 and p(ONE, ONE, 1, 64, 64, 2, ONE, ONE) == 3
    assert p(ONE, None, 1, 64, 64, 0, ONE, ONE) == 1 and p(ONE, ONE, 1, 64, 64, 0, ctypes.c_void_p(8), ONE) == 3
    g = lambda *a: lib.mx4_gemm(ONE, ONE, ONE, ONE, *a, None)  # noqa: E731
    assert g(4, 64, 64, 0, ONE, 63, None, 0) == 3 and g(4, 64, 0, 0, ONE, 64, None, 0) == 3 and g(4, 64, 64, 3, ONE, 64, None, 0) == 3
    assert g(4, 64, 64, 0, None, 64, None, 0) == 1 and g(4, 64, 64, 0, ODD, 64, None, 0) == 3
    assert g(4, 64, 64, 0, ONE, 64, None, 16) == 1 and g(4, 64, 64, 0, ONE, 64, ctypes.c_void_p(24), 64) == 5
    assert g(4, 64, 64, 0, ONE, 1 << 22, None, 0) == 3 and g(0, 64, 64, 0, None, 64, None, 0) == 0
    assert lib.mx4_grouped_gemm(ONE, ONE, None, ONE, ONE, 4, 2, 64, 64, 0, ONE, 64, None, 0, None) == 1
    assert lib.mx4_grouped_gemm(ONE, ONE, ONE, ONE, ONE, 4, 1025, 64, 64, 0, ONE, 64, None, 0, None) == 3
    r = lambda *a: lib.expert_route(ONE, *a, ONE, ONE, ONE, ONE, ONE, None, 0, None)  # noqa: E731
    assert r(7, 4, 8, 8, 2, 1) == 4 and r(0, 4, 8, 7, 2, 1) == 3 and r(0, 4, 8, 8, 9, 1) == 3 and r(0, 4, 8, 8, 0, 1) == 3 and r(0, 4, 8, 8, 2, 2) == 3
    assert r(0, 65, 8, 8, 2, 1) == 1                                                              # needs a workspace
    assert lib.expert_route(ONE, 0, 65, 8, 8, 2, 1, ONE, ONE, ONE, ONE, ONE, ONE, 8, None) == 5   # and a large enough one
    c = lambda *a: lib.expert_combine(ONE, 8, 64, 64, ONE, ONE, *a, None)  # noqa: E731
    assert c(4, 0, None, 0, ONE, 64) == 3 and c(4, 65, None, 0, ONE, 64) == 3 and c(4, 2, ONE, 63, ONE, 64) == 3 and c(4, 2, None, 0, ONE, 63) == 3
    assert c(4, 2, None, 0, None, 64) == 1 and c(4, 2, None, 0, ODD, 64) == 3


def test_more_threads_than_a_grid_counts(lib):
    n = 1 << 24
    assert lib.mx4_quant(ONE, 0, n, n, n, None, n, ONE, ONE, None) == 3 and lib.mx4_quant(ONE, 1, n, 1 << 13, n, None, n, ONE, ONE, None) == 3
    assert lib.mx4_dequant(ONE, ONE, n, 1 << 13, 1, ONE, n, None) == 3
    assert lib.mx4_pack(ONE, ONE, 1024, 1 << 18, n, 0, ONE, ONE, None) == 3
    assert lib.expert_combine(ONE, 8, 1 << 12, 1 << 12, ONE, ONE, n, 2, None, 0, ONE, 1 << 12, None) == 3


def test_oracle_against_closed_forms():
    v = np.array([[0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 6.9, -0.2, -0.26, 4.0, 0.0]])
    code, b = mo.quant(v)
    assert b[0, 0, 0] == 127 and (b[0, 0, 1:] == 0).all()
    assert mo.values(code, b)[0, :12].tolist() == [0, 1, 1, 2, 2, 4, 4, 6, 0, -0.5, 4, 0]
    for e in (-120, -3, 0, 5, 100):                                                                # a power of two moves the scale alone
        c2, b2 = mo.quant(v * 2.0 ** e)
        assert (c2 == code).all() and b2[0, 0, 0] == 127 + e
    rng = np.random.default_rng(0)
    x = rng.standard_normal((5, 700))
    code, b = mo.quant(x)
    got = mo.values(code, b)[:, :700]
    scale = np.ldexp(1.0, np.repeat(b.reshape(5, -1).astype(int) - 127, 32, axis=1))[:, :700]
    cand = np.concatenate([mo.GRID, -mo.GRID])
    best = np.min(np.abs(x[..., None] - cand * scale[..., None]), axis=-1)
    assert np.array_equal(np.abs(got - x), best)                                                   # no other value is nearer
    code, b = mo.quant(np.array([[1.0, np.nan] + [1.0] * 40]))
    assert b[0, 0, 0] == 255 and (code[0, 0, :32] == 0).all() and b[0, 0, 1] != 255 and np.isnan(mo.values(code, b)[0, :32]).all()
    ids, w, slots, rows, off = mo.route(np.array([[1.0, 2.0, 2.0, np.nan], [-np.inf] * 4]), 2)
    assert ids.tolist() == [[1, 2], [0, 1]] and w.tolist() == [[0.5, 0.5], [0, 0]]
    assert off.tolist() == [0, 1, 3, 4, 4] and rows.tolist() == [1, 0, 1, 0] and slots.tolist() == [[1, 3], [0, 2]]
