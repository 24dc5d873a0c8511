"""CPU reference of the microscaled 4-bit operators and of the expert layer's choice and sum (numpy, 64 bits), written from the definitions in
include/slidesparse.h; shares no code with the HIP path."""
from __future__ import annotations

import numpy as np

GRID = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


def quant(X):
    """X[R,K] float -> codes[R,U,256] (one per value), scale bytes [R,U,8]."""
    X = np.asarray(X, np.float64)
    R, K = X.shape
    U = -(-K // 256)
    x = np.zeros((R, U * 256))
    x[:, :K] = X
    sign = np.zeros(x.shape, bool)
    sign[:, :K] = np.signbit(X)
    x, sign = x.reshape(R, U * 8, 32), sign.reshape(R, U * 8, 32)
    bad = ~np.isfinite(x).all(-1)
    a = np.abs(np.where(bad[..., None], 0.0, x))
    top = np.frexp(a.max(-1))[1] - 1                           # floor(log2), of zero anything
    b = np.where(a.max(-1) > 0, np.maximum(top - 2 + 127, 0), 0)
    v = np.ldexp(a, (127 - b)[..., None])
    code = np.zeros(v.shape, np.int64)
    for i in range(1, 8):                                      # nearest, ties to the even code
        mid = (GRID[i - 1] + GRID[i]) / 2
        code += (v > mid) | ((v == mid) & (i % 2 == 0))
    code += 8 * sign
    code[bad] = 0
    b = np.where(bad, 255, b)
    return code.reshape(R, U, 256).astype(np.uint8), b.reshape(R, U, 8).astype(np.uint8)


def values(code, b):
    """[R, 256 U] of codes[R,U,256] and scale bytes [R,U,8]."""
    v = np.where(code >= 8, -1.0, 1.0) * GRID[code & 7]
    s = np.where(b == 255, np.nan, np.ldexp(1.0, b.astype(np.int64) - 127))
    return (v.reshape(*b.shape, 32) * s[..., None]).reshape(code.shape[0], -1)


def pack_codes(code):
    """[R,U,256] -> bytes [R, 128 U], the even value in the low half."""
    return (code[..., 0::2] | (code[..., 1::2] << 4)).reshape(code.shape[0], -1).astype(np.uint8)


def product(xv, wv, gated=False):
    """(Y, bound of what 32-bit sums of exact products may be off) of values xv[R,K], wv[rows,K]; gated: wv = gate's rows, then up's."""
    y, size = xv @ wv.T, np.abs(xv) @ np.abs(wv).T
    off = xv.shape[1] * 2.0 ** -23 * size
    if not gated:
        return y, off
    n = wv.shape[0] // 2
    g, u, eg, eu = y[:, :n], y[:, n:], off[:, :n], off[:, n:]
    with np.errstate(over="ignore"):
        silu = g / (1 + np.exp(-g))
    return silu * u, 1.1 * eg * (np.abs(u) + eu) + np.abs(silu) * eu + 2.0 ** -20 * np.abs(silu * u)      # |silu'| < 1.1


def route(x, k, renormalise=True):
    """ids, weights, slots, rows, offsets of scores x[M,E]."""
    x = np.asarray(x, np.float64)
    M, E = x.shape
    ids = np.empty((M, k), np.int64)
    weights = np.zeros((M, k))
    for m in range(M):
        order = sorted(range(E), key=lambda e: (np.isnan(x[m, e]), 0.0 if np.isnan(x[m, e]) else -x[m, e], e))
        ids[m] = order[:k]
        top = x[m, order[0]]
        if top == -np.inf:
            continue
        p = np.exp(x[m] - top)
        weights[m] = p[ids[m]] / (p[ids[m]].sum() if renormalise else p.sum())
    by_expert = sorted(range(M * k), key=lambda i: (ids.flat[i], i))
    slots = np.empty(M * k, np.int64)
    slots[by_expert] = np.arange(M * k)
    offsets = np.concatenate([[0], np.cumsum(np.bincount(ids.ravel(), minlength=E))])
    return ids, weights, slots.reshape(M, k), np.array(by_expert, np.int64) // k, offsets


def combine(Y, slots, weights, base=None):
    """(sum, bound of what 32-bit sums may be off)."""
    M, k = slots.shape
    out, size = np.zeros((M, Y.shape[1])), np.zeros((M, Y.shape[1]))
    for j in range(k):
        there = (slots[:, j] >= 0) & (slots[:, j] < Y.shape[0])
        t = np.where(there[:, None], weights[:, j, None] * Y[np.where(there, slots[:, j], 0)], 0.0)
        out, size = out + t, size + np.abs(t)
    if base is not None:
        out, size = out + base, size + np.abs(base)
    return out, (k + 1) * 2.0 ** -23 * size
