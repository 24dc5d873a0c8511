"""CPU reference of the operators on a paged cache of keys and values (numpy, 64 bits), written from the definitions in include/slidesparse.h; shares no code with the HIP path."""
from __future__ import annotations

import numpy as np

LARGEST = {"i8": 127.0, "fp8": 448.0}


def tables(lens, want, table, page, pool, left, N):
    """One request after the other -> new lens, left, slots[N], offsets[B + 1], table, pool."""
    lens, want, table, pool = ([int(x) for x in lens], [int(x) for x in want], np.array(table), list(map(int, pool)))
    B, W = table.shape
    P = len(pool)
    lens = [min(max(n, 0), W * page) for n in lens]
    want = [max(n, 0) for n in want]
    have, need = [-(-n // page) for n in lens], [-(-n // page) for n in want]
    top = min(max(int(left), 0), P)
    for b in range(B):
        if want[b] < lens[b]:
            for i in range(need[b], have[b]):
                if top < P:
                    pool[top] = int(table[b, i])
                    top += 1
    new_lens, slots, offsets, asked, row, taken = [], [-1] * N, [0], 0, 0, 0
    for b in range(B):
        if want[b] <= lens[b]:
            new_lens.append(want[b])
            offsets.append(min(row, N))
            continue
        rows = range(row, row + want[b] - lens[b])
        row = rows.stop
        offsets.append(min(row, N))
        possible = need[b] <= W and row <= N
        more = need[b] - have[b] if possible else 0
        asked += more
        if not possible or (more and asked > top):
            new_lens.append(lens[b])
            continue
        for i in range(more):
            table[b, have[b] + i] = pool[top - 1 - (asked - more) - i]
        if more:
            taken = asked
        for i, t in zip(rows, range(lens[b], want[b])):
            page_id = int(table[b, t // page])
            slots[i] = page_id * page + t % page if 0 <= page_id < P else -1
        new_lens.append(want[b])
    return new_lens, top - taken, slots, offsets, table, pool


def e4m3(x):
    """Nearest value of the 8-bit format, ties to even; |x| <= 448."""
    x = np.asarray(x, np.float64)
    step = np.exp2(np.maximum(np.frexp(x)[1], -5).astype(np.float64) - 4)
    return np.rint(x / step) * step


def bf16(x):
    """fp32 values rounded to nearest even, as fp32."""
    u = np.ascontiguousarray(x, np.float32).view(np.uint32).astype(np.uint64)
    bad = (u & 0x7FFFFFFF) > 0x7F800000
    u = np.where(bad, 0x7FC00000, (u + 0x7FFF + (u >> 16 & 1)) & 0xFFFF0000)
    return u.astype(np.uint32).view(np.float32)


def held(x, dtype):
    """x[..., D] fp32 -> what a cache of this type holds of it, fp32: rounded values, or codes times scales (in 32 bits, as kv_read gives them)."""
    x = np.asarray(x, np.float32)
    if dtype == "bf16":
        return bf16(x)
    if dtype == "fp16":
        with np.errstate(over="ignore"):
            return x.astype(np.float16).astype(np.float32)
    q = np.float32(LARGEST[dtype])
    with np.errstate(invalid="ignore", divide="ignore", over="ignore"):
        a = np.abs(x).max(-1, keepdims=True)
        bad, none = ~np.isfinite(a), a < np.float32(2.0 ** -100)
        a = np.where(bad | none, np.float32(1), a)
        y = np.clip(x * (q * (np.float32(1) / a)), -q, q)
        codes = np.rint(y) if dtype == "i8" else e4m3(y)
        codes = np.where(bad | none, 0, codes).astype(np.float32)
        scale = np.where(bad, np.float32(np.nan), np.where(none, np.float32(1), a / q))
        return (codes * scale).astype(np.float32)


def attention(q, k, v, scale, seen):
    """q[Hq,D], k and v [T,H,D], seen[T] -> out[Hq,D] and what bound() takes; nothing seen or all scores minus infinity: zeros."""
    q, k, v = np.asarray(q, np.float64), np.asarray(k, np.float64)[seen], np.asarray(v, np.float64)[seen]
    Hq, D = q.shape
    out, share = np.zeros((Hq, D)), np.zeros((Hq, D))
    if k.shape[0] == 0:
        return out, share, np.zeros(Hq), np.zeros(Hq), np.zeros(Hq)
    G = Hq // k.shape[1]
    sums, spread, floor = np.zeros(Hq), np.zeros(Hq), np.zeros(Hq)
    for h in range(Hq):
        kh, vh = k[:, h // G], v[:, h // G]
        with np.errstate(invalid="ignore"):
            s = (kh * q[h]).sum(-1) * scale
            top = s.max() if np.isnan(s).any() else max(s.max(), -np.inf)
            if top == -np.inf:
                continue
            p = np.exp(s - top)
            out[h] = (p[:, None] * vh).sum(0) / p.sum()
            share[h] = (p[:, None] * np.abs(vh)).sum(0) / p.sum()
            sums[h] = (np.abs(kh) * np.abs(q[h])).sum(-1).max() * abs(scale)
            floor[h] = np.abs(kh).sum(-1).max() * np.abs(q[h]).max() * abs(scale)
            spread[h] = np.abs(s - top).max() + np.abs(s).max()
    return out, share, sums, spread, floor


def bound(out, share, sums, spread, floor, D, T, dtype, fp32_q):
    """How far the kernel's bf16 result may be off.  Score: D + 8 roundings of 2^-24 of the sum of magnitudes; a query of 32 bits as two bf16 pieces 2^-16 of it, as two half pieces 2^-22; in
    half, values far below the head's largest 2^-24 of that one; the argument of the exponential 4 roundings of its size; e^delta - 1 counts twice (numerator and denominator).
    Probabilities 2^-16 (two bf16 pieces) or 2^-22 (two half pieces), exponential, scales and weights of parts 2^-20 in all; sums over T tokens T + 64 roundings of 2^-24.  The result 2^-8 of itself."""
    half = dtype == "fp16"
    delta = sums * ((D + 8) * 2.0 ** -24 + ((2.0 ** -22 if half else 2.0 ** -16) if fp32_q else 0.0)) + (2.0 ** -24 * floor if half else 0.0) + 4 * spread * 1.4427 * 2.0 ** -24
    rel = 2 * np.expm1(delta) + (2.0 ** -22 if half else 2.0 ** -16) + 2.0 ** -20 + (T + 64) * 2.0 ** -24
    return 2.0 ** -8 * np.abs(out) + share * rel[:, None] + 1e-37
