"""The low-bit serving operators from their definitions, in 64 bits on the CPU (test infrastructure only)."""
import math

import numpy as np

GROUP, TILE, BLOCK = 32, 16, 128


def e4m3(x):
    """Rounded to 3 fraction bits from 2^-6 on and to steps of 2^-9 below, ties to even; |x| <= 448."""
    e = np.floor(np.log2(np.maximum(np.abs(x), 2.0 ** -6)))
    u = np.exp2(e - 3)
    return np.rint(x / u) * u


def f8_cast(x, rows):
    """(codes as values, scales) of x [m, k] with a scale for each rows x 128 block."""
    x = np.asarray(x, np.float64)
    m, k = x.shape
    mb, kb = -(-m // rows), -(-k // BLOCK)
    scale = np.zeros((mb, kb))
    q = np.zeros_like(x)
    for i in range(mb):
        for j in range(kb):
            b = x[i * rows:(i + 1) * rows, j * BLOCK:(j + 1) * BLOCK]
            top = np.abs(b).max()
            e = max(-126, math.ceil(math.log2(top / 448))) if top > 0 else -126
            scale[i, j] = 2.0 ** e
            q[i * rows:(i + 1) * rows, j * BLOCK:(j + 1) * BLOCK] = e4m3(b / scale[i, j])
    return q, scale


def f8_values(q, scale, rows):
    m, k = q.shape
    return q * np.repeat(np.repeat(scale, rows, 0)[:m], BLOCK, 1)[:, :k]


def grid4(x):
    """(codes, steps, zero codes) of x [..., dim]: a min-max grid with 0 in its range for every 32 values."""
    y = np.asarray(x, np.float64).reshape(*x.shape[:-1], -1, GROUP)
    lo, hi = np.minimum(y.min(-1), 0), np.maximum(y.max(-1), 0)
    r = np.minimum((hi - lo) / 15, 2112.0)
    unit = np.exp2(np.floor(np.log2(np.maximum(r, 2.0 ** -14))) - 5)
    s = np.maximum(np.ceil(r / unit) * unit, 2.0 ** -19)
    z = np.clip(np.rint(-lo / s), 0, 15)
    c = np.clip(np.rint(y / s[..., None]) + z[..., None], 0, 15)
    return c.reshape(x.shape), s, z


def held4(x):
    c, s, z = grid4(x)
    g = c.reshape(*x.shape[:-1], -1, GROUP)
    return (s[..., None] * (g - z[..., None])).reshape(x.shape)


def tile_bytes(dim):
    return 2 * TILE * (dim // 2 + dim // GROUP * 2)


def pages_from(k, v):
    """[pages, heads, page, dim] values to the bytes of the cache [pages, heads, page / 16, bytes of a tile]."""
    p, h, n, dim = k.shape
    sides = []
    for x in (k, v):
        c, s, z = grid4(x)
        c = c.astype(np.uint8).reshape(p, h, n // TILE, TILE, dim)
        packed = (c[..., 0::2] | (c[..., 1::2] << 4)).reshape(p, h, n // TILE, -1)
        w = s.astype(np.float16).view(np.uint16) | z.astype(np.uint16)
        w = np.ascontiguousarray(w).view(np.uint8).reshape(p, h, n // TILE, -1)
        sides += [packed, w]
    return np.concatenate(sides, -1)


def plan(lens, new, table, free, page):
    """(table, slots, positions, cu, lens, taken) with the new tokens of every request placed."""
    table, slots, positions, cu, taken = table.copy(), [], [], [0], 0
    for b, (x, y) in enumerate(zip(lens, new)):
        for p in range(-(-x // page), -(-(x + y) // page)):
            table[b, p] = free[taken]
            taken += 1
        for p in range(x, x + y):
            slots.append(int(table[b, p // page]) * page + p % page)
            positions.append(p)
        cu.append(cu[-1] + y)
    return table, slots, positions, cu, [x + y for x, y in zip(lens, new)], taken


def attention(q, keys, values, length, scale, causal, window):
    """One request: q [n, heads, dim], keys and values [length, kv_heads, dim] -> (out, lse, what the tolerances need)."""
    n, heads, dim = q.shape
    ratio = heads // keys.shape[1]
    out, lse = np.zeros((n, heads, dim)), np.full((n, heads), -np.inf)
    mass, reach = np.zeros((n, heads, dim)), np.zeros((n, heads))
    j = np.arange(length)
    for i in range(n):
        p = length - n + i
        see = np.ones(length, bool)
        if causal:
            see &= j <= p
        if window > 0:
            see &= j > p - window
        if not see.any():
            continue
        for h in range(heads):
            k, v = keys[see, h // ratio], values[see, h // ratio]
            x = (k @ q[i, h]) * scale
            top = x.max()
            e = np.exp(x - top)
            lse[i, h] = top + np.log(e.sum())
            pr = e / e.sum()
            out[i, h] = pr @ v
            mass[i, h] = pr @ np.abs(v)                       # sum p |v|
            reach[i, h] = (np.abs(k) @ np.abs(q[i, h])).max() * abs(scale)
    return out, lse, mass, reach
