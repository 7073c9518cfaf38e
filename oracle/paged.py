"""Rotary positions and the paged KV cache in fp64: the definitions of
include/sps.h, one position at a time where that is affordable."""
import numpy as np


def frequencies(rot, base=10000.0, factor=1.0, original_len=0, low_turns=1.0, high_turns=32.0):
    i = np.arange(rot // 2, dtype=np.float64)
    f = np.float64(np.float32(base)) ** (-2.0 * i / rot)
    factor = np.float64(np.float32(factor))
    if original_len > 0:
        g = np.clip((original_len * f / (2 * np.pi) - np.float64(np.float32(low_turns))) /
                    (np.float64(np.float32(high_turns)) - np.float64(np.float32(low_turns))), 0.0, 1.0)
        return f * (g + (1.0 - g) / factor)
    return f / factor


def pairs(rot, layout):
    i = np.arange(rot // 2)
    return (i, i + rot // 2) if layout == "half" else (2 * i, 2 * i + 1)


def rope(x, pos, rot, layout="half", amplitude=1.0, backward=False, **kw):
    """x [rows][heads][D] at integer positions pos [rows]."""
    x = np.asarray(x, np.float64)
    y = x.copy()
    t = np.asarray(pos, np.float64)[:, None] * frequencies(rot, **kw)
    A = np.float64(np.float32(amplitude))
    c, s = A * np.cos(t)[:, None], A * np.sin(t)[:, None]
    if backward:
        s = -s
    ia, ib = pairs(rot, layout)
    a, b = x[..., ia], x[..., ib]
    y[..., ia], y[..., ib] = a * c - b * s, a * s + b * c
    return y


def key_at(p, d, D):
    return ((p // 16 * (D // 32) + d // 32) * 64 + p % 16 + 16 * (d % 32 // 8)) * 8 + d % 8


def value_at(p, d, D):
    w = p % 32
    return ((p // 32 * (D // 16) + d // 16) * 64 + d % 16 + 16 * (w % 16 // 4)) * 8 + 4 * (w // 16) + w % 4


def gather(plane, table, n, page, D, at):
    """[H][n][D] of positions 0 .. n - 1 of a sequence with that page table row."""
    p, d = np.arange(n)[:, None], np.arange(D)[None, :]
    pg = np.asarray(table)[np.arange(n) // page]
    off = at(p % page, d, D)
    return np.stack([plane[pg[:, None], h, off] for h in range(plane.shape[1])])


def append(kplane, vplane, table, pos0, k, v, page):
    """Write k, v [n][H][D] (rotated) at positions pos0 .. of one sequence."""
    n, H, D = k.shape
    d = np.arange(D)
    for j in range(n):
        p = pos0 + j
        for h in range(H):
            kplane[table[p // page], h, key_at(p % page, d, D)] = k[j, h]
            vplane[table[p // page], h, value_at(p % page, d, D)] = v[j, h]


def attention(q, K, V, pos0, scale, window=0, seen=None):
    """q [n][Hq][D] at positions pos0 + j, K and V [H][L][D]; seen: positions
    that may be attended to at all. Returns (out, lse, spread) with spread =
    sum_p w |V| and the largest sum_d |q_d k_d| scale, for error bounds."""
    n, Hq, D = q.shape
    H, L = K.shape[:2]
    G = Hq // H
    out, lse = np.zeros((n, Hq, D)), np.full((n, Hq), -np.inf)
    wabs, mag = np.zeros((n, Hq, D)), np.zeros((n, Hq))
    p = np.arange(L)
    for j in range(n):
        ok = p <= pos0 + j
        if window:
            ok &= p > pos0 + j - window
        if seen is not None:
            ok &= seen[:L]
        idx = p[ok]
        if not len(idx):
            continue
        for h in range(Hq):
            k, v = K[h // G][idx], V[h // G][idx]
            s = k @ q[j, h] * scale
            m = s.max()
            w = np.exp(s - m)
            z = w.sum()
            out[j, h], lse[j, h] = w @ v / z, m + np.log(z)
            wabs[j, h] = w @ np.abs(v) / z
            mag[j, h] = (np.abs(k) @ np.abs(q[j, h])).max() * scale
    return out, lse, wabs, mag
