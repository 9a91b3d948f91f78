"""Plain 64-bit definitions of the 4-bit rows, the attention that accumulates
weights and the eviction, in NumPy with loops over units.  Test infrastructure:
nothing here shares code with the library."""
from __future__ import annotations

import numpy as np

MAGNITUDES = np.array([0, 0.5, 1, 1.5, 2, 3, 4, 6], np.float64)


def encode(x):
    """Codes uint8 [..., d / 2] and scale bytes uint8 [..., d / 32] of rows x [..., d]."""
    x = np.asarray(x, np.float64)
    blocks = x.reshape(-1, 32)
    codes = np.zeros(blocks.shape, np.uint8)
    scales = np.zeros(len(blocks), np.uint8)
    for i, b in enumerate(blocks):
        if not np.isfinite(b).all():
            scales[i] = 255
            continue
        top = np.abs(b).max()
        e = -125
        while e < 125 and top > 7.0 * 2.0 ** e:
            e += 1
        scales[i] = e + 127
        a = np.abs(b) / 2.0 ** e
        dist = np.abs(a[:, None] - MAGNITUDES[None, :])
        best = dist.min(axis=1, keepdims=True)
        # of two codes equally near, the even one
        pick = np.where(dist == best, np.arange(8) % 2 + 0.0, 9.0).argmin(axis=1)
        codes[i] = pick.astype(np.uint8) | (np.signbit(b).astype(np.uint8) << 3)
    codes = codes.reshape(x.shape)
    return codes[..., 0::2] | (codes[..., 1::2] << 4), scales.reshape(*x.shape[:-1], x.shape[-1] // 32)


def decode(codes, scales):
    """Values (float64) of codes under their scale bytes."""
    c = np.stack([codes & 15, codes >> 4], axis=-1).reshape(*codes.shape[:-1], -1)
    v = np.where(c >= 8, -1.0, 1.0) * MAGNITUDES[c & 7]
    s = np.where(scales == 255, np.nan, 2.0 ** (scales.astype(np.float64) - 127))
    return v * np.repeat(s, 32, axis=-1)


def pool_rows_of(table, n, page_size, pool_rows):
    """Pool row of each logical row < n of one unit, -1 outside the pool."""
    i = np.arange(min(max(int(n), 0), len(table) * page_size))
    r = table[i // page_size].astype(np.int64) + i % page_size
    return np.where((r >= 0) & (r < pool_rows), r, -1)


def attention(q, k, v, table, n_rows, page_size, scale, weight=None, decay=1.0):
    """(out [B][Hq][d], weights, bound of sums): q [B][Hq][d], pools [rows][d] float64.

    `weights` is a list per unit of the new weights of its rows; the bounds, per
    output and per weight, are what |error| of an fp32 evaluation is a multiple
    of (see tolerance())."""
    B, Hq, d = q.shape
    Hkv = table.shape[1]
    G = Hq // Hkv
    out, size = np.zeros((B, Hq, d)), np.zeros((B, Hq, d))
    weights, sizes, steps = {}, {}, np.zeros((B, Hq))
    for b in range(B):
        for h in range(Hkv):
            rows = pool_rows_of(table[b, h], n_rows[b, h], page_size, len(k))
            w = np.zeros(len(rows)) if weight is None else decay * weight[b, h, :len(rows)].astype(np.float64)
            base, live = np.abs(w), rows >= 0
            add = np.zeros(len(rows))
            for g in range(h * G, (h + 1) * G):
                if not live.any():
                    continue
                kk, vv = k[rows[live]], v[rows[live]]
                z = scale * (kk @ q[b, g])
                p = np.exp(z - z.max())
                p = p / p.sum()
                out[b, g], size[b, g] = p @ vv, p @ np.abs(vv)
                add[live] += p
                steps[b, g] = tolerance(d, live.sum(), scale * (np.abs(kk) @ np.abs(q[b, g])).max())
            weights[b, h] = w + add
            sizes[b, h] = base * 2.0 ** -22 + add * (steps[b, h * G:(h + 1) * G].max() if len(rows) else 0.0)
    return out, size * steps[..., None] + 1e-37, weights, sizes


def tolerance(d, n, reach):
    """Bound of the relative error of a probability, and of a sum of them, in fp32.

    A logit is a sum of d products whose magnitudes add up to `reach` (scaled):
    its error is at most (d + 8) * 2^-23 * reach (each product and sum rounded or
    cut at 24 bits).  The probability then is off by twice that (numerator and
    denominator) and by the exponential's own 2^-22; sums over n rows add n *
    2^-24 each to numerator and denominator."""
    return 2.0 * (d + 8) * 2.0 ** -23 * max(reach, 1.0) + 2.0 ** -21 + 2 * n * 2.0 ** -24


def evict(n, budget, weight, pos, sinks, recent):
    """(k, moves [(to, from)], new weights [n], new positions [n]) of one unit."""
    n = int(n)
    k = min(max(int(budget), 0), n)

    def rank(i):
        guarded = pos[i] < sinks or (recent is not None and pos[i] >= recent)
        w = float(weight[i])
        if guarded:
            return (0, 0.0, i)
        return (2, 0.0, i) if np.isnan(w) else (1, -w + 0.0, i)

    kept = sorted(sorted(range(n), key=rank)[:k])
    stay = set(i for i in kept if i < k)
    move = list(zip([i for i in range(k) if i not in stay], [i for i in kept if i >= k]))
    w, p = np.zeros(n, np.float32), np.full(n, -1, np.int32)
    for i in stay:
        w[i], p[i] = weight[i], pos[i]
    for to, src in move:
        w[to], p[to] = weight[src], pos[src]
    return k, move, w, p
