"""The paged 8-bit latent cache and both forms of its attention in plain numpy, 64 bits: the definitions of
include/uzip_latent.h, row by row."""
from __future__ import annotations

import numpy as np

from .kv import code_values, encode, exponent


def store(codes, exps, latent, key_rot, slots, page: int, fmt: str) -> None:
    """latent [rows, C] and key_rot [rows, R], turned already, into codes [pages, page, C + R] and exps [pages, page, 2], in place."""
    for r, slot in enumerate(slots):
        if slot < 0 or slot >= codes.shape[0] * page:
            continue
        pg, at = divmod(int(slot), page)
        begin = 0
        for part, x in enumerate((latent[r], key_rot[r])):
            x = np.asarray(x, dtype=np.float64)
            e = exponent(float(np.abs(x[np.isfinite(x)]).max(initial=0.0)), fmt)
            exps[pg, at, part] = e
            codes[pg, at, begin:begin + len(x)] = encode(x * 2.0 ** (127 - e), fmt)
            begin += len(x)


def _row(z, values):
    m = z.max(axis=1, keepdims=True)
    w = np.exp(z - m)
    s = w.sum(axis=1, keepdims=True)
    return w / s, (m + np.log(s))[:, 0]


def attend(q, codes, exps, latent: int, fmt: str, table, lens, q_start, page: int, scale: float) -> dict:
    """Besides out and lse: `spread`, the sum of p |c| for each output, `size`, the largest scale * sum |q k| of a
    row, and `floor`, the sum of |code_t| over sum_t 2^(g_t - max g - e_t) with g_t = s_t log2(e) + e_t: what an error of 1 of a
    weight 2^(g_t - max g) on every token would make of an output; `tiles`, the same of an error of 1 relative to the largest
    weight of 64 tokens that begin at a multiple of 64."""
    q = np.asarray(q, dtype=np.float64)
    rows, heads, _ = q.shape
    out, spread, floor, tiles = (np.zeros((rows, heads, latent)) for _ in range(4))
    lse, size, shift = np.full((rows, heads), -np.inf), np.zeros((rows, heads)), np.zeros((rows, heads))
    values = code_values(fmt)
    for i in range(len(lens)):
        a, b = int(q_start[i]), int(q_start[i + 1])
        length = min(max(int(lens[i]), 0), table.shape[1] * page)
        t = np.arange(length)
        pg = table[i, t // page] if length else np.zeros(0, int)
        here = (pg >= 0) & (pg < codes.shape[0])
        t, pg = t[here], pg[here]
        raw = values[codes[pg, t % page]]
        e = exps[pg, t % page].astype(np.float64) - 127
        keys = raw * np.repeat(2.0 ** e, [latent, raw.shape[1] - latent], axis=1) if len(t) else raw
        for r in range(a, b):
            n = int(np.searchsorted(t, length - (b - a) + (r - a), side="right"))
            if not n:
                continue
            k = keys[:n]
            z = (q[r] @ k.T) * scale
            w, lse[r] = _row(z, k)
            out[r], spread[r] = w @ k[:, :latent], w @ np.abs(k[:, :latent])
            size[r] = (np.abs(q[r]) @ np.abs(k).T).max(axis=1) * abs(scale)
            g = z * np.log2(np.e) + e[:n, 0]
            under = (2.0 ** (g - g.max(axis=1, keepdims=True) - e[:n, 0])).sum(axis=1)
            floor[r] = np.abs(raw[:n, :latent]).sum(axis=0) / under[:, None]
            starts = np.flatnonzero(np.diff(t[:n] // 64, prepend=-1))
            most = 2.0 ** (np.maximum.reduceat(g, starts, axis=1) - g.max(axis=1, keepdims=True))
            tiles[r] = most @ np.add.reduceat(np.abs(raw[:n, :latent]), starts, axis=0) / under[:, None]
            shift[r] = np.abs(e[:n, 0]).max()
    return {"out": out, "lse": lse, "spread": spread, "size": size, "floor": floor, "tiles": tiles, "shift": shift}


def expanded(q, k, key_rot, v, q_start, k_start, scale: float) -> dict:
    q, k, key_rot, v = (np.asarray(x, dtype=np.float64) for x in (q, k, key_rot, v))
    rows, heads, _ = q.shape
    out, spread, floor = (np.zeros((rows, heads, v.shape[2])) for _ in range(3))
    lse, size = np.full((rows, heads), -np.inf), np.zeros((rows, heads))
    for i in range(len(k_start) - 1):
        a, b, c, d = int(q_start[i]), int(q_start[i + 1]), int(k_start[i]), int(k_start[i + 1])
        for h in range(heads):
            keys = np.concatenate([k[c:d, h], key_rot[c:d]], axis=1)
            for r in range(a, b):
                n = (d - c) - (b - a) + (r - a) + 1
                if n <= 0:
                    continue
                z = (q[r, h] @ keys[:n].T)[None] * scale
                w, e = _row(z, keys)
                lse[r, h] = e[0]
                out[r, h], spread[r, h] = w[0] @ v[c:c + n, h], w[0] @ np.abs(v[c:c + n, h])
                size[r, h] = (np.abs(q[r, h]) @ np.abs(keys[:n]).T).max() * abs(scale)
                floor[r, h] = np.abs(v[c:c + n, h]).sum(axis=0) / np.exp(z - z.max()).sum()
    return {"out": out, "lse": lse, "spread": spread, "size": size, "floor": floor}
