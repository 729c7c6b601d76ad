"""The paged 8-bit key/value cache in plain numpy, 64 bits throughout.

The definitions of include/uzip_kv.h, written request by request and row by
row; the tests compare the kernels with it.
"""
from __future__ import annotations

import numpy as np

# fraction bits, bias, largest value, largest exponent byte
FORMATS = {"e4m3fn": (3, 7, 448.0, 246), "e5m2": (2, 15, 57344.0, 239)}
EXP_MIN = 27
EINVAL, ENOSPC = -1, -2


def code_values(fmt: str) -> np.ndarray:
    """The 256 codes' values."""
    bits, bias, top, _ = FORMATS[fmt]
    c = np.arange(256)
    field, frac = (c & 127) >> bits, (c & ((1 << bits) - 1)) / (1 << bits)
    x = np.where(field > 0, (1 + frac) * 2.0 ** (field - bias), frac * 2.0 ** (1 - bias))
    if fmt == "e4m3fn":
        x[(c & 127) == 127] = np.nan
    else:
        x[(c & 127) == 0x7C] = np.inf
        x[(c & 127) > 0x7C] = np.nan
    return np.where(c >= 128, -x, x)


def decode(codes, fmt: str, exps=None) -> np.ndarray:
    x = code_values(fmt)[np.asarray(codes)]
    return x if exps is None else x * 2.0 ** (np.asarray(exps, dtype=np.float64) - 127)


def encode(x, fmt: str) -> np.ndarray:
    """The nearest code of each x (ties to the even one), the largest for values past it."""
    x = np.asarray(x, dtype=np.float64)
    table = code_values(fmt)[:128]
    finite = table[np.isfinite(table)]
    mag = np.minimum(np.abs(np.where(np.isfinite(x), x, 0.0)), finite[-1])
    up = np.clip(np.searchsorted(finite, mag), 1, len(finite) - 1)
    lo, hi = finite[up - 1], finite[up]
    down = (mag - lo < hi - mag) | ((mag - lo == hi - mag) & ((up - 1) % 2 == 0))
    c = np.where(down, up - 1, up)
    c = np.where(np.isinf(x), 0x7F if fmt == "e4m3fn" else 0x7C, c)
    c = np.where(np.isnan(x), 0x7F, c)
    return (c + 128 * np.signbit(x)).astype(np.uint8)


def exponent(amax: float, fmt: str) -> int:
    """The least exponent byte in the format's range with amax <= largest code * 2^(e - 127)."""
    _, _, top, most = FORMATS[fmt]
    e = EXP_MIN
    while e < most and amax > top * 2.0 ** (e - 127):
        e += 1
    return e


def max_runs(rows: int, reqs: int, page: int) -> int:
    return max(1, min(rows, rows // page + 2 * reqs))


def plan(old, new, free, table, page: int, rows: int) -> dict:
    """Lengths, first rows, slots, runs, counts, status; `table` as it is after the call."""
    table = table.copy()
    lens, q_start, slots, runs = [], [0], np.full(rows, -1, np.int64), []
    status, taken, at, row, short = 0, 0, 0, 0, False
    for i, (o, n) in enumerate(zip(old, new)):
        o, n = int(o), int(n)
        first = row
        row += max(n, 0)
        q_start.append(min(row, rows))
        have, want = -(-o // page), -(-(o + n) // page)
        if o < 0 or n < 0 or row > rows or o + n > 2 ** 31 - 1:
            status = min(status, EINVAL)
            lens.append(0)
            continue
        if want > table.shape[1]:
            status = min(status, ENOSPC)
            lens.append(0)
            continue
        if want > have and (short or at + want - have > len(free)):
            status, short = min(status, ENOSPC), True
            lens.append(0)
            continue
        for k in range(have, want):
            table[i, k] = free[at]
            at += 1
        taken = at
        lens.append(o + n)
        for j in range(n):
            pos = o + j
            pg = int(table[i, pos // page])
            slots[first + j] = pg * page + pos % page if pg >= 0 else -1
            if j == 0 or pos % page == 0:
                runs.append((first + j, min(page - pos % page, n - j)))
    return {"table": table, "lens": np.array(lens, np.int32), "q_start": np.array(q_start, np.int32), "slots": slots,
            "runs": np.array(runs, np.int32).reshape(-1, 2), "counts": np.array([taken, len(runs)], np.int32),
            "status": status}


def store(codes, exps, x, slots, runs, page: int, fmt: str) -> None:
    """Write rows x [rows, heads, dim] into codes [pages, heads, page, dim] and exps [pages, heads], in place."""
    x = np.asarray(x, dtype=np.float64)
    for first, n in runs:
        pg, off = divmod(int(slots[first]), page)
        for h in range(x.shape[1]):
            y = x[first:first + n, h]
            e = exponent(float(np.abs(y[np.isfinite(y)]).max(initial=0.0)), fmt)
            if off:
                was = int(exps[pg, h])
                if e > was:
                    codes[pg, h, :off] = encode(decode(codes[pg, h, :off], fmt) * 2.0 ** (was - e), fmt)
                e = max(e, was)
            exps[pg, h] = e
            codes[pg, h, off:off + n] = encode(y * 2.0 ** (127 - e), fmt)


def attend(q, k, k_exp, v, v_exp, fmt: str, table, lens, q_start, page: int, scale: float, window: int = 0) -> dict:
    """k and v: codes [pages, heads, page, dim] (v as k, not transposed).  Besides out and lse: `spread`, the sum of
    p |v| for each output, and `size`, the largest scale * sum |q k| of each row, which bound rounding errors."""
    q = np.asarray(q, dtype=np.float64)
    rows, heads, dim = q.shape
    pages, kv = k_exp.shape
    group = heads // kv
    out, spread = np.zeros((rows, heads, dim)), np.zeros((rows, heads, dim))
    lse, size = np.full((rows, heads), -np.inf), np.zeros((rows, heads))
    values = code_values(fmt)
    for i in range(len(lens)):
        a, b = int(q_start[i]), int(q_start[i + 1])
        length = min(max(int(lens[i]), 0), table.shape[1] * page)
        for r in range(a, b):
            p = length - (b - a) + (r - a)
            t = np.arange(max(0, p - window + 1) if window else 0, min(p + 1, length))
            pg = table[i, t // page] if len(t) else np.zeros(0, int)
            here = (pg >= 0) & (pg < pages)
            t, pg = t[here], pg[here]
            if not len(t):
                continue
            for h in range(kv):
                kk = values[k[pg, h, t % page]] * (2.0 ** (k_exp[pg, h].astype(float) - 127))[:, None]
                vv = values[v[pg, h, t % page]] * (2.0 ** (v_exp[pg, h].astype(float) - 127))[:, None]
                z = (q[r, h * group:(h + 1) * group] @ kk.T) * scale
                m = z.max(axis=1, keepdims=True)
                w = np.exp(z - m)
                s = w.sum(axis=1, keepdims=True)
                cols = slice(h * group, (h + 1) * group)
                out[r, cols], spread[r, cols] = (w / s) @ vv, (w / s) @ np.abs(vv)
                lse[r, cols] = (m + np.log(s))[:, 0]
                size[r, cols] = (np.abs(q[r, cols]) @ np.abs(kk).T).max(axis=1) * abs(scale)
    return {"out": out, "lse": lse, "spread": spread, "size": size}
