"""The 8-bit paged cache from its definition, for the tests: whole numbers in Python and fp64 in
numpy and torch on the CPU, one block and one row at a time. Shares no code with the library."""
import math

import numpy as np
import torch

TOP = {"e4m3": 448.0, "int8": 127.0}
DTYPE = {"e4m3": torch.float8_e4m3fn, "int8": torch.int8}


def schedule(old, new, free, table, block_size, max_rows):
    """(table, row_starts, kv_lens, slots, counts) by walking the requests and their tokens."""
    table = [list(r) for r in table]
    width = len(table[0]) if table else 0
    cap = width * block_size
    old, new = [max(0, x) for x in old], [max(0, x) for x in new]
    taken, starts, slots, kv = 0, [0], [], []
    for r, (o, n) in enumerate(zip(old, new)):
        k = min(o + n, cap)
        kv.append(k)
        for b in range(min(-(-o // block_size), width), -(-k // block_size)):
            table[r][b] = free[taken] if taken < len(free) else -1
            taken += 1
        for t in range(o, o + n):
            b = table[r][t // block_size] if t < cap else -1
            slots.append(b * block_size + t % block_size if b >= 0 else -1)
        starts.append(starts[-1] + n)
    counts = [taken, len(slots)]
    slots = (slots + [-1] * max_rows)[:max_rows]
    return table, [min(s, max_rows) for s in starts], kv, slots, counts


def nearest_codes(x, fmt):
    """fp64 values to the nearest code's value, ties to even, clamped; NaN to 0."""
    x = np.where(np.isnan(x), 0.0, x)
    x = np.clip(x, -TOP[fmt], TOP[fmt])
    if fmt == "int8":
        return np.rint(x)
    _, e = np.frexp(x)
    step = np.ldexp(1.0, np.maximum(e - 4, -9))
    return np.rint(x / step) * step


def scale_for(x, fmt):
    x = np.abs(x[np.isfinite(x)])
    m = float(x.max()) if x.size else 0.0
    k = -60
    while k < 60 and m > TOP[fmt] * 2.0 ** k:
        k += 1
    return 2.0 ** k


def append(codes, scale, rows, slots, block_size, fmt):
    """One head of K or V: codes [blocks, block_size, d] and scale [blocks] (fp64, changed in place)
    take rows [n, d] at `slots`."""
    i = 0
    while i < len(slots):
        s = int(slots[i])
        if s < 0 or s >= codes.shape[0] * block_size:
            i += 1
            continue
        n = 1
        while i + n < len(slots) and slots[i + n] == s + n and (s + n) % block_size:
            n += 1
        b, p = divmod(s, block_size)
        need = scale_for(rows[i:i + n], fmt)
        f = max(scale[b], need) if p else need
        if p and f > scale[b]:
            codes[b, :p] = nearest_codes(codes[b, :p] * (scale[b] / f), fmt)
        codes[b, p:p + n] = nearest_codes(rows[i:i + n] / f, fmt)
        scale[b] = f
        i += n


def attend(q, k, v, softmax_scale, limits):
    """One (request, query head): q [n, d], k and v [tokens, d] in fp64, row i over the first limits[i]
    tokens. Returns (out, lse, weighted magnitude sum p |v|, largest sum |q||k| scale)."""
    out, mag = (torch.zeros((len(q), v.shape[1]), dtype=torch.float64) for _ in range(2))
    lse, size = torch.full((len(q),), -math.inf, dtype=torch.float64), 0.0
    for i in range(len(q)):
        n = limits[i]
        if n <= 0:
            continue
        s = (k[:n] @ q[i]) * softmax_scale
        size = max(size, float(((k[:n].abs() @ q[i].abs()) * abs(softmax_scale)).max()))
        top = s.max()
        p = torch.exp(s - top)
        total = p.sum()
        out[i] = (p @ v[:n]) / total
        mag[i] = (p @ v[:n].abs()) / total
        lse[i] = top + torch.log(total)
    return out, lse, mag, size
