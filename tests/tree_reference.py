"""The operators around a tree of drafted tokens from their definitions, for the tests: whole numbers in Python, fp64 (and
fp32 where the definition rounds to it) in numpy, one row at a time. Shares no code with the library."""
import numpy as np

import qcache_reference as qref

UNIT = 1 << 42


def plan(starts, context, parents, rows, words):
    """(masks as whole numbers, positions), None for rows of no request. parents None: the row before."""
    masks, positions = [None] * rows, [None] * rows
    for r in range(len(starts) - 1):
        c = max(context[r], 0)
        depth = {}
        for i in range(starts[r + 1] - starts[r]):
            row = starts[r] + i
            a = i - 1 if parents is None else parents[row]
            if parents is None:
                positions[row] = min(c + i, 2 ** 31 - 1)
                masks[row] = (2 << i) - 1 if i < 32 * words else 0
                continue
            if i >= 32 * words:
                masks[row], positions[row] = 0, c
                continue
            has = 0 <= a < i
            masks[row] = 1 << i | (masks[starts[r] + a] if has else 0)
            depth[i] = depth[a] + 1 if has else 0
            positions[row] = min(c + depth[i], 2 ** 31 - 1)
    return masks, positions


def rotate(x, positions, weight, eps, theta):
    """x [rows, heads, d] in fp64. Returns (out, |y_j| + |y_{j + d/2}| for each element)."""
    d = x.shape[-1]
    y = x
    if weight is not None:
        root = np.sqrt((x ** 2).mean(-1, keepdims=True) + eps)
        y = np.where(root == 0, 0.0, x / np.where(root == 0, 1.0, root)) * weight
    turn = np.longdouble(theta) ** (-np.arange(0, d, 2, dtype=np.longdouble) / d)
    angle = np.fmod(positions.astype(np.longdouble)[:, None] * turn, 8 * np.arctan(np.longdouble(1)))[:, None].astype(np.float64)
    lo, hi = y[..., :d // 2], y[..., d // 2:]
    size = np.abs(lo) + np.abs(hi)
    return (np.concatenate([lo * np.cos(angle) - hi * np.sin(angle), hi * np.cos(angle) + lo * np.sin(angle)], -1),
            np.concatenate([size, size], -1))


def _clean(x):
    x = np.where(np.isnan(x), np.float32(0), x.astype(np.float32))
    return np.minimum(np.maximum(x, np.float32(0)), np.float32(1))


def _whole(x):
    return (x.astype(np.float64) * UNIT).astype(np.int64)


def verify(starts, parents, tokens, target, draft, accept, sample, max_nodes):
    """target, draft: fp32 arrays [rows, vocab]; accept, sample fp32. (path, kept, next_token)."""
    vocab = target.shape[1]
    path, kept, chosen = [], [], []
    for r in range(len(starts) - 1):
        base, n = starts[r], starts[r + 1] - starts[r]
        if n == 0:
            kept.append(0)
            chosen.append(-1)
            continue
        children = {}
        for i in range(min(n, max_nodes)):
            a, t = parents[base + i], tokens[base + i]
            if 0 <= a < i and 0 <= t < vocab:
                children.setdefault(a, []).append(i)
        walk = [0]
        while True:
            node = walk[-1]
            whole = w = _clean(target[base + node])
            q = None if draft is None else _clean(draft[base + node])
            z, taken = UNIT, None
            for c in children.get(node, []):
                t, u = tokens[base + c], float(accept[base + c])
                if q is None:
                    if u * (z / UNIT) < float(w[t]):
                        taken = c
                        break
                    z -= int(_whole(w[t:t + 1])[0])
                    w = w.copy()
                    w[t] = 0
                else:
                    scale = np.float32(z / UNIT)
                    if u * float(q[t]) * float(scale) < float(w[t]):
                        taken = c
                        break
                    rest = np.maximum(w - q * scale, np.float32(0))
                    total = int(_whole(rest).sum())
                    if total:
                        w, z = rest, total
            if taken is None:
                break
            walk.append(taken)
        if draft is None and not _whole(w).any():
            w = whole
        total, at, u = int(_whole(w).sum()), 0, float(sample[r])
        number = 0 if not u > 0 else min(int(min(u, 1.0) * 2 ** 32), 2 ** 32 - 1)
        point, token = total * number >> 32, -1
        if total:
            sums = np.cumsum(_whole(w))
            token = int(np.argmax(sums > point))
        kept.append(len(walk))
        chosen.append(token)
        path += walk + [-1] * (n - len(walk))
    return path, kept, chosen


def _again(codes, ratio, fmt):
    """Codes times an fp32 ratio to the nearest code: rounded to fp32 between for e4m3, at once for int8."""
    x = codes * float(ratio) if fmt == "int8" else codes.astype(np.float32) * ratio
    return qref.nearest_codes(x.astype(np.float64), fmt)


def keep_rows(table, context, kv, n, path, kept, block, num_blocks):
    """The moves ((block, place) from, to) of one request's path, and its length afterwards."""
    moves, before = [], -1
    kv = min(kv, len(table) * block)

    def place(token):
        if token >= kv or not 0 <= table[token // block] < num_blocks:
            return None
        return table[token // block], token % block

    for i in range(min(max(kept, 0), n, 256)):
        x = path[i]
        if not before < x < n or place(context + x) is None or place(context + i) is None:
            break
        moves.append((place(context + x), place(context + i)))
        before = x
    return moves


def keep(codes, scale, moves, fmt):
    """One layer and head of K or V: codes [blocks, block, d] fp64 and scale [blocks] fp32, changed in place."""
    still = True
    pending = []
    for frm, to in moves:
        still = still and frm == to
        if not still:
            pending.append((frm, to))
    while pending:
        b = pending[0][1][0]
        here = [m for m in pending if m[1][0] == b]
        pending = pending[len(here):]
        first = here[0][1][1]
        now = max([scale[f[0]] for f, _ in here] + ([scale[b]] if first else []))
        put = []
        for (x, at), _ in here:
            ratio = np.float32(scale[x] / now)
            put.append(codes[x, at].copy() if ratio == 1 else _again(codes[x, at], ratio, fmt))
        if first and now > scale[b]:
            codes[b, :first] = _again(codes[b, :first], np.float32(scale[b] / now), fmt)
        for x, (_, (_, at)) in zip(put, here):
            codes[b, at] = x
        scale[b] = now
