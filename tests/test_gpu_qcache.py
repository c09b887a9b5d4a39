"""The 8-bit paged cache on the GPU against its definition: block tables and slots, the cache
write and attention.

Tables, codes and scales are compared exactly: scales are powers of two, so every division is
exact and each code is rounded once.

Attention, from how it is computed: the result is rounded once to bf16 (half an ulp: 2^-8 of it),
each weight once to fp16 (2^-11 of it, so 2^-11 of sum p |v|, whatever the signs), and the fp32 part
(sums of at most a few thousand products, 2^-13 of sum p |v|; scores to 2^-20 of sum |q||k|, which
moves a weight by as much) is below that. Hence
    |out - ref| <= 2^-8 |ref| * (1 + 2^-6) + (2^-11 + 2^-12 + 2^-19 size) * sum p |v|
    |lse - ref| <= 2^-19 * (1 + |ref| + size),   size = the largest sum |q||k| * softmax_scale
"""
import importlib.util
import math
import os

import numpy as np
import pytest
import torch

import qcache_reference as ref

pytestmark = pytest.mark.gpu

cm = pytest.importorskip("paper_2607_01308_gb300")

DEV = "cuda:0"


@pytest.fixture(scope="module")
def ctx():
    c = cm.Context(0)
    yield c
    c.close()


def _i32(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


# ---------------------------------------------------------------- block tables

def _schedule(ctx, old, new, width, block, num_free=None, max_rows=None, seed=0):
    rng = np.random.default_rng(seed)
    need = sum(-(-max(0, o) // block) for o in old)
    fresh = sum(-(-(max(0, o) + max(0, n)) // block) for o, n in zip(old, new)) - need
    ids = rng.permutation(need + fresh + 5).tolist()
    table, at = [], 0
    for o in old:
        row = [-1] * width
        for b in range(min(width, -(-max(0, o) // block))):
            row[b] = ids[at]
            at += 1
        table.append(row)
    free = ids[at:]
    if num_free is not None:
        free = free[:num_free]
    rows = sum(max(0, n) for n in new) if max_rows is None else max_rows
    batch = cm.QBatch(ctx, len(old), width, rows, block)
    if old:
        batch.block_table.copy_(_i32(table).reshape(len(old), width))
    batch.slot_map.fill_(-7)
    batch.schedule(_i32(old), _i32(new), _i32(free))
    torch.cuda.synchronize()
    want = ref.schedule(old, new, free, table, block, rows)
    got = (batch.block_table.tolist(), batch.row_starts.tolist(), batch.kv_lens.tolist(),
           batch.slot_map.tolist(), batch.counts.tolist())
    for name, g, w in zip(("table", "starts", "kv", "slots", "counts"), got, want):
        assert g == w, name


@pytest.mark.parametrize("old,new,block", [
    ([5], [1], 16), ([16], [1], 16), ([0], [0], 16), ([15], [1], 16), ([0], [16], 16), ([31], [34], 32),
    ([0, 0, 0], [0, 7, 0], 16), ([3, 40, 0, 16], [0, 1, 100, 17], 16), ([256, 255, 1], [1, 1, 513], 256),
    ([0] * 5, [0] * 5, 64)])
def test_tables_small(ctx, old, new, block):
    width = max(1, max(-(-(o + n) // block) for o, n in zip(old, new)) + 2)
    _schedule(ctx, old, new, width, block)


@pytest.mark.parametrize("requests,most_old,most_new,block", [
    (1, 100, 5000, 16), (33, 900, 1, 16), (255, 70, 3, 32), (256, 70, 3, 32), (257, 70, 90, 64), (1500, 40, 2, 128)])
def test_tables_ragged(ctx, requests, most_old, most_new, block):
    rng = np.random.default_rng(requests)
    old = rng.integers(0, most_old + 1, requests).tolist()
    new = rng.integers(0, most_new + 1, requests).tolist()
    _schedule(ctx, old, new, -(-(most_old + most_new) // block) + 1, block, seed=requests)


def test_tables_many_requests(ctx):
    n = 16384
    rng = np.random.default_rng(1)
    old, new = rng.integers(0, 33, n).tolist(), rng.integers(0, 2, n).tolist()
    _schedule(ctx, old, new, 3, 16, seed=3)


def test_tables_out_of_blocks_width_and_rows(ctx):
    _schedule(ctx, [3, 20, 0], [40, 30, 60], 8, 16, num_free=4)        # the free list runs out
    _schedule(ctx, [3, 20, 0], [40, 30, 60], 8, 16, num_free=0)
    _schedule(ctx, [3, 100, 60], [40, 30, 60], 4, 16)                  # the table ends before the tokens
    _schedule(ctx, [3, 20, 0], [40, 30, 60], 8, 16, max_rows=50)       # fewer rows than tokens
    _schedule(ctx, [3, 20, 0], [40, 30, 60], 8, 16, max_rows=500)      # more
    _schedule(ctx, [-4, 7], [5, -9], 3, 16)                            # negative lengths count as none
    _schedule(ctx, [], [], 1, 16, max_rows=3)


# ---------------------------------------------------------------- the cache write

def _codes_f64(t):
    return t.float().double().cpu().numpy()


def _check_append(ctx, fmt, layers, heads, dim, block, num_blocks, slots, rows, layer=0, cache_layers=None,
                  order="blhtd", fill=0, k_values=None):
    """One append into a cache in use against the reference; returns the cache."""
    g = torch.Generator().manual_seed(fill + dim)
    cl = cache_layers or layers
    sizes = {"b": num_blocks, "l": cl, "h": heads, "t": block, "d": dim}
    names = "blhtd"

    def make():
        raw = torch.randint(-100, 100, [sizes[c] for c in order], generator=g)
        if fmt == "int8":
            t = raw.to(torch.int8)
        else:
            t = (raw / 8.0).to(torch.float8_e4m3fn)
        return t.to(DEV).permute([order.index(c) for c in names])

    k, v = make(), make()
    ks = torch.pow(2.0, torch.randint(-9, 2, (num_blocks, cl, heads), generator=g).float()).to(DEV)
    vs = torch.pow(2.0, torch.randint(-9, 2, (num_blocks, cl, heads), generator=g).float()).to(DEV)
    cache = cm.QCache.from_tensors(ctx, k, v, ks, vs)
    n = len(slots)
    new = []
    for which in range(2):
        x = torch.randn((layers, heads, n, dim), generator=g) * torch.exp2(torch.randint(-6, 4, (layers, heads, n, 1), generator=g).float())
        x = x.bfloat16()
        if k_values is not None:
            x = k_values(x, which)
        new.append(x)
    before = [t.clone() for t in (k.view(torch.uint8), v.view(torch.uint8), ks, vs)]
    want = []
    for codes, scale, x in ((k, ks, new[0]), (v, vs, new[1])):
        c, s = _codes_f64(codes), scale.double().cpu().numpy()
        for l in range(layers):
            for h in range(heads):
                ref.append(c[:, layer + l, h], s[:, layer + l, h], x[l, h].double().numpy(), slots, block, fmt)
        want.append((c, s))
    cache.append(new[0].to(DEV), new[1].to(DEV), torch.tensor(slots, dtype=torch.int64, device=DEV), layer=layer)
    torch.cuda.synchronize()
    # codes are compared as values: -0 and 0 are one
    for codes, scale, (c, s) in ((k, ks, want[0]), (v, vs, want[1])):
        np.testing.assert_array_equal(scale.double().cpu().numpy(), s)
        np.testing.assert_array_equal(_codes_f64(codes), c)
    return cache, before


def _slots_of(requests, block, num_blocks, seed):
    """Slots of [(old, new), ...] with shuffled blocks."""
    rng = np.random.default_rng(seed)
    ids = rng.permutation(num_blocks).tolist()
    slots = []
    for old, new in requests:
        mine = [ids.pop() for _ in range(-(-(old + new) // block))]
        slots += [mine[t // block] * block + t % block for t in range(old, old + new)]
    return slots


FORMATS = ["e4m3", "int8"]


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("dim,block,requests", [
    (128, 16, [(0, 1)]), (128, 16, [(15, 1), (16, 1), (7, 1)]), (128, 16, [(0, 53)]), (64, 32, [(5, 40), (31, 1), (0, 64), (33, 95)]),
    (16, 16, [(3, 30)]), (32, 64, [(1, 200), (63, 2)]), (256, 16, [(9, 20)]), (512, 16, [(4, 33), (0, 3)]),
    (128, 64, [(10, 150)]), (256, 128, [(100, 300), (127, 1)]), (512, 256, [(5, 260)])])
def test_append(ctx, fmt, dim, block, requests):
    num_blocks = sum(-(-(o + n) // block) for o, n in requests) + 2
    _check_append(ctx, fmt, 1, 3, dim, block, num_blocks, _slots_of(requests, block, num_blocks, dim), requests)


@pytest.mark.parametrize("fmt", FORMATS)
def test_append_layers_and_layouts(ctx, fmt):
    requests = [(5, 30), (0, 17)]
    slots = _slots_of(requests, 16, 9, 4)
    _check_append(ctx, fmt, 2, 2, 64, 16, 9, slots, requests, layer=1, cache_layers=4)
    _check_append(ctx, fmt, 1, 2, 64, 16, 9, slots, requests, order="lbthd")     # per-layer pools, token-major
    _check_append(ctx, fmt, 3, 5, 32, 16, 9, slots, requests, order="hlbtd")


@pytest.mark.parametrize("fmt", FORMATS)
def test_append_strided_rows_many_heads(ctx, fmt):
    """Rows [rows][H][d] (a projection's output) as a permuted view; more heads than one thread block has."""
    rows, H, d, block = 37, 7, 64, 16
    x = torch.randn(2, rows, H, d).bfloat16().to(DEV)
    a = cm.QCache(ctx, 4, block, 1, H, d, dtype=ref.DTYPE[fmt])
    b = cm.QCache(ctx, 4, block, 1, H, d, dtype=ref.DTYPE[fmt])
    slots = torch.arange(rows, device=DEV)
    a.append(x[0].permute(1, 0, 2)[None], x[1].permute(1, 0, 2)[None], slots)
    y = x.permute(0, 2, 1, 3).contiguous()
    b.append(y[0][None], y[1][None], slots)
    torch.cuda.synchronize()
    for s, t in ((a.k, b.k), (a.v, b.v)):
        assert torch.equal(s.view(torch.uint8), t.view(torch.uint8))
    assert torch.equal(a.k_scale, b.k_scale) and torch.equal(a.v_scale, b.v_scale)
    assert a.k_scale.gt(0).sum() == 3 * H


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("value", [math.inf, -math.inf, math.nan, 3.0e38, 1e-38, 0.0])
def test_append_extreme_values(ctx, fmt, value):
    def put(x, which):
        x[0, 0, :, 3] = value
        x[0, 1, 2, :] = value
        x[0, 2] = value
        return x
    _check_append(ctx, fmt, 1, 3, 64, 16, 4, list(range(5, 40)), None, k_values=put)


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("dim,block", [(64, 16), (128, 32), (128, 64), (256, 128), (512, 256)])
def test_append_not_finite_among_many(ctx, fmt, dim, block):
    """A NaN and infinities in long runs and in a single token of a cache in use."""
    requests = [(3, 2 * block + 5), (block - 1, 1)]

    def values(x, which):
        x[:, 0, 1, 3] = math.inf
        x[:, 1, block + 2, dim - 1] = -math.inf
        x[:, 1, block + 3, 0] = math.nan
        x[:, 0, -1, which] = math.nan
        return x

    num_blocks = sum(-(-(o + n) // block) for o, n in requests) + 1
    _check_append(ctx, fmt, 1, 2, dim, block, num_blocks, _slots_of(requests, block, num_blocks, dim), requests, k_values=values)


@pytest.mark.parametrize("fmt", FORMATS)
def test_append_skips_and_leaves_the_rest(ctx, fmt):
    slots = [-1, 3, 4, -1, 21, 22, 10 ** 12, 64, 35, 36, -5]      # four blocks: 64 is beyond the pool
    cache, before = _check_append(ctx, fmt, 1, 2, 32, 16, 4, slots, None)
    touched = torch.zeros(4, 16, dtype=torch.bool)
    for s in slots:
        if 0 <= s < 64:
            touched[s // 16, :s % 16 + 1] = True
    for t, b in ((cache.k, before[0]), (cache.v, before[1])):
        assert torch.equal(t.view(torch.uint8).cpu()[:, 0][:, :, ~touched[0]][0], b.cpu()[:, 0][:, :, ~touched[0]][0])
        assert torch.equal(t.view(torch.uint8)[3], b[3])


@pytest.mark.parametrize("fmt", FORMATS)
def test_append_token_by_token_equals_the_reference(ctx, fmt):
    """A block filled by single-token calls: scales grow as larger tokens come."""
    H, d, block = 2, 64, 16
    cache = cm.QCache(ctx, 2, block, 1, H, d, dtype=ref.DTYPE[fmt])
    g = torch.Generator().manual_seed(9)
    x = (torch.randn(2, H, 20, d, generator=g) * torch.exp2(torch.arange(20)[None, None, :, None] * 0.5 % 7)).bfloat16()
    c = [np.zeros((2, block, d)) for _ in range(2 * H)]
    s = [np.zeros(2) for _ in range(2 * H)]
    for t in range(20):
        cache.append(x[0][None, :, t:t + 1].to(DEV), x[1][None, :, t:t + 1].to(DEV), torch.tensor([t], device=DEV))
        for i in range(2 * H):
            ref.append(c[i], s[i], x[i // H, i % H, t:t + 1].double().numpy(), [t], block, fmt)
    torch.cuda.synchronize()
    for i in range(2 * H):
        codes, scale = (cache.k, cache.k_scale) if i < H else (cache.v, cache.v_scale)
        np.testing.assert_array_equal(_codes_f64(codes)[:, 0, i % H], c[i])
        np.testing.assert_array_equal(scale[:, 0, i % H].double().cpu().numpy(), s[i])


def test_append_past_32_bits(ctx):
    """Slots and code addresses beyond 2^32 bytes."""
    H, d, block = 1, 128, 16
    nb = (1 << 32) // (block * d) + 64
    cache = cm.QCache(ctx, nb, block, 1, H, d)
    x = torch.randn(1, H, 40, d).bfloat16().to(DEV)
    first = (nb - 3) * block
    cache.append(x, x, torch.arange(first, first + 40, device=DEV))
    small = cm.QCache(ctx, 3, block, 1, H, d)
    small.append(x, x, torch.arange(40, device=DEV))
    torch.cuda.synchronize()
    assert torch.equal(cache.k[-3:].view(torch.uint8), small.k.view(torch.uint8))
    assert torch.equal(cache.v_scale[-3:], small.v_scale)
    q = torch.randn(1, 2, d).bfloat16().to(DEV)
    outs = []
    for c, start in ((cache, nb - 3), (small, 0)):
        b = cm.QBatch(ctx, 1, 3, 1, block)
        b.block_table.copy_(_i32([[start, start + 1, start + 2]]))
        b.row_starts.copy_(_i32([0, 1]))
        b.kv_lens.fill_(40)
        outs.append(c.attend(q, b)[0])
    assert torch.equal(outs[0], outs[1])


# ---------------------------------------------------------------- attention

def _make_cache(ctx, fmt, layers, heads, dim, block, num_blocks, seed, order="blhtd", junk=True):
    g = torch.Generator().manual_seed(seed)
    sizes = {"b": num_blocks, "l": layers, "h": heads, "t": block, "d": dim}

    def make():
        x = torch.randn([sizes[c] for c in order], generator=g)
        t = (x * 30).round().clamp(-127, 127).to(torch.int8) if fmt == "int8" else (x * 20).clamp(-448, 448).to(torch.float8_e4m3fn)
        return t.to(DEV).permute([order.index(c) for c in "blhtd"])

    ks = (0.02 * torch.exp2(torch.randint(-2, 3, (num_blocks, layers, heads), generator=g).float())).to(DEV)
    vs = (0.05 * torch.rand((num_blocks, layers, heads), generator=g).add(0.2)).to(DEV)
    return cm.QCache.from_tensors(ctx, make(), make(), ks, vs)


def _check_attend(ctx, fmt, heads, group, dim, block, requests, causal=True, layers=1, layer=0, seed=0, order="blhtd",
                  missing=(), max_new=None, scale=None, q_scale=1.0, lse=True, extra_rows=0, heads_checked=None):
    """requests: [(tokens, query rows), ...]; missing: (request, block) entries that name no block."""
    rng = np.random.default_rng(seed)
    width = max(1, max(-(-kv // block) for kv, _ in requests)) + 1
    total = sum(-(-kv // block) for kv, _ in requests)
    cache = _make_cache(ctx, fmt, layers, heads, dim, block, total + 1, seed, order)
    ids = rng.permutation(total + 1).tolist()
    table = np.full((len(requests), width), -1)
    for r, (kv, _) in enumerate(requests):
        for b in range(-(-kv // block)):
            table[r, b] = ids.pop()
    # behind the last token of a request: NaN codes (e4m3) or the lowest value, and NaN scales in the spare block
    raw = {"k": cache.k.view(torch.uint8), "v": cache.v.view(torch.uint8)}
    for r, (kv, _) in enumerate(requests):
        if kv % block:
            for t in raw.values():
                t[int(table[r, kv // block]), :, :, kv % block:] = 0x7F if fmt == "e4m3" else 0x80
    for s in (cache.k_scale, cache.v_scale):
        s[ids[0]] = math.nan
    for r, b in missing:
        table[r, b] = [-1, total + 1, 2 ** 31 - 1][(r + b) % 3]
    n = sum(m for _, m in requests) + extra_rows
    g = torch.Generator().manual_seed(seed + 1)
    q = (torch.randn((n, heads * group, dim), generator=g) * q_scale).bfloat16().to(DEV)
    batch = cm.QBatch(ctx, len(requests), width, n, block)
    batch.block_table.copy_(torch.from_numpy(table).int())
    batch.row_starts.copy_(_i32(np.cumsum([0] + [m for _, m in requests]).tolist()))
    batch.kv_lens.copy_(_i32([kv for kv, _ in requests]))
    batch.max_new = max_new if max_new is not None else max(1, max(m for _, m in requests))
    out = torch.full_like(q, 7.0)
    got_lse = torch.full((n, heads * group), 7.0, device=DEV) if lse else None
    cache.attend(q, batch, layer=layer, out=out, lse=got_lse, causal=causal, softmax_scale=scale)
    torch.cuda.synchronize()
    f = scale if scale is not None else dim ** -0.5
    kc, vc = cache.k[:, layer].float().double().cpu(), cache.v[:, layer].float().double().cpu()
    ks, vs = cache.k_scale[:, layer].double().cpu(), cache.v_scale[:, layer].double().cpu()
    o, l, qd = out.double().cpu(), got_lse.double().cpu() if lse else None, q.double().cpu()
    at = 0
    for r, (kv, m) in enumerate(requests):
        t = np.arange(kv)
        entry = table[r, t // block]
        present = torch.from_numpy((entry >= 0) & (entry <= total))
        b, p = torch.from_numpy(entry)[present], torch.from_numpy(t % block)[present]
        # row i sees the tokens present among its first kv - m + i + 1
        seen = torch.cat([torch.zeros(1, dtype=torch.long), present.long().cumsum(0)])
        limits = [int(seen[min(kv, max(0, kv - m + i + 1)) if causal else kv]) for i in range(m)]
        for h in heads_checked or range(heads):
            k = kc[b, h, p] * ks[b, h][:, None]
            v = vc[b, h, p] * vs[b, h][:, None]
            for j in range(h * group, (h + 1) * group):
                w, wl, mag, size = ref.attend(qd[at:at + m, j], k, v, f, limits)
                err = (o[at:at + m, j] - w).abs()
                tol = w.abs() * 2 ** -8 * (1 + 2 ** -6) + (2 ** -11 + 2 ** -12 + 2 ** -19 * size) * mag
                assert bool((err <= tol).all()), (r, h, j, float((err - tol).max()), float(err.max()))
                if lse:
                    x = l[at:at + m, j]
                    fine = torch.isfinite(wl)
                    assert torch.equal(torch.isinf(x), ~fine) and not torch.isnan(x).any()
                    e = (x - wl)[fine].abs()
                    assert bool((e <= 2 ** -19 * (1 + wl[fine].abs() + size)).all()), (r, h, j, float(e.max()))
        at += m
    if extra_rows:
        assert bool((out[at:] == 7).all()) and (not lse or bool((got_lse[at:] == 7).all()))
    return cache, batch, q, out


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("heads,group,dim", [(2, 1, 32), (1, 4, 64), (2, 2, 128), (1, 5, 128), (1, 8, 256), (1, 12, 64),
                                             (1, 16, 128), (1, 16, 256)])
def test_attend_single_tokens(ctx, fmt, heads, group, dim):
    _check_attend(ctx, fmt, heads, group, dim, 16, [(1, 1), (2, 1), (15, 1), (16, 1), (17, 1), (63, 1), (64, 1), (65, 1),
                                                    (0, 1), (100, 0), (131, 1), (1000, 1)], seed=dim + group)


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("block", [16, 32, 64, 128, 256])
def test_attend_block_sizes(ctx, fmt, block):
    _check_attend(ctx, fmt, 1, 4, 64, block, [(block - 1, 1), (block, 1), (block + 1, 1), (3 * block + 7, 2)], seed=block)


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("heads,group,dim", [(2, 1, 64), (1, 4, 128), (1, 2, 256), (1, 3, 32)])
def test_attend_several_rows(ctx, fmt, causal, heads, group, dim):
    _check_attend(ctx, fmt, heads, group, dim, 16, [(70, 3), (5, 5), (200, 4), (3, 7), (0, 2), (33, 1)], causal=causal, seed=3)


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("heads,group,dim,rows,kv", [(1, 4, 128, 33, 33), (1, 4, 128, 130, 700), (2, 1, 64, 129, 129),
                                                     (1, 2, 256, 65, 200), (1, 8, 32, 40, 90), (1, 5, 128, 100, 101)])
def test_attend_prompts(ctx, fmt, heads, group, dim, rows, kv):
    _check_attend(ctx, fmt, heads, group, dim, 16, [(kv, rows), (rows - 7, rows), (kv + 11, 2)], seed=rows)


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("heads,group,dim,fmt", [(1, 1, 128, "e4m3"), (2, 3, 64, "int8"), (1, 2, 32, "e4m3"), (1, 1, 256, "int8")])
def test_attend_at_most_128_rows(ctx, heads, group, dim, fmt, causal):
    """One query tile over 0 to 7 tiles of tokens: rows that see nothing, one tile for two halves, odd counts."""
    requests = [(0, 33), (1, 40), (20, 42), (64, 33), (65, 34), (128, 42), (129, 36), (200, 35), (300, 42), (449, 33)]
    _check_attend(ctx, fmt, heads, group, dim, 16, requests, causal=causal, seed=21)


@pytest.mark.parametrize("rows", [1, 40])
def test_attend_split_long_axis(ctx, rows):
    """Few rows over many tokens: the parts of several thread blocks are joined; the same bits each time."""
    cache, batch, q, out = _check_attend(ctx, "e4m3", 2, 4, 128, 32, [(20011, rows)], heads_checked=[1], seed=5)
    for _ in range(3):
        again, _ = cache.attend(q, batch)
        assert torch.equal(again, out)


@pytest.mark.parametrize("rows", [1, 3, 50])
def test_attend_kernels_agree_with_a_wrong_expectation(ctx, rows):
    """max_new chooses the kernel only: rows beyond it are still right."""
    _check_attend(ctx, "e4m3", 1, 4, 64, 16, [(300, rows), (77, 1)], max_new=1, seed=11)
    _check_attend(ctx, "e4m3", 1, 4, 64, 16, [(300, rows), (77, 1)], max_new=1000, seed=11)


@pytest.mark.parametrize("rows", [1, 40])
def test_attend_missing_blocks(ctx, rows):
    _check_attend(ctx, "e4m3", 1, 2, 64, 16, [(100, rows), (16, 1), (90, 1)], missing=[(0, 0), (0, 3), (0, 6), (1, 0), (2, 5)], seed=2)


@pytest.mark.parametrize("rows", [1, 40])
def test_attend_layers_layouts_strides(ctx, rows):
    _check_attend(ctx, "e4m3", 2, 2, 64, 16, [(100, rows), (33, 1)], layers=3, layer=2, seed=6)
    _check_attend(ctx, "int8", 2, 2, 64, 32, [(100, rows), (33, 1)], layers=2, layer=1, order="lbthd", seed=6, extra_rows=3)
    _check_attend(ctx, "e4m3", 3, 2, 32, 16, [(100, rows), (33, 1)], order="hblt" + "d", seed=6, lse=False)


@pytest.mark.parametrize("rows", [1, 40])
@pytest.mark.parametrize("q_scale,scale", [(1e-30, 1e28), (1e20, 1e-21), (1.0, 0.0), (4.0, 3.0), (1.0, -0.2)])
def test_attend_query_and_score_ranges(ctx, rows, q_scale, scale):
    _check_attend(ctx, "e4m3", 1, 2, 64, 16, [(300, rows), (7, 1)], q_scale=q_scale, scale=scale, seed=8)


@pytest.mark.parametrize("rows", [1, 40])
def test_attend_block_scales_far_apart(ctx, rows):
    """V scales from 2^-60 to 2^60 and K scales of zero."""
    cache, batch, q, _ = _check_attend(ctx, "int8", 1, 2, 64, 16, [(160, rows)], seed=12)
    exps = [-60, 60, 0, -30, 5, -60, -1, 40, 2, -7, 0]
    for i, e in enumerate(exps):
        cache.v_scale[i] = 2.0 ** e
    cache.k_scale[2] = 0.0
    lse = torch.empty(q.shape[:2], device=DEV)
    out, _ = cache.attend(q, batch, lse=lse)
    torch.cuda.synchronize()
    b = batch.block_table[0].long().cpu()[torch.arange(160) // 16]
    p = torch.arange(160) % 16
    k = cache.k[:, 0, 0].double().cpu()[b, p] * cache.k_scale[:, 0, 0].double().cpu()[b][:, None]
    v = cache.v[:, 0, 0].double().cpu()[b, p] * cache.v_scale[:, 0, 0].double().cpu()[b][:, None]
    limits = [160 - rows + i + 1 for i in range(rows)]
    for j in range(2):
        w, wl, mag, size = ref.attend(q[:, j].double().cpu(), k, v, 64 ** -0.5, limits)
        err = (out[:, j].double().cpu() - w).abs()
        assert bool((err <= w.abs() * 2 ** -8 * (1 + 2 ** -6) + (2 ** -11 + 2 ** -12 + 2 ** -19 * size) * mag).all())
        assert bool(((lse[:, j].double().cpu() - wl).abs() <= 2 ** -19 * (1 + wl.abs() + size)).all())


def test_attend_on_another_stream_and_in_a_graph(ctx):
    cache, batch, q, out = _check_attend(ctx, "e4m3", 2, 4, 64, 16, [(900, 1), (70, 1), (5, 1)], seed=21)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    mine = torch.zeros_like(out)
    with torch.cuda.stream(side):
        cache.attend(q, batch, out=mine)
    side.synchronize()
    assert torch.equal(mine, out)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        cache.attend(q, batch, out=mine)
    for _ in range(3):
        mine.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(mine, out)


# ---------------------------------------------------------------- refusals

def test_attend_one_batch_for_several_head_dims(ctx):
    """A batch's workspace serves caches of any head_dim, in any order: same bits as with a batch of its own."""
    caches = [_make_cache(ctx, "e4m3", 1, 1, d, 16, 160, d) for d in (256, 128, 64)]
    g = torch.Generator().manual_seed(3)

    def batch(rows):
        b = cm.QBatch(ctx, 1, 160, rows, 16)
        b.block_table.copy_(torch.arange(160)[None].int())
        b.row_starts.copy_(_i32([0, rows]))
        b.kv_lens.fill_(2500)
        b.max_new = rows
        return b

    for rows in (1, 40):
        queries = [torch.randn((rows, 4, c.k.shape[4]), generator=g).bfloat16().to(DEV) for c in caches]
        own = [c.attend(q, batch(rows))[0] for c, q in zip(caches, queries)]
        shared = batch(rows)
        for i in (0, 1, 2, 1, 0, 2, 0, 1):
            out = caches[i].attend(queries[i], shared)[0]
            assert torch.equal(out, own[i])


def test_refusals(ctx):
    cache = cm.QCache(ctx, 4, 16, 2, 2, 64)
    batch = cm.QBatch(ctx, 2, 4, 8, 16)
    q = torch.zeros(3, 4, 64, dtype=torch.bfloat16, device=DEV)
    good = torch.zeros(1, 2, 3, 64, dtype=torch.bfloat16, device=DEV)
    slots = torch.zeros(3, dtype=torch.int64, device=DEV)
    for bad in (lambda: cache.append(good.float(), good.float(), slots),
                lambda: cache.append(good, good[:, :1], slots),
                lambda: cache.append(good, good, slots.int()),
                lambda: cache.append(good, good, torch.zeros(4, dtype=torch.int64, device=DEV)),
                lambda: cache.append(good.cpu(), good.cpu(), slots),
                lambda: cache.attend(q.float(), batch), lambda: cache.attend(q[..., :32], batch),
                lambda: cache.attend(q, batch, out=q[:2]), lambda: cache.attend(q, batch, lse=torch.zeros(3, 5, device=DEV)),
                lambda: batch.schedule(_i32([1]), _i32([1, 1]), _i32([0])),
                lambda: batch.schedule(torch.zeros(2, device=DEV), _i32([1, 1]), _i32([0])),
                lambda: cm.QCache(ctx, 4, 16, 2, 2, 64, dtype=torch.bfloat16),
                lambda: cm.QCache.from_tensors(ctx, cache.k, cache.v[:2], cache.k_scale, cache.v_scale)):
        with pytest.raises(ValueError):
            bad()
    S = cm.Status
    for status, bad in (
            (S.ERR_INVALID_ARG, lambda: cache.append(good, good, slots, layer=2)),
            (S.ERR_INVALID_ARG, lambda: cache.append(good, good, slots, layer=-1)),
            (S.ERR_INVALID_ARG, lambda: cache.attend(q, batch, layer=2)),
            (S.ERR_INVALID_ARG, lambda: cache.attend(q, batch, softmax_scale=math.inf)),
            (S.ERR_SHAPE_MISMATCH, lambda: cache.attend(q[:, :3], batch)),
            (S.ERR_SHAPE_MISMATCH, lambda: cache.attend(q, cm.QBatch(ctx, 2, 4, 8, 32))),
            (S.ERR_UNSUPPORTED, lambda: cache.attend(q, cm.QBatch(ctx, 4097, 1, 8, 16))),
            (S.ERR_UNSUPPORTED, lambda: cm.QBatch(ctx, 1, 1, 1, 24).schedule(_i32([1]), _i32([1]), _i32([0]))),
            (S.ERR_UNSUPPORTED, lambda: cm.QCache(ctx, 4, 8, 1, 1, 64).append(good[:, :1], good[:, :1], slots)),
            (S.ERR_INVALID_ARG, lambda: cm.QCache(ctx, 4, 16, 1, 1, 48).append(good[:, :1, :, :48], good[:, :1, :, :48], slots)),
            (S.ERR_UNSUPPORTED, lambda: cm.QCache(ctx, 4, 16, 1, 1, 16).attend(q[:, :1, :16], batch)),
            (S.ERR_ALIGNMENT, lambda: cache.attend(torch.zeros(3 * 4 * 64 + 1, dtype=torch.bfloat16, device=DEV)[1:].view(3, 4, 64), batch)),
            (S.ERR_INVALID_ARG, lambda: batch.schedule(batch.kv_lens, _i32([1, 1]), _i32([0])))):
        with pytest.raises(cm.CMError) as e:
            bad()
        assert e.value.status == status, (status, str(e.value))
    # nothing to do is no error
    cache.append(good[:, :, :0], good[:, :, :0], slots[:0])
    cache.attend(q[:0], batch)


@pytest.mark.parametrize("rows", [1, 40])
def test_steps_in_a_row_equal_steps_with_waits_between(ctx, rows):
    """Each call reads what the one before it wrote (tables, slots, codes, scales), with nothing between them that
    waits: the same bits as with a synchronisation after every call."""
    R, H, G, d, block, steps = 5, 2, 4, 64, 16, 24
    width = -(-(steps * rows + 200) // block)

    def run(wait):
        g = torch.Generator(device=DEV).manual_seed(17)
        cache = cm.QCache(ctx, R * width, block, 1, H, d)
        b = cm.QBatch(ctx, R, width, R * rows, block)
        b.max_new = rows
        free = torch.randperm(R * width, generator=torch.Generator().manual_seed(3)).int().to(DEV)
        held = [3 * r for r in range(R)]
        first = cm.QBatch(ctx, R, width, sum(held), block)
        first.schedule(_i32([0] * R), _i32(held), free)
        free = free[sum(-(-h // block) for h in held):].contiguous()
        b.block_table.copy_(first.block_table)
        x = torch.randn((2, 1, H, sum(held), d), generator=g, device=DEV).bfloat16()
        cache.append(x[0], x[1], first.slot_map)
        lens, new = _i32(held), _i32([rows] * R)
        inputs = [torch.randn((2, 1, H, R * rows, d), generator=g, device=DEV).bfloat16() for _ in range(steps)]
        queries = [torch.randn((R * rows, H * G, d), generator=g, device=DEV).bfloat16() for _ in range(steps)]
        frees = []
        for _ in range(steps):
            frees.append(free)
            free = free[sum(-(-(h + rows) // block) - -(-h // block) for h in held):].contiguous()
            held = [h + rows for h in held]
        lengths = [lens + t * rows for t in range(steps)]
        torch.cuda.synchronize()
        outs = []
        for t in range(steps):
            b.schedule(lengths[t], new, frees[t])
            if wait:
                torch.cuda.synchronize()
            cache.append(inputs[t][0], inputs[t][1], b.slot_map)
            if wait:
                torch.cuda.synchronize()
            outs.append(cache.attend(queries[t], b)[0])
            if wait:
                torch.cuda.synchronize()
        ctx.check()
        return outs

    for a, c in zip(run(True), run(False)):
        assert torch.equal(a, c)


@pytest.mark.parametrize("fmt", FORMATS)
def test_example_answers_from_merged_caches(fmt):
    """Render, schedule, append and attend together. A value's rounding is at most 2^-4 of it (e4m3, three bits
    behind the point) or 2^-6 of its block's largest (int8, power-of-two scale: up to 1 / 64), so an element is off
    by no more than 1 / 16 of a typical one, K and V each; three times both bounds any row's result."""
    path = os.path.join(os.path.dirname(os.path.abspath(__file__)), "..", "examples", "answer_from_merge.py")
    spec = importlib.util.spec_from_file_location("answer_from_merge", path)
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    r = example.main(requests=3, layers=2, kv_heads=2, group=4, dim=64, tokens=(20, 130), question=21, steps=3, fmt=fmt)
    assert r["merged_tokens"] > 3 * 40
    assert 0.0 < r["relative_error"] < 3 * 2 / 16
