"""The operators around a tree of drafted tokens on the GPU against their definitions (tree_reference.py).

Masks, positions, accepted paths, chosen tokens, moved codes and scales are compared exactly.

Norm and rotation, from how they are computed: one rounding to bf16 (2^-8 of the result); in fp32 the norm (at most 20 additions in a row,
rsqrt to 2^-22, three products: 2^-20 of y together), the angle (2^-25 half turns from its rounding to fp32, 2^-23 from sincospi, at the farthest
positions 2^-23 turns from the frequency's) and two products and a sum, all times |y_j| + |y_(j + d/2)|. Hence
    |out - ref| <= 2^-8 |ref| + 2^-18 (|y_j| + |y_(j + d/2)|)

Attention: as in test_gpu_qcache.py (the same kernels' arithmetic):
    |out - ref| <= 2^-8 |ref| * (1 + 2^-6) + (2^-11 + 2^-12 + 2^-19 size) * sum p |v|
    |lse - ref| <= 2^-19 * (1 + |ref| + size)
"""
import math

import numpy as np
import pytest
import torch

import tree_reference as ref

pytestmark = pytest.mark.gpu

cm = pytest.importorskip("paper_2607_01308_gb300")

DEV = "cuda:0"
THETA = 1.0e6


@pytest.fixture(scope="module")
def ctx():
    c = cm.Context(0, rope_theta=THETA)
    yield c
    c.close()


def _i32(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


def _trees(rng, sizes, fan=3):
    """Parents of random trees of those sizes."""
    out = []
    for n in sizes:
        out.append([-1] + [int(rng.integers(max(0, i - 2 * fan), i)) for i in range(1, n)] if n else [])
    return out


def _starts(sizes):
    return [0] + np.cumsum(sizes).tolist() if len(sizes) else [0]


def _batch(ctx, sizes, width=0, block=16, rows=None):
    rows = sum(sizes) if rows is None else rows
    batch = cm.QBatch(ctx, len(sizes), width, rows, block)
    batch.row_starts.copy_(_i32(_starts(sizes)))
    return batch


# ---------------------------------------------------------------- masks and positions

def _check_plan(ctx, sizes, context, parents, max_nodes, rows=None, batch=None):
    batch = batch or _batch(ctx, sizes, rows=rows)
    tree = cm.QTree(batch, max_nodes)
    tree.mask.fill_(77)
    tree.positions.fill_(-5)
    tree.plan(None if parents is None else _i32(parents), _i32(context))
    torch.cuda.synchronize()
    words = tree.mask.shape[1]
    masks, positions = ref.plan(_starts(sizes), context, parents, tree.mask.shape[0], words)
    got = [sum((int(w) & 0xffffffff) << 32 * k for k, w in enumerate(m)) for m in tree.mask.tolist()]
    untouched = sum(77 << 32 * k for k in range(words))
    limit = (1 << 32 * words) - 1
    assert got == [untouched if m is None else m & limit for m in masks]
    assert tree.positions.tolist() == [-5 if x is None else x for x in positions]


@pytest.mark.parametrize("sizes", [[1], [2], [31, 32, 33], [0, 5, 0, 0, 1], [64, 65, 1, 96], [255, 256], [7] * 40])
def test_plan_trees(ctx, sizes):
    rng = np.random.default_rng(len(sizes))
    parents = [p for t in _trees(rng, sizes) for p in t]
    _check_plan(ctx, sizes, rng.integers(0, 100000, len(sizes)).tolist(), parents, max(1, max(sizes)))


def test_plan_chains_and_stars_and_forests(ctx):
    n = 256
    _check_plan(ctx, [n, n, n], [0, 5, 2 ** 31 - 100], list(range(-1, n - 1)) + [-1] + [0] * (n - 1) + [-1] * n, n)


def test_plan_parents_that_are_none(ctx):
    parents = [0, 1, 5, -7, 3, 2 ** 31 - 1, -2 ** 31, 6]       # its own row, a later one, far outside
    _check_plan(ctx, [8], [3], parents, 8)


@pytest.mark.parametrize("max_nodes", [1, 32, 40, 256])
def test_plan_rows_behind_the_trees(ctx, max_nodes):
    rng = np.random.default_rng(3)
    sizes = [300, 10, 70]
    _check_plan(ctx, sizes, [9, -4, 0], [p for t in _trees(rng, sizes) for p in t], max_nodes)
    _check_plan(ctx, sizes, [9, -4, 2 ** 31 - 200], None, max_nodes)


def test_plan_long_rows_without_parents(ctx):
    _check_plan(ctx, [9000, 1, 4097], [1, 2, 3], None, 33)


def test_plan_leaves_rows_of_no_request(ctx):
    _check_plan(ctx, [4, 2], [1, 2], [-1, 0, 1, 1, -1, 0, -1, -1, 4], 32, rows=9)
    _check_plan(ctx, [0, 0], [1, 2], [-1, 0], 32, rows=2)


def test_plan_fewer_parents_than_rows(ctx):
    batch = _batch(ctx, [4, 2], rows=6)
    tree = cm.QTree(batch, 8)
    tree.mask.fill_(7)
    tree.plan(_i32([-1, 0, 1]), _i32([5, 6]))                  # the rows behind them are none
    assert tree.mask[:, 0].tolist() == [1, 3, 7, 7, 7, 7] and tree.positions.tolist()[:3] == [5, 6, 7]


def test_plan_many_requests(ctx):
    rng = np.random.default_rng(4)
    sizes = rng.integers(0, 4, 16384).tolist()
    _check_plan(ctx, sizes, rng.integers(0, 1000, 16384).tolist(), [p for t in _trees(rng, sizes) for p in t], 3)


def test_plan_row_starts_that_descend(ctx):
    batch = cm.QBatch(ctx, 3, 0, 6, 16)
    batch.row_starts.copy_(_i32([4, 2, -3, 100]))              # rows of no request, then rows 0 .. 5 of the last
    tree = cm.QTree(batch, 8)
    tree.plan(_i32([-1, 0, 1, 0, 3, -1]), _i32([1, 1, 10]))
    assert tree.mask[:, 0].tolist() == [1, 3, 7, 9, 25, 32] and tree.positions.tolist() == [10, 11, 12, 11, 12, 10]


# ---------------------------------------------------------------- norm and rotation

def _check_rotate(ctx, x, got, positions, weight, eps, theta=THETA):
    w = None if weight is None else weight.double().cpu().numpy()
    want, size = ref.rotate(x.double().cpu().numpy(), positions.cpu().numpy(), w, eps, theta)
    err = np.abs(got.double().cpu().numpy() - want)
    tol = 2.0 ** -8 * np.abs(want) + 2.0 ** -18 * size
    assert np.all(err <= tol), (err / np.maximum(tol, 1e-300)).max()


@pytest.mark.parametrize("d", [16, 32, 64, 128, 256, 512])
@pytest.mark.parametrize("rows,hq,hk", [(1, 1, 1), (1, 32, 8), (7, 5, 3), (130, 3, 1), (1, 0, 4), (3, 2, 0)])
@pytest.mark.parametrize("norm", [True, False])
def test_rotate(ctx, d, rows, hq, hk, norm):
    g = torch.Generator(device=DEV).manual_seed(d + rows)
    qkv = (torch.randn((rows, hq + 2 * hk, d), generator=g, device=DEV) * 3).bfloat16()
    q, k = qkv[:, :hq] if hq else None, qkv[:, hq:hq + hk] if hk else None
    before = qkv.clone()
    wq, wk = ((1 + torch.randn(d, generator=g, device=DEV)).bfloat16() if norm and n else None for n in (hq, hk))
    pos = torch.randint(0, 200000, (rows,), generator=g, device=DEV, dtype=torch.int32)
    oq, ok = cm.rotate_qk(ctx, q, k, pos, wq, wk, eps=1e-6)
    for x, o, w in ((q, oq, wq), (k, ok, wk)):
        if x is None:
            assert o is None
        else:
            _check_rotate(ctx, x, o, pos, w, 1e-6)
    assert torch.equal(qkv, before)


def test_rotate_one_weight_alone(ctx):
    g = torch.Generator(device=DEV).manual_seed(1)
    q, k = (torch.randn((9, h, 64), generator=g, device=DEV).bfloat16() for h in (5, 2))
    w = torch.randn(64, generator=g, device=DEV).bfloat16()
    pos = torch.arange(9, dtype=torch.int32, device=DEV)
    for wq, wk in ((w, None), (None, w)):
        oq, ok = cm.rotate_qk(ctx, q, k, pos, wq, wk)
        _check_rotate(ctx, q, oq, pos, wq, 1e-6)
        _check_rotate(ctx, k, ok, pos, wk, 1e-6)


def test_rotate_far_and_negative_positions(ctx):
    pos = _i32([0, 1, -1, 2 ** 20, 2 ** 24 + 1, -2 ** 24 - 3, 2 ** 31 - 1, -2 ** 31, 123456789])
    g = torch.Generator(device=DEV).manual_seed(2)
    q = torch.randn((9, 3, 128), generator=g, device=DEV).bfloat16()
    o, _ = cm.rotate_qk(ctx, q, None, pos)
    _check_rotate(ctx, q, o, pos, None, 0)
    for theta in (1e4, 0.5):                                   # below 1: several turns a position
        c = cm.Context(0, rope_theta=theta)
        o, _ = cm.rotate_qk(c, q[:4], None, pos[:4])
        _check_rotate(c, q[:4], o, pos[:4], None, 0, theta)
        c.close()


def test_rotate_in_place_and_padded_rows(ctx):
    g = torch.Generator(device=DEV).manual_seed(3)
    for rows in (1, 37, 700):
        base = torch.randn((rows, 12, 96), generator=g, device=DEV).bfloat16()
        q, k = base[:, 1:9, 16:80], base[:, 9:11, 16:80]       # head_dim 64 within rows of 96
        w = torch.randn(64, generator=g, device=DEV).bfloat16()
        pos = torch.randint(0, 5000, (rows,), generator=g, device=DEV, dtype=torch.int32)
        want = cm.rotate_qk(ctx, q, k, pos, w, w)
        kept = base.clone()
        oq, ok = cm.rotate_qk(ctx, q, k, pos, w, w, q_out=q, k_out=k)
        assert oq is q and ok is k
        assert torch.equal(q, want[0]) and torch.equal(k, want[1])
        base[:, 1:11, 16:80] = kept[:, 1:11, 16:80]
        assert torch.equal(base, kept)                         # nothing around them


def test_rotate_heads_first_outputs_and_shared_inputs(ctx):
    g = torch.Generator(device=DEV).manual_seed(4)
    k = torch.randn((1, 4, 128), generator=g, device=DEV).bfloat16()
    pos = torch.arange(50, dtype=torch.int32, device=DEV)
    out = torch.empty((4, 60, 128), dtype=torch.bfloat16, device=DEV)
    out.fill_(5)
    cm.rotate_qk(ctx, None, k.expand(50, 4, 128), pos, k_out=out[:, :50].transpose(0, 1))    # one row at 50 positions
    _check_rotate(ctx, k.expand(50, 4, 128), out[:, :50].transpose(0, 1), pos, None, 0)
    assert bool((out[:, 50:] == 5).all())


def test_rotate_special_values(ctx):
    q = torch.zeros((4, 2, 32), dtype=torch.bfloat16, device=DEV)
    q[1, 0, 3] = float("nan")
    q[2, 1, 30] = float("inf")
    q[3] = 1e-30
    w = torch.ones(32, dtype=torch.bfloat16, device=DEV)
    pos = _i32([5, 6, 7, 8])
    o, _ = cm.rotate_qk(ctx, q, None, pos, w, eps=0.0)
    assert bool((o[0] == 0).all()) and bool((o[1, 1] == 0).all()) and bool((o[2, 0] == 0).all())   # 0 / 0 is 0
    assert bool(o[1, 0].isnan().all()) and bool(o[2, 1, [14, 30]].isnan().all())
    o, _ = cm.rotate_qk(ctx, q, None, pos)                     # without a norm only the pair is lost
    assert o[1, 0].isnan().nonzero().flatten().tolist() == [3, 19] and not bool(o[1, 1].isnan().any())


def test_rotate_no_rows(ctx):
    q = torch.empty((0, 4, 64), dtype=torch.bfloat16, device=DEV)
    o, k = cm.rotate_qk(ctx, q, q, torch.empty(0, dtype=torch.int32, device=DEV))
    assert o.shape == q.shape and k.shape == q.shape


def test_rotate_many_rows(ctx):
    g = torch.Generator(device=DEV).manual_seed(5)
    qkv = torch.randn((5003, 24, 64), generator=g, device=DEV).bfloat16()
    w = torch.randn(64, generator=g, device=DEV).bfloat16()
    pos = torch.randint(0, 1000000, (5003,), generator=g, device=DEV, dtype=torch.int32)
    q, k = qkv[:, :15], qkv[:, 15:20]
    oq, ok = cm.rotate_qk(ctx, q, k, pos, w, None)
    _check_rotate(ctx, q, oq, pos, w, 1e-6)
    _check_rotate(ctx, k, ok, pos, None, 1e-6)


# ---------------------------------------------------------------- attention

def _cache(ctx, blocks, layers, heads, block, d, fmt, seed, spread=3):
    g = torch.Generator(device=DEV).manual_seed(seed)
    shape = (blocks, layers, heads, block, d)

    def codes():
        x = torch.randn(shape, generator=g, device=DEV)
        return (x * 40).clamp(-127, 127).round().to(torch.int8) if fmt == "int8" else (x * 60).to(torch.float8_e4m3fn)

    def scales():
        return torch.exp2(torch.randint(-6 - spread, -5, shape[:3], generator=g, device=DEV).float())

    return cm.QCache.from_tensors(ctx, codes(), codes(), scales(), scales())


def _values(cache, table, layer, head, tokens):
    blocks = table[:-(-tokens // cache.k.shape[3])].long()
    return [(c[blocks, layer, head].double() * s[blocks, layer, head].double()[:, None, None]).reshape(-1, c.shape[-1])[:tokens].cpu()
            for c, s in ((cache.k, cache.k_scale), (cache.v, cache.v_scale))]


def _seen(context, n, mask_rows, kv):
    """[n, kv] of truth values from the masks (whole numbers) of a request's rows."""
    seen = torch.zeros((n, kv), dtype=torch.bool)
    seen[:, :max(0, context)] = True
    for i in range(n):
        for j in range(n):
            if mask_rows[i] >> j & 1 and 0 <= context + j < kv:
                seen[i, context + j] = True
    return seen


def _check_attend(cache, q, out, lse, table, kv, starts, seen, group, layer, scale):
    for r, visible in enumerate(seen):
        a, b = starts[r], starts[r + 1]
        for h in range(cache.k.shape[2]):
            k, v = _values(cache, table[r], layer, h, kv[r])
            for g in range(group):
                x = q[a:b, h * group + g].double().cpu()
                if kv[r] == 0:
                    assert bool((out[a:b, h * group + g] == 0).all()) and bool((lse[a:b, h * group + g] == -math.inf).all())
                    continue
                s = (x @ k.T) * scale
                size = float(((x.abs() @ k.T.abs()) * abs(scale)).max()) if s.numel() else 0.0
                s = s.masked_fill(~visible, -math.inf)
                want_lse = torch.logsumexp(s, -1)
                p = torch.where(visible, torch.exp(s - torch.where(want_lse.isinf(), 0.0, want_lse)[:, None]), 0.0)
                want, mag = p @ v, p @ v.abs()
                got = out[a:b, h * group + g].double().cpu()
                tol = 2.0 ** -8 * want.abs() * (1 + 2.0 ** -6) + (2.0 ** -11 + 2.0 ** -12 + 2.0 ** -19 * size) * mag
                assert bool(((got - want).abs() <= tol).all()), (r, h, g, float(((got - want).abs() / tol.clamp(min=1e-30)).max()))
                got = lse[a:b, h * group + g].double().cpu()
                empty = ~visible.any(-1)
                assert torch.equal(got == -math.inf, empty)
                err = (got - want_lse)[~empty].abs()
                assert bool((err <= 2.0 ** -19 * (1 + want_lse[~empty].abs() + size)).all())


def _attend_case(ctx, context, sizes, heads, group, d, fmt, block=16, max_nodes=None, masks=None, layers=1, max_new=None, seed=0,
                 scale=None, cut=None, kv=None):
    rng = np.random.default_rng(seed)
    kv = [c + n for c, n in zip(context, sizes)] if kv is None else kv
    need = [-(-max(1, k) // block) for k in kv]
    width = max(need) + 1
    order = torch.randperm(sum(need) + 3, generator=torch.Generator().manual_seed(seed)).int()
    table, at = torch.full((len(sizes), width), -1, dtype=torch.int32), 0
    for r, n in enumerate(need):
        table[r, :n] = order[at:at + n]
        at += n
    table = table.to(DEV)
    cache = _cache(ctx, sum(need) + 3, layers, heads, block, d, fmt, seed)
    batch = _batch(ctx, sizes, width, block)
    batch.block_table.copy_(table)
    batch.kv_lens.copy_(_i32(kv))
    if cut is not None:
        batch.context_lens.copy_(_i32(cut))
    batch.max_new = max(sizes) if max_new is None else max_new
    tree = cm.QTree(batch, max_nodes or max(sizes))
    words = tree.mask.shape[1]
    if masks is None:
        parents = [p for t in _trees(rng, sizes) for p in t]
        masks, _ = ref.plan(_starts(sizes), context, parents, sum(sizes), words)
        tree.plan(_i32(parents), _i32(context))
    else:
        words_of = np.array([[m >> 32 * w & 0xffffffff for w in range(words)] for m in masks], dtype=np.uint32)
        tree.mask.copy_(torch.from_numpy(words_of.view(np.int32)))
    g = torch.Generator(device=DEV).manual_seed(seed + 1)
    q = torch.randn((sum(sizes), heads * group, d), generator=g, device=DEV).bfloat16()
    lse = torch.full(q.shape[:2], 99.0, device=DEV)
    scale = d ** -0.5 if scale is None else scale
    layer = layers - 1
    out, _ = cache.attend(q, batch, layer=layer, lse=lse, tree=tree, softmax_scale=scale)
    torch.cuda.synchronize()
    ctx.check()
    starts = _starts(sizes)
    limit = (1 << 32 * words) - 1
    seen = [_seen(c, n, [m & limit for m in masks[a:a + n]], k) for c, n, a, k in zip(context, sizes, starts, kv)]
    _check_attend(cache, q, out, lse, table, kv, starts, seen, group, layer, scale)
    return cache, batch, tree, q, out, lse


@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
@pytest.mark.parametrize("d", [32, 64, 128, 256])
@pytest.mark.parametrize("group,sizes,context", [
    (1, [1], [0]), (2, [5], [40]), (1, [8, 3, 1], [0, 63, 64]), (4, [4, 2], [17, 200]),          # few rows
    (4, [9, 26], [100, 0]), (8, [33], [70]), (5, [40, 1, 60], [1, 128, 5])])                       # many
def test_attend_trees(ctx, fmt, d, group, sizes, context):
    _attend_case(ctx, context, sizes, 2, group, d, fmt, seed=d + group)


@pytest.mark.parametrize("block", [16, 32, 64, 128, 256])
@pytest.mark.parametrize("group", [1, 4])
def test_attend_blocks(ctx, block, group):
    _attend_case(ctx, [block - 3, 2 * block, 1, 5 * block + 1], [7, 20, 12, 9], 2, group, 64, "e4m3", block=block, layers=2, seed=block)


@pytest.mark.parametrize("context", list(range(40, 90, 7)) + [63, 64, 65])
@pytest.mark.parametrize("nodes,group", [(8, 1), (6, 2), (64, 2)])
def test_attend_borders_of_tiles(ctx, context, nodes, group):
    _attend_case(ctx, [context], [nodes], 1, group, 128, "e4m3", seed=context)


@pytest.mark.parametrize("nodes,max_nodes", [(256, 256), (130, 160), (200, 40)])
@pytest.mark.parametrize("group,d", [(1, 64), (2, 128)])
def test_attend_large_trees(ctx, nodes, max_nodes, group, d):
    _attend_case(ctx, [77, 0], [nodes, 3], 2, group, d, "int8", max_nodes=max_nodes, seed=nodes)


@pytest.mark.parametrize("max_new", [1, 20, 100])               # few rows, one tile of queries, two
@pytest.mark.parametrize("d", [64, 128])
def test_attend_any_masks(ctx, max_new, d):
    """Masks that no tree has: nothing at all, later rows, bits beyond the rows, all."""
    rng = np.random.default_rng(5)
    masks = [0, 0, 0b10, (1 << 64) - 1, 1 << 40] + [int(x) for x in rng.integers(0, 1 << 62, 12)] + [0]
    _attend_case(ctx, [0, 33, 0], [5, 12, 1], 2, 2, d, "e4m3", max_nodes=64, masks=masks, max_new=max_new)


@pytest.mark.parametrize("max_new", [1, 20, 100])
def test_attend_rows_without_tokens(ctx, max_new):
    """Fewer tokens than rows: row i of n is token kv - n + i, and the first ones are not there."""
    cache, batch, tree, q, out, lse = _attend_case(ctx, [-3, -4], [6, 4], 1, 2, 64, "int8", kv=[3, 0], max_nodes=32,
                                                   masks=[0b111111] * 6 + [0b1111] * 4, max_new=max_new)
    assert bool((out[6:] == 0).all()) and bool((lse[6:] == -math.inf).all())


@pytest.mark.parametrize("max_new", [1, 20, 100])
def test_attend_requests_that_were_cut(ctx, max_new):
    """context_lens says where the rows of a request begin whose table ended before them."""
    _attend_case(ctx, [20, 10], [9, 7], 1, 2, 128, "e4m3", kv=[24, 17], cut=[20, -1], max_new=max_new,
                 masks=[0b1, 0b11, 0b111, 0b1111, 0b11111, 0b111111111, 0, 0b100000000, 0b10] + [1, 3, 5, 9, 17, 33, 65], max_nodes=9)


@pytest.mark.parametrize("max_new", [1, 20, 100])
@pytest.mark.parametrize("scale", [-0.3, 0.0])
def test_attend_scales(ctx, max_new, scale):
    _attend_case(ctx, [50], [11], 2, 2, 64, "e4m3", max_new=max_new, scale=scale)


@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
@pytest.mark.parametrize("group,nodes", [(1, 7), (4, 26)])
def test_attend_many_requests_and_long_ones(ctx, fmt, group, nodes):
    rng = np.random.default_rng(group)
    sizes = rng.integers(1, nodes + 1, 60).tolist()
    context = rng.integers(0, 300, 59).tolist() + [9001]
    _attend_case(ctx, context, sizes, 1, group, 128, fmt, seed=nodes)


def test_attend_a_chain_is_causal(ctx):
    """With masks of chains, to few rows the same kernel on the same tiles: bit for bit what causal attention gives."""
    cache, batch, tree, q, _, _ = _attend_case(ctx, [70, 0, 5], [4, 3, 8], 2, 1, 128, "e4m3", seed=9)
    tree.plan(None, _i32([70, 0, 5]))
    lse, lse2 = (torch.empty(q.shape[:2], device=DEV) for _ in range(2))
    a, _ = cache.attend(q, batch, tree=tree, lse=lse)
    b, _ = cache.attend(q, batch, lse=lse2)
    assert torch.equal(a, b) and torch.equal(lse, lse2)


def test_attend_leaves_rows_of_no_request_and_ignores_junk(ctx):
    cache, batch, tree, q, out, lse = _attend_case(ctx, [30, 90], [5, 6], 2, 2, 64, "e4m3", seed=11)
    batch.row_starts.copy_(_i32([0, 3, 9]))                    # rows 9 and 10 are no one's
    batch.kv_lens.copy_(_i32([33, 96]))
    raw = [t.view(torch.uint8) for t in (cache.k, cache.v)]
    first, _ = cache.attend(q, batch, tree=tree)
    for r, kv in enumerate([33, 96]):                          # NaN codes behind the last token
        b = int(batch.block_table[r, (kv - 1) // 16])
        for t in raw:
            t[b, :, :, (kv - 1) % 16 + 1:] = 0x7f
    mine = torch.full_like(q, 7.0)
    cache.attend(q, batch, tree=tree, out=mine)
    assert torch.equal(mine[:9], first[:9]) and bool((mine[9:] == 7.0).all())


def test_attend_missing_blocks(ctx):
    """Tokens whose table entry names no block are not attended, in the context or among the rows."""
    for max_new in (1, 40, 200):
        cache, batch, tree, q, _, _ = _attend_case(ctx, [60], [20], 1, 1, 64, "e4m3", seed=12, max_new=max_new)
        batch.block_table[0, 1] = -1
        batch.block_table[0, 4] = 10 ** 6                      # tokens 64 .. 79: rows 4 on
        lse = torch.empty(q.shape[:2], device=DEV)
        out, _ = cache.attend(q, batch, tree=tree, lse=lse)
        keep = torch.ones(80, dtype=torch.bool)
        keep[16:32] = False
        keep[64:] = False
        masks = [int(m) & 0xffffffff for m in tree.mask[:, 0].tolist()]
        table = batch.block_table.clamp(0, cache.k.shape[0] - 1)
        _check_attend(cache, q, out, lse, table, [80], [0, 20], [_seen(60, 20, masks, 80) & keep], 1, 0, 64 ** -0.5)


# ---------------------------------------------------------------- verification

def _check_verify(ctx, sizes, parents, tokens, target, draft, accept, sample, max_nodes=256, rows=None):
    batch = _batch(ctx, sizes, rows=rows)
    tree = cm.QTree(batch, max_nodes)
    for t in (tree.path, tree.kept, tree.next_token):
        t.fill_(-9)
    tree.verify(_i32(parents), _i32(tokens), target, accept.to(DEV), sample.to(DEV), draft=draft)
    torch.cuda.synchronize()
    host = [None if t is None else t.float().cpu().numpy() for t in (target, draft)]
    path, kept, chosen = ref.verify(_starts(sizes), parents, tokens, host[0], host[1], accept.numpy(), sample.numpy(), max_nodes)
    assert tree.kept.tolist() == kept
    assert tree.next_token.tolist() == chosen
    assert tree.path.tolist() == path + [-9] * (tree.path.numel() - len(path))
    return kept, chosen


def _probabilities(rows, vocab, seed, dtype=torch.float32, sharp=3.0, agree=0.7):
    g = torch.Generator(device=DEV).manual_seed(seed)
    x = torch.randn((rows, vocab), generator=g, device=DEV) * sharp
    y = 0.9 * x + agree * torch.randn((rows, vocab), generator=g, device=DEV)
    return torch.softmax(x, -1).to(dtype), torch.softmax(y, -1).to(dtype)


def _drawn(sizes, parents, draft, seed):
    """Tokens drawn from their parents' rows of draft."""
    base = np.repeat(_starts(sizes)[:-1], sizes)
    at = torch.tensor([b + max(p, 0) for b, p in zip(base, parents)], device=DEV)
    g = torch.Generator(device=DEV).manual_seed(seed)
    return torch.multinomial(draft.float()[at], 1, generator=g)[:, 0].tolist()


def _uniform(n, seed):
    return torch.rand(n, generator=torch.Generator().manual_seed(seed))


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("vocab", [1, 2, 5, 31, 257, 4096, 4099, 33333, 152001])
@pytest.mark.parametrize("drawn", [True, False])
def test_verify(ctx, dtype, vocab, drawn):
    rng = np.random.default_rng(vocab)
    sizes = [1, 2, 0, 12, 26, 5, 40, 0]
    parents = [p for t in _trees(rng, sizes) for p in t]
    target, draft = _probabilities(sum(sizes), vocab, vocab, dtype)
    tokens = _drawn(sizes, parents, draft, vocab)
    kept, _ = _check_verify(ctx, sizes, parents, tokens, target, draft if drawn else None, _uniform(sum(sizes), 1), _uniform(len(sizes), 2))
    # drawn from a draft that nearly agrees some are accepted; without chance each is with its own probability alone
    assert not drawn or vocab < 5 or max(kept) > 1


@pytest.mark.parametrize("drawn", [True, False])
@pytest.mark.parametrize("vocab", [7, 1000])
def test_verify_many_siblings(ctx, drawn, vocab):
    """Rows that nearly all are rejected: the whole list of a node's children is gone through, with tokens that come twice."""
    rng = np.random.default_rng(3)
    sizes = [64, 256, 2, 100]
    parents = [p for n in sizes for p in [-1] + [0] * (n - 1)]
    target, _ = _probabilities(sum(sizes), vocab, 4, sharp=2.0)
    _, draft = _probabilities(sum(sizes), vocab, 5, sharp=4.0)
    tokens = rng.integers(0, vocab, sum(sizes)).tolist()
    accept = 0.9 + 0.1 * _uniform(sum(sizes), 6)
    _check_verify(ctx, sizes, parents, tokens, target, draft if drawn else None, accept, _uniform(len(sizes), 7))


def test_verify_long_chains_are_accepted(ctx):
    sizes = [256, 100, 300]
    parents = [i - 1 for n in sizes for i in range(n)]
    target, _ = _probabilities(sum(sizes), 50, 8)
    tokens = _drawn(sizes, parents, target, 8)
    kept, _ = _check_verify(ctx, sizes, parents, tokens, target, target, _uniform(sum(sizes), 9), _uniform(3, 10))
    assert kept[:2] == [256, 100] and kept[2] == 256           # as many rows as are looked at
    _check_verify(ctx, sizes, parents, tokens, target, target, _uniform(sum(sizes), 9), _uniform(3, 10), max_nodes=33)


def test_verify_numbers_at_the_ends(ctx):
    sizes = [3] * 8
    parents = [-1, 0, 0] * 8
    target, draft = _probabilities(24, 300, 11)
    tokens = _drawn(sizes, parents, draft, 12)
    accept = torch.tensor([0.0, 0.0, 0.0, 0.0, 1.0, 1.0, 0.0, float("nan"), float("nan"), 0.0, -1.0, 0.0, 0.0, 2.0, 1.0 - 2.0 ** -24] + [0.5] * 9)
    sample = torch.tensor([0.0, 1.0, float("nan"), -3.0, 1.0 - 2.0 ** -24, float("inf"), 2.0 ** -30, 0.5])
    _check_verify(ctx, sizes, parents, tokens, target, draft, accept, sample)
    _check_verify(ctx, sizes, parents, tokens, target, None, accept, sample)


@pytest.mark.parametrize("drawn", [True, False])
def test_verify_odd_probabilities(ctx, drawn):
    """NaN, infinities, negative and large ones, rows of nothing, rows of one token, a draft that is the target."""
    sizes = [3] * 8
    parents = [-1, 0, 0] * 8
    target, draft = _probabilities(24, 77, 13)
    target[0, 5], target[0, 6], target[0, 7], target[0, 8] = float("nan"), float("inf"), -0.5, 3.0
    draft[0, 5], draft[0, 9] = float("nan"), float("inf")
    target[3:6] = 0                                            # nothing: no token
    target[6:9] = 0
    target[6:9, 20] = 1                                        # the token that is drafted, then another
    draft[9:12] = target[9:12]                                 # nothing is left of a rejection
    draft[12:15] = 0
    target[15:18] = float("nan")
    draft[18:21] = 1
    tokens = [1, 6, 8, 1, 2, 3, 0, 20, 20, 5, 6, 7, 1, 2, 3, 4, 5, 6, 7, 8, 9, 76, 76, 0]
    for seed in range(4):
        accept = _uniform(24, seed)
        accept[7:9] = 1.0                                      # 1 * 1 < 1 is not
        accept[10:12] = 1.0
        _, chosen = _check_verify(ctx, sizes, parents, tokens, target, draft if drawn else None, accept, _uniform(8, seed + 50))
        assert chosen[1] == -1 and chosen[5] == -1 and chosen[2] == 20


def test_verify_rows_that_are_none(ctx):
    """Parents behind their rows, of no row, trees without a root's children; tokens outside the vocabulary."""
    sizes = [6, 4, 3]
    parents = [-1, 1, 5, 0, 99, 3] + [-1, -1, 1, 2] + [2, 0, 1]
    target, draft = _probabilities(13, 40, 14)
    tokens = [1, 2, 3, -1, 5, 6, 1, 2, 3, 4, 0, 40, 2 ** 31 - 1]
    for d in (draft, None):
        kept, _ = _check_verify(ctx, sizes, parents, tokens, target, d, torch.zeros(13), _uniform(3, 15))
        assert kept == [1, 1, 1]


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("offset,pad,draft_pad", [(0, 0, 0), (1, 3, 3), (3, 1, 2), (0, 5, 4), (2, 0, 8)])
def test_verify_rows_that_begin_anywhere(ctx, dtype, offset, pad, draft_pad):
    """Rows within wider ones, so that they begin within a vector, alike or not."""
    sizes, vocab = [9, 14], 5001
    rng = np.random.default_rng(pad)
    parents = [p for t in _trees(rng, sizes) for p in t]
    a, b = _probabilities(23, vocab, 16, dtype)
    target = torch.full((23, vocab + pad + offset), 9.0, dtype=dtype, device=DEV)[:, offset:offset + vocab]
    draft = torch.full((23, vocab + draft_pad + offset), 9.0, dtype=dtype, device=DEV)[:, offset:offset + vocab]
    target.copy_(a)
    draft.copy_(b)
    tokens = _drawn(sizes, parents, draft, 17)
    for seed in range(3):
        _check_verify(ctx, sizes, parents, tokens, target, draft, 0.5 + 0.5 * _uniform(23, seed), _uniform(2, seed + 9))
        _check_verify(ctx, sizes, parents, tokens, target, None, 0.5 + 0.5 * _uniform(23, seed), _uniform(2, seed + 9))


def test_verify_the_largest_vocabulary_and_shared_rows(ctx):
    vocab = 1 << 20
    target, draft = _probabilities(1, vocab, 18)
    target, draft = target.expand(6, vocab), draft.expand(6, vocab)        # one row for all
    tokens = torch.multinomial(draft[0], 6, generator=torch.Generator(device=DEV).manual_seed(1)).tolist()
    for seed in range(3):
        _check_verify(ctx, [4, 2], [-1, 0, 0, 1, -1, 0], tokens, target, draft, _uniform(6, seed), _uniform(2, seed))
    _check_verify(ctx, [4, 2], [-1, 0, 0, 1, -1, 0], tokens, target, None, _uniform(6, 4), torch.tensor([0.0, 1.0]))


def test_verify_every_token_can_be_chosen(ctx):
    """The choice at numbers next to every border of a cumulative sum: probabilities that are whole multiples of 2^-24."""
    vocab, n = 37, 2 * 37
    rng = np.random.default_rng(2)
    w = rng.integers(1, 1000, vocab) * (rng.random(vocab) < 0.8)
    w[5] = 1 << 23
    w[-1] = (1 << 24) - w[:-1].sum()
    p = torch.tensor(w / 2.0 ** 24, dtype=torch.float32, device=DEV).expand(n, vocab)
    edges = np.cumsum(w)
    sample = torch.tensor(np.concatenate([edges, edges - 1]).clip(0, (1 << 24) - 1) / 2.0 ** 24, dtype=torch.float32)
    _check_verify(ctx, [1] * n, [-1] * n, [0] * n, p, None, torch.zeros(n), sample)


def test_verify_draws_the_targets_distribution(ctx):
    """The token behind the root over 16,384 requests; each frequency within five standard deviations."""
    n, vocab, fan = 16384, 8, 2
    rng = np.random.default_rng(4)
    p, q = (x / x.sum() for x in (rng.random(vocab) ** 2, rng.random(vocab)))
    tokens = rng.choice(vocab, n * (fan + 1), p=q)
    target = torch.tensor(p, dtype=torch.float32, device=DEV).expand(n * (fan + 1), vocab)
    draft = torch.tensor(q, dtype=torch.float32, device=DEV).expand(n * (fan + 1), vocab)
    for d in (draft, None):
        tree = cm.QTree(_batch(ctx, [fan + 1] * n), 3)
        if d is None:
            tokens = np.tile([0, 3, 6], n)
        tree.verify(_i32([-1, 0, 0] * n), _i32(tokens.tolist()), target, _uniform(len(tokens), 5).to(DEV), _uniform(n, 6).to(DEV), draft=d)
        kept, path, chosen = tree.kept.cpu().numpy(), tree.path.cpu().numpy().reshape(n, -1), tree.next_token.cpu().numpy()
        got = np.where(kept > 1, tokens.reshape(n, -1)[np.arange(n), path[:, 1].clip(0)], chosen)
        frequency = np.bincount(got, minlength=vocab) / n
        assert np.all(np.abs(frequency - p) <= 5 * np.sqrt(p * (1 - p) / n))


# ---------------------------------------------------------------- accepted rows

def _check_keep(ctx, context, sizes, paths, fmt, layers=2, heads=3, d=64, block=16, kv=None, order="blhtd", holes=(), kept=None,
                scales=None, seed=0, extra_width=1):
    """paths: entries of each request's path (any whole numbers); kept: their numbers if not all."""
    g = torch.Generator().manual_seed(seed)
    kv = [max(0, c) + n for c, n in zip(context, sizes)] if kv is None else kv
    need = [-(-max(0, c) // block) + -(-n // block) + 1 for c, n in zip(context, sizes)]
    width = max(need) + extra_width
    nb = sum(need) + 2
    ids = torch.randperm(nb, generator=g).tolist()
    table, at = [], 0
    for n in need:
        table.append(ids[at:at + n] + [-1] * (width - n))
        at += n
    for r, e, b in holes:
        table[r][e] = b
    size = {"b": nb, "l": layers, "h": heads, "t": block, "d": d}

    def codes():
        raw = torch.randint(-120, 121, [size[c] for c in order], generator=g)
        raw = raw.to(torch.int8) if fmt == "int8" else (raw / 4.0).to(torch.float8_e4m3fn)
        return raw.to(DEV).permute([order.index(c) for c in "blhtd"])

    def scale():
        s = torch.exp2(torch.randint(-6, -2, (nb, layers, heads), generator=g).float()) if scales is None else scales((nb, layers, heads), g)
        return s.to(DEV)

    k, v, ks, vs = codes(), codes(), scale(), scale()
    cache = cm.QCache.from_tensors(ctx, k, v, ks, vs)
    batch = _batch(ctx, sizes, width, block)
    batch.block_table.copy_(_i32(table))
    batch.kv_lens.copy_(_i32(kv))
    tree = cm.QTree(batch, 256)
    kept = [len(p) for p in paths] if kept is None else kept
    paths = [(list(p) + [-1] * n)[:n] for p, n in zip(paths, sizes)]
    flat = [x for p in paths for x in p]
    if flat:
        tree.path.copy_(_i32(flat))
    tree.kept.copy_(_i32(kept))
    want = []
    for c, s in ((k, ks), (v, vs)):
        want.append((c.float().double().cpu().numpy(), s.cpu().numpy().copy()))
    lens, freed = [], []
    for r, n in enumerate(sizes):
        moves = ref.keep_rows(table[r], max(0, context[r]), kv[r], n, paths[r], kept[r], block, nb)
        lens.append(max(0, context[r]) + len(moves))
        end = min(kv[r], width * block)
        freed += table[r][-(-lens[r] // block):-(-end // block)]
        for c, s in want:
            for l in range(layers):
                for h in range(heads):
                    view, scalar = c[:, l, h], s[:, l, h]
                    ref.keep(view, scalar, moves, fmt)
    cache.keep(batch, tree, _i32(context))
    torch.cuda.synchronize()
    for (c, s), got_c, got_s in zip(want, (k, v), (ks, vs)):
        assert np.array_equal(got_s.cpu().numpy(), s)
        assert np.array_equal(got_c.float().double().cpu().numpy(), c, equal_nan=True)
    assert tree.lens.tolist() == lens
    assert tree.freed_count.item() == len(freed)
    assert tree.freed.tolist() == (freed + [-1] * tree.freed.numel())[:tree.freed.numel()]
    return cache, batch, tree


@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
@pytest.mark.parametrize("d,block", [(16, 16), (32, 64), (64, 16), (64, 256), (128, 16), (128, 32), (256, 16), (512, 128)])
def test_keep(ctx, fmt, d, block):
    context = [0, 5, block - 1, block, 3 * block + 2, 7, 1]
    sizes = [1, 12, 26, 20, 2 * block + 9, 3, 0]
    paths = [[0], [0, 4, 7, 11], [0, 1, 2, 9, 25], [0, 19], list(range(0, 2 * block + 9, 2)), [0, 1, 2], []]
    _check_keep(ctx, context, sizes, paths, fmt, d=d, block=block)


@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
def test_keep_long_paths(ctx, fmt):
    """Paths over several blocks, in which what is written lies where other entries are read."""
    rng = np.random.default_rng(5)
    sizes = [256, 200, 255, 256]
    paths = [sorted(rng.choice(n, int(m), replace=False).tolist()) for n, m in zip(sizes, (200, 199, 17, 100))]
    paths.append(list(range(0, 256)))
    _check_keep(ctx, [3, 16, 0, 9, 5], sizes + [256], paths, fmt, layers=1, heads=2, d=128)
    _check_keep(ctx, [3, 16, 0, 9, 5], sizes + [256], [[x for x in range(1, n)] for n in sizes] + [[255]], fmt, layers=1, heads=2, d=32)


def test_keep_ends_at_what_is_no_path(ctx):
    sizes = [8] * 9
    paths = [[0, 2, 2, 5], [0, 3, 1], [-1, 2], [0, 8], [0, 5, 2 ** 31 - 1, 6], [2, 3, 4], [7], [0, 1, 2, 3, 4, 5, 6, 7], []]
    _check_keep(ctx, list(range(9)), sizes, paths, "int8")
    _check_keep(ctx, list(range(9)), sizes, [p + [7] for p in paths], "int8", kept=[99, -3, 2, 2, 3, 2, 0, 5, 0])


def test_keep_tokens_that_are_not_there(ctx):
    """Rows beyond the tokens (a request that was cut short), blocks that the table does not name, blocks of no pool."""
    sizes, paths = [30, 30, 30, 30], [[0, 3, 12, 20, 25]] * 4
    _check_keep(ctx, [10, 10, 10, 10], sizes, paths, "e4m3", kv=[40, 25, 10, 0])
    _check_keep(ctx, [10, 10, 10, 10], sizes, paths, "e4m3", holes=[(0, 1, -1), (1, 0, -1), (2, 2, 10 ** 6), (3, 1, -7)])
    _check_keep(ctx, [10, 10], [30, 30], paths[:2], "e4m3", kv=[10 ** 9, 40], extra_width=0)       # longer than the table
    _check_keep(ctx, [-5, 0], [4, 4], [[0, 2], [1]], "int8")


def test_keep_scales_that_are_no_powers_of_two(ctx):
    def odd(shape, g):
        return torch.rand(shape, generator=g) * 0.1 + 0.01
    for fmt in ("e4m3", "int8"):
        _check_keep(ctx, [5, 12], [40, 33], [[0, 3, 20, 21, 39], [2, 30]], fmt, scales=odd)


def test_keep_scales_alike_copies(ctx):
    """Codes whose scale does not change are copied as they are, a NaN too."""
    cache, batch, tree = _check_keep(ctx, [5], [20], [[0, 4, 9]], "e4m3", scales=lambda shape, g: torch.full(shape, 0.25))
    raw = cache.k.view(torch.uint8)
    b = batch.block_table[0].tolist()
    raw[b[0], :, :, 5 + 4] = 0x7f                              # row 4, in the request's first block
    cache.keep(batch, tree, _i32([5]))
    assert bool((raw[b[0], :, :, 6] == 0x7f).all())


@pytest.mark.parametrize("order", ["lbhtd", "bthld", "hbltd", "blthd"])
def test_keep_layouts(ctx, order):
    _check_keep(ctx, [5, 30], [20, 26], [[0, 4, 19], [0, 1, 3, 25]], "e4m3", layers=3, heads=2, d=32, order=order)


def test_keep_many_requests(ctx):
    n = 700
    rng = np.random.default_rng(6)
    sizes = rng.integers(0, 9, n).tolist()
    paths = [sorted(rng.choice(s, int(rng.integers(0, s + 1)), replace=False).tolist()) for s in sizes]
    _check_keep(ctx, rng.integers(0, 40, n).tolist(), sizes, paths, "int8", layers=1, heads=1, d=16)


def test_keep_without_room_for_the_blocks_and_without_requests(ctx):
    cache, batch, tree = _check_keep(ctx, [0], [70], [[0]], "int8")
    freed = torch.full((6,), -9, dtype=torch.int32, device=DEV)
    count, lens = torch.zeros(1, dtype=torch.int64, device=DEV), torch.zeros(1, dtype=torch.int32, device=DEV)
    cm.cm_qcache_keep(ctx.handle, cache._c, batch._c, _i32([0]).data_ptr(), tree.path.data_ptr(), tree.kept.data_ptr(), 70, lens.data_ptr(),
                      freed.data_ptr(), 2, count.data_ptr())
    assert freed.tolist() == batch.block_table[0, 1:3].tolist() + [-9] * 4 and count.item() == 4
    none = cm.QBatch(ctx, 0, 4, 0, 16)
    tree = cm.QTree(none, 4)
    tree.freed_count.fill_(5)
    cache.keep(none, tree, torch.empty(0, dtype=torch.int32, device=DEV))
    tree.plan(None, torch.empty(0, dtype=torch.int32, device=DEV))
    assert tree.freed_count.item() == 0


# ---------------------------------------------------------------- refusals

def test_refusals(ctx):
    batch = _batch(ctx, [3, 2], width=4)
    tree = cm.QTree(batch, 8)
    cache = cm.QCache(ctx, 16, 16, 1, 2, 64)
    lens, parents = _i32([5, 6]), _i32([-1, 0, 0, -1, 0])
    u5, u2 = torch.zeros(5, device=DEV), torch.zeros(2, device=DEV)
    p = torch.zeros((5, 10), device=DEV)
    q = torch.zeros((5, 2, 64), dtype=torch.bfloat16, device=DEV)
    pos = torch.zeros(5, dtype=torch.int32, device=DEV)
    for bad in (0, 257):
        with pytest.raises(ValueError):
            cm.QTree(batch, bad)
    for name in ("mask", "positions", "path", "kept", "next_token", "lens", "freed", "freed_count"):
        with pytest.raises(AttributeError):
            setattr(tree, name, torch.zeros(1))
    calls = [
        lambda: tree.plan(parents.long(), lens), lambda: tree.plan(parents, lens[:1]), lambda: tree.plan(parents.cpu(), lens),
        lambda: tree.plan(_i32([0] * 6), lens), lambda: tree.plan(_i32([0] * 10)[::2], lens),
        lambda: tree.verify(parents, parents, p.half(), u5, u2), lambda: tree.verify(parents, parents, p[:4], u5, u2),
        lambda: tree.verify(parents, parents, p, u5, u2, draft=p.bfloat16()), lambda: tree.verify(parents, parents, p, u5, u2, draft=p[:, :9]),
        lambda: tree.verify(parents, parents, p[:, ::2], u5, u2), lambda: tree.verify(parents, parents[:4], p, u5, u2),
        lambda: tree.verify(parents, parents, p, u5.double(), u2), lambda: tree.verify(parents, parents, p, u5, u5),
        lambda: tree.verify(parents, parents, p.cpu(), u5, u2), lambda: tree.verify(parents, parents.long(), p, u5, u2),
        lambda: cm.rotate_qk(ctx, None, None, pos), lambda: cm.rotate_qk(ctx, q.float(), None, pos), lambda: cm.rotate_qk(ctx, q, None, pos[:4]),
        lambda: cm.rotate_qk(ctx, q, q[:4], pos), lambda: cm.rotate_qk(ctx, q, q[..., :32], pos), lambda: cm.rotate_qk(ctx, q, None, pos.long()),
        lambda: cm.rotate_qk(ctx, q, None, pos, q_weight=torch.zeros(64, device=DEV)), lambda: cm.rotate_qk(ctx, q, None, pos, k_weight=q[0, 0]),
        lambda: cm.rotate_qk(ctx, q, q, pos, q_out=q[:, :1]), lambda: cm.rotate_qk(ctx, q.cpu(), None, pos),
        lambda: cm.rotate_qk(ctx, q.transpose(1, 2), None, pos),
        lambda: cache.attend(torch.zeros((6, 2, 64), dtype=torch.bfloat16, device=DEV), batch, tree=tree),
        lambda: cache.keep(batch, tree, lens.long()), lambda: cache.keep(batch, tree, lens[:1]), lambda: cache.keep(batch, cm.QTree(_batch(ctx, [5]), 8), lens),
    ]
    for i, call in enumerate(calls):
        with pytest.raises(ValueError):
            call()
            pytest.fail("call %d was not refused" % i)


def test_refusals_of_the_library(ctx):
    S = cm.Status

    def refused(status, call):
        with pytest.raises(cm.CMError) as e:
            call()
        assert e.value.status == status

    batch = _batch(ctx, [3, 2], width=4)
    tree = cm.QTree(batch, 8)
    cache = cm.QCache(ctx, 16, 16, 1, 2, 64)
    lens, parents = _i32([5, 6]), _i32([-1, 0, 0, -1, 0])
    L, P, M, X = lens.data_ptr(), parents.data_ptr(), tree.mask.data_ptr(), tree.positions.data_ptr()
    plan = lambda *a: cm.cm_qcache_tree(ctx.handle, batch._c, *a)      # noqa: E731
    for words in (0, 9, -1):
        refused(S.ERR_INVALID_ARG, lambda: plan(L, P, 5, words, M, X))
    refused(S.ERR_INVALID_ARG, lambda: plan(None, P, 5, 1, M, X))
    refused(S.ERR_INVALID_ARG, lambda: plan(L, P, -1, 1, M, X))
    refused(S.ERR_ALIGNMENT, lambda: plan(L, P + 2, 4, 1, M, X))
    refused(S.ERR_INVALID_ARG, lambda: plan(L, M, 5, 1, M, X))         # masks over the parents that are read
    refused(S.ERR_INVALID_ARG, lambda: plan(L, P, 5, 1, P + 8, X))
    plan(L, P, 0, 1, M, X)
    plan(L, None, 5, 1, None, None)

    q = torch.zeros((5, 2, 64), dtype=torch.bfloat16, device=DEV)
    pos = torch.zeros(5, dtype=torch.int32, device=DEV)

    def rows(**kw):
        r = cm.cm_qk_rows(q=q.data_ptr(), q_out=q.data_ptr(), positions=pos.data_ptr(), q_stride_row=128, q_stride_head=64, q_out_stride_row=128,
                          q_out_stride_head=64, num_rows=5, num_q_heads=2, head_dim=64, eps=0.0)
        for name, value in kw.items():
            setattr(r, name, value)
        cm.cm_qk_rotate(ctx.handle, r)

    elsewhere = torch.zeros(2048, dtype=torch.bfloat16, device=DEV)
    other = elsewhere.data_ptr()
    rows()
    rows(q_out=other, q_out_stride_row=64, q_out_stride_head=320)
    rows(q_out=other, q_out_stride_row=136, q_out_stride_head=72)
    rows(num_rows=1, q_out_stride_row=0)
    rows(num_q_heads=1, q_out_stride_head=0)
    for status, kw in ((S.ERR_INVALID_ARG, {"head_dim": 96}), (S.ERR_INVALID_ARG, {"head_dim": 8}), (S.ERR_INVALID_ARG, {"head_dim": 1024}),
                       (S.ERR_INVALID_ARG, {"reserved": 1}), (S.ERR_INVALID_ARG, {"num_rows": -1}), (S.ERR_INVALID_ARG, {"num_rows": 2 ** 31}),
                       (S.ERR_INVALID_ARG, {"eps": -1.0}), (S.ERR_INVALID_ARG, {"eps": float("nan")}), (S.ERR_INVALID_ARG, {"eps": float("inf")}),
                       (S.ERR_INVALID_ARG, {"num_kv_heads": 1}), (S.ERR_INVALID_ARG, {"q_out": None}), (S.ERR_INVALID_ARG, {"positions": None}),
                       (S.ERR_ALIGNMENT, {"q": q.data_ptr() + 2}), (S.ERR_ALIGNMENT, {"q_stride_row": 132}), (S.ERR_INVALID_ARG, {"q_stride_head": -64}),
                       (S.ERR_ALIGNMENT, {"q_weight": q.data_ptr() + 8}), (S.ERR_INVALID_ARG, {"q_out_stride_head": 32}),
                       (S.ERR_INVALID_ARG, {"q_out_stride_row": 0}), (S.ERR_INVALID_ARG, {"num_q_heads": 65536}),
                       # rows that lie on one another, in place with other strides
                       (S.ERR_INVALID_ARG, {"q_out": other, "q_out_stride_row": 64}), (S.ERR_INVALID_ARG, {"q_out": other, "q_out_stride_row": 120}),
                       (S.ERR_INVALID_ARG, {"q_out": other, "q_out_stride_row": 64, "q_out_stride_head": 312}),
                       (S.ERR_INVALID_ARG, {"q_out_stride_row": 136}), (S.ERR_INVALID_ARG, {"q_out_stride_head": 72, "q_out_stride_row": 136})):
        refused(status, lambda: rows(**kw))

    p = torch.zeros((5, 10), device=DEV)
    u5, u2 = torch.zeros(5, device=DEV), torch.zeros(2, device=DEV)

    def drafts(**kw):
        r = cm.cm_tree_drafts(row_starts=batch.row_starts.data_ptr(), parents=P, tokens=P, target=p.data_ptr(), accept=u5.data_ptr(), sample=u2.data_ptr(),
                              path=tree.path.data_ptr(), kept=tree.kept.data_ptr(), next_token=tree.next_token.data_ptr(), target_stride=10,
                              num_requests=2, total_rows=5, vocab=10, max_nodes=8, type=cm.CM_PROB_F32)
        for name, value in kw.items():
            setattr(r, name, value)
        cm.cm_tree_verify(ctx.handle, r)

    drafts()
    for status, kw in ((S.ERR_INVALID_ARG, {"type": 2}), (S.ERR_UNSUPPORTED, {"vocab": 0}), (S.ERR_UNSUPPORTED, {"vocab": (1 << 20) + 1}),
                       (S.ERR_INVALID_ARG, {"max_nodes": 0}), (S.ERR_INVALID_ARG, {"max_nodes": 257}), (S.ERR_INVALID_ARG, {"total_rows": -1}),
                       (S.ERR_UNSUPPORTED, {"num_requests": 16385}), (S.ERR_INVALID_ARG, {"target": None}), (S.ERR_INVALID_ARG, {"kept": None}),
                       (S.ERR_INVALID_ARG, {"sample": None}), (S.ERR_ALIGNMENT, {"target": p.data_ptr() + 2}), (S.ERR_ALIGNMENT, {"accept": u5.data_ptr() + 1}),
                       (S.ERR_INVALID_ARG, {"target_stride": -10})):
        refused(status, lambda: drafts(**kw))

    attend = lambda words, mask: cm.cm_qcache_attend_tree(            # noqa: E731
        ctx.handle, cache._c, 0, batch._c, cm.cm_qcache_query(q=q.data_ptr(), out=q.data_ptr(), q_stride_row=128, q_stride_head=64, out_stride_row=128,
                                                              out_stride_head=64, total_rows=5, num_q_heads=2, softmax_scale=1.0),
        mask, words, batch._workspace_ptr, batch._workspace_bytes)
    for words in (0, 9):
        refused(S.ERR_INVALID_ARG, lambda: attend(words, M))
    refused(S.ERR_INVALID_ARG, lambda: attend(1, None))
    refused(S.ERR_ALIGNMENT, lambda: attend(1, M + 2))

    T, K, F, C = tree.path.data_ptr(), tree.kept.data_ptr(), tree.freed.data_ptr(), tree.freed_count.data_ptr()
    keep = lambda *a: cm.cm_qcache_keep(ctx.handle, cache._c, batch._c, *a)     # noqa: E731
    refused(S.ERR_INVALID_ARG, lambda: keep(L, T, K, 5, L, F, 2, C))            # lens_out over what is read
    refused(S.ERR_INVALID_ARG, lambda: keep(L, T, K, 5, K, F, 2, C))
    refused(S.ERR_INVALID_ARG, lambda: keep(L, T, K, 5, batch.kv_lens.data_ptr(), F, 2, C))
    refused(S.ERR_INVALID_ARG, lambda: keep(L, None, K, 5, tree.lens.data_ptr(), F, 2, C))
    refused(S.ERR_INVALID_ARG, lambda: keep(L, T, K, 5, tree.lens.data_ptr(), None, 2, C))
    refused(S.ERR_INVALID_ARG, lambda: keep(L, T, K, 5, tree.lens.data_ptr(), F, -1, C))
    refused(S.ERR_ALIGNMENT, lambda: keep(L, T, K, 5, tree.lens.data_ptr(), F, 2, C + 4))
    other = cm.QBatch(ctx, 2, 4, 5, 32)
    refused(S.ERR_SHAPE_MISMATCH, lambda: cm.cm_qcache_keep(ctx.handle, cache._c, other._c, L, T, K, 5, tree.lens.data_ptr(), F, 2, C))
    torch.cuda.synchronize()
