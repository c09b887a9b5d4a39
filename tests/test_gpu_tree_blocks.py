"""What a step over trees gives back of the cache's blocks, and that none is lost: blocks that the free list did not have, table
entries that name none of the pool's, requests that were cut short. Blocks and lengths are compared exactly."""
import numpy as np
import pytest
import torch

import tree_reference as ref

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


def _put(tree, starts, paths):
    """The requests' paths and their numbers, as a check of their trees would have left them."""
    path = np.full(tree.path.numel(), -1)
    for at, p in zip(starts, paths):
        path[at:at + len(p)] = p
    tree.path.copy_(torch.from_numpy(path).int())
    tree.kept.copy_(_i32([len(p) for p in paths]))


@pytest.mark.parametrize("requests,block,width", [(1, 16, 7), (5, 32, 4), (300, 16, 3), (2, 16, 700)])
def test_only_blocks_of_the_pool_are_given_back(ctx, requests, block, width):
    rng = np.random.default_rng(requests)
    pool = requests * width
    cache = cm.QCache(ctx, pool, block, 1, 1, 16)
    rows = 3
    batch = cm.QBatch(ctx, requests, width, rows * requests, block)
    table = rng.permutation(pool).reshape(requests, width)
    for value in (-1, -7, pool, 10 ** 6, 2 ** 31 - 1, -2 ** 31):
        table[rng.integers(0, requests, requests), rng.integers(0, width, requests)] = value
    table = table.tolist()
    context = rng.integers(0, block, requests).tolist()
    kv = rng.integers(block, width * block + 1, requests).tolist()
    starts = [rows * r for r in range(requests + 1)]
    paths = [sorted(rng.choice(rows, int(rng.integers(0, rows + 1)), replace=False).tolist()) for _ in range(requests)]
    batch.block_table.copy_(_i32(table))
    batch.kv_lens.copy_(_i32(kv))
    batch.row_starts.copy_(_i32(starts))
    tree = cm.QTree(batch, rows)
    _put(tree, starts, paths)
    lens, want = [], []
    for r in range(requests):
        moves = ref.keep_rows(table[r], context[r], kv[r], rows, paths[r] + [-1] * rows, len(paths[r]), block, pool)
        lens.append(context[r] + len(moves))
        want += [b for b in table[r][-(-lens[r] // block):-(-kv[r] // block)] if 0 <= b < pool]
    for room in (requests * width, len(want), len(want) // 2, 0):
        freed = torch.full((requests * width + 3,), -9, dtype=torch.int32, device=DEV)
        count, got = torch.zeros(1, dtype=torch.int64, device=DEV), torch.zeros(requests, dtype=torch.int32, device=DEV)
        cm.cm_qcache_keep(ctx.handle, cache._c, batch._c, _i32(context).data_ptr(), tree.path.data_ptr(), tree.kept.data_ptr(), rows * requests,
                          got.data_ptr(), freed.data_ptr(), room, count.data_ptr())
        assert got.tolist() == lens and count.item() == len(want)
        assert freed.tolist() == (want + [-1] * room)[:room] + [-9] * (freed.numel() - room)


@pytest.mark.parametrize("seed", range(4))
def test_no_block_is_lost_where_the_free_list_is_too_short(ctx, seed):
    """Steps that want more blocks than there are: what the table got instead of them is not given back, and every block is either
    held by one request or free."""
    rng = np.random.default_rng(seed)
    R, block, n, width = 6, 16, 24, 12
    pool = 20
    cache = cm.QCache(ctx, pool, block, 2, 1, 32)
    batch = cm.QBatch(ctx, R, width, R * n, block)
    tree = cm.QTree(batch, n)
    new, starts = _i32([n] * R), [n * r for r in range(R + 1)]
    context = [0] * R
    free = _i32(rng.permutation(pool).tolist())
    short = 0
    for _ in range(14):
        batch.schedule(_i32(context), new, free)
        paths = [sorted(rng.choice(n, int(rng.integers(0, n)), replace=False).tolist()) for _ in range(R)]
        _put(tree, starts, paths)
        cache.keep(batch, tree, _i32(context))
        torch.cuda.synchronize()
        need, table = int(batch.counts[0]), batch.block_table.tolist()
        short += need > free.numel()
        free = torch.cat([tree.freed[:int(tree.freed_count)], free[need:]])
        kv = batch.kv_lens.tolist()
        context = [c + len(ref.keep_rows(t, c, k, n, p + [-1] * n, len(p), block, pool)) for t, c, k, p in zip(table, context, kv, paths)]
        assert tree.lens.tolist() == context
        held = [b for t, c in zip(table, context) for b in t[:-(-c // block)]]
        assert sorted(held + free.tolist()) == list(range(pool))
        if rng.random() < 0.4:                                 # a request ends: its blocks are free, the least recent first
            r = int(rng.integers(R))
            free = torch.cat([free, _i32(table[r][:-(-context[r] // block)])])
            context[r] = 0
    assert short >= 2


@pytest.mark.parametrize("old,new,rows,block,width", [
    ([0], [160], 16, 16, 12), ([5, 0, 40], [30, 100, 20], 40, 16, 8), ([0, 17, 3, 9], [70, 70, 70, 70], 1, 16, 8),
    ([3, 60, 20], [500, 40, 1], 90, 16, 6), ([10, 0], [33, 64], 200, 32, 4)])
def test_blocks_of_rows_that_were_cut_are_given_back(ctx, old, new, rows, block, width):
    """What a step has taken is held or given back, also for rows that had no room in the batch or in the table."""
    R = len(old)
    cache = cm.QCache(ctx, R * width + 5, block, 1, 1, 16)
    pool = np.random.default_rng(rows).permutation(R * width).tolist()
    table = []
    for c in old:
        need = -(-c // block)
        table.append(pool[:need] + [-1] * (width - need))
        pool = pool[need:]
    batch = cm.QBatch(ctx, R, width, rows, block)
    batch.block_table.copy_(_i32(table))
    tree, few = cm.QTree(batch, 256, max_freed=R * width), cm.QTree(batch, 256)
    assert tree.freed.numel() == R * width and few.freed.numel() == R + rows // block
    batch.schedule(_i32(old), _i32(new), _i32(pool))
    starts = batch.row_starts.tolist()
    paths = [list(range(0, min(n, 256), 2)) for n in np.diff(starts)]
    for t in (tree, few):
        _put(t, starts, paths)
        cache.keep(batch, t, _i32(old))
    table, taken, count = batch.block_table.tolist(), pool[:int(batch.counts[0])], int(tree.freed_count)
    lens = tree.lens.tolist()
    assert all(c <= n <= c + len(p) for c, n, p in zip(old, lens, paths))
    held = [b for t, c, n in zip(table, old, lens) for b in t[-(-c // block):-(-n // block)]]
    freed = tree.freed.tolist()
    assert sorted(held + freed[:count]) == sorted(taken) and freed[count:] == [-1] * (R * width - count)
    # a list that is too short holds the first of them, and the number of all
    assert few.freed_count.item() == count and few.freed.tolist() == (freed + [-1] * few.freed.numel())[:few.freed.numel()]
    if sum(new) <= rows:
        assert count <= few.freed.numel()
