"""The 8-bit paged cache where its buffers end, where a launch's limits lie and where its memory is used again:
requests that are cut short, the most requests of a call, graphs and other streams. Tolerances are those of
test_gpu_qcache.py, which derives them."""
import math

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


def _rows_of(cache, head, entries, block):
    """K and V values (fp64) of a head's tokens, whose blocks are `entries`, one per token."""
    e, p = torch.tensor(entries, dtype=torch.long), torch.arange(len(entries)) % block
    return tuple(c[:, 0, head].double().cpu()[e, p] * s[:, 0, head].double().cpu()[e][:, None]
                 for c, s in ((cache.k, cache.k_scale), (cache.v, cache.v_scale)))


def _assert_rows(out, lse, q, k, v, limits):
    """out, lse [n] of one query head against 64 bits: row i over the first limits[i] of k and v."""
    w, wl, mag, size = ref.attend(q.double().cpu(), k, v, q.shape[-1] ** -0.5, limits)
    err = (out.double().cpu() - w).abs()
    tol = w.abs() * 2 ** -8 * (1 + 2 ** -6) + (2 ** -11 + 2 ** -12 + 2 ** -19 * size) * mag
    assert bool((err <= tol).all()), float((err - tol).max())
    got, fine = lse.double().cpu(), torch.isfinite(wl)
    assert torch.equal(torch.isinf(got), ~fine) and not torch.isnan(got).any()
    assert bool(((got - wl)[fine].abs() <= 2 ** -19 * (1 + wl[fine].abs() + size)).all())


# ---------------------------------------------------------------- requests that are cut short

@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("max_new", [1, 1000])
@pytest.mark.parametrize("old,new,width,max_rows", [
    ([60], [30], 4, None),                       # the table ends after 4 of the new tokens
    ([60], [30], 9, 7),                          # 7 rows of 30
    ([60, 20], [30, 25], 9, 37),                 # the second request keeps 7 rows
    ([3, 20, 0], [40, 30, 60], 8, 50),           # a request cut, the last without a row
    ([3, 100, 60], [40, 30, 60], 4, None),       # one whose cached tokens already end at the table
    ([3, 100, 60], [40, 30, 60], 4, 85),         # both
    ([0], [200], 3, None), ([0], [200], 20, 1)])
def test_attend_after_a_cut(ctx, old, new, width, max_rows, max_new, causal):
    """Rows that got a place see their request's tokens up to their own and nothing that was never written; rows
    behind the table's end see what the table holds."""
    H, G, d, block = 1, 4, 64, 16
    R, cap = len(old), width * block
    rows = sum(new) if max_rows is None else max_rows
    cache = cm.QCache(ctx, sum(-(-(o + n) // block) for o, n in zip(old, new)), block, 1, H, d)
    for c in (cache.k, cache.v):
        c.view(torch.uint8).fill_(0x7F)           # NaN wherever nothing is written
    free = torch.randperm(cache.k.shape[0], generator=torch.Generator().manual_seed(1)).int().to(DEV)
    g = torch.Generator(device=DEV).manual_seed(2)

    def step(batch, before, lens, free):
        batch.schedule(_i32(before), _i32(lens), free)
        x = torch.randn((2, 1, H, batch.max_rows, d), generator=g, device=DEV).bfloat16()
        if batch.max_rows:
            cache.append(x[0], x[1], batch.slot_map)

    first = cm.QBatch(ctx, R, width, sum(old), block)
    step(first, [0] * R, old, free)
    batch = cm.QBatch(ctx, R, width, rows, block)
    batch.block_table.copy_(first.block_table)
    step(batch, old, new, free[int(first.counts[0]):].contiguous())
    batch.max_new = max_new
    q = torch.randn((rows, H * G, d), generator=g, device=DEV).bfloat16()
    lse = torch.empty(q.shape[:2], device=DEV)
    out, _ = cache.attend(q, batch, lse=lse, causal=causal)
    torch.cuda.synchronize()
    table, at = batch.block_table.tolist(), 0
    for r, (o, n) in enumerate(zip(old, new)):
        kept = min(n, rows - at)
        tokens = min(o + kept, cap)
        k, v = _rows_of(cache, 0, [table[r][t // block] for t in range(tokens)], block)
        assert torch.isfinite(k).all() and torch.isfinite(v).all()
        limits = [min(tokens, o + i + 1) if causal else tokens for i in range(kept)]
        for j in range(G):
            _assert_rows(out[at:at + kept, j], lse[at:at + kept, j], q[at:at + kept, j], k, v, limits)
        at += kept
    assert at == rows


def test_context_lens_of_a_schedule(ctx):
    """Only requests that were cut short have an entry; later steps without a cut take it back."""
    batch = cm.QBatch(ctx, 3, 4, 130, 16)
    batch.schedule(_i32([3, 100, 60]), _i32([40, 30, 60]), _i32(list(range(40))))
    assert batch.context_lens.tolist() == [-1, 100, 60]
    batch.schedule(_i32([3, -5, 60]), _i32([2, 64, 4]), _i32(list(range(40))))
    assert batch.context_lens.tolist() == [-1, -1, -1]
    few = cm.QBatch(ctx, 3, 4, 5, 16)
    few.schedule(_i32([3, 0, 7]), _i32([2, 4, 0]), _i32(list(range(40))))
    assert few.context_lens.tolist() == [-1, 0, -1]


def test_context_lens_of_the_caller(ctx):
    """Context lengths in the query descriptor, as a C program gives them; flags that are not known are refused."""
    import ctypes
    cache = cm.QCache(ctx, 4, 16, 1, 1, 64)
    x = torch.randn((2, 1, 1, 50, 64), generator=torch.Generator(device=DEV).manual_seed(1), device=DEV).bfloat16()
    cache.append(x[0], x[1], torch.arange(50, device=DEV))
    batch = cm.QBatch(ctx, 1, 4, 8, 16)
    batch.block_table.copy_(_i32([[0, 1, 2, 3]]))
    batch.row_starts.copy_(_i32([0, 8]))
    batch.kv_lens.fill_(50)
    q = torch.randn((8, 2, 64), generator=torch.Generator(device=DEV).manual_seed(2), device=DEV).bfloat16()
    out, lse = torch.empty_like(q), torch.empty((8, 2), device=DEV)
    context = _i32([20])
    space = torch.zeros(cm.cm_qcache_workspace(ctx.handle, 64), dtype=torch.uint8, device=DEV)
    d = cm.cm_qcache_query(q=q.data_ptr(), out=out.data_ptr(), lse=lse.data_ptr(), q_stride_row=128, q_stride_head=64,
                           out_stride_row=128, out_stride_head=64, total_rows=8, num_q_heads=2, max_rows_per_request=8,
                           causal=1, softmax_scale=0.125, flags=cm.CM_QCACHE_CONTEXT_LENS, context_lens=context.data_ptr())
    c = cache._c
    k, v = _rows_of(cache, 0, [t // 16 for t in range(50)], 16)
    for flags, limits in ((cm.CM_QCACHE_CONTEXT_LENS, [21 + i for i in range(8)]), (0, [43 + i for i in range(8)])):
        d.flags = flags
        cm.cm_qcache_attend(ctx.handle, c, 0, batch._c, d, space.data_ptr(), space.numel())
        torch.cuda.synchronize()
        for j in range(2):
            _assert_rows(out[:, j], lse[:, j], q[:, j], k, v, limits)
    d.reserved = 2
    assert d.flags == 2
    with pytest.raises(cm.CMError) as e:
        cm.cm_qcache_attend(ctx.handle, c, 0, batch._c, d, space.data_ptr(), space.numel())
    assert e.value.status == cm.Status.ERR_INVALID_ARG


# ---------------------------------------------------------------- many requests

def _attend_requests(ctx, requests, heads, group, dim, block, max_new, checked, seed, fmt="e4m3"):
    """requests: [(tokens, query rows), ...] over a pool whose blocks are shared; the rows of the requests `checked`
    against 64 bits."""
    rng = np.random.default_rng(seed)
    pool = 64
    g = torch.Generator(device=DEV).manual_seed(seed)
    cache = cm.QCache(ctx, pool, block, 1, heads, dim, dtype=ref.DTYPE[fmt])
    x = torch.randn((2, 1, heads, pool * block, dim), generator=g, device=DEV).bfloat16()
    cache.append(x[0], x[1], torch.arange(pool * block, device=DEV))
    width = max(1, max(-(-kv // block) for kv, _ in requests))
    table = rng.integers(0, pool, (len(requests), width))
    starts = np.cumsum([0] + [m for _, m in requests])
    batch = cm.QBatch(ctx, len(requests), width, int(starts[-1]), block)
    batch.block_table.copy_(torch.from_numpy(table).int())
    batch.row_starts.copy_(torch.from_numpy(starts).int())
    batch.kv_lens.copy_(_i32([kv for kv, _ in requests]))
    batch.max_new = max_new
    q = torch.randn((int(starts[-1]), heads * group, dim), generator=g, device=DEV).bfloat16()
    out, lse = torch.full_like(q, 7.0), torch.full(q.shape[:2], 7.0, device=DEV)
    cache.attend(q, batch, out=out, lse=lse)
    torch.cuda.synchronize()
    assert not (out == 7).all(-1).any() and not (lse == 7).any()       # every row is written
    for r in checked:
        (kv, m), at = requests[r], int(starts[r])
        for h in range(heads):
            k, v = _rows_of(cache, h, [int(table[r, t // block]) for t in range(kv)], block)
            for j in range(h * group, (h + 1) * group):
                _assert_rows(out[at:at + m, j], lse[at:at + m, j], q[at:at + m, j], k, v,
                             [max(0, kv - m + i + 1) for i in range(m)])


@pytest.mark.parametrize("requests,group", [(4060, 1), (4095, 1), (4096, 1), (3672, 16), (3711, 16)])
def test_attend_as_many_requests_as_shared_memory_holds(ctx, requests, group):
    """Request counts whose plan ends close to 48 KB of shared memory, up to the most of a call."""
    rng = np.random.default_rng(requests)
    lens = [(int(kv), 1) for kv in rng.integers(1, 40, requests)]
    _attend_requests(ctx, lens, 1, group, 128, 16, 1, [0, 1, 127, 128, 129, 2047, requests - 2, requests - 1], requests)


@pytest.mark.parametrize("requests", [129, 300, 700])
@pytest.mark.parametrize("heads,group,dim,fmt", [(2, 4, 64, "e4m3"), (1, 2, 256, "int8"), (1, 8, 32, "e4m3")])
@pytest.mark.parametrize("max_new", [1, 1000])
def test_attend_more_requests_than_the_plan_scans_at_a_time(ctx, requests, heads, group, dim, fmt, max_new):
    """Ragged requests, some without rows or tokens, beyond 128 (few-rows kernel) and 640 (many-rows kernel)."""
    rng = np.random.default_rng(requests + dim)
    lens = [(int(kv), int(m)) for kv, m in zip(rng.integers(0, 400, requests), rng.choice([0, 1, 1, 2, 5], requests))]
    lens[0], lens[128], lens[requests - 1] = (33, 1), (70, 2), (129, 1)
    checked = sorted({0, 1, 127, 128, requests // 2, requests - 2, requests - 1} | ({639, 640, 641} if requests > 641 else set()))
    _attend_requests(ctx, lens, heads, group, dim, 16, max_new, checked, requests, fmt)


@pytest.mark.parametrize("tokens,kv,group,dim,heads", [(1100, 1300, 8, 32, 1), (1100, 1100, 8, 64, 2), (600, 700, 16, 256, 1)])
def test_attend_more_row_tiles_than_a_warp_searches_at_a_time(ctx, tokens, kv, group, dim, heads):
    """More than 32 row tiles of a request and kv head, between requests of other sizes; a sample of the rows."""
    requests = [(50, 3), (kv, tokens), (0, 2), (77, 77)]
    block, pool = 16, 128
    g = torch.Generator(device=DEV).manual_seed(tokens + dim)
    cache = cm.QCache(ctx, pool, block, 1, heads, dim)
    x = torch.randn((2, 1, heads, pool * block, dim), generator=g, device=DEV).bfloat16()
    cache.append(x[0], x[1], torch.arange(pool * block, device=DEV))
    width = -(-kv // block)
    table = np.random.default_rng(dim).integers(0, pool, (len(requests), width))
    starts = np.cumsum([0] + [m for _, m in requests])
    batch = cm.QBatch(ctx, len(requests), width, int(starts[-1]), block)
    batch.block_table.copy_(torch.from_numpy(table).int())
    batch.row_starts.copy_(torch.from_numpy(starts).int())
    batch.kv_lens.copy_(_i32([n for n, _ in requests]))
    q = torch.randn((int(starts[-1]), heads * group, dim), generator=g, device=DEV).bfloat16()
    out, lse = torch.full_like(q, 7.0), torch.full(q.shape[:2], 7.0, device=DEV)
    cache.attend(q, batch, out=out, lse=lse)
    torch.cuda.synchronize()
    assert not (out == 7).all(-1).any() and not (lse == 7).any()
    assert tokens * group > 32 * (128 if dim == 256 else 256)
    for r, (n, m) in enumerate(requests):
        rows = sorted({0, 1, m // 3, m // 2, m - 2, m - 1, *([m - 60, 32 * 256 // group - 1, 32 * 256 // group] if m > 500 else [])})
        rows = [i for i in rows if 0 <= i < m]
        at = torch.tensor(rows) + int(starts[r])
        for h in range(heads):
            k, v = _rows_of(cache, h, [int(table[r, t // block]) for t in range(n)], block)
            for j in range(h * group, (h + 1) * group):
                _assert_rows(out[at, j], lse[at, j], q[at, j], k, v, [max(0, n - m + i + 1) for i in rows])


@pytest.mark.parametrize("max_new,T", [(1, 8192), (1000, 65536)])
def test_row_starts_that_do_not_ascend(ctx, max_new, T):
    """2,048 requests that claim all of the rows, in tiles of 8 or of 256: more work than 32 bits count. Such a call does
    nothing, and the batch can be used on."""
    R, width, group, dim, block = 4096, 256, 8, 32, 256
    assert 2048 * (T * group // (8 if max_new == 1 else 256)) * (width * block // 64) >= 2 ** 32
    cache = cm.QCache(ctx, width, block, 1, 1, dim)
    batch = cm.QBatch(ctx, R, width, T, block)
    batch.block_table.copy_(torch.arange(width, dtype=torch.int32)[None].expand(R, width))
    batch.row_starts.copy_((torch.arange(R + 1) % 2 * T).int())
    batch.kv_lens.fill_(width * block)
    batch.max_new = max_new
    q = torch.zeros((T, group, dim), dtype=torch.bfloat16, device=DEV)
    out = torch.full_like(q, 7.0)
    cache.attend(q, batch, out=out)
    ctx.check()
    assert bool((out == 7).all())
    batch.row_starts.copy_(torch.arange(R + 1, dtype=torch.int32))
    cache.attend(q, batch, out=out)
    ctx.check()
    assert bool((out[:R] == 0).all()) and bool((out[R:] == 7).all())


# ---------------------------------------------------------------- refusals

def _small(ctx, rows=3, heads=2, dim=64):
    cache = cm.QCache(ctx, 2, 16, 1, 1, dim)
    batch = cm.QBatch(ctx, 1, 1, rows, 16)
    batch.block_table.fill_(1)
    batch.row_starts.copy_(_i32([0, rows]))
    batch.kv_lens.fill_(rows)
    return cache, batch, torch.zeros((rows, heads, dim), dtype=torch.bfloat16, device=DEV)


@pytest.mark.parametrize("scale", [3e38, -3e38, math.inf, math.nan])
def test_scales_that_overflow_are_refused(ctx, scale):
    """A scale that is finite itself but not times log2 e would make every score NaN."""
    cache, batch, q = _small(ctx)
    with pytest.raises(cm.CMError) as e:
        cache.attend(q, batch, softmax_scale=scale)
    assert e.value.status == cm.Status.ERR_INVALID_ARG
    out, _ = cache.attend(q, batch, softmax_scale=math.copysign(2.3e38, scale))
    assert bool((out == 0).all())


def test_results_that_lie_on_one_another_are_refused(ctx):
    """An expanded tensor has no place of its own for every row; an expanded query is fine."""
    cache, batch, q = _small(ctx)
    one = torch.empty((1, 2, 64), dtype=torch.bfloat16, device=DEV)
    for out in (one.expand(3, 2, 64), one[:, :1].expand(1, 2, 64).expand(3, 2, 64), torch.empty_like(q)[:, :1].expand(3, 2, 64),
                torch.empty(400, dtype=torch.bfloat16, device=DEV).as_strided((3, 2, 64), (128, 32, 1))):
        with pytest.raises(cm.CMError) as e:
            cache.attend(q, batch, out=out)
        assert e.value.status == cm.Status.ERR_INVALID_ARG
    out, _ = cache.attend(q[:1].expand(3, 2, 64), batch)
    assert bool((out == 0).all())
    # a single row or head has no stride to speak of
    cache.attend(q[:1, :1], batch, out=one[:, :1])


# ---------------------------------------------------------------- memory that is used again

def _steps(ctx, rows, dim, seed=5, fmt="e4m3"):
    """A cache of some 2,500 tokens, a batch of one request that reads all of it, and a query."""
    block, tokens = 16, 2500
    n = -(-tokens // block)
    cache = cm.QCache(ctx, n, block, 1, 1, dim, dtype=ref.DTYPE[fmt])
    g = torch.Generator(device=DEV).manual_seed(seed)
    x = torch.randn((2, 1, 1, tokens, dim), generator=g, device=DEV).bfloat16()
    cache.append(x[0], x[1], torch.arange(tokens, device=DEV))
    batch = cm.QBatch(ctx, 1, n, rows, block)
    batch.block_table.copy_(torch.arange(n)[None].int())
    batch.row_starts.copy_(_i32([0, rows]))
    batch.kv_lens.fill_(tokens)
    batch.max_new = rows
    return cache, batch, torch.randn((rows, 4, dim), generator=g, device=DEV).bfloat16()


@pytest.mark.parametrize("rows", [1, 40])
def test_a_captured_attend_outlives_calls_of_other_head_dims(ctx, rows):
    """The first attend of a batch is captured; then the batch serves a larger head_dim; the graph still writes
    into memory that is the batch's, and gives the same bits."""
    cache, batch, q = _steps(ctx, rows, 64)
    wide, _, q_wide = _steps(ctx, rows, 128)
    want = cache.attend(q, _same(ctx, batch))[0]
    want_wide = wide.attend(q_wide, _same(ctx, batch))[0]
    out = torch.zeros_like(q)
    space = batch._workspace_ptr
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        cache.attend(q, batch, out=out)
    assert torch.equal(wide.attend(q_wide, batch)[0], want_wide)
    assert batch._workspace_ptr == space == batch._workspace.data_ptr()
    for _ in range(2):
        out.zero_()
        graph.replay()
        assert torch.equal(wide.attend(q_wide, batch)[0], want_wide)
        torch.cuda.synchronize()
        assert torch.equal(out, want)


def _same(ctx, batch):
    """Another batch of the same requests."""
    b = cm.QBatch(ctx, batch.kv_lens.numel(), batch.block_table.shape[1], batch.max_rows, 16)
    for a, c in ((b.block_table, batch.block_table), (b.row_starts, batch.row_starts), (b.kv_lens, batch.kv_lens)):
        a.copy_(c)
    b.max_new = batch.max_new
    return b


@pytest.mark.parametrize("rows", [1, 40])
def test_a_captured_step_is_the_step(ctx, rows):
    """schedule, append and attend in one graph, replayed over new inputs: the bits of the plain calls. The first
    calls of the batch are the captured ones."""
    R, H, G, d, block, width = 3, 2, 4, 64, 16, 40
    old = [3, 16, 200]
    g = torch.Generator(device=DEV).manual_seed(31)
    caches = [cm.QCache(ctx, R * width, block, 1, H, d) for _ in range(2)]
    batches = [cm.QBatch(ctx, R, width, R * rows, block) for _ in range(2)]
    first = cm.QBatch(ctx, R, width, sum(old), block)
    free = torch.randperm(R * width, generator=torch.Generator().manual_seed(3)).int().to(DEV)
    first.schedule(_i32([0] * R), _i32(old), free)
    x = torch.randn((2, 1, H, sum(old), d), generator=g, device=DEV).bfloat16()
    for c, b in zip(caches, batches):
        c.append(x[0], x[1], first.slot_map)
        b.block_table.copy_(first.block_table)
        b.max_new = rows
    lens, new = _i32(old), _i32([rows] * R)
    left = free[sum(-(-o // block) for o in old):].contiguous()
    kv = torch.empty((2, 1, H, R * rows, d), dtype=torch.bfloat16, device=DEV)
    q = torch.empty((R * rows, H * G, d), dtype=torch.bfloat16, device=DEV)
    outs = [torch.zeros_like(q) for _ in range(2)]

    def step(i):
        batches[i].schedule(lens, new, left)
        caches[i].append(kv[0], kv[1], batches[i].slot_map)
        caches[i].attend(q, batches[i], out=outs[i])

    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(0)
    held = list(old)
    for _ in range(3):
        kv.copy_(torch.randn(kv.shape, generator=g, device=DEV))
        q.copy_(torch.randn(q.shape, generator=g, device=DEV))
        graph.replay()
        step(1)
        torch.cuda.synchronize()
        assert torch.equal(outs[0], outs[1]) and bool(outs[0].abs().sum() > 0)
        for a, b in ((caches[0].k, caches[1].k), (caches[0].v, caches[1].v)):
            assert torch.equal(a.view(torch.uint8), b.view(torch.uint8))
        lens += rows                                  # the next step's, in the same memory
        taken = sum(-(-(h + rows) // block) - -(-h // block) for h in held)
        held = [h + rows for h in held]
        left.copy_(torch.cat([left[taken:], left[:taken]]))
    ctx.check()


@pytest.mark.parametrize("handle", [False, True])
@pytest.mark.parametrize("rows", [1, 40])
def test_results_are_made_on_the_stream_that_writes_them(ctx, rows, handle):
    """With stream= and no out, the result is memory of that stream: the current stream neither has it still in use nor
    gets it when the result is dropped."""
    cache, batch, q = _steps(ctx, rows, 64)
    want = cache.attend(q, batch)[0]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    torch.cuda.synchronize()
    out, _ = cache.attend(q, batch, stream=side.cuda_stream if handle else side)
    side.synchronize()
    assert torch.equal(out, want)
    torch.cuda.synchronize()
    at = out.data_ptr()
    del out
    assert torch.empty_like(q).data_ptr() != at           # of the current stream
    with torch.cuda.stream(side):
        assert torch.empty_like(q).data_ptr() == at
    assert torch.equal(cache.attend(q, batch, stream=0)[0], want)     # the default stream


@pytest.mark.parametrize("current", [False, True])
def test_a_dropped_batch_keeps_its_memory_from_others_until_its_stream_is_done(ctx, current):
    """A batch made on one stream, used on another (named, or the current one) and dropped while that one is busy:
    nobody else gets its memory before."""
    cache, batch, q = _steps(ctx, 1, 64)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    spaces = {t.data_ptr(): t.numel() for t in (batch._workspace, batch.block_table)}
    with torch.cuda.stream(side):
        torch.cuda._sleep(200_000_000)                    # some 0.1 s
    if current:
        with torch.cuda.stream(side):
            out, _ = cache.attend(q, batch)
    else:
        out, _ = cache.attend(q, batch, stream=side)
    del batch
    big = torch.empty(max(spaces.values()), dtype=torch.uint8, device=DEV)
    small = torch.empty(min(spaces.values()), dtype=torch.int32, device=DEV)
    assert not side.query()                               # it was still busy
    assert not {big.data_ptr(), small.data_ptr()} & set(spaces)
    side.synchronize()
    assert torch.isfinite(out).all()


# ---------------------------------------------------------------- waits that run out

def _withheld(ctx, cache, batch, q, out, what):
    """Attention with an arrival withheld: the host learns of it, once. Returns the call's time in ms."""
    n, heads, dim = q.shape
    d = cm.cm_qcache_query(q=q.data_ptr(), out=out.data_ptr(), q_stride_row=q.stride(0), q_stride_head=q.stride(1),
                           out_stride_row=out.stride(0), out_stride_head=out.stride(1), total_rows=n, num_q_heads=heads,
                           max_rows_per_request=n, causal=1, softmax_scale=dim ** -0.5)
    begin, end = (torch.cuda.Event(enable_timing=True) for _ in range(2))
    begin.record()
    st = cm.lib.cm_testing_qcache_attend_withheld(ctx.handle, cache._ref, 0, batch._ref, bytes(d), batch._workspace_ptr,
                                                  batch._workspace_bytes, what, torch.cuda.current_stream().cuda_stream or None)
    end.record()
    assert st == cm.Status.OK
    with pytest.raises(cm.CMError) as e:
        ctx.check()
    assert e.value.status == cm.Status.ERR_TIMEOUT
    ctx.check()
    return begin.elapsed_time(end)


@pytest.mark.parametrize("dim,fmt", [(32, "e4m3"), (64, "int8"), (128, "e4m3"), (256, "int8")])
def test_withheld_queries_time_out_and_the_next_call_is_right(ctx, dim, fmt):
    cache, batch, q = _steps(ctx, 70, dim, fmt=fmt)
    want = cache.attend(q, batch)[0]
    out = torch.zeros_like(q)
    for _ in range(2):
        _withheld(ctx, cache, batch, q, out, 1)
        assert torch.equal(cache.attend(q, batch)[0], want)
    ctx.check()


@pytest.mark.parametrize("dim,fmt", [(32, "e4m3"), (64, "int8"), (128, "e4m3"), (256, "int8")])
def test_withheld_lookups_time_out_and_read_nothing_outside(ctx, dim, fmt):
    """The loads go on without the places of their codes: they read none. (Shared memory that was never written is no
    address; what a wrong one would do is not tried.)"""
    cache, batch, q = _steps(ctx, 70, dim, fmt=fmt)
    want = cache.attend(q, batch)[0]
    out = torch.zeros_like(q)
    for _ in range(2):
        _withheld(ctx, cache, batch, q, out, 2)
        assert torch.equal(cache.attend(q, batch)[0], want)
    ctx.check()


def test_unknown_arrivals_are_not_withheld(ctx):
    cache, batch, q = _steps(ctx, 1, 64)
    for what in (0, 3, -1):
        assert cm.lib.cm_testing_qcache_attend_withheld(ctx.handle, cache._ref, 0, batch._ref, bytes(cm.cm_qcache_query()),
                                                        batch._workspace_ptr, batch._workspace_bytes, what,
                                                        None) == cm.Status.ERR_INVALID_ARG


def test_after_a_wait_ran_out_the_others_do_not_add_up(ctx):
    """A block with 64 * 2,052 / 152 = 864 tiles that are never looked up: the first wait takes 2e9 cycles (0.97 s at
    2,070 MHz, 1.43 s at 1,400), the three of each tile after it some microseconds (a millisecond each, which a try may take, would be 2.6 s)."""
    block, tokens, heads, dim, rows = 16, 1 << 17, 64, 32, 40
    n = tokens // block
    cache = cm.QCache(ctx, n, block, 1, heads, dim)
    batch = cm.QBatch(ctx, 1, n, rows, block)
    batch.block_table.copy_(torch.arange(n)[None].int())
    batch.row_starts.copy_(_i32([0, rows]))
    batch.kv_lens.fill_(tokens)
    q = torch.zeros((rows, heads, dim), dtype=torch.bfloat16, device=DEV)
    out = torch.zeros_like(q)
    assert 900 < _withheld(ctx, cache, batch, q, out, 2) < 1600
    cache.attend(q, batch, out=out)
    ctx.check()
    assert bool((out == 0).all())


def test_tensors_that_the_library_holds_cannot_be_replaced(ctx):
    """Assigning another tensor would leave the calls with the old one's memory; writing into it is the way."""
    cache, batch, q = _small(ctx)
    for obj, names in ((batch, ("block_table", "row_starts", "kv_lens", "context_lens", "slot_map", "counts")),
                       (cache, ("k", "v", "k_scale", "v_scale"))):
        for name in names:
            with pytest.raises(AttributeError):
                setattr(obj, name, getattr(obj, name).clone())
    batch.kv_lens[0] = 2
    batch.kv_lens += 1
    cache.k_scale *= 2
    assert batch.kv_lens.tolist() == [3]
    # fewer rows than the slot map has are fine, more are not
    batch.max_rows = 2
    for rows in (4, -1):
        with pytest.raises(ValueError):
            batch.max_rows = rows
    batch.slot_map.fill_(-9)
    batch.schedule(_i32([0]), _i32([5]), _i32([1]))
    assert batch.slot_map.tolist() == [16, 17, -9] and batch.row_starts.tolist() == [0, 2]


def test_a_batch_of_another_device_is_refused(ctx):
    """Its addresses mean nothing here. (One GPU: a batch that says it is elsewhere.)"""
    cache, batch, q = _small(ctx)
    batch._device = 1
    with pytest.raises(ValueError):
        cache.attend(q, batch)
