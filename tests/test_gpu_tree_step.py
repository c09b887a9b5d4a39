"""The operators around a tree of drafted tokens together, as a serving step uses them: what a step leaves in the cache is what its
accepted tokens alone would have left, a captured step repeats the eager one, streams and devices are the caller's."""
import importlib.util
import os

import numpy as np
import pytest
import torch

import tree_reference as ref

pytestmark = pytest.mark.gpu

cm = pytest.importorskip("paper_2607_01308_gb300")

DEV = "cuda:0"
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def ctx():
    c = cm.Context(0)
    yield c
    c.close()


def _i32(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


class Step:
    """One step of a small model's attention with everything that it needs: R requests, random trees."""

    def __init__(self, ctx, fmt="int8", R=5, layers=2, heads=2, group=2, d=64, block=16, vocab=500, seed=0, scale=1.0):
        rng = np.random.default_rng(seed)
        g = torch.Generator(device=DEV).manual_seed(seed)
        self.ctx, self.layers, self.group, self.block = ctx, layers, group, block
        self.sizes = rng.integers(1, 30, R).tolist()
        self.context = rng.integers(0, 90, R).tolist()
        n = sum(self.sizes)
        self.starts = [0] + np.cumsum(self.sizes).tolist()
        self.parents = [p for s in self.sizes for p in [-1] + [int(rng.integers(max(0, i - 4), i)) for i in range(1, s)]]
        width = 1 + max(-(-(c + s) // block) for c, s in zip(self.context, self.sizes))
        self.cache = cm.QCache(ctx, R * width, block, layers, heads, d, dtype=torch.int8 if fmt == "int8" else torch.float8_e4m3fn)
        self.free = torch.randperm(R * width, generator=torch.Generator().manual_seed(seed)).int().to(DEV)
        first = cm.QBatch(ctx, R, width, sum(self.context), block)
        first.schedule(_i32([0] * R), _i32(self.context), self.free)
        k, v = (scale * torch.randn((layers, heads, sum(self.context), d), generator=g, device=DEV).bfloat16() for _ in range(2))
        self.cache.append(k, v, first.slot_map)
        self.free = self.free[int(first.counts[0]):].contiguous()
        self.batch = cm.QBatch(ctx, R, width, n, block)
        self.batch.block_table.copy_(first.block_table)
        self.batch.max_new = max(self.sizes)
        self.tree = cm.QTree(self.batch, max(self.sizes))
        self.context_lens, self.new_lens, self.parent_rows = _i32(self.context), _i32(self.sizes), _i32(self.parents)
        self.qkv = (scale * torch.randn((layers, n, heads * (group + 2), d), generator=g, device=DEV)).bfloat16()
        self.weights = [(1 + 0.1 * torch.randn(d, generator=g, device=DEV)).bfloat16() for _ in range(2)]
        self.heads, self.q_heads = heads, heads * group
        x = torch.randn((n, vocab), generator=g, device=DEV) * 3
        self.target, self.draft = torch.softmax(x, -1), torch.softmax(x + 0.5 * torch.randn(x.shape, generator=g, device=DEV), -1)
        base = np.repeat(self.starts[:-1], self.sizes)
        at = torch.tensor([b + max(p, 0) for b, p in zip(base, self.parents)], device=DEV)
        self.tokens = torch.multinomial(self.draft[at], 1, generator=g)[:, 0].int()
        self.accept, self.sample = torch.rand(n, generator=g, device=DEV), torch.rand(R, generator=g, device=DEV)
        self.q_out = torch.empty((layers, n, self.q_heads, d), dtype=torch.bfloat16, device=DEV)
        self.k_out = torch.empty((layers, n, heads, d), dtype=torch.bfloat16, device=DEV)
        self.out = torch.empty_like(self.q_out)

    def run(self, stream=None):
        s = {"stream": stream}
        self.batch.schedule(self.context_lens, self.new_lens, self.free, **s)
        self.tree.plan(self.parent_rows, self.context_lens, **s)
        for l in range(self.layers):
            q, k, v = self.qkv[l].split([self.q_heads, self.heads, self.heads], 1)
            cm.rotate_qk(self.ctx, q, k, self.tree.positions, *self.weights, q_out=self.q_out[l], k_out=self.k_out[l], **s)
            self.cache.append(self.k_out[l].transpose(0, 1)[None], v.contiguous().transpose(0, 1)[None], self.batch.slot_map, layer=l, **s)
            self.cache.attend(self.q_out[l], self.batch, layer=l, out=self.out[l], tree=self.tree, **s)
        self.tree.verify(self.parent_rows, self.tokens, self.target, self.accept, self.sample, draft=self.draft, **s)
        self.cache.keep(self.batch, self.tree, self.context_lens, **s)

    def state(self):
        t, c = self.tree, self.cache
        return [x.clone() for x in (c.k.view(torch.uint8), c.v.view(torch.uint8), c.k_scale, c.v_scale, t.path, t.kept, t.next_token, t.lens,
                                    t.freed, t.freed_count, t.mask, t.positions, self.batch.block_table, self.out)]


@pytest.mark.parametrize("seed", [0, 1, 2])
@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
def test_a_step_leaves_its_accepted_tokens(ctx, fmt, seed):
    """Every accepted token's K and V are in the cache behind their request's context, each element off by at most half a step of the
    rows' own rounding and half a step of the move's, at the block's scale; the context within half a step of what it was."""
    s = Step(ctx, fmt, seed=seed, scale=1.7)
    before = [t.clone() for t in (s.cache.k, s.cache.v, s.cache.k_scale, s.cache.v_scale)]
    table_before = s.batch.block_table.clone()
    s.run()
    torch.cuda.synchronize()
    ctx.check()
    path, kept = s.tree.path.tolist(), s.tree.kept.tolist()
    want = ref.verify(s.starts, s.parents, s.tokens.tolist(), s.target.cpu().numpy(), s.draft.cpu().numpy(), s.accept.cpu().numpy(),
                      s.sample.cpu().numpy(), 256)
    assert (path, kept, s.tree.next_token.tolist()) == want
    assert max(kept) > 1 and s.tree.lens.tolist() == [c + n for c, n in zip(s.context, kept)]
    table = s.batch.block_table.long()

    def values(codes, scale, r, n, l, tab):
        tokens = torch.arange(n, device=DEV)
        b, at = tab[r, tokens // s.block], tokens % s.block
        return codes[b, l, :, at].float() * scale[b, l][..., None], scale[b, l][..., None]

    def half_step(x, scale):                                       # of a code with that value
        if fmt == "int8":
            return 0.5 * scale
        return torch.maximum(2.0 ** -4 * x.abs(), 2.0 ** -10 * scale)

    for l in range(s.layers):
        v_rows = s.qkv[l][:, s.q_heads + s.heads:]
        for which, (codes, scale, rows) in enumerate(((s.cache.k, s.cache.k_scale, s.k_out[l]), (s.cache.v, s.cache.v_scale, v_rows))):
            for r, (c, n) in enumerate(zip(s.context, kept)):
                got, z = values(codes, scale, r, c + n, l, table)
                old, _ = values(before[which], before[which + 2], r, c, l, table_before.long())
                # the scale may grow in the append and in the move: two roundings
                assert bool(((got[:c] - old).abs() <= 2 * half_step(old, z[:c]) * (1 + 2.0 ** -3)).all())
                mine = rows[[s.starts[r] + i for i in path[s.starts[r]:s.starts[r] + n]]].float()
                assert bool(((got[c:] - mine).abs() <= 2 * half_step(mine, z[c:]) * (1 + 2.0 ** -3)).all())
    # given back: what the step took and its tokens do not need
    taken = s.free[:int(s.batch.counts[0])].tolist()
    held = {int(b) for r, n in enumerate(s.tree.lens.tolist()) for b in table[r, :-(-n // s.block)]}
    freed = s.tree.freed[:int(s.tree.freed_count)].tolist()
    assert not held & set(freed) and set(freed) <= set(taken) and set(taken) - held == set(freed)


@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
def test_a_captured_step_repeats(ctx, fmt):
    a, b = Step(ctx, fmt, seed=7), Step(ctx, fmt, seed=7)
    a.run()
    want = a.state()
    stream = torch.cuda.Stream()
    warm = Step(ctx, fmt, seed=7)
    with torch.cuda.stream(stream):
        warm.run()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    start = [t.clone() for t in (b.cache.k.view(torch.uint8), b.cache.v.view(torch.uint8), b.cache.k_scale, b.cache.v_scale, b.batch.block_table)]
    with torch.cuda.graph(graph):
        b.run()
    for _ in range(2):
        for t, x in zip((b.cache.k.view(torch.uint8), b.cache.v.view(torch.uint8), b.cache.k_scale, b.cache.v_scale, b.batch.block_table), start):
            t.copy_(x)
        graph.replay()
        torch.cuda.synchronize()
        for x, y in zip(b.state(), want):
            assert torch.equal(x, y)


def test_streams(ctx):
    """Two steps on two streams at once, with batches and trees of their own, and one on a bare handle."""
    steps = [Step(ctx, seed=s) for s in (3, 4, 5)]
    want = [Step(ctx, seed=s) for s in (3, 4, 5)]
    for w in want:
        w.run()
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in steps]
    for s, t in zip(steps[:2], streams):
        s.run(t)
    steps[2].run(streams[2].cuda_stream)
    torch.cuda.synchronize()
    for s, w in zip(steps, want):
        for x, y in zip(s.state(), w.state()):
            assert torch.equal(x, y)


@pytest.mark.parametrize("what", [1, 2])
@pytest.mark.parametrize("d,nodes", [(32, 40), (64, 40), (128, 40), (128, 150), (256, 40)])
def test_waits_of_tree_attention_that_run_out(ctx, d, nodes, what):
    """An arrival that never comes, in one thread block: the call ends, the host learns of it once, and the next call is right."""
    block, tokens, heads = 16, 3000, 2
    n = -(-tokens // block)
    g = torch.Generator(device=DEV).manual_seed(d)
    cache = cm.QCache(ctx, n, block, 1, heads, d)
    batch = cm.QBatch(ctx, 1, n, nodes, block)
    tree = cm.QTree(batch, nodes)
    batch.block_table.copy_(torch.arange(n)[None].int())
    batch.row_starts.copy_(_i32([0, nodes]))
    batch.kv_lens.fill_(tokens)
    batch.max_new = nodes
    rows = torch.randn((1, heads, tokens, d), generator=g, device=DEV).bfloat16()
    cache.append(rows, rows, torch.arange(tokens, device=DEV))
    tree.plan(_i32([-1] + [i // 2 for i in range(nodes - 1)]), _i32([tokens - nodes]))
    q = torch.randn((nodes, heads, d), generator=g, device=DEV).bfloat16()
    want, _ = cache.attend(q, batch, tree=tree)
    out = torch.zeros_like(q)
    query = cm.cm_qcache_query(q=q.data_ptr(), out=out.data_ptr(), q_stride_row=heads * d, q_stride_head=d, out_stride_row=heads * d,
                               out_stride_head=d, total_rows=nodes, num_q_heads=heads, max_rows_per_request=nodes, softmax_scale=d ** -0.5)
    assert cm.lib.cm_testing_qcache_attend_tree_withheld(ctx.handle, cache._ref, 0, batch._ref, bytes(query), tree.mask.data_ptr(), tree.mask.shape[1],
                                                         batch._workspace_ptr, batch._workspace_bytes, what,
                                                         torch.cuda.current_stream().cuda_stream or None) == cm.Status.OK
    with pytest.raises(cm.CMError) as e:
        ctx.check()
    assert e.value.status == cm.Status.ERR_TIMEOUT
    assert torch.equal(cache.attend(q, batch, tree=tree)[0], want)
    ctx.check()


def test_repeated_calls_give_the_same_bits(ctx):
    runs = []
    for _ in range(3):
        s = Step(ctx, "e4m3", R=40, d=128, seed=11)
        s.run()
        runs.append(s.state())
    for other in runs[1:]:
        for x, y in zip(runs[0], other):
            assert torch.equal(x, y)


@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
def test_example(fmt):
    spec = importlib.util.spec_from_file_location("draft_trees", os.path.join(ROOT, "examples", "draft_trees.py"))
    mod = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(mod)
    r = mod.main(requests=6, layers=2, kv_heads=2, group=2, dim=64, vocab=300, tokens=(20, 70), steps=5, fmt=fmt)
    # weights in fp16 and the result in bf16 against fp32: 2^-11 and 2^-8 of the elements, and q's rounding that may fall the other way
    assert r["relative_error"] <= 2.0 ** -7
    assert r["context"] == [n + int(sum(a[2][i] for a in r["answers"])) for i, n in enumerate(r["lens"])]
    for drafted, path, kept, chosen in r["answers"]:
        assert bool(((chosen >= 0) & (chosen < 300)).all()) and bool((kept >= 1).all())
    for (_, _, _, chosen), (drafted, _, _, _) in zip(r["answers"], r["answers"][1:]):
        assert torch.equal(drafted[:, 0], chosen)
