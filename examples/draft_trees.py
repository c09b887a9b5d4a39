"""Several tokens a step from merged caches held in 8 bits: a drafter proposes a tree of tokens for each request, one pass of
the model checks all of them against the request's merged cache, the accepted path stays in it.

    python examples/draft_trees.py [--requests 16] [--layers 4] [--steps 12] [--format e4m3]

The caches and the decoder (attention, norms of q and k, random weights, tied embeddings) are synthetic, and the drafter is the
model's own embeddings with noise; what is shown is how the calls follow one another. With check the first layer's attention
is computed again in fp32 from the cache's values, and the printed error is the largest relative one.
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.join(os.path.dirname(os.path.abspath(__file__)), ".."))
import paper_2607_01308_gb300 as cm  # noqa: E402

THETA = 1.0e6


class Decoder:
    """Attention layers with residuals, norms of every head's q and k; random weights."""

    def __init__(self, layers, q_heads, kv_heads, d, vocab, gen):
        self.q_heads, self.kv_heads, self.d, self.hidden, self.layers = q_heads, kv_heads, d, q_heads * d, layers

        def weight(n, m, size):
            return (torch.randn((n, m), generator=gen, device="cuda") * size * n ** -0.5).bfloat16()

        self.qkv = [weight(self.hidden, (q_heads + 2 * kv_heads) * d, 1) for _ in range(layers)]
        self.out = [weight(self.hidden, self.hidden, 0.5) for _ in range(layers)]
        self.q_norm, self.k_norm = ([(1 + 0.1 * torch.randn(d, generator=gen, device="cuda")).bfloat16() for _ in range(layers)] for _ in range(2))
        self.embedding = torch.randn((vocab, self.hidden), generator=gen, device="cuda").bfloat16()

    def project(self, layer, x):
        h = (x.float() * torch.rsqrt(x.float().square().mean(-1, keepdim=True) + 1e-6)).bfloat16()
        return (h @ self.qkv[layer]).view(len(x), -1, self.d).split([self.q_heads, self.kv_heads, self.kv_heads], 1)

    def probabilities(self, x):
        return torch.softmax((x @ self.embedding.T).float() * (2.0 * self.hidden ** -0.5), -1)


def rope_f32(x, positions, weight):
    """What rotate_qk computes, in elementary operations."""
    d, y = x.shape[-1], x.float()
    y = y * torch.rsqrt((y * y).mean(-1, keepdim=True) + 1e-6) * weight.float()
    a = (positions.double()[:, None] * THETA ** (-torch.arange(0, d, 2, device=x.device, dtype=torch.float64) / d))[:, None]
    c, s, (lo, hi) = a.cos().float(), a.sin().float(), y.chunk(2, -1)
    return torch.cat([lo * c - hi * s, hi * c + lo * s], -1)


def static_tree(widths):
    """Parents of a tree that has widths[l] rows at level l, spread over the level before it."""
    parents, before = [-1], [0]
    for width in widths:
        level = range(len(parents), len(parents) + width)
        parents += [before[i * len(before) // width] for i in range(width)]
        before = list(level)
    return parents


def main(requests=16, layers=4, kv_heads=4, group=4, dim=64, vocab=2000, tokens=(200, 600), widths=(4, 6, 6, 4), steps=12, block=16,
         fmt="e4m3", check=True, seed=0):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    host = torch.Generator().manual_seed(seed)
    ctx = cm.Context(0, rope_theta=THETA)
    model = Decoder(layers, kv_heads * group, kv_heads, dim, vocab, gen)
    parents = static_tree(widths)
    n, fan = len(parents), max(parents.count(i) for i in range(len(parents)))
    assert n <= 256

    # Merged caches (here: random ones) in the pool's first blocks, room for every step behind them.
    lens = torch.randint(tokens[0], tokens[1], (requests,), generator=host).tolist()
    width = max(lens) // block + steps * n // block + 3
    cache = cm.QCache(ctx, requests * width, block, layers, kv_heads, dim, dtype=torch.int8 if fmt == "int8" else torch.float8_e4m3fn)
    free = torch.randperm(requests * width, generator=host).int().cuda()
    taken = cm.QBatch(ctx, requests, width, sum(lens), block)
    context = torch.zeros(requests, dtype=torch.int32, device="cuda")
    taken.schedule(context, torch.tensor(lens, dtype=torch.int32, device="cuda"), free)
    for l in range(layers):
        k, v = (torch.randn((1, kv_heads, sum(lens), dim), generator=gen, device="cuda").bfloat16() for _ in range(2))
        cache.append(k, v, taken.slot_map, layer=l)
    context.copy_(torch.tensor(lens, dtype=torch.int32))
    free = free[sum((x + block - 1) // block for x in lens):].contiguous()

    batch = cm.QBatch(ctx, requests, width, requests * n, block)
    batch.max_new = n
    batch.block_table.copy_(taken.block_table)
    tree = cm.QTree(batch, n)
    rows = requests * n
    all_parents = torch.tensor(parents * requests, dtype=torch.int32, device="cuda")
    new = torch.full((requests,), n, dtype=torch.int32, device="cuda")
    parent_row = (torch.arange(requests, device="cuda")[:, None] * n + torch.tensor([max(p, 0) for p in parents], device="cuda")).reshape(-1)
    drafted = torch.zeros(rows, dtype=torch.int32, device="cuda")
    root = torch.randint(0, vocab, (requests,), generator=gen, device="cuda", dtype=torch.int32)
    answers, worst = [], 0.0
    depth = []
    for p in parents:
        depth.append(depth[p] + 1 if p >= 0 else 0)
    for _ in range(steps):
        # The drafter: the embeddings of what it has so far say what comes next; siblings are drawn from one row.
        drafted.view(requests, n)[:, 0] = root
        draft = torch.empty((rows, vocab), device="cuda")
        for d in range(len(widths) + 1):
            at = torch.tensor([i for i in range(n) if depth[i] == d], device="cuda")
            here = (torch.arange(requests, device="cuda")[:, None] * n + at).reshape(-1)
            if d:
                picked = torch.multinomial(draft[parent_row[here]], 1, generator=gen)[:, 0]
                drafted[here] = picked.int()
            x = model.embedding[drafted[here].long()].float()
            draft[here] = model.probabilities((x + 0.3 * torch.randn(x.shape, generator=gen, device="cuda")).bfloat16())

        # One pass of the model over every row of every tree.
        batch.schedule(context, new, free)
        tree.plan(all_parents, context)
        x = model.embedding[drafted.long()]
        for l in range(layers):
            q, k, v = model.project(l, x)
            q, k = cm.rotate_qk(ctx, q, k, tree.positions, model.q_norm[l], model.k_norm[l])
            v = v.contiguous()
            cache.append(k.transpose(0, 1)[None], v.transpose(0, 1)[None], batch.slot_map, layer=l)
            out, _ = cache.attend(q, batch, layer=l, tree=tree)
            if check and l == 0:
                worst = max(worst, _error(cache, batch, tree, model, x, out, group, n))
            x = x + out.reshape(rows, -1) @ model.out[l]

        # What is accepted stays.
        tree.verify(all_parents, drafted, model.probabilities(x), torch.rand(rows, generator=gen, device="cuda"),
                    torch.rand(requests, generator=gen, device="cuda"), draft=draft)
        cache.keep(batch, tree, context)
        answers.append((drafted.view(requests, n).clone(), tree.path.view(requests, n).clone(), tree.kept.clone(), tree.next_token.clone()))
        context.copy_(tree.lens)
        root = tree.next_token.clone()
        # the free list loses what the step has taken from its front and gets back what no token is left in (one number of each
        # is read back: a program that must not wait reads the step's before)
        free = torch.cat([tree.freed[:int(tree.freed_count)], free[int(batch.counts[0]):]])
    ctx.check()
    kept = torch.stack([a[2] for a in answers]).float()
    return {"requests": requests, "rows": n, "steps": steps, "tokens_per_step": float(kept.mean()), "relative_error": worst,
            "answers": answers, "context": context.tolist(), "lens": lens, "parents": parents, "fan": fan}


def _error(cache, batch, tree, model, x, out, group, n):
    """The first layer's attention from the cache's values, in fp32."""
    q, _, _ = model.project(0, x)
    q = rope_f32(q, tree.positions, model.q_norm[0]).bfloat16().float()
    worst = 0.0
    for r in range(batch.block_table.shape[0]):
        kv = int(batch.kv_lens[r])
        blocks = batch.block_table[r, :(kv + cache.k.shape[3] - 1) // cache.k.shape[3]].long()
        k, v = ((c[blocks, 0].float() * s[blocks, 0][..., None, None]).transpose(0, 1).flatten(1, 2)[:, :kv].repeat_interleave(group, 0)
                for c, s in ((cache.k, cache.k_scale), (cache.v, cache.v_scale)))
        mine = slice(r * n, (r + 1) * n)
        words = tree.mask[mine].long() & 0xffffffff
        j = torch.arange(n, device="cuda")
        seen = torch.cat([torch.ones((n, kv - n), dtype=torch.bool, device="cuda"), (words[:, j // 32] >> (j % 32) & 1).bool()], 1)
        s = torch.einsum("nhd,htd->nht", q[mine], k) * q.shape[-1] ** -0.5
        want = torch.einsum("nht,htd->nhd", s.masked_fill(~seen[:, None], float("-inf")).softmax(-1), v)
        worst = max(worst, float((out[mine].float() - want).norm() / want.norm()))
    return worst


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__.split("\n\n")[0])
    ap.add_argument("--requests", type=int, default=16)
    ap.add_argument("--layers", type=int, default=4)
    ap.add_argument("--steps", type=int, default=12)
    ap.add_argument("--format", choices=["e4m3", "int8"], default="e4m3")
    a = ap.parse_args()
    r = main(a.requests, a.layers, steps=a.steps, fmt=a.format)
    print("%(requests)d requests, trees of %(rows)d rows: %(tokens_per_step).2f tokens a step" % r)
    print("largest relative error of the first layer's attention against fp32 on the same cache: %.5f" % r["relative_error"])
