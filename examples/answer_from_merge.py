"""Answering from merged caches held in 8 bits, the whole way: the agents' fragments of each request
are ingested and rendered into one canonical cache, the render goes into a paged 8-bit cache, a
question is read against it in one chunk and the answer is decoded token by token.

    python examples/answer_from_merge.py [--requests 16] [--layers 8] [--steps 32] [--format e4m3]

The fragments and the decoder (attention only, random weights) are synthetic; what is shown is how the
calls follow one another. Every attention result is also compared with one over the unquantised
cache in fp32; the printed error is what eight bits cost.
"""
import argparse
import os
import sys
import time

import torch

sys.path.insert(0, os.path.join(os.path.dirname(os.path.abspath(__file__)), ".."))
import paper_2607_01308_gb300 as cm  # noqa: E402

THETA = 1.0e6


def rope(x, positions):
    """x [rows, heads, d] rotated to its positions (element j pairs with j + d / 2)."""
    d = x.shape[-1]
    freq = THETA ** (-torch.arange(0, d, 2, device=x.device, dtype=torch.float64) / d)
    a = (positions.double()[:, None] * freq)[:, None]
    c, s = a.cos().float(), a.sin().float()
    lo, hi = x.float().chunk(2, -1)
    return torch.cat([lo * c - hi * s, hi * c + lo * s], -1).bfloat16()


def fragment(tokens, layers, heads, d, gen):
    """An agent's K (rotated to its own positions 0 .. tokens - 1) and V, [layers, heads, tokens, d]."""
    k, v = (torch.randn((layers, heads, tokens, d), generator=gen, device="cuda").bfloat16() for _ in range(2))
    pos = torch.arange(tokens, device="cuda")
    k = torch.stack([rope(k[l].transpose(0, 1), pos).transpose(0, 1) for l in range(layers)])
    return k.contiguous(), v


class Decoder:
    """Attention layers with residuals; random weights."""

    def __init__(self, layers, q_heads, kv_heads, d, gen):
        self.q_heads, self.kv_heads, self.d, self.hidden = q_heads, kv_heads, d, q_heads * d

        def weight(n, m):
            return (torch.randn((n, m), generator=gen, device="cuda") * n ** -0.5).bfloat16()

        self.qkv = [weight(self.hidden, (q_heads + 2 * kv_heads) * d) for _ in range(layers)]
        self.out = [weight(self.hidden, self.hidden) for _ in range(layers)]

    def project(self, layer, x, positions):
        h = (x.float() * torch.rsqrt(x.float().square().mean(-1, keepdim=True) + 1e-6)).bfloat16()
        q, k, v = (h @ self.qkv[layer]).view(len(x), -1, self.d).split([self.q_heads, self.kv_heads, self.kv_heads], 1)
        return rope(q, positions), rope(k, positions), v


def attention_f32(q, k, v, causal_from):
    """q [n, Hq, d] over k, v [H, t, d]; row i sees the first causal_from + i + 1 tokens."""
    n, hq, d = q.shape
    k, v = (x.float().repeat_interleave(hq // x.shape[0], 0) for x in (k, v))
    s = torch.einsum("nhd,htd->nht", q.float(), k) * d ** -0.5
    seen = torch.arange(k.shape[1], device=q.device) <= causal_from + torch.arange(n, device=q.device)[:, None]
    return torch.einsum("nht,htd->nhd", s.masked_fill(~seen[:, None], float("-inf")).softmax(-1), v)


def main(requests=16, layers=8, kv_heads=8, group=4, dim=128, tokens=(300, 900), question=33, steps=32, block=16,
         fmt="e4m3", check=True, seed=0):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    host = torch.Generator().manual_seed(seed)
    ctx = cm.Context(0, rope_theta=THETA)

    # What each request's agents bring: two fragments, one of them delivered twice (and absorbed once).
    sets, deliveries = [cm.FragmentSet(ctx) for _ in range(requests)], []
    for s in sets:
        a, b = (fragment(int(torch.randint(tokens[0], tokens[1], (), generator=host)), layers, kv_heads, dim, gen) for _ in range(2))
        deliveries += [(s, *a), (s, *b), (s, *a)]
    cm.ingest_many(deliveries)
    merged = []
    for s in sets:
        shape = (layers, kv_heads, s.seq_len(), dim)
        merged.append(tuple(torch.empty(shape, dtype=torch.bfloat16, device="cuda") for _ in range(2)))
    cm.render_many([(s, k, v) for s, (k, v) in zip(sets, merged)])
    lens = [k.shape[2] for k, _ in merged]

    # The pool, and the batch that names each request's blocks. The host knows the lengths, so it knows
    # how many blocks a step takes from the free list; nothing is read back.
    width = max((n + question + steps + block - 1) // block for n in lens)
    pool = sum((n + question + steps + block - 1) // block for n in lens)
    dtype = torch.int8 if fmt == "int8" else torch.float8_e4m3fn
    cache = cm.QCache(ctx, pool, block, layers, kv_heads, dim, dtype=dtype)
    free = torch.randperm(pool, generator=host).int().cuda()
    tables = torch.full((requests, width), -1, dtype=torch.int32, device="cuda")

    def schedule(batch, held, new):
        """Places `new` more rows for each request that holds `held` tokens."""
        nonlocal free, tables
        batch.block_table.copy_(tables)
        batch.schedule(torch.tensor(held, dtype=torch.int32).cuda(), torch.tensor(new, dtype=torch.int32).cuda(), free)
        tables = batch.block_table
        free = free[sum((h + n + block - 1) // block - (h + block - 1) // block for h, n in zip(held, new)):].contiguous()
        batch.max_new = max(new)

    # The merged caches go in: all layers of a request at once.
    taken = cm.QBatch(ctx, requests, width, sum(lens), block)
    schedule(taken, [0] * requests, lens)
    at = 0
    for (k, v), n in zip(merged, lens):
        cache.append(k, v, taken.slot_map[at:at + n])
        at += n

    # The question in one chunk, then the answer one token at a time.
    model = Decoder(layers, kv_heads * group, kv_heads, dim, gen)
    plain = [[list(kv) for kv in zip(k, v)] for k, v in merged] if check else None   # [request][layer] -> [K, V]
    x = torch.randn((requests * question, model.hidden), generator=gen, device="cuda").bfloat16()
    held, worst, timed = list(lens), 0.0, []
    one = cm.QBatch(ctx, requests, width, requests, block)
    for step in range(1 + steps):
        rows = question if step == 0 else 1
        batch = cm.QBatch(ctx, requests, width, requests * rows, block) if step == 0 else one
        torch.cuda.synchronize()
        begun = time.perf_counter()
        schedule(batch, held, [rows] * requests)
        positions = (torch.tensor(held).cuda()[:, None] + torch.arange(rows, device="cuda")).reshape(-1)
        for layer in range(layers):
            q, k, v = model.project(layer, x, positions)
            v = v.contiguous()                            # strides as K's, which its rotation has laid out anew
            # [rows, heads, d] is taken as it is, as a view [1, heads, rows, d]
            cache.append(k.transpose(0, 1)[None], v.transpose(0, 1)[None], batch.slot_map, layer=layer)
            out, _ = cache.attend(q, batch, layer=layer)
            if check:
                for r in range(requests):
                    mine = slice(r * rows, (r + 1) * rows)
                    kv = plain[r][layer]
                    kv[0], kv[1] = (torch.cat([old, new[mine].transpose(0, 1)], 1) for old, new in zip(kv, (k, v)))
                    want = attention_f32(q[mine], kv[0], kv[1], held[r])
                    worst = max(worst, float((out[mine].float() - want).norm() / want.norm()))
            x = x + out.reshape(len(x), -1) @ model.out[layer]
        ctx.check()
        timed.append(time.perf_counter() - begun)
        held = [h + rows for h in held]
        if step == 0:                                     # the last row of each question goes on
            x = x.view(requests, rows, -1)[:, -1].contiguous()
    codes = 2 * cache.k.numel() + 8 * cache.k_scale.numel()
    return {"requests": requests, "merged_tokens": sum(lens), "relative_error": worst, "cache_bytes": codes,
            "bf16_bytes": 4 * cache.k.numel(), "question_ms": timed[0] * 1e3, "step_ms": sorted(timed[1:])[len(timed) // 2] * 1e3 if steps else 0.0}


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__.split("\n\n")[0])
    ap.add_argument("--requests", type=int, default=16)
    ap.add_argument("--layers", type=int, default=8)
    ap.add_argument("--steps", type=int, default=32)
    ap.add_argument("--format", choices=["e4m3", "int8"], default="e4m3")
    a = ap.parse_args()
    r = main(a.requests, a.layers, steps=a.steps, fmt=a.format, check=True)
    print("%(requests)d requests, %(merged_tokens)d merged tokens; cache %(cache_bytes)d bytes (bf16: %(bf16_bytes)d)" % r)
    print("largest relative error of an attention result against the bf16 cache in fp32: %.4f" % r["relative_error"])
    r = main(a.requests, a.layers, steps=a.steps, fmt=a.format, check=False)
    print("without the comparison: question %(question_ms).2f ms, a step %(step_ms).2f ms" % r)
