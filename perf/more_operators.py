"""The serving operators that check a tree of drafted tokens against a paged cache held in 8 bits, as
cases to be timed: ancestor masks and positions from the drafts' parents ("plan"), the norm of every
head of q and k with their position rotation ("rotate"), attention in which a row sees its request's
context and its own ancestors ("attend"), the check of drafted tokens against the target's
probabilities from given random numbers ("verify"), and the move of the accepted rows to the front of
their request with the blocks behind them given back ("keep").

`run` computes them in elementary torch operations, in 32 bits (angles and acceptance tests in 64),
or, where `own` is true, through the package's public entry points.

A request's rows are a tree: row i was drafted behind row parents[i] < i of its request (-1: behind
the context alone); row 0 is the root, the token that the step before has chosen.

The check. At a node, beginning with the root: w is its row of target probabilities, z = 1. Its
children, in order, are accepted where u * q(token) * z < w(token), u the child's random number
and q the node's row of draft probabilities (q(token) = 1 without such rows). The first that is accepted
is the next node. One that is rejected leaves w = max(w - q z, 0) and z = sum w, unless that is 0 (w(token) = 0
and z less by it without draft rows). Where no child is left, the next token is the first whose cumulative
w passes v * sum w, v the request's random number (the target row itself, if w is all 0). Elements are fp32;
sums, exactly, of the whole multiples of 2^-42 that the elements reach; z is rounded to fp32 where it
multiplies a row.

The move. A moved row keeps its value up to one rounding: the scale of the block that takes rows becomes the
largest of its own (if it holds tokens in front of them) and those of the blocks that they come from.
"""
import random

import numpy as np
import torch

own = False      # True: the package's operators; False: the plain forms below

FORMATS = {"e4m3": torch.float8_e4m3fn, "int8": torch.int8}
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
THETA = 1.0e6
EPS = 1e-6


# ---------------------------------------------------------------- cases

def listed():
    return [
        # A drafter's trees of one step, all alike in size. Latency only.
        {"name": "plan_64_trees", "op": "plan", "requests": 64, "nodes_lo": 26, "nodes_hi": 26, "fan": 4,
         "old_lo": 600, "old_hi": 12000, "mix": 1},
        # A large ragged batch: from the root alone to trees of 200 rows, some nearly chains.
        {"name": "plan_509_ragged", "op": "plan", "requests": 509, "nodes_lo": 1, "nodes_hi": 200, "fan": 2,
         "old_lo": 0, "old_hi": 130000, "mix": 2},
        # One token of 48 requests: a layer's q and k between projection and cache.
        {"name": "rotate_decode_48", "op": "rotate", "rows": 48, "q_heads": 32, "kv_heads": 8, "dim": 128,
         "far": 12000, "norm": True, "mix": 3},
        # Odd sizes without norms, far positions.
        {"name": "rotate_ragged_d64", "op": "rotate", "rows": 1837, "q_heads": 12, "kv_heads": 12, "dim": 64,
         "far": 1000003, "norm": False, "mix": 4},
        # A long prompt's rows.
        {"name": "rotate_prompt_16384", "op": "rotate", "rows": 16384, "q_heads": 32, "kv_heads": 8, "dim": 128,
         "far": 40000, "norm": True, "mix": 5},
        # One request answers from a merge of 2 x 512 tokens with five drafted tokens in a row.
        {"name": "attend_chain_1x1041", "op": "attend", "requests": 1, "old_lo": 1041, "old_hi": 1041, "nodes_lo": 5,
         "nodes_hi": 5, "fan": 1, "layers": 2, "heads": 8, "group": 2, "dim": 128, "block": 16, "format": "e4m3", "mix": 6},
        # A step of 64 requests with trees over merged caches of ragged lengths.
        {"name": "attend_trees_64_ragged", "op": "attend", "requests": 64, "old_lo": 600, "old_hi": 12000, "nodes_lo": 10,
         "nodes_hi": 26, "fan": 4, "layers": 1, "heads": 8, "group": 4, "dim": 128, "block": 16, "format": "e4m3", "mix": 7},
        # Large trees over long contexts, int8, head_dim 64, many heads to a kv head.
        {"name": "attend_trees_5_long", "op": "attend", "requests": 5, "old_lo": 16000, "old_hi": 64000, "nodes_lo": 41,
         "nodes_hi": 64, "fan": 3, "layers": 1, "heads": 4, "group": 8, "dim": 64, "block": 32, "format": "int8", "mix": 8},
        # Chains of four drafted tokens without draft probabilities (a lookup's proposals).
        {"name": "verify_chains_16", "op": "verify", "requests": 16, "nodes_lo": 3, "nodes_hi": 5, "fan": 1, "vocab": 32003,
         "type": "bf16", "draft": False, "mix": 9},
        # Trees sampled from a draft model, a large vocabulary.
        {"name": "verify_trees_64", "op": "verify", "requests": 64, "nodes_lo": 10, "nodes_hi": 26, "fan": 4, "vocab": 152000,
         "type": "f32", "draft": True, "mix": 10},
        # Small batch, int8, head_dim 64: what one layer group of a small model keeps.
        {"name": "keep_6_int8", "op": "keep", "requests": 6, "old_lo": 3, "old_hi": 200, "nodes_lo": 4, "nodes_hi": 12, "fan": 2,
         "layers": 4, "heads": 12, "dim": 64, "block": 32, "format": "int8", "mix": 11},
        # 64 requests, all layers of a 36-layer model.
        {"name": "keep_64_layers_36", "op": "keep", "requests": 64, "old_lo": 3, "old_hi": 100, "nodes_lo": 10, "nodes_hi": 26,
         "fan": 3, "layers": 36, "heads": 8, "dim": 128, "block": 16, "format": "e4m3", "mix": 12},
    ]


_SHAPES = [(8, 128), (8, 128), (4, 64), (4, 256), (12, 64), (2, 32)]


def draw(rng):
    def size(lo, hi):
        return int(round(lo * (hi / lo) ** rng.random()))

    op = rng.choice(["plan", "rotate", "rotate", "attend", "attend", "attend", "verify", "verify", "keep", "keep"])
    case = {"op": op, "mix": rng.randrange(1 << 20)}
    if op == "rotate":
        heads, dim = rng.choice(_SHAPES)
        group = rng.choice([1, 2, 4, 5, 8])
        case.update(rows=size(1, max(2, min(20000, 80_000_000 // (heads * (group + 1) * dim)))), q_heads=heads * group, kv_heads=heads,
                    dim=dim, far=size(10, 2_000_000), norm=rng.random() < 0.7)
        return case
    nodes = size(1, 200 if op in ("plan", "keep") else 64)
    case.update(nodes_lo=max(1, nodes // rng.choice([1, 3, 10])), nodes_hi=nodes, fan=rng.choice([1, 2, 3, 4, 8]))
    if op == "plan":
        case.update(requests=size(1, 512), old_lo=0, old_hi=size(10, 130000))
        return case
    if op == "verify":
        draft = rng.random() < 0.6
        vocab = size(50, 160000)
        case.update(draft=draft, vocab=vocab, type=rng.choice(["f32", "f32", "bf16"]),
                    requests=size(1, max(1, min(128, 160_000_000 // (nodes * vocab)))))
        return case
    heads, dim = rng.choice(_SHAPES)
    case.update(heads=heads, dim=dim, format=rng.choice(["e4m3", "e4m3", "int8"]), block=rng.choice([16, 16, 32, 64, 128]))
    if op == "keep":
        layers = rng.choice([1, 2, 16, 36])
        old = size(3, 300)
        tokens = (old + nodes + 2 * case["block"]) * layers * heads * dim
        case.update(layers=layers, old_lo=rng.choice([0, old // 2, old]), old_hi=old,
                    requests=size(1, max(1, min(64, 100_000_000 // tokens))))
        return case
    group = rng.choice([1, 2, 4, 4, 5, 8])
    requests = size(1, 96)
    pairs = 6_000_000_000 // (heads * group * dim * nodes * requests)
    top = size(16, max(17, min(65536, pairs, 250_000_000 // (heads * dim * requests))))
    case.update(layers=rng.choice([1, 1, 2]), group=group, requests=requests, old_lo=top // rng.choice([1, 4, 40]), old_hi=top)
    return case


def _spread(rng, lo, hi):
    """A whole number of lo .. hi, spread over its logarithm."""
    return int(round((lo + 1) * ((hi + 1) / (lo + 1)) ** rng.random())) - 1


def _trees(case, seed=None):
    """The requests' cached token counts and trees (the parents of their rows). The trees' sizes are the case's; with
    a seed the rest is that seed's."""
    rng = random.Random(case["mix"])
    sizes = [_spread(rng, case["nodes_lo"], case["nodes_hi"]) for _ in range(case["requests"])]
    if seed is not None:
        rng = random.Random(case["mix"] * 1000003 + seed)
    old = [_spread(rng, case["old_lo"], case["old_hi"]) if "old_lo" in case else 0 for _ in sizes]
    trees = []
    for n in sizes:
        parents, left = [-1], [(0, case["fan"])]
        for i in range(1, n):
            at = rng.randrange(len(left))
            p, room = left[at]
            parents.append(p)
            if room > 1:
                left[at] = (p, room - 1)
            else:
                left.pop(at)
            left.append((i, case["fan"]))
        trees.append(parents)
    return old, trees


def _paths(case):
    """For "keep": a walk down each tree, as long as the check happened to accept."""
    old, trees = _trees(case)
    rng, paths = random.Random(case["mix"] + 1), []
    for parents in trees:
        path = [0]
        while rng.random() < 0.85:
            below = [i for i, p in enumerate(parents) if p == path[-1]]
            if not below:
                break
            path.append(rng.choice(below))
        paths.append(path)
    return old, trees, paths


def _depths(parents):
    depth = []
    for p in parents:
        depth.append(depth[p] + 1 if p >= 0 else 0)
    return depth


def _ceil(a, b):
    return -(-a // b)


def _words(trees):
    return _ceil(max(len(t) for t in trees), 32)


def work(case):
    op = case["op"]
    if op == "rotate":
        d, heads = case["dim"], case["q_heads"] + case["kv_heads"]
        return {"bytes": case["rows"] * (heads * d * 4 + 4), "flops": 0}
    if op == "keep":
        old, trees, paths = _paths(case)
        moved = sum(sum(i != p for i, p in enumerate(path)) for path in paths)
        return {"bytes": moved * case["layers"] * case["heads"] * case["dim"] * 4, "flops": 0}
    old, trees = _trees(case)
    rows = sum(len(t) for t in trees)
    if op == "plan":
        return {"bytes": rows * (8 + 4 * _words(trees)), "flops": 0}
    if op == "verify":
        # the rows at which the walks end
        size = 4 if case["type"] == "f32" else 2
        return {"bytes": len(trees) * case["vocab"] * size * (2 if case["draft"] else 1), "flops": 0}
    H, G, d = case["heads"], case["group"], case["dim"]
    tokens = sum(o + len(t) for o, t in zip(old, trees))
    blocks = sum(_ceil(o + len(t), case["block"]) for o, t in zip(old, trees))
    pairs = sum(len(t) * o + sum(x + 1 for x in _depths(t)) for o, t in zip(old, trees))
    return {"bytes": H * (tokens * d * 2 + blocks * 8) + 4 * blocks + rows * H * G * (4 * d + 4),
            "flops": 4.0 * pairs * H * G * d}


# ---------------------------------------------------------------- inputs

def _generator(seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    return gen


def _normal(shape, gen):
    return torch.randn(shape, generator=gen, device="cuda")


def _int32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def _pow2_scale(amax, fmt):
    """The smallest 2^k that brings amax within the format's largest code (448, or 127)."""
    e, m = (9, 0.875) if fmt == "e4m3" else (7, 0.9921875)
    mant, exp = torch.frexp(amax)
    return (((exp - e + (mant > m)).clamp(-60, 60).int() + 127) << 23).view(torch.float32)


def _codes(x, fmt):
    """x (already divided by its scale) as codes of the format: nearest even, clamped."""
    top = 448.0 if fmt == "e4m3" else 127.0
    x = x.clamp(-top, top)
    return x.round().to(torch.int8) if fmt == "int8" else x.to(torch.float8_e4m3fn)


def _cache(shape, fmt, gen):
    """Codes and scales [blocks, layers, heads, block, dim] of a cache in use: keys with a few
    strong channels, block scales that vary."""
    codes = torch.empty(shape, dtype=FORMATS[fmt], device="cuda")
    scale = torch.empty(shape[:3], device="cuda")
    step = max(1, (1 << 26) // max(1, codes[0].numel()))
    strong = 1 + 2 * (torch.rand(shape[-1], generator=gen, device="cuda") < 0.05)
    for b in range(0, shape[0], step):
        x = _normal((min(step, shape[0] - b),) + tuple(shape[1:]), gen) * strong
        x *= 0.4 + 1.6 * torch.rand(x.shape[:3] + (1, 1), generator=gen, device="cuda")
        s = _pow2_scale(x.abs().amax((-1, -2)), fmt)
        scale[b:b + step] = s
        codes[b:b + step] = _codes(x / s[..., None, None], fmt)
    return codes, scale


def _place(case, old, trees, seed):
    """Lengths on the GPU and a block table with blocks handed out in a shuffled order."""
    bs, kv = case["block"], [o + len(t) for o, t in zip(old, trees)]
    held = [_ceil(n, bs) for n in kv]
    width, total = max(held) + 2, sum(held)
    order = torch.randperm(total + 5, generator=_generator(seed + 1), device="cuda").int()
    table = torch.full((len(kv), width), -1, dtype=torch.int32, device="cuda")
    at = 0
    for r, n in enumerate(held):
        table[r, :n] = order[at:at + n]
        at += n
    return {"table": table, "kv": _int32(kv), "blocks": total + 5, "block": bs, "longest": max(kv)}


def prepare(case, seed):
    gen, op = _generator(seed), case["op"]
    state = {"op": op, "format": case.get("format")}
    if op == "rotate":
        rows, hq, hk, d = case["rows"], case["q_heads"], case["kv_heads"], case["dim"]
        # q, k and v as a projection leaves them: one row of all heads; some channels are strong
        qkv = (_normal((rows, hq + 2 * hk, d), gen) * (1 + 4 * (torch.rand(d, generator=gen, device="cuda") < 0.03))).bfloat16()
        state.update(q=qkv[:, :hq], k=qkv[:, hq:hq + hk], q_weight=None, k_weight=None,
                     positions=torch.randint(0, case["far"] + 1, (rows,), generator=gen, device="cuda", dtype=torch.int32))
        if case["norm"]:
            state.update(q_weight=(1 + 0.2 * _normal((d,), gen)).bfloat16(), k_weight=(1 + 0.2 * _normal((d,), gen)).bfloat16())
        if own:
            import paper_2607_01308_gb300 as cm
            state.update(ctx=_context(cm), rotate=cm.rotate_qk, q_out=torch.empty((rows, hq, d), dtype=torch.bfloat16, device="cuda"),
                         k_out=torch.empty((rows, hk, d), dtype=torch.bfloat16, device="cuda"))
        return state
    old, trees, paths = _paths(case)
    if op == "plan":
        old, trees = _trees(case, seed)
    n = [len(t) for t in trees]
    rows, most, starts = sum(n), max(n), [sum(n[:r]) for r in range(len(n) + 1)]
    state.update(rows=rows, most=most, depth=max(max(_depths(t)) for t in trees), fan=case["fan"], starts=_int32(starts),
                 parents=_int32([p for t in trees for p in t]), context=_int32(old), words=_words(trees))
    block = case.get("block", 16)
    if own:
        import paper_2607_01308_gb300 as cm
        place = _place(case, old, trees, seed) if op in ("attend", "keep") else {"table": torch.zeros((len(n), 0), device="cuda")}
        state["batch"] = batch = cm.QBatch(_context(cm), len(n), place["table"].shape[1], rows, block)
        batch.row_starts.copy_(state["starts"])
        batch.max_new = most
        state["tree"] = tree = cm.QTree(batch, most)
    if op == "plan":
        return state
    if op == "verify":
        return _prepare_verify(case, state, trees, gen)
    H, d, L = case["heads"], case["dim"], case["layers"]
    state.update(_place(case, old, trees, seed))
    for name in ("k", "v"):
        state[name], state[name + "_scale"] = _cache((state["blocks"], L, H, block, d), case["format"], gen)
    if op == "attend":
        mask, _ = _plan(state)
        state.update(mask=mask, layer=L - 1, group=case["group"], q=_normal((rows, H * case["group"], d), gen).bfloat16())
    else:
        path = [list(p) + [-1] * (k - len(p)) for p, k in zip(paths, n)]
        state.update(path=_int32([x for p in path for x in p]), kept=_int32([len(p) for p in paths]), longest_path=max(len(p) for p in paths))
    if own:
        batch.block_table.copy_(state["table"])
        batch.kv_lens.copy_(state["kv"])
        state["cache"] = cm.QCache.from_tensors(_context(cm), state["k"], state["v"], state["k_scale"], state["v_scale"])
        if op == "attend":
            tree.mask.copy_(state["mask"])
            state.update(out=torch.empty_like(state["q"]), lse=torch.empty(state["q"].shape[:2], device="cuda"))
        else:
            tree.path.copy_(state["path"])
            tree.kept.copy_(state["kept"])
    return state


def _prepare_verify(case, state, trees, gen):
    """Probabilities of a target and of a drafter that nearly agrees with it; the drafted tokens: drawn from the
    drafter's row at their parent, or, without draft probabilities, its likeliest ones."""
    rows, V, kind = state["rows"], case["vocab"], TYPES[case["type"]]
    place, rank = [], []                     # of each row: its parent's row, its order among the siblings
    for t in trees:
        at, seen = len(place), {}
        for p in t:
            place.append(at + max(p, 0))
            rank.append(seen.get(p, 0))
            seen[p] = rank[-1] + 1
    target = torch.empty((rows, V), dtype=kind, device="cuda")
    draft = torch.empty((rows, V), dtype=kind, device="cuda") if case["draft"] else None
    picks = torch.empty((rows, case["fan"]), dtype=torch.int64, device="cuda")
    step = max(1, (1 << 26) // V)
    for i in range(0, rows, step):
        x = _normal((min(step, rows - i), V), gen) * 3.5
        target[i:i + step] = torch.softmax(x, -1).to(kind)
        q = torch.softmax(0.9 * x + 0.7 * _normal(x.shape, gen), -1).to(kind)
        if draft is None:
            picks[i:i + step] = q.float().topk(case["fan"], -1).indices
        else:
            draft[i:i + step] = q
            picks[i:i + step] = torch.multinomial(q.float(), case["fan"], replacement=True, generator=gen)
    tokens = picks[torch.tensor(place, device="cuda"), torch.tensor(rank, device="cuda")].int()
    state.update(target=target, draft=draft, tokens=tokens, accept=torch.rand(rows, generator=gen, device="cuda"),
                 sample=torch.rand(len(trees), generator=gen, device="cuda"))
    return state


_contexts = []


def _context(cm):
    """One context for the life of the process, as a serving process keeps it."""
    if not _contexts:
        _contexts.append(cm.Context(0, rope_theta=THETA))
    return _contexts[0]


# ---------------------------------------------------------------- one pass

def run(state):
    op = state["op"]
    if own:
        if op == "rotate":
            q, k = state["rotate"](state["ctx"], state["q"], state["k"], state["positions"], q_weight=state["q_weight"],
                                   k_weight=state["k_weight"], eps=EPS, q_out=state["q_out"], k_out=state["k_out"])
            return {"q": q, "k": k}
        tree = state["tree"]
        if op == "plan":
            tree.plan(state["parents"], state["context"])
            return {"mask": tree.mask, "positions": tree.positions}
        if op == "verify":
            tree.verify(state["parents"], state["tokens"], state["target"], state["accept"], state["sample"], draft=state["draft"])
            return {"path": tree.path, "kept": tree.kept, "next": tree.next_token}
        cache = state["cache"]
        if op == "attend":
            out, lse = cache.attend(state["q"], state["batch"], layer=state["layer"], out=state["out"], lse=state["lse"], tree=tree)
            return {"out": out, "lse": lse}
        cache.keep(state["batch"], tree, state["context"])
        return {"k": cache.k, "v": cache.v, "k_scale": cache.k_scale, "v_scale": cache.v_scale,
                "lens": tree.lens, "freed": tree.freed, "count": tree.freed_count}
    if op == "rotate":
        return {name: _rotate(state[name], state["positions"], state[name + "_weight"]) for name in ("q", "k")}
    if op == "plan":
        mask, positions = _plan(state)
        return {"mask": mask, "positions": positions}
    if op == "verify":
        return _verify(state)
    return _attend(state) if op == "attend" else _keep(state)


def _owner(s):
    """The request of each row, and the first row of that request."""
    starts = s["starts"].long()
    r = torch.searchsorted(starts[1:].contiguous(), torch.arange(s["rows"], device="cuda"), right=True)
    return r, starts[r]


def _plan(s):
    """Bit j of a row's mask: row j of its request is the row itself or one of its ancestors."""
    r, first = _owner(s)
    row = torch.arange(s["rows"], device="cuda")
    seen = torch.zeros((s["rows"], 32 * s["words"]), dtype=torch.bool, device="cuda")
    depth = torch.zeros_like(row)
    at, parents = row - first, s["parents"].long()
    seen[row, at] = True
    for _ in range(s["depth"]):
        up = parents[first + at]
        has = up >= 0
        at = torch.where(has, up, at)
        seen[row, at] = True
        depth += has
    bits = torch.ones(32, dtype=torch.int64, device="cuda") << torch.arange(32, device="cuda")
    mask = (seen.view(s["rows"], s["words"], 32) * bits).sum(-1)
    return torch.where(mask >= 1 << 31, mask - (1 << 32), mask).int(), (s["context"].long()[r] + depth).int()


def _rotate(x, positions, weight):
    """Norm of each head's row, then element j and j + d / 2 turned by position * THETA^(-2j/d)."""
    d = x.shape[-1]
    y = x.float()
    if weight is not None:
        y = y * torch.rsqrt((y * y).mean(-1, keepdim=True) + EPS) * weight.float()
    freq = THETA ** (-torch.arange(0, d, 2, device="cuda", dtype=torch.float64) / d)
    a = (positions.double()[:, None] * freq)[:, None]
    c, s = a.cos().float(), a.sin().float()
    lo, hi = y[..., :d // 2], y[..., d // 2:]
    return torch.cat([lo * c - hi * s, hi * c + lo * s], -1).bfloat16()


def _attend(s):
    """softmax(q k^T / sqrt(d)) v over each request's own cached tokens: the context, and of its new rows those in the mask."""
    table, kv, starts, q, context = s["table"], s["kv"].long(), s["starts"].long(), s["q"], s["context"].long()
    bs, G, layer = s["block"], s["group"], s["layer"]
    H, d = s["k"].shape[2], s["k"].shape[4]
    R = len(kv)
    blocks = table[:, :_ceil(s["longest"], bs)].long().clamp(min=0)
    j = torch.arange(blocks.shape[1] * bs, device="cuda")
    inside = (j < kv[:, None])[:, None, :, None]                                  # [R, 1, n, 1]

    def read(name):
        x = s[name][:, layer][blocks].float() * s[name + "_scale"][:, layer][blocks][..., None, None]
        x = x.permute(0, 2, 1, 3, 4).reshape(R, H, -1, d)                         # [R, H, n, d]
        return torch.where(inside, x, 0.0)

    i = torch.arange(s["most"], device="cuda")
    row = (starts[:-1, None] + i).clamp(max=len(q) - 1)                           # [R, most]
    x = q[row].float().reshape(R, s["most"], H, G, d).permute(0, 2, 1, 3, 4).reshape(R, H, -1, d)
    score = ((x @ read("k").transpose(-1, -2)) * d ** -0.5).reshape(R, H, s["most"], G, -1)
    place = (j - context[:, None]).clamp(0, 32 * s["words"] - 1)                  # [R, n] among the new rows
    word = s["mask"].long()[row].gather(2, (place >> 5)[:, None].expand(-1, s["most"], -1))
    seen = ((word >> (place & 31)[:, None]) & 1).bool() & (j < kv[:, None])[:, None]
    seen |= (j < context[:, None])[:, None]                                       # [R, most, n]
    score = torch.where(seen[:, None, :, None, :], score, -torch.inf).reshape(R, H, s["most"] * G, -1)
    top = score.amax(-1, keepdim=True)
    top = torch.where(top == -torch.inf, 0.0, top)
    p = torch.exp(score - top)
    total = p.sum(-1, keepdim=True)
    out = (p @ read("v")) / torch.where(total > 0, total, 1.0)
    lse = (top + torch.log(total))[..., 0]
    out = out.reshape(R, H, s["most"], G, d).permute(0, 2, 1, 3, 4).reshape(R, s["most"], H * G, d)
    lse = lse.reshape(R, H, s["most"], G).permute(0, 2, 1, 3).reshape(R, s["most"], H * G)
    r, first = _owner(s)
    at = torch.arange(len(q), device="cuda") - first
    return {"out": out[r, at].bfloat16(), "lse": lse[r, at]}


_ONE = 1 << 42


def _clean(x):
    return torch.nan_to_num(x.float(), nan=0.0).clamp(0.0, 1.0)


def _fixed(x):
    """fp32 values of 0 .. 1 as whole multiples of 2^-42, rounded down."""
    return (x.double() * _ONE).long()


def _verify(s):
    """All requests walk their trees together, a level at a time."""
    starts, parents, tokens = s["starts"].long(), s["parents"].long(), s["tokens"].long()
    R, V, fan = len(starts) - 1, s["target"].shape[1], s["fan"]
    r, first = _owner(s)
    row = torch.arange(s["rows"], device="cuda")
    # child[row, c]: the c-th row whose parent it is, -1 behind the last
    order = torch.zeros_like(row)
    above = torch.where(parents >= 0, first + parents, -1 - row)                  # no two alike without a parent
    for back in range(1, s["most"]):
        order[back:] += above[back:] == above[:-back]
    child = torch.full((s["rows"] + 1, fan), -1, dtype=torch.int64, device="cuda")      # the roots' go behind the last
    child[torch.where(parents >= 0, above, s["rows"]), order] = row
    every = torch.arange(R, device="cuda")
    at, alive = starts[:-1].clone(), starts[1:] > starts[:-1]
    path = torch.full((s["rows"] + 1,), -1, dtype=torch.int64, device="cuda")
    path[at] = 0
    kept = alive.long()
    final, plain = torch.zeros((R, V), device="cuda"), torch.zeros((R, V), device="cuda")
    for _ in range(s["depth"] + 1):
        w = _clean(s["target"][at])
        whole = w
        q = _clean(s["draft"][at]) if s["draft"] is not None else None
        z = torch.full((R,), float(_ONE), dtype=torch.float64, device="cuda")     # in multiples of 2^-42
        found = torch.full((R,), -1, dtype=torch.int64, device="cuda")
        for c in range(fan):
            i = child[at, c]
            t = tokens[i.clamp(min=0)]
            there = alive & (found < 0) & (i >= 0) & (t >= 0) & (t < V)
            t = t.clamp(0, V - 1)
            u, have = s["accept"][i.clamp(min=0)].double(), w[every, t]
            if q is None:
                taken = u * (z / _ONE) < have.double()
            else:
                zf = (z / _ONE).float()
                taken = u * q[every, t].double() * zf.double() < have.double()
            found = torch.where(there & taken, i, found)
            lost = there & ~taken
            if q is None:
                z = torch.where(lost, z - _fixed(have).double(), z)
                w = torch.where(lost[:, None] & (torch.arange(V, device="cuda") == t[:, None]), 0.0, w)
            else:
                rest = (w - q * zf[:, None]).clamp(min=0.0)
                total = _fixed(rest).sum(-1)
                lost &= total > 0
                w, z = torch.where(lost[:, None], rest, w), torch.where(lost, total.double(), z)
        ends = alive & (found < 0)
        final, plain = torch.where(ends[:, None], w, final), torch.where(ends[:, None], whole, plain)
        alive &= found >= 0
        path[torch.where(alive, starts[:-1] + kept, s["rows"])] = found - starts[:-1]
        kept += alive
        at = torch.where(alive, found, at)
    final = torch.where(_fixed(final).sum(-1, keepdim=True) > 0, final, plain)
    sums = _fixed(final).cumsum(-1)
    total = sums[:, -1]
    v = (s["sample"].double() * 2.0 ** 32).long().clamp(0, (1 << 32) - 1)
    # floor(total * v / 2^32) in 64 bits
    high, low = total >> 32, total & 0xffffffff
    point = high * v + ((low * (v >> 16) + (low * (v & 0xffff) >> 16)) >> 16)
    chosen = torch.where(total > 0, (sums <= point[:, None]).sum(-1), -1)
    return {"path": path[:-1].int(), "kept": kept.int(), "next": chosen.int()}


def _keep(s):
    """Rows path[i] of each request to place i: first what is read, then what is written. Rows that are in place are
    written there again, and the first of a request stands for what is behind its last."""
    fmt, bs, K = s["format"], s["block"], s["longest_path"]
    context, kept, starts, kv = s["context"].long(), s["kept"].long(), s["starts"].long(), s["kv"].long()
    i = torch.arange(K, device="cuda")
    path = s["path"].long()[(starts[:-1, None] + i).clamp(max=s["rows"] - 1)]     # [R, K]
    inside = i < kept[:, None]
    same = (inside & (path == i)).long().cumprod(-1).bool()                       # in place, and so all before it
    still = context + same.sum(-1)                                                # tokens that stay where they are
    nb = s["k"].shape[0]

    def where(token):
        return s["table"].gather(1, token // bs).long().reshape(-1), (token % bs).reshape(-1)

    to, to_place = where(context[:, None] + torch.where(inside, i, 0))
    frm, frm_place = where(context[:, None] + torch.where(inside, path, path[:, :1]))
    # of the one block of a request that has tokens in place and takes others: how many
    held = torch.zeros(nb + 1, dtype=torch.int64, device="cuda")
    edge = still % bs
    block = s["table"].gather(1, (still // bs)[:, None])[:, 0].long()
    held[torch.where((edge > 0) & (inside & ~same).any(-1), block, nb)] = edge
    held = held[:nb]
    touched = torch.zeros(nb, dtype=torch.bool, device="cuda")
    touched[to] = True
    got = {}
    for name in ("k", "v"):
        codes, scale = s[name], s[name + "_scale"]
        low = torch.where((held > 0)[:, None, None], scale, 0.0)
        need = low.scatter_reduce(0, to[:, None, None].expand(-1, *scale.shape[1:]), scale[frm], "amax")
        fresh = torch.where(touched[:, None, None], need, scale)
        raw = codes.view(torch.uint8)
        rows = raw[frm, :, :, frm_place]                                          # [moved, L, H, d]
        ratio = (scale[frm] / fresh[to])[..., None]
        again = _codes(rows.view(codes.dtype).float() * ratio, fmt).view(torch.uint8)
        rows = torch.where(ratio == 1.0, rows, again)
        grown = (touched & (held > 0))[:, None, None] & (fresh > scale)
        place = torch.arange(bs, device="cuda") < held[:, None]
        which = grown[..., None, None] & place[:, None, None, :, None]
        factor = torch.where(grown, scale / fresh, 1.0)[..., None, None]
        raw.copy_(torch.where(which, _codes(codes.float() * factor, fmt).view(torch.uint8), raw))
        raw[to, :, :, to_place] = rows
        scale.copy_(fresh)
        got[name], got[name + "_scale"] = codes, scale
    lens = context + kept
    begin, end = (lens + bs - 1) // bs, (kv + bs - 1) // bs
    n = end - begin
    ends, room = n.cumsum(0), len(kv) + s["rows"] // bs
    at = torch.arange(room, device="cuda")
    r = torch.searchsorted(ends, at, right=True).clamp(max=len(kv) - 1)
    entry = (begin[r] + at - (ends - n)[r]).clamp(0, s["table"].shape[1] - 1)
    freed = torch.where(at < ends[-1], s["table"][r, entry], -1)
    return dict(got, lens=lens.int(), freed=freed.int(), count=ends[-1:])


# ---------------------------------------------------------------- in 64 bits

def exact(case, seed):
    """The definitions, request by request, in fp64 and whole numbers."""
    global own
    was, own = own, False
    s = prepare(case, seed)
    own = was
    if case["op"] == "rotate":
        return {name: _exact_rotate(s[name], s["positions"], s[name + "_weight"]) for name in ("q", "k")}
    if case["op"] == "plan":
        return _exact_plan(*_trees(case, seed))
    old, trees, paths = _paths(case)
    if case["op"] == "verify":
        return _exact_verify(s, trees)
    return _exact_attend(case, s, old, trees) if case["op"] == "attend" else _exact_keep(case, s, old, trees, paths)


def _exact_plan(old, trees):
    words, masks, positions = _words(trees), [], []
    for o, t in zip(old, trees):
        own_masks = []
        for i, p in enumerate(t):
            own_masks.append(1 << i | (own_masks[p] if p >= 0 else 0))
        masks += own_masks
        positions += [o + d for d in _depths(t)]
    out = np.array([[m >> 32 * w & 0xffffffff for w in range(words)] for m in masks], dtype=np.uint32).view(np.int32)
    return {"mask": torch.from_numpy(out), "positions": torch.tensor(positions, dtype=torch.int32)}


def _exact_rotate(x, positions, weight):
    out = torch.empty(x.shape, dtype=torch.float64, device="cuda")
    half = x.shape[-1] // 2
    for i in range(0, len(x), 2048):
        y = x[i:i + 2048].double()
        if weight is not None:
            y = y / torch.sqrt((y ** 2).mean(-1, keepdim=True) + EPS) * weight.double()
        angle = positions[i:i + 2048, None, None].double() / THETA ** (torch.arange(half, device="cuda", dtype=torch.float64) / half)
        turn = torch.polar(torch.ones_like(angle), angle) * torch.complex(y[..., :half], y[..., half:])
        out[i:i + 2048, :, :half], out[i:i + 2048, :, half:] = turn.real, turn.imag
    return out


def _exact_attend(case, s, old, trees):
    bs, G, H, d = case["block"], case["group"], case["heads"], case["dim"]
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
    lse = torch.full(s["q"].shape[:2], -torch.inf, dtype=torch.float64, device="cuda")
    at = 0
    for r, (o, t) in enumerate(zip(old, trees)):
        n, rows = o + len(t), slice(at, at + len(t))
        blocks = s["table"][r, :_ceil(n, bs)].long()
        hidden = torch.zeros((len(t), n), dtype=torch.bool)
        hidden[:, o:] = True
        for i, p in enumerate(t):
            if p >= 0:
                hidden[i] &= hidden[p]
            hidden[i, o + i] = False
        hidden = hidden.cuda()

        def read(name, h):
            x = s[name][blocks, s["layer"], h].double() * s[name + "_scale"][blocks, s["layer"], h].double()[:, None, None]
            return x.reshape(-1, d)[:n]

        for h in range(H):
            k, v, g = read("k", h), read("v", h), slice(h * G, (h + 1) * G)
            score = torch.einsum("ngd,td->ngt", s["q"][rows, g].double(), k) / d ** 0.5
            score.masked_fill_(hidden[:, None], -torch.inf)
            lse[rows, g] = torch.logsumexp(score, -1)
            out[rows, g] = torch.softmax(score, -1) @ v
        at += len(t)
    return {"out": out, "lse": lse}


def _exact_verify(s, trees):
    """One request after the other on the host; sums in whole numbers."""
    def host(x):
        return np.clip(np.nan_to_num(x.float().cpu().numpy(), nan=0.0), np.float32(0), np.float32(1))

    def whole(x):
        return np.floor(x.astype(np.float64) * _ONE).astype(np.int64)

    tokens, accept, sample = s["tokens"].tolist(), s["accept"].tolist(), s["sample"].tolist()
    path, kept, chosen, at = [], [], [], 0
    for r, t in enumerate(trees):
        walk = [0]
        while True:
            x = walk[-1]
            p = w = host(s["target"][at + x])
            q = host(s["draft"][at + x]) if s["draft"] is not None else None
            z, found = _ONE, None
            for c in [i for i in range(len(t)) if t[i] == x]:
                token = tokens[at + c]
                if q is None:
                    if accept[at + c] * (z / _ONE) < float(w[token]):
                        found = c
                        break
                    z -= int(whole(w[token:token + 1])[0])
                    w = w.copy()
                    w[token] = 0
                    continue
                scale = np.float32(z / _ONE)
                if accept[at + c] * float(q[token]) * float(scale) < float(w[token]):
                    found = c
                    break
                rest = np.maximum(w - q * scale, np.float32(0))
                if int(whole(rest).sum()):
                    w, z = rest, int(whole(rest).sum())
            if found is None:
                break
            walk.append(found)
        if not whole(w).any():
            w = p
        sums = np.cumsum(whole(w))
        point = int(sums[-1]) * min(max(int(sample[r] * 2 ** 32), 0), 2 ** 32 - 1) >> 32
        chosen.append(int(np.searchsorted(sums, point, side="right")) if sums[-1] else -1)
        path += walk + [-1] * (len(t) - len(walk))
        kept.append(len(walk))
        at += len(t)
    return {"path": torch.tensor(path, dtype=torch.int32), "kept": torch.tensor(kept, dtype=torch.int32),
            "next": torch.tensor(chosen, dtype=torch.int32)}


def _nearest(x, fmt):
    """x in fp64 to the nearest code, ties to even: int8, or e4m3 (steps of 2^-9 at least)."""
    if fmt == "int8":
        return torch.round(x).clamp(-127, 127)
    _, e = torch.frexp(x)
    step = torch.ldexp(torch.ones_like(x), (e - 4).clamp(min=-9))
    return (torch.round(x / step) * step).clamp(-448, 448)


def _exact_keep(case, s, old, trees, paths):
    bs, fmt = case["block"], case["format"]
    table = s["table"].tolist()
    got = {}
    for name in ("k", "v"):
        codes, scale = s[name].double(), s[name + "_scale"].double()
        for r, (o, path) in enumerate(zip(old, paths)):
            i = 0
            while i < len(path):
                # the rows that go into one block
                b, n = (o + i) // bs, 1
                while i + n < len(path) and (o + i + n) // bs == b:
                    n += 1
                rows, i = [(o + j, o + path[j]) for j in range(i, i + n) if path[j] != j], i + n
                if not rows:
                    continue
                here, first = table[r][b], rows[0][0] % bs
                sources = [table[r][f // bs] for _, f in rows]
                fresh = torch.stack([scale[x] for x in sources] + ([scale[here]] if first else [])).amax(0)
                put = [_nearest(codes[x, :, :, f % bs] * (scale[x] / fresh)[..., None], fmt) for x, (_, f) in zip(sources, rows)]
                if first:
                    ratio = (scale[here] / fresh)[..., None, None]
                    codes[here, :, :, :first] = _nearest(codes[here, :, :, :first] * ratio, fmt)
                for (t, _), x in zip(rows, put):
                    codes[here, :, :, t % bs] = x
                scale[here] = fresh
        # int8 codes are whole numbers: no rounding error to speak of
        got[name], got[name + "_scale"] = (codes if fmt == "e4m3" else None), scale
    lens, freed = [o + len(p) for o, p in zip(old, paths)], []
    for r, (o, t) in enumerate(zip(old, trees)):
        freed += table[r][_ceil(lens[r], bs):_ceil(o + len(t), bs)]
    room = len(trees) + s["rows"] // bs
    whole = {"lens": torch.tensor(lens, dtype=torch.int32), "count": torch.tensor([len(freed)]),
             "freed": torch.tensor(freed + [-1] * (room - len(freed)), dtype=torch.int32)}
    return {**{name: got[name] for name in ("k", "v", "k_scale", "v_scale")}, **whole}
