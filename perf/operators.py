"""The serving operators that stand behind a merged cache, as cases to be timed: block tables
and slot maps built on the GPU from request lengths ("tables"), K and V rows written into a
paged cache held in 8 bits with one scale for each block of tokens and head ("append"), and
attention that reads that cache ("attend"), from one token of one request to long prompts.

`run` computes them in elementary torch operations, in 32 bits, or, where `own` is true,
through the package's public entry points.

The 8-bit cache. A pool holds blocks of `block` tokens; the codes of K and V are
[blocks, layers, heads, block, dim] (8-bit floating point e4m3, or int8) and each (block,
layer, head) has one fp32 scale for K and one for V: a stored value is code * scale. A scale
that is written is the smallest power of two 2^k, k in [-60, 60], with max |x| <= 448 * 2^k
(e4m3) or 127 * 2^k (int8) over the finite values of the block; codes are rounded to nearest
even and clamped. A block that already holds tokens keeps its scale unless new tokens need a
larger one; then its codes are rounded again to the larger scale.
"""
import random

import torch

own = False      # True: the package's operators; False: the plain forms below

FORMATS = {"e4m3": torch.float8_e4m3fn, "int8": torch.int8}


# ---------------------------------------------------------------- cases

def listed():
    return [
        # One decoding step of a small batch: every request gets one token. Latency only.
        {"name": "tables_decode_16", "op": "tables", "requests": 16, "old_lo": 30, "old_hi": 3000,
         "new_lo": 1, "new_hi": 1, "prompts": 0, "block": 16, "mix": 1},
        # A mixed step of a large batch: most requests decode, some bring a prompt chunk.
        {"name": "tables_mixed_509", "op": "tables", "requests": 509, "old_lo": 1, "old_hi": 6000,
         "new_lo": 200, "new_hi": 2048, "prompts": 24, "block": 16, "mix": 2},
        # Merged caches of 64 serving requests are taken in at once (three fragments each,
        # about 5,000 tokens), nothing cached before.
        {"name": "tables_prompts_64", "op": "tables", "requests": 64, "old_lo": 0, "old_hi": 0,
         "new_lo": 1536, "new_hi": 12288, "prompts": 64, "block": 32, "mix": 3},
        # One layer's K and V of one new token for each of 48 requests (a decoding step).
        {"name": "append_decode_48", "op": "append", "requests": 48, "old_lo": 100, "old_hi": 3000,
         "new_lo": 1, "new_hi": 1, "prompts": 0, "layers": 1, "heads": 8, "dim": 128,
         "block": 16, "format": "e4m3", "mix": 4},
        # One layer of a ragged batch in int8 (head_dim 64, odd lengths, part-filled blocks).
        {"name": "append_ragged_int8", "op": "append", "requests": 37, "old_lo": 1, "old_hi": 900,
         "new_lo": 1, "new_hi": 1500, "prompts": 37, "layers": 1, "heads": 12, "dim": 64,
         "block": 32, "format": "int8", "mix": 5},
        # A rendered merge (Qwen3-4B shape, all 36 layers, about 5,200 tokens) goes into the
        # 8-bit cache of the request that will answer from it.
        {"name": "append_merge_4b", "op": "append", "requests": 1, "old_lo": 0, "old_hi": 0,
         "new_lo": 5208, "new_hi": 5208, "prompts": 1, "layers": 36, "heads": 8, "dim": 128,
         "block": 16, "format": "e4m3", "mix": 6},
        # One request answers from the Qwen3-1.7B-shaped merge of 2 x 512 tokens, one token
        # at a time: the smallest attention.
        {"name": "attend_17b_1x1041", "op": "attend", "requests": 1, "old_lo": 1040, "old_hi": 1040,
         "new_lo": 1, "new_hi": 1, "prompts": 0, "layers": 2, "heads": 8, "group": 2, "dim": 128,
         "block": 16, "format": "e4m3", "mix": 7},
        # A decoding step of 64 requests over merged caches of ragged lengths.
        {"name": "attend_4b_64_ragged", "op": "attend", "requests": 64, "old_lo": 600,
         "old_hi": 12000, "new_lo": 1, "new_hi": 1, "prompts": 0, "layers": 1, "heads": 8,
         "group": 4, "dim": 128, "block": 16, "format": "e4m3", "mix": 8},
        # Two long requests: few rows, a long axis.
        {"name": "attend_4b_2_long", "op": "attend", "requests": 2, "old_lo": 98304,
         "old_hi": 131072, "new_lo": 1, "new_hi": 1, "prompts": 0, "layers": 1, "heads": 8,
         "group": 4, "dim": 128, "block": 32, "format": "e4m3", "mix": 9},
        # A few tokens of each request at once (a draft being checked), int8, head_dim 64.
        {"name": "attend_int8_verify", "op": "attend", "requests": 29, "old_lo": 50,
         "old_hi": 4000, "new_lo": 3, "new_hi": 4, "prompts": 29, "layers": 2, "heads": 12,
         "group": 1, "dim": 64, "block": 16, "format": "int8", "mix": 10},
        # A chunk of the judge's prompt reads a merged cache of 4 x 4096 tokens.
        {"name": "attend_4b_chunk_2048", "op": "attend", "requests": 1, "old_lo": 16384,
         "old_hi": 16384, "new_lo": 2048, "new_hi": 2048, "prompts": 1, "layers": 1, "heads": 8,
         "group": 4, "dim": 128, "block": 16, "format": "e4m3", "mix": 11},
        # Ragged prompts without any cached tokens in front, head_dim 256, int8.
        {"name": "attend_d256_prompts", "op": "attend", "requests": 5, "old_lo": 0, "old_hi": 0,
         "new_lo": 150, "new_hi": 2300, "prompts": 5, "layers": 1, "heads": 4, "group": 2,
         "dim": 256, "block": 64, "format": "int8", "mix": 12},
    ]


_SHAPES = [(8, 128), (8, 128), (4, 64), (4, 256), (12, 64), (2, 32)]


def draw(rng):
    def size(lo, hi):
        return int(round(lo * (hi / lo) ** rng.random()))

    op = rng.choice(["tables", "append", "append", "attend", "attend", "attend"])
    case = {"op": op, "block": rng.choice([16, 16, 32, 64, 128]), "mix": rng.randrange(1 << 20)}
    if op == "tables":
        requests = size(1, 1024)
        prompts = rng.choice([0, min(requests, size(1, 48)), requests])
        most = max(1, min(12288, 600000 // max(1, prompts)))
        case.update(requests=requests, old_lo=rng.choice([0, 1, 100]), old_hi=size(100, 8000),
                    new_lo=1, new_hi=size(1, most) if prompts else 1, prompts=prompts)
        return case
    heads, dim = rng.choice(_SHAPES)
    case.update(heads=heads, dim=dim, format=rng.choice(["e4m3", "e4m3", "int8"]))
    if op == "append":
        layers = rng.choice([1, 1, 2, 16, 36])
        budget = 190_000_000 // (layers * heads * dim)          # tokens written at most
        requests = size(1, 128)
        prompts = rng.choice([0, requests])
        top = size(1, max(1, min(6000, budget // requests))) if prompts else 1
        pool = 190_000_000 // (layers * heads * dim * requests)  # cached tokens before, each
        case.update(requests=requests, old_lo=0, old_hi=max(1, min(3000, pool)),
                    new_lo=max(1, top // 8), new_hi=top, prompts=prompts, layers=layers)
        return case
    group = rng.choice([1, 2, 4, 4, 5, 8])
    case.update(layers=rng.choice([1, 1, 2]), group=group)
    if rng.random() < 0.6:                                       # single tokens, or a few
        requests = size(1, 160)
        budget = 300_000_000 // (heads * dim * requests)
        top = size(16, max(17, min(131072, budget)))
        few = rng.choice([1, 1, 1, 2, 4])
        case.update(requests=requests, old_lo=max(0, top // rng.choice([1, 4, 40])), old_hi=top,
                    new_lo=1, new_hi=few, prompts=requests if few > 1 else 0)
    else:                                                        # prompts and chunks of them
        requests = size(1, 8)
        new = size(17, 2048)
        old = rng.choice([0, size(16, 16384)])
        while requests > 1 and requests * heads * group * dim * new * (old + new) > 1.5e11:
            requests -= 1
        while heads * group * dim * new * (old + new) > 1.5e11:
            new //= 2
        case.update(requests=requests, old_lo=old // 2, old_hi=old, new_lo=max(1, new // 5),
                    new_hi=new, prompts=requests)
    return case


def _lengths(case):
    """The requests' cached and new token counts, spread over their ranges (by logarithm)."""
    rng = random.Random(case["mix"])

    def between(lo, hi):
        return int(round((lo + 1) * ((hi + 1) / (lo + 1)) ** rng.random())) - 1

    n = case["requests"]
    old = [between(case["old_lo"], case["old_hi"]) for _ in range(n)]
    new = [between(case["new_lo"], case["new_hi"]) if i < case["prompts"] else 1 for i in range(n)]
    both = list(zip(old, new))
    rng.shuffle(both)
    return [o for o, _ in both], [t for _, t in both]


def _ceil(a, b):
    return -(-a // b)


def work(case):
    old, new = _lengths(case)
    n, bs, rows = len(old), case["block"], sum(new)
    if case["op"] == "tables":
        fresh = sum(_ceil(o + t, bs) - _ceil(o, bs) for o, t in zip(old, new))
        # lengths, free blocks and the tables' part-filled entries in; entries, slots, starts out
        return {"bytes": 4 * n * 4 + 8 * fresh + 8 * rows, "flops": 0}
    H, d = case["heads"], case["dim"]
    if case["op"] == "append":
        L = case["layers"]
        # bf16 rows in, codes out; the scales of the blocks written; the slots
        blocks = sum(_ceil(o + t, bs) - o // bs for o, t in zip(old, new))
        return {"bytes": L * H * (rows * d * 2 * 3 + blocks * 8) + 8 * rows, "flops": 0}
    G = case["group"]
    tokens = sum(o + t for o, t in zip(old, new))
    blocks = sum(_ceil(o + t, bs) for o, t in zip(old, new))
    pairs = sum(t * o + t * (t + 1) // 2 for o, t in zip(old, new))
    return {"bytes": H * (tokens * d * 2 + blocks * 8) + 4 * blocks + rows * H * G * (4 * d + 4),
            "flops": 4.0 * pairs * H * G * d}


# ---------------------------------------------------------------- inputs

def _generator(seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    return gen


def _normal(shape, gen):
    return torch.randn(shape, generator=gen, device="cuda")


def _limit(fmt):
    """(largest code, its exponent and mantissa as frexp gives them)."""
    return (448.0, 9, 0.875) if fmt == "e4m3" else (127.0, 7, 0.9921875)


def _pow2(k, dtype=torch.float32):
    """2^k exactly, from its bits (a library power need not be exact)."""
    if dtype == torch.float32:
        return ((k.int() + 127) << 23).view(torch.float32)
    return ((k.long() + 1023) << 52).view(torch.float64)


def _pow2_scale(amax, fmt):
    """The smallest 2^k, k in [-60, 60], that brings amax within the format's largest code."""
    _, e, m = _limit(fmt)
    mant, exp = torch.frexp(amax)
    k = (exp - e + (mant > m)).clamp(-60, 60)
    k = torch.where(amax > 0, k, torch.full_like(k, -60))
    return _pow2(k)


def _codes(x, fmt):
    """x (already divided by its scale) as codes of the format: nearest even, clamped; no NaN."""
    top = _limit(fmt)[0]
    x = torch.nan_to_num(x, nan=0.0, posinf=top, neginf=-top).clamp(-top, top)
    return x.round().to(torch.int8) if fmt == "int8" else x.to(torch.float8_e4m3fn)


def _old_tokens(case, shape, gen):
    """Codes and scales [blocks, layers, heads, block, dim] of a cache in use: keys with a few
    strong channels, block scales that vary, garbage where nothing has been written."""
    fmt = case["format"]
    codes = torch.empty(shape, dtype=FORMATS[fmt], device="cuda")
    scale = torch.empty(shape[:3], device="cuda")
    step = max(1, (1 << 26) // max(1, codes[0].numel()))
    strong = 1 + 2 * (torch.rand(shape[-1], generator=gen, device="cuda") < 0.05)
    for b in range(0, shape[0], step):
        x = _normal((min(step, shape[0] - b),) + tuple(shape[1:]), gen) * strong
        x *= 0.5 + torch.rand(x.shape[:3] + (1, 1), generator=gen, device="cuda")
        s = _pow2_scale(x.abs().amax((-1, -2)), fmt)
        scale[b:b + step] = s
        codes[b:b + step] = _codes(x / s[..., None, None], fmt)
    return codes, scale


def _place(case, seed):
    """Lengths on the GPU, and the block tables before the step: the blocks of the cached
    tokens named, the others -1. Blocks are handed out in a shuffled order."""
    old, new = _lengths(case)
    bs = case["block"]
    width = max(_ceil(o + t, bs) for o, t in zip(old, new)) + 3
    total = sum(_ceil(o + t, bs) for o, t in zip(old, new))
    order = torch.randperm(total + 7, generator=_generator(seed + 1), device="cuda").int()
    old_t = torch.tensor(old, dtype=torch.int32, device="cuda")
    new_t = torch.tensor(new, dtype=torch.int32, device="cuda")
    held = (old_t.long() + bs - 1) // bs
    at = held.cumsum(0) - held
    j = torch.arange(width, device="cuda")
    table = torch.where(j < held[:, None], order[(at[:, None] + j).clamp(max=total + 6)],
                        torch.full((), -1, dtype=torch.int32, device="cuda"))
    return {"old": old_t, "new": new_t, "table": table, "free": order[int(held.sum()):].clone(),
            "rows": sum(new), "most": max(new), "longest": max(o + t for o, t in zip(old, new)),
            "blocks": total + 7, "block": bs}


def prepare(case, seed):
    place = _place(case, seed)
    state = dict(place, op=case["op"], seed=seed, format=case.get("format"))
    gen = _generator(seed)
    if own:
        import paper_2607_01308_gb300 as cm
        state["batch"] = cm.QBatch(_context(cm), len(place["old"]), place["table"].shape[1],
                                     place["rows"], place["block"])
        state["batch"].block_table.copy_(place["table"])
    if case["op"] == "tables":
        return state
    H, d, L, bs = case["heads"], case["dim"], case["layers"], case["block"]
    shape = (place["blocks"], L, H, bs, d)
    for name in ("k", "v"):
        state[name], state[name + "_scale"] = _old_tokens(case, shape, gen)
    table, starts, kv, slots, _ = _tables(place)
    state.update(starts=starts, kv=kv, slots=slots, layer=L - 1)
    if case["op"] == "append":
        for name in ("new_k", "new_v"):
            x = torch.empty((L, H, place["rows"], d), dtype=torch.bfloat16, device="cuda")
            for l in range(L):
                # some rows are larger than what their blocks were scaled for
                big = 1 + 5 * (torch.rand((H, place["rows"], 1), generator=gen, device="cuda") < 0.2)
                x[l] = _normal((H, place["rows"], d), gen) * big
            state[name] = x
    else:
        state["table"] = table
        state["group"] = case["group"]
        state["q"] = _normal((place["rows"], H * case["group"], d), gen).bfloat16()
        # what lies behind the last token of a request is not zero
        junk = 0x7F if case["format"] == "e4m3" else 77
        last = table.gather(1, ((kv.long() - 1) // bs)[:, None])[:, 0].long()
        tail = torch.arange(bs, device="cuda") > ((kv.long() - 1) % bs)[:, None]
        for name in ("k", "v"):
            raw = state[name].view(torch.uint8)
            raw[last] = torch.where(tail[:, None, None, :, None], torch.full((), junk, dtype=torch.uint8, device="cuda"), raw[last])
    if own:
        state["cache"] = cm.QCache.from_tensors(_context(cm), state["k"], state["v"],
                                                  state["k_scale"], state["v_scale"])
        if case["op"] == "attend":
            b = state["batch"]
            b.block_table.copy_(table)
            b.row_starts.copy_(starts)
            b.kv_lens.copy_(kv)
            b.max_new = place["most"]
            state["out"] = torch.empty_like(state["q"])
            state["lse"] = torch.empty(state["q"].shape[:2], device="cuda")
    return state


_contexts = []


def _context(cm):
    """One context for the life of the process, as a serving process keeps it."""
    if not _contexts:
        _contexts.append(cm.Context(0))
    return _contexts[0]


# ---------------------------------------------------------------- one pass

def run(state):
    op = state["op"]
    if own:
        if op == "tables":
            b = state["batch"]
            b.schedule(state["old"], state["new"], state["free"])
            return {"table": b.block_table, "starts": b.row_starts, "kv": b.kv_lens,
                    "slots": b.slot_map, "counts": b.counts}
        cache = state["cache"]
        if op == "append":
            cache.append(state["new_k"], state["new_v"], state["slots"])
            return {"k": cache.k, "v": cache.v, "k_scale": cache.k_scale, "v_scale": cache.v_scale}
        out, lse = cache.attend(state["q"], state["batch"], layer=state["layer"], out=state["out"],
                                lse=state["lse"])
        return {"out": out, "lse": lse}
    if op == "tables":
        table, starts, kv, slots, counts = _tables(state)
        return {"table": table, "starts": starts, "kv": kv, "slots": slots, "counts": counts}
    if op == "append":
        return _append(state)
    return _attend(state)


def _tables(s):
    """Blocks for the new tokens, taken from the free list in request order; the slot (block *
    block size + place in it) of each new row; where each request's rows start."""
    bs, old, new = s["block"], s["old"].long(), s["new"].long()
    kv = old + new
    first, last = (old + bs - 1) // bs, (kv + bs - 1) // bs
    need = last - first
    at = need.cumsum(0) - need
    j = torch.arange(s["table"].shape[1], device="cuda")
    fresh = (j >= first[:, None]) & (j < last[:, None])
    which = (at[:, None] + j - first[:, None]).clamp(0, len(s["free"]) - 1)
    table = torch.where(fresh, s["free"][which], s["table"])
    starts = torch.cat([torch.zeros_like(new[:1]), new.cumsum(0)])
    row = torch.arange(s["rows"], device="cuda")
    r = torch.searchsorted(starts[1:].contiguous(), row, right=True)
    pos = old[r] + row - starts[r]
    slots = table[r, pos // bs].long() * bs + pos % bs
    counts = torch.stack([need.sum(), starts[-1]])
    return table, starts.int(), kv.int(), slots, counts


def _append(s):
    """The rows into their slots: per block the largest magnitude, the scale it needs, the codes
    held before rounded again where the scale grows, the new codes."""
    fmt, slots = s["format"], s["slots"]
    nb, L, H, bs, d = s["k"].shape
    block, place = slots // bs, slots % bs
    begin = torch.full((nb,), bs, device="cuda").scatter_reduce(0, block, place, "amin")
    touched = torch.zeros(nb, dtype=torch.bool, device="cuda")
    touched[block] = True
    held = torch.arange(bs, device="cuda") < begin[:, None]                       # [nb, bs]
    got = {}
    for name in ("k", "v"):
        codes, scale, x = s[name], s[name + "_scale"], s["new_" + name]
        size = x.abs().float()
        size = torch.where(torch.isfinite(size), size, 0.0).amax(-1).permute(2, 0, 1)   # [rows, L, H]
        amax = torch.zeros((nb, L, H), device="cuda")
        amax.scatter_reduce_(0, block[:, None, None].expand(-1, L, H), size, "amax")
        needed = _pow2_scale(amax, fmt)
        fresh = torch.where((begin > 0)[:, None, None], torch.maximum(scale, needed), needed)
        fresh = torch.where(touched[:, None, None], fresh, scale)
        grown = (touched & (begin > 0))[:, None, None] & (fresh > scale)
        where = grown[..., None, None] & held[:, None, None, :, None]
        again = _codes(codes.float() * (scale / fresh)[..., None, None], fmt)
        kept = torch.where(where, again.view(torch.uint8), codes.view(torch.uint8))
        rows = _codes(x.float().permute(2, 0, 1, 3) / fresh[block][..., None], fmt)     # [rows, L, H, d]
        kept[block, :, :, place] = rows.view(torch.uint8)
        codes.view(torch.uint8).copy_(kept)
        scale.copy_(fresh)
        got[name], got[name + "_scale"] = codes, scale
    return got


def _attend(s):
    """softmax(q k^T / sqrt(d)) v over each request's own cached tokens, causal: row i of n
    new ones sees the first kv - n + i + 1 tokens."""
    table, kv, starts, q = s["table"], s["kv"].long(), s["starts"].long(), s["q"]
    bs, G, layer = s["block"], s["group"], s["layer"]
    H, d = s["k"].shape[2], s["k"].shape[4]
    R, N = len(kv), s["longest"]
    blocks = table[:, :(N + bs - 1) // bs].long().clamp(min=0)
    j = torch.arange(blocks.shape[1] * bs, device="cuda")
    inside = (j < kv[:, None])[:, None, :, None]                                  # [R, 1, n, 1]

    def read(name):
        x = s[name][:, layer][blocks].float() * s[name + "_scale"][:, layer][blocks][..., None, None]
        x = x.permute(0, 2, 1, 3, 4).reshape(R, H, -1, d)                         # [R, H, n, d]
        return torch.where(inside, x, 0.0)

    n = (starts[1:] - starts[:-1])
    i = torch.arange(s["most"], device="cuda")
    row = (starts[:-1, None] + i).clamp(max=len(q) - 1)                           # [R, most]
    x = q[row].float().reshape(R, s["most"], H, G, d).permute(0, 2, 1, 3, 4).reshape(R, H, -1, d)
    score = (x @ read("k").transpose(-1, -2)) * d ** -0.5
    last = (kv - n)[:, None] + i                                                  # [R, most]
    seen = j <= last[:, :, None]
    score = score.reshape(R, H, s["most"], G, -1)
    score = torch.where(seen[:, None, :, None, :], score, -torch.inf).reshape(R, H, s["most"] * G, -1)
    top = score.amax(-1, keepdim=True)
    top = torch.where(top == -torch.inf, 0.0, top)
    p = torch.exp(score - top)
    total = p.sum(-1, keepdim=True)
    out = (p @ read("v")) / torch.where(total > 0, total, 1.0)
    lse = (top + torch.log(total))[..., 0]
    out = out.reshape(R, H, s["most"], G, d).permute(0, 2, 1, 3, 4).reshape(R, s["most"], H * G, d)
    lse = lse.reshape(R, H, s["most"], G).permute(0, 2, 1, 3).reshape(R, s["most"], H * G)
    at = torch.arange(len(q), device="cuda")
    r = torch.searchsorted(starts[1:].contiguous(), at, right=True)
    return {"out": out[r, at - starts[r]].bfloat16(), "lse": lse[r, at - starts[r]]}


# ---------------------------------------------------------------- in 64 bits

def exact(case, seed):
    """The definitions, request by request (block by block for the append), in fp64."""
    if case["op"] == "tables":
        return None                    # whole numbers only
    global own
    was, own = own, False
    s = prepare(case, seed)
    own = was
    return _exact_append(case, s) if case["op"] == "append" else _exact_attend(case, s)


def _exact_append(case, s):
    bs, fmt = case["block"], case["format"]
    top = 448.0 if fmt == "e4m3" else 127.0
    old, new = _lengths(case)
    slots, got = s["slots"], {}
    for name in ("k", "v"):
        codes, scale = s[name].double(), s[name + "_scale"].double()
        rows = s["new_" + name]
        at = 0
        for o, t in zip(old, new):
            # the part-filled block first, then whole ones together, then the rest
            head = min(t, -o % bs)
            spans = [(at, head)] if head else []
            whole = (t - head) // bs
            if whole:
                spans.append((at + head, whole * bs))
            if t - head - whole * bs:
                spans.append((at + head + whole * bs, t - head - whole * bs))
            for begin, n in spans:
                per = min(n, bs)
                x = rows[:, :, begin:begin + n].double().unflatten(2, (n // per, per)).movedim(2, 0)
                b = slots[begin:begin + n:per] // bs
                p = int(slots[begin] % bs)
                size = x.abs().amax((-1, -2))
                k = torch.ceil(torch.log2(size / top)).clamp(-200, 200)
                up, half = _pow2(k, torch.float64), _pow2(k - 1, torch.float64)
                k += (size > top * up).double() - (size <= top * half).double()
                f = _pow2(k.clamp(-60, 60), torch.float64)
                if p:
                    f = torch.maximum(f, scale[b])
                    before = codes[b, :, :, :p] * scale[b][..., None, None]
                    codes[b, :, :, :p] = _nearest(before / f[..., None, None], fmt)
                codes[b, :, :, p:p + per] = _nearest(x / f[..., None, None], fmt)
                scale[b] = f
            at += t
        # int8 codes are whole numbers: no rounding error to speak of
        got[name], got[name + "_scale"] = (codes if fmt == "e4m3" else None), scale
    return {name: got[name] for name in ("k", "v", "k_scale", "v_scale")}


def _nearest(x, fmt):
    """x in fp64 to the nearest code, ties to even: int8, or e4m3 (steps of 2^-9 at least)."""
    if fmt == "int8":
        return torch.round(x).clamp(-127, 127)
    _, e = torch.frexp(x)
    step = _pow2((e - 4).clamp(min=-9), torch.float64)
    return (torch.round(x / step) * step).clamp(-448, 448)


def _exact_attend(case, s):
    old, new = _lengths(case)
    bs, G, H, d = case["block"], case["group"], case["heads"], case["dim"]
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
    lse = torch.full(s["q"].shape[:2], -torch.inf, dtype=torch.float64, device="cuda")
    at = 0
    for r, (o, t) in enumerate(zip(old, new)):
        n = o + t
        blocks = s["table"][r, :_ceil(n, bs)].long()

        def read(name, h):
            x = s[name][blocks, s["layer"], h].double() * s[name + "_scale"][blocks, s["layer"], h].double()[:, None, None]
            return x.reshape(-1, d)[:n]

        hidden = torch.arange(n, device="cuda") > o + torch.arange(t, device="cuda")[:, None]
        for h in range(H):
            k, v = read("k", h), read("v", h)
            for g in range(h * G, (h + 1) * G):
                score = s["q"][at:at + t, g].double() @ k.T / d ** 0.5
                score.masked_fill_(hidden, -torch.inf)
                lse[at:at + t, g] = torch.logsumexp(score, -1)
                out[at:at + t, g] = torch.softmax(score, -1) @ v
        at += t
    return {"out": out, "lse": lse}
