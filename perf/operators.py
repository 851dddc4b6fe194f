"""The operators around a paged cache of keys and values: what they are timed and checked on.

  tables      block tables and slot maps from request lengths: a decode step of 1 .. 1024 requests, chunks of up to 65536 tokens
  rotary      rotary positions: interleaved and half layouts, the whole head or a part of it, scaled frequencies, fp32 / bf16 / fp16,
              1 .. 32768 tokens; forward and gradient on tensors, or keys and values stored in the cache
  attention   new tokens over the cache, fp16 / bf16, head dim 32 / 64 / 96 / 128, 1 to 16 query heads to a key head: one token a request over
              1 .. 131072 keys, a few tokens a request, chunks of thousands of tokens

`own` false: the operators in elementary torch operations.  True: the calls of this library.  What both are given is the same.
"""
import math
import random

import numpy as np
import torch

own = False

DT = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
SIZE = {"f32": 4, "f16": 2, "bf16": 2}


def listed():
    return [
        # a decode step of a small batch: every request gets one token, now and then a page; nothing but latency
        {"name": "tables_decode", "op": "tables", "requests": 48, "tokens": 48, "block": 16, "width": 256, "new": "one"},
        # a large batch of prompts in chunks, some cut by the token budget
        {"name": "tables_chunks", "op": "tables", "requests": 515, "tokens": 32768, "block": 32, "width": 1024, "new": "chunk"},
        # the keys and values of a decode step, packed with the queries by the projection, into the cache
        {"name": "rotary_store_decode", "op": "rotary", "dtype": "bf16", "tokens": 32, "q_heads": 32, "k_heads": 8, "dim": 128, "rot": 128,
         "layout": "half", "store": True, "inverse": False, "block": 16, "far": 32768, "factor": 8.0},
        # ... of a chunk of a prompt, with half of the head rotated
        {"name": "rotary_store_chunk", "op": "rotary", "dtype": "f16", "tokens": 8191, "q_heads": 24, "k_heads": 24, "dim": 64, "rot": 32,
         "layout": "half", "store": True, "inverse": False, "block": 64, "far": 131072, "factor": 1.0},
        # a training batch in fp32, neighbouring elements as pairs
        {"name": "rotary_train_f32", "op": "rotary", "dtype": "f32", "tokens": 8192, "q_heads": 16, "k_heads": 16, "dim": 64, "rot": 64,
         "layout": "interleaved", "store": False, "inverse": False, "block": 0, "far": 2048, "factor": 1.0},
        # the gradient of a training batch of long sequences
        {"name": "rotary_gradient", "op": "rotary", "dtype": "bf16", "tokens": 16384, "q_heads": 32, "k_heads": 8, "dim": 128, "rot": 128,
         "layout": "half", "store": False, "inverse": True, "block": 0, "far": 16384, "factor": 4.0},
        # a decode step of a few short requests: latency
        {"name": "attention_decode_small", "op": "attention", "dtype": "f16", "requests": 4, "new": 1, "context": 500, "spread": "ragged",
         "q_heads": 8, "kv_heads": 2, "dim": 64, "block": 16, "order": "head", "window": 0, "lse": False, "pattern": 1},
        # a decode step of a server's batch, requests of very different lengths
        {"name": "attention_decode_batch", "op": "attention", "dtype": "bf16", "requests": 64, "new": 1, "context": 24000, "spread": "ragged",
         "q_heads": 32, "kv_heads": 8, "dim": 128, "block": 16, "order": "head", "window": 0, "lse": False, "pattern": 2},
        # one long document: a single row of work to share among all of the chip
        {"name": "attention_decode_long", "op": "attention", "dtype": "bf16", "requests": 1, "new": 1, "context": 131072, "spread": "even",
         "q_heads": 32, "kv_heads": 8, "dim": 128, "block": 64, "order": "token", "window": 0, "lse": False, "pattern": 3},
        # a few guessed tokens a request, checked in one go, with a sliding window and the log-sum-exp
        {"name": "attention_few_window", "op": "attention", "dtype": "f16", "requests": 37, "new": 5, "context": 9000, "spread": "ragged",
         "q_heads": 24, "kv_heads": 4, "dim": 96, "block": 32, "order": "token", "window": 4096, "lse": True, "pattern": 4},
        # prompts in chunks, and single tokens among them, behind long contexts
        {"name": "attention_chunk", "op": "attention", "dtype": "bf16", "requests": 8, "new": 1024, "context": 12000, "spread": "ragged",
         "q_heads": 32, "kv_heads": 8, "dim": 128, "block": 16, "order": "head", "window": 0, "lse": False, "pattern": 5},
        # whole prompts without a context before them, a key head for every query head
        {"name": "attention_prompt", "op": "attention", "dtype": "f16", "requests": 4, "new": 2048, "context": 2048, "spread": "even",
         "q_heads": 16, "kv_heads": 16, "dim": 64, "block": 128, "order": "head", "window": 0, "lse": True, "pattern": 6},
    ]


def _log(rng, lo, hi):
    """A whole number between lo and hi, spread over the logarithm; half of them odd."""
    n = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
    return max(lo, min(hi, n | 1 if rng.random() < 0.5 else n))


def draw(rng):
    op = rng.choice(("tables", "rotary", "attention", "attention"))
    if op == "tables":
        new = rng.choice(("one", "chunk"))
        requests = _log(rng, 1, 1024)
        block = rng.choice((8, 16, 32, 64, 128))
        return {"op": op, "requests": requests, "tokens": requests if new == "one" else _log(rng, 64, 65536), "block": block,
                "width": _log(rng, 16, 65536 // block), "new": new}
    if op == "rotary":
        store = rng.random() < 0.5
        dim = rng.choice((32, 64, 80, 96, 128, 256))
        k_heads = rng.choice((1, 2, 3, 4, 8, 12, 16))
        q_heads = k_heads * rng.choice((1, 1, 2, 4, 8))
        most = max(1, min(32768, (400 << 20) // ((q_heads + 2 * k_heads) * dim * 8)))
        return {"op": op, "dtype": rng.choice(("bf16", "f16") if store else ("bf16", "f16", "f32")), "tokens": _log(rng, 1, most), "q_heads": q_heads,
                "k_heads": k_heads, "dim": dim, "rot": rng.choice((dim, dim, dim // 2, 24)), "layout": rng.choice(("half", "interleaved")), "store": store,
                "inverse": not store and rng.random() < 0.5, "block": rng.choice((16, 32, 64, 128)) if store else 0,
                "far": _log(rng, 1, 1 << 20), "factor": rng.choice((1.0, 1.0, 4.0, 8.0))}
    kind = rng.choice(("one", "few", "chunk"))
    kv_heads = rng.choice((1, 2, 4, 8, 16) if kind != "chunk" else (1, 2, 4, 8))
    share = rng.choice((1, 2, 3, 4, 8, 16) if kind != "chunk" else (1, 2, 4, 8))
    dim = rng.choice((32, 64, 96, 128, 128))
    requests = _log(rng, 1, 128 if kind != "chunk" else 8)
    new = 1 if kind == "one" else _log(rng, 2, 8) if kind == "few" else _log(rng, 32, 2048)
    # keys in all: what the largest listed case of the kind has
    most = (64 * 24000 * 8 * 128) // (requests * kv_heads * dim)
    if kind != "one":
        most = min(most, (8 * 1024 * 12000 * 32) // (requests * kv_heads * share * new))
    context = _log(rng, 1, max(2, min(131072 if kind == "one" else 32768, most)))
    block = rng.choice((16, 32, 64, 128))
    return {"op": op, "dtype": rng.choice(("bf16", "f16")), "requests": requests, "new": new, "context": max(context, new), "spread": rng.choice(("ragged", "even")),
            "q_heads": kv_heads * share, "kv_heads": kv_heads, "dim": dim, "block": block, "order": rng.choice(("head", "token")),
            "window": rng.choice((0, 0, 0, 128, 1000, 4096)), "lse": rng.random() < 0.5, "pattern": rng.randrange(1 << 20)}


def prepare(case, seed):
    return {"tables": _prepare_tables, "rotary": _prepare_rotary, "attention": _prepare_attention}[case["op"]](case, seed)


def run(state):
    return {"tables": _run_tables, "rotary": _run_rotary, "attention": _run_attention}[state["op"]](state)


def exact(case, seed):
    return {"tables": _exact_tables, "rotary": _exact_rotary, "attention": _exact_attention}[case["op"]](case, seed)


def work(case):
    return {"tables": _work_tables, "rotary": _work_rotary, "attention": _work_attention}[case["op"]](case)


def _generator(seed):
    g = torch.Generator("cuda")
    g.manual_seed(seed)
    return g


def _int32(a):
    return torch.from_numpy(np.ascontiguousarray(a, dtype=np.int32)).cuda()


# ---------------------------------------------------------------------------------------------------- block tables

def _table_lengths(case, seed):
    """Tokens in the cache and new tokens of every request: a few idle, a few at the end of their row."""
    r = np.random.default_rng(seed)
    b, most = case["requests"], case["block"] * case["width"]
    cached = np.exp(r.uniform(0, math.log(most), b)).astype(np.int64)
    if case["new"] == "one":
        fresh = (r.random(b) > 0.05).astype(np.int64)
    else:
        fresh = r.integers(0, max(2, 5 * case["tokens"] // (2 * b)), b)
        cached[r.random(b) < 0.3] = 0
    cached[r.random(b) < 0.05] = most - 1
    return cached, fresh


def _prepare_tables(case, seed):
    r = np.random.default_rng(seed + 1)
    b, w, block = case["requests"], case["width"], case["block"]
    cached, fresh = _table_lengths(case, seed)
    n_free = case["tokens"] // block + b
    held = np.minimum(-(-cached // block), w)
    blocks = int(held.sum()) + n_free
    pages = r.permutation(blocks).astype(np.int32)
    table = np.full((b, w), -1, np.int32)
    table[np.arange(w)[None, :] < held[:, None]] = pages[:held.sum()]
    s = {"op": "tables", "cached": _int32(cached), "fresh": _int32(fresh), "free": _int32(pages[held.sum():]), "table": _int32(table), "tokens": case["tokens"],
         "block": block, "blocks": blocks}
    if own:
        from paper_1911_11576_amd import Plan
        e = lambda *n: torch.empty(n, dtype=torch.int32, device="cuda")  # noqa: E731
        s["plan"] = Plan.block_tables(requests=b, tokens=case["tokens"], blocks=blocks, block_size=block, table_blocks=w, free_blocks=n_free)
        s["outputs"] = [s["table"], e(b), e(b + 1), e(case["tokens"]), e(case["tokens"]), e(2)]
    return s


def _run_tables(s):
    if own:
        s["plan"].launch([s["cached"], s["fresh"], s["free"]], s["outputs"])
        return s["outputs"]
    table, block, free = s["table"], s["block"], s["free"]
    b, w = table.shape
    most = w * block
    cached = s["cached"].long().clamp(0, most)
    fresh = torch.minimum(s["fresh"].long().clamp(min=0), most - cached)
    ends = fresh.cumsum(0).clamp(max=s["tokens"])
    starts = torch.cat([torch.zeros_like(ends[:1]), ends])
    lengths = cached + starts[1:] - starts[:-1]
    have, need = (cached + block - 1) // block, (lengths + block - 1) // block
    ends_of_pages = (need - have).cumsum(0)
    taken_before = ends_of_pages - (need - have)
    # the entries that are new, from the front of the free list
    j = torch.arange(w, device="cuda")
    place = taken_before[:, None] + j - have[:, None]
    page = torch.where(place < len(free), free[place.clamp(0, len(free) - 1)], -1)
    table.copy_(torch.where((j >= have[:, None]) & (j < need[:, None]), page, table))
    # the tokens' positions and slots
    t = torch.arange(s["tokens"], device="cuda")
    request = torch.searchsorted(ends, t, right=True).clamp(max=b - 1)
    there = t < ends[-1]
    position = torch.where(there, cached[request] + t - starts[request], 0)
    page = table[request, (position // block).clamp(max=w - 1)].long()
    slot = torch.where(there & (page >= 0) & (page < s["blocks"]), page * block + position % block, -1)
    wanted = ends_of_pages[-1]
    i32 = lambda v: v.to(torch.int32)  # noqa: E731
    return [table, i32(lengths), i32(starts), i32(position), i32(slot), i32(torch.stack([wanted.clamp(max=len(free)), wanted]))]


def _exact_tables(case, seed):
    s = _prepare_tables(case, seed)
    cached, fresh, free, table = (s[k].cpu().numpy().astype(np.int64) for k in ("cached", "fresh", "free", "table"))
    block, budget, used = case["block"], case["tokens"], 0
    lengths, starts = [], [0]
    position, slot = np.zeros(budget, np.int64), np.full(budget, -1, np.int64)
    for b in range(case["requests"]):
        n = int(min(fresh[b], table.shape[1] * block - cached[b], budget - starts[-1]))
        have, need = -(-int(cached[b]) // block), -(-(int(cached[b]) + n) // block)
        for j in range(have, need):
            table[b, j] = free[used] if used < len(free) else -1
            used += 1
        p = cached[b] + np.arange(n)
        page = table[b, p // block]
        position[starts[-1]:starts[-1] + n] = p
        slot[starts[-1]:starts[-1] + n] = np.where((page >= 0) & (page < s["blocks"]), page * block + p % block, -1)
        lengths.append(int(cached[b]) + n)
        starts.append(starts[-1] + n)
    return [v.astype(np.int32) for v in (table, np.array(lengths), np.array(starts), position, slot, np.array([min(used, len(free)), used]))]


def _work_tables(case):
    b, t = case["requests"], case["tokens"]
    return {"bytes": 4 * (2 * b + 2 * b + 1 + 2 * t + 2 * (t // case["block"]) + b + 2), "flops": 0}


# ---------------------------------------------------------------------------------------------------- rotary positions

def _frequencies(case):
    """Radians a position for every pair; long waves are stretched by `factor`, short ones kept, those in between blended."""
    f = 10000.0 ** (-np.arange(0, case["rot"], 2, dtype=np.float64) / case["rot"])
    if case["factor"] == 1.0:
        return f
    smooth = np.clip((8192 * f / (2 * math.pi) - 1.0) / (4.0 - 1.0), 0.0, 1.0)
    return (1 - smooth) * f / case["factor"] + smooth * f


def _prepare_rotary(case, seed):
    g, dt = _generator(seed), DT[case["dtype"]]
    t, hq, hk, d = case["tokens"], case["q_heads"], case["k_heads"], case["dim"]
    random_ = lambda *n: torch.randn(n, device="cuda", generator=g).to(dt)  # noqa: E731
    s = {"op": "rotary", "case": case, "frequencies": torch.from_numpy(_frequencies(case)).cuda(), "magnitude": 1.0 + 0.1 * math.log(case["factor"]),
         "positions": torch.randint(0, case["far"], (t,), device="cuda", generator=g, dtype=torch.int32)}
    if case["store"]:
        # queries, keys and values as one projection leaves them
        qkv = random_(t, (hq + 2 * hk) * d)
        s["q"], s["k"], s["v"] = (x.unflatten(1, (-1, d)) for x in qkv.split([hq * d, hk * d, hk * d], 1))
        blocks = -(-t // case["block"]) + 3
        s["slots"] = torch.randperm(blocks * case["block"], device="cuda", generator=g)[:t].to(torch.int32)
        s["k_cache"] = torch.zeros((blocks, hk, case["block"], d), dtype=dt, device="cuda")
        s["v_cache"] = torch.zeros_like(s["k_cache"])
    else:
        s["q"], s["k"] = random_(t, hq, d), random_(t, hk, d)
    if own:
        from paper_1911_11576_amd import Plan
        args = dict(dtype=case["dtype"], tokens=t, q_heads=hq, k_heads=hk, head_dim=d, rotary_dim=case["rot"], interleaved=case["layout"] == "interleaved",
                    inverse=case["inverse"], magnitude=s["magnitude"])
        q_out = torch.empty((t, hq, d), dtype=dt, device="cuda")
        if case["store"]:
            stride = (hq + 2 * hk) * d
            s["plan"] = Plan.rotary(**args, q_stride=stride, k_stride=stride, v_stride=stride, blocks=blocks, block_size=case["block"])
            s["inputs"] = [s["q"], s["k"], s["v"], s["positions"], s["frequencies"], s["slots"]]
            s["outputs"] = [q_out, s["k_cache"], s["v_cache"]]
        else:
            s["plan"] = Plan.rotary(**args)
            s["inputs"] = [s["q"], s["k"], s["positions"], s["frequencies"]]
            s["outputs"] = [q_out, torch.empty((t, hk, d), dtype=dt, device="cuda")]
    return s


def _rotate(x, cos, sin, rot, interleaved):
    """x[T, H, D] in 32 bits, cos and sin [T, 1, rot / 2]: pairs of neighbours, or of one from each half, turned; the rest as it is."""
    head, rest = x[..., :rot], x[..., rot:]
    a, b = (head[..., 0::2], head[..., 1::2]) if interleaved else (head[..., :rot // 2], head[..., rot // 2:])
    y0, y1 = a * cos - b * sin, b * cos + a * sin
    turned = torch.stack([y0, y1], -1).flatten(-2) if interleaved else torch.cat([y0, y1], -1)
    return torch.cat([turned, rest], -1)


def _run_rotary(s):
    if own:
        s["plan"].launch(s["inputs"], s["outputs"])
        return s["outputs"]
    case = s["case"]
    angle = s["positions"].double()[:, None] * s["frequencies"]
    cos, sin = (s["magnitude"] * angle.cos()).float()[:, None], (s["magnitude"] * angle.sin()).float()[:, None]
    if case["inverse"]:
        sin = -sin
    dt, inter = s["q"].dtype, case["layout"] == "interleaved"
    q = _rotate(s["q"].float(), cos, sin, case["rot"], inter).to(dt)
    k = _rotate(s["k"].float(), cos, sin, case["rot"], inter).to(dt)
    if not case["store"]:
        return [q, k]
    page, at = s["slots"].long() // case["block"], s["slots"].long() % case["block"]
    s["k_cache"][page, :, at] = k
    s["v_cache"][page, :, at] = s["v"]
    return [q, s["k_cache"], s["v_cache"]]


def _exact_rotary(case, seed):
    s = _prepare_rotary(case, seed)
    n = case["rot"] // 2
    turn = torch.polar(torch.full((), s["magnitude"], dtype=torch.float64, device="cuda"),
                       (s["positions"].double().outer(s["frequencies"]) * (-1 if case["inverse"] else 1)))

    def rotated(x):
        y = x.double().clone()
        at = (slice(0, 2 * n, 2), slice(1, 2 * n, 2)) if case["layout"] == "interleaved" else (slice(0, n), slice(n, 2 * n))
        z = torch.complex(y[..., at[0]].contiguous(), y[..., at[1]].contiguous()) * turn[:, None]
        y[..., at[0]], y[..., at[1]] = z.real, z.imag
        return y

    if not case["store"]:
        return [rotated(s["q"]), rotated(s["k"])]
    caches = []
    for x in (rotated(s["k"]), s["v"].double()):
        rows = torch.zeros((s["k_cache"].shape[0] * case["block"], *x.shape[1:]), dtype=torch.float64, device="cuda")
        rows[s["slots"].long()] = x
        caches.append(rows.unflatten(0, (-1, case["block"])).transpose(1, 2))
    return [rotated(s["q"]), *caches]


def _work_rotary(case):
    t, d, e = case["tokens"], case["dim"], SIZE[case["dtype"]]
    heads = case["q_heads"] + case["k_heads"] * (2 if case["store"] else 1)
    return {"bytes": 2 * t * heads * d * e + t * (8 if case["store"] else 4) + 4 * case["rot"], "flops": 3 * t * (case["q_heads"] + case["k_heads"]) * case["rot"]}


# ---------------------------------------------------------------------------------------------------- attention over the cache

def _lengths(case):
    """Keys and new tokens of every request, the same whatever the seed, so that a pass has the work that work() says."""
    r = random.Random(case["pattern"])
    keys, new = [], []
    for i in range(case["requests"]):
        if case["spread"] == "even" or i == 0:
            keys.append(case["context"])
            new.append(case["new"])
            continue
        n = case["new"] if case["new"] == 1 else r.choice((1, case["new"], r.randint(1, case["new"])))
        keys.append(max(n, int(round(math.exp(r.uniform(math.log(max(1, case["context"] / 30)), math.log(case["context"])))))))
        new.append(n)
    return keys, new


def _prepare_attention(case, seed):
    g, dt = _generator(seed), DT[case["dtype"]]
    keys, new = _lengths(case)
    block, hk, d = case["block"], case["kv_heads"], case["dim"]
    held = [-(-n // block) for n in keys]
    width, blocks, t = max(held) + 2, sum(held) + 5, sum(new)
    pages = torch.randperm(blocks, generator=torch.Generator().manual_seed(seed)).numpy()
    table, at = np.full((len(keys), width), -1, np.int32), 0
    for b, n in enumerate(held):
        table[b, :n] = pages[at:at + n]
        at += n
    shape = (blocks, hk, block, d) if case["order"] == "head" else (blocks, block, hk, d)
    s = {"op": "attention", "case": case, "longest": max(keys), "most": max(new), "scale": d ** -0.5,
         "q": torch.randn((t, case["q_heads"], d), device="cuda", generator=g, dtype=dt),
         "k_cache": torch.randn(shape, device="cuda", generator=g, dtype=dt), "v_cache": torch.randn(shape, device="cuda", generator=g, dtype=dt),
         "table": _int32(table), "lengths": _int32(keys), "starts": _int32(np.concatenate([[0], np.cumsum(new)]))}
    if own:
        from paper_1911_11576_amd import Plan
        strides = {} if case["order"] == "head" else dict(block_stride=block * hk * d, head_stride=d, slot_stride=hk * d)
        s["plan"], nbytes = Plan.paged_attention(dtype=case["dtype"], requests=len(keys), tokens=t, q_heads=case["q_heads"], kv_heads=hk, head_dim=d, blocks=blocks,
                                                 block_size=block, table_blocks=width, scale=s["scale"], window=case["window"], max_new=max(new), lse=case["lse"], **strides)
        s["inputs"] = [s[k] for k in ("q", "k_cache", "v_cache", "table", "lengths", "starts")]
        s["outputs"] = [torch.empty_like(s["q"])] + ([torch.empty((t, case["q_heads"]), device="cuda")] if case["lse"] else [])
        s["partials"] = [torch.empty(nbytes, dtype=torch.uint8, device="cuda")] if nbytes else []
    return s


def _run_attention(s):
    if own:
        s["plan"].launch(s["inputs"], s["outputs"] + s["partials"])
        return s["outputs"]
    case, q, starts, lengths = s["case"], s["q"], s["starts"].long(), s["lengths"].long()
    t, hq, d = q.shape
    hk, block = case["kv_heads"], case["block"]
    share, b, most = hq // hk, len(lengths), s["most"]
    # every request's queries, padded to the most new tokens: [B, kv head, token x share, D]
    i = torch.arange(most, device="cuda")
    new = starts[1:] - starts[:-1]
    rows = torch.where(i < new[:, None], starts[:-1, None] + i, t)
    queries = q[rows.clamp(max=t - 1)].float().unflatten(2, (hk, share)).permute(0, 2, 1, 3, 4).flatten(2, 3)
    # its keys and values, padded to the longest: [B, kv head, key, D]; pages that a row has not are any page, masked below
    pages = s["table"][:, :-(-s["longest"] // block)].long().clamp(min=0)

    def gathered(cache):
        x = cache[pages]                                                     # [B, pages, kv head, slot, D], or slot and kv head changed about
        x = x.transpose(1, 2) if case["order"] == "head" else x.permute(0, 3, 1, 2, 4)
        return x.flatten(2, 3).float()

    j = torch.arange(pages.shape[1] * block, device="cuda")
    position = lengths[:, None] - new[:, None] + i                           # [B, token]
    seen = (j <= position[..., None]) & (j < lengths[:, None, None])
    if case["window"]:
        seen &= j > position[..., None] - case["window"]
    seen = seen.repeat_interleave(share, 1)[:, None]                         # [B, 1, token x share, key]
    scores = torch.matmul(queries * s["scale"], gathered(s["k_cache"]).transpose(2, 3))
    scores = scores.masked_fill_(~seen, -math.inf)
    top = scores.amax(-1, keepdim=True).clamp(min=-3e38)
    scores = scores.sub_(top).exp_()
    total = scores.sum(-1, keepdim=True)
    out = torch.matmul(scores, gathered(s["v_cache"])) / total.clamp(min=1e-38)
    tokens = lambda v: v.unflatten(2, (most, share)).permute(0, 2, 1, 3, *range(4, v.dim() + 1)).flatten(2, 3).flatten(0, 1)  # noqa: E731
    result = [torch.zeros((t + 1, hq, d), device="cuda").index_copy_(0, rows.flatten(), tokens(out))[:t].to(q.dtype)]
    if case["lse"]:
        lse = (top + total.log()).squeeze(-1)
        result.append(torch.zeros((t + 1, hq), device="cuda").index_copy_(0, rows.flatten(), tokens(lse))[:t])
    return result


def _exact_attention(case, seed):
    keys, new = _lengths(case)
    if 4 * case["dim"] * case["q_heads"] * sum(n * k for n, k in zip(new, keys)) > 2e12:
        return None
    s = _prepare_attention(case, seed)
    share, window = case["q_heads"] // case["kv_heads"], case["window"]
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
    lse = torch.zeros(s["q"].shape[:2], dtype=torch.float64, device="cuda")
    first = 0
    for b, (n, m) in enumerate(zip(keys, new)):
        page = s["table"][b, :-(-n // case["block"])].long()
        k, v = (s[c][page].transpose(1, 2) if case["order"] == "head" else s[c][page] for c in ("k_cache", "v_cache"))     # [pages, slot, head, D]
        at = torch.arange(n, device="cuda")
        for h in range(case["q_heads"]):
            kh, vh = (x[:, :, h // share].reshape(-1, case["dim"])[:n].double() for x in (k, v))
            z = s["scale"] * (s["q"][first:first + m, h].double() @ kh.T)
            mine = torch.arange(n - m, n, device="cuda")[:, None]
            z[(at > mine) | ((at <= mine - window) if window else False)] = -math.inf
            lse[first:first + m, h] = torch.logsumexp(z, 1)
            out[first:first + m, h] = torch.softmax(z, 1) @ vh
        first += m
    return [out, lse] if case["lse"] else [out]


def _work_attention(case):
    keys, new = _lengths(case)
    e, d, w = SIZE[case["dtype"]], case["dim"], case["window"]
    seen = lambda n, m: sum(min(p + 1, w or p + 1) for p in range(n - m, n))  # noqa: E731
    pairs = sum(seen(n, m) for n, m in zip(keys, new))
    read = sum(min(n, w + m - 1) if w else n for n, m in zip(keys, new))
    nbytes = 2 * sum(new) * case["q_heads"] * d * e + 2 * read * case["kv_heads"] * d * e + 4 * read // case["block"]
    return {"bytes": nbytes + (4 * sum(new) * case["q_heads"] if case["lse"] else 0), "flops": 4 * pairs * case["q_heads"] * d}
