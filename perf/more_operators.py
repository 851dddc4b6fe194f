"""The operators of a paged cache held in 8 bits, a scale for each block of tokens and head: what they are timed and checked on.

  store       new keys and values quantised as they are written, fp16 / bf16 into e4m3 or int8 codes: single tokens behind tokens that
              are there (their block's scale may grow) and chunks of up to 65536 tokens, as parts of a projection
  read        a request's tokens as numbers again, 1 .. 65536 tokens
  attention   new tokens over such a cache, fp16 / bf16, head dim 32 / 64 / 96 / 128, 1 to 16 query heads to a key head: one token a
              request over 1 .. 131072 keys, a few tokens a request, chunks of thousands of tokens

A code c of block b and head h stands for c * scales[b, h].  `own` false: the operators in elementary torch operations.  True: the
calls of this library.  What both are given is the same.
"""
import math
import random

import numpy as np
import torch

own = False

DT = {"f16": torch.float16, "bf16": torch.bfloat16}
CODE = {"e4m3": torch.float8_e4m3fn, "int8": torch.int8}
LARGEST = {"e4m3": 448.0, "int8": 127.0}


def listed():
    return [
        # a decode step of a server's batch: a token a request, mostly into a block that others are in; nothing but latency
        {"name": "store_decode", "op": "store", "dtype": "bf16", "code": "e4m3", "requests": 48, "new": 1, "context": 6000, "heads": 8, "dim": 128, "block": 16,
         "order": "head", "packed": 32, "pattern": 11},
        # chunks of prompts of several requests, keys and values as one projection leaves them
        {"name": "store_chunk", "op": "store", "dtype": "bf16", "code": "e4m3", "requests": 9, "new": 2048, "context": 9000, "heads": 8, "dim": 128, "block": 16,
         "order": "head", "packed": 32, "pattern": 12},
        # whole prompts into large blocks, a key head for every query head, heads of a token side by side
        {"name": "store_prompt_int8", "op": "store", "dtype": "f16", "code": "int8", "requests": 5, "new": 8000, "context": 8000, "heads": 16, "dim": 64, "block": 64,
         "order": "token", "packed": 0, "pattern": 13},
        # one short prefix read back
        {"name": "read_short", "op": "read", "dtype": "f16", "code": "int8", "requests": 1, "new": 77, "context": 500, "heads": 4, "dim": 96, "block": 32, "order": "head",
         "pattern": 14},
        # the prefixes of a batch read back, to move them or to attend over them elsewhere
        {"name": "read_prefixes", "op": "read", "dtype": "bf16", "code": "e4m3", "requests": 24, "new": 9000, "context": 9000, "heads": 8, "dim": 128, "block": 16,
         "order": "head", "pattern": 15},
        # a decode step of a few short requests: latency
        {"name": "attention8_decode_small", "op": "attention", "dtype": "f16", "code": "int8", "requests": 5, "new": 1, "context": 700, "spread": "ragged", "q_heads": 8,
         "heads": 2, "dim": 64, "block": 16, "order": "head", "window": 0, "lse": False, "pattern": 16},
        # a decode step of a server's batch, requests of very different lengths
        {"name": "attention8_decode_batch", "op": "attention", "dtype": "bf16", "code": "e4m3", "requests": 80, "new": 1, "context": 30000, "spread": "ragged", "q_heads": 32,
         "heads": 8, "dim": 128, "block": 16, "order": "head", "window": 0, "lse": False, "pattern": 17},
        # one long document in whole numbers, heads of a token side by side
        {"name": "attention8_decode_long", "op": "attention", "dtype": "bf16", "code": "int8", "requests": 1, "new": 1, "context": 131072, "spread": "even", "q_heads": 32,
         "heads": 8, "dim": 128, "block": 64, "order": "token", "window": 0, "lse": False, "pattern": 18},
        # a few guessed tokens a request, checked in one go, with a sliding window and the log-sum-exp
        {"name": "attention8_few_window", "op": "attention", "dtype": "f16", "code": "e4m3", "requests": 41, "new": 4, "context": 12000, "spread": "ragged", "q_heads": 24,
         "heads": 4, "dim": 96, "block": 32, "order": "token", "window": 5000, "lse": True, "pattern": 19},
        # prompts in chunks, and single tokens among them, behind long contexts
        {"name": "attention8_chunk", "op": "attention", "dtype": "bf16", "code": "e4m3", "requests": 7, "new": 1200, "context": 10000, "spread": "ragged", "q_heads": 32,
         "heads": 8, "dim": 128, "block": 16, "order": "head", "window": 0, "lse": False, "pattern": 20},
        # whole prompts without a context before them, a key head for every query head
        {"name": "attention8_prompt", "op": "attention", "dtype": "f16", "code": "int8", "requests": 3, "new": 2500, "context": 2500, "spread": "even", "q_heads": 16,
         "heads": 16, "dim": 64, "block": 64, "order": "head", "window": 0, "lse": True, "pattern": 21},
    ]


def _log(rng, lo, hi):
    """A whole number between lo and hi, spread over the logarithm; half of them odd."""
    n = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
    return max(lo, min(hi, n | 1 if rng.random() < 0.5 else n))


def draw(rng):
    op = rng.choice(("store", "read", "attention", "attention"))
    dtype, code, order = rng.choice(("bf16", "f16")), rng.choice(("e4m3", "int8")), rng.choice(("head", "token"))
    block, pattern = rng.choice((16, 32, 64, 128)), rng.randrange(1 << 20)
    if op in ("store", "read"):
        heads, dim = rng.choice((1, 2, 3, 4, 8, 16)), rng.choice((32, 64, 80, 96, 128, 256))
        requests = _log(rng, 1, 256)
        most = max(2, (65536 * 8 * 128) // (requests * heads * dim))      # tokens of a request
        new = 1 if op == "store" and rng.random() < 0.4 else _log(rng, 1, min(65536, most))
        case = {"op": op, "dtype": dtype, "code": code, "requests": requests, "new": new, "context": new + rng.choice((0, _log(rng, 1, max(2, min(32768, most))))),
                "heads": heads, "dim": dim, "block": block, "order": order, "pattern": pattern}
        return dict(case, packed=rng.choice((0, heads, 4 * heads))) if op == "store" else case
    kind = rng.choice(("one", "few", "chunk"))
    heads = rng.choice((1, 2, 4, 8, 16) if kind != "chunk" else (1, 2, 4, 8))
    share = rng.choice((1, 2, 3, 4, 8, 16) if kind != "chunk" else (1, 2, 4, 8))
    dim = rng.choice((32, 64, 96, 128, 128))
    requests = _log(rng, 1, 128 if kind != "chunk" else 8)
    new = 1 if kind == "one" else _log(rng, 2, 8) if kind == "few" else _log(rng, 32, 2048)
    # keys in all: no more than the largest listed case of the kind has
    most = (64 * 24000 * 8 * 128) // (requests * heads * dim)
    if kind != "one":
        most = min(most, (7 * 1200 * 10000 * 32) // (requests * heads * share * new))
    context = _log(rng, 1, max(2, min(131072 if kind == "one" else 32768, most)))
    return {"op": op, "dtype": dtype, "code": code, "requests": requests, "new": new, "context": max(context, new), "spread": rng.choice(("ragged", "even")),
            "q_heads": heads * share, "heads": heads, "dim": dim, "block": block, "order": order, "window": rng.choice((0, 0, 0, 128, 1000, 4096)), "lse": rng.random() < 0.5,
            "pattern": pattern}


def prepare(case, seed):
    return {"store": _prepare_store, "read": _prepare_read, "attention": _prepare_attention}[case["op"]](case, seed)


def run(state):
    return {"store": _run_store, "read": _run_read, "attention": _run_attention}[state["case"]["op"]](state)


def exact(case, seed):
    return {"store": _exact_store, "read": _exact_read, "attention": _exact_attention}[case["op"]](case, seed)


def work(case):
    return {"store": _work_store, "read": _work_read, "attention": _work_attention}[case["op"]](case)


def _int32(a):
    return torch.from_numpy(np.ascontiguousarray(a, dtype=np.int32)).cuda()


def _lengths(case):
    """Tokens of every request and new ones among them, the same whatever the seed, so that a pass has the work that work() says."""
    r = random.Random(case["pattern"])
    keys, new = [], []
    for i in range(case["requests"]):
        if case.get("spread") == "even" or i == 0:
            keys.append(case["context"])
            new.append(case["new"])
            continue
        n = case["new"] if case["new"] == 1 else r.choice((1, case["new"], r.randint(1, case["new"])))
        keys.append(max(n, int(round(math.exp(r.uniform(math.log(max(1, case["context"] / 30)), math.log(case["context"])))))))
        new.append(n)
    return keys, new


def _cache(case, seed):
    """A cache in use: its requests' tables, and codes and scales as earlier steps have left them, blocks and heads of different ranges."""
    g = torch.Generator("cuda")
    g.manual_seed(seed)
    keys, new = _lengths(case)
    block, heads, dim = case["block"], case["heads"], case["dim"]
    held = [-(-n // block) for n in keys]
    width, blocks = max(held) + 2, sum(held) + 5
    pages = torch.randperm(blocks, generator=torch.Generator().manual_seed(seed)).numpy()
    table, at = np.full((len(keys), width), -1, np.int32), 0
    for b, n in enumerate(held):
        table[b, :n] = pages[at:at + n]
        at += n
    shape = (blocks, heads, block, dim) if case["order"] == "head" else (blocks, block, heads, dim)
    spread, base = (64.0, 2.0 ** -6) if case["code"] == "e4m3" else (32.0, 2.0 ** -5)

    def codes():
        x = torch.randn(shape, device="cuda", generator=g, dtype=torch.bfloat16).mul_(spread)
        return x.to(CODE["e4m3"]) if case["code"] == "e4m3" else x.round_().clamp_(-127, 127).to(torch.int8)

    def scales():
        return base * torch.exp2(torch.randint(-1, 2, (blocks, heads), device="cuda", generator=g).float())

    s = {"case": case, "k_cache": codes(), "v_cache": codes(), "k_scales": scales(), "v_scales": scales(), "table": _int32(table), "lengths": _int32(keys),
         "starts": _int32(np.concatenate([[0], np.cumsum(new)])), "longest": max(keys), "most": max(new)}
    strides = {} if case["order"] == "head" else dict(block_stride=block * heads * dim, head_stride=dim, slot_stride=heads * dim)
    args = dict(dtype=case["dtype"], code=case["code"], requests=len(keys), tokens=sum(new), kv_heads=heads, head_dim=dim, blocks=blocks, block_size=block, table_blocks=width,
                **strides)
    return s, g, args


def _places(s):
    """Of every new token its block, its place there and its position; and the requests that they belong to."""
    starts, lengths, block = s["starts"].long(), s["lengths"].long(), s["case"]["block"]
    t = torch.arange(s["tokens"], device="cuda")
    request = torch.searchsorted(starts[1:].contiguous(), t, right=True)
    position = lengths[request] - starts[request + 1] + t
    return s["table"].long()[request, position // block], position % block, position, request


def _rows(cache, order):
    """The cache as [block, place, head, D], bytes: indexing knows no type of 8 bits but those of whole numbers."""
    return (cache.transpose(1, 2) if order == "head" else cache).view(torch.uint8)


# ---------------------------------------------------------------------------------------------------- store

def _prepare_store(case, seed):
    s, g, args = _cache(case, seed)
    t, heads, dim = args["tokens"], case["heads"], case["dim"]
    s["tokens"] = t
    # with `packed` query heads before them in a row of one projection; a request's tokens have a range of their own
    row = (case["packed"] + 2 * heads) * dim
    far = torch.exp2(2 * torch.rand((t, 1), device="cuda", generator=g) - 1)
    qkv = (torch.randn((t, row), device="cuda", generator=g) * far).to(DT[case["dtype"]])
    s["k"], s["v"] = (x.unflatten(1, (heads, dim)) for x in qkv[:, case["packed"] * dim:].split([heads * dim] * 2, 1))
    if own:
        from paper_1911_11576_amd import Plan
        s["plan"] = Plan.cache_store8(**args, k_stride=row, v_stride=row)
        s["inputs"] = [s[x] for x in ("k", "v", "table", "lengths", "starts")]
        s["outputs"] = [s[x] for x in ("k_cache", "v_cache", "k_scales", "v_scales")]
    return s


def _run_store(s):
    """-> codes of keys and of values, which stand for multiples of the scales that come with them."""
    if own:
        s["plan"].launch(s["inputs"], s["outputs"])
        return s["outputs"]
    case = s["case"]
    order, int8, block = case["order"], case["code"] == "int8", case["block"]
    page, place, position, request = _places(s)
    # blocks that hold tokens from before: a request's first new token is not the first of its block
    starts, lengths = s["starts"].long(), s["lengths"].long()
    first = lengths - starts[1:] + starts[:-1]
    begun = (first % block > 0) & (starts[1:] > starts[:-1])
    begun_page = s["table"].long().gather(1, (first // block)[:, None].clamp(max=s["table"].shape[1] - 1))[:, 0]
    old = torch.arange(block, device="cuda") < torch.where(begun, first % block, 0)[:, None]      # [B, place]
    for name in ("k", "v"):
        x, cache, scales, code = s[name].float(), _rows(s[name + "_cache"], order), s[name + "_scales"], CODE[case["code"]]
        # the least power of two whose largest code reaches the largest of a block's new values; no less than what its old ones have
        top = torch.zeros_like(scales).index_reduce_(0, page, x.abs().amax(-1), "amax")
        part, exponent = torch.frexp(top)
        exponent = exponent - (7 if int8 else 9) + (part > (127 / 128 if int8 else 0.875))
        need = torch.exp2(exponent.clamp(min=-126).float())
        touched = torch.zeros(len(scales), dtype=torch.bool, device="cuda").index_fill_(0, page, True)[:, None]
        kept = torch.zeros(len(scales), dtype=torch.bool, device="cuda").index_put_((begun_page,), begun)[:, None]
        now = torch.where(touched, torch.where(kept, torch.maximum(scales, need), need), scales)
        # the old codes of those blocks in their new scales
        ratio = (scales / now)[begun_page][:, None, :, None]
        codes = cache[begun_page]
        again = codes.view(code).float() * ratio
        again = (again.round() if int8 else again).to(code).view(torch.uint8)
        cache[begun_page] = torch.where(old[:, :, None, None], again, codes)
        # the new ones
        y = x / now[page][..., None]
        cache[page, place] = (y.round() if int8 else y).to(code).view(torch.uint8)
        scales.copy_(now)
    return [s[n] for n in ("k_cache", "v_cache", "k_scales", "v_scales")]


def _exact_store(case, seed):
    s = _prepare_store(case, seed)
    keys, new = _lengths(case)
    block, most = case["block"], LARGEST[case["code"]]

    def coded(y):
        if case["code"] == "int8":
            return y.round()
        step = torch.exp2(torch.frexp(y.abs()).exponent.clamp(min=-5).double() - 4)      # three bits behind the first one, down to 2^-9
        return (y / step).round() * step

    result = []
    for name in ("k", "v"):
        cache, scales = s[name + "_cache"].float().double(), s[name + "_scales"].double()
        cache = cache.transpose(1, 2) if case["order"] == "head" else cache
        at = 0
        for b, (n, m) in enumerate(zip(keys, new)):
            x, p = s[name][at:at + m].double(), n - m
            at += m
            while len(x):
                page, lo = int(s["table"][b, p // block]), p % block
                hi = min(block, lo + len(x))
                here, x, p = x[:hi - lo], x[hi - lo:], p + hi - lo
                part, power = torch.frexp((here.abs().amax((0, 2)) / most).clamp(min=2.0 ** -126))
                scale = torch.ldexp(torch.ones_like(part), power - (part == 0.5).int())
                if lo:
                    before = scales[page]
                    scale = torch.maximum(scale, before)
                    cache[page, :lo] = coded(cache[page, :lo] * (before / scale)[:, None])
                cache[page, lo:hi] = coded(here / scale[:, None])
                scales[page] = scale
        result.append((cache.transpose(1, 2) if case["order"] == "head" else cache, scales))
    return [result[0][0], result[1][0], result[0][1], result[1][1]]


def _work_store(case):
    keys, new = _lengths(case)
    pages = sum(-(-n // case["block"]) - (n - m) // case["block"] for n, m in zip(keys, new))
    t, row = sum(new), case["heads"] * case["dim"]
    return {"bytes": 2 * t * row * 2 + 2 * t * row + 2 * pages * case["heads"] * 4 + 4 * (pages + 2 * len(keys) + 1), "flops": 4 * t * row}


# ---------------------------------------------------------------------------------------------------- read

def _prepare_read(case, seed):
    s, _, args = _cache(case, seed)
    s["tokens"] = args["tokens"]
    if own:
        from paper_1911_11576_amd import Plan
        s["plan"] = Plan.cache_read8(**args)
        s["inputs"] = [s[x] for x in ("k_cache", "v_cache", "k_scales", "v_scales", "table", "lengths", "starts")]
        s["outputs"] = [torch.empty((s["tokens"], case["heads"], case["dim"]), dtype=DT[case["dtype"]], device="cuda") for _ in range(2)]
    return s


def _run_read(s):
    if own:
        s["plan"].launch(s["inputs"], s["outputs"])
        return s["outputs"]
    case = s["case"]
    page, place, _, _ = _places(s)
    return [(_rows(s[n + "_cache"], case["order"])[page, place].view(CODE[case["code"]]).float() * s[n + "_scales"][page][..., None]).to(DT[case["dtype"]]) for n in ("k", "v")]


def _exact_read(case, seed):
    s = _prepare_read(case, seed)
    keys, new = _lengths(case)
    result = []
    for name in ("k", "v"):
        parts = []
        for b, (n, m) in enumerate(zip(keys, new)):
            page = s["table"][b, :-(-n // case["block"])].long()
            x = s[name + "_cache"].view(torch.uint8)[page].view(CODE[case["code"]]).float().double()
            x = (x.transpose(1, 2) if case["order"] == "head" else x) * s[name + "_scales"][page].double()[:, None, :, None]
            parts.append(x.flatten(0, 1)[n - m:n])
        result.append(torch.cat(parts))
    return result


def _work_read(case):
    keys, new = _lengths(case)
    pages = sum(-(-n // case["block"]) - (n - m) // case["block"] for n, m in zip(keys, new))
    t, row = sum(new), case["heads"] * case["dim"]
    return {"bytes": 2 * t * row + 2 * t * row * 2 + 2 * pages * case["heads"] * 4 + 4 * (pages + 2 * len(keys) + 1), "flops": 2 * t * row}


# ---------------------------------------------------------------------------------------------------- attention

def _prepare_attention(case, seed):
    s, g, args = _cache(case, seed)
    t = args["tokens"]
    s["scale"] = case["dim"] ** -0.5
    s["q"] = torch.randn((t, case["q_heads"], case["dim"]), device="cuda", generator=g, dtype=DT[case["dtype"]])
    if own:
        from paper_1911_11576_amd import Plan
        s["plan"], nbytes = Plan.paged_attention8(**args, q_heads=case["q_heads"], scale=s["scale"], window=case["window"], max_new=s["most"], lse=case["lse"])
        s["inputs"] = [s[x] for x in ("q", "k_cache", "v_cache", "k_scales", "v_scales", "table", "lengths", "starts")]
        s["outputs"] = [torch.empty_like(s["q"])] + ([torch.empty((t, case["q_heads"]), device="cuda")] if case["lse"] else [])
        s["partials"] = [torch.empty(nbytes, dtype=torch.uint8, device="cuda")] if nbytes else []
    return s


def _run_attention(s):
    if own:
        s["plan"].launch(s["inputs"], s["outputs"] + s["partials"])
        return s["outputs"]
    case, q, starts, lengths = s["case"], s["q"], s["starts"].long(), s["lengths"].long()
    t, hq, d = q.shape
    heads, block = case["heads"], case["block"]
    share, most = hq // heads, s["most"]
    # every request's queries, padded to the most new tokens: [B, key head, token x share, D]
    i = torch.arange(most, device="cuda")
    new = starts[1:] - starts[:-1]
    rows = torch.where(i < new[:, None], starts[:-1, None] + i, t)
    queries = q[rows.clamp(max=t - 1)].float().unflatten(2, (heads, share)).permute(0, 2, 1, 3, 4).flatten(2, 3)
    # its keys and values, padded to the longest: [B, key head, key, D]; pages that a row has not are any page, masked below
    pages = s["table"][:, :-(-s["longest"] // block)].long().clamp(min=0)

    def gathered(name):
        x = s[name + "_cache"].view(torch.uint8)[pages].view(CODE[case["code"]]).float()      # [B, pages, head, place, D], or place and head changed about
        x = x.transpose(1, 2) if case["order"] == "head" else x.permute(0, 3, 1, 2, 4)
        return (x * s[name + "_scales"][pages].transpose(1, 2)[..., None, None]).flatten(2, 3)

    j = torch.arange(pages.shape[1] * block, device="cuda")
    position = lengths[:, None] - new[:, None] + i                           # [B, token]
    seen = (j <= position[..., None]) & (j < lengths[:, None, None])
    if case["window"]:
        seen &= j > position[..., None] - case["window"]
    seen = seen.repeat_interleave(share, 1)[:, None]                         # [B, 1, token x share, key]
    scores = torch.matmul(queries * s["scale"], gathered("k").transpose(2, 3))
    scores = scores.masked_fill_(~seen, -math.inf)
    top = scores.amax(-1, keepdim=True).clamp(min=-3e38)
    scores = scores.sub_(top).exp_()
    total = scores.sum(-1, keepdim=True)
    out = torch.matmul(scores, gathered("v")) / total.clamp(min=1e-38)
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
    share, window = case["q_heads"] // case["heads"], case["window"]
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
    lse = torch.zeros(s["q"].shape[:2], dtype=torch.float64, device="cuda")
    first = 0
    for b, (n, m) in enumerate(zip(keys, new)):
        page = s["table"][b, :-(-n // case["block"])].long()
        mine = torch.arange(n - m, n, device="cuda")[:, None]
        at = torch.arange(n, device="cuda")
        hidden = at > mine
        if window:
            hidden |= at <= mine - window
        for h in range(case["heads"]):
            part = (slice(None), h) if case["order"] == "head" else (slice(None), slice(None), h)
            k, v = ((s[x + "_cache"].view(torch.uint8)[page][part].contiguous().view(CODE[case["code"]]).float().double() * s[x + "_scales"][page, h].double()[:, None, None]).reshape(-1, case["dim"])[:n] for x in ("k", "v"))
            for i in range(h * share, (h + 1) * share):
                z = (s["scale"] * (s["q"][first:first + m, i].double() @ k.T)).masked_fill_(hidden, -math.inf)
                lse[first:first + m, i] = torch.logsumexp(z, 1)
                out[first:first + m, i] = torch.softmax(z, 1) @ v
        first += m
    return [out, lse] if case["lse"] else [out]


def _work_attention(case):
    keys, new = _lengths(case)
    d, w = case["dim"], case["window"]
    seen = lambda n, m: sum(min(p + 1, w or p + 1) for p in range(n - m, n))  # noqa: E731
    pairs = sum(seen(n, m) for n, m in zip(keys, new))
    read = sum(min(n, w + m - 1) if w else n for n, m in zip(keys, new))
    nbytes = 2 * sum(new) * case["q_heads"] * d * 2 + 2 * read * case["heads"] * d + (4 + 8 * case["heads"]) * read // case["block"]
    return {"bytes": nbytes + (4 * sum(new) * case["q_heads"] if case["lse"] else 0), "flops": 4 * pairs * case["q_heads"] * d}
