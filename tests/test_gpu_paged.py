"""The operators around a paged cache on the GPU, against their definitions in 64 bits (oracle/paged.py).

Tolerances.  u: half a step of the storage type, relative (fp32 2^-24).
  rotary     The angle is exact to 2^-26 turns of rounding to fp32, 2 pi times that, and its product with 2 pi (two more roundings of at most
             pi / 4): 1.5e-7 in all, or 2.5 steps of 2^-24; the polynomials' own roundings and remainders are two more, the magnitude one,
             the two products and their sum two: 8 * 2^-24 * magnitude * (|x0| + |x1|), and u |y| for the store (fp16: and 2^-25).
  attention  Products of 16-bit numbers are exact in fp32; a score's sum of D of them and its scaling err by at most (D + 4) 2^-24 sum |q k| scale, the exponent's
             argument by three roundings of a number up to 2 max |s| more, the exponential and the sums of weights by 2^-20: d in all, once
             in the numerator and once in the denominator; the weight itself is rounded to the type (u, and 2^-25 of the largest weight where fp16's
             numbers end), the result at the store:  (u + 2 d) sum w |v| + 2^-25 sum |v| / sum e + u |o| (fp16: + 2^-25).
             Log-sum-exp: d + 2^-22 |lse| + 2^-22.
"""
import numpy as np
import pytest
import torch

from oracle import paged
from paper_1911_11576_amd import Plan, fs_rotary_frequencies

pytestmark = pytest.mark.gpu

DT = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
U = {"f32": 2.0**-24, "f16": 2.0**-11, "bf16": 2.0**-8}


def i32(a):
    return torch.as_tensor(np.ascontiguousarray(a, dtype=np.int32), device="cuda")


def f64(t):
    return t.detach().double().cpu().numpy()


def within(got, want, bound, what):
    """|got - want| <= bound wherever want is a number; where it is none `got` is the same none."""
    got, want, bound = (np.broadcast_to(np.asarray(a, np.float64), np.shape(want)) for a in (got, want, bound))
    odd = ~np.isfinite(want)
    assert np.array_equal(got[odd], want[odd], equal_nan=True), f"{what}: infinities or NaN differ"
    err = np.abs(got[~odd] - want[~odd])
    bad = ~(err <= bound[~odd])
    assert not bad.any(), f"{what}: {bad.sum()} of {bad.size} outside, worst {np.nanmax(err / np.maximum(bound[~odd], 1e-300)):.3g} times the bound"


# ---------------------------------------------------------------------------------------------------- block tables

def run_tables(cached, fresh, free, tables, tokens, blocks, block_size, stream=None, static=False):
    b, w = np.asarray(tables).reshape(len(cached), -1).shape if len(cached) else (0, 3)
    t = i32(tables) if len(cached) else torch.zeros(0, dtype=torch.int32, device="cuda")
    outs = [t] + [torch.full((n,), -77, dtype=torch.int32, device="cuda") for n in (b, b + 1, tokens, tokens, 2)]
    with Plan.block_tables(b, tokens, blocks, block_size, w, len(free)) as plan:
        ins = [i32(cached), i32(fresh), i32(free)]
        (plan.launch_static if static else plan.launch)(ins, outs, stream)
        torch.cuda.synchronize()
    return [o.cpu().numpy() for o in outs]


def check_tables(cached, fresh, free, tables, tokens, blocks, block_size, **kw):
    want = paged.block_tables(cached, fresh, free, tables, tokens, blocks, block_size)
    got = run_tables(cached, fresh, free, tables, tokens, blocks, block_size, **kw)
    for name, g, w in zip(("tables", "lengths", "starts", "positions", "slots", "taken"), got, want):
        assert np.array_equal(g.reshape(-1), np.asarray(w).reshape(-1)), name


@pytest.mark.parametrize("requests, tokens, block_size, width, n_free", [
    (1, 1, 16, 4, 1), (1, 0, 16, 4, 3), (3, 1000, 1, 50, 60), (64, 64, 16, 9, 70), (65, 64, 16, 9, 10), (200, 1500, 32, 5, 1000), (257, 6000, 8, 33, 700),
    (1000, 999, 1024, 2, 40), (4096, 70000, 16, 17, 9000), (2, 5000, 64, 100, 100)])
@pytest.mark.parametrize("kind", ["one", "chunk", "odd"])
def test_tables(requests, tokens, block_size, width, n_free, kind):
    rng = np.random.default_rng(requests + tokens)
    most = width * block_size
    cached = rng.integers(0, most + 1, requests)
    fresh = np.ones(requests, int) if kind == "one" else rng.integers(0, max(2, 3 * tokens // requests), requests)
    if kind == "odd":      # idle requests, lengths below 0 and beyond the row, new tokens that pass 31 bits in all
        cached = np.where(rng.random(requests) < 0.2, rng.choice([-5, 0, most, most + 7, 2**31 - 1], requests), cached)
        fresh = np.where(rng.random(requests) < 0.2, rng.choice([-3, 0, 2**31 - 1], requests), fresh)
    blocks = width * requests + n_free
    pages = rng.permutation(blocks)
    tables = np.where(np.arange(width) < -(-np.clip(cached, 0, most) // block_size)[:, None], pages[:requests * width].reshape(requests, width), -1)
    free = pages[requests * width:]
    if kind == "odd":
        tables = np.where(rng.random(tables.shape) < 0.1, rng.choice([-9, blocks, 2**31 - 1], tables.shape), tables)
        blocks -= 1
    check_tables(cached, fresh, free, tables, tokens, blocks, block_size, static=kind == "odd")


def test_tables_without_requests_and_without_room():
    check_tables([], [], [1, 2], [], 5, 4, 16)
    check_tables([3, 0], [4, 5], [], [[], []], 6, 0, 16)
    check_tables([3, 0], [40, 5], [], [[1], [-1]], 60, 2, 16)


# ---------------------------------------------------------------------------------------------------- rotary positions

def rotary_bound(x, want, freqs, interleaved, magnitude, dtype):
    n = len(freqs)
    room = np.zeros_like(want)
    i0, i1 = (np.arange(0, 2 * n, 2), np.arange(1, 2 * n, 2)) if interleaved else (np.arange(n), np.arange(n, 2 * n))
    s = 8 * 2.0**-24 * magnitude * (np.abs(x[..., i0]) + np.abs(x[..., i1]))
    room[..., i0], room[..., i1] = s, s
    return room + U[dtype] * np.abs(want) + (2.0**-25 if dtype == "f16" else 0)


def positions_of(rng, t, far):
    p = rng.integers(0, far, t)
    p[: min(t, 3)] = [0, far - 1, 1][: min(t, 3)]
    return p


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("tokens, q_heads, k_heads, dim, rot, far", [
    (1, 1, 0, 2, 2, 10), (5, 3, 1, 6, 4, 1 << 20), (7, 2, 2, 10, 10, 100), (33, 32, 8, 128, 128, 1 << 20), (129, 5, 5, 80, 24, 4000), (17, 4, 1, 64, 32, 1 << 27), (300, 1, 1, 96, 96, 3),
    (3, 40, 8, 512, 510, 50), (9, 7, 3, 256, 64, 1 << 17), (1000, 2, 1, 20, 12, 999)])
def test_rotary(dtype, interleaved, tokens, q_heads, k_heads, dim, rot, far):
    rng = np.random.default_rng(dim + rot)
    g = torch.Generator("cuda").manual_seed(1)
    freqs = fs_rotary_frequencies(rot, 10000.0, 4.0, 1.0, 4.0, 8192.0)
    pos = positions_of(rng, tokens, far)
    heads = [q_heads] + ([k_heads] if k_heads else [])
    x = [torch.randn((tokens, h, dim), device="cuda", generator=g).to(DT[dtype]) for h in heads]
    frq, p = torch.tensor(freqs, dtype=torch.float64, device="cuda"), i32(pos)
    kw = dict(dtype=dtype, tokens=tokens, q_heads=q_heads, k_heads=k_heads, head_dim=dim, rotary_dim=rot, interleaved=interleaved)
    for inverse, magnitude in ((False, 1.0), (True, 1.25)):
        outs = [torch.full_like(t, float("nan")) for t in x]
        with Plan.rotary(**kw, inverse=inverse, magnitude=magnitude) as plan:
            plan.launch([*x, p, frq], outs)
            for t, o in zip(x, outs):
                want = paged.rotary(f64(t), pos, freqs, interleaved, inverse, magnitude)
                within(f64(o), want, rotary_bound(f64(t), want, freqs, interleaved, magnitude, dtype), "rotary")
            same = [t.clone() for t in x]      # in place
            plan.launch([*same, p, frq], same)
            assert all(torch.equal(a, b) for a, b in zip(same, outs))


@pytest.mark.parametrize("interleaved", [False, True])
def test_rotary_of_parts_of_a_projection(interleaved):
    t, hq, hk, d, row = 19, 6, 2, 32, 6 * 32 + 2 * 2 * 32 + 24
    g = torch.Generator("cuda").manual_seed(2)
    qkv = torch.randn((t, row), device="cuda", generator=g).to(torch.bfloat16)
    before = qkv.clone()
    q, k = qkv[:, : hq * d].unflatten(1, (hq, d)), qkv[:, hq * d: (hq + hk) * d].unflatten(1, (hk, d))
    pos, freqs = np.arange(t) * 37, fs_rotary_frequencies(d)
    want = [paged.rotary(f64(x), pos, freqs, interleaved) for x in (q, k)]
    room = [rotary_bound(f64(x), w, freqs, interleaved, 1.0, "bf16") for x, w in zip((q, k), want)]
    with Plan.rotary("bf16", t, hq, hk, d, interleaved=interleaved, q_stride=row, k_stride=row, q_out_stride=row, k_out_stride=row) as plan:
        plan.launch([q, k, i32(pos), torch.tensor(freqs, dtype=torch.float64, device="cuda")], [q, k])
    within(f64(q), want[0], room[0], "q in place")
    within(f64(k), want[1], room[1], "k in place")
    assert torch.equal(qkv[:, (hq + hk) * d:], before[:, (hq + hk) * d:])


@pytest.mark.parametrize("dtype", ["f16", "bf16", "f32"])
@pytest.mark.parametrize("tokens, q_heads, k_heads, dim, rot, block_size, order", [
    (1, 1, 1, 64, 64, 16, "head"), (70, 32, 8, 128, 128, 16, "token"), (33, 6, 2, 80, 24, 1, "head"), (257, 3, 3, 6, 2, 128, "token"), (12, 4, 4, 64, 32, 1024, "head")])
def test_rotary_store(dtype, tokens, q_heads, k_heads, dim, rot, block_size, order):
    rng = np.random.default_rng(tokens)
    g = torch.Generator("cuda").manual_seed(3)
    row = (q_heads + 2 * k_heads) * dim
    qkv = torch.randn((tokens, row), device="cuda", generator=g).to(DT[dtype])
    pad = 16 // qkv.element_size() - 1      # parts of a projection begin at 16 bytes
    if (q_heads * dim) % (pad + 1) or (k_heads * dim) % (pad + 1):
        parts = [qkv[:, a * dim:b * dim].contiguous() for a, b in ((0, q_heads), (q_heads, q_heads + k_heads), (q_heads + k_heads, q_heads + 2 * k_heads))]
        strides = {}
    else:
        parts, strides = qkv.split([q_heads * dim, k_heads * dim, k_heads * dim], 1), dict(q_stride=row, k_stride=row, v_stride=row)
    blocks = -(-tokens // block_size) + 2
    slots = rng.permutation(blocks * block_size)[:tokens]
    padding = rng.random(tokens) < 0.2
    slots[padding] = rng.choice([-1, -2**31, blocks * block_size, 2**31 - 1], padding.sum())
    freqs, pos = fs_rotary_frequencies(rot), positions_of(rng, tokens, 100000)
    shape = (blocks, k_heads, block_size, dim) if order == "head" else (blocks, block_size, k_heads, dim)
    caches = [torch.full(shape, 7.0, dtype=DT[dtype], device="cuda") for _ in range(2)]
    q_out = torch.full((tokens, q_heads, dim), 5.0, dtype=DT[dtype], device="cuda")
    if order == "token":
        strides |= dict(block_stride=block_size * k_heads * dim, head_stride=dim, slot_stride=k_heads * dim)
    with Plan.rotary(dtype, tokens, q_heads, k_heads, dim, rot, blocks=blocks, block_size=block_size, **strides) as plan:
        plan.launch([*parts, i32(pos), torch.tensor(freqs, dtype=torch.float64, device="cuda"), i32(slots)], [q_out, *caches])
    xq, xk, xv = (f64(x.reshape(tokens, -1, dim)) for x in parts)
    want = paged.rotary(xq, pos, freqs)
    room = rotary_bound(xq, want, freqs, False, 1.0, dtype)
    want[padding], room[padding] = 5.0, 0
    within(f64(q_out), want, room, "q")
    for cache, rows, x in ((caches[0], paged.rotary(xk, pos, freqs), xk), (caches[1], xv, None)):
        bound = rotary_bound(x, rows, freqs, False, 1.0, dtype) if x is not None else np.zeros_like(rows)
        cache = cache if order == "head" else cache.transpose(1, 2)
        empty = np.full((blocks, k_heads, block_size, dim), 7.0)
        within(f64(cache), paged.stored(empty, rows, slots), paged.stored(0 * empty, bound, slots), "cache")


@pytest.mark.parametrize("dtype, heads, dim, rot, interleaved, store", [
    ("f16", 72, 64, 32, False, True), ("bf16", 72, 64, 64, False, False), ("f16", 24, 128, 96, False, False), ("bf16", 36, 128, 128, False, True), ("bf16", 60, 96, 32, False, True),
    ("f16", 99, 32, 16, False, False), ("bf16", 48, 64, 32, True, True), ("f32", 45, 64, 48, True, False), ("f32", 21, 128, 64, False, True), ("bf16", 3, 256, 64, False, False),
    ("f16", 3, 512, 512, False, True)])
def test_rotary_of_many_rows(dtype, heads, dim, rot, interleaved, store):
    """Enough rows that threads have several heads: with angles of their own and of a workgroup's, one vector of a head and two, in place too."""
    width = 4 if dtype == "f32" else 8
    tokens = -(-4 * 131072 * 2 * width // (dim * heads)) + 1
    rng, g = np.random.default_rng(dim + heads), torch.Generator("cuda").manual_seed(heads)
    k_heads = heads // 3
    x = [torch.randn((tokens, h, dim), device="cuda", generator=g).to(DT[dtype]) for h in (heads - k_heads * (1 + store), *([k_heads] * (1 + store)))]
    freqs, pos = fs_rotary_frequencies(rot), positions_of(rng, tokens, 1 << 20)
    frq, p = torch.tensor(freqs, dtype=torch.float64, device="cuda"), i32(pos)
    kw = dict(interleaved=interleaved, inverse=not store, magnitude=1.25)
    want = [paged.rotary(f64(t), pos, freqs, interleaved, not store, 1.25) for t in x[:2]]
    room = [rotary_bound(f64(t), w, freqs, interleaved, 1.25, dtype) for t, w in zip(x, want)]
    if not store:
        with Plan.rotary(dtype, tokens, x[0].shape[1], k_heads, dim, rot, **kw) as plan:
            outs = [torch.full_like(t, float("nan")) for t in x]
            plan.launch([*x, p, frq], outs)
            for o, w, b in zip(outs, want, room):
                within(f64(o), w, b, "rotary")
            plan.launch([*x, p, frq], x)
            assert all(torch.equal(a, b) for a, b in zip(x, outs))
        return
    blocks = -(-tokens // 16) + 2
    slots = rng.permutation(blocks * 16)[:tokens]
    padding = rng.random(tokens) < 0.1
    slots[padding] = -1
    caches = [torch.full((blocks, k_heads, 16, dim), 7.0, dtype=DT[dtype], device="cuda") for _ in range(2)]
    q_out = torch.full_like(x[0], 5.0)
    with Plan.rotary(dtype, tokens, x[0].shape[1], k_heads, dim, rot, blocks=blocks, block_size=16, **kw) as plan:
        plan.launch([*x, p, frq, i32(slots)], [q_out, *caches])
        want[0][padding], room[0][padding] = 5.0, 0
        within(f64(q_out), want[0], room[0], "q")
        empty = np.full((blocks, k_heads, 16, dim), 7.0)
        within(f64(caches[0]), paged.stored(empty, want[1], slots), paged.stored(0 * empty, room[1], slots), "k")
        assert np.array_equal(f64(caches[1]), paged.stored(empty, f64(x[2]), slots))
        same = x[0].clone()      # in place: padding rows stay as they are
        plan.launch([same, *x[1:], p, frq, i32(slots)], [same, *caches])
        keep = torch.tensor(padding, device="cuda")
        assert torch.equal(same[~keep], q_out[~keep]) and torch.equal(same[keep], x[0][keep])


@pytest.mark.parametrize("dtype, q_heads, k_heads, dim, rot, interleaved, store, pad, each", [
    ("bf16", 11, 9, 80, 40, False, False, 0, 4), ("f16", 32, 8, 128, 24, False, True, 0, 4), ("f16", 7, 7, 20, 12, True, False, 4, 4), ("bf16", 13, 4, 36, 20, False, False, 2, 8),
    ("f16", 9, 9, 22, 22, False, True, 0, 8), ("bf16", 16, 1, 24, 24, False, False, 3, 8), ("f16", 5, 1, 24, 10, True, False, 6, 4), ("f32", 12, 4, 36, 20, False, False, 2, 4), ("f32", 15, 1, 10, 10, False, False, 1, 8),
    ("f32", 5, 2, 64, 64, False, True, 0, 4), ("f32", 2, 1, 64, 64, True, False, 0, 1), ("f32", 9, 1, 80, 24, False, False, 4, 4), ("bf16", 2, 1, 80, 40, False, False, 0, 1)])
def test_rotary_of_many_rows_in_narrow_vectors(dtype, q_heads, k_heads, dim, rot, interleaved, store, pad, each):
    """Rotated parts and strides that leave vectors of less than 16 bytes, or few heads: as many heads to a thread as their rule says, rows of outputs
    further apart than their heads."""
    rng, g = np.random.default_rng(dim + rot), torch.Generator("cuda").manual_seed(dim)
    tokens = 4 * 131072 // (q_heads + k_heads) // max(1, dim // 16) + 3
    heads = [q_heads, k_heads] + [k_heads] * store
    wide = [torch.randn((tokens, h * dim + pad), device="cuda", generator=g).to(DT[dtype]) for h in heads]
    x = [f64(w[:, :h * dim]).reshape(tokens, h, dim) for w, h in zip(wide, heads)]
    freqs, pos = fs_rotary_frequencies(rot), positions_of(rng, tokens, 1 << 17)
    frq, p = torch.tensor(freqs, dtype=torch.float64, device="cuda"), i32(pos)
    want = [paged.rotary(a, pos, freqs, interleaved, magnitude=0.75) for a in x[:2]]
    room = [rotary_bound(a, w, freqs, interleaved, 0.75, dtype) for a, w in zip(x, want)]
    kw = dict(interleaved=interleaved, magnitude=0.75, q_stride=q_heads * dim + pad, k_stride=k_heads * dim + pad, q_out_stride=q_heads * dim + pad)
    out = [torch.full_like(w, 5.0) for w in wide[:2]]
    if store:
        blocks = -(-tokens // 32) + 1
        slots = rng.permutation(blocks * 32)[:tokens]
        slots[::7] = -1
        caches = [torch.full((blocks, k_heads, 32, dim), 7.0, dtype=DT[dtype], device="cuda") for _ in range(2)]
        kw |= dict(v_stride=k_heads * dim + pad, blocks=blocks, block_size=32)
        ins, outs = [*wide, p, frq, i32(slots)], [out[0], *caches]
        want[0][slots < 0], room[0][slots < 0] = 5.0, 0
    else:
        kw |= dict(k_out_stride=k_heads * dim + pad)
        ins, outs = [*wide, p, frq], out
    with Plan.rotary(dtype, tokens, q_heads, k_heads, dim, rot, **kw) as plan:
        assert f"heads_each={each};" in plan.describe(), plan.describe()
        plan.launch(ins, outs)
    within(f64(out[0][:, :q_heads * dim]).reshape(tokens, q_heads, dim), want[0], room[0], "q")
    assert (out[0][:, q_heads * dim:] == 5).all()
    if store:
        empty = np.full((blocks, k_heads, 32, dim), 7.0)
        within(f64(caches[0]), paged.stored(empty, want[1], slots), paged.stored(0 * empty, room[1], slots), "k")
        assert np.array_equal(f64(caches[1]), paged.stored(empty, x[2], slots))
    else:
        within(f64(out[1][:, :k_heads * dim]).reshape(tokens, k_heads, dim), want[1], room[1], "k")
        assert (out[1][:, k_heads * dim:] == 5).all()


def test_rotary_gradient():
    """Against the formula's own (the transpose) and against differences, through torch's autograd."""
    t, h, d = 6, 2, 32
    freqs, pos = fs_rotary_frequencies(d, 100.0), np.arange(t) * 3
    frq, p = torch.tensor(freqs, dtype=torch.float64, device="cuda"), i32(pos)

    class Rotary(torch.autograd.Function):
        @staticmethod
        def forward(ctx, q, k):
            outs = [torch.empty_like(q), torch.empty_like(k)]
            forward.launch([q, k, p, frq], outs)
            return tuple(outs)

        @staticmethod
        def backward(ctx, dq, dk):
            outs = [torch.empty_like(dq), torch.empty_like(dk)]
            backward.launch([dq.contiguous(), dk.contiguous(), p, frq], outs)
            return tuple(outs)

    with Plan.rotary("f32", t, h, h, d, interleaved=True, magnitude=1.5) as forward, Plan.rotary("f32", t, h, h, d, interleaved=True, magnitude=1.5, inverse=True) as backward:
        g = torch.Generator("cuda").manual_seed(4)
        q, k, a, b = (torch.randn((t, h, d), device="cuda", generator=g) for _ in range(4))
        q.requires_grad_()
        k.requires_grad_()
        loss = lambda: sum((o * w).sum() for o, w in zip(Rotary.apply(q, k), (a, b)))  # noqa: E731
        loss().backward()
        for x, w in ((q, a), (k, b)):
            want = paged.rotary(f64(w), pos, freqs, True, True, 1.5)
            within(f64(x.grad), want, rotary_bound(f64(w), want, freqs, True, 1.5, "f32"), "gradient")
        # the call is linear: a step of 1 along a direction changes the loss by the gradient's product with it
        step = torch.randn((t, h, d), device="cuda", generator=g)
        with torch.no_grad():
            before = [o.double() for o in Rotary.apply(q, k)]
            after = [o.double() for o in Rotary.apply(q + step, k)]
            change = ((after[0] - before[0]) * a).sum().item()
            along = (q.grad.double() * step).sum().item()
        # 2 t h d outputs, each off by at most 8 steps of 1.5 * (|x0| + |x1|) < 20 in both launches, and q + step by one of 8
        assert abs(change - along) <= t * h * d * (2 * 8 * 2.0**-24 * 20 + 2.0**-24 * 8) * a.abs().max().item()


# ---------------------------------------------------------------------------------------------------- attention over the cache

def problem(rng, dtype, keys, new, q_heads, kv_heads, dim, block_size, order="head", pad_rows=0, spread=1.0):
    """Everything of a call: caches filled with NaN behind the lengths and in blocks of nobody."""
    g = torch.Generator("cuda").manual_seed(int(rng.integers(1 << 30)))
    held = [-(-n // block_size) for n in keys]
    width, blocks = max(held + [0]) + 1, sum(held) + 2
    pages = rng.permutation(blocks)
    tables, at = np.full((len(keys), width), -1), 0
    caches = [torch.full((blocks, kv_heads, block_size, dim), float("nan"), dtype=DT[dtype], device="cuda") for _ in range(2)]
    for b, n in enumerate(keys):
        tables[b, :held[b]] = pages[at:at + held[b]]
        at += held[b]
        if n:
            j = torch.arange(n, device="cuda")
            page = i32(tables[b]).long()[j // block_size]
            for c in caches:
                c[page, :, j % block_size] = (spread * torch.randn((n, kv_heads, dim), device="cuda", generator=g)).to(DT[dtype])
    t = sum(new) + pad_rows
    q = torch.randn((t, q_heads, dim), device="cuda", generator=g).to(DT[dtype])
    if order == "token":
        caches = [c.transpose(1, 2).contiguous() for c in caches]
    return dict(dtype=dtype, q=q, caches=caches, tables=tables, lengths=np.array(keys), starts=np.concatenate([[0], np.cumsum(new)]).astype(int), order=order, block_size=block_size,
                kv_heads=kv_heads, scale=dim ** -0.5)


def plan_of(c, window=0, causal=True, max_new=0, lse=True, q_stride=0, out_stride=0):
    t, h, d = c["q"].shape
    blocks = c["caches"][0].shape[0]
    strides = {} if c["order"] == "head" else dict(block_stride=c["block_size"] * c["kv_heads"] * d, head_stride=d, slot_stride=c["kv_heads"] * d)
    return Plan.paged_attention(c["dtype"], len(c["lengths"]), t, h, c["kv_heads"], d, blocks, c["block_size"], c["tables"].shape[1], c["scale"], causal, window, max_new, lse,
                                q_stride, out_stride, **strides)


def buffers(c, nbytes, lse=True):
    t, h, d = c["q"].shape
    return ([torch.full((t, h, d), 3.0, dtype=DT[c["dtype"]], device="cuda")] + ([torch.full((t, h), 3.0, device="cuda")] if lse else []) +
            ([torch.full((nbytes,), 255, dtype=torch.uint8, device="cuda")] if nbytes else []))


def inputs(c):
    return [c["q"], *c["caches"], i32(c["tables"]), i32(c["lengths"]), i32(c["starts"])]


def wanted(c, window=0, causal=True):
    k, v = (f64(x if c["order"] == "head" else x.transpose(1, 2)) for x in c["caches"])
    return paged.attention(f64(c["q"]), k, v, c["tables"], c["lengths"], c["starts"], c["scale"], causal, window)


def check_out(c, outs, want, what=""):
    out, lse, weight, small, top = want
    u, d = U[c["dtype"]], c["q"].shape[2]
    none = np.isnan(lse)
    off = (d + 4) * 2.0**-24 * top + 6 * 2.0**-24 * top + 2.0**-20
    room = (u + 2 * off[..., None]) * weight + 2.0**-25 * small + u * np.abs(out) + (2.0**-25 if c["dtype"] == "f16" else 0)
    got = f64(outs[0])
    assert (got[none] == 3.0).all(), what + ": a row of no request was written"
    within(got[~none], out[~none], room[~none], what + " out")
    if len(outs) > 1 and outs[1].dtype == torch.float32:
        got = f64(outs[1])
        assert (got[none] == 3.0).all(), what
        within(got[~none], lse[~none], (off + 2.0**-22 * np.abs(np.where(np.isfinite(lse), lse, 0)) + 2.0**-22)[~none], what + " lse")


def check_attention(c, window=0, causal=True, max_new=0):
    plan, nbytes = plan_of(c, window, causal, max_new)
    with plan:
        outs = buffers(c, nbytes)
        plan.launch(inputs(c), outs)
        torch.cuda.synchronize()
    check_out(c, outs, wanted(c, window, causal), plan_text(c, window, causal, max_new))
    return outs


def plan_text(c, *rest):
    return f"{c['dtype']} {tuple(c['q'].shape)} kv_heads {c['kv_heads']} lengths {c['lengths'].tolist()[:8]} starts {c['starts'].tolist()[:8]} block {c['block_size']} {c['order']} {rest}"


SHAPES = [   # keys, new tokens, q heads, kv heads, block size
    ([1], [1], 1, 1, 16),
    ([5, 0, 17, 1], [1, 0, 1, 1], 8, 2, 16),
    ([300, 33, 32, 31, 129, 128, 127], [1] * 7, 8, 2, 16),
    ([64, 65, 0, 600], [4, 0, 0, 7], 12, 4, 32),
    ([200, 7, 1000], [200, 7, 3], 4, 4, 64),
    ([513, 90], [130, 1], 16, 2, 128),
    ([2000], [1], 32, 2, 16),
    ([70, 3, 40], [70, 5, 1], 6, 2, 1),
    ([900, 1500], [1, 2], 5, 1, 1024),
    ([257, 258], [33, 64], 3, 3, 8),
]


@pytest.mark.parametrize("dtype, dim", [("bf16", 128), ("f16", 64), ("bf16", 96), ("f16", 128), ("bf16", 32)])
@pytest.mark.parametrize("shape", range(len(SHAPES)))
def test_attention(dtype, dim, shape):
    keys, new, q_heads, kv_heads, block = SHAPES[shape]
    rng = np.random.default_rng(shape)
    c = problem(rng, dtype, keys, new, q_heads, kv_heads, dim, block, order=("head", "token")[shape % 2], pad_rows=shape % 3)
    check_attention(c, max_new=(0, max(new))[shape % 2])


@pytest.mark.parametrize("shape", range(len(SHAPES)))
def test_attention_of_fp16_heads_of_96(shape):
    keys, new, q_heads, kv_heads, block = SHAPES[shape]
    c = problem(np.random.default_rng(shape), "f16", keys, new, q_heads, kv_heads, 96, block, order=("token", "head")[shape % 2], pad_rows=shape % 3)
    check_attention(c, max_new=(max(new), 0)[shape % 2])
    check_attention(c, window=60)


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("dim", [32, 64, 96, 128])
def test_attention_of_many_query_heads_to_a_key_head(dtype, dim):
    """17 and 32 of them: tiles of 32 rows beside tiles of 128, alone, in equal runs, and a workgroup each."""
    rng = np.random.default_rng(dim)
    for keys, new, share in (([300, 90, 40, 700, 5], [1, 30, 2, 1, 0], 17), ([40, 200], [5, 1], 32), ([3000, 64, 1700], [1, 1, 1], 32), ([200, 17, 1000], [1, 1, 1], 17)):
        c = problem(rng, dtype, keys, new, 2 * share, 2, dim, 16, order=("head", "token")[share == 32], pad_rows=1)
        check_attention(c, max_new=max(new))
    check_attention(c, max_new=0)
    check_attention(c, causal=False)
    keys = [int(k) for k in rng.integers(1, 60, 140)]
    check_attention(problem(rng, dtype, keys, [1] * 140, 34, 2, dim, 16), max_new=1)      # more tiles than CUs


@pytest.mark.parametrize("shape", [1, 3, 4, 5, 7, 9])
@pytest.mark.parametrize("window, causal", [(0, False), (1, True), (13, True), (64, True), (100, True), (100000, True)])
def test_attention_masks(shape, window, causal):
    keys, new, q_heads, kv_heads, block = SHAPES[shape]
    check_attention(problem(np.random.default_rng(shape), "bf16", keys, new, q_heads, kv_heads, 64, block), window, causal)


@pytest.mark.parametrize("max_new", [0, 1, 2, 8, 200])
def test_attention_takes_any_hint(max_new):
    c = problem(np.random.default_rng(5), "f16", [300, 40, 700, 129], [100, 1, 9, 33], 8, 2, 64, 16)
    check_attention(c, max_new=max_new)


@pytest.mark.parametrize("new", [1, 40])
def test_attention_bad_blocks(new):
    rng = np.random.default_rng(6)
    c = problem(rng, "bf16", [300, 90, 64], [new, new, new], 8, 2, 128, 16)
    c["tables"][0, [0, 3, 18]] = [-1, c["caches"][0].shape[0], 2**31 - 1]
    c["tables"][2, :] = -2**31                       # a request with no block at all: rows of zeros
    outs = check_attention(c)
    assert (f64(outs[0])[-new:] == 0).all() and (f64(outs[1])[-new:] == -np.inf).all()


@pytest.mark.parametrize("lengths, starts", [
    ([-5, 2**31 - 1, 30], [0, 2, 5, 9]), ([30, 30, 30], [-4, 2, 2, 2**31 - 1]), ([30, 20, 30], [0, 4, 4, 4]), ([0, 0, 0], [0, 3, 6, 9]), ([2, 30, 1], [0, 5, 7, 9])])
def test_attention_odd_lengths(lengths, starts):
    c = problem(np.random.default_rng(7), "f16", [40, 40, 40], [3, 3, 3], 4, 2, 32, 16)
    for x in c["caches"]:
        x.nan_to_num_(0.5)                           # lengths that pass what was stored read all of a block
    c["tables"][:, 3] = c["tables"][:, 0]
    c["lengths"], c["starts"] = np.array(lengths), np.array(starts)
    check_attention(c)


@pytest.mark.parametrize("starts", [[0, 9, 0, 9], [9, 0, 9, 0], [5, 5, 1, 9], [0, 9, 9, 9]])
@pytest.mark.parametrize("max_new", [0, 1])
def test_attention_rows_of_several_requests(starts, max_new):
    """Rows that no request or only one has are right whatever the others claim."""
    c = problem(np.random.default_rng(14), "bf16", [40, 40, 40], [3, 3, 3], 48, 3, 64, 16)
    c["starts"] = np.array(starts)
    claims = np.array([sum(starts[b] <= t < starts[b + 1] for b in range(3)) for t in range(9)])
    plan, nbytes = plan_of(c, max_new=max_new)
    with plan:
        outs = buffers(c, nbytes)
        plan.launch(inputs(c), outs)
    want = [a[claims < 2] for a in wanted(c)]
    check_out(dict(c, q=c["q"][claims < 2]), [outs[0][claims < 2], outs[1][claims < 2]], want, f"starts {starts}")


@pytest.mark.parametrize("q_heads, kv_heads", [(64, 1), (33, 1), (24, 1), (7, 7)])
@pytest.mark.parametrize("requests", [3, 70, 130])
def test_attention_of_many_requests(q_heads, kv_heads, requests):
    """More requests than a wavefront has lanes, single tokens and chunks among each other, runs of heads beyond a tile's rows."""
    rng = np.random.default_rng(requests)
    new = [int(n) for n in rng.choice([0, 1, 1, 2, 5, 40], requests)]
    keys = [n + int(k) for n, k in zip(new, rng.choice([0, 1, 30, 200], requests))]
    c = problem(rng, "bf16", keys, new, q_heads, kv_heads, 32, 16, order="token", pad_rows=2)
    check_attention(c)
    check_attention(c, window=2**31 - 1)


@pytest.mark.parametrize("requests, chunks", [(64, 3), (65, 3), (130, 64), (130, 65), (300, 1), (512, 5), (513, 5)])
def test_attention_of_chunks_among_many_requests(requests, chunks):
    """A few long chunks, whose keys are split, scattered among single tokens; as many chunks as one line takes, and one more."""
    rng = np.random.default_rng(requests + chunks)
    new, keys = rng.integers(0, 3, requests), rng.integers(3, 40, requests)
    for b in rng.permutation(requests)[:chunks]:
        new[b] = rng.integers(5, 70)
        keys[b] = rng.integers(new[b], 2500 if chunks < 10 else 300)
    c = problem(rng, "f16", [int(k) for k in keys], [int(n) for n in new], 8, 2, 64, 16)
    check_attention(c)
    check_attention(c, window=500)
    check_attention(c, causal=False)


@pytest.mark.parametrize("singles, behind, split", [(0, 0, True), (500, 448, False), (30, 12, True)])
def test_attention_counts_short_requests_in_the_shares(singles, behind, split):
    """A chunk of 32 steps of 64 keys is split over workgroups where it is all there is, not where hundreds of requests of seven steps a head
    make an even share longer than it.  Parts of split tiles are written to the last 2 * 512 places of the partial results."""
    dim, heads = 32, 8
    c = problem(np.random.default_rng(singles), "f16", [behind] * (singles // 2) + [2048] + [behind] * (singles - singles // 2), [1] * (singles // 2) + [128] + [1] * (singles - singles // 2),
                heads, heads, dim, 16)
    outs = check_attention(c)
    assert bool((outs[-1][-2 * 512 * 128 * (dim + 2) * 4:] != 255).any()) == split


@pytest.mark.parametrize("table_keys, long", [(64, 60), (2048, 1900)])
def test_attention_of_thousands_of_requests(table_keys, long):
    """More than 4096 requests, single tokens: a workgroup each tile, and equal runs whose ends are searched behind the first 4096."""
    requests = 4300
    rng = np.random.default_rng(table_keys)
    lengths = rng.integers(0, 4, requests)
    new = np.minimum(lengths, rng.integers(0, 2, requests))
    for b in (0, 63, 64, 4095, 4096, 4200, 4299):
        lengths[b], new[b] = long - b % 7, 1
    blocks, size, dim, heads = 600, 16, 32, 2
    g = torch.Generator("cuda").manual_seed(5)
    caches = [torch.randn((blocks, 1, size, dim), device="cuda", generator=g).half() for _ in range(2)]
    tables = rng.integers(0, blocks, (requests, table_keys // size))
    c = dict(dtype="f16", q=torch.randn((int(new.sum()) + 1, heads, dim), device="cuda", generator=g).half(), caches=caches, tables=tables, lengths=lengths,
             starts=np.concatenate([[0], np.cumsum(new)]), order="head", block_size=size, kv_heads=1, scale=dim ** -0.5)
    check_attention(c, max_new=1)


@pytest.mark.parametrize("order", ["head", "token"])
@pytest.mark.parametrize("kv_heads, dim", [(1, 64), (2, 32), (6, 96), (12, 128), (32, 32), (48, 64), (64, 32), (100, 32), (7, 96)])
def test_attention_of_sets_of_key_heads(kv_heads, dim, order):
    """Heads whose workgroups walk the same keys: no set, one, several; less work than workgroups; single tokens alone and beside a chunk."""
    rng = np.random.default_rng(kv_heads + dim)
    for keys, new, share in (([1500, 3, 700, 64], [1, 1, 1, 1], 2), ([2, 0], [1, 0], 3), ([1300, 90, 5], [1, 70, 0], 1)):
        c = problem(rng, "bf16", keys, new, share * kv_heads, kv_heads, dim, 16, order=order)
        c["tables"] = np.pad(c["tables"], ((0, 0), (0, 100)), constant_values=-1)      # more than 1024 keys to a row
        check_attention(c, max_new=max(new))


@pytest.mark.parametrize("new", [1, 3, 90])
def test_attention_behind_a_billion_keys(new):
    """2^30 - 5 keys, the most that a row of the table may name but five, of which a window leaves the last ones: as of a request of the same end alone."""
    rng, g = np.random.default_rng(new), torch.Generator("cuda").manual_seed(new)
    blocks, size, dim, row, keys = 7, 1024, 64, 1 << 20, 2**30 - 5
    caches = [torch.randn((blocks, 2, size, dim), device="cuda", generator=g).bfloat16() for _ in range(2)]
    tables = rng.integers(0, blocks, (2, row))
    c = dict(dtype="bf16", q=torch.randn((new + 2, 6, dim), device="cuda", generator=g).bfloat16(), caches=caches, tables=tables, lengths=np.array([keys, 40]), starts=np.array([0, new, new + 2]),
             order="head", block_size=size, kv_heads=2, scale=0.125)
    end = dict(c, tables=np.where([[True], [False]], tables[:, -3:], tables[:, :3]), lengths=np.array([keys - (row - 3) * size, 40]))
    plan, nbytes = plan_of(c, 700, max_new=new)
    with plan:
        outs = buffers(c, nbytes)
        plan.launch(inputs(c), outs)
        torch.cuda.synchronize()
    check_out(c, outs, wanted(end, 700))


@pytest.mark.parametrize("new", [1, 2, 60])
def test_attention_of_one_long_request(new):
    """Keys of one tile over many workgroups: the parts are joined in the order of the keys."""
    c = problem(np.random.default_rng(15), "bf16", [40000, 3], [new, 1], 4, 1, 128, 64)
    check_attention(c, max_new=new)
    check_attention(c, max_new=new, window=20000)


@pytest.mark.parametrize("new, keys", [(3, 40), (70, 200), (150, 150)])
@pytest.mark.parametrize("value", [float("nan"), float("inf"), float("-inf")])
def test_attention_values_that_some_rows_do_not_see(new, keys, value):
    """NaN or infinity in keys and values of later tokens: the rows before them are as if it were not there."""
    rng = np.random.default_rng(8)
    c = problem(rng, "bf16", [keys], [new], 4, 2, 64, 16)
    for window in (0, 20):
        j = [keys - new // 2, keys - 1] + ([0] if window else [])
        for x in c["caches"]:
            for k in j:
                x[c["tables"][0, k // 16], :, k % 16, ::5] = value
        plan, nbytes = plan_of(c, window)
        with plan:
            outs = buffers(c, nbytes)
            plan.launch(inputs(c), outs)
        got = f64(outs[0])
        clean = [k for k in range(new) if not any(keys - new + k - (window or keys) < b <= keys - new + k for b in j)]
        assert clean
        with np.errstate(all="ignore"):
            want = wanted(c, window)
        full = np.array([k not in clean for k in range(new)])
        assert np.isfinite(got[clean]).all()
        touched = got[full][:, :, ::5]
        assert not np.isfinite(touched).any() or not np.isnan(value)      # a row that sees a NaN has it
        part = [np.array(a) for a in want]
        check_out(dict(c, q=c["q"][clean]), [outs[0][clean], outs[1][clean]], [a[clean] for a in part], f"rows before a {value}")


def put_value(c, request, key, value, every=5):
    """`value` in every fifth element of the value of a request's key, whose key itself stays as it is."""
    page = int(c["tables"][request, key // c["block_size"]])
    v = c["caches"][1] if c["order"] == "head" else c["caches"][1].transpose(1, 2)
    v[page, :, key % c["block_size"], ::every] = value


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("value", [float("inf"), float("-inf"), float("nan")])
@pytest.mark.parametrize("keys, new, places, window", [
    (3, 3, [0], 0), (40, 3, [0, 38], 0), (40, 3, [20, 37], 20), (500, 1, [0, 250, 499], 0), (40000, 2, [0, 20000, 39999], 0),      # few rows: one workgroup, several
    (150, 150, [0], 0), (150, 150, [63, 149], 0), (300, 70, [0, 230, 299], 0), (300, 150, [150, 200], 100), (9000, 60, [0, 4000, 8990], 0)])      # tiles; of split keys
def test_attention_of_values_that_are_infinite(dtype, value, keys, new, places, window):
    """Infinities or NaN in values alone, their keys numbers: the rows that see them have them as the definition does, the others do not."""
    c = problem(np.random.default_rng(keys), dtype, [keys, 7], [new, 1], 4, 2, 64, 16)
    for k in places:
        put_value(c, 0, k, value)
    with np.errstate(invalid="ignore"):
        want = wanted(c, window)
    plan, nbytes = plan_of(c, window)
    with plan:
        outs = buffers(c, nbytes)
        plan.launch(inputs(c), outs)
    check_out(c, outs, want, plan_text(c, window, value))


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("keys, new", [(600, 1), (40000, 2), (150, 150), (9000, 60)])
def test_attention_of_infinite_values_behind_a_small_weight(dtype, keys, new):
    """Scores of the last keys are 320 above those before them: what was summed up until then is taken times e^-320, which fp32 has no number
    for, and an infinity among it stays one, inside a run of keys, between wavefronts and between parts."""
    c = problem(np.random.default_rng(keys), dtype, [keys], [new], 4, 2, 64, 16)
    high = 64 if keys == 150 else keys - 64
    c["q"] = torch.ones_like(c["q"])
    for k in range(high, keys):
        c["caches"][0][c["tables"][0, k // 16], :, k % 16] = 40.0
    put_value(c, 0, 0, float("inf"))
    with np.errstate(invalid="ignore"):
        want = wanted(c)
    assert np.isposinf(want[0]).any()
    plan, nbytes = plan_of(c)
    with plan:
        outs = buffers(c, nbytes)
        plan.launch(inputs(c), outs)
    check_out(c, outs, want, plan_text(c))


@pytest.mark.parametrize("keys, new", [(40, 3), (3000, 1), (150, 150), (9000, 60)])
def test_attention_of_scores_of_minus_infinity(keys, new):
    """Keys whose scores are -inf have no weight; a row of nothing else is like one that sees no key."""
    c = problem(np.random.default_rng(keys), "bf16", [keys, keys], [new, new], 4, 2, 64, 16)
    c["q"][..., 0] = 1.0
    low = list(range(0, keys, 3)) + list(range(keys - keys // 4, keys - 1))
    for b, some in ((0, [k for k in low if k != 1]), (1, range(keys))):
        for k in some:
            c["caches"][0][c["tables"][b, k // 16], :, k % 16, 0] = float("-inf")
    plan, nbytes = plan_of(c)
    with plan:
        outs = buffers(c, nbytes)
        plan.launch(inputs(c), outs)
    with np.errstate(invalid="ignore"):
        out, lse, weight, small, top = (a[:new] for a in wanted(c))
    seen = np.isfinite(out).all((1, 2))                               # (the first row of a prompt sees one key, whose score is -inf)
    assert seen[1:].all()
    top[:] = 64 * 0.125 * 36                                          # of the finite ones: |q| and |k| are below 6
    check_out(dict(c, q=c["q"][:new][seen]), [outs[0][:new][seen], outs[1][:new][seen]], [a[seen] for a in (out, lse, weight, small, top)], plan_text(c))
    none = np.concatenate([~seen, np.ones(new, bool)])
    assert (f64(outs[0])[none] == 0).all() and (f64(outs[1])[none] == -np.inf).all()


def test_attention_scores_of_any_size():
    c = problem(np.random.default_rng(9), "bf16", [500, 90], [1, 60], 4, 2, 64, 16, spread=8.0)
    check_attention(c)
    c["scale"] = 0.0
    check_attention(c)
    c["scale"] = -0.3
    check_attention(c)


def test_attention_of_parts_of_a_projection():
    c = problem(np.random.default_rng(10), "f16", [100, 30], [1, 25], 4, 2, 64, 16)
    t, h, d = c["q"].shape
    row = h * d + 72
    wide, out = torch.zeros((t, row), dtype=torch.float16, device="cuda"), torch.full((t, row), 3.0, dtype=torch.float16, device="cuda")
    wide[:, :h * d] = c["q"].flatten(1)
    plan, nbytes = plan_of(c, q_stride=row, out_stride=row)
    with plan:
        outs = [out] + buffers(c, nbytes)[1:]
        plan.launch([wide, *inputs(c)[1:]], outs)
    check_out(c, [out[:, :h * d].unflatten(1, (h, d)), outs[1]], wanted(c), "parts")
    assert (out[:, h * d:] == 3).all()


def test_attention_without_lse_and_twice_the_same():
    c = problem(np.random.default_rng(11), "bf16", [3000, 40, 900], [1, 1, 30], 16, 2, 128, 16)
    outs = check_attention(c)
    plan, nbytes = plan_of(c, lse=False)
    with plan:
        for _ in range(3):
            again = buffers(c, nbytes, lse=False)
            plan.launch(inputs(c), again)
            assert torch.equal(again[0], outs[0])


def test_attention_behind_32_bits():
    """A cache of more than 2^32 elements: the last blocks of it, in both orders."""
    blocks, heads, size, dim = 1050, 8, 1024, 512      # strides of 512, of which 128 are a head's: 2 * 4.4e9 elements
    raw = torch.zeros(blocks * heads * size * dim + 4096, dtype=torch.float16, device="cuda")
    assert raw.numel() > 2**32
    rng = np.random.default_rng(12)
    for strides in ((heads * size * dim, size * dim, dim), (size * heads * dim, dim, heads * dim)):
        k = raw.as_strided((blocks, heads, size, 128), (strides[0], strides[1], strides[2], 1))
        v = raw.as_strided((blocks, heads, size, 128), (strides[0], strides[1], strides[2], 1), 128)
        page = [blocks - 1, 3, blocks - 2]
        small_k, small_v = torch.zeros((3, heads, size, 128), dtype=torch.float16, device="cuda"), torch.zeros((3, heads, size, 128), dtype=torch.float16, device="cuda")
        for i, b in enumerate(page):
            k[b], v[b] = torch.randn((heads, size, 128), device="cuda"), torch.randn((heads, size, 128), device="cuda")
            small_k[i], small_v[i] = k[b], v[b]
        q = torch.randn((1, heads, 128), dtype=torch.float16, device="cuda")
        plan, nbytes = Plan.paged_attention("f16", 1, 1, heads, heads, 128, blocks, size, 3, 0.1, lse=True, block_stride=strides[0], head_stride=strides[1], slot_stride=strides[2])
        with plan:
            outs = [torch.empty_like(q), torch.empty((1, heads), device="cuda")] + ([torch.empty(nbytes, dtype=torch.uint8, device="cuda")] if nbytes else [])
            plan.launch([q, k, v, i32([page]), i32([2500]), i32([0, 1])], outs)
        c = dict(dtype="f16", q=q, kv_heads=heads)
        check_out(c, outs, paged.attention(f64(q), f64(small_k), f64(small_v), [[0, 1, 2]], [2500], [0, 1], 0.1), "far blocks")
    with Plan.rotary("f16", 2, 1, heads, 128, blocks=blocks, block_size=size, block_stride=strides[0], head_stride=strides[1], slot_stride=strides[2]) as plan:
        x = torch.randn((2, heads, 128), dtype=torch.float16, device="cuda")
        freqs = torch.tensor(fs_rotary_frequencies(128), dtype=torch.float64, device="cuda")
        plan.launch([x[:, :1].contiguous(), x, x, i32([0, 0]), freqs, i32([blocks * size - 1, 5])], [torch.empty((2, 1, 128), dtype=torch.float16, device="cuda"), k, v])
        assert torch.equal(k[blocks - 1, :, size - 1], x[0]) and torch.equal(v[0, :, 5], x[1])


# ---------------------------------------------------------------------------------------------------- together, streams, graphs

class Server:
    """A cache, its plans for steps of up to `tokens` rows, and the calls of a step in their order."""

    def __init__(self, requests, tokens, block_size, width, q_heads, kv_heads, dim, dtype, n_blocks):
        e = lambda *n: torch.zeros(n, dtype=torch.int32, device="cuda")  # noqa: E731
        self.cached, self.fresh, self.free = e(requests), e(requests), torch.randperm(n_blocks, device="cuda").to(torch.int32)
        self.table = torch.full((requests, width), -1, dtype=torch.int32, device="cuda")
        self.lengths, self.starts, self.positions, self.slots, self.taken = e(requests), e(requests + 1), e(tokens), e(tokens), e(2)
        self.caches = [torch.full((n_blocks, kv_heads, block_size, dim), float("nan"), dtype=DT[dtype], device="cuda") for _ in range(2)]
        self.qkv = torch.zeros((tokens, (q_heads + 2 * kv_heads) * dim), dtype=DT[dtype], device="cuda")
        self.parts = self.qkv.split([q_heads * dim, kv_heads * dim, kv_heads * dim], 1)
        self.freqs = torch.tensor(fs_rotary_frequencies(dim), dtype=torch.float64, device="cuda")
        self.q, self.out = (torch.zeros((tokens, q_heads, dim), dtype=DT[dtype], device="cuda") for _ in range(2))
        row = self.qkv.shape[1]
        self.tables_plan = Plan.block_tables(requests, tokens, n_blocks, block_size, width, n_blocks)
        self.rotary_plan = Plan.rotary(dtype, tokens, q_heads, kv_heads, dim, blocks=n_blocks, block_size=block_size, q_stride=row, k_stride=row, v_stride=row)
        self.attention_plan, nbytes = Plan.paged_attention(dtype, requests, tokens, q_heads, kv_heads, dim, n_blocks, block_size, width, dim ** -0.5)
        self.partials = [torch.empty(nbytes, dtype=torch.uint8, device="cuda")] if nbytes else []

    def step(self):
        self.tables_plan.launch([self.cached, self.fresh, self.free], [self.table, self.lengths, self.starts, self.positions, self.slots, self.taken])
        self.rotary_plan.launch([*self.parts, self.positions, self.freqs, self.slots], [self.q, *self.caches])
        self.attention_plan.launch([self.q, *self.caches, self.table, self.lengths, self.starts], [self.out, *self.partials])

    def next(self):
        """What a server does between steps: the tokens are cached now, their blocks are gone from the free list."""
        self.cached.copy_(self.lengths)
        self.free = torch.roll(self.free, -int(self.taken[0]))


def test_steps_of_a_server():
    """Prompts in chunks under a token budget, then single tokens: every step's rows against attention over all that the requests were given."""
    rng = np.random.default_rng(13)
    hq, hk, d, dtype = 8, 2, 64, "bf16"
    s = Server(5, 48, 16, 12, hq, hk, d, dtype, 60)
    prompts = [70, 3, 0, 33, 90]
    given = [np.zeros((0, (hq + 2 * hk) * d)) for _ in prompts]
    freqs = fs_rotary_frequencies(d)
    for step in range(9):
        left = [max(0, p - len(g)) for p, g in zip(prompts, given)]
        new = [n if n else int(rng.random() < 0.8 and step > 3) for n in left]
        s.fresh.copy_(i32(new))
        s.qkv.copy_(torch.randn(s.qkv.shape, device="cuda"))
        s.out.fill_(3.0)
        s.step()
        starts, rows = s.starts.cpu().numpy(), f64(s.qkv)
        for b in range(len(prompts)):
            given[b] = np.concatenate([given[b], rows[starts[b]:starts[b + 1]]])
        assert s.lengths.cpu().tolist() == [len(g) for g in given]
        out = f64(s.out)
        assert (out[starts[-1]:] == 3.0).all()
        for b, g in enumerate(given):
            n, m = len(g), starts[b + 1] - starts[b]
            if not m:
                continue
            q, k, v = (x.reshape(n, -1, d) for x in np.split(g, [hq * d, (hq + hk) * d], 1))
            q, k = paged.rotary(q, np.arange(n), freqs), paged.rotary(k, np.arange(n), freqs)
            want, _, weight, small, top = paged.attention(q[n - m:], k.transpose(1, 0, 2)[None], v.transpose(1, 0, 2)[None].copy(), [[0]], [n], [0, m], d ** -0.5)
            # as in check_out, and q and k are rounded on their way into the cache: the scores by 2 u of their absolute sum more
            u = U[dtype]
            off = 2.5 * u * top + 2.0**-16
            within(out[starts[b]:starts[b + 1]], want, (u + 2 * off[..., None]) * weight + u * np.abs(want), f"step {step} request {b}")
        s.next()
    assert len(given[4]) > 90      # its prompt is through, single tokens followed


def test_two_launches_of_a_plan_at_once():
    """On two streams, with outputs and partial results of their own."""
    c = problem(np.random.default_rng(16), "f16", [5000, 700, 20000], [1, 1, 30], 8, 2, 64, 16)
    plan, nbytes = plan_of(c, max_new=0)
    streams = [torch.cuda.Stream() for _ in range(2)]
    with plan:
        ins, sets = inputs(c), [buffers(c, nbytes) for _ in range(2)]
        alone = buffers(c, nbytes)
        plan.launch(ins, alone)
        torch.cuda.synchronize()
        for _ in range(5):
            for s, outs in zip(streams, sets):
                plan.launch(ins, outs, s.cuda_stream)
        torch.cuda.synchronize()
    for outs in sets:
        assert torch.equal(outs[0], alone[0]) and torch.equal(outs[1], alone[1])
    check_out(c, alone, wanted(c), "two streams")


def test_steps_in_a_graph():
    """The step captured once and replayed with new lengths, between eager steps of the same server on another stream."""
    s = Server(6, 32, 16, 20, 8, 4, 128, "f16", 130)
    s.fresh.copy_(i32([3, 20, 0, 5, 1, 9]))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    s.qkv.copy_(torch.randn(s.qkv.shape, device="cuda"))
    with torch.cuda.stream(side):
        s.step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        s.step()
    for new in ([1] * 6, [9, 0, 0, 9, 30, 1], [0] * 6, [1, 1, 0, 1, 1, 1], [32, 1, 1, 1, 1, 1]):
        s.cached.copy_(s.lengths)
        s.fresh.copy_(i32(new))
        s.free.copy_(torch.roll(s.free, -int(s.taken[0])))
        s.qkv.copy_(torch.randn(s.qkv.shape, device="cuda"))
        watched = [s.table, s.lengths, s.starts, s.positions, s.slots, s.taken, s.q, *s.caches, s.out]
        before = [t.clone() for t in watched]
        graph.replay()
        torch.cuda.synchronize()
        replayed = [t.clone() for t in watched]
        for t, b in zip(watched, before):
            t.copy_(b)
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            s.step()
        torch.cuda.synchronize()
        for t, r in zip(watched, replayed):
            assert torch.equal(t.view(torch.int16) if t.dtype == torch.float16 else t, r.view(torch.int16) if r.dtype == torch.float16 else r)
