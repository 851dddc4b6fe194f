"""The paged cache in 8 bits on the GPU, against its definitions in 64 bits (oracle/paged8.py, oracle/paged.py).

Tolerances.  u: half a step of the storage type, relative.
  store, read  None: codes and scales are powers of two and single roundings of exact numbers.  Scales that are no powers of two, read: the product is rounded
               to fp32 and then to the type: u |x| + 2^-24 |x|, fp16 also 2^-25 where its numbers end.
  attention    As over a cache of numbers (test_gpu_paged.py), with two more roundings of a score (its scale times the call's, and the product with it) and one of a
               weight.  Scales that are no powers of two: keys' and values' numbers may be rounded to the type once more, u of each (fp16 values: and 2^-25).
"""
import numpy as np
import pytest
import torch

from oracle import paged, paged8
from paper_1911_11576_amd import Plan, fs_rotary_frequencies
from test_gpu_paged import DT, U, f64, i32, rotary_bound, within

pytestmark = pytest.mark.gpu

CODES = ["e4m3", "int8"]


def u8(a):
    return torch.as_tensor(np.ascontiguousarray(a).view(np.uint8), device="cuda")


def placed(a, order):
    """[blocks, heads, place, D] as it lies on the device, and back."""
    return a if order == "head" else np.ascontiguousarray(a.transpose(0, 2, 1, 3))


def strides_of(order, heads, size, dim):
    return {} if order == "head" else dict(block_stride=size * heads * dim, head_stride=dim, slot_stride=heads * dim)


def cache_of(rng, code, lengths, heads, dim, size, scale="powers", extra=2):
    """Tables, codes and scales of a cache in use: what is behind a length or in blocks of nobody are codes and scales that are no numbers."""
    held = [-(-max(0, n) // size) for n in lengths]
    width, blocks = max(held + [0]) + 1, sum(held) + extra
    pages = rng.permutation(blocks)
    tables, at = np.full((len(lengths), width), -1), 0
    garbage = 0x7F if code == "e4m3" else 0x80
    codes = [np.full((blocks, heads, size, dim), garbage, np.uint8) for _ in range(2)]
    scales = [np.full((blocks, heads), np.nan, np.float32) for _ in range(2)]
    for b, n in enumerate(lengths):
        tables[b, :held[b]] = pages[at:at + held[b]]
        at += held[b]
        for k in range(2):
            for j, page in enumerate(tables[b, :held[b]]):
                m = min(size, n - j * size)
                codes[k][page, :, :m] = paged8.coded(np.clip(rng.standard_normal((heads, m, dim)) * (64 if code == "e4m3" else 30), -127, 127), code)
                s = 2.0 ** rng.integers(-8, -4, heads)
                scales[k][page] = s if scale == "powers" else (s * rng.uniform(1, 2, heads)).astype(np.float32)
    return tables, codes, scales


# ---------------------------------------------------------------------------------------------------- store

def run_store(dtype, code, x, tables, codes, scales, lengths, starts, size, order="head", pad=0, static=False, stream=None):
    """x: k and v, [T, H, D] on the device; -> codes and scales of both, in the oracle's order."""
    t, heads, dim = x[0].shape
    blocks = codes[0].shape[0]
    wide = [torch.cat([a.reshape(t, heads * dim), torch.full((t, pad), 9.0, dtype=a.dtype, device="cuda")], 1).contiguous() for a in x]
    outs = [u8(placed(c, order)) for c in codes] + [torch.tensor(s, device="cuda") for s in scales]
    with Plan.cache_store8(dtype, code, len(lengths), t, heads, dim, blocks, size, tables.shape[1], k_stride=heads * dim + pad, v_stride=heads * dim + pad,
                           **strides_of(order, heads, size, dim)) as plan:
        (plan.launch_static if static else plan.launch)([*wide, i32(tables), i32(lengths), i32(starts)], outs, stream)
        torch.cuda.synchronize()
    got = [o.cpu().numpy() for o in outs]
    return [placed(c, order) for c in got[:2]], got[2:]


def check_store(dtype, code, x, tables, codes, scales, lengths, starts, size, **kw):
    got_codes, got_scales = run_store(dtype, code, x, tables, codes, scales, lengths, starts, size, **kw)
    for k in range(2):
        want = paged8.store(f64(x[k]), codes[k], scales[k], tables, lengths, starts, code, dtype)
        assert np.array_equal(got_scales[k], want[1].astype(np.float32), equal_nan=True), "scales of " + "kv"[k]
        wrong = got_codes[k] != want[0]
        assert not wrong.any(), f"{'kv'[k]}: {wrong.sum()} codes differ, the first at {np.argwhere(wrong)[0]}: {got_codes[k][wrong][0]} for {want[0][wrong][0]}"
    return got_codes, got_scales


def numbers_of(g, dtype, t, heads, dim):
    """Rows of different ranges, some of zeros."""
    far = torch.exp2(8 * torch.rand((t, heads, 1), device="cuda", generator=g) - 5)
    x = torch.randn((t, heads, dim), device="cuda", generator=g) * far
    return torch.where(torch.rand((t, heads, 1), device="cuda", generator=g) < 0.1, 0.0, x).to(DT[dtype])


STORES = [   # lengths, new tokens, heads, dim, block size
    ([1], [1], 1, 16, 8),
    ([5, 0, 17, 33], [1, 0, 1, 1], 8, 128, 16),
    ([300, 33, 32, 31, 129, 128, 127], [1] * 7, 3, 64, 16),
    ([64, 65, 0, 600], [4, 0, 0, 7], 4, 96, 32),
    ([200, 7, 1000], [200, 7, 3], 2, 80, 64),
    ([513, 90, 8], [130, 1, 8], 5, 32, 128),
    ([2000], [1500], 2, 128, 1024),
    ([70, 3, 40], [70, 2, 33], 1, 512, 8),
    ([900, 1500], [899, 1100], 2, 256, 256),
    ([31, 47, 16, 15, 32], [30, 17, 16, 15, 1], 16, 48, 16),
]


@pytest.mark.parametrize("code", CODES)
@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("shape", range(len(STORES)))
def test_store(dtype, code, shape):
    lengths, new, heads, dim, size = STORES[shape]
    rng, g = np.random.default_rng(shape), torch.Generator("cuda").manual_seed(shape)
    tables, codes, scales = cache_of(rng, code, lengths, heads, dim, size)
    t = sum(new) + shape % 3
    x = [numbers_of(g, dtype, t, heads, dim) for _ in range(2)]
    starts = np.concatenate([[0], np.cumsum(new)])
    check_store(dtype, code, x, tables, codes, scales, lengths, starts, size, order=("head", "token")[shape % 2], pad=(0, 16, 8)[shape % 3], static=shape % 2 == 1)


@pytest.mark.parametrize("code", CODES)
@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
def test_store_of_odd_numbers(dtype, code):
    """Infinities and NaN, the largest numbers, subnormal ones, both zeros; a head of each in a block of its own, single and behind others."""
    biggest = {"f16": 65504.0, "bf16": float(2.0**127 * (2 - 2.0**-7)), "f32": float(np.finfo(np.float32).max)}[dtype]
    least = {"f16": 2.0**-24, "bf16": 2.0**-133, "f32": 2.0**-149}[dtype]
    odd = [np.inf, -np.inf, np.nan, biggest, -biggest, 0.97 * biggest, 0.875 * biggest, least, -3 * least, 2.0**-14, -0.0, 0.0]
    heads, dim, size, n = len(odd), 32, 16, 21
    rng, g = np.random.default_rng(5), torch.Generator("cuda").manual_seed(5)
    x = [torch.randn((n, heads, dim), device="cuda", generator=g).to(DT[dtype]) for _ in range(2)]
    for k, row in enumerate(((7, 20), (0, 16))):
        for h, value in enumerate(odd):
            x[k][:, h] *= 0 if h >= 7 else 1
            for r in row:
                x[k][r, h, (3 * h + r) % dim] = value
    tables, codes, scales = cache_of(rng, code, [n], heads, dim, size)
    check_store(dtype, code, x, tables, codes, scales, [n], [0, n], size)                               # all new
    check_store(dtype, code, [a[:8] for a in x], tables, codes, scales, [13], [0, 8], size)             # behind five others
    check_store(dtype, code, [a[20:] for a in x], tables, codes, scales, [n], [0, 1], size)


@pytest.mark.parametrize("code", CODES)
def test_store_behind_scales_of_others(code):
    """A block begun under a scale of 0, no power of two, below 0, infinite, NaN, subnormal, or beyond 2^127."""
    odd = np.array([0.0, 3.0, 0.75, -0.5, np.inf, np.nan, 1e-40, 3e38, 2.0**100, 2.0**-126], np.float32)
    heads, g = len(odd), torch.Generator("cuda").manual_seed(1)
    tables, codes, scales = cache_of(np.random.default_rng(1), code, [9], heads, 64, 16)
    for s in scales:
        s[tables[0, 0]] = odd
    x = [torch.randn((2, heads, 64), device="cuda", generator=g).to(torch.bfloat16) for _ in range(2)]
    check_store("bf16", code, x, tables, codes, scales, [9], [0, 2], 16)


@pytest.mark.parametrize("new, lengths, starts", [
    (40, [37, 90, -4], [0, 12, 40, 40]), (9, [5, 100000, 3], [0, 9, 9, 9]), (12, [30, 0, 8], [0, 3, 8, 99]), (12, [30, 0, 8], [-5, 3, 8, 10]), (6, [30, 20, 8], [2, 3, 3, 5])])
def test_store_of_odd_lengths(new, lengths, starts):
    """More new tokens than a request has, lengths below 0 and beyond the table's row, starts outside the rows."""
    g = torch.Generator("cuda").manual_seed(3)
    tables, codes, scales = cache_of(np.random.default_rng(3), "e4m3", [64, 64, 64], 2, 64, 16)
    x = [numbers_of(g, "bf16", new, 2, 64) for _ in range(2)]
    check_store("bf16", "e4m3", x, tables, codes, scales, lengths, starts, 16)


def test_store_into_bad_blocks():
    g = torch.Generator("cuda").manual_seed(4)
    tables, codes, scales = cache_of(np.random.default_rng(4), "int8", [70, 50], 3, 32, 16)
    tables[0, 1], tables[0, 3], tables[1, 3] = -1, 2**31 - 1, len(codes[0])
    x = [numbers_of(g, "f16", 110, 3, 32) for _ in range(2)]
    check_store("f16", "int8", x, tables, codes, scales, [70, 50], [0, 65, 110], 16)


@pytest.mark.parametrize("starts", [[0, 9, 0, 9], [9, 0, 9, 0], [5, 5, 1, 9]])
def test_store_of_rows_of_several_requests(starts):
    """Undefined rows, but nothing outside the requests' blocks is written."""
    g = torch.Generator("cuda").manual_seed(4)
    tables, codes, scales = cache_of(np.random.default_rng(4), "e4m3", [20, 30, 40], 2, 32, 16)
    x = [numbers_of(g, "f16", 9, 2, 32) for _ in range(2)]
    got, got_scales = run_store("f16", "e4m3", x, tables, codes, scales, [20, 30, 40], starts, 16)
    others = np.setdiff1d(np.arange(len(codes[0])), tables)
    assert all(np.array_equal(a[others], b[others]) for a, b in zip(got, codes)) and all(np.array_equal(a[others], b[others], equal_nan=True) for a, b in zip(got_scales, scales))


@pytest.mark.parametrize("requests, heads", [(1000, 1), (4097, 3)])
def test_store_of_many_requests(requests, heads):
    rng, g = np.random.default_rng(requests), torch.Generator("cuda").manual_seed(1)
    new = rng.integers(0, 3, requests)
    lengths = np.where(new > 0, rng.integers(2, 40, requests), rng.integers(0, 40, requests))
    tables, codes, scales = cache_of(rng, "e4m3", lengths, heads, 16, 8)
    x = [numbers_of(g, "bf16", int(new.sum()), heads, 16) for _ in range(2)]
    check_store("bf16", "e4m3", x, tables, codes, scales, lengths, np.concatenate([[0], np.cumsum(new)]), 8)


@pytest.mark.parametrize("code", CODES)
@pytest.mark.parametrize("dim, size", [(128, 64), (64, 256), (512, 8), (80, 128)])
def test_store_of_a_long_request_among_single_tokens(code, dim, size):
    """What registers hold goes by the requests' mean share; the long one's blocks have more, and begin behind many tokens from before."""
    rng, g = np.random.default_rng(dim), torch.Generator("cuda").manual_seed(dim)
    new = np.array([1] * 30 + [2 * size + 77] + [1] * 30)
    lengths = new + rng.integers(0, 3 * size, len(new))
    lengths[30] = new[30] + size - 5
    tables, codes, scales = cache_of(rng, code, lengths, 2, dim, size)
    x = [numbers_of(g, "bf16", int(new.sum()), 2, dim) for _ in range(2)]
    x[0][5:9] *= 64      # (their blocks grow)
    check_store("bf16", code, x, tables, codes, scales, lengths, np.concatenate([[0], np.cumsum(new)]), size, order=("head", "token")[size % 3 == 1])


def test_store_of_more_than_a_grid():
    """More heads and more places of requests' blocks than the grid has rows and columns: a workgroup takes several of both."""
    requests, heads = 4200, 2080
    rng, g = np.random.default_rng(9), torch.Generator("cuda").manual_seed(9)
    new, lengths = np.zeros(requests, int), np.zeros(requests, int)
    for b, n, m in [(0, 3, 11), (1, 1, 8), (700, 9, 9), (4090, 1, 2), (4097, 17, 30), (4199, 2, 9)]:
        new[b], lengths[b] = n, m
    tables, codes, scales = cache_of(rng, "e4m3", lengths, heads, 16, 8)
    x = [numbers_of(g, "bf16", int(new.sum()), heads, 16) for _ in range(2)]
    check_store("bf16", "e4m3", x, tables, codes, scales, lengths, np.concatenate([[0], np.cumsum(new)]), 8)


def test_store_past_the_caches():
    """More than 64 MiB of keys and values: they are read past the caches."""
    new, heads, dim, size = [9000, 7900, 500], 16, 64, 64
    g = torch.Generator("cuda").manual_seed(8)
    lengths = np.array(new) + [0, 1000, 70]
    tables, codes, scales = cache_of(np.random.default_rng(8), "int8", [0, 1000, 70], heads, dim, size, extra=300)
    free = np.setdiff1d(np.arange(len(codes[0])), tables)
    wide, at = np.full((3, 200), -1), 0
    for b, n in enumerate(lengths):
        held, need = -(-[0, 1000, 70][b] // size), -(-n // size)
        wide[b, :held] = tables[b, :held]
        wide[b, held:need] = free[at:at + need - held]
        at += need - held
    x = [numbers_of(g, "f16", sum(new), heads, dim) for _ in range(2)]
    check_store("f16", "int8", x, wide, codes, scales, lengths, np.concatenate([[0], np.cumsum(new)]), size, order="token")


# ---------------------------------------------------------------------------------------------------- read

def run_read(dtype, code, t, tables, codes, scales, lengths, starts, size, order="head", pad=0):
    blocks, heads, _, dim = codes[0].shape
    outs = [torch.full((t, heads * dim + pad), 5.0, dtype=DT[dtype], device="cuda") for _ in range(2)]
    with Plan.cache_read8(dtype, code, len(lengths), t, heads, dim, blocks, size, tables.shape[1], k_stride=heads * dim + pad, v_stride=heads * dim + pad,
                          **strides_of(order, heads, size, dim)) as plan:
        plan.launch([*(u8(placed(c, order)) for c in codes), *(torch.tensor(s, device="cuda") for s in scales), i32(tables), i32(lengths), i32(starts)], outs)
        torch.cuda.synchronize()
    assert all((o[:, heads * dim:] == 5).all() for o in outs)
    return [o[:, :heads * dim].reshape(t, heads, dim) for o in outs]


def check_read(dtype, code, t, tables, codes, scales, lengths, starts, size, powers=True, **kw):
    got = run_read(dtype, code, t, tables, codes, scales, lengths, starts, size, **kw)
    for k in range(2):
        want, mine = paged8.read(paged8.numbers(codes[k], scales[k], code), tables, lengths, starts, t)
        want[~mine] = 5.0
        rounded = f64(torch.tensor(want, device="cuda").to(DT[dtype]))
        room = 0.0 if powers else (U[dtype] + 2.0**-24) * np.abs(want) + 2.0**-25 * (dtype == "f16")
        within(f64(got[k]), rounded if powers else want, room, "kv"[k])


@pytest.mark.parametrize("code", CODES)
@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("shape", range(len(STORES)))
def test_read(dtype, code, shape):
    lengths, new, heads, dim, size = STORES[shape]
    powers = shape % 2 == 0
    tables, codes, scales = cache_of(np.random.default_rng(shape), code, lengths, heads, dim, size, "powers" if powers else "any")
    check_read(dtype, code, sum(new) + shape % 3, tables, codes, scales, lengths, np.concatenate([[0], np.cumsum(new)]), size, powers, order=("token", "head")[shape % 2],
               pad=(0, 8, 16)[shape % 3])


def test_read_of_odd_lengths_blocks_and_scales():
    tables, codes, scales = cache_of(np.random.default_rng(3), "e4m3", [64, 64, 64], 2, 64, 16)
    tables[0, 1], tables[1, 0], tables[2, 2] = -1, 2**31 - 1, len(codes[0])
    scales[0][tables[2, 0]], scales[1][tables[2, 1]] = 0.0, -np.inf
    codes[1][tables[0, 0], 1, 3, 7] = 0xFF      # NaN
    for t, lengths, starts in ((40, [37, 90, -4], [0, 12, 40, 40]), (90, [40, 40, 60], [0, 30, 30, 90]), (12, [30, 0, 8], [-5, 3, 8, 10]), (9, [5, 100000, 3], [0, 9, 9, 9])):
        check_read("bf16", "e4m3", t, tables, codes, scales, lengths, starts, 16)


def test_read_of_thousands_of_requests():
    rng = np.random.default_rng(7)
    new = rng.integers(0, 4, 5000)
    lengths = new + rng.integers(0, 30, 5000)
    tables, codes, scales = cache_of(rng, "int8", lengths, 1, 16, 8)
    check_read("f16", "int8", int(new.sum()) + 5, tables, codes, scales, lengths, np.concatenate([[0], np.cumsum(new)]), 8)


@pytest.mark.parametrize("code", CODES)
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_store_and_read(dtype, code):
    """Tokens stored in turns of 1, 5 and 40: what is read back is off by half a step of the codes, and by less than a step of the last scale in all where whole
    numbers' blocks have grown."""
    g, heads, dim, size, total = torch.Generator("cuda").manual_seed(2), 3, 64, 16, 100
    x = [numbers_of(g, dtype, total, heads, dim) for _ in range(2)]
    tables = np.arange(8)[None, ::-1].copy()
    codes, scales = [np.zeros((8, heads, size, dim), np.uint8) for _ in range(2)], [np.full((8, heads), np.nan, np.float32) for _ in range(2)]
    n, turns = 0, (1, 5, 40, 1, 1, 1, 5, 1, 40, 5)
    for m in turns:
        codes, scales = check_store(dtype, code, [a[n:n + m] for a in x], tables, codes, scales, [n + m], [0, m], size)
        n += m
    assert n == total
    got = run_read(dtype, code, n, tables, codes, scales, [n], [0, n], size)
    for k in range(2):
        want = f64(x[k])
        step = scales[k].astype(np.float64)[tables[0, np.arange(n) // size]][:, :, None]
        # e4m3: half of the 16th between neighbours, and of its least numbers half a step once more for every growth: less than one in all
        room = step if code == "int8" else 2.0**-4 * np.abs(want) + 2.0**-9 * step
        within(f64(got[k]), want, np.broadcast_to(room, want.shape), "kv"[k])


# ---------------------------------------------------------------------------------------------------- attention

def problem(seed, dtype, code, keys, new, q_heads, heads, dim, size, order="head", pad_rows=0, scale="powers"):
    rng, g = np.random.default_rng(seed), torch.Generator("cuda").manual_seed(seed)
    tables, codes, scales = cache_of(rng, code, keys, heads, dim, size, scale)
    q = torch.randn((sum(new) + pad_rows, q_heads, dim), device="cuda", generator=g).to(DT[dtype])
    return dict(dtype=dtype, code=code, q=q, tables=tables, codes=codes, scales=scales, lengths=np.array(keys), starts=np.concatenate([[0], np.cumsum(new)]).astype(int), order=order,
                size=size, heads=heads, scale=dim ** -0.5, powers=scale == "powers")


def plan_of(c, window=0, causal=True, max_new=0, lse=True, **kw):
    t, h, d = c["q"].shape
    return Plan.paged_attention8(c["dtype"], c["code"], len(c["lengths"]), t, h, c["heads"], d, len(c["codes"][0]), c["size"], c["tables"].shape[1], c["scale"], causal, window,
                                 max_new, lse, **strides_of(c["order"], c["heads"], c["size"], d), **kw)


def inputs(c):
    return [c["q"], *(u8(placed(x, c["order"])) for x in c["codes"]), *(torch.tensor(s, device="cuda") for s in c["scales"]), i32(c["tables"]), i32(c["lengths"]), i32(c["starts"])]


def buffers(c, nbytes, lse=True):
    t, h, d = c["q"].shape
    return ([torch.full((t, h, d), 3.0, dtype=DT[c["dtype"]], device="cuda")] + ([torch.full((t, h), 3.0, device="cuda")] if lse else []) +
            ([torch.full((nbytes,), 255, dtype=torch.uint8, device="cuda")] if nbytes else []))


def wanted(c, window=0, causal=True):
    k, v = (paged8.numbers(x, s, c["code"]) for x, s in zip(c["codes"], c["scales"]))
    return paged.attention(f64(c["q"]), k, v, c["tables"], c["lengths"], c["starts"], c["scale"], causal, window)


def check_out(c, outs, want, what=""):
    out, lse, weight, small, top = want
    u, d = U[c["dtype"]], c["q"].shape[2]
    none = np.isnan(lse)
    more = 0 if c["powers"] else u
    off = (d + 6) * 2.0**-24 * top + 6 * 2.0**-24 * top + 2.0**-20 + more * top
    room = (u + more + 2 * off[..., None]) * weight + 2.0**-25 * small + u * np.abs(out) + (2.0**-25 if c["dtype"] == "f16" else 0) * (1 if c["powers"] else 2)
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
    check_out(c, outs, wanted(c, window, causal), f"{c['dtype']} {c['code']} {tuple(c['q'].shape)} heads {c['heads']} lengths {c['lengths'].tolist()[:8]} block {c['size']} {c['order']} "
              f"{(window, causal, max_new)}")
    return outs


SHAPES = [   # keys, new tokens, q heads, key heads, block size
    ([1], [1], 1, 1, 16),
    ([5, 0, 17, 1], [1, 0, 1, 1], 8, 2, 16),
    ([300, 33, 32, 31, 129, 128, 127], [1] * 7, 8, 2, 16),
    ([64, 65, 0, 600], [4, 0, 0, 7], 12, 4, 32),
    ([200, 7, 1000], [200, 7, 3], 4, 4, 64),
    ([513, 90], [130, 1], 16, 2, 128),
    ([2000], [1], 32, 2, 16),
    ([70, 9, 40], [70, 5, 1], 6, 2, 8),
    ([900, 1500], [1, 2], 5, 1, 1024),
    ([257, 258], [33, 64], 3, 3, 8),
]


@pytest.mark.parametrize("code", CODES)
@pytest.mark.parametrize("dtype, dim", [("bf16", 128), ("f16", 64), ("bf16", 96), ("f16", 128), ("bf16", 32), ("f16", 96), ("f16", 32), ("bf16", 64)])
@pytest.mark.parametrize("shape", range(len(SHAPES)))
def test_attention(dtype, dim, code, shape):
    keys, new, q_heads, heads, size = SHAPES[shape]
    c = problem(shape, dtype, code, keys, new, q_heads, heads, dim, size, ("head", "token")[shape % 2], shape % 3)
    check_attention(c, max_new=(0, max(new))[shape % 2])


@pytest.mark.parametrize("code", CODES)
@pytest.mark.parametrize("dtype, dim", [("bf16", 128), ("f16", 64), ("f16", 128)])
@pytest.mark.parametrize("shape", range(len(SHAPES)))
def test_attention_with_any_scales(dtype, dim, code, shape):
    keys, new, q_heads, heads, size = SHAPES[shape]
    c = problem(shape, dtype, code, keys, new, q_heads, heads, dim, size, ("token", "head")[shape % 2], scale="any")
    check_attention(c, max_new=(0, max(new))[shape % 2])


@pytest.mark.parametrize("code", CODES)
@pytest.mark.parametrize("window, causal", [(1, True), (5, True), (64, True), (200, True), (0, False)])
@pytest.mark.parametrize("keys, new", [([300, 7, 64, 900], [1, 1, 2, 1]), ([300, 70, 900], [150, 70, 33])])
def test_attention_masks(code, window, causal, keys, new):
    for dtype, dim in (("bf16", 128), ("f16", 64)):
        check_attention(problem(window, dtype, code, keys, new, 4, 2, dim, 16), window, causal, max(new))


@pytest.mark.parametrize("q_heads, heads", [(64, 1), (24, 1), (7, 7)])
@pytest.mark.parametrize("requests", [3, 70, 130])
def test_attention_of_many_requests(q_heads, heads, requests):
    rng = np.random.default_rng(requests)
    keys, new = rng.integers(1, 700, requests), rng.choice([1, 1, 1, 2, 3], requests)
    keys = np.maximum(keys, new)
    check_attention(problem(1, "bf16", "e4m3", keys.tolist(), new.tolist(), q_heads, heads, 64, 16), max_new=3)


@pytest.mark.parametrize("requests, chunks", [(65, 3), (130, 65), (513, 5)])
def test_attention_of_chunks_among_many_requests(requests, chunks):
    rng = np.random.default_rng(requests)
    new = np.ones(requests, int)
    new[rng.permutation(requests)[:chunks]] = rng.integers(20, 60, chunks)
    keys = new + rng.integers(0, 200, requests)
    check_attention(problem(2, "f16", "int8", keys.tolist(), new.tolist(), 8, 2, 32, 16))


@pytest.mark.parametrize("table_keys, long", [(64, 60), (2048, 1900)])
def test_attention_of_thousands_of_requests(table_keys, long):
    """4200 requests, a few long ones behind the first 4096: whole tiles, and a line of units."""
    rng = np.random.default_rng(table_keys)
    keys = rng.integers(1, 40, 4200)
    keys[[3, 4100, 4199]] = long
    c = problem(13, "bf16", "e4m3", keys.tolist(), [1] * 4200, 4, 2, 32, 8)
    wide = np.full((4200, table_keys // 8), -1)
    wide[:, :c["tables"].shape[1]] = c["tables"][:, :wide.shape[1]]
    c["tables"] = wide
    check_attention(c, max_new=1)


@pytest.mark.parametrize("order", ["head", "token"])
@pytest.mark.parametrize("heads, dim", [(1, 64), (2, 32), (6, 96), (12, 128), (32, 32), (7, 96)])
def test_attention_of_sets_of_key_heads(heads, dim, order):
    check_attention(problem(3, "bf16", "int8", [1500, 40, 2100], [1, 2, 1], 2 * heads, heads, dim, 16, order), max_new=2)


@pytest.mark.parametrize("code", CODES)
@pytest.mark.parametrize("new", [1, 2, 60])
def test_attention_of_one_long_request(new, code):
    check_attention(problem(4, "bf16", code, [20000], [new], 4, 2, 128, 16), max_new=new)


@pytest.mark.parametrize("new", [1, 40])
def test_attention_bad_blocks(new):
    c = problem(5, "bf16", "e4m3", [200, 300], [new, new], 4, 2, 64, 16)
    c["tables"][0, 2], c["tables"][0, 5], c["tables"][1, :4] = -1, 2**31 - 1, len(c["codes"][0])
    check_attention(c)


@pytest.mark.parametrize("lengths, starts", [([-5, 500, 3], [0, 1, 2, 3]), ([40, 2**31 - 1, 20], [0, 30, 40, 60]), ([2, 1, 0], [0, 20, 40, 60]), ([64, 64, 64], [-7, 3, 40, 99])])
def test_attention_odd_lengths(lengths, starts):
    c = problem(6, "f16", "int8", [64, 64, 64], [20, 20, 20], 4, 2, 64, 16)
    table = c["tables"]
    table[table < 0] = 0      # (block 0: some request's, or nobody's)
    c["scales"] = [np.where(np.isnan(s), np.float32(2.0**-5), s) for s in c["scales"]]
    c["lengths"], c["starts"] = np.array(lengths), np.array(starts)
    check_attention(c)


@pytest.mark.parametrize("starts", [[0, 9, 0, 9], [9, 0, 9, 0], [5, 5, 1, 9]])
@pytest.mark.parametrize("max_new", [0, 1])
def test_attention_rows_of_several_requests(starts, max_new):
    """Undefined rows; the launch ends and rows of no request stay."""
    c = problem(7, "bf16", "e4m3", [20, 300, 64], [3, 3, 3], 8, 2, 64, 16)
    c["starts"] = np.array(starts)
    plan, nbytes = plan_of(c, max_new=max_new)
    with plan:
        outs = buffers(c, nbytes)
        plan.launch(inputs(c), outs)
        torch.cuda.synchronize()


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("new, keys", [(3, 40), (70, 200), (150, 150)])
def test_attention_codes_that_some_rows_do_not_see(dtype, new, keys):
    """NaN codes of values and keys in tokens that the first new tokens do not see yet: they reach the rows behind them alone."""
    for which in (0, 1):
        c = problem(8, dtype, "e4m3", [keys], [new], 4, 2, 64, 16)
        at = keys - 2
        c["codes"][which][c["tables"][0, at // 16], :, at % 16, 5] = 0xFF
        k, v = (paged8.numbers(x, s, "e4m3") for x, s in zip(c["codes"], c["scales"]))
        plan, nbytes = plan_of(c, max_new=new)
        with plan:
            outs = buffers(c, nbytes)
            plan.launch(inputs(c), outs)
            torch.cuda.synchronize()
        clean = dict(c, starts=np.array([0, new - 2]), lengths=np.array([keys - 2]), q=c["q"][:new - 2])
        check_out(clean, [o[:new - 2] for o in outs[:2]], wanted(clean), "rows before")
        tail = f64(outs[0])[new - 2:]
        assert np.isnan(tail if which == 0 else tail[:, :, 5]).all()
        if which == 1:
            keep = np.delete(np.arange(64), 5)
            assert np.isfinite(tail[:, :, keep]).all()


@pytest.mark.parametrize("code", CODES)
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("value", [float("nan"), float("inf"), 0.0])
@pytest.mark.parametrize("new, keys", [(3, 50), (70, 210), (150, 166)])
def test_attention_scales_that_some_rows_do_not_see(dtype, code, value, new, keys):
    """A scale that is none, in a block that the first new tokens do not see: they are as without it, those behind are not numbers (0: the keys' scores are 0)."""
    for which in (0, 1):
        c = problem(9, dtype, code, [keys], [new], 4, 2, 64, 16)
        first = (keys - 1) // 16 * 16      # the block's first key
        c["scales"][which][c["tables"][0, first // 16]] = value
        plan, nbytes = plan_of(c, max_new=new)
        with plan:
            outs = buffers(c, nbytes)
            plan.launch(inputs(c), outs)
            torch.cuda.synchronize()
        before = max(0, new - (keys - first))
        clean = dict(c, starts=np.array([0, before]), lengths=np.array([first]), q=c["q"][:before])
        if before:
            check_out(clean, [o[:before] for o in outs[:2]], wanted(clean), "rows before")
        tail = f64(outs[0])[before:]
        if np.isnan(value):
            assert np.isnan(tail).all()
        elif value == 0:
            rest = dict(c, q=c["q"][before:], starts=np.array([0, new - before]))
            check_out(rest, [o[before:] for o in outs[:2]], wanted(rest), "rows behind")


@pytest.mark.parametrize("code", CODES)
@pytest.mark.parametrize("new, keys", [(2, 100), (90, 300)])
def test_attention_in_fp16_of_numbers_beyond_its_range(code, new, keys):
    """Values of a block that only the last rows see are beyond fp16's numbers: infinities there, nothing elsewhere."""
    c = problem(10, "f16", code, [keys], [new], 4, 2, 64, 16)
    first = (keys - 1) // 16 * 16
    c["scales"][1][c["tables"][0, first // 16]] = 2.0**14
    page = c["codes"][1][c["tables"][0, first // 16]]
    page[:] = 0
    page[:, 0, ::2] = 0x48 if code == "e4m3" else 100      # 4 * 2^14, 100 * 2^14
    plan, nbytes = plan_of(c, max_new=new)
    with plan:
        outs = buffers(c, nbytes)
        plan.launch(inputs(c), outs)
        torch.cuda.synchronize()
    before = max(0, new - (keys - first))
    if before:
        clean = dict(c, starts=np.array([0, before]), lengths=np.array([first]), q=c["q"][:before])
        check_out(clean, [o[:before] for o in outs[:2]], wanted(clean), "rows before")
    tail = f64(outs[0])[before:]
    assert np.isfinite(tail[:, :, 1::2]).all() and (np.isposinf(tail[:, :, ::2]) | (tail[:, :, ::2] < 65520)).all() and not np.isnan(tail).any()


@pytest.mark.parametrize("new", [1, 60])
def test_attention_scores_of_any_size_and_sign(new):
    for scale in (0.0, -0.2, 40.0):
        c = problem(11, "bf16", "e4m3", [200, 90], [new, new], 4, 2, 64, 16)
        c["scale"] = scale
        check_attention(c)


def test_attention_of_parts_of_a_projection_and_twice_the_same():
    c = problem(12, "bf16", "int8", [130, 700], [40, 1], 4, 2, 128, 16)
    t, h, d = c["q"].shape
    row = (h + 4) * d
    wide = torch.zeros((t, row), dtype=torch.bfloat16, device="cuda")
    wide[:, :h * d] = c["q"].reshape(t, h * d)
    out = torch.full((t, h * d + 8), 3.0, dtype=torch.bfloat16, device="cuda")
    plan, nbytes = plan_of(c, q_stride=row, out_stride=h * d + 8, lse=False)
    with plan:
        ins, parts = inputs(c), buffers(c, nbytes, False)[1:]
        plan.launch([wide, *ins[1:]], [out, *parts])
        first = out.clone()
        for p in parts:
            p.fill_(255)
        plan.launch([wide, *ins[1:]], [out, *parts])
        torch.cuda.synchronize()
        assert torch.equal(out, first) and (out[:, h * d:] == 3).all()
    check_out(c, [out[:, :h * d].reshape(t, h, d)], wanted(c))


def test_behind_32_bits():
    """Blocks more than 2^32 codes behind the cache's first one: stored, read and attended to; scales more than 2^31 numbers are not reached by any cache here."""
    heads, dim, size, blocks = 8, 128, 16, 300000      # 4.9e9 codes
    free = torch.cuda.mem_get_info()[0]
    assert free > 14 << 30
    caches = [torch.full((blocks, heads, size, dim), 0x7F, dtype=torch.uint8, device="cuda") for _ in range(2)]
    scales = [torch.full((blocks, heads), float("nan"), device="cuda") for _ in range(2)]
    pages = [blocks - 1, 5, blocks - 7, 262144, 262143]
    n, g = 5 * size - 3, torch.Generator("cuda").manual_seed(1)
    tables, lengths, starts = np.array([pages]), [n], [0, n]
    x = [torch.randn((n, heads, dim), device="cuda", generator=g).to(torch.bfloat16) for _ in range(2)]
    q = torch.randn((n, 2 * heads, dim), device="cuda", generator=g).to(torch.bfloat16)
    t, le, st = i32(tables), i32(lengths), i32(starts)
    kw = dict(dtype="bf16", code="e4m3", requests=1, tokens=n, kv_heads=heads, head_dim=dim, blocks=blocks, block_size=size, table_blocks=5)
    with Plan.cache_store8(**kw) as plan:
        plan.launch([*x, t, le, st], [*caches, *scales])
    back = [torch.empty_like(a) for a in x]
    with Plan.cache_read8(**kw) as plan:
        plan.launch([*caches, *scales, t, le, st], back)
    small = [c[pages].cpu().numpy() for c in caches], [s[pages].cpu().numpy() for s in scales]
    here = np.arange(5)[None]
    c = dict(dtype="bf16", code="e4m3", q=q, tables=here, codes=small[0], scales=small[1], lengths=np.array(lengths), starts=np.array(starts), order="head", size=size, heads=heads,
             scale=0.1, powers=True)
    for k in range(2):
        empty = np.full((5, heads, size, dim), 0x7F, np.uint8), np.full((5, heads), np.nan)
        want = paged8.store(f64(x[k]), *empty, here, lengths, starts, "e4m3", "bf16")
        assert np.array_equal(small[0][k], want[0]) and np.array_equal(small[1][k], want[1].astype(np.float32), equal_nan=True)
        assert np.array_equal(f64(back[k]), paged8.read(paged8.numbers(*want, "e4m3"), here, lengths, starts, n)[0])
    for rows in (n, 1):      # tiles of many rows, and of few
        plan, nbytes = Plan.paged_attention8(q_heads=2 * heads, scale=0.1, lse=True, max_new=rows, **dict(kw, tokens=rows))
        c["q"], c["starts"] = q[:rows], np.array([0, rows])
        with plan:
            outs = buffers(c, nbytes)
            plan.launch([c["q"], *caches, *scales, t, le, i32([0, rows])], outs)
            torch.cuda.synchronize()
        check_out(c, outs, wanted(c))


# ---------------------------------------------------------------------------------------------------- together

class Server:
    """Block tables, rotary positions, the store and attention of steps of a few requests, as a program that serves a model makes them."""

    def __init__(self, code, requests=3, most=24, q_heads=4, heads=2, dim=64, size=16, blocks=40, width=8):
        self.code, self.requests, self.most, self.q_heads, self.heads, self.dim, self.size, self.blocks, self.width = code, requests, most, q_heads, heads, dim, size, blocks, width
        e = lambda *n, **kw: torch.zeros(n, device="cuda", **kw)  # noqa: E731
        i = lambda *n: torch.zeros(n, dtype=torch.int32, device="cuda")  # noqa: E731
        row = (q_heads + 2 * heads) * dim
        self.qkv = e(most, row, dtype=torch.bfloat16)
        self.q, self.k, self.v = (x.unflatten(1, (-1, dim)) for x in self.qkv.split([q_heads * dim, heads * dim, heads * dim], 1))
        self.cached, self.fresh, self.free = i(requests), i(requests), torch.arange(blocks - 1, -1, -1, dtype=torch.int32, device="cuda")
        self.table, self.lengths, self.starts, self.positions, self.slots, self.taken = i(requests, width).fill_(-1), i(requests), i(requests + 1), i(most), i(most), i(2)
        self.frequencies = torch.tensor(fs_rotary_frequencies(dim), dtype=torch.float64, device="cuda")
        self.q_turned, self.k_turned = e(most, q_heads, dim, dtype=torch.bfloat16), e(most, heads, dim, dtype=torch.bfloat16)
        self.caches = [torch.full((blocks, heads, size, dim), 0x7F, dtype=torch.uint8, device="cuda") for _ in range(2)]
        self.scales = [torch.full((blocks, heads), float("nan"), device="cuda") for _ in range(2)]
        self.out = e(most, q_heads, dim, dtype=torch.bfloat16)
        kw = dict(dtype="bf16", code=code, requests=requests, tokens=most, kv_heads=heads, head_dim=dim, blocks=blocks, block_size=size, table_blocks=width)
        self.tables_plan = Plan.block_tables(requests, most, blocks, size, width, blocks)
        self.rotary_plan = Plan.rotary("bf16", most, q_heads, heads, dim, q_stride=row, k_stride=row)
        self.store_plan = Plan.cache_store8(**kw, v_stride=row)
        self.attend_plan, nbytes = Plan.paged_attention8(q_heads=q_heads, scale=dim ** -0.5, **kw)
        self.partials = [torch.empty(nbytes, dtype=torch.uint8, device="cuda")] if nbytes else []

    def step(self):
        self.tables_plan.launch([self.cached, self.fresh, self.free], [self.table, self.lengths, self.starts, self.positions, self.slots, self.taken])
        self.rotary_plan.launch([self.q, self.k, self.positions, self.frequencies], [self.q_turned, self.k_turned])
        self.store_plan.launch([self.k_turned, self.v, self.table, self.lengths, self.starts], [*self.caches, *self.scales])
        self.attend_plan.launch([self.q_turned, *self.caches, *self.scales, self.table, self.lengths, self.starts], [self.out, *self.partials])

    def state(self):
        return [self.table, self.lengths, *self.caches, *self.scales, self.out]


def fill(server, rng, fresh):
    """The next step's lengths and numbers; the free list without what the last step took."""
    taken = int(server.taken[0])
    if taken:
        server.free.copy_(torch.cat([server.free[taken:], torch.full((taken,), -1, dtype=torch.int32, device="cuda")]))
    server.cached.copy_(server.lengths)
    server.fresh.copy_(i32(fresh))
    server.qkv.copy_(torch.as_tensor(rng.standard_normal(server.qkv.shape) * 2.0 ** rng.integers(-2, 3), dtype=torch.float32))


STEPS = [[7, 0, 12], [1, 5, 1], [1, 1, 1], [0, 14, 1], [1, 1, 1], [9, 1, 9], [1, 1, 1]]


@pytest.mark.parametrize("code", CODES)
def test_steps_of_a_server(code):
    rng, s = np.random.default_rng(0), Server(code)
    codes, scales = [np.full(c.shape, 0x7F, np.uint8) for c in s.caches], [np.full(x.shape, np.nan) for x in s.scales]
    for fresh in STEPS:
        fill(s, rng, fresh)
        s.step()
        torch.cuda.synchronize()
        n = sum(fresh)
        tables, lengths, starts = (t.cpu().numpy() for t in (s.table, s.lengths, s.starts))
        assert starts[-1] == n
        freqs = fs_rotary_frequencies(s.dim)
        want = paged.rotary(f64(s.k)[:n], s.positions.cpu().numpy()[:n], freqs)
        within(f64(s.k_turned)[:n], want, rotary_bound(f64(s.k)[:n], want, freqs, False, 1.0, "bf16"), "k turned")
        for k, x in enumerate((s.k_turned, s.v)):
            codes[k], scales[k] = paged8.store(f64(x), codes[k], scales[k], tables, lengths, starts, code, "bf16")
            assert np.array_equal(s.caches[k].cpu().numpy(), codes[k]) and np.array_equal(s.scales[k].cpu().numpy(), scales[k].astype(np.float32), equal_nan=True)
        c = dict(dtype="bf16", code=code, q=s.q_turned, tables=tables, codes=codes, scales=scales, lengths=lengths, starts=starts, scale=s.dim ** -0.5, powers=True)
        out, lse, *_ = want = wanted(c)
        got = s.out.clone()
        got[n:] = 3.0
        check_out(c, [got], want)


@pytest.mark.parametrize("code", CODES)
def test_steps_in_a_graph(code):
    """Captured once and replayed with other lengths, eager steps of another server's between the replays; every replay against its eager twin."""
    a, b, other = Server(code), Server(code), Server(code)
    ra, rb, ro = (np.random.default_rng(3) for _ in range(3))
    graph = None
    for i, fresh in enumerate(STEPS):
        fill(a, ra, fresh)
        a.step()
        fill(b, rb, fresh)
        if i == 0:
            b.step()
        elif graph is None:
            stream = torch.cuda.Stream()
            stream.wait_stream(torch.cuda.current_stream())
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.stream(stream), torch.cuda.graph(graph, stream=stream):
                b.step()
            torch.cuda.current_stream().wait_stream(stream)
            graph.replay()
        else:
            graph.replay()
        fill(other, ro, fresh[::-1])
        other.step()
        torch.cuda.synchronize()
        n = sum(fresh)
        for x, y in zip(a.state()[:-1], b.state()[:-1]):
            assert torch.equal(x.nan_to_num(nan=-1.0) if x.is_floating_point() else x, y.nan_to_num(nan=-1.0) if y.is_floating_point() else y)
        assert torch.equal(a.out[:n], b.out[:n])


def test_two_launches_of_a_plan_at_once():
    """One plan on two streams, partial results of their own."""
    c, d = (problem(s, "bf16", "e4m3", [9000, 40, 5000], [1, 1, 2], 8, 2, 128, 16) for s in (20, 21))
    plan, nbytes = plan_of(c, max_new=2)
    with plan:
        ins, outs, streams = [inputs(c), inputs(d)], [buffers(c, nbytes), buffers(d, nbytes)], [torch.cuda.Stream() for _ in range(2)]
        torch.cuda.synchronize()
        for _ in range(5):
            for k in range(2):
                with torch.cuda.stream(streams[k]):
                    plan.launch(ins[k], outs[k])
        torch.cuda.synchronize()
    check_out(c, outs[0], wanted(c))
    check_out(d, outs[1], wanted(d))
