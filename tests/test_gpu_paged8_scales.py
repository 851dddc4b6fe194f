"""Attention over the paged cache in 8 bits: scales of blocks that not every row sees, scales that are none, numbers beyond fp16's range, rows of nobody.  Tolerances as in
test_gpu_paged8.py.

The first tests are of steps of the few-rows kernel whose keys not every row sees and which have another step behind them, in front of a window and around blocks that are
none: the scales of the two steps must not be taken for each other's.  A step is 32 or 64 keys of each of four or eight wavefronts, so a wavefront has a step behind a masked one in windows of 256 keys and more.
"""
import numpy as np
import pytest
import torch

from oracle import paged8
from test_gpu_paged import f64
from test_gpu_paged8 import CODES, buffers, check_attention, check_out, inputs, plan_of, problem, wanted

pytestmark = pytest.mark.gpu

SIZE = 16
CASES = [   # window, new tokens, query heads, key heads, head dim, keys of the shortest request, requests, new tokens of one more request
    (512, 1, 4, 2, 64, 700, 32, 0),        # whole tiles, eight wavefronts
    (512, 3, 4, 2, 128, 700, 32, 0),
    (256, 1, 4, 2, 64, 300, 160, 0),       # ... four
    (256, 3, 4, 2, 32, 300, 160, 0),
    (512, 1, 4, 2, 128, 1500, 32, 0),      # a line of units
    (512, 3, 4, 2, 96, 1500, 32, 0),
    (1000, 3, 16, 2, 64, 1500, 32, 0),     # two tiles of rows, two steps in LDS
    (1000, 3, 16, 2, 96, 1500, 32, 0),
    (256, 1, 4, 2, 64, 600, 32, 60),       # among chunks
    (256, 3, 4, 2, 128, 600, 32, 60),
    (512, 1, 20, 1, 64, 600, 32, 60),
]

EVERY = [("f16", c) for c in CASES] + [("bf16", c) for c in (CASES[0], CASES[3], CASES[7], CASES[8])]      # (bf16 takes the scales of values another way, into the weights)


def windowed(case, dtype, code):
    """Requests of every remainder by 32, and block 0 nobody's."""
    window, new, q_heads, heads, dim, keys, requests, chunk = case
    lengths, fresh = [keys + b for b in range(32)] * (requests // 32), [new] * requests
    if chunk:
        lengths, fresh = lengths + [keys + 77], fresh + [chunk]
    c = problem(window + new, dtype, code, lengths, fresh, q_heads, heads, dim, SIZE, ("head", "token")[new == 3])
    block_0_of_nobody(c)
    return c, window, 0 if chunk else new


def block_0_of_nobody(c):
    spare = np.setdiff1d(np.arange(len(c["codes"][0])), c["tables"])[0]
    for a in (*c["codes"], *c["scales"]):
        a[[0, spare]] = a[[spare, 0]]
    c["tables"][c["tables"] == 0] = spare


@pytest.mark.parametrize("value", [float("nan"), 2.0**14])
@pytest.mark.parametrize("code", CODES)
@pytest.mark.parametrize("dtype, case", EVERY, ids=str)
def test_window_behind_which_block_0_is_nobodys(dtype, case, code, value):
    """Lanes without a key have the scale of block 0."""
    c, window, max_new = windowed(case, dtype, code)
    for s in c["scales"]:
        s[0] = value
    check_attention(c, window, True, max_new)


@pytest.mark.parametrize("value", [float("nan"), float("inf")])
@pytest.mark.parametrize("code", CODES)
@pytest.mark.parametrize("dtype, case", EVERY, ids=str)
def test_scale_that_is_none_in_a_windows_first_block(dtype, case, code, value):
    """Values of the block with the first key that a request's last token sees, finite ones behind it: no result of the request is a number."""
    c, window, max_new = windowed(case, dtype, code)
    for b, n in enumerate(c["lengths"]):
        c["scales"][1][c["tables"][b, (n - window) // SIZE]] = value
    plan, nbytes = plan_of(c, window, True, max_new)
    with plan:
        outs = buffers(c, nbytes)
        plan.launch(inputs(c), outs)
        torch.cuda.synchronize()
    got = f64(outs[0])
    assert np.isnan(got).all() if np.isnan(value) else not np.isfinite(got).any()


@pytest.mark.parametrize("code", CODES)
@pytest.mark.parametrize("dtype, case", EVERY, ids=str)
def test_large_scales_behind_a_windows_first_keys(dtype, case, code):
    """Large codes of values under a small scale in the window's first half, small codes under a scale in the second half with which the large ones would leave
    fp16's range."""
    c, window, max_new = windowed(case, dtype, code)
    rng = np.random.default_rng(1)
    most, scale, small = (448, 2.0**8, 1) if code == "e4m3" else (127, 2.0**10, 8)
    for b, n in enumerate(c["lengths"]):
        for j in range(-(-int(n) // SIZE)):
            page = c["tables"][b, j]
            m = min(SIZE, int(n) - j * SIZE)
            shape = c["codes"][1][page, :, :m].shape
            behind = j * SIZE >= n - window // 2
            x = rng.uniform(-small, small, shape) if behind else rng.uniform(0.6 * most, most, shape) * rng.choice([-1, 1], shape)
            c["codes"][1][page, :, :m] = paged8.coded(x, code)
            c["scales"][1][page] = scale if behind else 2.0**-6
    check_attention(c, window, True, max_new)


@pytest.mark.parametrize("value", [float("nan"), 2.0**14])
@pytest.mark.parametrize("code", CODES)
@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("new, q_heads, heads, dim, keys, window, chunk", [
    (1, 4, 2, 128, 3000, 0, 0), (3, 16, 2, 64, 3000, 0, 0), (2, 4, 2, 64, 900, 0, 0), (1, 4, 2, 96, 3000, 1000, 0), (1, 4, 2, 64, 900, 0, 50), (1, 20, 1, 32, 900, 0, 50)])
def test_blocks_that_are_none_in_the_middle(new, q_heads, heads, dim, keys, window, chunk, dtype, code, value):
    """A sixth of all blocks: their lanes have the scale of block 0."""
    lengths, fresh = [keys, keys - 13, keys - 300, keys // 2], [new] * 4
    if chunk:
        lengths, fresh = lengths + [keys - 50], fresh + [chunk]
    c = problem(keys + new, dtype, code, lengths, fresh, q_heads, heads, dim, SIZE)
    block_0_of_nobody(c)
    for s in c["scales"]:
        s[0] = value
    rng = np.random.default_rng(keys)
    c["tables"] = np.where(rng.random(c["tables"].shape) < 1 / 6, rng.choice([-1, len(c["codes"][0]), 2**31 - 1], c["tables"].shape), c["tables"])
    check_attention(c, window, True, 0 if chunk else new)


def launched(c, **kw):
    plan, nbytes = plan_of(c, **kw)
    with plan:
        outs = buffers(c, nbytes)
        plan.launch(inputs(c), outs)
        torch.cuda.synchronize()
    return outs


@pytest.mark.parametrize("code", CODES)
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("which", [0, 1], ids=["keys", "values"])
@pytest.mark.parametrize("new, keys", [(1, 30), (3, 50), (2, 900), (70, 210), (150, 166)])
def test_infinite_scale_of_the_last_block(dtype, code, which, new, keys):
    """Rows that see it: not a number wherever the definition has none there, and an infinity where it has one (or NaN, where the weight is rounded to 0).  Rows before: as
    without it."""
    c = problem(9, dtype, code, [keys], [new], 4, 2, 64, 16)
    first = (keys - 1) // 16 * 16
    c["scales"][which][c["tables"][0, first // 16]] = np.inf
    outs = launched(c, max_new=new)
    before = max(0, new - (keys - first))
    if before:
        clean = dict(c, starts=np.array([0, before]), lengths=np.array([first]), q=c["q"][:before])
        check_out(clean, [o[:before] for o in outs[:2]], wanted(clean), "rows before")
    with np.errstate(invalid="ignore"):
        want = wanted(c)[0][before:]
    got, none = f64(outs[0])[before:], ~np.isfinite(want)
    assert none.all() and not np.isfinite(got).any()
    inf = np.isinf(want)
    assert (np.isnan(got[inf]) | (got[inf] == want[inf])).all()


@pytest.mark.parametrize("code", CODES)
@pytest.mark.parametrize("new, keys", [(1, 30), (2, 100), (3, 900), (90, 300)])
def test_values_beyond_fp16_are_infinite_or_right(code, new, keys):
    """One key of the last block has values of 4 * 2^14 or 100 * 2^14 in every other column: an infinity there, or the sum that the numbers have; elsewhere nothing."""
    c = problem(10, "f16", code, [keys], [new], 4, 2, 64, 16)
    first = (keys - 1) // 16 * 16
    last = c["tables"][0, first // 16]
    c["scales"][1][last] = 2.0**14
    c["codes"][1][last] = 0
    c["codes"][1][last][:, 0, ::2] = 0x48 if code == "e4m3" else 100
    outs, want = launched(c, max_new=new), wanted(c)
    got, exact, weight, small = f64(outs[0]), want[0], want[2], want[3]
    before = max(0, new - (keys - first))
    off = (64 + 12) * 2.0**-24 * want[4] + 2.0**-20
    room = (2.0**-11 + 2 * off[..., None]) * weight + 2.0**-25 * small + 2.0**-11 * np.abs(exact) + 2.0**-25
    right = (np.abs(got - exact) <= room) | (np.isposinf(got) & (exact + room >= 65520))
    assert right[:before].all() and right[:, :, 1::2].all()
    assert (right | np.isposinf(got)).all()


@pytest.mark.parametrize("max_new", [0, 1])
@pytest.mark.parametrize("starts, nobody", [([5, 5, 1, 9], [0]), ([3, 1, 5, 6], [0, 6, 7, 8]), ([2, 4, 4, 7], [0, 1, 7, 8])])
def test_rows_of_no_request_stay(starts, nobody, max_new):
    c = problem(7, "bf16", "e4m3", [20, 300, 64], [3, 3, 3], 8, 2, 64, 16)
    c["starts"] = np.array(starts)
    outs = launched(c, max_new=max_new)
    assert (outs[0][nobody] == 3).all() and (outs[1][nobody] == 3).all()
    others = np.setdiff1d(np.arange(9), nobody)
    assert (outs[0][others] != 3).any(dim=2).all()


@pytest.mark.parametrize("code", CODES)
@pytest.mark.parametrize("dtype, powers", [("f16", (-20, -14)), ("f16", (-32, -20)), ("bf16", (-100, -90)), ("bf16", (-126, -117))])
@pytest.mark.parametrize("new, keys, dim", [(1, 300, 128), (3, 900, 64), (90, 300, 128), (40, 100, 32)])
def test_small_scales(dtype, powers, code, new, keys, dim):
    """Powers of two with which fp16 does not hold all that the codes stand for: keys and values may be rounded to it, 2^-25 of each at its end.  And the least that a
    store makes, in bf16."""
    c = problem(21, dtype, code, [keys, keys // 2], [new, 1], 4, 2, dim, 16)
    rng = np.random.default_rng(keys)
    for s in c["scales"]:
        there = np.isfinite(s)
        s[there] = 2.0 ** rng.integers(*powers, there.sum())
    c["powers"] = dtype == "bf16"
    outs, want = launched(c, max_new=new), list(wanted(c))
    if dtype == "f16":      # a score, by as much of every key
        want[4] = want[4] + c["scale"] * np.abs(f64(c["q"])).sum(2) * 2.0**-25 / 2.0**-11
    check_out(c, outs, want)
