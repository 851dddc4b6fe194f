"""The store into a paged cache in 8 bits, bit by bit against its definition (oracle/paged8.py), where a scale is not the one that the store itself would have given the
block: numbers at the end of the type's range, and codes from before written again."""
import numpy as np
import pytest
import torch

from oracle import paged8
from test_gpu_paged import DT
from test_gpu_paged8 import CODES, check_store, run_read

pytestmark = pytest.mark.gpu

LARGE = {"f16": [65504.0, 65024.0, 64992.0, 64544.0, 64512.0, 63520.0, 61472.0, 61440.0, 40000.0],
         "bf16": [m * 2.0**127 for m in (1.9921875, 1.984375, 1.9765625, 1.96875, 1.890625, 1.875, 1.25)]}
LARGE["f32"] = [float(np.finfo(np.float32).max), *LARGE["bf16"]]
POWERS = {"f16": [8, 9, 10, 11, 12, 14, 15, 16, 17, 20, 21, 22, 23, 25, 26], "bf16": range(119, 128), "f32": range(119, 128)}


@pytest.mark.parametrize("code", CODES)
@pytest.mark.parametrize("dtype", ["f16", "bf16", "f32"])
@pytest.mark.parametrize("held", [0, 3])
def test_store_cuts_by_the_scale_of_the_block(dtype, code, held):
    """Behind tokens under larger scales, and in new blocks: what is read back is finite, and nothing is cut whose code stands for a finite number."""
    pairs = [(m, p) for m in LARGE[dtype] for p in (POWERS[dtype] if held else [0])]
    heads, dim, rng = len(pairs), 64, np.random.default_rng(held)
    x = [np.empty((2, heads, dim)) for _ in range(2)]
    tables, codes, scales = np.array([[1]]), [np.zeros((2, heads, 8, dim), np.uint8) for _ in range(2)], [np.full((2, heads), np.nan, np.float32) for _ in range(2)]
    for h, (most, power) in enumerate(pairs):
        for k in range(2):
            x[k][:, h] = most * rng.uniform(0.45, 1, (2, dim)) * rng.choice([-1, 1], (2, dim))
            x[k][:, h, 1::5] = most * (1 - rng.integers(0, 40, (2, 13)) * 2.0**-11)
            x[k][1, h, 3 * k] = (-1)**k * most
            codes[k][1, h, :held] = paged8.coded(rng.uniform(-100, 100, (held, dim)), code)
            scales[k][1, h] = 2.0**power
    x = [torch.tensor(a, device="cuda").to(DT[dtype]) for a in x]
    assert all(torch.isfinite(a).all() for a in x)
    got_codes, got_scales = check_store(dtype, code, x, tables, codes, scales, [held + 2], [0, 2], 8)
    assert all(torch.isfinite(r).all() for r in run_read(dtype, code, 2, tables, got_codes, got_scales, [held + 2], [0, 2], 8))


def near_ties(code):
    """Codes z and scales s, in 24 bits, for which z * s is next to the middle of two codes and in fp32 that middle: to the even one of the two it would be
    rounded, not to the nearest."""
    grid = paged8.E4M3[:127] if code == "e4m3" else np.arange(128.0)
    middles, found = (grid[:-1] + grid[1:]) / 2, []
    for z in grid[1:]:
        s = (middles / z).astype(np.float32)
        twice = (z.astype(np.float32) * s).astype(np.float64)
        near = (s > 0.5) & (s < 1) & (twice == middles) & (z * s.astype(np.float64) != middles)
        found += [(z, t) for t, m in zip(s[near], middles[near]) if paged8.coded([z * float(t)], code) != paged8.coded([m], code)]
    return found


@pytest.mark.parametrize("code", CODES)
@pytest.mark.parametrize("exponent", [0, -9])
def test_codes_written_again_are_rounded_once(code, exponent):
    """Scales of others from before, no powers of two: 0.7 times the code 5, for one, is above 3.5 in fp32's number next to 0.7, and their product in fp32 is 3.5."""
    found = near_ties(code)
    assert len(found) > 100
    heads, dim = len(found), 16
    tables, codes, scales = np.array([[1]]), [np.zeros((2, heads, 8, dim), np.uint8) for _ in range(2)], [np.ones((2, heads), np.float32) for _ in range(2)]
    for h, (z, s) in enumerate(found):
        codes[0][1, h, :3] = paged8.coded(np.array([1, -1, 0.5, 0] * 4) * z, code)
        codes[1][1, h, :3] = paged8.coded(np.full(dim, -z), code)
        for k in range(2):
            scales[k][1, h] = np.ldexp(s, exponent)
    x = [torch.full((1, heads, dim), 0.25 * 2.0**exponent, device="cuda") for _ in range(2)]
    check_store("f32", code, x, tables, codes, scales, [4], [0, 1], 8)
