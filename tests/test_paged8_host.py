"""The paged cache in 8 bits without a GPU: refusals of plans and launches, what plans report, and the oracle's own definitions."""
import ctypes as C

import numpy as np
import pytest
import torch

from oracle import paged8
from paper_1911_11576_amd import FsError, Plan, binding
from test_paged_host import check_launch_arguments, refused

CACHE = dict(dtype="bf16", code="e4m3", requests=2, tokens=3, kv_heads=2, head_dim=64, blocks=9, block_size=16, table_blocks=4)
ATTENTION = dict(CACHE, q_heads=4, scale=0.125)
INVALID, UNSUPPORTED = binding.FS_ERR_INVALID, binding.FS_ERR_UNSUPPORTED


@pytest.mark.parametrize("make", [Plan.cache_store8, Plan.cache_read8])
@pytest.mark.parametrize("change, status, text", [
    (dict(requests=-1), INVALID, "requests"), (dict(requests=65537), INVALID, "requests"), (dict(tokens=-1), INVALID, "tokens"), (dict(tokens=2**30 + 1), INVALID, "tokens"),
    (dict(kv_heads=0), INVALID, "kv_heads"), (dict(kv_heads=65537), INVALID, "kv_heads"), (dict(head_dim=0), INVALID, "head_dim"), (dict(blocks=-1), INVALID, "blocks"),
    (dict(table_blocks=-1), INVALID, "blocks"), (dict(block_size=12), INVALID, "power of two"), (dict(block_size=2048), INVALID, "power of two"),
    (dict(blocks=2**28), INVALID, "2^31"), (dict(table_blocks=2**28), INVALID, "2^31"), (dict(k_stride=127), INVALID, "k_stride"), (dict(v_stride=-16), INVALID, "v_stride"),
    (dict(slot_stride=-16), INVALID, "negative"), (dict(slot_stride=32, head_stride=1024, block_stride=4096), INVALID, "overlap"),
    (dict(head_dim=24), UNSUPPORTED, "head_dim"), (dict(head_dim=528), UNSUPPORTED, "head_dim"), (dict(k_stride=132), UNSUPPORTED, "16 bytes"),
    (dict(dtype="f32", v_stride=130), UNSUPPORTED, "16 bytes"), (dict(block_size=4), UNSUPPORTED, "block_size"),
    (dict(slot_stride=136, head_stride=64, block_stride=4352), UNSUPPORTED, "multiples of 16")])
def test_cache_refused(make, change, status, text):
    refused(make, status, text, **dict(CACHE, **change))


@pytest.mark.parametrize("change, status, text", [
    (dict(requests=-1), INVALID, "requests"), (dict(tokens=2**30), INVALID, "tokens"), (dict(q_heads=3), INVALID, "q_heads"), (dict(kv_heads=0), INVALID, "kv_heads"),
    (dict(window=-1), INVALID, "window"), (dict(window=5, causal=False), INVALID, "window"), (dict(causal=2), INVALID, "0 or 1"), (dict(max_new=-1), INVALID, "max_new"),
    (dict(scale=float("nan")), INVALID, "scale"), (dict(q_stride=128), INVALID, "q_stride"), (dict(block_size=12), INVALID, "power of two"),
    (dict(dtype="f32"), UNSUPPORTED, "f16 and bf16"), (dict(head_dim=48), UNSUPPORTED, "head_dim"), (dict(head_dim=256), UNSUPPORTED, "head_dim"),
    (dict(q_stride=258), UNSUPPORTED, "multiples of 8"), (dict(block_size=4), UNSUPPORTED, "block_size"),
    (dict(slot_stride=136, head_stride=64, block_stride=4352), UNSUPPORTED, "multiples of 16")])
def test_attention_refused(change, status, text):
    refused(Plan.paged_attention8, status, text, **dict(ATTENTION, **change))


def test_attention_of_more_tiles_than_a_grid_has():
    change = dict(requests=32760, tokens=100, q_heads=512, kv_heads=512, max_new=0)
    Plan.paged_attention8(**dict(ATTENTION, **change))[0].close()
    refused(Plan.paged_attention8, UNSUPPORTED, "too many tiles", **dict(ATTENTION, **dict(change, requests=32768)))


def test_null_arguments_and_unknown_codes():
    L, out, n = binding.lib(), C.c_void_p(), C.c_int64()
    for create in (L.fs_plan_create_cache_store8, L.fs_plan_create_cache_read8):
        assert create(None, C.byref(out)) == INVALID
        d = binding.fs_cache8_desc(2, 0, 1, 1, 1, 64, 1, 16, 1, 0, 0, 0, 0, 0, 0)
        assert create(C.byref(d), None) == INVALID
        for field, value in (("reserved", 1), ("code", 2), ("code", -1), ("dtype", 3)):
            bad = binding.fs_cache8_desc.from_buffer_copy(d)
            setattr(bad, field, value)
            assert create(C.byref(bad), C.byref(out)) == INVALID and not out.value
    assert L.fs_plan_create_paged_attention8(None, C.byref(n), C.byref(out)) == INVALID
    d = binding.fs_paged_attention8_desc(2, 0, 1, 1, 1, 1, 64, 1, 16, 1, 1, 0, 0, 0, 0, 0, 0, 0, 0, 0.1)
    assert L.fs_plan_create_paged_attention8(C.byref(d), None, C.byref(out)) == INVALID and not out.value
    assert L.fs_plan_create_paged_attention8(C.byref(d), C.byref(n), None) == INVALID
    d.code = 2
    assert L.fs_plan_create_paged_attention8(C.byref(d), C.byref(n), C.byref(out)) == INVALID and not out.value
    with pytest.raises(KeyError):
        Plan.cache_store8(**dict(CACHE, code="e5m2"))


def test_launch_arguments():
    with Plan.cache_store8(**CACHE) as p:
        check_launch_arguments(p, 5, 4)
    with Plan.cache_read8(**CACHE) as p:
        check_launch_arguments(p, 7, 2)
    plan, nbytes = Plan.paged_attention8(**ATTENTION, lse=True)
    with plan:
        check_launch_arguments(plan, 8, 2 + (nbytes > 0))


@pytest.mark.parametrize("none", [dict(tokens=0), dict(requests=0)])
def test_nothing_to_do_launches_nothing(none):
    with Plan.cache_store8(**dict(CACHE, **none)) as p:
        p.launch([0] * 5, [0] * 4, 0)
        p.launch_static([0] * 5, [0] * 4, 0)
    with Plan.cache_read8(**dict(CACHE, **none)) as p:
        p.launch([0] * 7, [0] * 2, 0)
    plan, nbytes = Plan.paged_attention8(**dict(ATTENTION, **none))
    with plan:
        plan.launch([1 << 20 if "requests" in none else 0] + [0] * 7, [1 << 21 if "requests" in none else 0] + [0] * (nbytes > 0), 0)


def test_plans_report():
    with Plan.cache_store8(**CACHE) as p:
        assert p.info()["schedule"] == "cache_store8" and p.info()["n_kernels"] == 1 and p.info()["workspace_bytes"] == 0 and "cache_store8" in p.describe()
        assert p.info()["algorithmic_bytes"] == 2 * 3 * 128 * 3 + 8 * 4 * 2 + 4 * (4 + 4)
    with Plan.cache_read8(**CACHE) as p:
        assert p.info()["schedule"] == "cache_read8" and "cache_read8" in p.describe()
    plan, _ = Plan.paged_attention8(**ATTENTION)
    with plan:
        assert plan.info()["schedule"] == "paged_attention8" and plan.info()["algorithmic_bytes"] > 0 and "paged_attention8" in plan.describe()


def test_oracle_codes():
    every = np.arange(256, dtype=np.uint8)
    want = torch.from_numpy(every).view(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(paged8.values(every, "e4m3"), want, equal_nan=True)
    y = np.concatenate([np.random.default_rng(0).standard_normal(4000) * 100, np.linspace(-0.03, 0.03, 1001), (paged8.E4M3[:126] + paged8.E4M3[1:127]) / 2]).astype(np.float32)
    y = np.clip(y, -448, 448)
    assert np.array_equal(paged8.coded(y, "e4m3"), torch.from_numpy(y).to(torch.float8_e4m3fn).view(torch.uint8).numpy())
    assert paged8.coded([0.5, 1.5, -2.5, 126.6, -127.0], "int8").view(np.int8).tolist() == [0, 2, -2, 127, -127]


@pytest.mark.parametrize("code, most, power", [("e4m3", 448.0, 0), ("e4m3", 448.5, 1), ("e4m3", 1.75, -8), ("e4m3", 1.0, -8), ("e4m3", 2.0, -7), ("int8", 127.0, 0), ("int8", 128.0, 1),
                                               ("int8", 63.5, -1), ("int8", 3.0, -5), ("e4m3", 0.0, -126), ("int8", 1e-45, -126), ("e4m3", 65504.0, 8), ("int8", 65504.0, 10)])
def test_oracle_scale(code, most, power):
    assert paged8.least_power(most, code) == power


def test_oracle_store_grows_a_block():
    """Two tokens in a block, then two more in it and one in a new block; the second ones four times as large."""
    x = np.array([1.0, -0.3, 0.7, 0.0] * 4).reshape(1, 1, 16)
    codes, scales = np.full((3, 1, 4, 16), 0x55, np.uint8), np.full((3, 1), 9.0)
    a = paged8.store(np.concatenate([x, x]), codes, scales, [[2, 1]], [2], [0, 2], "e4m3", "bf16")
    assert a[1].tolist() == [[9.0], [9.0], [2.0**-8]] and (a[0][2, 0, 2:] == 0x55).all()
    b = paged8.store(np.concatenate([4 * x, x, x / 8]), *a, [[2, 1]], [5], [0, 3], "e4m3", "bf16")
    assert b[1].tolist() == [[9.0], [2.0**-11], [2.0**-6]]
    assert np.array_equal(paged8.numbers(*a, "e4m3")[2, :, :2], paged8.numbers(*b, "e4m3")[2, :, :2])      # a power of two: nothing is lost
    assert paged8.numbers(*b, "e4m3")[2, 0, 2, 0] == 4.0
    c = paged8.store(np.full((1, 1, 16), np.inf), *b, [[2, 1]], [3], [0, 1], "e4m3", "bf16")
    assert np.isnan(c[1][2, 0]) and np.isnan(paged8.numbers(*c, "e4m3")[2]).all()
    rows, mine = paged8.read(paged8.numbers(*b, "e4m3"), [[2, 1], [7, 0]], [5, 3], [0, 2, 3], 4)
    assert mine.tolist() == [True, True, True, False] and rows[0, 0, 0] == 1.0 and rows[1, 0, 0] == 0.125 and (rows[2] == 0).all()


@pytest.mark.parametrize("code", ["e4m3", "int8"])
@pytest.mark.parametrize("dtype, top, powers, numbers", [("f16", 65504.0, range(8, 27), 65504.0 - 32 * np.arange(1000)), ("bf16", 2.0**127 * (2 - 2.0**-7), range(120, 128), 2.0**120 * np.arange(60, 256))])
def test_oracle_cuts_only_what_would_be_infinite(code, dtype, top, powers, numbers):
    """Of fp16's numbers the greatest int8 code under 2^9 stands for 65024, which is one; under 2^11 63.5 and more would round to one that is none."""
    every = np.sort(paged8.values(np.arange(128, dtype=np.uint8), code)[:127 if code == "e4m3" else 128])
    for power in powers:
        x = numbers[numbers <= every[-1] * 2.0**power]
        if not len(x):
            continue
        codes, scales = np.zeros((1, 1, 8, len(x)), np.uint8), np.array([[2.0**power]])
        got, scale = paged8.store(np.stack([x, -x])[:, None], codes, scales, [[0]], [3], [0, 2], code, dtype)
        assert scale[0, 0] == 2.0**power
        nearest = paged8.values(paged8.coded(x / 2.0**power, code), code)
        want = np.where(nearest * 2.0**power > top, every[every * 2.0**power <= top].max(), nearest)
        assert np.array_equal(paged8.values(got[0, 0, 1], code), want) and np.array_equal(paged8.values(got[0, 0, 2], code), -want)


@pytest.mark.parametrize("change, shared", [({}, 0), (dict(tokens=5000, block_size=64), 0), (dict(tokens=5000, block_size=128), 16), (dict(kv_heads=1, head_dim=16), 0)])
def test_shared_memory_of_store_and_read(change, shared):
    """A maximum of each of four wavefronts, where a block has more new tokens than one holds (64 rows of 64 numbers); the read has none."""
    with Plan.cache_read8(**dict(CACHE, **change)) as p:
        assert p.info()["lds_bytes"] == 0
    with Plan.cache_store8(**dict(CACHE, **change)) as p:
        assert p.info()["lds_bytes"] == shared and ("head=4" if shared else "head=1") in p.describe()
