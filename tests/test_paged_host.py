"""The operators around a paged cache, without a GPU: refusals of plans and launches, what plans report, frequencies, and
the oracle's own edge cases."""
import ctypes as C

import numpy as np
import pytest

from oracle import paged
from paper_1911_11576_amd import FsError, Plan, binding, fs_rotary_frequencies

TABLES = dict(requests=4, tokens=8, blocks=10, block_size=16, table_blocks=3, free_blocks=2)
ROTARY = dict(dtype="bf16", tokens=4, q_heads=2, k_heads=1, head_dim=64)
STORE = dict(ROTARY, blocks=5, block_size=16)
ATTENTION = dict(dtype="bf16", requests=2, tokens=3, q_heads=4, kv_heads=2, head_dim=64, blocks=9, block_size=16, table_blocks=4, scale=0.125)


def refused(make, status, text, **kwargs):
    with pytest.raises(FsError) as e:
        make(**kwargs)
    assert e.value.status == status and text in e.value.message, e.value.message


@pytest.mark.parametrize("change, text", [
    (dict(requests=-1), "requests"), (dict(requests=4097), "requests"), (dict(tokens=-1), "tokens"), (dict(tokens=2**30 + 1), "tokens"),
    (dict(blocks=-1), "blocks"), (dict(free_blocks=-1), "blocks"), (dict(table_blocks=-1), "blocks"), (dict(block_size=0), "power of two"),
    (dict(block_size=24), "power of two"), (dict(block_size=2048), "power of two"), (dict(blocks=2**27), "2^31"), (dict(table_blocks=2**27), "2^31")])
def test_tables_refused(change, text):
    refused(Plan.block_tables, binding.FS_ERR_INVALID, text, **dict(TABLES, **change))


@pytest.mark.parametrize("change, text", [
    (dict(tokens=-1), "tokens"), (dict(q_heads=0), "q_heads"), (dict(k_heads=-1), "k_heads"), (dict(head_dim=63), "head_dim"), (dict(head_dim=514), "head_dim"),
    (dict(rotary_dim=66), "rotary_dim"), (dict(rotary_dim=3), "rotary_dim"), (dict(rotary_dim=0), "rotary_dim"), (dict(interleaved=2), "0 or 1"),
    (dict(inverse=-1), "0 or 1"), (dict(magnitude=float("nan")), "magnitude"), (dict(magnitude=1e300), "magnitude"), (dict(q_stride=127), "q_stride"),
    (dict(k_stride=-1), "k_stride"), (dict(q_out_stride=2**41), "q_out_stride"), (dict(interleaved=True, q_stride=129), "even"),
    (dict(block_size=16), "without blocks"), (dict(v_stride=64), "without blocks"), (dict(blocks=-1), "blocks"),
    (dict(blocks=5, block_size=16, k_heads=0), "k_heads"), (dict(blocks=5, block_size=10), "power of two"), (dict(blocks=5, block_size=16, k_out_stride=64), "k_out_stride"),
    (dict(blocks=5, block_size=16, block_stride=1024, head_stride=0, slot_stride=32), "overlap"),
    (dict(blocks=5, block_size=16, block_stride=512, head_stride=64, slot_stride=64), "overlap"),
    (dict(blocks=5, block_size=16, block_stride=-1), "negative")])
def test_rotary_refused(change, text):
    refused(Plan.rotary, binding.FS_ERR_INVALID, text, **dict(ROTARY, **change))


@pytest.mark.parametrize("change, text", [
    (dict(requests=-1), "requests"), (dict(tokens=-1), "tokens"), (dict(tokens=2**30), "tokens"), (dict(q_heads=3), "q_heads"), (dict(kv_heads=0), "kv_heads"),
    (dict(head_dim=0), "head_dim"), (dict(block_size=12), "power of two"), (dict(blocks=2**28), "2^31"), (dict(table_blocks=2**28), "2^31"), (dict(causal=2), "0 or 1"),
    (dict(window=-1), "window"), (dict(window=5, causal=False), "window"), (dict(max_new=-1), "max_new"), (dict(scale=float("inf")), "scale"), (dict(scale=3e38), "scale"), (dict(requests=65537), "requests"),
    (dict(q_stride=128), "q_stride"), (dict(out_stride=-8), "out_stride"), (dict(slot_stride=32, head_stride=1024, block_stride=4096), "overlap")])
def test_attention_refused(change, text):
    refused(Plan.paged_attention, binding.FS_ERR_INVALID, text, **dict(ATTENTION, **change))


@pytest.mark.parametrize("change, text", [
    (dict(dtype="f32"), "f16 and bf16"), (dict(head_dim=48), "head_dim"), (dict(head_dim=256), "head_dim"), (dict(q_stride=258), "multiples of 8"),
    (dict(slot_stride=132, head_stride=64, block_stride=4224), "multiples of 8")])
def test_attention_unsupported(change, text):
    refused(Plan.paged_attention, binding.FS_ERR_UNSUPPORTED, text, **dict(ATTENTION, **change))


def test_attention_of_more_tiles_than_a_grid_has():
    """Tiles of 128 rows: tokens * share / 128 + requests places for every key head, 256 threads each, below 2^32 of them."""
    change = dict(requests=32760, tokens=100, q_heads=512, kv_heads=512, max_new=0)
    Plan.paged_attention(**dict(ATTENTION, **change))[0].close()
    refused(Plan.paged_attention, binding.FS_ERR_UNSUPPORTED, "too many tiles", **dict(ATTENTION, **dict(change, requests=32768)))


def test_null_arguments():
    L, out, n = binding.lib(), C.c_void_p(), C.c_int64()
    assert L.fs_plan_create_block_tables(None, C.byref(out)) == binding.FS_ERR_INVALID
    assert L.fs_plan_create_rotary(None, C.byref(out)) == binding.FS_ERR_INVALID
    assert L.fs_plan_create_paged_attention(None, C.byref(n), C.byref(out)) == binding.FS_ERR_INVALID
    assert L.fs_plan_create_block_tables(C.byref(binding.fs_block_tables_desc(1, 1, 1, 1, 1, 1)), None) == binding.FS_ERR_INVALID
    d = binding.fs_paged_attention_desc(2, 1, 1, 1, 1, 64, 1, 16, 1, 1, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0.1)
    assert L.fs_plan_create_paged_attention(C.byref(d), None, C.byref(out)) == binding.FS_ERR_INVALID and not out.value
    d.reserved = 1
    assert L.fs_plan_create_paged_attention(C.byref(d), C.byref(n), C.byref(out)) == binding.FS_ERR_INVALID and not out.value
    assert L.fs_rotary_frequencies(64, 1e4, 1.0, 0.0, 0.0, 0.0, None) == binding.FS_ERR_INVALID


def launches_refused(plan, ins, outs, text):
    with pytest.raises(FsError) as e:
        plan.launch(ins, outs, 0)
    assert e.value.status == binding.FS_ERR_INVALID and text in e.value.message, e.value.message


def addresses(n, first=1 << 20):
    return [first + 4096 * i for i in range(n)]


def check_launch_arguments(plan, n_in, n_out):
    """Counts, alignment, NULL and shared buffers are refused before anything is launched."""
    ins, outs = addresses(n_in), addresses(n_out, 1 << 30)
    launches_refused(plan, ins[:-1], outs, "n_in")
    launches_refused(plan, ins, outs + [1 << 31], "n_out")
    for k in range(n_in):
        launches_refused(plan, ins[:k] + [0] + ins[k + 1:], outs, "NULL")
        launches_refused(plan, ins[:k] + [ins[k] + 4] + ins[k + 1:], outs, "aligned")
    for k in range(n_out):
        launches_refused(plan, ins, outs[:k] + [0] + outs[k + 1:], "NULL")
        launches_refused(plan, ins, outs[:k] + [outs[k] + 8] + outs[k + 1:], "aligned")
        if k:
            launches_refused(plan, ins, outs[:k] + [outs[0]] + outs[k + 1:], "share")
        launches_refused(plan, ins, outs[:k] + [ins[2]] + outs[k + 1:], "shares")


def test_launch_arguments():
    with Plan.block_tables(**TABLES) as p:
        check_launch_arguments(p, 3, 6)
    with Plan.rotary(**ROTARY) as p:
        check_launch_arguments(p, 4, 2)
    with Plan.rotary(**STORE) as p:
        check_launch_arguments(p, 6, 3)
    plan, nbytes = Plan.paged_attention(**ATTENTION, lse=True)
    with plan:
        check_launch_arguments(plan, 6, 2 + (nbytes > 0))


def test_in_place_needs_the_same_strides():
    q = addresses(4)
    with Plan.rotary(**ROTARY, q_stride=256) as p:
        launches_refused(p, q, [q[0], 1 << 30], "shares")
    with Plan.rotary(**ROTARY) as p:      # the other's buffer
        launches_refused(p, q, [q[1], 1 << 30], "shares")


def test_nothing_to_do_launches_nothing():
    with Plan.rotary(**dict(ROTARY, tokens=0)) as p:
        p.launch([0] * 4, [0] * 2, 0)
        p.launch_static([0] * 4, [0] * 2, 0)
    for none in (dict(tokens=0), dict(requests=0)):
        plan, nbytes = Plan.paged_attention(**dict(ATTENTION, **none))
        with plan:
            plan.launch([1 << 20, 0, 0, 0, 0, 0] if "requests" in none else [0] * 6, [1 << 21 if "requests" in none else 0] + [0] * (nbytes > 0), 0)


def test_plans_report():
    with Plan.block_tables(**TABLES) as p:
        assert p.info()["schedule"] == "block_tables" and p.info()["n_kernels"] == 1 and p.info()["workspace_bytes"] == 0
        assert "block_tables" in p.describe()
    with Plan.rotary(**STORE) as p:
        assert p.info()["schedule"] == "rotary" and "cache" in p.describe()
        assert p.info()["algorithmic_bytes"] == 2 * 4 * 64 * 4 * 2 + 4 * 8 + 4 * 64
    plan, _ = Plan.paged_attention(**ATTENTION)
    with plan:
        assert plan.info()["schedule"] == "paged_attention" and plan.info()["algorithmic_bytes"] > 0 and "paged_attention" in plan.describe()


@pytest.mark.parametrize("change, once", [
    (dict(), True), (dict(dtype="f32", head_dim=64), True), (dict(q_out_stride=32 * 128 + 64), True), (dict(q_out_stride=32 * 128 + 32, k_out_stride=8 * 128 + 32), True),
    (dict(q_out_stride=32 * 128 + 8), False), (dict(k_out_stride=8 * 128 + 8), False), (dict(dtype="f32", q_out_stride=32 * 128 + 16), False), (dict(q_stride=32 * 128 + 2), False),
    (dict(q_out_stride=32 * 128 + 2), False), (dict(rotary_dim=64), False), (dict(head_dim=64), False), (dict(k_heads=0), True), (dict(blocks=600, block_size=16), False)])
def test_rotary_stores_past_the_caches_in_whole_lines_alone(change, once):
    with Plan.rotary(**dict(dict(dtype="bf16", tokens=8192, q_heads=32, k_heads=8, head_dim=128), **change)) as p:
        assert ("past the caches" in p.describe()) == once, p.describe()


@pytest.mark.parametrize("dim", [2, 24, 128])
@pytest.mark.parametrize("args", [{}, dict(base=5e5), dict(factor=4.0), dict(factor=8.0, low=1.0, high=4.0, original=8192.0), dict(factor=2.0, low=1.0, high=32.0, original=100.0)])
def test_frequencies(dim, args):
    got, want = fs_rotary_frequencies(dim, **args), paged.frequencies(dim, **args)
    assert np.allclose(got, want, rtol=1e-14, atol=0)


@pytest.mark.parametrize("args", [dict(rotary_dim=3), dict(rotary_dim=0), dict(rotary_dim=8, base=0.0), dict(rotary_dim=8, factor=0.5), dict(rotary_dim=8, base=float("nan")),
                                  dict(rotary_dim=8, factor=2.0, low=1.0), dict(rotary_dim=8, factor=2.0, low=4.0, high=4.0, original=10.0),
                                  dict(rotary_dim=8, factor=2.0, low=1.0, high=4.0)])
def test_frequencies_refused(args):
    with pytest.raises(FsError):
        fs_rotary_frequencies(**args)


def test_oracle_tables():
    t = [[7, 9, -1], [3, -1, -1], [-1, -1, -1]]
    tables, lengths, starts, positions, slots, taken = paged.block_tables([17, 0, 5], [20, 3, 9], [4, 11, 6], t, 24, 10, 16)
    assert tables.tolist() == [[7, 9, 4], [11, -1, -1], [-1, -1, -1]]      # a block of request 0 and of request 1; the third's first entry is not touched
    assert lengths.tolist() == [37, 3, 6] and starts.tolist() == [0, 20, 23, 24] and taken.tolist() == [2, 2]
    assert positions.tolist() == [*range(17, 37), 0, 1, 2, 5]
    assert slots[:16].tolist() == [9 * 16 + i for i in range(1, 16)] + [64] and slots[20:].tolist() == [-1] * 4      # block 11 is outside, -1 too


def test_oracle_attention_masks():
    rng = np.random.default_rng(0)
    k, v, q = (rng.standard_normal(s) for s in ((3, 1, 4, 8), (3, 1, 4, 8), (3, 2, 8)))
    out, lse, *_ = paged.attention(q, k, v, [[2, 7, 0], [1, -1, 0]], [9, 1], [0, 2, 2], 0.3)
    assert np.isnan(out[2]).all()                                          # no request's row
    rows = np.concatenate([k[2, 0], k[0, 0, :1]]), np.concatenate([v[2, 0], v[0, 0, :1]])
    for t, n in ((0, 4), (1, 5)):                                          # block 7 is no block: its four keys are not seen
        s = 0.3 * rows[0][:n] @ q[t, 1]
        assert np.allclose(out[t, 1], np.exp(s) @ rows[1][:n] / np.exp(s).sum()) and np.isclose(lse[t, 1], np.log(np.exp(s).sum()))
    out, lse, *_ = paged.attention(q, k, v, [[2, 7, 0]], [1], [0, 3], 0.3)    # more new tokens than keys
    assert (out[:2] == 0).all() and (lse[:2] == -np.inf).all() and np.allclose(out[2], v[2, 0, 0])
