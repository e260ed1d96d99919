"""The cache operators without a GPU: sizes, refusals, and pins of their oracle."""
import math

import numpy as np
import pytest
import torch  # (before the library: the HIP runtime that both use is the one that comes with it)

from oracle import cache_ops as co
from paper_2510_05688_amd import binding as vb

ARG, SHAPE, NO_DEVICE, SMALL = vb.VATT_E_INVALID_ARG, vb.VATT_E_UNSUPPORTED_SHAPE, vb.VATT_E_NO_DEVICE, vb.VATT_E_WORKSPACE_TOO_SMALL


def _plan(q_len=1, fmt=0, block=None, rotary=None, **over):
    p = dict(batch=2, n_q_heads=8, n_kv_heads=2, head_dim=128, n_max=1000, kv_layout=0, page_size=0, num_blocks=0, sink=20, window=40,
             topk_abs=0, topk_frac=0.1, base_abs=0, base_frac=0.025, epsilon=0.05, delta=0.05, target=0, sm_scale=0.0,
             budget_cap_frac=1.0)
    p.update(over)
    plan = vb.vatt_plan_create_chunk(p, q_len, -1)
    vb.vatt_plan_set_option(plan, vb.VATT_OPT_KV_FORMAT, fmt)
    if block:
        vb.vatt_plan_set_option(plan, vb.VATT_OPT_BLOCK_TOKENS, block)
    if rotary:
        vb.vatt_plan_set_rotary(plan, rotary)
    return plan


class Mem:
    """A device buffer in name: the calls below must end before anything reads it."""

    def __init__(self, at=4096, size=1 << 40):
        self.at, self.size = at, size

    def data_ptr(self):
        return self.at

    def numel(self):
        return self.size

    def element_size(self):
        return 1


@pytest.mark.parametrize("fmt,row,scales", [(0, 256, 0), (1, 128, 4), (2, 64, 4)])
def test_sizes_of_a_cache(fmt, row, scales):
    plan = _plan(fmt=fmt)
    codes = 2 * 2 * 1000 * row
    off = codes if fmt == 0 else -(-codes // 256) * 256
    assert vb.vatt_kv_scale_offset(plan) == off
    assert vb.vatt_kv_cache_bytes(plan) == off + 2 * 2 * 1000 * scales
    odd = _plan(fmt=fmt, n_max=1001)  # the scales of a KV head are padded to a multiple of 8 rows
    assert vb.vatt_kv_cache_bytes(odd) == vb.vatt_kv_scale_offset(odd) + 2 * 2 * 1008 * scales
    paged = _plan(fmt=fmt, kv_layout=1, page_size=16, num_blocks=77)
    assert vb.vatt_kv_cache_bytes(paged) == 77 * 2 * 16 * (row + scales)
    for p in (plan, odd, paged):
        vb.vatt_plan_destroy(p)


def test_sizes_of_summaries_and_lists():
    plan = _plan(block=32)
    assert vb.vatt_block_summary_bytes(plan) == 2 * 2 * 32 * 2 * 128 * 2
    # sink 20: 1 block, window 40: at most 3, k = 100: 3
    assert vb.vatt_block_list_capacity(plan) == 1 + 3 + 3
    vb.vatt_plan_destroy(plan)
    plan = _plan(kv_layout=1, page_size=64, num_blocks=9, block=64, topk_frac=1.0)
    assert vb.vatt_block_summary_bytes(plan) == 9 * 2 * 2 * 128 * 2
    assert vb.vatt_block_list_capacity(plan) == 16
    vb.vatt_plan_destroy(plan)
    plan = _plan(kv_layout=1, page_size=8, num_blocks=9)  # pages smaller than a block
    assert vb.vatt_block_summary_bytes(plan) == vb.vatt_block_list_capacity(plan) == 0
    vb.vatt_plan_destroy(plan)


def test_every_list_fits_its_capacity():
    rng = np.random.default_rng(1)
    for _ in range(200):
        c = int(rng.choice([16, 32, 64, 128, 256]))
        n_max = int(rng.integers(1, 3000))
        p = dict(sink=int(rng.integers(0, 300)), window=int(rng.integers(0, 300)), topk_abs=int(rng.integers(0, 2) * rng.integers(1, 2000)),
                 topk_frac=float(rng.uniform()))
        plan = _plan(block=c, n_max=n_max, **p)
        cap = vb.vatt_block_list_capacity(plan)
        for n in {1, n_max, *rng.integers(1, n_max + 1, size=20).tolist()}:
            lo, hi, total, take = co.parts(n, p, c)
            assert lo + take + total - hi <= cap, (n, c, p)
            assert take * c <= vb.vatt_plan_index_segment(plan, 3) - vb.vatt_plan_index_segment(plan, 2)
        vb.vatt_plan_destroy(plan)


@pytest.mark.parametrize("option,value,code", [
    (vb.VATT_OPT_KV_FORMAT, 3, ARG), (vb.VATT_OPT_KV_FORMAT, -1, ARG), (vb.VATT_OPT_BLOCK_TOKENS, 8, ARG),
    (vb.VATT_OPT_BLOCK_TOKENS, 48, ARG), (vb.VATT_OPT_BLOCK_TOKENS, 512, ARG), (vb.VATT_OPT_BLOCK_TOKENS, 128, SHAPE)])
def test_options_are_checked(option, value, code):
    plan = _plan(kv_layout=1, page_size=64, num_blocks=9)
    with pytest.raises(vb.VattError) as e:
        vb.vatt_plan_set_option(plan, option, value)
    assert e.value.status == code
    vb.vatt_plan_destroy(plan)


GOOD = dict(theta=10000.0)


@pytest.mark.parametrize("over,code", [
    (dict(rotary_dim=24), SHAPE), (dict(rotary_dim=144), SHAPE), (dict(rotary_dim=-16), ARG), (dict(layout=2), ARG), (dict(scaling=4), ARG),
    (dict(theta=1.0), ARG), (dict(theta=math.inf), ARG), (dict(theta=math.nan), ARG), (dict(attention=-1.0), ARG),
    (dict(scaling=1), ARG), (dict(scaling=1, factor=0.5), ARG), (dict(scaling=2, factor=8.0, low=1.0, high=4.0), ARG),
    (dict(scaling=2, factor=8.0, low=4.0, high=4.0, original_len=100), ARG), (dict(scaling=3, factor=8.0, low=0.0, high=4.0, original_len=100), ARG),
    (dict(scaling=3, factor=math.nan, low=1.0, high=4.0, original_len=100), ARG)])
def test_rotations_are_checked(over, code):
    plan = _plan()
    with pytest.raises(vb.VattError) as e:
        vb.vatt_plan_set_rotary(plan, dict(GOOD, **over))
    assert e.value.status == code
    vb.vatt_plan_set_rotary(plan, GOOD)
    vb.vatt_plan_set_rotary(plan, None)
    vb.vatt_plan_destroy(plan)


def _write(plan, **over):
    a = dict(q=None, k_new=Mem(), v_new=Mem(), q_stride=0, k_stride=256, v_stride=256, n_new=3, first=Mem(), new_lens=None, k=Mem(), v=Mem(),
             block_table=None, summary=None, out_q=None, out_lens=None)
    a.update(over)
    vb.vatt_write_kv(plan, *a.values())


def _status(f, *args, **kw):
    with pytest.raises(vb.VattError) as e:
        f(*args, **kw)
    return e.value.status


def test_refusals_of_write():
    plan = _plan(rotary=GOOD)
    assert _status(_write, plan) == NO_DEVICE  # nothing else is wrong with it
    q = dict(q=Mem(), out_q=Mem(8192), q_stride=1024)
    assert _status(_write, plan, **q) == NO_DEVICE
    for over in (dict(k_new=None), dict(v_new=None), dict(first=None), dict(k=None), dict(v=None), dict(k_new=Mem(4104)), dict(v=Mem(4100)),
                 dict(n_new=0), dict(n_new=1001), dict(k_stride=248), dict(k_stride=260), dict(v_stride=255), dict(v_stride=0),
                 dict(q=Mem()), dict(out_q=Mem()), dict(q, q_stride=1016), dict(q, q_stride=1028), dict(q, out_q=q["q"]),
                 dict(summary=Mem(4098)), dict(first=Mem(64), out_lens=Mem(64)), dict(new_lens=Mem(64), out_lens=Mem(64))):
        assert _status(_write, plan, **over) == ARG, over
    vb.vatt_plan_set_rotary(plan, None)
    assert _status(_write, plan, **q) == ARG  # queries are only rotated
    vb.vatt_plan_destroy(plan)
    plan = _plan(kv_layout=1, page_size=8, num_blocks=9)
    assert _status(_write, plan, summary=Mem(), block_table=Mem()) == SHAPE
    assert _status(_write, plan, block_table=Mem()) == NO_DEVICE
    vb.vatt_plan_destroy(plan)


def test_refusals_of_the_other_calls():
    plan, m = _plan(), Mem()
    ok = [m, m, None, m, None, 5, m, m]
    assert _status(vb.vatt_read_kv, plan, *ok) == NO_DEVICE
    for i, x in ((0, None), (1, None), (3, None), (5, 0), (5, 1001), (6, Mem(8)), (7, Mem(4097))):
        assert _status(vb.vatt_read_kv, plan, *(ok[:i] + [x] + ok[i + 1:])) == ARG, i
    assert _status(vb.vatt_read_kv, plan, m, m, None, m, None, 5, None, None) == ARG
    ok = [m, None, m, m]
    assert _status(vb.vatt_block_summary_fill, plan, *ok) == NO_DEVICE
    for i, x in ((0, None), (0, Mem(8)), (2, None), (3, None), (3, Mem(24))):
        assert _status(vb.vatt_block_summary_fill, plan, *(ok[:i] + [x] + ok[i + 1:])) == ARG, i
    ok = [m, m, None, m, m, m, m, m, m]
    assert _status(vb.vatt_select_blocks, plan, *ok) == NO_DEVICE
    for i, x in ((0, None), (0, Mem(8)), (1, None), (1, Mem(8)), (3, None), (5, None), (6, None), (7, None), (8, None)):
        assert _status(vb.vatt_select_blocks, plan, *(ok[:i] + [x] + ok[i + 1:])) == ARG, i
    ok = [m, m, m, None, m, m, m, m, m, m]
    assert _status(vb.vatt_block_decode, plan, *ok) == NO_DEVICE
    for i, x in ((0, None), (1, None), (2, None), (2, Mem(8)), (4, None), (5, None), (6, None), (8, None)):
        assert _status(vb.vatt_block_decode, plan, *(ok[:i] + [x] + ok[i + 1:])) == ARG, i
    vb.vatt_plan_destroy(plan)
    plan = _plan(kv_layout=1, page_size=8, num_blocks=9)
    assert _status(vb.vatt_block_summary_fill, plan, m, m, m, m) == SHAPE
    assert _status(vb.vatt_select_blocks, plan, m, m, m, m, m, m, m) == SHAPE
    assert _status(vb.vatt_block_decode, plan, m, m, m, m, m, m, m, m, m, m) == SHAPE
    vb.vatt_plan_destroy(plan)


def test_oracle_formats():
    e4m3 = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(co.code_values(co.E4M3), e4m3, equal_nan=True)
    assert co.code_values(co.E2M1).tolist() == [0, .5, 1, 1.5, 2, 3, 4, 6, -0., -.5, -1, -1.5, -2, -3, -4, -6]
    x = torch.randn(500) * torch.exp(20 * torch.randn(500))
    assert np.array_equal(co.bf16_round(x.double().numpy()), x.to(torch.bfloat16).double().numpy())
    row = np.zeros(64)
    row[:6] = [448.0, 17.0, 19.0, -2.0 ** -10, 3 * 2.0 ** -10, 1e-9]
    codes, scales = co.encode(row, co.E4M3)
    assert scales.tolist() == [127, 0]
    assert co.decode(codes, scales, co.E4M3)[:6].tolist() == [448.0, 16.0, 20.0, -0.0, 2.0 ** -8, 0.0]  # ties to even
    row[:6] = [6.0 * 2 ** 100, 2.5 * 2 ** 100, 3.5 * 2 ** 100, -5.0 * 2 ** 100, 0.25 * 2 ** 100, 1.25 * 2 ** 100]
    codes, scales = co.encode(row, co.E2M1)
    assert scales.tolist() == [227, 0] and (co.decode(codes, scales, co.E2M1)[:6] / 2 ** 100).tolist() == [6, 2, 4, -4, 0, 1]
    row[0] = np.nextafter(6.0 * 2 ** 100, math.inf)
    assert co.encode(row, co.E2M1)[1][0] == 228
    row[40] = math.inf
    assert co.encode(row, co.E2M1)[1].tolist() == [228, 255]


def test_oracle_rotation():
    x = np.random.default_rng(0).normal(size=64)
    for layout in (0, 1):
        r = dict(theta=10000.0, layout=layout, rotary_dim=32)
        assert np.array_equal(co.rotate(x, 0, r), x)
        y, z = co.rotate(x, 11, r), co.rotate(co.rotate(x, 5, r), 6, r)  # angles add
        assert np.allclose(y, z, atol=1e-12) and np.array_equal(y[32:], x[32:])
        # what attention sees depends on the distance only
        a, b = np.random.default_rng(1).normal(size=(2, 64))
        assert np.isclose(co.rotate(a, 900, r) @ co.rotate(b, 890, r), co.rotate(a, 10, r) @ co.rotate(b, 0, r))
    plain = co.frequencies(dict(theta=1e4), 64)[0]
    long = dict(theta=1e4, factor=4.0, original_len=256, low=1.0, high=8.0)
    assert np.allclose(co.frequencies(dict(long, scaling=1), 64)[0], np.array(plain) / 4)
    for scaling in (2, 3):  # the fast pairs keep their angles, the slow ones have a quarter of them
        f, factor = co.frequencies(dict(long, scaling=scaling), 64)
        assert f[0] == plain[0] and np.isclose(f[-1], plain[-1] / 4) and all(p / 4 <= x <= p for x, p in zip(f, plain))
        assert factor == (1.0 if scaling == 2 else 0.1 * math.log(4.0) + 1.0)


def test_oracle_selection_is_a_bound():
    rng = np.random.default_rng(2)
    k = rng.normal(size=(10, 16, 32))
    q = rng.normal(size=(4, 32))
    top, low = k.max(1), k.min(1)
    u = co.bound(q, top, low)
    assert (u >= (k @ q.T).max(axis=(1, 2)) * (1 - 1e-6) - 1e-6).all()
    p = dict(sink=20, window=1, topk_abs=40, topk_frac=0.0)
    taken, chosen = co.select(np.array([9, 9, 1, 5, 5, 5, 0, 0, 0, 0]), 150, p, 16)
    assert taken == [0, 1, 3, 4, 9] and chosen == [3, 4]  # ties to the lower block
    taken, chosen = co.select(np.array([9, 9, 1, 5, 5, math.nan, 0, 0, 0, 0]), 150, p, 16)
    assert chosen == [3, 5]
