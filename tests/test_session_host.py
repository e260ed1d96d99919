"""What DecodeSession checks before a call goes to the library, without a GPU: nothing here may reach a kernel."""
import numpy as np
import pytest
import torch

from paper_2510_05688_amd import session as sm


class Calls:
    """The binding with every call that would launch something written down instead."""

    def __init__(self, monkeypatch, *names):
        self.made = []
        for name in names:
            monkeypatch.setattr(sm.vb, name, lambda *a, _name=name, **kw: self.made.append((_name, a)))


def _session(q_len=1, batch=2, hq=8, hkv=2, d=64, n_max=100, k_max=30, page=0):
    """A session as its constructor leaves it, on the CPU: no plan, no workspace."""
    s = sm.DecodeSession.__new__(sm.DecodeSession)
    s.plan, s.plain, s.device, s.q_len, s.kv_format, s.block_tokens = None, None, torch.device("cpu"), q_len, 0, None
    s.params = dict(batch=batch, n_q_heads=hq, n_kv_heads=hkv, head_dim=d, n_max=n_max, page_size=page)
    s.B, s.Hq, s.Hkv, s.d, s.n_max, s.paged, s.seg = batch * q_len, hq, hkv, d, n_max, page > 0, [0, 4, 8, 8 + k_max, 60]
    s.workspace = s.out_o = s.out_lse = s.k = s.v = s.q = s.seq_seeds = s.block_table = s.summary = s.blocks = s.block_count = s.rcache = s.cache_seeds = None
    s.seq_lens = torch.full((batch,), 50, dtype=torch.int32)
    s._stream = lambda: 0
    return s


def _ints(*x):
    return torch.tensor(x, dtype=torch.int32)


def test_rows_back_are_asked_for_by_one_int32_per_sequence(monkeypatch):
    calls, s = Calls(monkeypatch, "vatt_read_kv"), _session()
    for bad in ([1, 2], 5.0, np.array([1, 2], dtype=np.int32), _ints(1), _ints(1, 2, 3), _ints(1, 2).long(), _ints(1, 0, 2, 0)[::2]):
        with pytest.raises(ValueError):
            s.read_rows(bad, 3)
    assert not calls.made
    s.read_rows(_ints(1, 2), 3)
    s.read_rows(None, 3)
    for number in (0, 5):  # the same first row for all, never an address
        s.read_rows(number, 3)
    assert [name for name, _ in calls.made] == ["vatt_read_kv"] * 4
    assert calls.made[1][1][5] is None and [calls.made[i][1][5].tolist() for i in (0, 2, 3)] == [[1, 2], [0, 0], [5, 5]]


@pytest.mark.parametrize("q_len", [1, 3])
def test_queries_of_the_block_calls(monkeypatch, q_len):
    calls, s = Calls(monkeypatch, "vatt_select_blocks", "vatt_block_decode"), _session(q_len)
    q = torch.zeros(2, q_len, 8, 64, dtype=torch.bfloat16)
    for call in (s.select_blocks, s.block_decode):
        for bad in (4096, q[:1], q[..., :32], q[:, :, :4], q.float(), q.transpose(2, 3).contiguous().transpose(2, 3),
                    torch.cat([q, q], 1), q.view(torch.int16), q.to("meta")):
            with pytest.raises(ValueError):
                call(bad)
    assert not calls.made
    s.select_blocks(q)
    s.block_decode(q.view(2 * q_len, 8, 64))  # [B, Hq, d] as the plan's other calls have it
    s.q = q
    s.select_blocks()
    s.block_decode()
    assert [name for name, _ in calls.made] == ["vatt_select_blocks", "vatt_block_decode"] * 2


def test_token_lists_of_the_choice(monkeypatch):
    calls, s = Calls(monkeypatch, "vatt_select_blocks"), _session(2)
    q, idx, cnt = torch.zeros(2, 2, 8, 64, dtype=torch.bfloat16), torch.zeros(4, 8, 30, dtype=torch.int32), torch.zeros(4, 8, dtype=torch.int32)
    for a, b in ((idx[:2], cnt), (idx[..., :29], cnt), (idx.long(), cnt), (idx.to("meta"), cnt), (idx.mT.contiguous().mT, cnt),
                 (idx, cnt[:3]), (idx, cnt.long()), (idx, cnt.to("meta")), (4096, cnt), (idx, 4096)):
        with pytest.raises(ValueError):
            s.select_blocks(q, a, b)
    assert not calls.made
    s.select_blocks(q, idx, cnt)
    assert len(calls.made) == 1


def test_an_upload_into_a_quantised_plan_has_its_bytes(monkeypatch):
    """bf16 rows for a plan whose kernels read codes and scales would be taken for those, and can be shorter than the cache."""
    p = dict(batch=1, n_q_heads=2, n_kv_heads=1, head_dim=64, n_max=1, kv_layout=0, page_size=0, num_blocks=0, sink=4, window=4, topk_abs=0,
             topk_frac=0.1, base_abs=0, base_frac=0.1, epsilon=0.1, delta=0.1, target=0, sm_scale=0.0, budget_cap_frac=1.0)
    for fmt, n_max in ((1, 1), (2, 1), (1, 50), (2, 77)):
        s = _session(batch=1, hq=2, hkv=1, n_max=n_max)
        s.plan, s.kv_format = sm.vb.vatt_plan_create(dict(p, n_max=n_max), -1), fmt
        sm.vb.vatt_plan_set_option(s.plan, sm.vb.VATT_OPT_KV_FORMAT, fmt)
        q, rows, size = np.zeros((1, 2, 64), np.uint16), np.zeros((1, 1, n_max, 64), np.uint16), sm.vb.vatt_kv_cache_bytes(s.plan)
        whole = np.arange(size // 2, dtype=np.uint16)
        for k, v in ((rows, rows), (whole, rows), (rows, whole), (whole[:-1], whole[:-1])):
            with pytest.raises(ValueError):
                s.upload(q, k, v, [1], [0])
        assert s.q is None and s.k is None
        s.upload(q, whole, whole, [1], [0])  # a cache that was written somewhere else
        assert s.k.view(torch.int16).numpy().view(np.uint16).tolist() == whole.tolist()
        s.close()
    s = _session(batch=1, hq=2, hkv=1, n_max=50)
    s.plan, s.kv_format = sm.vb.vatt_plan_create(dict(p, n_max=50), -1), 0
    s.upload(np.zeros((1, 2, 64), np.uint16), *[np.zeros((1, 1, 50, 64), np.uint16)] * 2, [50], [0])
    assert s.k.shape == (1, 1, 50, 64)
    s.close()


def _host_session(page=0, block=16, **over):
    """A session with a plan that is of no device."""
    p = dict(batch=2, n_q_heads=8, n_kv_heads=2, head_dim=64, n_max=100, kv_layout=1 if page else 0, page_size=page, num_blocks=30 if page else 0,
             sink=4, window=4, topk_abs=0, topk_frac=0.3, base_abs=0, base_frac=0.1, epsilon=0.1, delta=0.1, target=0, sm_scale=0.0,
             budget_cap_frac=1.0)
    p.update(over)
    s = _session(page=page)
    s.params, s.block_tokens = p, block
    s.plan = s._new_plan()
    return s


def test_a_cache_on_pages_needs_its_whole_block_table():
    s = _host_session(page=16)
    table = np.arange(14, dtype=np.int32).reshape(2, 7)
    for bad in (table[:1], table[:, :6], np.arange(13)):
        with pytest.raises(ValueError):
            s.make_cache(bad)
    assert s.k is None and s.block_table is None
    s.make_cache(table)
    assert s.block_table.tolist() == table.tolist()
    s.close()
    s = _host_session().make_cache()
    assert s.block_table is None
    s.close()


def test_a_new_cache_leaves_nothing_of_the_last_one():
    """Queries, seeds and the random cache of other sequences would be used without a word."""
    s = _host_session()
    s.upload(np.zeros((2, 8, 64), np.uint16), *[np.zeros((2, 2, 100, 64), np.uint16)] * 2, [5, 5], [1, 2])
    s.rcache = s.cache_seeds = torch.zeros(1)
    s.make_cache()
    assert s.q is None and s.seq_seeds is None and s.rcache is None and s.cache_seeds is None
    assert s.seq_lens.tolist() == [0, 0]
    s.close()


def test_queries_of_tokens_that_are_not_written(monkeypatch):
    """Padding, and tokens of a full sequence, which the call leaves as they were: zeros, not what lay in the memory."""
    s, calls = _host_session(), []
    s.make_cache()
    monkeypatch.setattr(sm.vb, "vatt_write_kv", lambda *a: calls.append(a))
    q, kv = torch.ones(2, 3, 8, 64, dtype=torch.bfloat16), torch.ones(2, 3, 2, 64, dtype=torch.bfloat16)
    was = torch.are_deterministic_algorithms_enabled()
    torch.use_deterministic_algorithms(True)  # (memory nobody has written is then NaN)
    try:
        out = s.write(q, kv, kv, _ints(1, 0))
    finally:
        torch.use_deterministic_algorithms(was)
    assert calls and not out.any()
    s.close()


def test_lengths_of_new_tokens_lie_one_behind_the_other(monkeypatch):
    s, calls = _host_session(), Calls(monkeypatch, "vatt_write_kv")
    s.make_cache()
    kv = torch.ones(2, 3, 2, 64, dtype=torch.bfloat16)
    for bad in (_ints(1, 9, 2, 9)[::2], _ints(1).expand(2), _ints(1), _ints(1, 2).long(), 2):
        with pytest.raises(ValueError):
            s.write(None, kv, kv, bad)
    assert not calls.made
    s.write(None, kv, kv, _ints(1, 2))
    s.close()


def test_appended_tokens_reach_the_summaries(monkeypatch):
    calls, s = Calls(monkeypatch, "vatt_append_kv", "vatt_append_kv_cached", "vatt_write_kv"), _host_session()
    x = torch.zeros(2, 2, 64, dtype=torch.bfloat16)
    s.append_device(x, x)
    s.append_device_cached(x, x)
    assert [name for name, _ in calls.made] == ["vatt_append_kv", "vatt_append_kv_cached"]  # there are none
    s.make_cache()
    calls.made.clear()
    s.append_device(x, x)
    s.append_device_cached(x, x)
    assert [name for name, _ in calls.made] == ["vatt_write_kv", "vatt_append_kv", "vatt_write_kv", "vatt_append_kv_cached"]
    assert all(a[0] is s.plain is not s.plan for name, a in calls.made if name == "vatt_write_kv")  # nothing is rotated
    sm.vb.vatt_plan_set_option(s.plan, sm.vb.VATT_OPT_KV_FORMAT, 1)  # the append is refused: nothing may be written before
    calls.made.clear()
    s.append_device(x, x)
    assert [name for name, _ in calls.made] == ["vatt_append_kv"]
    s.close()


def test_summaries_of_an_uploaded_cache(monkeypatch):
    calls, s = Calls(monkeypatch, "vatt_block_summary_fill"), _host_session()
    s.upload(np.zeros((2, 8, 64), np.uint16), *[np.zeros((2, 2, 100, 64), np.uint16)] * 2, [5, 5], [1, 2])
    s.fill_summary()
    assert calls.made[0][1][1:5] == (s.k, None, s.seq_lens, s.summary) and s.summary.numel() == 2 * 2 * 7 * 2 * 64
    assert s.blocks.shape == (2, 2, s.block_capacity) and s.block_count.shape == (2, 2)
    s.close()


def test_the_verified_step_takes_queries(monkeypatch):
    """What write() returns goes into the step with a supplied top-k set as it goes into the others."""
    calls, s = Calls(monkeypatch, "vatt_decode_given_topk", "vatt_decode_given_topk_cached"), _host_session()
    s.make_cache()
    s.out_idx = s.out_counts = s.out_budget_raw = s.out_stats = None
    q, idx, cnt = torch.zeros(2, 1, 8, 64, dtype=torch.bfloat16), torch.zeros(2, 8, 30, dtype=torch.int32), torch.zeros(2, 8, dtype=torch.int32)
    s.decode_given_topk(idx, cnt, q=q)
    s.decode_given_topk_cached(idx, cnt, q=q)
    assert [a[1] is q for _, a in calls.made] == [True, True]
    for call in (s.decode_given_topk, s.decode_given_topk_cached):
        with pytest.raises(ValueError):
            call(idx, cnt, q=q[:1])
    s.close()


@pytest.mark.parametrize("q_len", [1, 4])
def test_queries_of_the_steps_over_all_tokens(monkeypatch, q_len):
    """write() returns as many queries as it was given tokens; a plan takes q_len of them."""
    calls, s = Calls(monkeypatch, "vatt_dense_decode", "vatt_decode", "vatt_score"), _session(q_len)
    s.dense_o = s.dense_lse = s.out_idx = s.out_counts = s.out_budget_raw = s.out_stats = None
    for call in (s.dense, s.decode, s.score):
        for tokens in (1, 2, 4, 5):
            q = torch.zeros(2, tokens, 8, 64, dtype=torch.bfloat16)
            if tokens == q_len:
                call(q)
                assert calls.made.pop()[1][1] is q
                continue
            with pytest.raises(ValueError):
                call(q)
    assert not calls.made


def test_queries_into_a_buffer_of_the_callers(monkeypatch):
    """It is handed on as it is: nothing is cleared, nothing allocated."""
    calls, s = Calls(monkeypatch, "vatt_write_kv"), _host_session()
    s.make_cache()
    q, kv = torch.ones(2, 3, 8, 64, dtype=torch.bfloat16), torch.ones(2, 3, 2, 64, dtype=torch.bfloat16)
    out = torch.full_like(q, 7.0)
    for bad in (out[:1], out[:, :2], out.float(), out.to("meta"), out.transpose(0, 1), 4096):
        with pytest.raises(ValueError):
            s.write(q, kv, kv, out_q=bad)
    with pytest.raises(ValueError):
        s.write(None, kv, kv, out_q=out)
    assert not calls.made
    assert s.write(q, kv, kv, out_q=out) is out and calls.made[0][1][14] is out and (out == 7.0).all()
    s.close()


@pytest.mark.parametrize("block", [16, 32, 64])
def test_options_set_on_the_plan_itself(monkeypatch, block):
    """Blocks and formats that the constructor was not told of: appended rows go into summaries of that layout, uploads are still checked."""
    calls, s, x = Calls(monkeypatch, "vatt_append_kv", "vatt_write_kv"), _host_session(block=None), torch.zeros(2, 2, 64, dtype=torch.bfloat16)
    sm.vb.vatt_plan_set_option(s.plan, sm.vb.VATT_OPT_BLOCK_TOKENS, block)
    s.make_cache()
    s.append_device(x, x)
    used = [a[0] for name, a in calls.made if name == "vatt_write_kv"]
    assert len(used) == 1 and sm.vb.vatt_block_summary_bytes(used[0]) == sm.vb.vatt_block_summary_bytes(s.plan) == 2 * s.summary.numel()
    sm.vb.vatt_plan_set_option(s.plan, sm.vb.VATT_OPT_KV_FORMAT, 2)
    with pytest.raises(ValueError):
        s.upload(np.zeros((2, 8, 64), np.uint16), *[np.zeros((2, 2, 100, 64), np.uint16)] * 2, [5, 5], [1, 2])
    s.close()
