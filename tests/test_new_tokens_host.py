"""Attention of new tokens without a GPU: workspace sizes, refusals, and pins of its oracle."""
import numpy as np
import pytest
import torch  # (before the library: the HIP runtime that both use is the one that comes with it)

from oracle import cache_ops as co
from paper_2510_05688_amd import binding as vb
from paper_2510_05688_amd import session as sm
from test_cache_ops_host import ARG, NO_DEVICE, SHAPE, Mem, _plan, _status
from test_session_host import Calls, _ints, _session


def _chunk(plan, **over):
    a = dict(q=Mem(), q_stride=1024, n_new=3, first=Mem(), new_lens=None, k=Mem(), v=Mem(), block_table=None, sink=0, window=0, workspace=Mem(),
             out_type=vb.VATT_OUT_F32, out_o=Mem(8192), out_lse=None)
    a.update(over)
    vb.vatt_chunk_attend(plan, *a.values())


def test_refusals_of_chunks():
    plan = _plan()
    assert _status(_chunk, plan) == NO_DEVICE  # nothing else is wrong with it
    for over in (dict(new_lens=Mem()), dict(out_lse=Mem()), dict(out_type=vb.VATT_OUT_BF16), dict(sink=1 << 30, window=1 << 30), dict(n_new=1000),
                 dict(q_stride=2048)):
        assert _status(_chunk, plan, **over) == NO_DEVICE, over
    for over in (dict(q=None), dict(first=None), dict(k=None), dict(v=None), dict(out_o=None), dict(q=Mem(8)), dict(k=Mem(4104)), dict(v=Mem(4100)),
                 dict(out_o=Mem(8200)), dict(n_new=0), dict(n_new=-1), dict(n_new=1001), dict(q_stride=1016), dict(q_stride=1028), dict(q_stride=0),
                 dict(sink=-1), dict(window=-1), dict(out_type=2), dict(out_type=-1), dict(out_o=Mem())):
        assert _status(_chunk, plan, **over) == ARG, over
    vb.vatt_plan_destroy(plan)


def test_refusals_of_window_decode():
    plan, m = _plan(), Mem()
    ok = [m, m, m, None, m, 4, 10, m, m, m]
    assert _status(vb.vatt_window_decode, plan, *ok) == NO_DEVICE
    for i, x in ((0, None), (0, Mem(8)), (1, None), (1, Mem(8)), (2, None), (2, Mem(24)), (4, None), (5, -1), (6, 0), (6, -3), (8, None)):
        assert _status(vb.vatt_window_decode, plan, *(ok[:i] + [x] + ok[i + 1:])) == ARG, i
    vb.vatt_plan_destroy(plan)


def test_workspace_of_chunks():
    plan = _plan()
    assert [vb.vatt_chunk_workspace_bytes(plan, n) for n in (0, -1, 1001)] == [0, 0, 0]
    few = vb.vatt_chunk_workspace_bytes(plan, 1)
    # sums of 16 vectors for 126 workgroups per KV head and the 4 jobs (sequence, KV head), and the jobs' list
    assert few == (126 * 2 + 4) * 16 * (128 + 2) * 4 + 4 * 8
    many = vb.vatt_chunk_workspace_bytes(plan, 500)
    assert many > 0 and many % (128 * (128 + 2) * 4) == 0  # of whole tiles of 128 rows
    vb.vatt_plan_destroy(plan)
    short = _plan(n_max=640)  # nothing to share out: one workgroup has all keys of its rows
    assert [vb.vatt_chunk_workspace_bytes(short, n) for n in (1, 8, 9, 640)] == [0, 0, 0, 0]
    vb.vatt_plan_destroy(short)
    one = _plan(batch=1, n_kv_heads=8, n_max=2048, n_q_heads=32)  # tiles for all compute units, or for a few
    assert vb.vatt_chunk_workspace_bytes(one, 2048) == 0 and vb.vatt_chunk_workspace_bytes(one, 64) > 0
    vb.vatt_plan_destroy(one)
    one = _plan(batch=1, n_kv_heads=8, n_max=65536, n_q_heads=32)  # of many new tokens a few may count
    assert vb.vatt_chunk_workspace_bytes(one, 2048) > 0
    vb.vatt_plan_destroy(one)


def test_launches_without_room():
    plan = _plan(batch=65535, n_q_heads=64, n_kv_heads=64, n_max=100000, head_dim=64)
    assert _status(_chunk, plan, q_stride=4096, n_new=100000) == SHAPE
    assert _status(_chunk, plan, q_stride=4096, n_new=1) == NO_DEVICE
    vb.vatt_plan_destroy(plan)


def test_oracle_visible():
    assert co.visible(5, 0, 0).tolist() == [0, 1, 2, 3, 4, 5]
    assert co.visible(9, 2, 3).tolist() == [0, 1, 7, 8, 9]
    assert co.visible(3, 2, 3).tolist() == [0, 1, 2, 3] and co.visible(0, 0, 1).tolist() == [0] and co.visible(4, 9, 1).tolist() == [0, 1, 2, 3, 4]
    assert [co.new_tokens(f, w, 8, 100) for f, w in ((0, 9), (95, 8), (-1, 8), (100, 8), (3, -2), (99, 1))] == [8, 5, 0, 0, 0, 1]
    # a window that reaches everything is plain causal attention
    rng = np.random.default_rng(0)
    k, v, q = rng.normal(size=(3, 20, 16))
    for p in (0, 7, 19):
        whole, one = co.visible(p, 0, 0), co.visible(p, 0, 20)
        assert np.array_equal(whole, one) and np.array_equal(co.attend(q[p], k[whole], v[whole], 0.2)[0], co.attend(q[p], k[one], v[one], 0.2)[0])


# ---- what DecodeSession checks -------------------------------------------------------------------------------------------------

def test_a_session_checks_the_tensors_of_attend(monkeypatch):
    calls, s = Calls(monkeypatch, "vatt_write_kv", "vatt_chunk_attend"), _session()
    monkeypatch.setattr(sm.vb, "vatt_chunk_workspace_bytes", lambda plan, n_new: 512)
    q, kv = (torch.zeros(2, 3, h, 64, dtype=torch.bfloat16) for h in (8, 2))
    with pytest.raises(ValueError):
        s.attend(q)  # nothing was written
    s.write(None, kv, kv)
    for bad in (q[:1], q[..., :32], q[:, :, :4], q.float(), q.transpose(2, 3).contiguous().transpose(2, 3), q[0], q.to("meta")):
        with pytest.raises(ValueError):
            s.attend(bad)
    for over in (dict(new_lens=_ints(1)), dict(new_lens=_ints(1, 2).long()), dict(new_lens=[1, 2]), dict(first=_ints(1, 2, 3)), dict(first=5),
                 dict(dtype=torch.float16), dict(out=torch.zeros(2, 3, 8, 64, dtype=torch.float16)), dict(out=torch.zeros(2, 3, 8, 32)),
                 dict(out=torch.zeros(2, 3, 64, 8).transpose(2, 3)), dict(lse=torch.zeros(2, 3, 4)), dict(lse=torch.zeros(2, 3, 8).double())):
        with pytest.raises(ValueError):
            s.attend(q, **over)
    assert [name for name, _ in calls.made] == ["vatt_write_kv"]
    out, lse = s.attend(q, _ints(3, 1), sink=4, window=9)
    assert out.dtype == torch.bfloat16 and out.shape == q.shape and lse.shape == (2, 3, 8) and not out.any() and not lse.any()
    a = calls.made[-1][1]
    assert a[1] is q and a[2:4] == (512, 3) and a[4] is s.first and a[4].tolist() == [50, 50] and a[9:11] == (4, 9) and a[11].numel() == 512
    own = torch.ones(2, 3, 8, 64)
    out, lse = s.attend(q, out=own, first=_ints(1, 2))
    assert out is own and own.all() and calls.made[-1][1][12] == vb.VATT_OUT_F32 and calls.made[-1][1][4].tolist() == [1, 2]
    wide = torch.zeros(2, 3, 12 * 64, dtype=torch.bfloat16)[..., :8 * 64].unflatten(-1, (8, 64))  # out of a fused projection
    s.attend(wide, dtype=torch.float32)
    assert calls.made[-1][1][2] == 12 * 64


def test_appended_tokens_end_what_the_last_write_says(monkeypatch):
    calls, s = Calls(monkeypatch, "vatt_write_kv", "vatt_chunk_attend", "vatt_append_kv", "vatt_append_kv_cached"), _session()
    monkeypatch.setattr(sm.vb, "vatt_chunk_workspace_bytes", lambda plan, n_new: 0)
    q, kv = (torch.zeros(2, 1, h, 64, dtype=torch.bfloat16) for h in (8, 2))
    for append in (s.append_device, s.append_device_cached):
        s.write(None, kv, kv)
        s.attend(q)
        assert calls.made[-1][1][11] is None  # no workspace
        append(kv[:, 0], kv[:, 0])
        with pytest.raises(ValueError):
            s.attend(q)
        s.attend(q, first=s.seq_lens - 1)


def test_a_session_checks_the_queries_of_window_decode(monkeypatch):
    calls, s = Calls(monkeypatch, "vatt_window_decode"), _session(3)
    q = torch.zeros(2, 3, 8, 64, dtype=torch.bfloat16)
    for bad in (4096, q[:1], q.float(), q[..., :32]):
        with pytest.raises(ValueError):
            s.window_decode(4, 10, bad)
    assert not calls.made
    s.window_decode(4, 10, q)
    assert calls.made[-1][1][1] is q and calls.made[-1][1][6:8] == (4, 10)
