"""Attention of new tokens without a GPU: refused addresses, and what DecodeSession hands on."""
import pytest
import torch  # (before the library: the HIP runtime that both use is the one that comes with it)

from paper_2510_05688_amd import binding as vb
from paper_2510_05688_amd import session as sm
from test_cache_ops_host import ARG, NO_DEVICE, Mem, _plan, _status
from test_session_host import _ints, _session


@pytest.mark.parametrize("at", [4, 8, 12])
def test_window_decode_refuses_an_output_that_its_stores_cannot_write(at):
    """Results of a workgroup that has a sequence alone go out 16 bytes at a time."""
    plan, m = _plan(), Mem()
    call = [m, m, m, None, m, 4, 10, m, Mem(8192), m]
    assert _status(vb.vatt_window_decode, plan, *call) == NO_DEVICE  # nothing else is wrong with it
    assert _status(vb.vatt_window_decode, plan, *(call[:8] + [Mem(8192 + at)] + call[9:])) == ARG
    assert _status(vb.vatt_window_decode, plan, *(call[:9] + [Mem(8192 + 4)])) == NO_DEVICE  # lse is written value by value
    vb.vatt_plan_destroy(plan)


@pytest.mark.parametrize("which", ["seq_lens", "first", "part of one buffer"])
def test_write_takes_its_own_lengths_for_new_lens(monkeypatch, which):
    """As many new tokens as there are: seq_lens is what the call writes to, so that it gets a copy."""
    s = _session()
    kv = torch.zeros(2, 60, 2, 64, dtype=torch.bfloat16)
    made = []

    def write_kv(*a):
        made.append(a)
        first, new_lens, after = a[8], a[9], a[15]
        ends = {x.data_ptr(): x.data_ptr() + 4 * x.numel() for x in (first, after, new_lens)}
        assert len(ends) == 3 and all(not (p < e and q < f) for q, e in ends.items() for p, f in ends.items() if p > q)
        after.copy_(first + new_lens)

    monkeypatch.setattr(sm.vb, "vatt_write_kv", write_kv)
    s.write(None, kv, kv, _ints(5, 7))
    assert s.seq_lens.tolist() == [55, 57] and s.first.tolist() == [50, 50]
    if which == "part of one buffer":
        both = _ints(55, 57, 4)
        s.seq_lens, new = both[:2], both[1:]
    else:
        new = getattr(s, which)
    want = new.tolist()
    s.write(None, kv, kv, new)
    assert made[-1][9].tolist() == want and s.first.tolist() == [55, 57]
    assert s.seq_lens.tolist() == [55 + want[0], 57 + want[1]]
    other = _ints(1, 2)
    s.write(None, kv, kv, other)
    assert made[-1][9] is other  # (no copy where none is needed)
