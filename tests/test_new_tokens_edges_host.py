"""Attention of new tokens without a GPU: refused addresses, and what DecodeSession hands on."""
import pytest
import torch  # (before the library: the HIP runtime that both use is the one that comes with it)

from paper_2510_05688_amd import binding as vb
from test_cache_ops_host import ARG, NO_DEVICE, Mem, _plan, _status


@pytest.mark.parametrize("at", [4, 8, 12])
def test_window_decode_refuses_an_output_that_its_stores_cannot_write(at):
    """Results of a workgroup that has a sequence alone go out 16 bytes at a time."""
    plan, m = _plan(), Mem()
    call = [m, m, m, None, m, 4, 10, m, Mem(8192), m]
    assert _status(vb.vatt_window_decode, plan, *call) == NO_DEVICE  # nothing else is wrong with it
    assert _status(vb.vatt_window_decode, plan, *(call[:8] + [Mem(8192 + at)] + call[9:])) == ARG
    assert _status(vb.vatt_window_decode, plan, *(call[:9] + [Mem(8192 + 4)])) == NO_DEVICE  # lse is written value by value
    vb.vatt_plan_destroy(plan)
