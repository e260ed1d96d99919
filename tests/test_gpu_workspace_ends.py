"""Attention of new tokens and decode steps over a window keep to the workspace that they ask for: what lies behind it stays."""
import pytest
import torch

from test_gpu_cache_ops import Setup, _bf16
from test_gpu_new_tokens import SHARED, WINDOWS, _check_rows, _chunk, _decode_places, _stream, _window

pytestmark = pytest.mark.gpu

BEHIND, PATTERN = 1 << 20, 0xa5


def _workspace(need):
    ws = torch.full((need + BEHIND,), PATTERN, dtype=torch.uint8, device="cuda")
    return ws, ws[:need]


class Zeros(Setup):
    def random_cache(self):
        return torch.zeros(self.vb.vatt_kv_cache_bytes(self.plan), dtype=torch.uint8, device="cuda")


# Rows in pieces up to the room that there is: 700 and 2048 new tokens, all or few of them, on long rows; rests of tiles; halved pieces
WIDE = [(1, 32, 8, 128, 32768, 64, 0, 700, [32068], None, 0, 0), (1, 32, 8, 64, 32768, 0, 1, 2304, [30464], None, 0, 0),
        (5, 32, 8, 64, 16384, 0, 2, 256, [16128, 16100, 16000, 15000, 16128], None, 0, 0), (1, 32, 8, 128, 65536, 0, 0, 2048, [65000], [64], 0, 0),
        (9, 32, 8, 64, 8192, 16, 1, 256, [7936] * 9, None, 0, 0), (3, 32, 4, 128, 16384, 0, 0, 33, [16351, 9000, 5000], None, 0, 0)]


@pytest.mark.parametrize("case", SHARED + WIDE, ids=lambda c: "-".join(str(x) for x in c[:8]) + f"-{c[10]}-{c[11]}")
def test_chunk(case):
    batch, hq, hkv, d, n_max, page, fmt, n_new, first, new, sink, window = case
    s = Zeros(batch, hq, hkv, d, n_max, page, fmt, None, seed=1)
    q = torch.zeros(batch, n_new, hq, d, dtype=torch.bfloat16, device="cuda")
    need = s.vb.vatt_chunk_workspace_bytes(s.plan, n_new)
    buf, ws = _workspace(need)
    for bf16 in (False, True):
        o, lse = torch.empty(q.shape, dtype=torch.bfloat16 if bf16 else torch.float32, device="cuda"), torch.empty(q.shape[:3], device="cuda")
        s.vb.vatt_chunk_attend(s.plan, q, hq * d, n_new, s.ints(first), None if new is None else s.ints(new), s.k, s.v, s.table, sink, window,
                               ws if need else None, s.vb.VATT_OUT_BF16 if bf16 else s.vb.VATT_OUT_F32, o, lse, _stream())
    torch.cuda.synchronize()
    assert (buf[need:] == PATTERN).all()


PART = (1, 1, 1, 128, 700, 0, 0, 17, [700], 0, 700)  # (room for 102 of 126 workgroups)


@pytest.mark.parametrize("case", WINDOWS + [(1, 8, 8, 128, 8192, 0, 0, 1, [8192], 0, 8000), (1, 1, 1, 128, 9000, 0, 0, 1, [9000], 0, 9000),
                                            (1, 4, 4, 128, 16384, 0, 0, 1, [16384], 0, 16000), PART],
                         ids=lambda c: "-".join(str(x) for x in c[:8]) + f"-{c[9]}-{c[10]}")
def test_window_decode(case):
    batch, hq, hkv, d, n_max, page, fmt, q_len, lens, sink, window = case
    s = Zeros(batch, hq, hkv, d, n_max, page, fmt, None, q_len, seed=1, topk_frac=0.025, base_frac=0.025)
    q = torch.zeros(batch, q_len, hq, d, dtype=torch.bfloat16, device="cuda")
    need = s.vb.vatt_plan_workspace_bytes(s.plan)
    buf, ws = _workspace(need)
    o, lse = torch.empty(q.shape, device="cuda"), torch.empty(q.shape[:3], device="cuda")
    s.vb.vatt_window_decode(s.plan, q, s.k, s.v, s.table, s.ints(lens), sink, window, ws, o, lse, _stream())
    torch.cuda.synchronize()
    assert (buf[need:] == PATTERN).all()


@pytest.mark.parametrize("hq,hkv,d,n", [(8, 8, 128, 8192), (1, 1, 128, 9000), (4, 4, 128, 16384), (4, 2, 64, 3000), (32, 8, 128, 2000)])
def test_window_decode_has_room_for_all_workgroups(hq, hkv, d, n):
    """In the plan's workspace, which other calls size: the tokens are dealt out as vatt_chunk_attend does it in a workspace of its own, to the same bits."""
    s = Setup(1, hq, hkv, d, n, 0, 1, None, seed=n, topk_frac=0.025, base_frac=0.025)
    q = _bf16(s.rng.normal(size=(1, 1, hq, d)))
    o, lse = _window(s, q, [n], 0, n)
    _check_rows(s, q, [[n - 1]], 0, n, o, lse, False)
    for a, b in zip((o, lse), _chunk(s, q, [n - 1], None, 0, 0, False)):
        assert torch.equal(a, b)


def test_window_decode_with_room_for_a_part_of_the_workgroups():
    batch, hq, hkv, d, n_max, page, fmt, q_len, lens, sink, window = PART
    s = Setup(batch, hq, hkv, d, n_max, page, fmt, None, q_len, seed=1, topk_frac=0.025, base_frac=0.025)
    q = _bf16(s.rng.normal(size=(batch, q_len, hq, d)))
    _check_rows(s, q, _decode_places(s, lens), sink, window, *_window(s, q, lens, sink, window), False)
