"""Attention of new tokens over the cache (vatt_chunk_attend) and decode steps over a window and the first tokens
(vatt_window_decode) against the 64-bit oracle."""
import math

import numpy as np
import pytest
import torch

from oracle import cache_ops as co
from test_gpu_cache_ops import HALF_BF16, Setup, _bf16, _np

pytestmark = pytest.mark.gpu

FILL = 7.5  # what output rows hold that nobody writes
INF, NAN = math.inf, math.nan


def _stream():
    return torch.cuda.current_stream().cuda_stream


def _chunk(s, q, first, new, sink, window, bf16, stride=None, lse=True):
    batch, n_new = q.shape[:2]
    o = torch.full((batch, n_new, s.hq, s.d), FILL, dtype=torch.bfloat16 if bf16 else torch.float32, device="cuda")
    out_lse = torch.full((batch, n_new, s.hq), FILL, device="cuda") if lse else None
    need = s.vb.vatt_chunk_workspace_bytes(s.plan, n_new)
    ws = torch.full((need,), 255, dtype=torch.uint8, device="cuda") if need else None  # (NaN, in whatever way it is read)
    s.vb.vatt_chunk_attend(s.plan, q, stride or s.vb.token_stride(q), n_new, s.ints(first), None if new is None else s.ints(new), s.k, s.v, s.table,
                           sink, window, ws, s.vb.VATT_OUT_BF16 if bf16 else s.vb.VATT_OUT_F32, o, out_lse, _stream())
    torch.cuda.synchronize()
    return o, out_lse


def _close(got, want, size, bf16, at):
    """got against want for one row; size: the weighted mean of |V| per column.  32 bits: scores and weights as in vatt_dense_decode.  bf16:
    every weight off by half a step of bf16, then the result by half a step, with what 32 bits leave in between."""
    ok = np.isfinite(want)
    assert np.array_equal(got[~ok], want[~ok], equal_nan=True), at
    norm = np.linalg.norm(want[ok])
    if not bf16:
        assert np.linalg.norm(got[ok] - want[ok]) <= 2e-5 * norm, at
        return
    weights = HALF_BF16 * size[ok] + 2e-5 * norm
    assert (np.abs(got[ok] - want[ok]) <= weights + HALF_BF16 * (np.abs(want[ok]) + weights)).all(), at


def _check_rows(s, q, places, sink, window, o, lse, bf16, finite=True):
    """places[b]: positions of the query tokens of sequence b that count; q, o, lse [B, n_new, Hq, ..]."""
    qh, oh, lh = _np(q), _np(o), None if lse is None else _np(lse)
    g, scale = s.hq // s.hkv, s.params["sm_scale"] or 1 / math.sqrt(s.d)
    for b, ps in enumerate(places):
        rest = oh[b, len(ps):]
        assert (rest == FILL).all() and (lh is None or (lh[b, len(ps):] == FILL).all()), ("rows that do not count", b)
        for h in range(s.hkv if len(ps) else 0):
            n = max(ps) + 1
            k, v = s.rows(s.k, b, h, range(n)), s.rows(s.v, b, h, range(n))
            heads = slice(h * g, (h + 1) * g)
            if finite:  # all rows at once
                there = np.zeros((len(ps), n), dtype=bool)
                for t, p in enumerate(ps):
                    there[t, co.visible(p, sink, window)] = True
                x = scale * np.einsum("tgd,nd->tgn", qh[b, :len(ps), heads], k)
                x = np.where(there[:, None], x, -INF)
                m = x.max(-1, keepdims=True)
                w = np.exp(x - m)
                total = w.sum(-1, keepdims=True)
                want, size, ln = (w @ v) / total, (w @ np.abs(v)) / total, (m + np.log(total))[..., 0]
            for t, p in enumerate(ps):
                for j in range(g):
                    if finite:
                        a, z, e = want[t, j], size[t, j], ln[t, j]
                    else:
                        at = co.visible(p, sink, window)
                        with np.errstate(invalid="ignore", over="ignore"):
                            a, e = co.attend(qh[b, t, h * g + j], k[at], v[at], scale)
                            z = co.attend(qh[b, t, h * g + j], k[at], np.abs(v[at]), scale)[0]
                    where = (b, t, h * g + j)
                    _close(oh[b, t, h * g + j], a, z, bf16, where)
                    if lh is not None:
                        got = lh[b, t, h * g + j]
                        if math.isfinite(e):
                            assert abs(got - e) <= 2e-5 * max(1.0, abs(e)), where
                        else:
                            assert np.array_equal(got, e, equal_nan=True), where


def _places(s, first, new, n_new):
    new = [n_new] * s.batch if new is None else new
    return [list(range(f, f + co.new_tokens(f, m, n_new, s.n_max))) for f, m in zip(first, new)]


# ---- chunks --------------------------------------------------------------------------------------------------------------------

CHUNKS = [
    # (batch, hq, hkv, d, n_max, page, fmt, n_new, first, new_lens, sink, window)
    (1, 1, 1, 64, 1, 0, 0, 1, [0], None, 0, 0),                                    # one token, the first one
    (1, 1, 1, 128, 1, 8, 1, 1, [0], [1], 3, 1),
    (2, 4, 2, 128, 100, 0, 0, 1, [99, 0], None, 0, 0),
    (2, 4, 1, 128, 65, 0, 0, 65, [0, 0], [65, 64], 0, 0),                          # one key behind a tile's end
    (1, 8, 1, 64, 300, 16, 0, 300, [0], None, 0, 0),
    (3, 8, 2, 128, 333, 0, 0, 100, [233, 0, 97], [100, 0, 31], 0, 0),              # one without new tokens
    (4, 2, 2, 64, 200, 0, 0, 70, [150, -1, 200, 5], [70, 70, 70, -4], 0, 0),        # the end of the cache, firsts outside it
    (2, 16, 2, 128, 520, 64, 0, 33, [487, 200], None, 0, 0),                       # groups of 8
    (2, 4, 4, 64, 257, 0, 0, 257, [0, 0], [257, 129], 0, 0),                       # groups of 1
    (1, 4, 1, 128, 1000, 8, 0, 37, [963], None, 0, 0),                             # pages of 8
    (2, 4, 2, 128, 390, 16, 1, 190, [200, 3], None, 0, 0),
    (1, 8, 2, 64, 501, 0, 1, 501, [0], None, 0, 0),                                # scales of a contiguous cache
    (2, 4, 2, 128, 301, 0, 2, 150, [151, 20], [150, 77], 0, 0),
    (2, 8, 1, 64, 320, 256, 2, 20, [300, 17], None, 0, 0),
    (1, 4, 2, 128, 700, 0, 0, 700, [0], None, 4, 100),                             # windows: with first tokens, ...
    (2, 4, 2, 128, 640, 16, 0, 300, [340, 0], [300, 211], 130, 64),                # ... more than the window, beyond a tile
    (1, 8, 1, 64, 500, 0, 0, 200, [300], None, 0, 1),                              # ... each its own token only
    (1, 2, 2, 128, 500, 64, 1, 200, [300], None, 1, 1),
    (2, 4, 1, 128, 400, 0, 2, 130, [270, 0], None, 37, 65),
    (1, 4, 1, 64, 300, 0, 0, 300, [0], None, 0, 300),                              # as wide as the cache
    (1, 4, 1, 64, 300, 0, 0, 300, [0], None, 1 << 30, 5),                          # every token is a first one
    (1, 4, 1, 128, 300, 0, 0, 77, [200], None, 100, 1 << 30),
    (1, 2, 1, 128, 2000, 0, 0, 3, [1990], None, 0, 0),                             # few rows, many splits
    (1, 8, 1, 128, 3001, 32, 1, 5, [2996], None, 70, 1500),
    (1, 1, 1, 128, 130, 0, 0, 129, [1], None, 0, 0),                               # one row behind a tile of rows
    (40, 8, 8, 64, 64, 16, 0, 9, [(i * 37) % 64 for i in range(40)], [i % 10 for i in range(40)], 0, 0),
]


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("case", CHUNKS, ids=lambda c: "-".join(str(x) for x in c[:8]) + f"-{c[10]}-{c[11]}")
def test_chunk(case, bf16):
    batch, hq, hkv, d, n_max, page, fmt, n_new, first, new, sink, window = case
    s = Setup(batch, hq, hkv, d, n_max, page, fmt, None, seed=n_max + n_new)
    q = _bf16(s.rng.normal(size=(batch, n_new, hq, d)))
    o, lse = _chunk(s, q, first, new, sink, window, bf16)
    _check_rows(s, q, _places(s, first, new, n_new), sink, window, o, lse, bf16)


@pytest.mark.parametrize("bf16", [False, True])
def test_queries_of_a_fused_projection_and_no_lse(bf16):
    s = Setup(2, 4, 2, 128, 260, 0, 0, None, seed=1)
    x = _bf16(s.rng.normal(size=(2, 130, (4 + 2 + 2) * 128)))
    q = x[..., :4 * 128].unflatten(-1, (4, 128))
    o, _ = _chunk(s, q, [0, 130], None, 0, 0, bf16, lse=False)
    _check_rows(s, q, _places(s, [0, 130], None, 130), 0, 0, o, None, bf16)


@pytest.mark.parametrize("bf16", [False, True])
def test_few_queries_of_a_fused_projection(bf16):
    s = Setup(2, 4, 2, 64, 700, 16, 1, None, seed=17)
    x = _bf16(s.rng.normal(size=(2, 5, (4 + 2 + 2) * 64)))
    q = x[..., 2 * 64:6 * 64].unflatten(-1, (4, 64))
    o, lse = _chunk(s, q, [690, 17], [5, 2], 0, 0, bf16)
    _check_rows(s, q, _places(s, [690, 17], [5, 2], 5), 0, 0, o, lse, bf16)


@pytest.mark.parametrize("page", [0, 16])
def test_a_cache_in_host_memory(page):
    """K and V in pinned host memory: the same results, bit for bit."""
    s = Setup(2, 4, 2, 128, 400, page, 0, None, seed=18)
    q = _bf16(s.rng.normal(size=(2, 150, 4, 128)))
    one = q[:, 0].contiguous()
    res = []
    for host in (False, True):
        if host:
            kept = [torch.empty(x.shape, dtype=x.dtype, pin_memory=True).copy_(x) for x in (s.k, s.v)]
            s.k, s.v = (s.vb.vatt_host_kv_device_pointer(x) for x in kept)
        res.append([*_chunk(s, q, [250, 0], [150, 90], 0, 0, True), *_chunk(s, q, [250, 0], [150, 90], 3, 70, False),
                    *_chunk(s, q[:, :3].contiguous(), [397, 5], None, 0, 0, False), *_window(s, one, [400, 77], 5, 60)])
    assert all(torch.equal(a, b) for a, b in zip(*res))


class Large(Setup):
    """A cache of more than 4 GiB per buffer of which the last sequence (contiguous) or the last pages hold what small's first one does."""

    def __init__(self, small, batch, n_max, blocks):
        self.vb, self.rng, self.hq, self.hkv, self.d, self.fmt, self.page, self.q_len = small.vb, small.rng, small.hq, small.hkv, small.d, small.fmt, small.page, 1
        self.batch, self.n_max = batch, n_max
        self.params = dict(small.params, batch=batch, n_max=n_max, num_blocks=blocks)
        self.plan = self.vb.vatt_plan_create_chunk(self.params, 1, 0)
        self.vb.vatt_plan_set_option(self.plan, self.vb.VATT_OPT_KV_FORMAT, self.fmt)
        self.ws = torch.empty(self.vb.vatt_plan_workspace_bytes(self.plan), dtype=torch.uint8, device="cuda")
        self.table = small.table + (blocks - small.pages) if self.page else None
        row, ends = {0: 2 * self.d, 1: self.d, 2: self.d // 2}[self.fmt], self.d // 32
        for name in "kv":
            big = torch.zeros(self.vb.vatt_kv_cache_bytes(self.plan), dtype=torch.uint8, device="cuda")
            assert big.numel() > 1 << 32
            for x, s in ((big, self), (getattr(small, name), small)):
                off = self.vb.vatt_kv_scale_offset(s.plan)
                n8 = (s.n_max + 7) // 8 * 8
                shape = (s.pages if s is small else blocks, s.hkv, s.page) if s.page else (s.batch, s.hkv, s.n_max)
                scales = shape if s.page else (s.batch, s.hkv, n8)
                views = [x[:math.prod(shape) * row].view(*shape, row)]
                if self.fmt:
                    views.append(x[off:off + math.prod(scales) * ends].view(*scales, ends))
                if s is self:
                    into = views
            for a, b in zip(into, views):
                if self.page:
                    a[-small.pages:] = b
                else:
                    a[-1, :, :b.shape[2]] = b[0]
            setattr(self, name, big)


@pytest.mark.parametrize("page", [0, 16])
@pytest.mark.parametrize("fmt", [0, 1, 2])
def test_offsets_beyond_32_bits(fmt, page):
    s = Setup(1, 4, 2, 128, 600, page, fmt, None, seed=21)
    batch = 1 if page else (60, 104, 208)[fmt]
    big = Large(s, batch, 600 if page else 170752, (600000, 1100000, 2200000)[fmt] if page else 0)
    for n_new, bf16, sink, window in ((3, False, 0, 0), (70, True, 0, 0), (70, False, 5, 300)):
        q = torch.zeros(batch, n_new, 4, 128, dtype=torch.bfloat16, device="cuda")
        q[-1] = _bf16(s.rng.normal(size=(n_new, 4, 128)))
        o, lse = _chunk(big, q, [-1] * (batch - 1) + [600 - n_new], None, sink, window, bf16)
        _check_rows(s, q[-1:], [list(range(600 - n_new, 600))], sink, window, o[-1:], lse[-1:], bf16)
    q = torch.zeros(batch, 1, 4, 128, dtype=torch.bfloat16, device="cuda")
    q[-1] = _bf16(s.rng.normal(size=(1, 4, 128)))
    for sink, window in ((3, 200), (0, 900)):
        o, lse = _window(big, q, [1] * (batch - 1) + [600], sink, window)
        _check_rows(s, q[-1:], [[599]], sink, window, o[-1:], lse[-1:], False)


@pytest.mark.parametrize("scale", [0.01, 3.0])
@pytest.mark.parametrize("fmt", [0, 2])
def test_chunk_with_another_scale(scale, fmt):
    """Nearly uniform weights, and ones that the largest score has nearly alone (scores of some 100)."""
    s = Setup(1, 4, 2, 128, 400, 0, fmt, None, seed=2, sm_scale=scale)
    q = _bf16(s.rng.normal(size=(1, 200, 4, 128)))
    for bf16 in (False, True):
        o, lse = _chunk(s, q, [200], None, 3, 90, bf16)
        _check_rows(s, q, _places(s, [200], None, 200), 3, 90, o, lse, bf16)


def test_chunk_scores_far_apart():
    """Weights over the whole range of exp; the largest score first, last and in the middle, so that the running maximum moves often."""
    s = Setup(3, 2, 1, 64, 700, 0, 0, None, sm_scale=1.0)
    for b, at in enumerate((0, 350, 699)):
        for tok in range(700):
            s.set_row(s.k, b, 0, tok, values=np.full(64, -abs(tok - at) / 64.0 / 4.0))
    q = _bf16(np.ones((3, 100, 2, 64)) * np.array([1.0, 8.0])[:, None])
    for bf16 in (False, True):
        o, lse = _chunk(s, q, [600] * 3, None, 0, 0, bf16)
        _check_rows(s, q, _places(s, [600] * 3, None, 100), 0, 0, o, lse, bf16)


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("sink,window", [(0, 0), (5, 40)])
@pytest.mark.parametrize("page,n_new", [(0, 150), (16, 150), (0, 3)])
def test_infinity_and_nan_reach_only_the_queries_that_see_them(page, n_new, sink, window, bf16):
    s = Setup(2, 4, 2, 128, 336, page, 0, None, seed=5)
    n = [333, 190]
    first = [x - n_new for x in n]
    for b in range(2):
        for h in range(2):
            for tok, value in ((n[b] - 1, [INF, 1.0, NAN]), (n[b] - 2, [INF, -INF, 1.0]), (first[b] + 1, [-INF, 1.0, 1.0]), (3, [1.0, NAN, 1.0]),
                               (n[b] // 3, [1.0, 1.0, INF])):
                row = s.rng.normal(size=128)
                row[3:6] = value
                s.set_row(s.v, b, h, tok, values=row)
            for tok in range(n[b], min(n[b] + 70, 336)):  # behind the sequence
                s.set_row(s.v, b, h, tok, values=np.full(128, NAN))
                s.set_row(s.k, b, h, tok, values=np.full(128, INF))
            low = s.rng.normal(size=128)
            low[0] = -INF
            s.set_row(s.k, b, h, n[b] - n_new // 2, values=low)  # a score of -Inf
    q = s.rng.normal(size=(2, n_new, 4, 128))
    q[..., 0] = np.abs(q[..., 0]) + 0.1
    q = _bf16(q)
    o, lse = _chunk(s, q, first, None, sink, window, bf16)
    _check_rows(s, q, _places(s, first, None, n_new), sink, window, o, lse, bf16, finite=False)


@pytest.mark.parametrize("fmt", [1, 2])
def test_groups_that_are_nan_reach_only_the_queries_that_see_them(fmt):
    s = Setup(1, 4, 1, 128, 203, 0, fmt, None, seed=6)
    odd = np.array([120, 255, 120, 120], dtype=np.uint8)
    s.set_row(s.v, 0, 0, 150, scales=odd)
    s.set_row(s.v, 0, 0, 202, scales=odd)
    s.set_row(s.k, 0, 0, 180, scales=odd)
    q = _bf16(s.rng.normal(size=(1, 100, 4, 128)))
    for window in (0, 12):
        for bf16 in (False, True):
            o, lse = _chunk(s, q, [100], [90], 0, window, bf16)
            _check_rows(s, q, _places(s, [100], [90], 100), 0, window, o, lse, bf16, finite=False)


def test_first_scores_all_minus_infinity():
    """A query all of whose scores are -Inf has no softmax (NaN); one that sees a finite score as well has its value."""
    s = Setup(1, 2, 1, 64, 200, 0, 0, None, seed=7)
    for tok in range(0, 130):
        row = s.rng.normal(size=64)
        row[0] = -INF
        s.set_row(s.k, 0, 0, tok, values=row)
    q = s.rng.normal(size=(1, 140, 2, 64))
    q[..., 0] = np.abs(q[..., 0]) + 0.1
    q = _bf16(q)
    for bf16 in (False, True):
        o, lse = _chunk(s, q, [60], None, 0, 0, bf16)
        _check_rows(s, q, _places(s, [60], None, 140), 0, 0, o, lse, bf16, finite=False)


# (batch, hq, hkv, d, n_max, page, fmt, n_new, first, new_lens, sink, window)
SHARED = [
    # tiles that are cut into pieces: one long sequence, the same among short ones, in a window, with a last piece of one tile
    (1, 4, 1, 128, 4000, 16, 0, 33, [3967], None, 0, 0),
    (3, 4, 2, 64, 6000, 0, 1, 40, [5960, 100, 3], [40, 40, 0], 0, 0),
    (2, 8, 1, 128, 3500, 64, 2, 70, [3430, 900], [70, 3], 300, 2500),
    (1, 2, 1, 64, 5001, 0, 0, 200, [4801], [131], 0, 0),
    # the same sizes with few new tokens: the kernel of the decode steps, in several workgroups
    (1, 4, 1, 128, 4000, 16, 0, 8, [3991], None, 0, 0), (3, 4, 2, 64, 6000, 0, 1, 3, [5960, 100, 3], [2, 3, 0], 0, 0),
    (2, 8, 1, 128, 3500, 64, 2, 4, [3430, 900], [4, 3], 300, 2500), (2, 1, 1, 64, 5001, 0, 0, 17, [4984, 17], None, 0, 0),
    # ... of which some have none, dealt out over several waves' lanes, and more than there are threads
    (70, 4, 2, 64, 900, 16, 1, 2, [(i * 137) % 930 - 10 for i in range(70)], [i % 3 for i in range(70)], 0, 0),
    (200, 2, 1, 64, 700, 0, 0, 1, [(i * 37) % 700 for i in range(200)], None, 0, 0), (270, 2, 1, 64, 700, 0, 2, 1, [(i * 37) % 700 for i in range(270)], None, 5, 660),
    (3, 4, 1, 128, 1000, 0, 0, 1, [-1, 1000, 999], None, 0, 0), (2, 4, 1, 128, 1000, 0, 0, 1, [500, 999], [0, 0], 0, 0),
    (1, 4, 1, 128, 1000, 0, 0, 2, [500], [0], 0, 0),
    # ... four KV heads with 202 and 239 pieces of 128 tokens each, for 504 workgroups: shares of two pieces, one head in 102 to 121 of them
    (1, 4, 4, 64, 25856, 16, 1, 1, [25855], None, 0, 0), (1, 4, 4, 64, 30600, 0, 0, 1, [30591], None, 0, 0),
    # more tiles than run at a time, and a rest that is cut: of one tile per KV head, of a few sequences, in a window
    (1, 64, 8, 64, 2640, 0, 0, 1040, [1600], None, 0, 0), (5, 64, 8, 64, 1900, 16, 1, 230, [1600, 1670, 1590, 1600, 1655], [230, 230, 229, 230, 225], 0, 0),
    (1, 64, 8, 64, 2700, 0, 2, 1090, [1600], [1087], 30, 1570),
    # ... and tiles whose pieces, rounded to the nearest number, would be a few too many
    (1, 16, 2, 64, 9000, 0, 0, 600, [8400], None, 0, 0), (3, 16, 4, 64, 2600, 0, 0, 230, [2370, 2000, 2200], None, 0, 0),
    # more sequences than a wave has lanes, and than it looks through
    (130, 2, 2, 64, 96, 16, 0, 33, [(i * 37) % 90 for i in range(130)], [(i * 5) % 34 for i in range(130)], 0, 0),
    (300, 4, 1, 64, 64, 0, 1, 20, [(i * 37) % 60 - 1 for i in range(300)], [(i * 7) % 21 for i in range(300)], 2, 9),
    (260, 8, 1, 64, 90, 0, 0, 50, [(i * 37) % 90 - 1 for i in range(260)], [(i * 7) % 51 for i in range(260)], 0, 0),
]


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("case", SHARED, ids=lambda c: "-".join(str(x) for x in c[:8]) + f"-{c[10]}-{c[11]}")
def test_chunk_of_shared_work(case, bf16):
    batch, hq, hkv, d, n_max, page, fmt, n_new, first, new, sink, window = case
    s = Setup(batch, hq, hkv, d, n_max, page, fmt, None, seed=n_max + n_new)
    q = _bf16(s.rng.normal(size=(batch, n_new, hq, d)))
    o, lse = _chunk(s, q, first, new, sink, window, bf16)
    _check_rows(s, q, _places(s, first, new, n_new), sink, window, o, lse, bf16)


@pytest.mark.parametrize("n_new", [3, 40])
def test_infinity_and_nan_in_pieces(n_new):
    """As above, where several workgroups have the keys: pieces that a NaN lies in, and pieces that it does not reach."""
    s = Setup(1, 4, 1, 128, 3000, 0, 0, None, seed=14)
    for tok, value in ((2999, [INF, 1.0, NAN]), (2998, [INF, -INF, 1.0]), (1500, [1.0, NAN, 1.0]), (70, [-INF, 1.0, 1.0])):
        row = s.rng.normal(size=128)
        row[3:6] = value
        s.set_row(s.v, 0, 0, tok, values=row)
    s.set_row(s.k, 0, 0, 1000, values=np.full(128, NAN))
    q = _bf16(s.rng.normal(size=(1, n_new, 4, 128)))
    for sink, window in ((0, 0), (60, 1400), (71, 1450), (0, 1900)):
        for bf16 in (False, True):
            o, lse = _chunk(s, q, [3000 - n_new], None, sink, window, bf16)
            _check_rows(s, q, _places(s, [3000 - n_new], None, n_new), sink, window, o, lse, bf16, finite=False)


# ---- decode steps over a window --------------------------------------------------------------------------------------------------

WINDOWS = [
    # (batch, hq, hkv, d, n_max, page, fmt, q_len, lens, sink, window)
    (1, 1, 1, 64, 1, 0, 0, 1, [1], 0, 1), (2, 4, 2, 128, 100, 0, 0, 1, [100, 3], 4, 10), (2, 8, 2, 128, 600, 16, 0, 1, [600, 77], 128, 128),
    (3, 8, 1, 64, 700, 0, 0, 1, [700, 129, 9], 0, 200), (2, 4, 4, 128, 640, 64, 1, 1, [640, 333], 7, 1), (2, 4, 1, 64, 500, 0, 2, 1, [499, 500], 9, 255),
    (2, 8, 2, 128, 401, 0, 0, 4, [401, 3], 5, 30), (1, 8, 1, 128, 300, 8, 0, 5, [299], 16, 17), (2, 4, 2, 64, 350, 16, 1, 17, [350, 40], 3, 33),
    (1, 8, 1, 128, 900, 0, 2, 12, [899], 70, 500), (1, 2, 1, 128, 1000, 256, 0, 40, [998], 1, 300), (2, 2, 2, 64, 150, 0, 1, 3, [150, 2], 200, 4),
    (1, 4, 1, 128, 9000, 0, 0, 1, [8999], 4, 4096), (1, 4, 1, 64, 170752, 64, 1, 1, [170752], 128, 128), (2, 2, 1, 64, 300, 0, 0, 2, [300, 299], 0, 1 << 30),
    (40, 2, 1, 64, 64, 16, 1, 1, [1 + (i * 37) % 64 for i in range(40)], 2, 7), (1, 4, 4, 128, 64, 0, 0, 1, [64], 1 << 30, 1),
    # several workgroups for a sequence's tokens
    (2, 4, 1, 128, 3000, 16, 1, 1, [3000, 700], 128, 1000), (2, 8, 1, 64, 3000, 0, 2, 1, [2999, 5], 0, 2000), (1, 8, 2, 128, 2500, 64, 0, 2, [2500], 300, 900),
    (2, 4, 2, 64, 2000, 0, 0, 11, [2000, 1300], 37, 700), (1, 2, 2, 128, 2000, 8, 2, 3, [1999], 5, 1500), (2, 4, 4, 64, 1500, 0, 1, 7, [1500, 3], 0, 1 << 30),
    (70, 8, 8, 64, 700, 0, 0, 1, [1 + (i * 137) % 700 for i in range(70)], 9, 690),
    # ... dealt out over sequences of several waves' lanes, and more than there are threads
    (40, 4, 4, 64, 700, 0, 1, 1, [1 + (i * 137) % 700 for i in range(40)], 9, 690), (200, 2, 1, 64, 800, 16, 0, 1, [1 + (i * 317) % 800 for i in range(200)], 0, 700),
    (300, 2, 2, 64, 800, 0, 2, 1, [1 + (i * 317) % 800 for i in range(300)], 3, 650), (1, 4, 4, 64, 30600, 16, 2, 1, [30600], 100, 25700), (5, 4, 1, 128, 2000, 64, 0, 9, [1999, 9, 2000, 700, 1], 40, 1300),
]


def _window(s, q, lens, sink, window, lse=True):
    o = torch.full((s.batch, s.q_len, s.hq, s.d), FILL, device="cuda")
    out_lse = torch.full((s.batch, s.q_len, s.hq), FILL, device="cuda") if lse else None
    s.ws.fill_(255)
    s.vb.vatt_window_decode(s.plan, q, s.k, s.v, s.table, s.ints(lens), sink, window, s.ws, o, out_lse, _stream())
    torch.cuda.synchronize()
    return o, out_lse


def _decode_places(s, lens):
    return [[max(n - s.q_len + t, 0) for t in range(s.q_len)] for n in lens]


@pytest.mark.parametrize("case", WINDOWS, ids=lambda c: "-".join(str(x) for x in c[:8]) + f"-{c[9]}-{c[10]}")
def test_window_decode(case):
    batch, hq, hkv, d, n_max, page, fmt, q_len, lens, sink, window = case
    s = Setup(batch, hq, hkv, d, n_max, page, fmt, None, q_len, seed=n_max + q_len)
    q = _bf16(s.rng.normal(size=(batch, q_len, hq, d)))
    o, lse = _window(s, q, lens, sink, window)
    _check_rows(s, q, _decode_places(s, lens), sink, window, o, lse, False)


@pytest.mark.parametrize("q_len", [1, 6])
@pytest.mark.parametrize("page", [0, 16])
def test_window_decode_infinity_and_nan(page, q_len):
    s = Setup(2, 4, 2, 128, 336, page, 0, None, q_len, seed=8)
    lens = [333, 90]
    for b, n in enumerate(lens):
        for h in range(2):
            for tok, value in ((n - 1, [INF, 1.0, NAN]), (n - 30, [INF, -INF, 1.0]), (n - 31, [1.0, NAN, 1.0]), (3, [-INF, 1.0, 1.0]), (12, [NAN, NAN, NAN])):
                row = s.rng.normal(size=128)
                row[3:6] = value
                s.set_row(s.v, b, h, tok, values=row)
            for tok in range(n, min(n + 16, 336)):
                s.set_row(s.v, b, h, tok, values=np.full(128, NAN))
                s.set_row(s.k, b, h, tok, values=np.full(128, INF))
            s.set_row(s.k, b, h, 13, values=np.full(128, NAN))  # between the first tokens and the window
    q = _bf16(s.rng.normal(size=(2, q_len, 4, 128)))
    for sink, window in ((4, 30), (11, 25), (0, 1), (0, 29)):
        o, lse = _window(s, q, lens, sink, window)
        _check_rows(s, q, _decode_places(s, lens), sink, window, o, lse, False, finite=False)


@pytest.mark.parametrize("q_len", [1, 2, 6])
def test_window_decode_infinity_and_nan_in_pieces(q_len):
    s = Setup(1, 4, 1, 128, 3000, 0, 0, None, q_len, seed=15)
    for tok, value in ((2999, [INF, 1.0, NAN]), (2000, [1.0, NAN, 1.0]), (5, [-INF, 1.0, 1.0])):
        row = s.rng.normal(size=128)
        row[3:6] = value
        s.set_row(s.v, 0, 0, tok, values=row)
    s.set_row(s.k, 0, 0, 1200, values=np.full(128, NAN))
    low = s.rng.normal(size=128)
    low[0] = -INF
    s.set_row(s.k, 0, 0, 2500, values=low)
    q = s.rng.normal(size=(1, q_len, 4, 128))
    q[..., 0] = np.abs(q[..., 0]) + 0.1
    q = _bf16(q)
    for lens in ([2999], [3000]):
        for sink, window in ((4, 900), (6, 1700), (0, 998), (0, 1802)):
            o, lse = _window(s, q, lens, sink, window)
            _check_rows(s, q, _decode_places(s, lens), sink, window, o, lse, False, finite=False)


def test_windows_as_wide_as_the_sequence_are_dense_attention():
    s = Setup(2, 8, 2, 128, 512, 16, 0, None, 3, seed=9)
    q, lens = _bf16(s.rng.normal(size=(2, 3, 8, 128))), [500, 77]
    o, lse = _window(s, q, lens, 0, 512)
    do, dlse = torch.empty_like(o), torch.empty_like(lse)
    s.vb.vatt_dense_decode(s.plan, q, s.k, s.v, s.table, s.ints(lens), s.ws, do, dlse, _stream())
    co_, clse = _chunk(s, q, [497, 74], None, 0, 0, False)
    torch.cuda.synchronize()
    for a, b in ((o, do), (lse, dlse), (co_, do), (clse, dlse)):
        assert float((a - b).norm() / b.norm()) < 1e-5


# ---- together ------------------------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("fmt,page", [(0, 0), (0, 64), (1, 16), (2, 0)])
def test_a_prompt_in_pieces_then_tokens(fmt, page):
    """A ragged prompt written and attended to in two pieces gives what it gives whole; single tokens follow, windowed and not."""
    rot = dict(theta=10000.0)
    s, whole = (Setup(2, 8, 2, 128, 640, page, fmt, None, rotary=rot, seed=10) for _ in range(2))
    x = [_bf16(s.rng.normal(size=(2, 400, h, 128))) for h in (8, 2, 2)]
    lens, got = [370, 201], []

    def piece(c, t0, t1, first, new, sink, window):
        part = [t[:, t0:t1].contiguous() for t in x]
        out_q = torch.zeros_like(part[0])
        c.write(*part, c.ints(first), c.ints(new), None, out_q, None)
        return out_q, [_chunk(c, out_q, first, new, sink, w, False) for w in (0, window)]

    q, all_at_once = piece(whole, 0, 400, [0, 0], lens, 4, 90)
    for t0, t1 in ((0, 150), (150, 400)):
        got.append(piece(s, t0, t1, [t0, t0], [max(min(n, t1) - t0, 0) for n in lens], 4, 90)[1])
    for w in range(2):
        for b, n in enumerate(lens):
            for y in range(2):
                one, two = all_at_once[w][y][b, :n], torch.cat([g[w][y][b] for g in got])[:n]
                assert float((one - two).norm() / one.norm()) < 1e-5
    _check_rows(whole, q, _places(whole, [0, 0], lens, 400), 4, 90, *all_at_once[1], False)
    for t in range(2):
        first = [n + t for n in lens]
        out_q, (dense, windowed) = piece(s, t, t + 1, first, [1, 1], 4, 90)
        o, lse = _window(s, out_q, [f + 1 for f in first], 4, 90)
        for a, b in ((o, windowed[0]), (lse, windowed[1])):
            assert float((a - b).norm() / b.norm()) < 1e-5
        _check_rows(s, out_q, [[f] for f in first], 0, 0, *dense, False)


@pytest.mark.parametrize("fmt,page,n_new", [(1, 16, 40), (0, 0, 1), (0, 0, 150)])
def test_captured(fmt, page, n_new):
    """Write, chunk and windowed step captured once and replayed with other inputs in the same buffers, the program's own work between."""
    s = Setup(3, 8, 2, 128, 512, page, fmt, None, rotary=dict(theta=10000.0), seed=11)
    x = [_bf16(s.rng.normal(size=(3, n_new, h, 128))) for h in (8, 2, 2)]
    first, new, after = s.ints([300, 17, 255]), s.ints([n_new, n_new // 2, n_new]), s.ints([0, 0, 0])
    out_q = torch.zeros_like(x[0])
    last = torch.zeros((3, 8, 128), dtype=torch.bfloat16, device="cuda")
    need = s.vb.vatt_chunk_workspace_bytes(s.plan, n_new)
    ws = torch.empty(max(need, 256), dtype=torch.uint8, device="cuda")
    o, lse = torch.zeros((3, n_new, 8, 128), device="cuda"), torch.zeros((3, n_new, 8), device="cuda")
    wo, wlse = torch.zeros((3, 8, 128), device="cuda"), torch.zeros((3, 8), device="cuda")

    def step():
        st = _stream()
        s.write(*x, first, new, None, out_q, after)
        s.vb.vatt_chunk_attend(s.plan, out_q, 8 * 128, n_new, first, new, s.k, s.v, s.table, 4, 100, ws, s.vb.VATT_OUT_F32, o, lse, st)
        last.copy_(out_q[:, 0])
        s.vb.vatt_window_decode(s.plan, last, s.k, s.v, s.table, after, 4, 33, s.ws, wo, wlse, st)

    outs = (out_q, after, o, lse, wo, wlse)
    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for i in range(4):
        for t in x:
            t.copy_(_bf16(s.rng.normal(size=tuple(t.shape))))
        first.copy_(s.ints([300 + i, 17 + 3 * i, 255 + 30 * i]))
        for t in (o, lse, wo, wlse):
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in outs]
        for t in (o, lse, wo, wlse):
            t.zero_()
        step()
        torch.cuda.synchronize()
        for a, b in zip(got, outs):
            assert torch.equal(a, b)


def test_another_stream():
    s = Setup(2, 8, 2, 128, 512, 0, 1, None, seed=12)
    q = _bf16(s.rng.normal(size=(2, 70, 8, 128)))
    one = _bf16(s.rng.normal(size=(2, 1, 8, 128)))
    side, res = torch.cuda.Stream(), []
    for stream in (torch.cuda.current_stream(), side):
        stream.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(stream):
            res.append([*_chunk(s, q, [400, 3], [70, 50], 0, 0, True), *_window(s, one, [470, 53], 4, 50)])
        stream.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(*res))


def test_calls_at_once():
    """Calls of one plan under way on two streams, each with its own workspace: what each gives alone."""
    s = Setup(2, 8, 2, 128, 4000, 16, 1, None, seed=22)
    q = [_bf16(s.rng.normal(size=(2, n, 8, 128))) for n in (40, 3)]
    firsts = [s.ints([3900, 1200]), s.ints([3990, 2100])]
    lens = s.ints([4000, 2500])

    def calls(i, o, ws, st):
        s.vb.vatt_chunk_attend(s.plan, q[i], 8 * 128, q[i].shape[1], firsts[i], None, s.k, s.v, s.table, 0, 0, ws[0], s.vb.VATT_OUT_F32, o[0], o[1], st)
        s.vb.vatt_window_decode(s.plan, q[i], s.k, s.v, s.table, lens, 9, 900 + i, ws[1], o[2], o[3], st)

    sides = [torch.cuda.Stream() for _ in range(2)]
    outs = [[[torch.zeros(2, x.shape[1], 8, 128, device="cuda"), torch.zeros(2, x.shape[1], 8, device="cuda"), torch.zeros(2, 8, 128, device="cuda"),
              torch.zeros(2, 8, device="cuda")] for x in q] for _ in range(2)]
    ws = [[torch.empty(s.vb.vatt_chunk_workspace_bytes(s.plan, x.shape[1]), dtype=torch.uint8, device="cuda"), torch.empty_like(s.ws)] for x in q]
    torch.cuda.synchronize()
    for i in range(2):
        calls(i, outs[0][i], ws[i], _stream())
        torch.cuda.synchronize()
    for _ in range(20):
        for i in range(2):
            calls(i, outs[1][i], ws[i], sides[i].cuda_stream)
    torch.cuda.synchronize()
    for a, b in zip(outs[0], outs[1]):
        assert all(torch.equal(x, y) for x, y in zip(a, b))


@pytest.mark.parametrize("n_new", [2, 40])
def test_as_many_sequences_as_a_plan_takes(n_new):
    s = Setup(65535, 1, 1, 64, 48, 0, 0, None, seed=23)
    q = torch.randn(65535, n_new, 1, 64, device="cuda", generator=torch.Generator("cuda").manual_seed(3)).to(torch.bfloat16)
    first = torch.arange(65535, device="cuda", dtype=torch.int32) * 7 % (49 - n_new)
    o, lse = torch.zeros(q.shape, device="cuda"), torch.zeros(q.shape[:3], device="cuda")
    need = s.vb.vatt_chunk_workspace_bytes(s.plan, n_new)
    assert need == 0
    s.vb.vatt_chunk_attend(s.plan, q, 64, n_new, first, None, s.k, s.v, None, 3, 30, None, s.vb.VATT_OUT_F32, o, lse, _stream())
    wo, wlse = torch.zeros(65535, 1, 64, device="cuda"), torch.zeros(65535, 1, device="cuda")
    one, lens = q[:, 0].contiguous(), first + 1
    s.vb.vatt_window_decode(s.plan, one, s.k, s.v, None, lens, 3, 30, s.ws, wo, wlse, _stream())
    torch.cuda.synchronize()
    for b0 in range(0, 65535, 8192):
        b = slice(b0, b0 + 8192)
        k, v = (x.view(torch.bfloat16).view(65535, 48, 64)[b].double().cpu() for x in (s.k, s.v))
        p = (first[b, None] + torch.arange(n_new, device="cuda")).cpu()[..., None]
        i = torch.arange(48)
        x = torch.bmm(q[b, :, 0].double().cpu(), k.transpose(1, 2).contiguous()) / 8
        x = x.masked_fill(~((i <= p) & ((i < 3) | (i > p - 30))), -INF)
        want, ln = torch.bmm(x.softmax(-1), v), x.logsumexp(-1)
        for got, exp in ((o[b, :, 0], want), (wo[b], want[:, :1])):
            assert ((got.double().cpu() - exp).norm(dim=-1) <= 2e-5 * exp.norm(dim=-1)).all(), b0
        for got, exp in ((lse[b, :, 0], ln), (wlse[b], ln[:, :1])):
            assert ((got.double().cpu() - exp).abs() <= 2e-5 * exp.abs().clamp(min=1)).all(), b0


@pytest.mark.parametrize("fmt", [0, 1])
def test_a_session(fmt):
    """As a program does it through DecodeSession: a ragged prompt, a second piece, then tokens over all rows and over a window."""
    from paper_2510_05688_amd.session import DecodeSession
    s = Setup(2, 8, 2, 128, 256, 32, fmt, None, rotary=dict(theta=10000.0), seed=13)
    sess = DecodeSession(s.params, kv_format=fmt, rotary=dict(theta=10000.0)).make_cache(s.table.cpu().numpy())
    s.k, s.v = sess.k, sess.v
    x = [_bf16(s.rng.normal(size=(2, 210, h, 128))) for h in (8, 2, 2)]

    def check(q, places, sink, window, o, lse):
        whole = [t.float().clone() for t in (o, lse)]
        for b, ps in enumerate(places):
            assert not o[b, len(ps):].any() and not lse[b, len(ps):].any()
            for t in whole:
                t[b, len(ps):] = FILL
        _check_rows(s, q, places, sink, window, *whole, o.dtype == torch.bfloat16)

    new = s.ints([130, 77])
    q = sess.write(*[t[:, :130].contiguous() for t in x], new)
    check(q, [range(130), range(77)], 0, 0, *sess.attend(q, new))
    check(q, [range(130), range(77)], 4, 50, *sess.attend(q, new, 4, 50, torch.float32))
    q = sess.write(*[t[:, 130:190].contiguous() for t in x])
    assert sess.seq_lens.tolist() == [190, 137] and sess.first.tolist() == [130, 77]
    check(q, [range(130, 190), range(77, 137)], 0, 0, *sess.attend(q))
    for t in range(190, 193):
        q = sess.write(*[y[:, t:t + 1].contiguous() for y in x])
        o, lse = sess.attend(q, dtype=torch.float32)
        sess.dense(q)
        assert float((o.view(2, 8, 128) - sess.dense_o).norm() / sess.dense_o.norm()) < 1e-5
        sess.window_decode(4, 50, q)
    check(q, [[192], [139]], 4, 50, sess.out_o[:, None], sess.out_lse[:, None])
    sess.close()


def test_a_session_captured():
    """A token's write, attention over all rows and over a window through DecodeSession, captured once: every replay goes on where the last
    one ended."""
    from paper_2510_05688_amd.session import DecodeSession
    s = Setup(2, 8, 2, 128, 256, 32, 1, None, rotary=dict(theta=10000.0), seed=21)
    table = s.table.cpu().numpy()
    one, two = (DecodeSession(s.params, kv_format=1, rotary=dict(theta=10000.0)).make_cache(table) for _ in range(2))
    x = [_bf16(s.rng.normal(size=(2, 150, h, 128))) for h in (8, 2, 2)]
    now = [t[:, :3].clone() for t in x]
    outs = [[torch.zeros(2, 3, 8, 128, device="cuda"), torch.zeros(2, 3, 8, device="cuda")] for _ in range(2)]

    def step(sess, out):
        q = sess.write(*now)
        sess.attend(q, out=out[0], lse=out[1])
        sess.window_decode(2, 40, q[:, 2].contiguous())

    for sess, out in zip((one, two), outs):
        sess.write(*x, s.ints([150, 93]))
        step(sess, out)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(one, outs[0])
    for i in range(4):
        for t in now:
            t.copy_(_bf16(s.rng.normal(size=tuple(t.shape))))
        graph.replay()
        step(two, outs[1])
        torch.cuda.synchronize()
        assert one.seq_lens.tolist() == two.seq_lens.tolist() == [156 + 3 * i, 99 + 3 * i]
        for a, b in zip((*outs[0], one.out_o, one.out_lse, one.k), (*outs[1], two.out_o, two.out_lse, two.k)):
            assert torch.equal(a, b)
