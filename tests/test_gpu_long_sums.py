"""Attention over very many tokens of equal weight, where every rounding of a running sum can go the same way: 32-bit outputs and lse keep
the tolerance of the other tests however long a row is."""
import math

import pytest
import torch

from test_gpu_cache_ops import Setup

pytestmark = pytest.mark.gpu

LN2 = math.log(2.0)
# Outputs and lse as in the other tests of 32-bit results: 2e-5 of a row's norm, and of lse (or of 1).
TOL = 2e-5


class Even(Setup):
    """Every sequence has the same n tokens (paged: the same pages).  K is 0 but for the first token, whose first column is 1; a column of V is the
    same for all tokens."""

    def __init__(self, batch, hq, hkv, d, n, page=0, fmt=0, q_len=1, odd=()):
        super().__init__(batch, hq, hkv, d, n, page, fmt, None, q_len, sm_scale=1.0, **(dict(num_blocks=-(-n // page)) if page else {}))
        if page:
            self.table = torch.arange(-(-n // page), dtype=torch.int32, device="cuda").expand(batch, -1).contiguous()
        row = {0: 2 * d, 1: d, 2: d // 2}[fmt]
        off = self.vb.vatt_kv_scale_offset(self.plan)
        one, some = {0: ([0x80, 0x3f], [0x33, 0x3f, 0xa0, 0x3f]), 1: ([0x38], [0x33, 0x3a]), 2: ([0x02], [0x31, 0x23])}[fmt]  # 1; two values of V
        k, v = (x[:off // row * row].view(-1, row) for x in (self.k, self.v))
        v[:] = torch.tensor(some * (row // len(some)), dtype=torch.uint8, device="cuda")
        if fmt:
            self.k[off:], self.v[off:] = 127, 127
        starts = [h * page for h in range(hkv)] if page else [i * n for i in range(batch * hkv)]
        for at in starts:
            k[at, :len(one)] = torch.tensor(one, dtype=torch.uint8, device="cuda")
        for tok in odd:  # (rows of V that are NaN)
            v[torch.tensor(starts, device="cuda") + tok] = 255
        self.value = {0: [0.69921875, 1.25], 1: [0.6875, 1.25], 2: [0.5, 1.5, 1.5, 1.0]}[fmt]

    def random_cache(self):
        return torch.zeros(self.vb.vatt_kv_cache_bytes(self.plan), dtype=torch.uint8, device="cuda")

    def queries(self, batch, n_new):
        """The first token's weight is 2^x times another's, x from 0 to 8, a different one for every query."""
        count = batch * n_new * self.hq
        q = torch.zeros(batch, n_new, self.hq, self.d, device="cuda")
        q[..., 0] = (torch.arange(count, device="cuda") * (8.0 / count) * LN2).view(batch, n_new, self.hq)
        return q.to(torch.bfloat16)

    def worst(self, q, places, o, lse):
        """The largest errors of o and lse.  places [B, n_new]: positions of the query tokens, all of which see everything before them."""
        s0 = q[..., 0].double()
        first = torch.exp(s0)
        want = torch.log(first + places[..., None].double())
        v = torch.tensor(self.value * (self.d // len(self.value)), dtype=torch.float64, device="cuda")
        err = torch.linalg.norm(o.double() - v, dim=-1) / torch.linalg.norm(v)
        return float(err.max()), float(((lse.double() - want).abs() / want.abs().clamp(min=1)).max())


def chunk(s, q, first, bf16=False, sink=0, window=0, new=None):
    n_new = q.shape[1]
    o = torch.zeros(q.shape, dtype=torch.bfloat16 if bf16 else torch.float32, device="cuda")
    lse = torch.zeros(q.shape[:3], device="cuda")
    need = s.vb.vatt_chunk_workspace_bytes(s.plan, n_new)
    ws = torch.empty(need, dtype=torch.uint8, device="cuda") if need else None
    s.vb.vatt_chunk_attend(s.plan, q, s.vb.token_stride(q), n_new, first, new, s.k, s.v, s.table, sink, window, ws,
                           s.vb.VATT_OUT_BF16 if bf16 else s.vb.VATT_OUT_F32, o, lse, torch.cuda.current_stream().cuda_stream)
    torch.cuda.synchronize()
    return o, lse


def chunk_errors(n, d, fmt, bf16, odd=(), n_new=960):
    """960 new tokens: 480 tiles of rows, as many as run at a time, none of which is cut."""
    s = Even(1, 64, 8, d, n, 0, fmt, odd=odd)
    q = s.queries(1, n_new)
    first = torch.tensor([n - n_new], dtype=torch.int32, device="cuda")
    places = first[:, None] + torch.arange(n_new, device="cuda")
    if odd:  # (the tokens before the NaN)
        o, lse = chunk(s, q, first, bf16)
        m = n_new - (n - min(odd))
        return s.worst(q[:, :m], places[:, :m], o[:, :m], lse[:, :m])
    return s.worst(q, places, *chunk(s, q, first, bf16))


def decode_errors(batch, hkv, n, fmt, dense=False, q_len=1, hq=None, odd=()):
    """Decode steps of so many sequences that a workgroup has a whole row."""
    s = Even(batch, hq or hkv, hkv, 64, n, 256, fmt, q_len, odd=odd)
    q = s.queries(batch, q_len)
    lens = torch.full((batch,), n, dtype=torch.int32, device="cuda")
    o, lse = torch.zeros(q.shape, device="cuda"), torch.zeros(q.shape[:3], device="cuda")
    st = torch.cuda.current_stream().cuda_stream
    if dense:
        s.vb.vatt_dense_decode(s.plan, q, s.k, s.v, s.table, lens, s.ws, o, lse, st)
    else:
        s.vb.vatt_window_decode(s.plan, q, s.k, s.v, s.table, lens, 0, n, s.ws, o, lse, st)
    torch.cuda.synchronize()
    places = (lens[:, None] - q_len + torch.arange(q_len, device="cuda"))
    m = q_len - len(odd)
    return s.worst(q[:, :m], places[:, :m], o[:, :m], lse[:, :m])


def _bf16_tol(n):
    """Every weight off by half a step of bf16, the same way, then the result by half a step; a matrix instruction adds 16 rows and cuts the sum off (off
    by 2^-23 of the sum so far, which is half the last one on average)."""
    half = 2.0 ** -8
    return half + half * (1 + half) + n / 16 * 2.0 ** -24 + TOL


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("n", [65536, 170752])
@pytest.mark.parametrize("d,fmt", [(128, 0), (64, 0), (64, 1), (128, 2)])
def test_chunk_of_equal_weights(n, d, fmt, bf16):
    o, lse = chunk_errors(n, d, fmt, bf16)
    assert lse <= TOL and o <= (_bf16_tol(n) if bf16 else TOL)


@pytest.mark.parametrize("n_new", [64, 200])
def test_pieces_of_equal_weights(n_new):
    """32 and 104 tiles of rows, in pieces of 64 and 114 tiles of keys."""
    assert max(chunk_errors(65536, 64, 0, False, n_new=n_new)) <= TOL


def test_rows_worked_out_again():
    """The last token's V is NaN: the rows that share a tile with its queries are worked out again, and keep the tolerance."""
    assert max(chunk_errors(65536, 128, 0, False, odd=(65535,))) <= TOL
    assert max(decode_errors(257, 1, 65536, 0, q_len=2, odd=(65535,))) <= TOL


# (sequences, KV heads, tokens, format, dense, queries): window decode, and dense decode of a quantised cache, by one workgroup per sequence and KV head
@pytest.mark.parametrize("case", [(257, 1, 170752, 0, False, 1), (256, 4, 170752, 0, False, 1), (256, 4, 65536, 2, False, 17), (256, 4, 65536, 1, False, 6),
                                  (256, 4, 170752, 1, True, 1)], ids=str)
def test_decode_of_equal_weights(case):
    batch, hkv, n, fmt, dense, q_len = case
    assert max(decode_errors(batch, hkv, n, fmt, dense, q_len)) <= TOL


@pytest.mark.parametrize("low", [False, True])
@pytest.mark.parametrize("n,d,n_new,sink,window", [(12000, 64, 768, 0, 0), (12000, 128, 768, 0, 0), (12000, 64, 768, 100, 9000), (12000, 128, 40, 0, 0),
                                                   (12000, 64, 61, 700, 10000), (65536, 128, 64, 0, 0)])
def test_maxima_that_move_over_long_rows(n, d, n_new, sink, window, low):
    """Scores that rise over all tokens, in whole rows and in pieces of them; low: the first 4000 scores are -Inf.  The last 5 query tokens do not
    count."""
    s = Even(1, 64, 8, d, n)
    g = torch.Generator("cuda").manual_seed(d + n_new)
    k, v = (torch.randn(8, n, d, generator=g, device="cuda") for _ in range(2))
    k[..., 0] = torch.arange(n, device="cuda") * (20.0 / n)
    if low:
        k[:, :4000, 0] = -math.inf
    for x, buf in ((k, s.k), (v, s.v)):
        buf.view(torch.bfloat16).view(8, n, d).copy_(x)
    k, v = (buf.view(torch.bfloat16).view(8, n, d).double() for buf in (s.k, s.v))
    q = torch.randn(1, n_new, 64, d, generator=g, device="cuda") / 4
    q[..., 0] = 1.0
    q = q.to(torch.bfloat16)
    first = torch.tensor([n - n_new], dtype=torch.int32, device="cuda")
    o, lse = chunk(s, q, first, False, sink, window, torch.tensor([n_new - 5], dtype=torch.int32, device="cuda"))
    assert not o[:, n_new - 5:].any() and not lse[:, n_new - 5:].any()
    p, i = torch.arange(n - n_new, n, device="cuda")[:, None, None], torch.arange(n, device="cuda")
    hidden = (i > p) | ((window > 0) & (i >= sink) & (i <= p - window))
    for h in range(8):
        x = q[0, :, 8 * h:8 * h + 8].double().flatten(0, 1) @ k[h].T.contiguous()
        x = x.view(n_new, 8, n).masked_fill(hidden, -math.inf)
        want, ln = x.softmax(-1).flatten(0, 1) @ v[h], x.logsumexp(-1)
        got = o[0, :, 8 * h:8 * h + 8].double().flatten(0, 1)
        assert ((got - want).norm(dim=-1) <= TOL * want.norm(dim=-1))[:8 * (n_new - 5)].all(), h
        assert ((lse[0, :, 8 * h:8 * h + 8].double() - ln).abs() <= TOL * ln.abs().clamp(min=1))[:n_new - 5].all(), h
