"""The cache operators where one workgroup does many rounds: launches are as large as it takes for several KV heads per tile and several
rows per lane (writes), several tiles of summaries per workgroup (choice), many chunks of keys per workgroup and more than one
look-up of the list (attention).  The sizes follow from the launch rules for 256 compute units, which the tests check."""
import math

import numpy as np
import pytest
import torch

from oracle import cache_ops as co
from test_gpu_cache_ops import HALF_BF16, Setup, _bf16, _block_decode, _check_select, _dense, _np, _seen, _select

pytestmark = pytest.mark.gpu


class Long(Setup):
    """A Setup whose cache is made on the device, and looked at there."""

    def random_cache(self):
        gen = torch.Generator(device="cuda").manual_seed(int(self.rng.integers(1 << 30)))
        size, off = self.vb.vatt_kv_cache_bytes(self.plan), self.vb.vatt_kv_scale_offset(self.plan)
        if self.fmt == co.BF16:
            return torch.randn(size // 2, generator=gen, device="cuda", dtype=torch.bfloat16).view(torch.uint8)
        raw = torch.randint(0, 256, (size,), generator=gen, device="cuda", dtype=torch.uint8)
        if self.fmt == co.E4M3:
            raw[:off] &= 0xfe  # no NaN
        raw[off:] = raw[off:] % 3 + (120 if self.fmt == co.E2M1 else 118)
        return raw

    def values(self, buf, b, h, n):
        """Rows of tokens 0 .. n - 1 as fp64 [n, d]."""
        tok = torch.arange(n, device="cuda")
        if self.page:
            at = scale_at = (self.table[b].long()[tok // self.page] * self.hkv + h) * self.page + tok % self.page
        else:
            at, scale_at = (b * self.hkv + h) * self.n_max + tok, (b * self.hkv + h) * ((self.n_max + 7) // 8 * 8) + tok
        off, size = self.vb.vatt_kv_scale_offset(self.plan), {0: 2 * self.d, 1: self.d, 2: self.d // 2}[self.fmt]
        codes = buf[:off // size * size].view(-1, size)[at]
        if self.fmt == co.BF16:
            return codes.view(torch.bfloat16).double()
        if self.fmt == co.E2M1:
            codes = torch.stack([codes & 15, codes >> 4], -1).view(n, self.d)
        scales = buf[off:].view(-1, self.d // 32)[scale_at].long()
        units = torch.from_numpy(2.0 ** (np.arange(256) - 127.0)).cuda()  # (powers on the device are off by their last bit)
        return torch.from_numpy(co.code_values(self.fmt)).cuda()[codes.long()] * units[scales].repeat_interleave(32, 1)


def _cus():
    return torch.cuda.get_device_properties(0).multi_processor_count


# ---- writing -----------------------------------------------------------------------------------------------------------------

WRITES = [
    # (batch, hq, hkv, d, n_max, page, fmt, block, n_new, first, new_lens, rotation, fused; KV heads per tile, passes per workgroup)
    (3, 20, 5, 128, 9100, 0, 0, 16, 9000, [0, 17, 99], [9000, 3001, 8999], dict(theta=1e4), True, 4, 8),
    (2, 20, 5, 64, 20100, 64, 2, 16, 20001, [3, 90], [20001, 19000], dict(theta=1e4, layout=1, rotary_dim=32), False, 3, 5),
    (1, 20, 5, 128, 7100, 0, 1, None, 7000, [33], None, dict(theta=1e4), False, 0, 5),
    (1, 32, 32, 128, 9100, 64, 1, 64, 9001, [5], None, dict(theta=5e5, rotary_dim=64), True, 2, 8),
    (2, 24, 24, 64, 20000, 0, 0, 32, 19960, [0, 31], [19960, 12345], None, True, 8, 6),
]


@pytest.mark.parametrize("case", WRITES, ids=lambda c: "-".join(str(x) for x in c[:9]))
def test_a_long_write_is_its_pieces(case):
    """One launch with many rounds per workgroup against launches with one each, bit for bit, and rows of it against the oracle."""
    batch, hq, hkv, d, n_max, page, fmt, block, n_new, first, new_lens, rotary, fused, k_heads, row_passes = case
    rows = 256 // (d // 8)  # of a pass
    if block:
        tile = max(block, rows)
        assert max(1, min(8, hkv, batch * ((n_new + tile - 2) // tile + 1) * hkv // (8 * _cus()))) == k_heads
    passes = [-(-hq // (rows // 8)) if rotary else 0, -(-hkv // (rows // 8))]
    assert max(1, min(8, max(passes), batch * -(-n_new // 8) * sum(passes) // (8 * _cus()))) == row_passes
    s = Long(batch, hq, hkv, d, n_max, page, fmt, block, rotary=rotary, seed=n_new)
    gen = torch.Generator(device="cuda").manual_seed(n_new)
    x = torch.randn(batch, n_new, (hq + 2 * hkv) * d + 8, generator=gen, device="cuda", dtype=torch.bfloat16)
    x *= torch.exp(2 * torch.randn(batch, n_new, 1, generator=gen, device="cuda")).bfloat16()
    at = [0, hq * d, (hq + hkv) * d, (hq + 2 * hkv) * d]
    q, kn, vn = (x[..., at[i]:at[i + 1]].unflatten(-1, (-1, d)) for i in range(3))
    if not fused:
        q, kn, vn = q.contiguous(), kn.contiguous(), vn.contiguous()
    start, lens = (s.k.clone(), s.v.clone()), new_lens or [n_new] * batch
    got = []
    for step in (n_new, 400):
        s.k, s.v = start[0].clone(), start[1].clone()
        summary = torch.full(s.summary_shape(), 3.25, dtype=torch.bfloat16, device="cuda") if block else None
        out_q = torch.full((batch, n_new, hq, d), 7.5, dtype=torch.bfloat16, device="cuda") if rotary else None
        now, after = s.ints(first), s.ints([0] * batch)
        for j in range(0, n_new, step):
            m = min(step, n_new - j)
            # (the last piece is shorter than the others for some of the sequences, and there may be none for them)
            part = q[:, j:j + m].contiguous(), kn[:, j:j + m].contiguous(), vn[:, j:j + m].contiguous()
            out = None if out_q is None else out_q[:, j:j + m].contiguous()
            here = s.ints([min(max(n - j, 0), m) for n in lens])
            if step == n_new:
                part, out, here = (q, kn, vn), out_q, None if new_lens is None else here
            s.write(part[0] if rotary else None, part[1], part[2], now, here, summary, out, after)
            if out is not None and out is not out_q:
                out_q[:, j:j + m] = out
            now, after = after, now
        torch.cuda.synchronize()
        got.append((s.k, s.v, summary, out_q, now))
    assert got[0][4].tolist() == got[1][4].tolist() == [f + n for f, n in zip(first, lens)]
    for one, two in zip(*got):
        assert one is two is None or torch.equal(one, two)
    s.k, s.v = got[0][:2]
    summary, out_q = got[0][2:4]
    half = {0: HALF_BF16, 1: 2.0 ** -4, 2: 2.0 ** -2}[fmt]
    for b in range(batch):
        for h in range(hkv):
            k, v = (_np(s.values(t, b, h, first[b] + lens[b])) for t in (s.k, s.v))
            for j in {0, lens[b] - 1, *s.rng.integers(0, lens[b], size=20).tolist()}:
                pos = first[b] + j
                new = _np(vn[b, j, h])
                assert np.array_equal(v[pos], co.stored(new, fmt)), (b, h, j)
                new = _np(kn[b, j, h])
                want = co.rotate(new, pos, rotary) if rotary else new
                # as in test_write; a quantised value is off by half a step of the value or of the smallest step of its 32
                slack = 4 * 2.0 ** -24 * 1.2 * np.abs(new).max() * 2
                unit = np.repeat(np.abs(want).reshape(-1, 32).max(1), 32)
                least = {0: 2.0 ** -133, 1: unit * 2.0 ** -10 / 224, 2: unit / 4 / 3}[fmt]
                assert (np.abs(k[pos] - want) <= np.maximum(half * np.abs(want), least) + 1.3 * slack).all(), (b, h, j)
            for blk in {0, *s.rng.integers(0, -(-(first[b] + lens[b]) // block), size=20).tolist()} if block else ():
                if (blk + 1) * block > first[b]:
                    top, low = co.summary(k[blk * block:(blk + 1) * block])
                    ends = _np(s.summary_of(summary, b, h, blk))
                    assert np.array_equal(ends[0], top) and np.array_equal(ends[1], low), (b, h, blk)
        for h in range(hq if rotary else 0):
            for j in s.rng.integers(0, lens[b], size=20).tolist():
                new = _np(q[b, j, h])
                want = co.rotate(new, first[b] + j, rotary)
                slack = 4 * 2.0 ** -24 * 1.2 * np.abs(new).max() * 2
                assert (np.abs(_np(out_q[b, j, h]) - want) <= HALF_BF16 * np.abs(want) + 1.01 * slack + 2.0 ** -133).all(), (b, h, j)


# ---- choosing ----------------------------------------------------------------------------------------------------------------

SELECTS = [
    # (batch, hq, hkv, d, n_max, page, block, q_len, lens; tiles of the first workgroup)
    (16, 64, 64, 64, 4160, 0, 16, 1, [4160 - 61 * i for i in range(15)] + [70], 3),
    (8, 128, 64, 64, 8192, 64, 16, 1, [8192, 8191, 5000, 1025, 1024, 16, 4097, 7000], 2),
    (8, 256, 64, 64, 4160, 32, 16, 5, [4160, 4150, 3000, 2050, 2049, 7, 1, 4111], 2),
    (16, 128, 32, 128, 5000, 0, 16, 1, [5000 - 300 * i for i in range(16)], 2),
]


@pytest.mark.parametrize("kind", ["normal", "odd"])
@pytest.mark.parametrize("case", SELECTS, ids=lambda c: "-".join(str(x) for x in c[:8]))
def test_a_choice_with_many_tiles_per_workgroup(case, kind):
    batch, hq, hkv, d, n_max, page, block, q_len, lens, tiles = case
    blocks = -(-n_max // block)
    splits = min(-(-blocks // 64), -(-8 * _cus() // (batch * hkv)))
    assert -(-(-(-blocks // 64)) // splits) == tiles
    s = Long(batch, hq, hkv, d, n_max, page, 0, block, q_len, seed=n_max, topk_frac=0.06)
    gen = torch.Generator(device="cuda").manual_seed(batch)
    ends = torch.randn(s.summary_shape(), generator=gen, device="cuda", dtype=torch.bfloat16).sort(-2, descending=True)[0].contiguous()
    if kind == "odd":  # a few rows take the way of values that are no numbers
        odd = torch.rand(s.summary_shape()[:3], generator=gen, device="cuda") < 2e-4
        ends[..., 5].masked_fill_(odd[..., None], math.nan)
        ends *= torch.where(torch.rand(s.summary_shape()[:3], generator=gen, device="cuda") < 1e-3, 1e30, 1.0)[..., None, None].bfloat16()
    q = torch.randn(batch, q_len, hq, d, generator=gen, device="cuda", dtype=torch.bfloat16)
    got = _select(s, q, ends, lens, q_len == 1)
    s.table = None if s.table is None else s.table.cpu()
    _check_select(s, q, ends, lens, got)


# ---- attention ---------------------------------------------------------------------------------------------------------------

def _staircase(s, lens):
    """K and V through vatt_write_kv: N(0, 1) / 2, and a first column that makes the scores rise, fall, peak in the middle, rise and fall
    again within every 1024 tokens, or stay, by some 40 in all, one way after the other over the sequences and KV heads."""
    gen = torch.Generator(device="cuda").manual_seed(s.n_max)
    n = max(lens)
    step = max(1, (1 << 27) // (s.batch * s.hkv * s.d))
    t = torch.arange(n, device="cuda", dtype=torch.float64)
    ways = torch.stack([t / n, 1 - t / n, 1 - (2 * t / n - 1).abs(), 1 - (2 * (t % 1024) / 1024 - 1).abs(), 0 * t + 0.5])
    way = (torch.arange(s.batch, device="cuda")[:, None] * 3 + torch.arange(s.hkv, device="cuda")) % 5
    for j in range(0, n, step):
        m = min(step, n - j)
        k, v = (torch.randn(s.batch, m, s.hkv, s.d, generator=gen, device="cuda", dtype=torch.bfloat16) * f for f in (0.5, 1.0))
        k[..., 0] = (40 * ways[way][..., j:j + m] - 20).permute(0, 2, 1).bfloat16()
        k[..., 1:32] = 0  # (the scale of the first group is the staircase's)
        s.write(None, k, v, s.ints([j] * s.batch), s.ints([min(max(x - j, 0), m) for x in lens]))


def _compare(s, q, lens, o, lse, seen_of=None):
    """Against softmax in 64 bits on the device.  seen_of(row, h): the tokens listed, or all that the query sees."""
    qd, g, scale = q.double().view(s.batch, s.q_len, s.hq, s.d), s.hq // s.hkv, s.params["sm_scale"] or 1 / math.sqrt(s.d)
    seen, o, lse = _seen(s, lens), o.double().view(s.batch, s.q_len, s.hq, s.d), lse.double().view(s.batch, s.q_len, s.hq)
    worst = torch.zeros(2, device="cuda", dtype=torch.float64)
    for b in range(s.batch):
        for h in range(s.hkv):
            k, v = s.values(s.k, b, h, lens[b]), s.values(s.v, b, h, lens[b])
            for t in range(s.q_len):
                r = b * s.q_len + t
                kt, vt = (k[:seen[r]], v[:seen[r]]) if seen_of is None else (k[seen_of(r, h)], v[seen_of(r, h)])
                score = scale * (qd[b, t, h * g:(h + 1) * g] @ kt.T)
                want = torch.softmax(score, -1) @ vt
                err = (o[b, t, h * g:(h + 1) * g] - want).norm(dim=-1) / want.norm(dim=-1)
                total = torch.logsumexp(score, -1)
                err2 = (lse[b, t, h * g:(h + 1) * g] - total).abs() / total.abs().clamp(min=1.0)
                worst = torch.maximum(worst, torch.stack([err.max(), err2.max()]))
    # 32-bit scores and weights, as in test_gpu_cache_ops
    assert worst[0] <= 2e-5 and worst[1] <= 2e-5, worst.tolist()


DENSE = [
    # (batch, hq, hkv, d, n_max, page, fmt, q_len, lens): one workgroup per KV head, of 1 .. 5, 6 .. 8, 9 .. 16, 17 .. 32 and more vectors
    (8, 128, 128, 64, 10007, 0, 2, 1, [10007, 9999, 8193, 8192, 8320, 129, 1, 5000]),
    (8, 512, 128, 64, 2007, 64, 2, 1, [2007, 2000, 1025, 1024, 700, 1, 128, 1999]),
    (8, 1024, 128, 64, 2007, 0, 1, 1, [2007, 2000, 1025, 1024, 700, 1, 128, 1999]),
    (8, 512, 128, 128, 1500, 0, 1, 3, [1500, 1499, 1025, 1024, 3, 1, 130, 1400]),
    (8, 1024, 128, 64, 8500, 0, 2, 3, [8500, 8499, 8193, 1024, 3, 1, 130, 8192]),
    (8, 512, 64, 128, 1300, 32, 2, 5, [1300, 1299, 1025, 1024, 5, 1, 130, 1200]),
]


@pytest.mark.parametrize("case", DENSE, ids=lambda c: "-".join(str(x) for x in c[:8]))
def test_dense_with_many_chunks_per_workgroup(case):
    batch, hq, hkv, d, n_max, page, fmt, q_len, lens = case
    vectors = hq // hkv * q_len
    assert batch * hkv * (1 if vectors <= 16 else -(-vectors // 32)) >= 4 * _cus()
    s = Long(batch, hq, hkv, d, n_max, page, fmt, None, q_len, seed=n_max, topk_frac=0.01, base_frac=0.01, budget_cap_frac=0.01, sm_scale=1.0)
    _staircase(s, lens)
    gen = torch.Generator(device="cuda").manual_seed(1)
    q = torch.randn(batch, q_len, hq, d, generator=gen, device="cuda", dtype=torch.bfloat16) / 4
    q[..., 0] = 1.0
    _compare(s, q, lens, *_dense(s, q, lens))


BLOCKS = [
    # (batch, hq, hkv, d, n_max, page, fmt, block, q_len, lens): up to four query vectors and eight
    (4, 256, 256, 64, 9000, 0, 0, 16, 1, [9000, 8999, 8193, 17]),
    (4, 1024, 256, 64, 1900, 64, 2, 32, 1, [1900, 1500, 1025, 33]),
    (4, 1024, 128, 128, 1900, 0, 1, 64, 2, [1900, 1899, 1025, 2]),
    (8, 1024, 128, 64, 8700, 0, 2, 256, 1, [8700, 8699, 8193, 8192, 1, 257, 4000, 8300]),
]


@pytest.mark.parametrize("case", BLOCKS, ids=lambda c: "-".join(str(x) for x in c[:9]))
def test_lists_with_many_chunks_per_workgroup(case):
    batch, hq, hkv, d, n_max, page, fmt, block, q_len, lens = case
    assert batch * q_len * hkv >= 4 * _cus()
    s = Long(batch, hq, hkv, d, n_max, page, fmt, block, q_len, seed=n_max, topk_frac=1.0, base_frac=0.01, budget_cap_frac=0.01, sm_scale=1.0)
    _staircase(s, lens)
    gen = torch.Generator(device="cuda").manual_seed(1)
    q = torch.randn(batch, q_len, hq, d, generator=gen, device="cuda", dtype=torch.bfloat16) / 4
    q[..., 0] = 1.0
    cap = s.vb.vatt_block_list_capacity(s.plan)
    rows, seen = batch * q_len, _seen(s, lens)
    blocks, count = np.full((rows, hkv, cap), 2 ** 30, dtype=np.int32), np.zeros((rows, hkv), dtype=np.int32)
    for r, n in enumerate(seen):
        total = -(-n // block)
        for h in range(hkv):  # nearly all, in order, in reverse, in any order
            pick = [np.arange(total), np.arange(total)[::-1], s.rng.permutation(total)][(r + h) % 3][:max(1, total - h % 4)]
            blocks[r, h, :len(pick)], count[r, h] = pick, len(pick)

    def listed(r, h):
        tok = (torch.from_numpy(blocks[r, h, :count[r, h]].astype(np.int64)).cuda()[:, None] * block + torch.arange(block, device="cuda")).flatten()
        return tok[tok < seen[r]]

    _compare(s, q, lens, *_block_decode(s, q, lens, torch.from_numpy(blocks).cuda(), torch.from_numpy(count).cuda()), listed)
