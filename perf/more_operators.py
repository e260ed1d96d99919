"""The attention operators for new tokens over the cache that performance work on this library is measured on, each in its plain form and as
the library's call.

A case is one call of the kind a serving loop makes for one layer, through the public entry points:

  op "chunk"    vatt_chunk_attend: the n_new newest tokens of every sequence (a prompt, a piece of one, drafted tokens) attend over
                the cache that already holds their rows; `window` > 0: over the first `sink` tokens and the last `window` only.
  op "window"   vatt_window_decode: a decode step (q_len query tokens per sequence) over the first `sink` and the last
                `window` tokens.

`fmt`: "bf16", "e4m3" (8 bits a value) or "e2m1" (4 bits a value), the latter two with one power-of-two scale for 32 columns.
`page` 0 is the contiguous layout.  `out`: "f32" or "bf16", the type of a chunk's output (a decode step's is f32).  Sequences are ragged
where n_lo < n, and their new tokens where new_lo < n_new.

Inputs: K ~ N(0, 1) in even KV heads and N(0, 1/4) in odd ones, every sixteenth column four times as large (real keys have such
columns, and scales feel them); V and q ~ N(0, 1), q smaller in the large columns.
"""
import math

import torch

own = False

VALUES = {"e4m3": 448.0, "e2m1": 6.0}  # largest value of a format
FMT = {"bf16": 0, "e4m3": 1, "e2m1": 2}
E2M1 = [0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0]
TYPE = {"f32": torch.float32, "bf16": torch.bfloat16}
PLAIN_SCORES = 1 << 29  # scores that the plain form makes at a time


def _case(op, batch, n, **over):
    c = dict(op=op, batch=batch, n=n, n_lo=n, hq=32, hkv=8, d=128, q_len=1, n_new=1, new_lo=0, fmt="bf16", page=0, sink=0, window=0,
             out="bf16" if op == "chunk" else "f32")
    c.update(over)
    c["new_lo"] = c["new_lo"] or c["n_new"]
    return c


def listed():
    return [
        # a few drafted tokens of one chat on a small model: launch and latency only
        _case("chunk", 1, 1024, name="chunk 1 x 7 on 1k", n_new=7, hq=8, hkv=2, d=64, out="f32"),
        # drafted tokens of several chats, eight query heads to a KV head
        _case("chunk", 3, 16384, name="chunk 3 x 33 on 5k-16k, groups of 8", n_lo=5003, n_new=33, hq=32, hkv=4),
        # continuous batching: single tokens and pieces of prompts in one padded batch, an 8-bit cache on pages of 16 tokens
        _case("chunk", 24, 8000, name="chunk 24 x 1-256 on 0.5k-8k e4m3 paged", n_lo=509, n_new=256, new_lo=1, fmt="e4m3", page=16),
        # one prompt
        _case("chunk", 1, 2048, name="prompt 1 x 2k", n_new=2048),
        # prompts of several lengths in one padded batch, on pages
        _case("chunk", 4, 8192, name="prompts 4 x 0.7k-8k paged", n_lo=701, n_new=8192, new_lo=701, page=64),
        # a piece of a long document
        _case("chunk", 1, 65536, name="chunk 1 x 2k on 64k paged", n_new=2048, page=64),
        # prompts of a model with narrow heads and as many KV heads, a 4-bit cache, output in 32 bits
        _case("chunk", 2, 4999, name="prompts 2 x 5k e2m1, heads of 64, f32", n_new=4999, fmt="e2m1", hq=16, hkv=16, d=64, out="f32"),
        # a long prompt in a layer that sees a window and the first tokens
        _case("chunk", 1, 32768, name="windowed prompt 1 x 32k", n_new=32768, sink=4, window=4096, page=64),
        # ragged prompts, narrow window, 8-bit cache
        _case("chunk", 6, 2999, name="windowed prompts 6 x 0.3k-3k e4m3", n_lo=301, n_new=2999, new_lo=301, fmt="e4m3", sink=128, window=500),
        # the decode step of one chat in such a layer, with the sizes of the deterministic set
        _case("window", 1, 32768, name="window 1 x 32k, 128 + 128", sink=128, window=128),
        # a large batch with a long window, 8-bit cache on pages
        _case("window", 48, 65536, name="window 48 x 1k-64k, 4 + 4096 e4m3 paged", n_lo=1021, sink=4, window=4096, fmt="e4m3", page=16),
        # drafted tokens on a narrow model with a 4-bit cache
        _case("window", 5, 9001, name="window 5 x 9k, 64 + 1000 e2m1, 3 queries", sink=64, window=1000, fmt="e2m1", hq=16, hkv=2, d=64, q_len=3),
    ]


SHAPES = [(32, 8, 128), (32, 8, 128), (32, 4, 128), (16, 16, 64), (16, 8, 64), (8, 8, 128), (8, 2, 64)]
MOST_FLOPS, MOST_ROWS = 2.0e12, 3_000_000  # of a drawn case: below the largest listed one


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """Any operator, shape, format, layout and length within the limits of the listed cases."""
    op = rng.choice(["chunk", "chunk", "chunk", "window"])
    hq, hkv, d = rng.choice(SHAPES)
    over = dict(hq=hq, hkv=hkv, d=d, page=rng.choice([0, 0, 16, 64, 128]), fmt=rng.choice(["bf16", "bf16", "e4m3", "e2m1"]))
    n = _log(rng, 1, 65536)
    if op == "window" or rng.random() < 0.5:
        over["sink"], over["window"] = rng.choice([0, 1, 4, 37, 128, 300]), _log(rng, 1, 8192)
    if op == "window":
        over["q_len"] = min(n, rng.choice([1, 1, 1, 2, 5, 11]))
    else:
        over["n_new"] = n if rng.random() < 0.4 else _log(rng, 1, min(n, 4096))
        over["out"] = rng.choice(["bf16", "bf16", "f32"])
    batch = _log(rng, 1, 48)
    ragged, most_ragged = rng.random() < 0.6, rng.random() < 0.5
    while True:  # fewer sequences, then shorter ones, until the case is small enough
        over["n_lo"] = over["new_lo"] = 0
        if ragged and batch > 1:
            over["n_lo"] = max(1, n // 16)
            if op == "chunk":
                over["new_lo"] = 1 if most_ragged else max(1, over["n_new"] // 9)
        over["n_lo"] = max(over["n_lo"] or n, over["q_len"] if op == "window" else over["n_new"] if over["n_new"] < n else 1)
        c = _case(op, batch, n, **over)
        if work(c)["flops"] <= MOST_FLOPS and batch * hkv * n <= MOST_ROWS:
            return c
        if batch > 1:
            batch = batch // 2
        else:
            n = max(1, n * 3 // 4)
            if op == "chunk":
                over["n_new"] = min(over["n_new"], n)


# ---- sizes, which follow from the case alone -----------------------------------------------------------------------------

def _spread(hi, lo, count):
    """hi, and the others evenly down to lo, in a scattered order."""
    if count == 1 or lo == hi:
        return [hi] * count
    got = [hi - (hi - lo) * i // (count - 1) for i in range(count)]
    return [got[(i * 7 + 3) % count] if math.gcd(7, count) == 1 else got[i] for i in range(count)]


def _lengths(c):
    """Tokens of every sequence, the new ones among them."""
    return _spread(c["n"], c["n_lo"], c["batch"])


def _new(c):
    """New tokens of every sequence: the query tokens that count."""
    if c["op"] == "window":
        return [c["q_len"]] * c["batch"]
    return [min(m, n) for m, n in zip(_spread(c["n_new"], c["new_lo"], c["batch"]), _lengths(c))]


def _queries(c):
    return c["q_len"] if c["op"] == "window" else c["n_new"]


def _n_max(c):
    return -(-c["n"] // c["page"]) * c["page"] if c["page"] else c["n"]


def _row_bytes(c):
    return {"bf16": 2 * c["d"], "e4m3": c["d"], "e2m1": c["d"] // 2}[c["fmt"]]


def _stored(c):
    """Bytes that one row of K or V takes, its scales included."""
    return _row_bytes(c) + (0 if c["fmt"] == "bf16" else c["d"] // 32)


def _sizes(c):
    """(physical pages of a paged cache, rows, rows of scales, byte offset of the scales) of a K or V buffer."""
    pages = c["batch"] * (_n_max(c) // c["page"]) + 3 if c["page"] else 0
    rows = pages * c["hkv"] * c["page"] if c["page"] else c["batch"] * c["hkv"] * _n_max(c)
    scales = rows if c["page"] else c["batch"] * c["hkv"] * (-(-_n_max(c) // 8) * 8)
    return pages, rows, scales, -(-rows * _row_bytes(c) // 256) * 256


# ---- inputs --------------------------------------------------------------------------------------------------------------

def _gen(seed, what):
    g = torch.Generator(device="cuda")
    g.manual_seed(1000003 * int(seed) + what)
    return g


def _columns(d):
    one = torch.ones(d, device="cuda")
    one[::16] = 4.0
    return one


def _fill(c, g, keys):
    """A cache buffer of K or V in the case's format, with values in every row that the layout has."""
    pages, rows, scales, off = _sizes(c)
    d, hkv = c["d"], c["hkv"]
    per = c["page"] or _n_max(c)
    head = torch.ones(hkv, device="cuda")
    head[1::2] = 0.5 if keys else 1.0
    cols = _columns(d) if keys else torch.ones(d, device="cuda")
    units = rows // (hkv * per)  # pages or sequences
    step = max(1, (1 << 25) // (hkv * per * d))
    out = []
    buf = torch.zeros(off + scales * (d // 32), dtype=torch.uint8, device="cuda") if c["fmt"] != "bf16" else None
    for u in range(0, units, step):
        m = min(step, units - u)
        x = torch.randn((m, hkv, per, d), generator=g, device="cuda") * head[:, None, None] * cols
        x = x.to(torch.bfloat16)
        if buf is None:
            out.append(x)
            continue
        codes, exps = _quantise(x.float(), c["fmt"])
        r = u * hkv * per
        buf[:rows * _row_bytes(c)].view(rows, -1)[r:r + m * hkv * per] = codes.reshape(m * hkv * per, -1)
        wide = per if c["page"] else scales // (units * hkv)
        buf[off:].view(units, hkv, wide, d // 32)[u:u + m, :, :per] = exps
    if buf is not None:
        return buf
    return torch.cat(out) if len(out) > 1 else out[0]


def _two(e):
    """2^e in 64 bits, from its bits: pow() need not be exact."""
    return ((e.long() + 1023) << 52).view(torch.float64)


def _quantise(x, fmt):
    """Finite fp32 [..., d] -> (codes uint8 [..., d or d / 2], scale bytes uint8 [..., d / 32]): per 32 columns the smallest power of
    two at which no magnitude is above the format's largest; values to the nearest, ties to even."""
    groups = x.unflatten(-1, (-1, 32))
    mant, exp = torch.frexp(groups.abs().amax(-1))  # mant in [1/2, 1)
    lm, le = math.frexp(VALUES[fmt])
    e = torch.where(mant > 0, torch.where(mant > lm, exp - le + 1, exp - le), -127).clamp(min=-127)
    y = (groups.double() * _two(-e)[..., None]).float()
    if fmt == "e4m3":
        codes = y.to(torch.float8_e4m3fn).view(torch.uint8).flatten(-2)
    else:
        a = y.abs()
        step = torch.where(a < 2, 0.5, torch.where(a < 4, 1.0, 2.0))
        r = torch.round(a / step) * step
        code = torch.where(r < 2, r * 2, torch.where(r < 4, r + 2, r / 2 + 4)).to(torch.uint8)
        code = (code | (torch.signbit(y).to(torch.uint8) << 3)).flatten(-2).unflatten(-1, (-1, 2))
        codes = code[..., 0] | (code[..., 1] << 4)
    return codes, (e + 127).to(torch.uint8)


def _plan(c):
    """The library's plan of a case with its workspace: what a serving process keeps for a layer."""
    from paper_2510_05688_amd import binding as vb

    class Kept:
        def __init__(self):
            pages = _sizes(c)[0]
            self.plan = vb.vatt_plan_create_chunk(
                dict(batch=c["batch"], n_q_heads=c["hq"], n_kv_heads=c["hkv"], head_dim=c["d"], n_max=_n_max(c),
                     kv_layout=1 if c["page"] else 0, page_size=c["page"], num_blocks=pages, sink=128, window=128,
                     topk_abs=0, topk_frac=0.025, base_abs=0, base_frac=0.025, epsilon=0.05, delta=0.05, target=0,
                     sm_scale=0.0, budget_cap_frac=1.0), c["q_len"], torch.cuda.current_device())
            vb.vatt_plan_set_option(self.plan, vb.VATT_OPT_KV_FORMAT, FMT[c["fmt"]])
            need = vb.vatt_plan_workspace_bytes(self.plan) if c["op"] == "window" else vb.vatt_chunk_workspace_bytes(self.plan, c["n_new"])
            self.workspace = torch.empty(need, dtype=torch.uint8, device="cuda")

        def __del__(self):
            vb.vatt_plan_destroy(self.plan)

    return Kept()


def prepare(case, seed):
    c = dict(case)
    b, hq, d, t = c["batch"], c["hq"], c["d"], _queries(c)
    s = dict(case=c, kept=_plan(c) if own else None, table=None)
    if c["page"]:
        s["table"] = torch.randperm(_sizes(c)[0], generator=_gen(seed, 1), device="cuda")[:b * (_n_max(c) // c["page"])].int().reshape(b, -1).contiguous()
    s["lens"] = torch.tensor(_lengths(c), dtype=torch.int32, device="cuda")
    s["new"] = torch.tensor(_new(c), dtype=torch.int32, device="cuda")
    s["first"] = s["lens"] - s["new"]
    s["k"], s["v"] = _fill(c, _gen(seed, 2), True), _fill(c, _gen(seed, 3), False)
    s["q"] = (torch.randn((b, t, hq, d), generator=_gen(seed, 4), device="cuda") / _columns(d).sqrt()).to(torch.bfloat16)
    s["o"] = torch.zeros((b, t, hq, d), dtype=TYPE[c["out"]], device="cuda")
    s["lse"] = torch.zeros((b, t, hq), dtype=torch.float32, device="cuda")
    return s


# ---- plain form ----------------------------------------------------------------------------------------------------------

def _load(s, buf, tokens):
    """Rows of `tokens` ([B, T] positions) for every KV head in fp32: [B, Hkv, T, d]."""
    c = s["case"]
    b, hkv, d = c["batch"], c["hkv"], c["d"]
    heads = torch.arange(hkv, device="cuda").view(1, hkv, 1)
    if c["page"]:
        page = torch.gather(s["table"].long(), 1, tokens // c["page"])
        at = scale_at = (page[:, None] * hkv + heads) * c["page"] + (tokens % c["page"])[:, None]
    else:
        base = torch.arange(b, device="cuda").view(b, 1, 1) * hkv + heads
        at, scale_at = base * _n_max(c) + tokens[:, None], base * (-(-_n_max(c) // 8) * 8) + tokens[:, None]
    if c["fmt"] == "bf16":
        return buf.view(-1, d)[at].float()
    pages, rows, scales, off = _sizes(c)
    codes, exps = buf[:rows * _row_bytes(c)].view(rows, -1)[at], buf[off:off + scales * (d // 32)].view(scales, -1)[scale_at]
    if c["fmt"] == "e4m3":
        v = codes.view(torch.float8_e4m3fn).float()
    else:
        table = torch.tensor(E2M1 + [-x for x in E2M1], device="cuda")
        v = torch.stack([table[(codes & 15).long()], table[(codes >> 4).long()]], -1).flatten(-2)
    return (v.unflatten(-1, (-1, 32)) * _two(exps.int() - 127).float()[..., None]).flatten(-2)


def _attend(s):
    c = s["case"]
    b, hq, hkv, d, sink, window = c["batch"], c["hq"], c["hkv"], c["d"], c["sink"], c["window"]
    group, count, last = hq // hkv, _queries(c), _n_max(c) - 1
    lengths, new = _lengths(c), _new(c)
    t0 = 0
    while t0 < count:
        if window:
            step = min(count - t0, max(1, min(512, PLAIN_SCORES // (b * hq * (sink + window + 512)))))
        else:
            step = min(count - t0, max(1, PLAIN_SCORES // (b * hq * c["n"])))
        t = torch.arange(t0, t0 + step, device="cuda")
        place = s["first"].long()[:, None] + t  # the query tokens' positions
        if window:
            # the first tokens, then those from the first query's window on
            start = (place[:, :1] - window + 1).clamp(min=sink)
            tokens = torch.cat([torch.arange(sink, device="cuda").expand(b, -1), start + torch.arange(window + step - 1, device="cuda")], 1)
        else:
            end = max(n - m + min(m, t0 + step) for n, m in zip(lengths, new))
            tokens = torch.arange(end, device="cuda").expand(b, -1)
        there = tokens[:, None] <= place[..., None]
        if window:
            there &= (tokens[:, None] < sink) | (tokens[:, None] > place[..., None] - window)
        k, v = (_load(s, s[x], tokens.clamp(max=last)) for x in "kv")
        q = s["q"][:, t0:t0 + step].float().view(b, step, hkv, group, d).transpose(1, 2).flatten(2, 3)
        x = (q @ k.transpose(-1, -2).contiguous()) / math.sqrt(d)
        x = x.unflatten(2, (step, group)).masked_fill_(~there[:, None, :, None], -torch.inf).flatten(2, 3)
        m = x.amax(-1, keepdim=True)
        p = x.sub_(m).exp_()
        total = p.sum(-1, keepdim=True)
        o = ((p @ v) / total).unflatten(2, (step, group)).transpose(1, 2).reshape(b, step, hq, d)
        lse = (m + total.log()).unflatten(2, (step, group)).transpose(1, 2).reshape(b, step, hq)
        valid = (t < s["new"][:, None])[..., None]
        now_o, now_lse = s["o"][:, t0:t0 + step], s["lse"][:, t0:t0 + step]
        now_o.copy_(torch.where(valid[..., None], o.to(s["o"].dtype), now_o))
        now_lse.copy_(torch.where(valid, lse, now_lse))
        t0 += step
    return dict(o=s["o"], lse=s["lse"])


# ---- one pass ------------------------------------------------------------------------------------------------------------

def run(state):
    s, c = state, state["case"]
    if not own:
        return _attend(s)
    from paper_2510_05688_amd import binding as vb

    plan, ws = s["kept"].plan, s["kept"].workspace
    stream = torch.cuda.current_stream().cuda_stream
    if c["op"] == "chunk":
        vb.vatt_chunk_attend(plan, s["q"], vb.token_stride(s["q"]), c["n_new"], s["first"], s["new"], s["k"], s["v"], s["table"], c["sink"],
                             c["window"], ws, vb.VATT_OUT_BF16 if c["out"] == "bf16" else vb.VATT_OUT_F32, s["o"], s["lse"], stream)
    else:
        vb.vatt_window_decode(plan, s["q"], s["k"], s["v"], s["table"], s["lens"], c["sink"], c["window"], ws, s["o"], s["lse"], stream)
    return dict(o=s["o"], lse=s["lse"])


def _seen_sum(c, upto):
    """Tokens seen by the queries at positions 0 .. upto - 1 together."""
    if not c["window"]:
        return upto * (upto + 1) // 2
    most = c["sink"] + c["window"]
    ramp = min(upto, most)
    return ramp * (ramp + 1) // 2 + (upto - ramp) * most


def work(case):
    """Inputs read once, outputs written once: every row that some query sees, queries, outputs."""
    c = case
    nbytes = flops = 0.0
    for n, m in zip(_lengths(c), _new(c)):
        rows = n
        if c["window"]:
            lo = max(n - m - c["window"] + 1, 0)
            rows = n - lo + min(c["sink"], lo)
        seen = _seen_sum(c, n) - _seen_sum(c, n - m)
        nbytes += 2 * c["hkv"] * rows * _stored(c) + m * c["hq"] * (c["d"] * (2 + (2 if c["out"] == "bf16" else 4)) + 4)
        flops += 4.0 * c["d"] * c["hq"] * seen
    return dict(bytes=nbytes, flops=flops)


# ---- the definition in 64 bits -------------------------------------------------------------------------------------------

def _exact_rows(c, s, buf, b, head, count):
    """The first `count` rows of one sequence and KV head in 64 bits."""
    tokens = torch.arange(count, device="cuda")
    if c["page"]:
        at = (s["table"][b].long()[tokens // c["page"]] * c["hkv"] + head) * c["page"] + tokens % c["page"]
        scale_at = at
    else:
        at = (b * c["hkv"] + head) * _n_max(c) + tokens
        scale_at = (b * c["hkv"] + head) * (-(-_n_max(c) // 8) * 8) + tokens
    d = c["d"]
    if c["fmt"] == "bf16":
        return buf.view(-1, d)[at].double()
    pages, rows, scales, off = _sizes(c)
    codes = buf[:rows * _row_bytes(c)].view(rows, -1)[at].long()
    exps = buf[off:off + scales * (d // 32)].view(scales, -1)[scale_at].double() - 127
    if c["fmt"] == "e4m3":
        e, m = (codes >> 3) & 15, codes & 7
        mag = torch.where(e > 0, (8 + m).double() * _two(e - 10), m.double() * 2.0 ** -9)
        val = torch.where(codes >= 128, -mag, mag)
    else:
        code = torch.stack([codes & 15, codes >> 4], -1).flatten(-2)
        e, m = (code >> 1) & 3, code & 1
        mag = torch.where(e > 0, (2 + m).double() * _two(e - 2), m.double() * 0.5)
        val = torch.where(code >= 8, -mag, mag)
    return val * _two(exps).repeat_interleave(32, -1)


def exact(case, seed):
    global own
    mine, own = own, False  # (the inputs alone)
    try:
        s = prepare(case, seed)
    finally:
        own = mine
    c = s["case"]
    group, sink, window = c["hq"] // c["hkv"], c["sink"], c["window"]
    o, lse = s["o"].double(), s["lse"].double()
    for i, (n, m) in enumerate(zip(_lengths(c), _new(c))):
        for h in range(c["hkv"]):
            k, v = _exact_rows(c, s, s["k"], i, h, n), _exact_rows(c, s, s["v"], i, h, n)
            heads = slice(h * group, (h + 1) * group)
            for t in range(0, m, 512):
                to = min(t + 512, m)
                place = torch.arange(n - m + t, n - m + to, device="cuda")[:, None]
                lo, hi = (max(n - m + t - window + 1, 0) if window else 0), n - m + to
                head = min(sink, lo)
                at = torch.cat([torch.arange(head, device="cuda"), torch.arange(lo, hi, device="cuda")])
                hidden = at > place
                if window:
                    hidden |= (at <= place - window) & (at >= sink)
                x = s["q"][i, t:to, heads].double().flatten(0, 1) @ torch.cat([k[:head], k[lo:hi]]).T.contiguous() / math.sqrt(c["d"])
                x = x.masked_fill(hidden.repeat_interleave(group, 0), -math.inf)
                o[i, t:to, heads] = (torch.softmax(x, -1) @ torch.cat([v[:head], v[lo:hi]])).unflatten(0, (-1, group))
                lse[i, t:to, heads] = torch.logsumexp(x, -1).unflatten(0, (-1, group))
    return dict(o=o, lse=lse)
