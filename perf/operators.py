"""The cache operators that performance work on this library is measured on, each in its plain form and as the library's call.

A case is one call of the kind a serving loop makes for one layer, through the public entry points:

  op "write"    vatt_write_kv: new tokens' q and k rows are rotated to their positions, k and v rows go into the cache in
                its format, the summaries of the blocks they touch are renewed.  `back`: followed by vatt_read_kv of the
                rows just written, which is how a quantised row is looked at.
  op "read"     vatt_read_kv: a run of rows of every sequence, back in bf16.
  op "select"   vatt_select_blocks: every KV head's best blocks by the upper bound of their scores.
  op "blocks"   vatt_block_decode: attention over listed blocks.
  op "dense"    vatt_dense_decode on a quantised cache.

`fmt`: "bf16", "e4m3" (8 bits a value) or "e2m1" (4 bits a value), the latter two with one power-of-two scale for 32 columns.
`page` 0 is the contiguous layout.  `block` is the number of tokens per block.  Sequences are ragged where n_lo < n.

Inputs: K ~ N(0, 1) in even KV heads and N(0, 1/4) in odd ones, every sixteenth column four times as large (real keys have
such columns, and scales and summaries feel them); V and q ~ N(0, 1), q smaller in the large columns.
"""
import math

import torch

own = False

VALUES = {"bf16": None, "e4m3": 448.0, "e2m1": 6.0}  # largest value of a format
FMT = {"bf16": 0, "e4m3": 1, "e2m1": 2}
E2M1 = [0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0]
LARGEST = 1.5 * 2.0 ** 127  # larger magnitudes are quantised as this


def _case(op, batch, n, **over):
    c = dict(op=op, batch=batch, n=n, n_lo=n, hq=32, hkv=8, d=128, q_len=1, fmt="bf16", page=0, block=16, sink=128, window=128,
             topk=0.025, n_new=1, new_lo=1, rotary=128, interleaved=False, scaling="none", fused=False, back=False, lists=False)
    c.update(over)
    return c


def listed():
    return [
        # the token of one chat on a small model: launch and latency only
        _case("write", 1, 1024, name="write 1 token", hq=8, hkv=2, d=64, rotary=64),
        # continuous batching on 16-token pages, the cache held in 8 bits, rotary stretched for long contexts by wavelength
        _case("write", 32, 8000, name="write 32 tokens e4m3 paged", n_lo=701, fmt="e4m3", page=16, scaling="wavelength", back=True),
        # prompts of several lengths in one padded batch, out of a fused projection; half of the head rotated, pairs side by side
        _case("write", 4, 2048, name="write prompts 4 x 0.3k-2k", n_lo=2048, n_new=2048, new_lo=331, rotary=64, interleaved=True, fused=True),
        # a long prompt into a 4-bit cache, and its rows back
        _case("write", 2, 16384, name="write prompts 2 x 16k e2m1", fmt="e2m1", n_new=16384, new_lo=16384, scaling="yarn", back=True),
        # a prefix handed to another program: ragged, odd lengths, 8-bit pages
        _case("read", 7, 4999, name="read 7 x 0.5k-5k e4m3 paged", n_lo=517, fmt="e4m3", page=64),
        # whole sequences of a 4-bit cache
        _case("read", 8, 16384, name="read 8 x 16k e2m1", fmt="e2m1", d=64, hq=16),
        # one sequence at the benchmark's 32K context
        _case("select", 1, 32768, name="select 1 x 32k"),
        # a batch up to the 128K capacity of the model family the shapes come from, token lists for the verified step
        _case("select", 12, 131072, name="select 12 x 8k-128k paged", n_lo=8192, page=64, lists=True),
        # the same two settings' attention over the blocks chosen
        _case("blocks", 1, 32768, name="blocks 1 x 32k"),
        _case("blocks", 12, 65536, name="blocks 12 x 4k-64k e4m3 paged, 2 queries", n_lo=4099, fmt="e4m3", page=64, q_len=2, topk=0.05),
        # layers that are kept dense, on a quantised cache
        _case("dense", 16, 32768, name="dense 16 x 32k e4m3", fmt="e4m3"),
        _case("dense", 3, 9001, name="dense 3 x 1k-9k e2m1, 3 queries", n_lo=1003, fmt="e2m1", hq=16, hkv=2, d=64, q_len=3),
    ]


SHAPES = [(32, 8, 128), (32, 8, 128), (32, 4, 128), (16, 16, 64), (16, 8, 64), (8, 8, 128)]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """Any operator, shape, format, layout and length within the limits of the listed cases."""
    op = rng.choice(["write", "write", "read", "select", "blocks", "blocks", "dense"])
    hq, hkv, d = rng.choice(SHAPES)
    page = rng.choice([0, 0, 16, 64, 128])
    fmt = rng.choice(["e4m3", "e2m1"] if op == "dense" else ["bf16", "e4m3", "e2m1"])
    most = dict(write=32768, read=131072, select=800000, blocks=400000, dense=500000)[op] * 8 // max(8, hkv)
    n = _log(rng, 1 if op in ("write", "read") else 40, min(most, 131072))
    batch = max(1, min(_log(rng, 1, 48), most // n))
    ragged = batch > 1 and rng.random() < 0.6
    over = dict(n_lo=max(1, n // 16) if ragged else n, hq=hq, hkv=hkv, d=d, page=page, fmt=fmt)
    over["block"] = rng.choice([b for b in (16, 16, 32, 64) if not page or b <= page])
    if op == "write":
        prompt = rng.random() < 0.6
        over["n_new"] = n if prompt else rng.choice([1, 1, 1, 4])
        over["new_lo"] = max(1, n // 9) if prompt and ragged else over["n_new"]
        over["n_lo"] = n if prompt else max(over["n_lo"], over["n_new"])
        n = max(n, over["n_new"])
        over["n_lo"] = min(n, max(over["n_lo"], over["n_new"]))
        over["rotary"] = rng.choice([d, d, d // 2, d // 4])
        over["interleaved"] = rng.random() < 0.4
        over["scaling"] = rng.choice(["none", "linear", "wavelength", "yarn"])
        over["fused"] = rng.random() < 0.5
        over["back"] = fmt != "bf16"
    if op in ("select", "blocks", "dense"):
        over["q_len"] = rng.choice([1, 1, 1, 2, 5])
        over["n_lo"] = max(over["n_lo"], over["q_len"])
        if batch * n * over["q_len"] > most:
            over["q_len"] = 1
        over["sink"], over["window"] = rng.choice([(128, 128), (128, 512), (4, 64), (0, 0)])
        over["topk"] = rng.choice([0.01, 0.025, 0.05, 0.1])
        over["lists"] = op == "select" and rng.random() < 0.5
    if op == "select":
        over["fmt"] = "bf16"
    return _case(op, batch, n, **over)


# ---- sizes, which follow from the case alone -----------------------------------------------------------------------------

def _spread(hi, lo, count):
    """hi, and the others evenly down to lo, in a scattered order."""
    if count == 1 or lo == hi:
        return [hi] * count
    got = [hi - (hi - lo) * i // (count - 1) for i in range(count)]
    return [got[(i * 7 + 3) % count] if math.gcd(7, count) == 1 else got[i] for i in range(count)]


def _lengths(c):
    """Tokens of every sequence, the new ones of a write among them."""
    return _spread(c["n"], c["n_lo"], c["batch"])


def _new(c):
    return _spread(c["n_new"], c["new_lo"], c["batch"])


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


def _parts(c, n):
    """How a query that sees n tokens divides its blocks: (sink blocks, first window block, blocks, blocks to choose)."""
    bs = c["block"]
    total = -(-n // bs)
    lo, hi = -(-min(c["sink"], n) // bs), max(n - max(c["window"], 1), 0) // bs
    if lo >= hi:
        return total, total, total, 0
    return lo, hi, total, min(_topk(c, n) // bs, hi - lo)


def _topk(c, n):
    return int(math.floor(_f32(c["topk"]) * n))


def _f32(x):
    return float(torch.tensor(x, dtype=torch.float32))


def _list_room(c):
    """Entries that a list of blocks has room for."""
    bs = c["block"]
    return min(-(-_n_max(c) // bs), -(-c["sink"] // bs) + c["window"] // bs + 2 + _topk(c, _n_max(c)) // bs)


def _seen(c):
    """Tokens that each query token of each sequence sees."""
    return [[max(n - (c["q_len"] - 1 - t), 1) for t in range(c["q_len"])] for n in _lengths(c)]


def _attended(c):
    """Tokens of the lists that prepare() makes, for every query."""
    got = []
    for row in _seen(c):
        for n in row:
            lo, hi, total, m = _parts(c, n)
            got.append(n if lo >= hi else lo * c["block"] + m * c["block"] + n - hi * c["block"])
    return got


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


def _plan(c):
    """The library's plan of a case with its workspace: what a serving process keeps for a layer."""
    from paper_2510_05688_amd import binding as vb

    class Kept:
        def __init__(self):
            pages = _sizes(c)[0]
            self.plan = vb.vatt_plan_create_chunk(
                dict(batch=c["batch"], n_q_heads=c["hq"], n_kv_heads=c["hkv"], head_dim=c["d"], n_max=_n_max(c),
                     kv_layout=1 if c["page"] else 0, page_size=c["page"], num_blocks=pages, sink=c["sink"], window=c["window"],
                     topk_abs=0, topk_frac=c["topk"], base_abs=0, base_frac=0.025, epsilon=0.05, delta=0.05, target=0,
                     sm_scale=0.0, budget_cap_frac=1.0), c["q_len"], torch.cuda.current_device())
            vb.vatt_plan_set_option(self.plan, vb.VATT_OPT_KV_FORMAT, FMT[c["fmt"]])
            vb.vatt_plan_set_option(self.plan, vb.VATT_OPT_BLOCK_TOKENS, c["block"])
            if c["op"] == "write":
                vb.vatt_plan_set_rotary(self.plan, _rotary(c))
            self.workspace = None
            if c["op"] in ("select", "blocks", "dense"):
                self.workspace = torch.empty(vb.vatt_plan_workspace_bytes(self.plan), dtype=torch.uint8, device="cuda")

        def __del__(self):
            vb.vatt_plan_destroy(self.plan)

    return Kept()


def _rotary(c):
    r = dict(rotary_dim=c["rotary"], layout=1 if c["interleaved"] else 0, theta=500000.0)
    if c["scaling"] == "linear":
        r.update(scaling=1, factor=4.0)
    if c["scaling"] == "wavelength":
        r.update(scaling=2, factor=8.0, low=1.0, high=4.0, original_len=8192)
    if c["scaling"] == "yarn":
        r.update(scaling=3, factor=4.0, low=1.0, high=32.0, original_len=8192)
    return r


def _lists(c, g):
    """Block lists as a selection leaves them: sink blocks, random ones between, window blocks, ascending."""
    b, q, hkv, room = c["batch"], c["q_len"], c["hkv"], _list_room(c)
    parts = torch.tensor([_parts(c, n) for row in _seen(c) for n in row], device="cuda")
    lo, hi, total, m = (parts[:, i, None, None] for i in range(4))
    nb = -(-_n_max(c) // c["block"])
    at = torch.arange(nb, device="cuda")
    order = torch.rand((b * q, hkv, nb), generator=g, device="cuda").masked_fill((at < lo) | (at >= hi), 2.0)
    rank = order.argsort(-1).argsort(-1)
    return _ascending((rank < m) | (at < lo) | ((at >= hi) & (at < total)), room)


def _ascending(chosen, room):
    """(the chosen places in ascending order, -1 behind them; how many)"""
    nb = chosen.shape[-1]
    at = torch.arange(nb, device=chosen.device)
    places = torch.where(chosen, at, nb).sort(-1).values
    places = torch.nn.functional.pad(places, (0, max(0, room - nb)), value=nb)[..., :room]
    return torch.where(places < nb, places, -1).int().contiguous(), chosen.sum(-1).int()


def prepare(case, seed):
    c = dict(case)
    b, hq, hkv, d, q = c["batch"], c["hq"], c["hkv"], c["d"], c["q_len"]
    s = dict(case=c, kept=_plan(c) if own else None, table=None)
    pages, rows, scales, off = _sizes(c)
    if c["page"]:
        s["table"] = torch.randperm(pages, generator=_gen(seed, 1), device="cuda")[:b * (_n_max(c) // c["page"])].int().reshape(b, -1).contiguous()
    s["lens"] = torch.tensor(_lengths(c), dtype=torch.int32, device="cuda")
    if c["op"] != "select":
        s["k"], s["v"] = _fill(c, _gen(seed, 2), True), _fill(c, _gen(seed, 3), False)
    cols = _columns(d)
    if c["op"] == "write":
        n_new = c["n_new"]
        first = [n - m for n, m in zip(_lengths(c), _new(c))]
        s["first"] = torch.tensor(first, dtype=torch.int32, device="cuda")
        s["new"] = torch.tensor(_new(c), dtype=torch.int32, device="cuda")
        s["after"] = torch.zeros(b, dtype=torch.int32, device="cuda")
        wide = (hq + 2 * hkv) * d
        x = torch.randn((b, n_new, wide), generator=_gen(seed, 4), device="cuda").to(torch.bfloat16)
        x[..., hq * d:(hq + hkv) * d] *= cols.to(torch.bfloat16).repeat(hkv)
        at = [0, hq * d, (hq + hkv) * d, wide]
        heads = [x[..., at[i]:at[i + 1]].unflatten(-1, (-1, d)) for i in range(3)]
        s["q"], s["k_new"], s["v_new"] = heads if c["fused"] else [h.contiguous() for h in heads]
        s["out_q"] = torch.zeros((b, n_new, hq, d), dtype=torch.bfloat16, device="cuda")
        s["summary"] = torch.zeros(_summary_shape(c), dtype=torch.bfloat16, device="cuda")
    else:
        x = torch.randn((b, q, hq, d), generator=_gen(seed, 4), device="cuda") / cols.sqrt()
        s["q"] = x.to(torch.bfloat16)
    if c["op"] == "read" or c["back"]:
        count = c["n_new"] if c["back"] else c["n"]
        s["back"] = [torch.zeros((b, hkv, count, d), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
        s["from"] = s["first"] if c["back"] else torch.tensor([min(3 * i, n - 1) for i, n in enumerate(_lengths(c))], dtype=torch.int32, device="cuda")
    if c["op"] == "select":
        x = torch.randn(_summary_shape(c), generator=_gen(seed, 5), device="cuda") * 0.5
        head = torch.ones(hkv, device="cuda")
        head[1::2] = 0.5
        x[..., 0, :], x[..., 1, :] = x[..., 0, :] + 1.7, x[..., 1, :] - 1.7  # the expected extremes of 16 rows, and their spread
        s["summary"] = (x * cols * head[:, None, None, None]).to(torch.bfloat16)
        room, k_max = _list_room(c), _topk(c, _n_max(c))
        s["blocks"] = torch.full((b * q, hkv, room), -1, dtype=torch.int32, device="cuda")
        s["count"] = torch.zeros((b * q, hkv), dtype=torch.int32, device="cuda")
        if c["lists"]:
            s["topk"] = torch.full((b * q, hq, max(k_max, 1)), -1, dtype=torch.int32, device="cuda")
            s["topk_count"] = torch.zeros((b * q, hq), dtype=torch.int32, device="cuda")
    if c["op"] == "blocks":
        s["blocks"], s["count"] = _lists(c, _gen(seed, 6))
    if c["op"] in ("blocks", "dense"):
        s["o"] = torch.zeros((b * q, hq, d), dtype=torch.float32, device="cuda")
        s["lse"] = torch.zeros((b * q, hq), dtype=torch.float32, device="cuda")
    return s


def _summary_shape(c):
    if c["page"]:
        return (_sizes(c)[0], c["hkv"], c["page"] // c["block"], 2, c["d"])
    return (c["batch"], c["hkv"], -(-_n_max(c) // c["block"]), 2, c["d"])


# ---- plain forms ---------------------------------------------------------------------------------------------------------

def _two(e):
    """2^e in 64 bits, from its bits: pow() need not be exact."""
    return ((e.long() + 1023) << 52).view(torch.float64)


def _quantise(x, fmt):
    """fp32 [..., d] -> (codes uint8 [..., d or d / 2], scale bytes uint8 [..., d / 32]): per 32 columns the smallest power of
    two at which no magnitude is above the format's largest; values to the nearest, ties to even; a group with an Inf or a NaN
    has scale byte 255 and codes 0."""
    groups = x.unflatten(-1, (-1, 32))
    finite = torch.isfinite(groups).all(-1)
    groups = groups.clamp(-LARGEST, LARGEST)
    mant, exp = torch.frexp(groups.abs().amax(-1))  # mant in [1/2, 1)
    limit = VALUES[fmt]
    lm, le = math.frexp(limit)
    e = torch.where(mant > lm, exp - le + 1, exp - le)
    e = torch.where(mant > 0, e, -127).clamp(min=-127)
    e = torch.where(finite, e, 0)
    y = torch.where(finite[..., None], groups, 0.0)
    y = (y.double() * _two(-e)[..., None]).float()
    if fmt == "e4m3":
        codes = y.to(torch.float8_e4m3fn).view(torch.uint8).flatten(-2)
    else:
        a = y.abs()
        step = torch.where(a < 2, 0.5, torch.where(a < 4, 1.0, 2.0))
        r = torch.round(a / step) * step
        code = torch.where(r < 2, r * 2, torch.where(r < 4, r + 2, r / 2 + 4)).to(torch.uint8)
        code = (code | (torch.signbit(y).to(torch.uint8) << 3)).flatten(-2).unflatten(-1, (-1, 2))
        codes = code[..., 0] | (code[..., 1] << 4)
    return codes, torch.where(finite, e + 127, 255).to(torch.uint8)


def _values(codes, exps, fmt):
    """What codes and scale bytes stand for, in fp32."""
    if fmt == "e4m3":
        v = codes.view(torch.float8_e4m3fn).float()
    else:
        table = torch.tensor(E2M1 + [-x for x in E2M1], device=codes.device)
        v = torch.stack([table[(codes & 15).long()], table[(codes >> 4).long()]], -1).flatten(-2)
    v = (v.unflatten(-1, (-1, 32)).double() * _two(exps.int() - 127)[..., None]).float()
    return torch.where(exps[..., None] == 255, torch.nan, v).flatten(-2)


def _row_index(s, tokens, scales=False):
    """Physical rows of `tokens` ([B, ...] positions) for every KV head: [B, Hkv, ...]."""
    c = s["case"]
    b, hkv = c["batch"], c["hkv"]
    more = (1,) * (tokens.dim() - 1)
    heads = torch.arange(hkv, device=tokens.device).view(1, hkv, *more)
    if c["page"]:
        page = torch.gather(s["table"].long(), 1, (tokens // c["page"]).reshape(b, -1)).reshape(tokens.shape)
        return (page[:, None] * hkv + heads) * c["page"] + (tokens % c["page"])[:, None]
    per = -(-_n_max(c) // 8) * 8 if scales else _n_max(c)
    seqs = torch.arange(b, device=tokens.device).view(b, 1, *more)
    return (seqs * hkv + heads) * per + tokens[:, None]


def _load(s, buf, tokens):
    """Rows of `tokens` in fp32: [B, Hkv, ..., d]."""
    return _load_rows(s, buf, _row_index(s, tokens), _row_index(s, tokens, True))


def _load_rows(s, buf, rows_at, scales_at):
    c = s["case"]
    d = c["d"]
    if c["fmt"] == "bf16":
        return buf.view(-1, d)[rows_at].float()
    pages, rows, scales, off = _sizes(c)
    codes = buf[:rows * _row_bytes(c)].view(rows, -1)[rows_at]
    return _values(codes, buf[off:off + scales * (d // 32)].view(scales, -1)[scales_at], c["fmt"])


def _store(s, buf, tokens, valid, x):
    """fp32 rows x [B, Hkv, T, d] to the cache, where valid ([B, T])."""
    c = s["case"]
    keep = valid[:, None].expand(-1, c["hkv"], -1)
    at = _row_index(s, tokens)[keep]
    if c["fmt"] == "bf16":
        buf.view(-1, c["d"])[at] = x[keep].to(torch.bfloat16)
        return
    pages, rows, scales, off = _sizes(c)
    codes, exps = _quantise(x[keep], c["fmt"])
    buf[:rows * _row_bytes(c)].view(rows, -1)[at] = codes
    buf[off:off + scales * (c["d"] // 32)].view(scales, -1)[_row_index(s, tokens, True)[keep]] = exps


def _frequencies(c):
    """(angle per position of each rotated pair, factor of the rotated values), in 64 bits."""
    half = c["rotary"] // 2
    i = torch.arange(half, dtype=torch.float64, device="cuda")
    f = 500000.0 ** (-i / half)
    if c["scaling"] == "linear":
        return f / 4.0, 1.0
    if c["scaling"] == "wavelength":  # turns within the original length decide how much of a frequency is divided
        turns = 8192 * f / (2 * math.pi)
        keep = ((turns - 1.0) / (4.0 - 1.0)).clamp(0.0, 1.0)
        return f * keep + f / 8.0 * (1 - keep), 1.0
    if c["scaling"] == "yarn":  # the same by a ramp over the pair's number between the pairs of 32 and of 1 turn
        def pair(turns):
            return c["rotary"] * math.log(8192 / (turns * 2 * math.pi)) / (2 * math.log(500000.0))
        lo, hi = max(math.floor(pair(32.0)), 0), min(math.ceil(pair(1.0)), c["rotary"] - 1)
        keep = 1 - ((i - lo) / max(hi - lo, 0.001)).clamp(0.0, 1.0)
        return f * keep + f / 4.0 * (1 - keep), 0.1 * math.log(4.0) + 1.0
    return f, 1.0


def _rotate(c, x, positions):
    """x [B, T, H, d] in fp32, rotated to `positions` [B, T]; angles in 64 bits."""
    f, factor = _frequencies(c)
    angle = positions[..., None].double() * f
    cos, sin = (factor * angle.cos()).float()[:, :, None], (factor * angle.sin()).float()[:, :, None]
    r = c["rotary"]
    if c["interleaved"]:
        a, b = x[..., 0:r:2], x[..., 1:r:2]
        return torch.cat([torch.stack([a * cos - b * sin, b * cos + a * sin], -1).flatten(-2), x[..., r:]], -1)
    a, b = x[..., :r // 2], x[..., r // 2:r]
    return torch.cat([a * cos - b * sin, b * cos + a * sin, x[..., r:]], -1)


def _write(s):
    c = s["case"]
    d, bs, hkv = c["d"], c["block"], c["hkv"]
    j = torch.arange(c["n_new"], device="cuda")
    positions = s["first"].long()[:, None] + j
    valid = (j < s["new"][:, None]) & (positions < _n_max(c))
    tokens = positions.clamp(max=_n_max(c) - 1)
    q, k = _rotate(c, s["q"].float(), positions), _rotate(c, s["k_new"].float(), positions)
    s["out_q"].copy_(torch.where(valid[..., None, None], q.to(torch.bfloat16), s["out_q"]))
    _store(s, s["k"], tokens, valid, k.transpose(1, 2))
    _store(s, s["v"], tokens, valid, s["v_new"].float().transpose(1, 2))
    s["after"].copy_(s["first"] + valid.sum(1))
    # the blocks that got a row: their extremes over all tokens that the sequence has now
    some = (c["n_new"] + bs - 2) // bs + 1
    blocks = s["first"].long()[:, None] // bs + torch.arange(some, device="cuda")
    at = blocks[..., None] * bs + torch.arange(bs, device="cuda")
    there = at < s["after"][:, None, None]
    rows = _load(s, s["k"], at.clamp(max=_n_max(c) - 1).flatten(1)).unflatten(2, (some, bs)).to(torch.bfloat16)
    top = torch.where(there[:, None, ..., None], rows, -torch.inf).amax(3)
    low = torch.where(there[:, None, ..., None], rows, torch.inf).amin(3)
    got = there[..., 0][:, None].expand(-1, hkv, -1)
    per = c["page"] // bs if c["page"] else _summary_shape(c)[2]
    if c["page"]:
        head = torch.arange(hkv, device="cuda")[None, :, None]
        page = torch.gather(s["table"].long(), 1, (blocks * bs // c["page"]).clamp(max=s["table"].shape[1] - 1))[:, None]
        place = (page * hkv + head) * per + (blocks % per)[:, None]
    else:
        place = torch.arange(c["batch"] * hkv, device="cuda").view(c["batch"], hkv, 1) * per + blocks[:, None]
    s["summary"].view(-1, 2, d)[place[got]] = torch.stack([top, low], -2)[got]
    out = dict(q=s["out_q"], summary=s["summary"], after=s["after"])
    if c["back"]:
        out.update(_read(s))
    else:
        out.update(k=s["k"], v=s["v"])
    return out


def _read(s):
    c = s["case"]
    count = s["back"][0].shape[2]
    tokens = s["from"].long()[:, None] + torch.arange(count, device="cuda")
    end = s["after"] if c["back"] else s["lens"]
    there = (tokens < end[:, None])[:, None, :, None]
    tokens = tokens.clamp(max=_n_max(c) - 1)
    for buf, out in zip((s["k"], s["v"]), s["back"]):
        out.copy_(torch.where(there, _load(s, buf, tokens).to(torch.bfloat16), out))
    return dict(back_k=s["back"][0], back_v=s["back"][1])


def _summaries(s):
    """[B, Hkv, blocks, 2, d]"""
    c = s["case"]
    if not c["page"]:
        return s["summary"]
    x = s["summary"][s["table"].long()]  # [B, pages, Hkv, blocks per page, 2, d]
    return x.transpose(1, 2).flatten(2, 3)


def _select(s):
    c = s["case"]
    b, q, hkv, d, bs = c["batch"], c["q_len"], c["hkv"], c["d"], c["block"]
    ends = _summaries(s)
    nb = ends.shape[2]
    qs = s["q"].double().reshape(b, q, hkv, -1, d).permute(0, 2, 1, 3, 4).flatten(2, 3)  # [B, Hkv, q * group, d]
    score = qs.clamp(min=0) @ ends[..., 0, :].double().transpose(-1, -2).contiguous()
    score += qs.clamp(max=0) @ ends[..., 1, :].double().transpose(-1, -2).contiguous()
    score = score.unflatten(2, (q, -1)).amax(3).float().transpose(1, 2).flatten(0, 1)  # [B * q, Hkv, blocks]
    seen = (s["lens"].long()[:, None] - (q - 1) + torch.arange(q, device="cuda")).clamp(min=1).flatten()
    total = (seen + bs - 1) // bs
    lo = (seen.clamp(max=c["sink"]) + bs - 1) // bs
    hi = (seen - max(c["window"], 1)).clamp(min=0) // bs
    lo, hi = torch.where(lo < hi, lo, total), torch.where(lo < hi, hi, total)
    m = torch.minimum((_f32(c["topk"]) * seen.double()).floor().long() // bs, hi - lo)
    lo, hi, total, m = (x[:, None, None] for x in (lo, hi, total, m))
    at = torch.arange(nb, device="cuda")
    between = (at >= lo) & (at < hi)
    rank = torch.where(between, score, -torch.inf).sort(dim=-1, descending=True, stable=True).indices.argsort(-1)
    best = between & (rank < m)
    blocks, count = _ascending(best | (at < lo) | ((at >= hi) & (at < total)), s["blocks"].shape[2])
    s["blocks"].copy_(torch.where(blocks >= 0, blocks, s["blocks"]))
    s["count"].copy_(count)
    out = dict(blocks=s["blocks"], count=s["count"])
    if c["lists"]:
        room = s["topk"].shape[2]
        chosen, number = _ascending(best, -(-room // bs))
        tokens = (chosen[..., None] * bs + torch.arange(bs, dtype=torch.int32, device="cuda")).flatten(2)[..., :room]
        per_head = torch.where(torch.arange(room, device="cuda") < (number * bs)[..., None], tokens, -1)
        s["topk"].copy_(per_head.repeat_interleave(c["hq"] // hkv, 1))
        s["topk_count"].copy_((number * bs).repeat_interleave(c["hq"] // hkv, 1))
        out.update(topk=s["topk"], topk_count=s["topk_count"])
    return out


def _attend(s, q, k, v, there):
    """q [..., G, d], k and v [..., T, d], there [..., 1, T]: softmax(q k^T) v over the tokens that are there, and ln of its sum."""
    x = (q @ k.transpose(-1, -2).contiguous()) / math.sqrt(q.shape[-1])
    x = torch.where(there, x, -torch.inf)
    m = x.amax(-1, keepdim=True)
    p = (x - m).exp()
    total = p.sum(-1, keepdim=True)
    return (p @ v) / total, (m + total.log()).squeeze(-1)


def _blocks(s):
    c = s["case"]
    b, q, hkv, d, bs = c["batch"], c["q_len"], c["hkv"], c["d"], c["block"]
    lists = s["blocks"].long().view(b, q, hkv, -1)
    tokens = (lists[..., None] * bs + torch.arange(bs, device="cuda")).flatten(3)  # [B, q, Hkv, T]
    seen = (s["lens"].long()[:, None] - (q - 1) + torch.arange(q, device="cuda")).clamp(min=1)
    there = (lists >= 0)[..., None].expand(-1, -1, -1, -1, bs).flatten(3) & (tokens < seen[..., None, None])
    tokens = tokens.clamp(0, _n_max(c) - 1)
    head = torch.arange(hkv, device="cuda")[:, None]
    if c["page"]:
        page = torch.gather(s["table"].long(), 1, (tokens // c["page"]).flatten(1)).view(tokens.shape)
        rows = (page * hkv + head) * c["page"] + tokens % c["page"]
        scales = rows
    else:
        base = torch.arange(b, device="cuda").view(b, 1, 1, 1) * hkv + head
        rows, scales = base * _n_max(c) + tokens, base * (-(-_n_max(c) // 8) * 8) + tokens
    k, v = (_load_rows(s, s[x], rows, scales) for x in "kv")
    o, lse = _attend(s, s["q"].float().view(b, q, hkv, -1, d), k, v, there[..., None, :])
    s["o"].copy_(o.view(s["o"].shape))
    s["lse"].copy_(lse.view(s["lse"].shape))
    return dict(o=s["o"], lse=s["lse"])


def _dense(s):
    c = s["case"]
    b, q, hkv, d = c["batch"], c["q_len"], c["hkv"], c["d"]
    tokens = torch.arange(c["n"], device="cuda").expand(b, -1)
    k, v = (_load(s, s[x], tokens) for x in "kv")
    qs = s["q"].float().view(b, q, hkv, -1, d).transpose(1, 2).flatten(2, 3)  # [B, Hkv, q * group, d]
    seen = (s["lens"].long()[:, None] - (q - 1) + torch.arange(q, device="cuda")).clamp(min=1)
    there = (tokens[:, None] < seen[..., None]).repeat_interleave(c["hq"] // hkv, 1)[:, None]
    o, lse = _attend(s, qs, k, v, there)
    s["o"].copy_(o.unflatten(2, (q, -1)).transpose(1, 2).reshape(s["o"].shape))
    s["lse"].copy_(lse.unflatten(2, (q, -1)).transpose(1, 2).reshape(s["lse"].shape))
    return dict(o=s["o"], lse=s["lse"])


# ---- one pass ------------------------------------------------------------------------------------------------------------

def run(state):
    s, op = state, state["case"]["op"]
    if not own:
        return dict(write=_write, read=_read, select=_select, blocks=_blocks, dense=_dense)[op](s)
    from paper_2510_05688_amd import binding as vb

    plan, ws = s["kept"].plan, s["kept"].workspace
    stream = torch.cuda.current_stream().cuda_stream
    if op == "write":
        strides = [vb.token_stride(s[x]) for x in ("q", "k_new", "v_new")]
        vb.vatt_write_kv(plan, s["q"], s["k_new"], s["v_new"], *strides, s["case"]["n_new"], s["first"], s["new"], s["k"], s["v"],
                         s["table"], s["summary"], s["out_q"], s["after"], stream)
        out = dict(q=s["out_q"], summary=s["summary"], after=s["after"])
        if not s["case"]["back"]:
            out.update(k=s["k"], v=s["v"])
            return out
        vb.vatt_read_kv(plan, s["k"], s["v"], s["table"], s["after"], s["first"], s["case"]["n_new"], s["back"][0], s["back"][1],
                        stream)
        out.update(back_k=s["back"][0], back_v=s["back"][1])
        return out
    if op == "read":
        vb.vatt_read_kv(plan, s["k"], s["v"], s["table"], s["lens"], s["from"], s["case"]["n"], s["back"][0], s["back"][1], stream)
        return dict(back_k=s["back"][0], back_v=s["back"][1])
    if op == "select":
        vb.vatt_select_blocks(plan, s["q"], s["summary"], s["table"], s["lens"], ws, s["blocks"], s["count"], s.get("topk"),
                              s.get("topk_count"), stream)
        out = dict(blocks=s["blocks"], count=s["count"])
        if s["case"]["lists"]:
            out.update(topk=s["topk"], topk_count=s["topk_count"])
        return out
    if op == "blocks":
        vb.vatt_block_decode(plan, s["q"], s["k"], s["v"], s["table"], s["lens"], s["blocks"], s["count"], ws, s["o"], s["lse"], stream)
    else:
        vb.vatt_dense_decode(plan, s["q"], s["k"], s["v"], s["table"], s["lens"], ws, s["o"], s["lse"], stream)
    return dict(o=s["o"], lse=s["lse"])


def work(case):
    """Inputs read once, outputs written once."""
    c = case
    hq, hkv, d, q, op = c["hq"], c["hkv"], c["d"], c["q_len"], c["op"]
    row, bs = _stored(c), c["block"]
    nbytes = flops = 0.0
    if op == "write":
        for n, m in zip(_lengths(c), _new(c)):
            first = n - m
            touched = -(-n // bs) - first // bs
            nbytes += m * (hq + 2 * hkv) * d * 2 + m * hq * d * 2 + 2 * m * hkv * row
            nbytes += hkv * (touched * 4 * d + (first % bs) * row)
            nbytes += 2 * m * hkv * 2 * d if c["back"] else 0  # (the rows come back from what was just written)
            flops += m * (hq + hkv) * c["rotary"] * 3.0
    elif op == "read":
        rows = sum(n - min(3 * i, n - 1) for i, n in enumerate(_lengths(c)))
        nbytes += 2 * hkv * rows * (row + 2 * d)
        flops += 2.0 * hkv * rows * d
    elif op == "select":
        for row_ in _seen(c):
            read = 0
            for n in row_:
                lo, hi, total, m = _parts(c, n)
                read = max(read, hi - lo)
                flops += 2.0 * hq * (hi - lo) * d
                nbytes += hkv * 4 * (total if lo >= hi else lo + m + total - hi) + (4 * hq * m * bs if c["lists"] else 0)
            nbytes += hkv * read * 4 * d + q * hq * d * 2
    elif op == "blocks":
        for n in _attended(c):
            nbytes += 2 * hkv * n * row + hq * d * 6 + hkv * 4 * (n // bs)
            flops += 4.0 * hq * n * d
    else:
        for n in _lengths(c):
            nbytes += 2 * hkv * n * row + q * hq * d * 6
            flops += 4.0 * hq * q * n * d
    return dict(bytes=nbytes, flops=flops)


# ---- the definitions in 64 bits ------------------------------------------------------------------------------------------

def _grid(c, x):
    """x rounded to what the case's format can hold, in 64 bits."""
    if c["fmt"] == "bf16":
        return x
    g = x.clamp(-LARGEST, LARGEST).unflatten(-1, (-1, 32))
    top = g.abs().amax(-1, keepdim=True)
    e = torch.ceil(torch.log2(torch.where(top > 0, top, 1.0) / VALUES[c["fmt"]]))
    e = e + (top > VALUES[c["fmt"]] * _two(e)).double() - (top <= VALUES[c["fmt"]] * _two(e - 1)).double()
    unit = _two(torch.where(top > 0, e, -127.0).clamp(min=-127))
    y = g / unit
    least, bits = (-6, 3) if c["fmt"] == "e4m3" else (0, 1)
    octave = torch.frexp(y.abs().clamp(min=2.0 ** least)).exponent - 1
    ulp = _two(octave - bits)
    return (torch.round(y / ulp) * ulp * unit).flatten(-2)


def _exact_rows(c, s, buf, b, head, tokens):
    """Rows of one sequence and KV head in 64 bits."""
    if c["page"]:
        page = s["table"][b].long()[tokens // c["page"]]
        at = (page * c["hkv"] + head) * c["page"] + tokens % c["page"]
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
    b, hq, hkv, d, q, op = c["batch"], c["hq"], c["hkv"], c["d"], c["q_len"], c["op"]
    if op == "select":
        return None  # whole numbers
    if op in ("blocks", "dense"):
        o = torch.zeros((b * q, hq, d), dtype=torch.float64, device="cuda")
        lse = torch.zeros((b * q, hq), dtype=torch.float64, device="cuda")
        grp = hq // hkv
        lens = _lengths(c)
        lists = [[None] * hkv for _ in range(b * q)] if op == "dense" else s["blocks"].tolist()
        for i in range(b):
            for h in range(hkv):
                if op == "dense":
                    k, v = (_exact_rows(c, s, s[x], i, h, torch.arange(lens[i], device="cuda")) for x in "kv")
                for t in range(q):
                    n = max(lens[i] - (q - 1 - t), 1)
                    if op == "blocks":
                        at = torch.tensor([x for x in lists[i * q + t][h] if x >= 0], device="cuda")
                        at = (at[:, None] * c["block"] + torch.arange(c["block"], device="cuda")).flatten()
                        k, v = (_exact_rows(c, s, s[x], i, h, at[at < n]) for x in "kv")
                        n = k.shape[0]
                    x = s["q"][i, t, h * grp:(h + 1) * grp].double() @ k[:n].T.contiguous() / math.sqrt(d)
                    o[i * q + t, h * grp:(h + 1) * grp] = torch.softmax(x, -1) @ v[:n]
                    lse[i * q + t, h * grp:(h + 1) * grp] = torch.logsumexp(x, -1)
        return dict(o=o, lse=lse)
    if op == "read":
        back = [x.double() for x in s["back"]]
        for i, n in enumerate(_lengths(c)):
            first = int(s["from"][i])
            for h in range(hkv):
                for x, out in zip("kv", back):
                    out[i, h, :n - first] = _exact_rows(c, s, s[x], i, h, torch.arange(first, n, device="cuda"))
        return dict(back_k=back[0], back_v=back[1])
    # write
    f, factor = _frequencies(c)
    half = c["rotary"] // 2
    out_q, back = s["out_q"].double(), [x.double() for x in s.get("back", [])]
    summary = s["summary"].double().view(-1, 2, d)
    cache = [s[x].view(-1, d).double() for x in "kv"] if not c["back"] else None
    for i, (n, m) in enumerate(zip(_lengths(c), _new(c))):
        first = n - m
        turn = torch.polar(torch.tensor(factor, dtype=torch.float64, device="cuda"), torch.arange(first, n, device="cuda").double()[:, None] * f)[:, None]
        rows = []
        for x in (s["q"], s["k_new"]):
            x = x[i, :m].double()
            r = x[..., :c["rotary"]]
            z = torch.view_as_complex(r.unflatten(-1, (half, 2)).contiguous()) if c["interleaved"] else torch.complex(r[..., :half], r[..., half:])
            z = z * turn
            r = torch.view_as_real(z).flatten(-2) if c["interleaved"] else torch.cat([z.real, z.imag], -1)
            rows.append(torch.cat([r, x[..., c["rotary"]:]], -1))
        out_q[i, :m] = rows[0]
        new_k, new_v = _grid(c, rows[1]), _grid(c, s["v_new"][i, :m].double())
        start = first // c["block"] * c["block"]
        for h in range(hkv):
            if c["back"]:
                back[0][i, h, :m], back[1][i, h, :m] = new_k[:, h], new_v[:, h]
            else:
                at = torch.arange(first, n, device="cuda")
                page = s["table"][i].long()[at // c["page"]] if c["page"] else None
                at = (page * hkv + h) * c["page"] + at % c["page"] if c["page"] else (i * hkv + h) * _n_max(c) + at
                cache[0][at], cache[1][at] = new_k[:, h], new_v[:, h]
            k = torch.cat([_exact_rows(c, s, s["k"], i, h, torch.arange(start, first, device="cuda")), new_k[:, h]])
            gap = -len(k) % c["block"]
            top = torch.nn.functional.pad(k, (0, 0, 0, gap), value=-math.inf).unflatten(0, (-1, c["block"])).amax(1)
            low = torch.nn.functional.pad(k, (0, 0, 0, gap), value=math.inf).unflatten(0, (-1, c["block"])).amin(1)
            blocks = torch.arange(start // c["block"], -(-n // c["block"]), device="cuda")
            if c["page"]:
                per = c["page"] // c["block"]
                place = (s["table"][i].long()[blocks // per] * hkv + h) * per + blocks % per
            else:
                place = (i * hkv + h) * _summary_shape(c)[2] + blocks
            summary[place] = torch.stack([top, low], 1)
    out = dict(q=out_q, summary=summary.view(s["summary"].shape), after=None)
    if c["back"]:
        out.update(back_k=back[0], back_v=back[1])
    else:
        out.update(k=cache[0].view(s["k"].shape), v=cache[1].view(s["v"].shape))
    return out
