"""Reference in 64 bits for the cache operators of libvatt: formats, rotary positions, block summaries, block selection and
attention over blocks.  Written from the definitions in include/vatt.h with NumPy, one sequence and one KV head at a time; it
shares no code with the library or its bindings.
"""
from __future__ import annotations

import math

import numpy as np

BF16, E4M3, E2M1 = 0, 1, 2
LARGEST = 1.5 * 2.0 ** 127


# ---- numbers -------------------------------------------------------------------------------------------------------------

def bf16_round(x):
    """fp64 -> the nearest bf16 value (ties to even), as fp64.  Inf and NaN stay."""
    x = np.asarray(x, dtype=np.float64)
    out = x.copy()
    ok = np.isfinite(x) & (x != 0)
    e = np.maximum(np.frexp(x[ok])[1] - 8, -133)  # unit of the last of 8 significant bits, subnormals at 2^-133
    r = np.ldexp(np.rint(np.ldexp(x[ok], -e)), e)
    out[ok] = np.where(np.abs(r) >= 2.0 ** 128, np.copysign(np.inf, r), r)
    return out


def code_values(fmt):
    """The value of every code of a quantised format, from its fields."""
    vals = []
    for code in range(256 if fmt == E4M3 else 16):
        bits, bias = (3, 7) if fmt == E4M3 else (1, 1)
        top = 7 if fmt == E4M3 else 3
        sign = -1.0 if code >> top else 1.0
        e, m = (code & ((1 << top) - 1)) >> bits, code & ((1 << bits) - 1)
        v = m * 2.0 ** (1 - bias - bits) if e == 0 else (1 + m / 2.0 ** bits) * 2.0 ** (e - bias)
        if fmt == E4M3 and code & 0x7f == 0x7f:
            v = math.nan
        vals.append(sign * v)
    return np.array(vals)


def encode(x, fmt):
    """fp64 row (d values) -> (codes, one per value; scale bytes, one per 32)."""
    vals = code_values(fmt)
    half = len(vals) // 2
    mags = vals[:half][np.isfinite(vals[:half])]
    codes, scales = [], []
    for group in np.asarray(x, dtype=np.float64).reshape(-1, 32):
        if not np.isfinite(group).all():
            codes += [0] * 32
            scales.append(255)
            continue
        g = np.clip(group, -LARGEST, LARGEST)
        top, e = np.abs(g).max(), -127
        while top > mags[-1] * 2.0 ** e:
            e += 1
        scales.append(e + 127)
        for v in g:
            y = abs(v) * 2.0 ** -e
            i = int(np.searchsorted(mags, y))
            if i > 0 and (i == len(mags) or y < mags[i]):  # between mags[i - 1] and mags[i]
                below, above = y - mags[i - 1], mags[i] - y
                i = i - 1 if below < above or (below == above and (i - 1) % 2 == 0) else i
            codes.append(i + (half if np.signbit(v) else 0))
    return np.array(codes), np.array(scales)


def decode(codes, scales, fmt):
    """What codes and scale bytes stand for."""
    v = code_values(fmt)[np.asarray(codes)].reshape(-1, 32)
    s = np.where(np.asarray(scales) == 255, math.nan, 2.0 ** (np.asarray(scales, dtype=np.float64) - 127))
    return (v * s[:, None]).reshape(-1)


def unpack(raw, fmt):
    """Bytes of a row -> codes."""
    raw = np.asarray(raw, dtype=np.uint8)
    return raw.astype(np.int64) if fmt == E4M3 else np.stack([raw & 15, raw >> 4], -1).reshape(-1).astype(np.int64)


def pack(codes, fmt):
    codes = np.asarray(codes, dtype=np.uint8)
    return codes if fmt == E4M3 else codes[0::2] | (codes[1::2] << 4)


def stored(x, fmt):
    """What the cache holds of an fp64 row."""
    return bf16_round(x) if fmt == BF16 else decode(*encode(x, fmt), fmt)


# ---- rotary positions ------------------------------------------------------------------------------------------------------

def frequencies(r, head_dim):
    """(angle per position of every pair, factor) for a dict with the fields of vatt_rotary."""
    dim = r.get("rotary_dim", 0) or head_dim
    scaling, theta = r.get("scaling", 0), r["theta"]
    f = [theta ** (-2.0 * i / dim) for i in range(dim // 2)]
    factor = r.get("attention", 0.0) or (0.1 * math.log(r["factor"]) + 1.0 if scaling == 3 else 1.0)
    if scaling == 1:
        f = [x / r["factor"] for x in f]
    if scaling == 2:
        keep = [min(max((r["original_len"] * x / (2 * math.pi) - r["low"]) / (r["high"] - r["low"]), 0.0), 1.0) for x in f]
        f = [x * k + x / r["factor"] * (1 - k) for x, k in zip(f, keep)]
    if scaling == 3:
        def pair(turns):
            return dim * math.log(r["original_len"] / (2 * math.pi * turns)) / (2 * math.log(theta))
        lo, hi = max(math.floor(pair(r["high"])), 0), min(math.ceil(pair(r["low"])), dim - 1)
        keep = [1 - min(max((i - lo) / max(hi - lo, 0.001), 0.0), 1.0) for i in range(dim // 2)]
        f = [x * k + x / r["factor"] * (1 - k) for x, k in zip(f, keep)]
    return f, factor


def rotate(x, position, r):
    """A row of head_dim values, rotated, in 64 bits."""
    x = np.array(x, dtype=np.float64)
    f, factor = frequencies(r, len(x))
    half = len(f)
    y = x.copy()
    for i in range(half):
        a, b = (2 * i, 2 * i + 1) if r.get("layout", 0) == 1 else (i, i + half)
        c, s = factor * math.cos(position * f[i]), factor * math.sin(position * f[i])
        y[a], y[b] = x[a] * c - x[b] * s, x[b] * c + x[a] * s
    return y


# ---- blocks ----------------------------------------------------------------------------------------------------------------

def summary(rows):
    """(largest, smallest) of every column; NaN where a row has one."""
    return np.max(rows, axis=0), np.min(rows, axis=0)


def parts(n, params, c):
    """(lo, hi, total, take): blocks [0, lo) and [hi, total) are always taken, `take` of those between are chosen."""
    total = (n + c - 1) // c
    lo = (min(params["sink"], n) + c - 1) // c
    hi = max(n - max(params["window"], 1), 0) // c
    if lo >= hi:
        return total, total, total, 0
    k = params["topk_abs"] if params["topk_abs"] > 0 else int(math.floor(float(np.float32(params["topk_frac"])) * n))
    return lo, hi, total, min(k // c, hi - lo)


def bound(q, top, low):
    """Upper bounds of <q, K[i]> for blocks [.., d], as if in 64 bits and rounded to 32; q [group, d]; the group's largest."""
    best = None
    for row in np.asarray(q, dtype=np.float64):
        with np.errstate(invalid="ignore", over="ignore"):
            s = (row * np.where(row < 0, low, top)).sum(-1).astype(np.float32)
        best = s if best is None else np.maximum(best, s)  # (NaN stays)
    return best


def select(scores, n, params, c):
    """(blocks taken, ascending; the chosen ones among them) from the bounds of all blocks."""
    lo, hi, total, take = parts(n, params, c)
    mid = list(range(lo, hi))
    key = [(-math.inf if math.isnan(scores[j]) else -float(scores[j]) if scores[j] == scores[j] else 0.0,
            0 if math.isnan(scores[j]) else 1, j) for j in mid]
    chosen = sorted(j for _, _, j in sorted(key)[:take])
    return list(range(lo)) + chosen + list(range(hi, total)), chosen


def tokens_of(blocks, n, c):
    """Tokens below n of listed blocks, in list order; entries that are no block of the sequence are left out."""
    out = []
    for j in blocks:
        if 0 <= j * c < n:
            out += range(j * c, min(j * c + c, n))
    return np.array(out, dtype=np.int64)


def attend(q, k, v, scale):
    """softmax(scale q K^T) V and ln of the sum for one query row over the given rows; (0, -Inf) without any."""
    if len(k) == 0:
        return np.zeros(len(q)), -math.inf
    with np.errstate(invalid="ignore", over="ignore"):
        s = scale * (np.asarray(k, dtype=np.float64) @ np.asarray(q, dtype=np.float64))
        m = s.max()
        if m == -math.inf:
            return np.full(len(q), math.nan), -math.inf
        p = np.exp(s - m)
        return (p[:, None] * v).sum(0) / p.sum(), m + math.log(p.sum()) if not math.isnan(p.sum()) else math.nan


# ---- new tokens ------------------------------------------------------------------------------------------------------------

def visible(p, sink, window):
    """Tokens that a query at position p sees: all up to its own, or (window > 0) the first `sink` and the last `window` of them."""
    i = np.arange(p + 1)
    return i if window == 0 else i[(i < sink) | (i > p - window)]


def new_tokens(first, want, n_new, n_max):
    """How many of a sequence's new tokens count: none where the first one's position is outside the cache, none behind its end."""
    if first < 0 or first >= n_max:
        return 0
    return min(max(0, min(want, n_new)), n_max - first)
