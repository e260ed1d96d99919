"""Rows of the cache that no query sees: what they hold changes nothing, not a bit and not the way that a result is worked out."""
import numpy as np
import pytest
import torch

from test_gpu_cache_ops import Setup, _bf16
from test_gpu_new_tokens import _check_rows, _chunk, _places, _window

pytestmark = pytest.mark.gpu


def _spoil(s, buf, tokens):
    """NaN in rows `tokens` of every sequence and KV head."""
    for b in range(s.batch):
        for h in range(s.hkv):
            for tok in tokens:
                if s.fmt:
                    s.set_row(buf, b, h, tok, scales=np.full(s.d // 32, 255, dtype=np.uint8))
                else:
                    s.set_row(buf, b, h, tok, values=np.full(s.d, np.nan))


# (hq, hkv, d, page, n_new, first, sink, window): hidden from all queries are sink .. first - window
HIDDEN = [(8, 2, 128, 0, 200, 500, 5, 150), (8, 2, 64, 16, 200, 500, 70, 150), (2, 2, 128, 16, 130, 400, 0, 77), (8, 1, 64, 0, 60, 600, 64, 64),
          (8, 2, 128, 8, 150, 300, 130, 140), (4, 2, 128, 0, 3, 500, 5, 150)]


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("fmt", [0, 1, 2])
@pytest.mark.parametrize("case", HIDDEN, ids=str)
def test_chunk(case, fmt, bf16):
    hq, hkv, d, page, n_new, first, sink, window = case
    s = Setup(2, hq, hkv, d, first + n_new + 20, page, fmt, None, seed=n_new)
    q = _bf16(s.rng.normal(size=(2, n_new, hq, d)))
    clean = _chunk(s, q, [first, first], None, sink, window, bf16)
    _check_rows(s, q, _places(s, [first] * 2, None, n_new), sink, window, *clean, bf16)
    hidden = [*range(sink, first - window + 1), *range(first + n_new, s.n_max)]
    _spoil(s, s.v, hidden)
    _spoil(s, s.k, hidden)
    for a, b in zip(clean, _chunk(s, q, [first, first], None, sink, window, bf16)):
        assert torch.equal(a, b)


@pytest.mark.parametrize("fmt", [0, 1, 2])
@pytest.mark.parametrize("sink,window", [(5, 150), (0, 1500), (70, 900)])
def test_window_decode(sink, window, fmt):
    s = Setup(2, 8, 2, 128, 1900, 16, fmt, None, seed=window)
    q = _bf16(s.rng.normal(size=(2, 1, 8, 128)))
    clean = _window(s, q, [1880, 1880], sink, window)
    hidden = [*range(sink, 1880 - window), *range(1880, 1900)]
    _spoil(s, s.v, hidden)
    _spoil(s, s.k, hidden)
    for a, b in zip(clean, _window(s, q, [1880, 1880], sink, window)):
        assert torch.equal(a, b)
