"""Attention over the paged cache with scales next to the largest and smallest that fp32 holds, and with scales of pages that no query sees:
results are finite and right wherever the definition's are.

Tolerances as in test_gpu_cache.py: terms rounded to bf16, a result once more."""
import math

import numpy as np
import pytest
import torch

from oracle import softmax_attention as sa
from test_gpu_cache import HALF, Pool, TERMS, _append_both, _attend, _freqs, _np, _tokens

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("page,at,window,sinks", [(16, 300, 100, 0), (16, 290, 100, 4), (16, 310, 100, 0), (32, 300, 60, 4), (64, 310, 40, 0)])
@pytest.mark.parametrize("d,Hq", [(128, 2), (64, 40)])
def test_attend_scales_of_pages_that_nobody_sees(page, at, window, sinks, d, Hq):
    """A page wholly before the window and behind the sinks may have been given to another sequence, and its scale be anything."""
    for Tq in (1, 3):
        length = at + window + Tq - 1                        # the first query's window begins at `at` or behind it
        pool = Pool(1, 1, d, page, length + 20, 5)
        q = _tokens(1, Tq, Hq, d, 6)
        clean = _attend(pool, q, [length], window, sinks)
        first = length - Tq - window + 1                     # the first key that a query sees
        hidden = [p for p in range(1, first // page) if p * page >= sinks]
        assert hidden
        for value in (math.nan, math.inf, 3e38):
            for x in (pool.ks, pool.vs):
                x[pool.table[0, hidden]] = value
            assert torch.equal(_attend(pool, q, [length], window, sinks), clean), (Tq, value)


def _check_relative(pool, q, lens, window=0, sinks=0, rows=None, **kw):
    """The attention over the cache without a floor under its tolerance: a result may be of any size."""
    o = _attend(pool, q, lens, window, sinks, **kw)
    ref, bound = sa.cache_attention(_np(q), pool.k, pool.v, pool.ks, pool.vs, pool.table, lens, window, sinks)
    got = _np(o)
    assert np.isfinite(got).all()
    off = np.abs(got - ref) - (TERMS * bound * (1 + HALF) + (HALF if kw.get("out_dtype") == torch.bfloat16 else 2.0 ** -20) * np.abs(ref))
    assert (off <= 0).all(), "%g beyond its bound at %s" % (off.max(), np.unravel_index(off.argmax(), off.shape))
    return o


@pytest.mark.parametrize("out_dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("low,high", [(119, 119), (60, 119), (20, 70), (-20, 119), (-40, 64), (-45, -39), (-100, -60), (-115, -110)])
@pytest.mark.parametrize("d,Tq,Hq,page,lens", [(128, 2, 4, 64, [3000, 700, 17, 64]), (64, 8, 24, 16, [900, 40, 300, 9]), (64, 1, 2, 128, [33000, 5000, 300, 1])])
def test_attend_values_of_any_size(d, Tq, Hq, page, lens, low, high, out_dtype):
    """Scales of values from 2^-115 to 2^119, each page and head its own."""
    pool = Pool(4, 1, d, page, max(lens) + 20, 5, nan_behind=lens)
    g = np.random.default_rng(low + 200)
    pool.vs = np.float32(2.0) ** g.integers(low, high + 1, pool.vs.shape).astype(np.float32)
    pool.v &= 0xFF if low < 100 else 0x7F                    # (of one sign: the sums grow with every key)
    q = (_tokens(4, Tq, Hq, d, 5).float() * 0.1).to(torch.bfloat16)
    _check_relative(pool, q, lens, out_dtype=out_dtype)
    if high - low <= 10:
        for window, sinks in ((200, 4), (20, 0)):
            _check_relative(pool, q, lens, window, sinks, out_dtype=out_dtype)


def test_attend_ordinary_scales_keep_their_bits_beside_large_ones():
    """A head's results do not depend on another head's scales, nor on those of pages that are not its own."""
    lens = [3000, 100]
    pool = Pool(2, 2, 128, 64, 3040, 5)
    q = _tokens(2, 4, 8, 128, 6)
    clean = _attend(pool, q, lens)
    pool.vs[:, 1] *= np.float32(2.0 ** 120)
    got = _check_relative(pool, q, lens)
    assert torch.equal(got[:, :, :4], clean[:, :, :4])


@pytest.mark.parametrize("exponent", [124, 100, -90])
def test_attend_over_an_append_of_large_and_small_values(exponent):
    """What the append stores of the largest and smallest values is attended over as it stands."""
    pool = Pool(3, 2, 128, 32, 200, 6)
    lens, T = [0, 0, 0], 150
    k, v = _tokens(3, T, 2, 128, 7), (_tokens(3, T, 2, 128, 8).float().clamp(-4, 4) * 2.0 ** exponent).to(torch.bfloat16)
    _append_both(pool, k, v, lens, freqs=_freqs(64))
    _check_relative(pool, (_tokens(3, 4, 4, 128, 9).float() * 0.2).to(torch.bfloat16), [T] * 3)


def test_attend_keys_of_any_size():
    """Scales of keys up to 2^100 and down to 2^-90, with queries as small or large: the logits are ordinary."""
    for exponent in (100, -90):
        pool = Pool(2, 2, 64, 32, 700, 8)
        pool.ks *= np.float32(2.0 ** exponent)
        _check_relative(pool, (_tokens(2, 2, 4, 64, 9).float() * 2.0 ** -exponent).to(torch.bfloat16), [700, 33])
