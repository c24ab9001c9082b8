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
