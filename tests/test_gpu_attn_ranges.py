"""Softmax attention of values next to the largest and smallest that fp32 holds: results are finite and right wherever the definition's are.

Tolerances as in test_gpu_window_attn.py: terms rounded to bf16, a result once more."""
import math

import numpy as np
import pytest
import torch

from oracle import softmax_attention as sa
from test_gpu_window_attn import _check_bwd, _check_fwd, _grads, _make, _np

pytestmark = pytest.mark.gpu


def _large(x, head, exponent):
    """v of one key head: up to 2^(exponent + 2), all of one sign, so that sums grow with every key."""
    x["v"][:, :, head] = (x["v"][:, :, head].float().abs().clamp(max=4) * 2.0 ** exponent).to(torch.bfloat16)
    return x


@pytest.mark.parametrize("out_dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("B,T,Hq,Hk,d,window,sinks,q_std", [
    (1, 500, 4, 2, 64, 0, 0, 0.1), (2, 500, 4, 2, 128, 0, 0, 0.1), (1, 700, 4, 2, 128, 90, 4, 1.5), (2, 333, 2, 2, 64, 40, 0, 0.1), (48, 261, 12, 3, 128, 70, 5, 0.1)])
def test_forward_of_large_values(B, T, Hq, Hk, d, window, sinks, q_std, out_dtype):
    import paper_2510_26692_amd as kda
    x = _make(B, T, Hq, Hk, d, T, q_std)
    call = lambda: kda.kda_window_attn_fwd(*(x[n].cuda() for n in "qkv"), window=window, sinks=sinks, out_dtype=out_dtype)
    clean = call()
    _large(x, 1, 125)
    o, lse = call()
    _check_fwd(x, o, lse, sa.attention(*(_np(x[n]) for n in "qkv"), window, sinks), out_dtype)
    others = [h for h in range(Hq) if h // (Hq // Hk) != 1]
    assert torch.equal(o[:, :, others], clean[0][:, :, others]) and torch.equal(lse, clean[1])


@pytest.mark.parametrize("d", [64, 128])
def test_large_values_beside_one_that_is_not_finite(d):
    import paper_2510_26692_amd as kda
    T, window, sinks = 420, 50, 3
    x = _large(_make(1, T, 2, 2, d, 3, 0.1), 1, 125)
    x["v"][0, 200, 1, 7] = math.inf
    o, _ = kda.kda_window_attn_fwd(*(x[n].cuda() for n in "qkv"), window=window, sinks=sinks)
    sees = sa.visible(np.arange(T), [200], window, sinks)[:, 0]
    assert torch.equal(~torch.isfinite(o).all(-1).cpu()[0, :, 1], torch.from_numpy(sees)) and bool(torch.isfinite(o[:, :, 0]).all())
    y = {n: t.clone() for n, t in x.items()}
    y["v"][0, 200, 1, 7] = 0
    ref = sa.attention(*(_np(y[n]) for n in "qkv"), window, sinks)
    _check_fwd(y, o[:, ~sees], None, {n: t[:, ~sees] for n, t in ref.items() if n != "lse"}, torch.float32)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("window,sinks", [(0, 0), (90, 4)])
def test_gradients_with_large_values(d, window, sinks):
    """Gradients of o as small as v is large: those of q and k are ordinary numbers."""
    x = _large(_make(1, 400, 4, 2, d, 9, 0.5), 1, 124)
    x["do"][:, :, 2:] = (x["do"][:, :, 2:].float() * 2.0 ** -124).to(torch.bfloat16)
    _check_bwd(x, _grads(x, window, sinks)[2], window, sinks)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("window,sinks", [(0, 0), (60, 4)])
def test_a_key_of_infinities_is_unseen_by_queries_that_point_away_from_it(d, window, sinks):
    """Logits of minus infinity are terms of zero; those of plus infinity make their rows NaN."""
    import paper_2510_26692_amd as kda
    T = 300
    x = _make(1, T, 2, 1, d, 13)
    x["k"][0, :, 0, 5] = 0                                    # (the channel is that key's alone)
    x["k"][0, 100, 0, 5] = math.inf
    away = torch.arange(T) % 3 != 0
    x["q"][0, :, :, 5] = torch.where(away[:, None], -1.0, 1.0).to(torch.bfloat16)
    o, lse = kda.kda_window_attn_fwd(*(x[n].cuda() for n in "qkv"), window=window, sinks=sinks)
    hit = torch.from_numpy(sa.visible(np.arange(T), [100], window, sinks)[:, 0]) & ~away
    assert bool(hit.any()) and bool(torch.isnan(o[0, hit]).all()) and bool(torch.isnan(lse[0, :, hit]).all())
    x["k"][0, 100, 0, 5] = 2.0 ** 15                         # (a term of e^-2000 and less, next to none)
    ref = sa.attention(*(_np(x[n]) for n in "qkv"), window, sinks)
    _check_fwd(x, o[:, ~hit], lse[:, :, ~hit], {n: (t[:, :, ~hit] if n == "lse" else t[:, ~hit]) for n, t in ref.items()}, torch.float32)
