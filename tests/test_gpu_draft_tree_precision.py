"""Tree attention with results in fp32: the softmax's terms go to the product with the values to 2^-16 of themselves.

A term exp(x_j - m) is off by 2^-16, by the rounding of its logit, (d + 16) 2^-24 scale |q| . |k_j| (a sum of d products, the scale and the difference from the
maximum), and by 2^-18 for the exponential and the factors that join parts with other maxima (ten of 2^-22 at most); sums of n terms by n 2^-24 of what they add
up.  That is in the numerators, which with p_j normalised weigh |v_j|, and once more in the sum that divides them."""
import numpy as np
import pytest
import torch

from oracle import draft_trees as dt
from test_gpu_cache import Pool, _np, _tokens
from test_gpu_draft_trees import _attend, _attend_refs, _cached, _within, random_trees

pytestmark = pytest.mark.gpu

# few rows a key head (no tiles), 64 and 128 rows a workgroup, several workgroups
KINDS = [(64, 4, 4, 2), (64, 16, 4, 2), (64, 40, 4, 1), (64, 64, 8, 2), (128, 8, 2, 1), (128, 20, 2, 2), (128, 40, 8, 2), (128, 64, 4, 1)]


def _off(pool, q, lens, parents, window, sinks, scale, got):
    """How far rows are off, over what they may be."""
    o, bound = _attend_refs(pool, q, lens, parents, window, sinks, scale)
    N, T, Hq, d = q.shape
    tol = np.zeros(o.shape)
    for n, held in enumerate(lens):
        k = np.abs(_cached(pool, "k", n, held + T)[0])
        size = max(float((np.abs(_np(q[n, :, h])) @ k[:, h // (Hq // k.shape[1])].T).max()) for h in range(Hq))
        tol[n] = 2 * bound[n] * (2.0 ** -16 + 2.0 ** -18 + (d + 16) * 2.0 ** -24 * scale * size + (held + T) * 2.0 ** -24) + 1e-30
    return np.abs(_np(got) - o) / tol


@pytest.mark.parametrize("d,T,Hq,Hk", KINDS)
@pytest.mark.parametrize("window,sinks", [(0, 0), (40, 4)])
def test_results_in_fp32(d, T, Hq, Hk, window, sinks):
    lens, scale = [0, 1, 30, 200, 430], 2.0 ** -6
    N = len(lens)
    pool = Pool(N, Hk, d, 16, max(lens) + T, d + T, nan_behind=[n + T for n in lens])
    q, parents = _tokens(N, T, Hq, d, 3), random_trees(N, T, 3, T, max(1, T // 2), roots=True)
    got = _attend(pool, q, lens, parents, window, sinks, scale=scale)
    off = _off(pool, q, lens, parents, window, sinks, scale, got)
    assert (off <= 1).all(), off.max()
    # scales that the codes cannot take on their way
    g = np.random.default_rng(3)
    pool.ks, pool.vs = np.float32(pool.ks * g.uniform(0.5, 1, pool.ks.shape)), np.float32(pool.vs * g.uniform(-2, 2, pool.vs.shape))
    off = _off(pool, q, lens, parents, window, sinks, scale, _attend(pool, q, lens, parents, window, sinks, scale=scale))
    assert (off <= 1).all(), off.max()
    # in bf16 the same call rounds its terms and its result to bf16
    _within(_attend(pool, q, lens, parents, window, sinks, torch.bfloat16, scale=scale), *_attend_refs(pool, q, lens, parents, window, sinks, scale), torch.bfloat16)


@pytest.mark.parametrize("d,T,Hq,Hk", KINDS)
def test_results_in_fp32_beside_values_that_are_no_numbers(d, T, Hq, Hk):
    """The walk that is repeated with care holds the terms as the other does."""
    held, scale = 120, 2.0 ** -6
    pool = Pool(1, Hk, d, 16, held + T, d + T)
    q, parents = _tokens(1, T, Hq, d, 3), random_trees(1, T, 3, T, roots=True)
    slot = held + T // 2
    page, at = pool.table[0, slot // 16], slot % 16
    want = _off(pool, q, [held], parents, 0, 0, scale, _attend(pool, q, [held], parents, scale=scale))
    assert (want <= 1).all()
    pool.v[page, :, at, 5] = 0x7F
    got = _attend(pool, q, [held], parents, scale=scale)
    pool.v[page, :, at, 5] = 0
    seen = dt.tree_mask(parents[0], held, 0, 0)[:, slot]
    hit = np.zeros(got.shape[1:], bool)
    hit[seen, :, 5] = True
    assert np.array_equal(np.isnan(_np(got[0])), hit)
    off = _off(pool, q, [held], parents, 0, 0, scale, torch.nan_to_num(got))[0]
    assert (off[~hit] <= 1).all(), off[~hit].max()
