"""Tree attention with results in bf16, whose kernels hold the softmax's terms in bf16 (those of fp32 results are others): masks, scales, what is not finite,
lengths far apart, a graph and offsets beyond 32 bits."""
import math

import numpy as np
import pytest
import torch

from oracle import draft_trees as dt
from test_gpu_cache import Pool, _np, _tokens
from test_gpu_draft_tree_edges import KINDS
from test_gpu_draft_trees import _attend, _attend_refs, _within, int32, random_trees

pytestmark = pytest.mark.gpu
BF16 = torch.bfloat16


@pytest.mark.parametrize("d,T,Hq,Hk", KINDS)
@pytest.mark.parametrize("window,sinks", [(0, 0), (40, 4), (3, 2)])
def test_lengths_masks_and_pages_that_are_not_there(d, T, Hq, Hk, window, sinks):
    lens = [0, 15, 16, 33, 700, 3000, -1, 64]
    N = len(lens)
    pool = Pool(N, Hk, d, 16, 3000 + T, d + T, nan_behind=[max(0, n) + T for n in lens])
    pool.table[4, 9] = -1
    q, parents = _tokens(N, T, Hq, d, 3), random_trees(N, T, 4, T, max(1, T // 2), roots=True)
    got = _attend(pool, q, lens, parents, window, sinks, BF16)
    _within(got, *_attend_refs(pool, q, lens, parents, window, sinks), BF16)
    empty = torch.tensor([[not x for x in dt.lines(p)] for p in parents])
    assert not bool(got.cpu()[empty].any()) and not bool(got[6].any())


@pytest.mark.parametrize("d,T,Hq,Hk", KINDS)
def test_values_and_keys_that_are_no_numbers(d, T, Hq, Hk):
    held = 500
    pool = Pool(1, Hk, d, 16, held + T, d + T)
    q, parents = _tokens(1, T, Hq, d, 3), random_trees(1, T, 4, T, roots=True)
    ref, bound = _attend_refs(pool, q, [held], parents)
    for slot in (held - 2, held, held + T - 1):
        page, at = pool.table[0, slot // 16], slot % 16
        seen = dt.tree_mask(parents[0], held, 0, 0)[:, slot]
        was = pool.v[page, 0, at, 7]
        pool.v[page, 0, at, 7] = 0x7F
        got = _attend(pool, q, [held], parents, out_dtype=BF16)
        pool.v[page, 0, at, 7] = was
        hit = np.zeros(ref.shape, bool)
        hit[0, seen, :Hq // Hk, 7] = True
        assert np.array_equal(np.isnan(_np(got)), hit)
        _within(torch.tensor(np.where(hit, ref, _np(got))), ref, bound, BF16)
        was = pool.k[page, 0, at, 9]
        pool.k[page, 0, at, 9] = 0xFF
        got = _attend(pool, q, [held], parents, out_dtype=BF16)
        pool.k[page, 0, at, 9] = was
        hit = np.zeros(ref.shape, bool)
        hit[0, seen, :Hq // Hk] = True
        assert np.array_equal(np.isnan(_np(got)), hit)
        _within(torch.tensor(np.where(hit, ref, _np(got))), ref, bound, BF16)


@pytest.mark.parametrize("d,T,Hq,Hk", KINDS)
def test_scales_of_any_size(d, T, Hq, Hk):
    held = [500, 40]
    pool = Pool(2, Hk, d, 16, 500 + T, d + T)
    g = np.random.default_rng(3)
    ks, vs = pool.ks.copy(), pool.vs.copy()
    q, parents = _tokens(2, T, Hq, d, 3), random_trees(2, T, 4, 5)
    for kind in range(6):
        pool.ks, pool.vs = ks.copy(), vs.copy()
        if kind == 0:
            pool.ks = np.float32(ks * g.uniform(0.5, 2, ks.shape))
        elif kind == 1:
            pool.vs = np.float32(vs * g.uniform(-2, 2, vs.shape))
        elif kind == 2:
            pool.vs = np.float32(vs * 2.0 ** 100)
        elif kind == 3:
            pool.vs = np.float32(vs * 2.0 ** -70)
        elif kind == 4:
            pool.vs = np.float32(np.where(g.random(vs.shape) < 0.5, 2.0 ** 117, 2.0 ** 90))
        else:
            pool.ks[::2], pool.vs[1::3] = 0, 0
        got = _attend(pool, q, held, parents, out_dtype=BF16)
        assert bool(torch.isfinite(got).all())
        _within(got, *_attend_refs(pool, q, held, parents), BF16)


@pytest.mark.parametrize("d,T,Hq,Hk", KINDS)
def test_rows_that_see_nothing_and_other_sequences_pages(d, T, Hq, Hk):
    pool = Pool(2, Hk, d, 16, 700 + T, 9)
    q, parents = _tokens(2, T, Hq, d, 3), random_trees(2, T, 3, 1)
    pool.table[0, :] = -1
    for p in pool.table[1, :600 // 16 - 3]:                  # (behind every row's window)
        pool.k[p], pool.v[p] = 0x7F, 0xFF
        pool.ks[p] = pool.vs[p] = math.nan
    got = _attend(pool, q, [600, 600], parents, 20, 0, BF16)
    assert not bool(got[0].any())
    _within(got, *_attend_refs(pool, q, [600, 600], parents, 20, 0), BF16)


@pytest.mark.parametrize("d,T,Hq", [(128, 20, 8), (64, 40, 8), (128, 35, 16)])
def test_one_long_sequence_of_a_batch(d, T, Hq):
    N, Hk, page, long = 64, 8, 128, 17000
    pool = Pool(N, Hk, d, page, 256, T)
    g = np.random.default_rng(T)
    held = g.integers(0, 256 - T, N)
    held[[3, 40]] = -1, 0
    wide = np.full((N, (long + T + page - 1) // page), -1, pool.table.dtype)
    wide[:, :pool.table.shape[1]] = pool.table
    wide[17] = g.integers(0, pool.P, wide.shape[1])          # (read only, so the pages may be others' too)
    held[17] = long
    pool.table = wide
    q, parents = _tokens(N, T, Hq, d, 3), random_trees(N, T, 4, T, (T + 1) // 2)
    got = _attend(pool, q, held, parents, out_dtype=BF16, max_kv_len=long + T)
    _within(got, *_attend_refs(pool, q, held, parents), BF16)
    assert torch.equal(got, _attend(pool, q, held, parents, out_dtype=BF16))


@pytest.mark.parametrize("d", [64, 128])
def test_both_results_in_a_graph(d):
    """The same call with either result, captured and replayed: two kernels, each with its own parts."""
    import paper_2510_26692_amd as kda
    T = 64
    pool = Pool(2, 2, d, 32, 2000, 3)
    q, parents, lens, cache = _tokens(2, T, 8, d, 4).cuda(), int32(random_trees(2, T, 4, 1)), int32([1900, 77]), pool.device()
    call = lambda out_dtype: kda.kda_cache_tree_attn(q, *cache, lens, parents, out_dtype=out_dtype)
    call(BF16)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        o = [call(BF16), call(torch.float32)]
    for seed in (5, 6, 7):
        parents.copy_(int32(random_trees(2, T, 4, seed)))
        q.copy_(_tokens(2, T, 8, d, seed).cuda())
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(o[0], call(BF16)) and torch.equal(o[1], call(torch.float32))


def test_offsets_beyond_32_bits():
    import paper_2510_26692_amd as kda
    Hk, page, d, T, held = 8, 128, 128, 9, 300
    P = (1 << 32) // (Hk * page * d) + 40
    small = Pool(1, Hk, d, page, held + T, 3)
    codes = [torch.zeros(P, Hk, page, d, dtype=torch.uint8, device="cuda") for _ in range(2)]
    scales = [torch.ones(P, Hk, device="cuda") for _ in range(2)]
    at = P - small.P
    for big, part in zip(codes + scales, (small.k, small.v, small.ks, small.vs)):
        big[at:] = torch.from_numpy(part).cuda()
    f8 = [x.view(torch.float8_e4m3fn) for x in codes]
    table = torch.from_numpy(small.table + at).to(torch.int32).cuda()
    for Hq in (16, 32):                                      # few rows, and tiles
        q, parents = _tokens(1, T, Hq, d, 3), random_trees(1, T, 3, 1)
        got = kda.kda_cache_tree_attn(q.cuda(), *f8, *scales, table, int32([held]), int32(parents), out_dtype=BF16)
        _within(got, *_attend_refs(small, q, [held], parents), BF16)
