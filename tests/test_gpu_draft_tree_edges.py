"""Draft trees and shared pages at the edges: what is not finite and whom it reaches, offsets beyond 32 bits, the native and the general way of
marshalling, the largest trees in a graph, and answers that are the same every time."""
import math

import numpy as np
import pytest
import torch

from oracle import draft_trees as dt
from oracle import softmax_attention as sa
from test_gpu_cache import Pool, _np, _tokens
from test_gpu_draft_trees import _attend, _attend_refs, _check_steps, _inputs, _within, int32, random_trees

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("T,d,dtype", [(16, 128, torch.bfloat16), (40, 64, torch.float32), (64, 128, torch.float32), (64, 128, torch.bfloat16)])
@pytest.mark.parametrize("what", ["q", "k", "v", "log_alpha", "beta"])
@pytest.mark.parametrize("value", [math.nan, math.inf])
def test_what_is_not_finite_reaches_a_token_and_its_descendants(T, d, dtype, what, value):
    """A drafted token that is not finite makes NaN of itself and of what descends from it (a query: of itself; one channel of v: of that
    channel), and leaves every other row as it is without that token."""
    import paper_2510_26692_amd as kda
    x = dict(zip(("q", "k", "v", "log_alpha", "beta"), _inputs(1, T, 2, d, dtype, T)))
    S = (torch.randn(1, 2, d, d, generator=torch.Generator().manual_seed(2)) * 0.3).cuda()
    parents = random_trees(1, T, 3, T)
    line = dt.lines(parents[0])
    bad = next(t for t in range(T) if 1 < sum(t in x for x in line) < T - 2)
    run = lambda: kda.kda_tree_steps(*(y.cuda() for y in x.values()), S, int32(parents), scale=0.1)
    want = run()
    if what == "beta":
        x[what][0, bad, 1] = value
    else:
        x[what][0, bad, 1, 5] = value
    got = run()
    hit = torch.zeros(T, dtype=torch.bool)
    hit[[t for t in range(T) if t == bad or (what != "q" and bad in line[t])]] = True
    odd = torch.zeros(1, T, 2, d, dtype=torch.bool)
    if what == "v":
        odd[0, hit, 1, 5] = True
    else:
        odd[0, hit, 1] = True
    if what == "log_alpha" and value == math.inf:
        return                                               # (no decay: not a call that the contract knows)
    assert bool(torch.equal(got.cpu()[~odd], want.cpu()[~odd]))
    assert not bool(torch.isfinite(got.cpu()[odd]).any())


def test_a_state_that_is_not_finite_reaches_its_columns():
    import paper_2510_26692_amd as kda
    T, d = 16, 128
    x = [y.cuda() for y in _inputs(2, T, 1, d, torch.bfloat16, 1)]
    S = (torch.randn(2, 1, d, d, generator=torch.Generator().manual_seed(2)) * 0.3).cuda()
    parents = random_trees(2, T, 3, 5)
    parents[0, 9:] = -2
    want = kda.kda_tree_steps(*x, S, int32(parents))
    S[0, 0, 3, 40] = math.inf
    got = kda.kda_tree_steps(*x, S, int32(parents))
    odd = torch.zeros(2, T, 1, d, dtype=torch.bool, device="cuda")
    odd[0, :9, 0, 40] = True
    assert bool(torch.equal(got[~odd], want[~odd])) and not bool(torch.isfinite(got[odd]).any())


def test_offsets_beyond_32_bits():
    """A pool of more than 4 GiB of keys: tree attention, accepted tokens and copies in its last pages."""
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
    q, parents = _tokens(1, T, 16, d, 3), random_trees(1, T, 3, 1)
    got = kda.kda_cache_tree_attn(q.cuda(), *f8, *scales, table, int32([held]), int32(parents))
    _within(got, *_attend_refs(small, q, [held], parents), torch.float32)
    kept = [[0, 2, 5, 8, -1]]
    kda.kda_cache_keep(*f8, *scales, table, int32([held]), int32(kept))
    for c, s in ((small.k, small.ks), (small.v, small.vs)):
        dt.keep(c, s, small.table, [held], kept)
    for big, part in zip(codes + scales, (small.k, small.v, small.ks, small.vs)):
        assert np.array_equal(big[at:].cpu().numpy(), part)
    kda.kda_cache_copy_pages(*f8, *scales, int32([[P - 1, 5], [P - 2, P - 30]]))
    for big in codes + scales:
        assert torch.equal(big[5], big[P - 1]) and torch.equal(big[P - 30], big[P - 2])


def test_states_and_rotations_beyond_32_bits():
    import paper_2510_26692_amd as kda
    H, d, T = 4, 128, 5
    P = (1 << 31) // (H * d * d) + 3
    S = torch.zeros(P, H, d, d, device="cuda")
    S[P - 1] = torch.randn(H, d, d, generator=torch.Generator().manual_seed(1)).cuda() * 0.3
    x = _inputs(1, T, H, d, torch.bfloat16, 2)
    parents, idx = random_trees(1, T, 2, 1), torch.tensor([P - 1], dtype=torch.int32)
    o = kda.kda_tree_steps(*(y.cuda() for y in x), S, int32(parents), state_indices=idx.cuda(), scale=0.1)
    last = S[P - 1].cpu()
    _check_steps(*x, last[None], np.zeros(1, int), parents, 0.1, torch.float32, o)
    kda.kda_tree_commit(*(y.cuda() for y in x[1:]), S, int32([[0, -1]]), state_indices=idx.cuda())
    ref = dt.commit(_np(x[1][0]), _np(x[2][0]), np.exp(_np(x[3][0])), _np(x[4][0]), _np(last), [0])
    assert float(np.abs(_np(S[P - 1]) - ref).max()) < 1e-4 and not bool(S[0].any())
    del S
    T = (1 << 31) // (16 * d) + 70
    q = torch.zeros(1, T, 16, d, dtype=torch.bfloat16, device="cuda")
    q[0, -3:] = _tokens(1, 3, 16, d, 1).cuda()[0]
    pos = torch.full((1, T), 77, dtype=torch.int32, device="cuda")
    f = torch.from_numpy(np.float32(10000.0 ** (-np.arange(64) / 64))).cuda()
    out, _ = kda.kda_rotate(q, None, pos, f)
    want, _ = kda.kda_rotate(q[:, -3:].contiguous(), None, pos[:, -3:].contiguous(), f)
    assert torch.equal(out[:, -3:], want) and not bool(out[0, :5].any())


def test_the_native_and_the_general_way_are_the_same(monkeypatch):
    import paper_2510_26692_amd as kda
    from paper_2510_26692_amd import kda as binding
    pool = Pool(3, 2, 128, 16, 300, 9)
    q, k = (_tokens(3, 12, H, 128, H).cuda() for H in (8, 2))
    parents = random_trees(3, 12, 3, 1, 6)
    kept = int32([[0, 2, 5, -1], [1, 3, -1, 0], [-1, 0, 1, 2]])
    x = [y.cuda() for y in _inputs(3, 12, 2, 64, torch.float32, 1)]
    f = torch.from_numpy(np.float32(10000.0 ** (-np.arange(64) / 64))).cuda()
    lens = int32([250, 40, 0])

    def all_calls():
        S = (torch.randn(4, 2, 64, 64, generator=torch.Generator().manual_seed(2)) * 0.3).cuda()
        cache = pool.device()
        idx = int32([3, -1, 0])
        out = list(kda.kda_rotate(q, k, lens[:, None].expand(3, 12).contiguous(), f, axes=[0] * 64, interleaved=True, inverse=True))
        out.append(kda.kda_cache_tree_attn(q, *cache, lens, int32(parents), window=40, sinks=2, scale=0.2, max_kv_len=280, out_dtype=torch.bfloat16))
        out.append(kda.kda_tree_steps(*x, S, int32(parents), state_indices=idx, scale=0.3))
        kda.kda_tree_commit(*x[1:], S, kept, state_indices=idx)
        kda.kda_cache_keep(*cache, lens, kept)
        kda.kda_cache_copy_pages(*cache[:4], int32([[0, 5], [-1, -1], [3, 7]]))
        refs = torch.from_numpy(dt.count(pool.table, pool.P)).cuda()
        table = cache[4].clone()
        kda.kda_pages_fork(table, refs, int32([0, 0, -1]))
        out += kda.kda_pages_reserve(table, lens, lens + 20, refs, 16)
        out.append(kda.kda_pages_compact(table, refs))
        return out + [S, table, refs] + [c.view(torch.uint8) if c.dtype == torch.float8_e4m3fn else c for c in cache]

    assert binding._native is not None
    calls = []
    real = binding._native

    class Counting:
        def __getattr__(self, name):
            def call(*args):
                done = getattr(real, name)(*args)
                calls.append((name, done is not None))
                return done
            return call

    monkeypatch.setattr(binding, "_native", Counting())
    one = all_calls()
    assert [c[0] for c in calls] == ["rotate", "tree_attend", "tree_steps", "tree_commit", "keep", "copy_pages", "fork", "reserve"] and all(c[1] for c in calls)
    monkeypatch.setattr(binding, "_native", None)
    two = all_calls()
    assert all(torch.equal(a, b) for a, b in zip(one, two))


def test_refused_calls_raise_either_way():
    import paper_2510_26692_amd as kda
    q = _tokens(2, 65, 4, 128, 1).cuda()
    pool = Pool(2, 2, 128, 16, 300, 9)
    parents = int32(np.tile(np.arange(-1, 64), (2, 1)))
    with pytest.raises(kda.KdaError, match="64"):
        kda.kda_cache_tree_attn(q, *pool.device(), int32([3, 4]), parents)
    f = torch.ones(64, device="cuda")
    with pytest.raises(kda.KdaError, match="axis"):
        kda.kda_rotate(q, None, int32(np.zeros((2, 65))), f, axes=[0] * 63 + [1])
    with pytest.raises((TypeError, ValueError)):
        kda.kda_rotate(q, None, int32(np.zeros((2, 65))), f, axes=64)
    with pytest.raises(ValueError):
        kda.kda_rotate(q, None, int32(np.zeros((2, 65))), f, axes=[0] * 60)
    with pytest.raises(ValueError):
        kda.kda_rotate(q, None, int32(np.zeros((2, 64))), f)
    x = [y.cuda() for y in _inputs(1, 65, 1, 64, torch.bfloat16, 1)]
    with pytest.raises(kda.KdaError, match="64"):
        kda.kda_tree_steps(*x, torch.zeros(1, 1, 64, 64, device="cuda"), int32([np.arange(-1, 64)]))
    with pytest.raises(ValueError):
        kda.kda_tree_steps(*x, torch.zeros(1, 1, 64, 64, device="cuda"), int32([np.arange(-1, 60)]))
    with pytest.raises(ValueError):
        kda.kda_cache_keep(*pool.device(), int32([3, 4]), int32([1, 2]))


@pytest.mark.parametrize("d", [64, 128])
def test_the_largest_trees_in_a_graph(d):
    """64 tokens, whose workgroups take more LDS than the runtime gives unasked, captured in a process's first call of its size or not, and replayed."""
    import paper_2510_26692_amd as kda
    T = 64
    pool = Pool(2, 2, d, 32, 2000, 3)
    q = _tokens(2, T, 8, d, 4).cuda()
    x = [y.cuda() for y in _inputs(2, T, 3, d, torch.float32, 1)]
    S = (torch.randn(2, 3, d, d, generator=torch.Generator().manual_seed(2)) * 0.3).cuda()
    parents, kept, lens, cache = int32(random_trees(2, T, 4, 1)), int32([list(range(64))] * 2), int32([1900, 77]), pool.device()
    f = torch.ones(d // 2, device="cuda")
    kda.kda_rotate(q, None, parents, f)                      # (the library is loaded, and the stream has worked)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        o = kda.kda_cache_tree_attn(q, *cache, lens, parents)
        o2 = kda.kda_tree_steps(*x, S, parents)
        kda.kda_tree_commit(*x[1:], S, kept)
    for seed in (5, 6, 7):
        parents.copy_(int32(random_trees(2, T, 4, seed)))
        q.copy_(_tokens(2, T, 8, d, seed).cuda())
        before = S.clone()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(o, kda.kda_cache_tree_attn(q, *cache, lens, parents))
        assert torch.equal(o2, kda.kda_tree_steps(*x, before, parents))
        kda.kda_tree_commit(*x[1:], before, kept)
        assert torch.equal(S, before)


def test_answers_are_the_same_every_time_and_whatever_the_batch():
    """A sequence's rows alone and among others (other places, other rounds of workgroups) agree within the attention's rounding, and a call with
    itself bit for bit; more sequences than a round holds, ranked by length."""
    N, T = 70, 24
    pool = Pool(N, 8, 64, 16, 700, 3)
    lens = np.random.default_rng(1).integers(0, 670, N).tolist()
    lens[7], lens[33] = -1, 0
    q, parents = _tokens(N, T, 16, 64, 3), random_trees(N, T, 4, 1, 10)
    got = _attend(pool, q, lens, parents, max_kv_len=64)
    assert torch.equal(got, _attend(pool, q, lens, parents, max_kv_len=64))
    _within(got, *_attend_refs(pool, q, lens, parents), torch.float32)


def test_compaction_of_counts_below_zero_stays_inside():
    """Counts that a caller broke are nobody's promise, but no write leaves the pool."""
    import paper_2510_26692_amd as kda
    refs = int32([1, -3, 0, 2, -1, 0, 1, 1])
    table = int32([[0, 3, 6, 7]])
    moves = kda.kda_pages_compact(table, refs)
    assert table.tolist() == [[0, 3, 1, 2]] and moves.tolist() == [[6, 1], [7, 2], [-1, -1], [-1, -1]] and refs.tolist()[:4] == [1, 1, 1, 2]


@pytest.mark.parametrize("d,T,Hq,Hk", [(64, 8, 8, 2), (64, 32, 2, 2), (64, 33, 2, 2), (128, 16, 2, 2), (128, 17, 2, 2), (128, 4, 8, 2), (64, 3, 8, 1), (128, 5, 5, 1), (64, 1, 64, 1)])
@pytest.mark.parametrize("window,sinks", [(0, 0), (40, 4), (3, 2)])
def test_few_rows_a_key_head(d, T, Hq, Hk, window, sinks):
    """Either side of where a tree's rows go to the kernel without tiles: masks, codes that are no numbers behind the last token, pages that are not
    there, skipped sequences, long ones that are split."""
    lens = [0, 15, 16, 33, 700, 3000, -1, 64]
    N = len(lens)
    pool = Pool(N, Hk, d, 16, 3000 + T, d + T, nan_behind=[max(0, n) + T for n in lens])
    pool.table[4, 9] = -1
    q, parents = _tokens(N, T, Hq, d, 3), random_trees(N, T, 4, T, max(1, T // 2), roots=True)
    for out_dtype in (torch.float32, torch.bfloat16):
        got = _attend(pool, q, lens, parents, window, sinks, out_dtype)
        _within(got, *_attend_refs(pool, q, lens, parents, window, sinks), out_dtype)
    # a value that is not a number, of the context and of the tree
    n, held = 5, 3000
    for slot in (held - 2, held):
        page, at = pool.table[n, slot // 16], slot % 16
        was = pool.v[page, 0, at, 7]
        pool.v[page, 0, at, 7] = 0x7F
        got = np.isnan(_np(_attend(pool, q, lens, parents, window, sinks))[n])
        pool.v[page, 0, at, 7] = was
        want = np.zeros(got.shape, bool)
        want[dt.tree_mask(parents[n], held, window, sinks)[:, slot], :Hq // Hk, 7] = True
        assert np.array_equal(got, want)


KINDS = [(64, 16, 4, 2), (64, 40, 4, 1), (128, 8, 2, 1), (128, 20, 2, 2), (128, 40, 8, 2), (128, 64, 4, 1)]        # few rows, 64 and 128 a workgroup


@pytest.mark.parametrize("d,T,Hq,Hk", KINDS)
def test_scales_of_any_size_whichever_the_kernel(d, T, Hq, Hk):
    """Scales that are no powers of two, that differ from page to page, that are negative, large, small or zero: exact in fp32, and finite where the
    result is."""
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
            pool.vs = np.float32(np.where(g.random(vs.shape) < 0.5, 2.0 ** 118, 2.0 ** 90))
        else:
            pool.ks[::2], pool.vs[1::3] = 0, 0
        got = _attend(pool, q, held, parents)
        assert bool(torch.isfinite(got).all())
        _within(got, *_attend_refs(pool, q, held, parents), torch.float32)


@pytest.mark.parametrize("d,T,Hq,Hk", KINDS)
def test_rows_that_see_nothing_and_other_sequences_pages(d, T, Hq, Hk):
    """A window with no page under it; and pages that no row sees, whose scales and codes are no numbers."""
    pool = Pool(2, Hk, d, 16, 700 + T, 9)
    q, parents = _tokens(2, T, Hq, d, 3), random_trees(2, T, 3, 1)
    pool.table[0, :] = -1
    before = 600 // 16 - 3
    for p in pool.table[1, :before]:                         # (behind every row's window)
        pool.k[p], pool.v[p] = 0x7F, 0xFF
        pool.ks[p] = pool.vs[p] = math.nan
    got = _attend(pool, q, [600, 600], parents, 20, 0)
    assert not bool(got[0].any())
    _within(got, *_attend_refs(pool, q, [600, 600], parents, 20, 0), torch.float32)


@pytest.mark.parametrize("d,T,Hq,Hk", KINDS)
def test_scales_at_float32_s_edge_in_the_keys(d, T, Hq, Hk):
    """Keys' scales of 2^80 with a scale of 2^-91 for the logits, and the other way round: what is multiplied first does not matter."""
    pool = Pool(1, Hk, d, 32, 300 + T, 9)
    q, parents = _tokens(1, T, Hq, d, 3), random_trees(1, T, 4, 5)
    for up in (80, -80):                                     # (the logits' scale has to be within 1e-30 to 1e30)
        pool.ks[:] = np.float32(2.0 ** up)
        scale = 2.0 ** (-up - 11)
        got = _attend(pool, q, [300], parents, scale=scale)
        _within(got, *_attend_refs(pool, q, [300], parents, scale=scale), torch.float32)


@pytest.mark.parametrize("d,T,Hq", [(128, 3, 8), (128, 20, 8), (64, 40, 8), (128, 35, 16), (64, 5, 16)])
def test_one_long_sequence_of_a_batch(d, T, Hq):
    """Of 64 sequences one is of 17 000 tokens and walked in parts, with the others' few pages walked in the same launch."""
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
    got = _attend(pool, q, held, parents, max_kv_len=long + T)
    _within(got, *_attend_refs(pool, q, held, parents), torch.float32)
    assert torch.equal(got, _attend(pool, q, held, parents))


@pytest.mark.parametrize("T,d", [(24, 64), (24, 128), (64, 64), (64, 128)])
@pytest.mark.parametrize("value", [math.nan, math.inf, -math.inf])
def test_a_state_that_is_not_finite_reaches_its_columns_in_larger_trees(T, d, value):
    import paper_2510_26692_amd as kda
    x = [y.cuda() for y in _inputs(2, T, 2, d, torch.float32, 1)]
    S = (torch.randn(2, 2, d, d, generator=torch.Generator().manual_seed(2)) * 0.3).cuda()
    parents = random_trees(2, T, 3, 5)
    parents[0, T - 5:] = -2
    want = kda.kda_tree_steps(*x, S, int32(parents))
    S[0, 1, d - 3, 41] = value
    got = kda.kda_tree_steps(*x, S, int32(parents))
    odd = torch.zeros(2, T, 2, d, dtype=torch.bool, device="cuda")
    odd[0, :T - 5, 1, 41] = True
    assert bool(torch.equal(got[~odd], want[~odd])) and not bool(torch.isfinite(got[odd]).any())


@pytest.mark.parametrize("T,d", [(16, 128), (17, 64), (32, 128), (50, 64), (64, 128)])
def test_states_of_any_size(T, d):
    """The largest numbers, some far apart, and small ones down to 2^-90: products with the state are off by fp32's steps of its columns."""
    import paper_2510_26692_amd as kda
    x = list(_inputs(1, T, 2, d, torch.float32, T))
    parents = random_trees(1, T, 3, T)
    run = lambda S: _check_steps(*x, S, None, parents, 2.0 ** -6, torch.float32,
                                 kda.kda_tree_steps(*(y.cuda() for y in x), S.cuda(), int32(parents), scale=2.0 ** -6))
    g = torch.Generator().manual_seed(2)
    S = torch.randn(1, 2, d, d, generator=g) * 2.0 ** torch.randint(-30, 31, (1, 2, d, d), generator=g)
    run(S)
    run(S * 2.0 ** 85)
    x[2] = x[2] * 2.0 ** -90
    run(torch.randn(1, 2, d, d, generator=g) * 2.0 ** -90)
    x[2] = x[2] * 0
    S = torch.zeros(1, 2, d, d)
    S[0, :, 5, 3], S[0, :, d - 1, 8] = torch.finfo(torch.float32).max, -3.4e38
    run(S)
