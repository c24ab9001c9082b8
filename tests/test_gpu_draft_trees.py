"""Draft trees: attention over the paged cache, KDA over the tree, the accepted path, and a step of a hybrid stack with all of them, against
the fp64 oracle.

Attention: softmax terms rounded to bf16 (2^-8, and 2^-11 for what is fp32), a bf16 result once more (2^-8), as for kda_cache_attn.

KDA, all fp32 (half a step: 2^-24): a dot product of D terms is off by at most D 2^-24 of its factors' lengths; a decay by 2^-24 |log alpha| and two
steps of the hardware's exponential, and a line's product of them by as often as it is long.  Corrections pass to a line's later tokens through steps
that lengthen nothing (unit keys, beta and alpha up to 1), so that with M the largest length of a state's column or value of v and unit
queries, an output is off by less than  scale (depth + 2) M (2 (D + 16) 2^-24 + 2^-22 (1 + max |log alpha|))."""
import math

import numpy as np
import pytest
import torch

from oracle import draft_trees as dt
from oracle import softmax_attention as sa
from test_gpu_cache import HALF, TERMS, Pool, _np, _tokens

pytestmark = pytest.mark.gpu


def random_trees(N, T, spread, seed, fewest=None, roots=False):
    """Parents of random trees; with `fewest`, sequences of fewer tokens, what is missing at the end or, every third one, anywhere."""
    g = np.random.default_rng(seed)
    out = np.full((N, T), -2, np.int64)
    for n in range(N):
        there = T if fewest is None else int(g.integers(fewest, T + 1))
        for t in range(there):
            out[n, t] = -1 if t == 0 or (roots and g.random() < 0.3) else int(g.integers(max(0, t - spread), t))
        if fewest is not None and n % 3 == 2 and T > 2:
            out[n, int(g.integers(1, T))] = int(g.choice([-2, -7, T, T + 60, 2 ** 31 - 1, -2 ** 31]))
    return out


def int32(x):
    return torch.tensor(np.asarray(x), dtype=torch.int32, device="cuda")


def _cached(pool, which, n, count):
    """Tokens 0..count of a sequence in fp64 [count,Hk,d], and which of them have a page."""
    codes, scale = (pool.k, pool.ks) if which == "k" else (pool.v, pool.vs)
    out, there = np.zeros((count, codes.shape[1], codes.shape[3])), np.zeros(count, bool)
    for t in range(count):
        p = pool.table[n, t // pool.page] if t // pool.page < pool.table.shape[1] else -1
        if 0 <= p < pool.P:
            out[t], there[t] = sa.E4M3[codes[p, :, t % pool.page]] * scale[p][:, None].astype(np.float64), True
    return out, there


def _attend(pool, q, lens, parents, window=0, sinks=0, out_dtype=None, scale=None, max_kv_len=0, **kw):
    import paper_2510_26692_amd as kda
    kd, vd, ksd, vsd, td = pool.device()
    return kda.kda_cache_tree_attn(q.cuda(), kd, vd, ksd, vsd, td, int32(lens), int32(parents), window=window, sinks=sinks, scale=scale,
                                   max_kv_len=max_kv_len, out_dtype=out_dtype, **kw)


def _attend_refs(pool, q, lens, parents, window=0, sinks=0, scale=None):
    T = q.shape[1]
    outs = []
    for n, held in enumerate(lens):
        if held < 0:
            outs.append((np.zeros(q.shape[1:]),) * 2)
            continue
        (k, there), (v, _) = (_cached(pool, x, n, held + T) for x in "kv")
        outs.append(dt.tree_attention(_np(q[n]), k, v, parents[n], held, window, sinks, scale, there))
    return np.stack([o for o, _ in outs]), np.stack([b for _, b in outs])


def _within(got, ref, bound, out_dtype):
    got = _np(got)
    off = np.abs(got - ref) - (TERMS * bound + (HALF * (np.abs(ref) + TERMS * bound) if out_dtype == torch.bfloat16 else 0) + 1e-30)
    assert (off <= 0).all(), (off.max(), np.argwhere(off > 0)[:4].tolist())


ATTEND = [  # d, page, tokens, held, Hq, Hk, spread, fewest, window, sinks
    (128, 64, 16, [100, 0, 63, 64, 65, 500], 8, 2, 4, None, 0, 0), (128, 16, 64, [0, 1, 15, 16, 300], 4, 2, 8, 40, 0, 0),
    (64, 32, 17, [31, 0, 33, 200], 6, 1, 1, None, 0, 0), (128, 128, 33, [127, 128, 1000, 5], 10, 2, 64, 20, 0, 0),
    (64, 16, 64, [0, 47, 48, 49, 700], 4, 4, 2, 30, 0, 0), (128, 64, 1, [0, 1, 640], 4, 1, 1, None, 0, 0),
    (128, 64, 2, [61, 62, 63, 64], 2, 2, 2, None, 0, 0), (128, 32, 64, [100, 3000], 16, 2, 16, None, 0, 0),
    (128, 64, 31, [100, 0, 64, 500], 8, 2, 3, 9, 64, 4), (128, 16, 64, [0, 3, 100, 900], 4, 2, 1, 50, 7, 3),
    (64, 64, 40, [10, 200, 1500], 8, 1, 4, None, 200, 64), (128, 128, 20, [500, 129], 8, 8, 2, 12, 1, 0),
    (128, 16, 24, [300, 64, 0], 5, 1, 4, None, 33, 1), (64, 128, 64, [1, 127, 513], 2, 1, 1, None, 40, 17),
]


@pytest.mark.parametrize("d,page,T,lens,Hq,Hk,spread,fewest,window,sinks", ATTEND)
@pytest.mark.parametrize("out_dtype", [torch.float32, torch.bfloat16])
def test_tree_attention(d, page, T, lens, Hq, Hk, spread, fewest, window, sinks, out_dtype):
    N = len(lens)
    pool = Pool(N, Hk, d, page, max(lens) + T, T + d, nan_behind=[n + T for n in lens])
    q, parents = _tokens(N, T, Hq, d, 3), random_trees(N, T, spread, T + page, fewest, roots=True)
    got = _attend(pool, q, lens, parents, window, sinks, out_dtype, max_kv_len=max(lens) + T if T % 2 else 0)
    _within(got, *_attend_refs(pool, q, lens, parents, window, sinks), out_dtype)
    empty = torch.tensor([[not x for x in dt.lines(p)] for p in parents])
    assert not bool(got.cpu()[empty].any())


def test_tree_attention_of_a_chain_is_cache_attention():
    import paper_2510_26692_amd as kda
    for T, window, sinks in ((8, 0, 0), (5, 40, 2)):
        pool = Pool(3, 2, 128, 32, 400, 5)
        q, held = _tokens(3, T, 8, 128, 4), [300, 0, 33]
        chain = np.tile(np.arange(-1, T - 1), (3, 1))
        kd, vd, ksd, vsd, td = pool.device()
        one = kda.kda_cache_attn(q.cuda(), kd, vd, ksd, vsd, td, int32([h + T for h in held]), window=window, sinks=sinks)
        two = _attend(pool, q, held, chain, window, sinks)
        ref, bound = _attend_refs(pool, q, held, chain, window, sinks)
        _within(one, ref, bound, torch.float32)
        _within(two, ref, bound, torch.float32)


def test_tree_attention_pages_that_are_not_there_skipped_sequences_and_lengths_beyond_the_table():
    pool = Pool(6, 2, 128, 16, 96, 9)
    pool.table[1, 1] = -1                                    # tokens 16..31
    pool.table[2, 0] = pool.P
    pool.table[3, 5] = np.iinfo(np.int32).max                # the last tokens of the tree
    lens = [-1, 60, 3, 70, 84, 96]                           # the last two: drafted tokens without a column
    T = 20
    q, parents = _tokens(6, T, 4, 128, 3), random_trees(6, T, 3, 1)
    for window, sinks in ((0, 0), (30, 4)):
        got = _attend(pool, q, lens, parents, window, sinks)
        _within(got, *_attend_refs(pool, q, lens, parents, window, sinks), torch.float32)
        assert not bool(got[0].any())


def test_tree_attention_where_everything_is_out_of_sight():
    """A window and no page under it: rows that see nothing are zeros, whatever the split."""
    pool = Pool(2, 1, 64, 16, 700, 9)
    pool.table[0, :] = -1
    pool.table[1, 600 // 16 - 3:] = -1
    q, parents = _tokens(2, 9, 2, 64, 3), random_trees(2, 9, 3, 1)
    got = _attend(pool, q, [600, 600], parents, 20, 0)
    assert not bool(got.any())


@pytest.mark.parametrize("where", ["context", "tree", "window"])
def test_tree_attention_values_that_are_no_numbers_reach_those_that_see_them(where):
    T, held, window = 12, 200, 30 if where == "window" else 0
    pool = Pool(1, 2, 128, 16, held + T, 9)
    parents = random_trees(1, T, 4, 5)
    slot = {"context": 77, "tree": held + 3, "window": held - window + 2}[where]
    line = dt.lines(parents[0])
    seen = dt.tree_mask(parents[0], held, window, 0)[:, slot]
    assert seen.any() and (where == "context" or not seen.all())
    page, at = pool.table[0, slot // 16], slot % 16
    q = _tokens(1, T, 4, 128, 3)
    ref, bound = _attend_refs(pool, q, [held], parents, window)
    pool.v[page, 1, at, 5] = 0x7F
    got = _np(_attend(pool, q, [held], parents, window))[0]
    off = ~np.isnan(got)
    want = np.ones(got.shape, bool)
    want[np.ix_(seen, [2, 3], [5])] = False                  # (heads 2 and 3 read key head 1)
    assert np.array_equal(off, want), line
    _within(torch.tensor(np.where(want, got, ref[0])), ref[0], bound[0], torch.float32)
    pool.v[page, 1, at, 5] = 0
    pool.k[page, 0, at, 9] = 0xFF
    got = _np(_attend(pool, q, [held], parents, window))[0]
    want = np.zeros(got.shape, bool)
    want[np.ix_(seen, [0, 1], np.arange(128))] = True
    assert np.array_equal(np.isnan(got), want)


def test_tree_attention_scales_of_any_size():
    """Scales that are no powers of two, large and small ones: what they do to the logits and to the values is exact in fp32."""
    T, held = 16, 300
    pool = Pool(2, 2, 64, 32, held + T, 11)
    g = np.random.default_rng(3)
    pool.ks = (pool.ks * g.uniform(0.5, 2, pool.ks.shape)).astype(np.float32)
    pool.vs = np.float32(g.uniform(0.5, 2, pool.vs.shape))
    q, parents = _tokens(2, T, 4, 64, 3), random_trees(2, T, 4, 5)
    for factor in (1.0, 2.0 ** 100, 2.0 ** -60):
        pool.vs = np.float32(pool.vs * np.float32(factor))
        got = _attend(pool, q, [held, 40], parents)
        _within(got, *_attend_refs(pool, q, [held, 40], parents), torch.float32)
        pool.vs = np.float32(pool.vs / np.float32(factor))
    pool.vs[:] = np.float32(2.0 ** 118)
    got = _attend(pool, q, [held, 40], parents)
    assert bool(torch.isfinite(got).all())
    _within(got, *_attend_refs(pool, q, [held, 40], parents), torch.float32)


def test_tree_attention_spaced_queries_given_output_and_workspace():
    import paper_2510_26692_amd as kda
    pool = Pool(2, 2, 128, 64, 3000, 9)
    fused = torch.randn(2, 20, 12 * 128, generator=torch.Generator().manual_seed(1)).to(torch.bfloat16).cuda()
    q = fused[..., :8 * 128].view(2, 20, 8, 128)
    assert not q.is_contiguous()
    parents, lens = random_trees(2, 20, 3, 8), [2900, 700]
    kd, vd, ksd, vsd, td = pool.device()
    o = torch.full((2, 20, 8, 128), 7.0, device="cuda")
    got = kda.kda_cache_tree_attn(q, kd, vd, ksd, vsd, td, int32(lens), int32(parents), o=o)
    assert got is o
    _within(o, *_attend_refs(pool, q.cpu(), lens, parents), torch.float32)
    again = kda.kda_cache_tree_attn(q.contiguous(), kd, vd, ksd, vsd, td, int32(lens), int32(parents))
    assert torch.equal(o, again)


# ---- KDA ----

def _inputs(N, T, H, d, dtype, seed, decay=-0.3):
    g = torch.Generator().manual_seed(seed)
    unit = lambda: torch.nn.functional.normalize(torch.randn(N, T, H, d, generator=g), dim=-1).to(dtype)
    q, k, v = unit(), unit(), torch.randn(N, T, H, d, generator=g).to(dtype)
    return q, k, v, (decay * torch.rand(N, T, H, d, generator=g)).to(dtype), torch.rand(N, T, H, generator=g).to(dtype)


def _delta_tol(d, depth, size, la, scale):
    # (unit vectors in bf16 are up to 2^-8 longer, which the lines' lengths see twice a token)
    return scale * (depth + 2) * size * (2 * (d + 16) * 2.0 ** -24 + 2.0 ** -22 * (1 + float(np.abs(la).max()))) * (1 + 2.0 ** -8) ** (2 * depth + 2)


def _check_steps(q, k, v, la, beta, S, idx, parents, scale, out_dtype, o, scalar=False):
    N, T, H, d = q.shape
    for n in range(N):
        slot = n if idx is None else int(idx[n])
        got = _np(o[n])
        if slot < 0:
            assert not got.any()
            continue
        a = np.exp(_np(la[n]))
        a = np.broadcast_to(a[..., None], (T, H, d)) if scalar else a
        ref, size = dt.tree_steps(_np(q[n]), _np(k[n]), _np(v[n]), a, _np(beta[n]), _np(S[slot]), parents[n], scale)
        depth = max([len(x) for x in dt.lines(parents[n])])
        tol = _delta_tol(d, depth, size, _np(la[n]), abs(scale))
        off = np.abs(got - ref) - tol - (HALF * (np.abs(ref) + tol) if out_dtype == torch.bfloat16 else 0)
        assert (off <= 0).all(), (n, off.max(), tol)
        for t, line in enumerate(dt.lines(parents[n])):
            assert line or not got[t].any()


STEPS = [  # N, T, H, d, dtype, spread, fewest
    (3, 16, 2, 128, torch.bfloat16, 4, None), (2, 16, 3, 128, torch.float32, 1, None), (3, 7, 2, 64, torch.bfloat16, 2, 3),
    (3, 32, 1, 128, torch.bfloat16, 8, 17), (2, 64, 2, 128, torch.bfloat16, 16, 30), (2, 64, 1, 128, torch.float32, 1, None),
    (3, 64, 2, 64, torch.float32, 64, 10), (2, 33, 2, 64, torch.bfloat16, 1, None), (2, 1, 2, 128, torch.bfloat16, 1, None),
    (3, 49, 1, 128, torch.float32, 3, 40), (1, 17, 5, 128, torch.bfloat16, 2, None), (4, 2, 1, 64, torch.float32, 1, 1),
]


@pytest.mark.parametrize("N,T,H,d,dtype,spread,fewest", STEPS)
@pytest.mark.parametrize("out_dtype", [torch.float32, torch.bfloat16])
def test_tree_steps(N, T, H, d, dtype, spread, fewest, out_dtype):
    import paper_2510_26692_amd as kda
    q, k, v, la, beta = _inputs(N, T, H, d, dtype, T + d)
    S = torch.randn(N + 2, H, d, d, generator=torch.Generator().manual_seed(2)) * 0.3
    parents = random_trees(N, T, spread, T, fewest, roots=True)
    idx = torch.arange(N + 1, 1, -1, dtype=torch.int32)
    Sd = S.cuda()
    o = kda.kda_tree_steps(*(x.cuda() for x in (q, k, v, la, beta)), Sd, int32(parents), state_indices=idx.cuda(), scale=d ** -0.5, out_dtype=out_dtype)
    assert o.dtype == out_dtype and torch.equal(Sd.cpu(), S)
    _check_steps(q, k, v, la, beta, S, idx, parents, d ** -0.5, out_dtype, o)


def test_tree_steps_skipped_and_shared_states_scalar_gate_and_inputs_that_are_not_there():
    import paper_2510_26692_amd as kda
    N, T, H, d = 4, 12, 2, 128
    q, k, v, la, beta = _inputs(N, T, H, d, torch.bfloat16, 5)
    S = torch.randn(3, H, d, d, generator=torch.Generator().manual_seed(2)) * 0.3
    parents = random_trees(N, T, 3, 1, 5)
    parents[3, 6:] = -2
    idx = torch.tensor([1, -1, 1, 2], dtype=torch.int32)
    for x in (q, k, v, la, beta):                            # (tokens that are not there may be anything)
        x[3, 6:] = math.nan
    for scalar in (False, True):
        g = la[..., 0].contiguous() if scalar else la
        o = torch.full((N, T, H, d), 7.0, device="cuda")
        kda.kda_tree_steps(q.cuda(), k.cuda(), v.cuda(), g.cuda(), beta.cuda(), S.cuda(), int32(parents), state_indices=idx.cuda(), scale=0.5, o=o,
                           scalar_gate=scalar)
        clean = [torch.nan_to_num(x) for x in (q, k, v, g, beta)]
        _check_steps(*clean, S, idx, parents, 0.5, torch.float32, o, scalar)


def test_tree_steps_of_a_chain_are_decode_steps_and_strong_decays_vanish():
    import paper_2510_26692_amd as kda
    N, T, H, d = 2, 8, 2, 128
    for decay in (-0.3, -60.0):
        q, k, v, la, beta = (x.cuda() for x in _inputs(N, T, H, d, torch.bfloat16, 5, decay))
        S = (torch.randn(N, H, d, d, generator=torch.Generator().manual_seed(2)) * 0.3).cuda()
        o = kda.kda_tree_steps(q, k, v, la, beta, S, int32(np.tile(np.arange(-1, T - 1), (N, 1))))
        kept = int32(np.tile(np.arange(T), (N, 1)))
        S1, S2 = S.clone(), S.clone()
        o1 = kda.kda_recurrent_steps_pooled(q, k, v, la, beta, S1)
        kda.kda_tree_commit(k, v, la, beta, S2, kept)
        tol = _delta_tol(d, T, 8.0, _np(la), 1.0)            # (no column or value is longer than 8)
        assert float((o - o1).abs().max()) <= 2 * tol and float((S1 - S2).abs().max()) <= 2 * tol


@pytest.mark.parametrize("N,T,H,d,dtype,most", [(4, 16, 2, 128, torch.bfloat16, 16), (5, 64, 1, 128, torch.float32, 64), (4, 20, 3, 64, torch.bfloat16, 9),
                                                (3, 9, 2, 64, torch.float32, 12), (3, 1, 1, 128, torch.bfloat16, 1)])
@pytest.mark.parametrize("scalar", [False, True])
def test_tree_commit(N, T, H, d, dtype, most, scalar):
    import paper_2510_26692_amd as kda
    _, k, v, la, beta = _inputs(N, T, H, d, dtype, T + d)
    la = la[..., 0].contiguous() if scalar else la
    g = np.random.default_rng(T)
    kept = np.full((N, most), -1)
    for n in range(N):
        path = np.sort(g.permutation(T)[:g.integers(0, min(T, most) + 1)])
        kept[n, :len(path)] = path
    if most > 4:
        kept[0, :5] = [0, 1, 1, 2, 3]                        # (an entry that is not above the one before ends the path)
        kept[1, :4] = [0, 2, T, T + 1]                       # (and one behind the tokens)
    idx = torch.tensor([N + 1 - n if n != N - 1 else -1 for n in range(N)], dtype=torch.int32)
    S = torch.randn(N + 2, H, d, d, generator=torch.Generator().manual_seed(2)) * 0.3
    Sd = S.cuda()
    assert kda.kda_tree_commit(k.cuda(), v.cuda(), la.cuda(), beta.cuda(), Sd, int32(kept), state_indices=idx.cuda(), scalar_gate=scalar) is None
    ref = _np(S)
    size = 0.0
    for n in range(N):
        if idx[n] >= 0:
            a = np.exp(_np(la[n]))
            a = np.broadcast_to(a[..., None], (T, H, d)) if scalar else a
            ref[idx[n]] = dt.commit(_np(k[n]), _np(v[n]), a, _np(beta[n]), _np(S[idx[n]]), kept[n])
    size = max(np.sqrt((ref ** 2).sum(2)).max(), np.sqrt((_np(S) ** 2).sum(2)).max(), np.abs(_np(v)).max())
    off = np.abs(_np(Sd) - ref).max()
    assert off <= _delta_tol(d, min(T, most), size, _np(la), 1.0), off
    untouched = [i for i in range(N + 2) if i not in idx.tolist() or kept[idx.tolist().index(i)][0] < 0]
    assert torch.equal(Sd.cpu()[untouched], S[untouched])


# ---- the accepted path in the cache ----

def _stack(L, N, Hk, d, page, most, seed):
    pools = [Pool(N, Hk, d, page, most, seed + i) for i in range(L)]
    for p in pools[1:]:
        p.table = pools[0].table
    return pools


def _device_stack(pools):
    f8 = lambda x: torch.from_numpy(np.stack(x)).cuda().view(torch.float8_e4m3fn)
    f32 = lambda x: torch.from_numpy(np.stack(x)).cuda()
    return [f8([p.k for p in pools]), f8([p.v for p in pools]), f32([p.ks for p in pools]), f32([p.vs for p in pools])]


def _same_codes(got, want):
    got = got.view(torch.uint8).cpu().numpy()
    same = (got == want) | (((got & 127) == 127) & ((want & 127) == 127))
    assert same.all(), np.argwhere(~same)[:4].tolist()


@pytest.mark.parametrize("L,d,page,T,lens", [
    (3, 128, 64, 16, [0, 1, 50, 63, 64, 500]), (2, 64, 16, 64, [15, 16, 17, 0, 47, 100]), (1, 128, 16, 64, [15, 1, 0, 13, 31, 33]),
    (2, 128, 128, 33, [120, 127, 128, 100, 5, 0]), (1, 64, 32, 1, [31, 32, 0, 3, 4, 5]), (2, 64, 128, 40, [90, 126, 127, 200, 255, 3])])
def test_keep(L, d, page, T, lens):
    import paper_2510_26692_amd as kda
    N = len(lens)
    pools = _stack(L, N, 2, d, page, max(lens) + T, 7)
    g = np.random.default_rng(T + page)
    kept = np.full((N, T), -1)
    for n in range(N):
        path = np.sort(g.permutation(T)[:g.integers(1, T + 1)])
        kept[n, :len(path)] = path
    if T > 4:
        kept[1] = -1
        kept[2, :5] = [0, 1, 4, 4, 5]
    args = _device_stack(pools)
    kda.kda_cache_keep(*args, torch.from_numpy(pools[0].table).cuda(), int32(lens), int32(kept))
    for p in pools:
        for c, s in ((p.k, p.ks), (p.v, p.vs)):
            dt.keep(c, s, p.table, lens, kept)
    for i, p in enumerate(pools):
        _same_codes(args[0][i], p.k)
        _same_codes(args[1][i], p.v)
        np.testing.assert_array_equal(args[2][i].cpu().numpy(), p.ks)
        np.testing.assert_array_equal(args[3][i].cpu().numpy(), p.vs)


def test_keep_of_one_layer_without_pages_skipped_sequences_and_scales_of_any_size():
    import paper_2510_26692_amd as kda
    pool = Pool(5, 3, 128, 16, 96, 9)
    pool.table[1, 3] = -1                                    # tokens 48..63: gone, wherever they are wanted or would go
    pool.table[2, 1] = pool.P
    lens = [-1, 40, 14, 90, 2 ** 31 - 1]
    kept = np.tile(np.array([1, 3, 4, 8, 9, 12, 13, 20, 30, 50, -1, 60]), (5, 1))
    pool.ks = (pool.ks * np.random.default_rng(1).uniform(0.5, 2, pool.ks.shape)).astype(np.float32)
    kd, vd, ksd, vsd, td = pool.device()
    kda.kda_cache_keep(kd, vd, ksd, vsd, td, int32(lens), int32(kept))
    for c, s in ((pool.k, pool.ks), (pool.v, pool.vs)):
        dt.keep(c, s, pool.table, lens[:4], kept)
    # (codes whose scale changes by no power of two: fp32 division and product, each rounded once, as the oracle's)
    _same_codes(kd, pool.k)
    _same_codes(vd, pool.v)
    np.testing.assert_array_equal(ksd.cpu().numpy(), pool.ks)
    np.testing.assert_array_equal(vsd.cpu().numpy(), pool.vs)


# ---- all of it ----

def _flow(seed, device="cuda"):
    """A step of a hybrid stack's two kinds of layers: a tree is drafted, verified and its accepted path kept; then the next token is decoded as if
    the path had been appended token by token."""
    import paper_2510_26692_amd as kda
    N, T, Hq, Hk, d, page, held = 3, 12, 8, 2, 128, 16, [30, 61, 0]
    pool = Pool(N, Hk, d, page, 120, seed)
    kd, vd, ksd, vsd, td = (x.to(device) for x in pool.device())
    i32 = lambda x: torch.tensor(np.asarray(x), dtype=torch.int32, device=device)
    parents = random_trees(N, T, 4, seed)
    depth = np.array([[len(x) - 1 for x in dt.lines(p)] for p in parents])
    kept = np.full((N, T), -1)
    for n in range(N):
        path = dt.lines(parents[n])[T - 1 - n]
        kept[n, :len(path)] = path
    k, v, q = (_tokens(N, T, H, d, seed + H).to(device) for H in (Hk, Hk, Hq))
    v = v * 0.5
    f = torch.from_numpy(np.float32(10000.0 ** (-np.arange(64) / 64))).to(device)
    lens = i32(held)
    qr, kr = kda.kda_rotate(q, k, lens[:, None] + i32(depth), f)
    caches = (kd, vd, ksd, vsd)
    kda.kda_cache_append(kr, v, *caches, td, lens)
    o = kda.kda_cache_tree_attn(qr, *caches, td, lens, i32(parents))
    kda.kda_cache_keep(*caches, td, lens, i32(kept))
    count = (kept >= 0).sum(1)
    # the same tokens, one after the other
    pool2 = Pool(N, Hk, d, page, 120, seed)
    kd2, vd2, ksd2, vsd2, td2 = (x.to(device) for x in pool2.device())
    o2 = []
    for n in range(N):
        outs = []
        for i in range(count[n]):
            t = int(kept[n, i])
            # (one sequence at a time; the others are skipped)
            only = i32([held[n] + i if m == n else -1 for m in range(N)])
            row = lambda x: x[:, t:t + 1].contiguous()
            q1, _ = kda.kda_cache_append(row(k), row(v), kd2, vd2, ksd2, vsd2, td2, only, inv_freq=f, q=row(q))
            outs.append(kda.kda_cache_attn(q1, kd2, vd2, ksd2, vsd2, td2, torch.where(only >= 0, only + 1, only))[n, 0])
        o2.append(torch.stack(outs))
    return o, o2, kept, count, (kd, vd, ksd, vsd, td), (kd2, vd2, ksd2, vsd2, td2), held


def test_a_verified_step_is_the_same_as_its_tokens_one_by_one():
    """Attention of the accepted tokens over the drafted tree and over the cache that grows token by token see the same keys, but for codes: pages'
    scales may differ where a larger token that was not accepted stood with them, by one rounding to e4m3 more (2^-4 of a value, 2^-10 of a page's
    smallest step)."""
    o, o2, kept, count, one, two, held = _flow(3)
    for n in range(3):
        path = torch.tensor(kept[n, :count[n]], device=o.device)
        a, b = o[n, path], o2[n]
        # values up to 2 and keys up to 7: terms differ by exp of the logits' difference, 2 2^-4 |q||k| / sqrt(d) at the very most
        assert float((a - b).abs().max()) <= 0.25, n
        length = held[n] + int(count[n])
        for c in (0, 1):
            for t in range(length):
                x, y = (s[c].float()[s[4][n, t // 16].long(), :, t % 16] * s[2 + c][s[4][n, t // 16].long()][:, None] for s in (one, two))
                step = torch.maximum(one[2 + c][one[4][n, t // 16].long()], two[2 + c][two[4][n, t // 16].long()])[:, None]
                # (both are roundings of the same value, to 2^-4 of it or half the smallest step, once or, where a scale grew, twice or thrice)
                assert bool(((x - y).abs() <= 4 * (2.0 ** -4 * torch.maximum(x.abs(), y.abs()) + 2.0 ** -10 * step)).all()), (n, c, t)


def test_a_captured_step_replays():
    """The whole step in a graph, replayed with other contents of its buffers between eager work; two graphs with their own workspaces."""
    import paper_2510_26692_amd as kda
    N, T, Hq, Hk, d, page = 2, 16, 8, 2, 128, 64
    dev = "cuda"

    def make(seed):
        pool = Pool(N, Hk, d, page, 3000, seed)
        k, v, q = (_tokens(N, T, H, d, seed + H).to(dev) for H in (Hk, Hk, Hq))
        kq, kk, kv, la, beta = (x.to(dev) for x in _inputs(N, T, 4, d, torch.bfloat16, seed))
        S = (torch.randn(N, 4, d, d, generator=torch.Generator().manual_seed(seed)) * 0.3).to(dev)
        parents = random_trees(N, T, 4, seed)
        kept = np.full((N, T), -1)
        for n in range(N):
            path = dt.lines(parents[n])[T - 1]
            kept[n, :len(path)] = path
        depth = int32([[len(x) - 1 for x in dt.lines(p)] for p in parents])
        lens = int32([2900 - seed, 100 + seed])
        return [q, k, v, kq, kk, kv, la, beta, S, int32(parents), int32(kept), lens[:, None] + depth, lens, *pool.device()]

    f = torch.from_numpy(np.float32(10000.0 ** (-np.arange(64) / 64))).cuda()

    def run(s):
        q, k, v, kq, kk, kv, la, beta, S, parents, kept, pos, lens, kd, vd, ksd, vsd, td = s
        qr, kr = kda.kda_rotate(q, k, pos, f)
        kda.kda_cache_append(kr, v, kd, vd, ksd, vsd, td, lens)
        o = kda.kda_cache_tree_attn(qr, kd, vd, ksd, vsd, td, lens, parents, max_kv_len=3000)
        o2 = kda.kda_tree_steps(kq, kk, kv, la, beta, S, parents)
        kda.kda_cache_keep(kd, vd, ksd, vsd, td, lens, kept)
        kda.kda_tree_commit(kk, kv, la, beta, S, kept)
        return o, o2

    graphs = []
    for i in range(2):
        s = make(1)
        run(s)
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            out = run(s)
        graphs.append((g, s, out))
    for seed in (2, 3, 4):
        for g, s, out in graphs:
            fresh = make(seed)
            for a, b in zip(s, fresh):
                a.copy_(b) if a.dtype != torch.float8_e4m3fn else a.view(torch.uint8).copy_(b.view(torch.uint8))
            want = run(fresh)
            torch.cuda.synchronize()
            g.replay()
            torch.cuda.synchronize()
            assert all(torch.equal(x, y) for x, y in zip(out, want))
            bits = lambda x: x.view(torch.uint8) if x.dtype == torch.float8_e4m3fn else x
            assert all(torch.equal(bits(x), bits(y)) for x, y in zip(s, fresh))


def test_calls_on_two_streams_at_once():
    streams = [torch.cuda.Stream() for _ in range(2)]
    T = 24
    jobs = []
    for i in range(2):
        pool = Pool(2, 2, 128, 64, 3000, 20 + i)
        jobs.append((pool, _tokens(2, T, 8, 128, 30 + i), [2800, 900 + i], random_trees(2, T, 3, i)))
    want = [_attend(*j) for j in jobs]
    torch.cuda.synchronize()
    got = [[], []]
    for _ in range(4):
        for i, st in enumerate(streams):
            with torch.cuda.stream(st):
                got[i].append(_attend(*jobs[i]))
    torch.cuda.synchronize()
    for w, g in zip(want, got):
        assert all(torch.equal(w, x) for x in g)


def test_nothing_is_written_outside():
    """Outputs between guards, with rows that belong to nobody."""
    import paper_2510_26692_amd as kda
    N, T, H, d = 2, 5, 3, 64
    q, k, v, la, beta = (x.cuda() for x in _inputs(N, T, H, d, torch.float32, 1))
    S = torch.zeros(N, H, d, d, device="cuda")
    room = torch.full((N * T * H * d + 512,), 7.0, device="cuda")
    o = room[256:-256].view(N, T, H, d)
    kda.kda_tree_steps(q, k, v, la, beta, S, int32(random_trees(N, T, 2, 1)), o=o)
    assert bool((room[:256] == 7).all()) and bool((room[-256:] == 7).all()) and not bool((o == 7).any())
    pool = Pool(N, 1, d, 16, 60, 3)
    kd, vd, ksd, vsd, td = pool.device()
    room.fill_(7.0)
    kda.kda_cache_tree_attn(_tokens(N, T, H, d, 1).cuda(), kd, vd, ksd, vsd, td, int32([40, 3]), int32(random_trees(N, T, 2, 1)), o=o)
    assert bool((room[:256] == 7).all()) and bool((room[-256:] == 7).all()) and not bool((o == 7).any())
