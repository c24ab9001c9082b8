"""The paged 8-bit cache: appending with the rotation on the way, and attention over it, against the fp64 oracle.

Codes and scales are compared bit by bit: the kernel turns keys by angles held in 64 bits and rounds once to fp32, as the oracle does.
Rotated queries and keys in bf16 are within half a step (2^-8) of the exact rotation, and 2^-18 of the pair's length for queries,
whose sine and cosine are the hardware's.  Attention: softmax terms rounded to bf16 (2^-8, and 2^-11 for what is fp32), the
result once more."""
import math

import numpy as np
import pytest
import torch

from helpers import Guarded
from oracle import softmax_attention as sa

pytestmark = pytest.mark.gpu

TERMS = 2.0 ** -8 + 2.0 ** -11
HALF = 2.0 ** -8


def _np(t):
    return t.detach().cpu().double().numpy()


class Pool:
    """A cache on the host and on the device: random codes (NaN ones among them where nothing valid stands) and scales, shuffled pages."""

    def __init__(self, N, Hk, d, page, max_len, seed, spare=3, nan_behind=None):
        g = np.random.default_rng(seed)
        self.cols = -(-max_len // page)
        self.P = N * self.cols + spare
        self.k, self.v = (sa.e4m3_encode(g.standard_normal((self.P, Hk, page, d)) * 80) for _ in range(2))
        self.ks, self.vs = (np.float32(2.0) ** g.integers(-8, -4, (self.P, Hk)).astype(np.float32) for _ in range(2))
        self.table = g.permutation(self.P)[:N * self.cols].reshape(N, self.cols).astype(np.int32)
        self.page = page
        if nan_behind is not None:                           # codes behind the last token are not numbers
            valid = np.zeros((self.P, page), bool)
            for n, length in enumerate(nan_behind):
                for t in range(max(0, length)):
                    valid[self.table[n, t // page], t % page] = True
            for x in (self.k, self.v):
                x[np.broadcast_to(~valid[:, None, :, None], x.shape)] = 0x7F

    def device(self):
        f8 = lambda x: torch.from_numpy(x).cuda().view(torch.float8_e4m3fn)
        return f8(self.k), f8(self.v), torch.from_numpy(self.ks).cuda(), torch.from_numpy(self.vs).cuda(), torch.from_numpy(self.table).cuda()


def _tokens(N, T, H, d, seed, cu=None):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(N, T, H, d, generator=g) * 1.3).to(torch.bfloat16)


def _positions(B, T, lens, cu):
    if cu is None:
        return [np.arange(T) + lens[b] for b in range(B)]
    return [np.concatenate([np.zeros(cu[0], np.int64)] + [np.arange(e - s) + lens[n] for n, (s, e) in enumerate(zip(cu[:-1], cu[1:]))] + [np.zeros(T - cu[-1], np.int64)])]


def _freqs(n, base=10000.0):
    return np.float32(base ** (-np.arange(n) / max(1, n)))


def _append_both(pool, k, v, lens, cu=None, freqs=None, inter=False, q=None, want_k=False):
    """The call and the oracle on the same cache; returns the device's (q_out, k_out) and the exact rotated q and k."""
    import paper_2510_26692_amd as kda
    dev = pool.device()
    kd, vd, ksd, vsd, td = dev
    cud = None if cu is None else torch.tensor(cu, dtype=torch.int32, device="cuda")
    out = kda.kda_cache_append(k.cuda(), v.cuda(), kd, vd, ksd, vsd, td, torch.tensor(lens, dtype=torch.int32, device="cuda"), cu_seqlens=cud,
                               inv_freq=None if freqs is None else torch.from_numpy(freqs).cuda(), interleaved=inter, q=None if q is None else q.cuda(),
                               want_k=want_k)
    torch.cuda.synchronize()
    B, T = k.shape[:2]
    pos = _positions(B, T, lens, cu)
    turn = lambda x: np.stack([_np(x[b]) if freqs is None else sa.rotate(_np(x[b]), pos[b], freqs, inter) for b in range(B)])
    kr = turn(k)
    sa.append(kr.astype(np.float32), _np(v).astype(np.float32), pool.k, pool.v, pool.ks, pool.vs, pool.table, lens, cu)
    for name, got, want in (("k", kd, pool.k), ("v", vd, pool.v)):
        got = got.view(torch.uint8).cpu().numpy()
        # (a code that is not a number has no sign to speak of)
        same = (got == want) | (((got & 127) == 127) & ((want & 127) == 127))
        assert same.all(), "%s codes differ at %s" % (name, np.argwhere(~same)[:4].tolist())
    np.testing.assert_array_equal(ksd.cpu().numpy(), pool.ks)
    np.testing.assert_array_equal(vsd.cpu().numpy(), pool.vs)
    return out, (None if q is None else turn(q)), kr


def _turned_within(got, exact, raw):
    length = np.abs(_np(raw)).max(-1, keepdims=True)
    off = np.abs(_np(got) - exact) - (HALF * np.abs(exact) + 2.0 ** -18 * (1 + HALF) * 2 * length)
    assert (off <= 0).all(), off.max()


@pytest.mark.parametrize("d,page,T,lens,freqs,inter", [
    (128, 64, 1, [0, 1, 63, 64, 65, 500], 64, False), (64, 16, 1, [15, 16, 17, 31, 0, 200], 32, True), (128, 128, 8, [0, 120, 121, 127, 128, 300], 64, True),
    (64, 32, 5, [30, 0, 27, 28, 31, 64], 16, False), (128, 16, 7, [9, 10, 15, 0, 3, 100], 24, False), (128, 64, 9, [0, 55, 56, 63, 64, 1], 64, False),
    (64, 128, 200, [0, 1, 127, 128, 129, 60], 32, False), (128, 32, 100, [0, 31, 5, 64, 33, 90], 32, True), (128, 16, 33, [0, 15, 16, 17, 1, 2], 0, False),
    (128, 128, 130, [0, 127, 126, 1, 200, 3], None, False),
])
def test_append_fixed(d, page, T, lens, freqs, inter):
    N, Hk, Hq = len(lens), 2, 6
    pool = Pool(N, Hk, d, page, max(lens) + T, T + d)
    k, v, q = _tokens(N, T, Hk, d, 1), _tokens(N, T, Hk, d, 2), _tokens(N, T, Hq, d, 3)
    f = None if freqs is None else _freqs(freqs)
    (q_out, k_out), q_ref, k_ref = _append_both(pool, k, v, lens, freqs=f, inter=inter, q=q, want_k=True)
    _turned_within(q_out, q_ref, q)
    _turned_within(k_out, k_ref, k)


@pytest.mark.parametrize("lens_new,before,behind,held,page,d", [
    ([5, 0, 300, 64, 1, 129], 3, 6, [0, 7, 61, 64, 31, 100], 64, 128), ([200], 0, 0, [13], 128, 64), ([0, 0, 16], 5, 5, [1, 2, 0], 16, 128),
    ([1, 1, 1, 1], 0, 0, [15, 16, 0, 31], 16, 64), ([40, 500], 0, 3, [0, 127], 32, 64)])
def test_append_packed(lens_new, before, behind, held, page, d):
    T = before + sum(lens_new) + behind
    cu = (before + np.concatenate([[0], np.cumsum(lens_new)])).tolist()
    pool = Pool(len(held), 2, d, page, max(h + n for h, n in zip(held, lens_new)), T)
    k, v, q = _tokens(1, T, 2, d, 1), _tokens(1, T, 2, d, 2), _tokens(1, T, 10, d, 3)
    (q_out, k_out), q_ref, k_ref = _append_both(pool, k, v, held, cu=cu, freqs=_freqs(d // 2), q=q, want_k=True)
    rows = slice(cu[0], cu[-1])
    _turned_within(q_out[:, rows], q_ref[:, rows], q[:, rows])
    _turned_within(k_out[:, rows], k_ref[:, rows], k[:, rows])
    for t in (q_out, k_out):
        assert not bool(t[:, :cu[0]].any()) and not bool(t[:, cu[-1]:].any())


def test_append_skips_sequences_and_pages_that_are_not_there():
    pool = Pool(5, 2, 128, 16, 64, 9)
    pool.table[1, 1] = -1                                    # the page of tokens 16..31
    pool.table[2, 0] = pool.P
    pool.table[3, 3] = np.iinfo(np.int32).max
    lens = [-1, 14, 3, 60, 62]                               # the last one: beyond the table's columns
    k, v, q = _tokens(5, 7, 2, 128, 1), _tokens(5, 7, 2, 128, 2), _tokens(5, 7, 4, 128, 3)
    (q_out, k_out), q_ref, k_ref = _append_both(pool, k, v, lens, freqs=_freqs(64), q=q, want_k=True)
    _turned_within(q_out[1:], q_ref[1:], q[1:])
    _turned_within(k_out[1:], k_ref[1:], k[1:])
    assert not bool(q_out[0].any()) and not bool(k_out[0].any())


def test_append_rows_of_nobody_in_what_is_passed_in_and_what_is_allocated():
    """Skipped sequences and unowned tokens: untouched in q_out and k_out that the caller brings, zeros in fresh ones; a batch of no
    sequences at all."""
    import paper_2510_26692_amd as kda
    pool = Pool(3, 2, 64, 16, 64, 9)
    kd, vd, ksd, vsd, td = pool.device()
    f = torch.from_numpy(_freqs(32)).cuda()
    k, v, q = (_tokens(1, 30, h, 64, h).cuda() for h in (2, 2, 4))
    lens = torch.tensor([4, -3, 9], dtype=torch.int32, device="cuda")
    cu = torch.tensor([2, 10, 15, 27], dtype=torch.int32, device="cuda")
    nobody = torch.ones(30, dtype=torch.bool)
    nobody[2:10] = nobody[15:27] = False
    outs = []
    for given in (False, True):
        q_in, k_in = (torch.full_like(t, 7) for t in (q, k)) if given else (None, None)
        q_out, k_out = kda.kda_cache_append(k, v, kd, vd, ksd, vsd, td, lens, cu_seqlens=cu, inv_freq=f, q=q, q_out=q_in, k_out=k_in, want_k=True)
        for t in (q_out, k_out):
            assert bool((t[0, nobody] == (7 if given else 0)).all())
        outs.append((q_out[0, ~nobody], k_out[0, ~nobody]))
    assert all(torch.equal(a, b) for a, b in zip(*outs))
    only_k = kda.kda_cache_append(k, v, kd, vd, ksd, vsd, td, lens, cu_seqlens=cu, inv_freq=f, want_k=True)
    assert only_k[0] is None and torch.equal(only_k[1][0, ~nobody], outs[0][1]) and not bool(only_k[1][0, nobody].any())
    none = torch.zeros(1, dtype=torch.int32, device="cuda")
    q_out, k_out = kda.kda_cache_append(k, v, kd, vd, ksd, vsd, td[:0], lens[:0], cu_seqlens=none, inv_freq=f, q=q, want_k=True)
    assert not bool(q_out.any()) and not bool(k_out.any())


def test_append_turns_keys_and_queries_in_place():
    import paper_2510_26692_amd as kda
    for T, inter in ((3, False), (70, True)):
        pool = Pool(2, 2, 128, 32, 200, 9)
        k, v, q = (_tokens(2, T, h, 128, h).cuda() for h in (2, 2, 4))
        lens = torch.tensor([4, 100], dtype=torch.int32, device="cuda")
        f = torch.from_numpy(_freqs(64)).cuda()
        outs = []
        for place in (False, True):
            kd, vd, ksd, vsd, td = pool.device()
            ki, qi = k.clone(), q.clone()
            qo, ko = kda.kda_cache_append(ki, v, kd, vd, ksd, vsd, td, lens, inv_freq=f, interleaved=inter, q=qi, q_out=qi if place else None,
                                          k_out=ki if place else None, want_k=True)
            assert (qo is qi and ko is ki) if place else bool((qi == q).all() and (ki == k).all())
            outs.append([qo, ko, kd.view(torch.uint8), vd.view(torch.uint8), ksd, vsd])
        assert all(torch.equal(x, y) for x, y in zip(*outs))


def test_cache_calls_on_two_streams_at_once():
    import paper_2510_26692_amd as kda
    f = torch.from_numpy(_freqs(64)).cuda()
    jobs = []
    for i in range(2):
        pool = Pool(3, 2, 128, 64, 3000, 20 + i)
        k, v, q = (_tokens(3, 2, h, 128, 30 + 3 * i + h).cuda() for h in (2, 2, 8))
        jobs.append((pool, k, v, q, torch.tensor([2900, 64, 1000 + i], dtype=torch.int32, device="cuda")))

    def run(job, times):
        pool, k, v, q, lens = job
        dev = pool.device()
        torch.cuda.synchronize()
        outs = []
        for _ in range(times):
            qo, _ = kda.kda_cache_append(k, v, *dev, lens, inv_freq=f, q=q)
            outs.append(kda.kda_cache_attn(qo, *dev, lens + 2))
        return outs

    want = [run(j, 1)[0] for j in jobs]
    torch.cuda.synchronize()
    got = []
    for j, s in zip(jobs, [torch.cuda.Stream(), torch.cuda.Stream()]):
        with torch.cuda.stream(s):
            got.append(run(j, 4))
    torch.cuda.synchronize()
    assert all(torch.equal(w, o) for w, outs in zip(want, got) for o in outs)


def test_append_token_by_token_rounds_older_codes_again():
    import paper_2510_26692_amd as kda
    pool = Pool(2, 2, 64, 32, 96, 4)
    g = torch.Generator().manual_seed(5)
    lens = [0, 20]
    for t in range(40):                                      # growing magnitudes: scales grow on the way
        k, v = ((torch.randn(2, 1, 2, 64, generator=g) * 1.15 ** t).to(torch.bfloat16) for _ in range(2))
        _append_both(pool, k, v, lens, freqs=_freqs(32))
        lens = [n + 1 for n in lens]


@pytest.mark.parametrize("T", [3, 20])
def test_append_of_extreme_values(T):
    pool = Pool(6, 1, 64, 16, 64, 6)
    k, v = _tokens(6, T, 1, 64, 7), _tokens(6, T, 1, 64, 8)
    k[0, 1, 0, 3], v[0, 0, 0, 5], v[0, 1, 0, 6] = math.nan, math.inf, -math.inf
    k[1], v[1] = 0, 0
    k[2], v[2] = k[2] * 2.0 ** -120, v[2] * 2.0 ** -126
    k[3], v[3] = k[3] * 2.0 ** 120, v[3] * 2.0 ** 124
    k[4], v[4] = 448 * 2.0 ** 3, 450
    v[5] = math.nan
    _append_both(pool, k, v, [0, 5, 9, 15, 1, 0])


@pytest.mark.parametrize("inter", [False, True])
def test_rotation_at_far_positions(inter):
    """Positions up to 2^31: no page stands there, the rotated queries and keys come all the same."""
    import paper_2510_26692_amd as kda
    pool = Pool(4, 1, 128, 16, 64, 2)
    lens = [2 ** 31 - 5, 10 ** 9, 10 ** 6 + 1, 77]
    k, v, q = (_tokens(4, 2, 1, 128, i) for i in range(3))
    kd, vd, ksd, vsd, td = pool.device()
    f = _freqs(64)
    q_out, k_out = kda.kda_cache_append(k.cuda(), v.cuda(), kd, vd, ksd, vsd, td, torch.tensor(lens, dtype=torch.int32, device="cuda"),
                                        inv_freq=torch.from_numpy(f).cuda(), interleaved=inter, q=q.cuda(), want_k=True)
    for got, x in ((q_out, q), (k_out, k)):
        exact = np.stack([sa.rotate(_np(x[n]), lens[n] + np.arange(2), f, inter) for n in range(4)])
        # (at 2^31 an angle held in 64 bits is good to 2^-20 of a turn: 6e-6)
        off = np.abs(_np(got) - exact) - (HALF * np.abs(exact) + 2.0 ** -16 * np.abs(_np(x)).max(-1, keepdims=True))
        assert (off <= 0).all()


def _attend(pool, q, lens, window=0, sinks=0, out_dtype=torch.float32, **kw):
    import paper_2510_26692_amd as kda
    kd, vd, ksd, vsd, td = pool.device()
    o = Guarded(q.shape, out_dtype, fill=7)
    kda.kda_cache_attn(q.cuda(), kd, vd, ksd, vsd, td, torch.tensor(lens, dtype=torch.int32, device="cuda"), window=window, sinks=sinks, o=o.tensor, **kw)
    o.assert_untouched("o")
    return o.tensor


def _check_attend(pool, q, lens, window=0, sinks=0, out_dtype=torch.float32, scale=None, **kw):
    o = _attend(pool, q, lens, window, sinks, out_dtype, scale=scale, **kw)
    ref, bound = sa.cache_attention(_np(q), pool.k, pool.v, pool.ks, pool.vs, pool.table, lens, window, sinks, scale)
    got = _np(o)
    assert np.isfinite(got).all()
    off = np.abs(got - ref) - (TERMS * bound * (1 + HALF) + (HALF if out_dtype == torch.bfloat16 else 2.0 ** -20) * np.abs(ref) + 1e-30)
    assert (off <= 0).all(), "%g beyond its bound at %s" % (off.max(), np.unravel_index(off.argmax(), off.shape))
    return o


@pytest.mark.parametrize("out_dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("Tq,Hq,Hk,d,page,lens,window,sinks", [
    (1, 1, 1, 128, 64, [0, 1, 2, 16, 17, 63], 0, 0), (1, 4, 1, 64, 16, [31, 32, 33, 64, 65, 15], 0, 0), (1, 8, 2, 128, 128, [127, 128, 129, 500, 1000, 1], 0, 0),
    (8, 16, 2, 128, 32, [8, 9, 3, 40, 100, 0], 0, 0), (4, 8, 1, 64, 64, [4, 300, 70, 64, 66, 1], 0, 0), (3, 5, 1, 128, 16, [200, 3, 50, 16, 18, 2], 0, 0),
    (8, 32, 2, 64, 32, [600, 8, 33, 31, 5, 64], 0, 0), (8, 24, 1, 128, 64, [300, 90, 8, 7, 64, 200], 0, 0), (1, 4, 2, 128, 64, [700, 64, 33, 10, 1, 0], 20, 4),
    (5, 4, 2, 64, 16, [700, 64, 33, 10, 6, 5], 17, 40), (2, 8, 1, 128, 128, [900, 130, 100, 65, 64, 63], 64, 64), (8, 16, 1, 64, 32, [500, 40, 12, 8, 4, 300], 1, 0),
    (4, 8, 4, 128, 16, [777, 400, 34, 30, 33, 12], 33, 1), (1, 10, 2, 64, 64, [5000, 3000, 100, 1, 4999, 2500], 0, 0),
    (2, 6, 2, 128, 16, [4100, 2000, 1000, 3, 4097, 64], 2000, 5)])
def test_attend(Tq, Hq, Hk, d, page, lens, window, sinks, out_dtype):
    pool = Pool(len(lens), Hk, d, page, max(lens) + 40, Tq + Hq, nan_behind=lens)
    _check_attend(pool, _tokens(len(lens), Tq, Hq, d, 5), lens, window, sinks, out_dtype)


@pytest.mark.parametrize("d,Hq,window,sinks", [(128, 4, 0, 0), (64, 3, 20000, 7)])
def test_attend_parts_of_long_sequences_joined_by_several_waves(d, Hq, window, sinks):
    """Few heads and many keys: more parts than one wave joins, in sequences that fill them, some of them, one or none."""
    lens = [33000, 9000, 12, 0]
    pool = Pool(4, 1, d, 64, 33040, 71, nan_behind=lens)
    q = _tokens(4, 2, Hq, d, 72)
    clean = _check_attend(pool, q, lens, window, sinks)
    pool.k[pool.table[0, 32000 // 64], 0, 32000 % 64, 1] = 0xFF
    got = _attend(pool, q, lens, window, sinks)
    assert not bool(torch.isfinite(got[0]).any()) and torch.equal(got[1:], clean[1:])


def test_attend_lengths_of_nothing_give_zeros():
    pool = Pool(4, 2, 128, 64, 200, 1)
    o = _attend(pool, _tokens(4, 3, 4, 128, 1), [0, -5, -(2 ** 31), 1])
    assert not bool(o[:3].any()) and not bool(o[3, :2].any()) and bool(o[3, 2].any())


def test_attend_longer_than_the_table_and_missing_pages():
    pool = Pool(4, 2, 64, 16, 96, 3)
    pool.table[1, 2] = -1
    pool.table[2, :] = pool.P
    pool.table[3, 0] = 2 ** 30
    for lens in ([96, 90, 80, 70], [100, 96, 96, 2 ** 31 - 1][:3] + [96]):
        for window, sinks in ((0, 0), (20, 4)):
            _check_attend(pool, _tokens(4, 4, 4, 64, 2), lens, window, sinks)


def test_attend_any_scales_and_any_split():
    pool = Pool(3, 2, 128, 64, 3000, 8)
    g = np.random.default_rng(1)
    pool.ks, pool.vs = (np.exp(g.uniform(-6, -3, pool.ks.shape)).astype(np.float32) for _ in range(2))
    lens, q = [3000, 1234, 17], _tokens(3, 2, 8, 128, 9)
    outs = [_check_attend(pool, q, lens, max_kv_len=m, scale=0.05) for m in (0, 3000, 500, 64, 1)]
    # (the split regroups sums of the same rounded terms: 2^-8 where a running maximum differs, as the bound allows)
    assert torch.equal(outs[0], outs[1])


@pytest.mark.parametrize("d,Hq", [(64, 2), (128, 2), (128, 40), (64, 40)])
def test_attend_codes_that_are_not_numbers_reach_the_rows_that_see_them(d, Hq):
    lens = [500, 40]
    q = _tokens(2, 8, Hq, d, 3)
    for window, sinks in ((0, 0), (30, 2)):
        for which, at in (("v", 496), ("v", 466), ("k", 495), ("v", 1), ("k", 0)):
            pool = Pool(2, 1, d, 16, 540, 5, nan_behind=lens)
            clean = _attend(pool, q, lens, window, sinks)
            x = pool.k if which == "k" else pool.v
            x[pool.table[0, at // 16], 0, at % 16, d - 3] = 0xFF
            got = _attend(pool, q, lens, window, sinks)
            sees = sa.visible(500 - 8 + np.arange(8), [at], window, sinks)[:, 0]
            bad = ~torch.isfinite(got).all(-1).all(-1).cpu().numpy()
            assert bad[0].tolist() == sees.tolist() and not bad[1].any(), (which, at, window)
            rest = torch.from_numpy(~sees).cuda()
            assert torch.equal(got[0, rest], clean[0, rest]) and torch.equal(got[1], clean[1])


def test_attend_slices_and_a_workspace_of_the_exact_size():
    import ctypes

    import paper_2510_26692_amd as kda
    pool = Pool(2, 2, 128, 64, 2000, 4)
    lens = torch.tensor([2000, 1500], dtype=torch.int32, device="cuda")
    qkv = _tokens(2, 3, 12, 128, 6).cuda()
    q = qkv[:, :, 2:10]
    dev = pool.device()
    kd, vd, ksd, vsd, td = dev
    cache = kda.attn._cache(kd, vd, ksd, vsd, td, lens, 8, 2, 128, 2)
    need = int(kda.load_library().kda_cache_attn_workspace_size(ctypes.byref(cache), ctypes.byref(kda.KdaCacheQuery(tokens=3, scale=0.1, out_dtype=0))))
    ws = Guarded((need,), torch.uint8)
    assert need > 0
    a = kda.kda_cache_attn(q, kd, vd, ksd, vsd, td, lens, scale=0.1, workspace=ws.tensor)
    ws.assert_untouched("workspace")
    b = kda.kda_cache_attn(q.contiguous(), kd, vd, ksd, vsd, td, lens, scale=0.1)
    assert torch.equal(a, b)
    k, v, qa = qkv[:, :, :2], qkv[:, :, 4:6], qkv[:, :, 6:10]
    f = torch.from_numpy(_freqs(64)).cuda()
    lens0 = torch.tensor([1000, 33], dtype=torch.int32, device="cuda")
    outs = []
    for args in ((k, v, qa), (k.contiguous(), v.contiguous(), qa.contiguous())):
        c = [t.clone() for t in dev]
        q_out, k_out = kda.kda_cache_append(args[0], args[1], *c[:4], td, lens0, inv_freq=f, q=args[2], want_k=True)
        outs.append([q_out, k_out] + [t.view(torch.uint8) for t in c[:2]] + c[2:4])
    assert all(torch.equal(x, y) for x, y in zip(*outs))


def test_cache_of_more_than_2_31_bytes():
    import paper_2510_26692_amd as kda
    P, page, d = 140000, 128, 128
    kc, vc = (torch.zeros(P, 1, page, d, dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn) for _ in range(2))
    assert kc.numel() > 1 << 31
    ks, vs = (torch.ones(P, 1, device="cuda") for _ in range(2))
    table = torch.tensor([[P - 1, 0, P - 2]], dtype=torch.int32, device="cuda")
    k, v, q = (_tokens(1, 300, 1, d, i) for i in range(3))
    lens0 = torch.zeros(1, dtype=torch.int32, device="cuda")
    kda.kda_cache_append(k.cuda(), v.cuda(), kc, vc, ks, vs, table, lens0)
    pick = lambda t: t.view(torch.uint8)[[P - 1, 0, P - 2]].cpu().numpy() if t.dim() == 4 else t[[P - 1, 0, P - 2]].cpu().numpy()
    small = [np.zeros((3, 1, page, d), np.uint8) for _ in range(2)] + [np.ones((3, 1), np.float32) for _ in range(2)]
    sa.append(_np(k).astype(np.float32), _np(v).astype(np.float32), *small, np.array([[0, 1, 2]]), [0])
    for got, want in zip((kc, vc, ks, vs), small):
        np.testing.assert_array_equal(pick(got), want)
    o = kda.kda_cache_attn(q[:, -2:].cuda(), kc, vc, ks, vs, table, lens0 + 300)
    ref, bound = sa.cache_attention(_np(q[:, -2:]), *small, np.array([[0, 1, 2]]), [300])
    assert (np.abs(_np(o) - ref) <= TERMS * bound * (1 + HALF) + 2.0 ** -20 * np.abs(ref)).all()


def test_append_and_attend_replayed_from_a_graph():
    import paper_2510_26692_amd as kda
    pool = Pool(3, 2, 128, 64, 1200, 12)
    kd, vd, ksd, vsd, td = pool.device()
    lens = torch.tensor([1000, 63, 500], dtype=torch.int32, device="cuda")
    f = torch.from_numpy(_freqs(64)).cuda()
    k, v, q = (torch.zeros(3, 1, h, 128, dtype=torch.bfloat16, device="cuda") for h in (2, 2, 8))

    def step(c, n):
        q_out, _ = kda.kda_cache_append(k, v, *c, td, n, inv_freq=f, q=q)
        n.add_(1)
        return kda.kda_cache_attn(q_out, *c, td, n)

    caches = [[t.clone() for t in (kd, vd, ksd, vsd)] for _ in range(2)]
    lengths = [lens.clone() for _ in range(2)]
    step([t.clone() for t in caches[0]], lens.clone())       # first use outside the capture
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        o = step(caches[0], lengths[0])
    for rep in range(5):
        for t, i in ((k, 0), (v, 1), (q, 2)):
            t.copy_(_tokens(3, 1, t.shape[2], 128, 10 * rep + i))
        want = step(caches[1], lengths[1])                   # eager work of the program between the replays
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(o, want) and torch.equal(lengths[0], lengths[1])
        assert all(torch.equal(x.view(torch.uint8) if x.dim() == 4 else x, y.view(torch.uint8) if y.dim() == 4 else y) for x, y in zip(*caches))
