"""Softmax attention in the forms that large calls take: several heads of a group in one workgroup of the dK / dV walk, several heads of a
page and several query heads behind the same angles in the append.  Small sequences, but as many as bring these forms about."""
import math

import numpy as np
import pytest
import torch

from helpers import Guarded
from oracle import softmax_attention as sa
from test_gpu_cache import Pool, _append_both, _freqs, _tokens, _turned_within
from test_gpu_window_attn import HALF, TERMS, TINY, _check_bwd, _check_fwd, _grads, _make, _np, _within

pytestmark = pytest.mark.gpu


def _form(B, T, Hq, Hk, d, window, sinks, sequences):
    """(heads of a group's walk in one workgroup, what is summed apart), as the size of the workspace tells."""
    import paper_2510_26692_amd as kda
    tokens, group = B * T, Hq // Hk
    dims = kda.KdaAttnDims(batch=B, seqlen=T, heads_q=Hq, heads_kv=Hk, dim=d, num_seqs=sequences, in_dtype=1, out_dtype=1, scale=1.0, window=window, sinks=sinks)
    size = kda.kda_window_attn_bwd_workspace_size(dims)
    up = lambda n: -(-n // 256) * 256
    found = []
    for splits in (s for s in range(1, group + 1) if group % s == 0):
        tiles = max(8, (window + 128) // 64)
        sink_slots = 0 if not sinks else B * -(-T // (64 * tiles)) if B > 1 else T // (64 * tiles) + sequences
        sink = up(sink_slots * 2 * splits * Hk * 64 * d * 4)
        for kind, rows in (("direct", 0), ("first keys", sequences * 64), ("parts", tokens)):
            fits = kind == "parts" or (splits == 1 and (kind == "direct") == (not sinks))
            if fits and size == up(tokens * Hq * 8) + 2 * up(splits * rows * Hk * d * 4) + 2 * sink:
                found.append((group // splits, kind))
    assert len(found) == 1, found
    return found[0]


FORMS = [  # B, T, Hq, Hk, d, window, sinks, form
    (128, 130, 16, 4, 64, 0, 0, (4, "direct")), (64, 130, 16, 4, 128, 0, 0, (2, "parts")), (128, 200, 12, 4, 128, 40, 5, (3, "first keys")),
    (128, 50, 16, 8, 64, 20, 3, (2, "parts")), (90, 130, 12, 2, 128, 0, 0, (2, "parts")), (90, 150, 12, 2, 64, 33, 64, (2, "parts")),
    (60, 330, 16, 8, 128, 70, 0, (2, "direct")), (60, 330, 32, 8, 64, 70, 33, (4, "first keys")), (128, 129, 8, 8, 128, 1, 0, (1, "direct"))]


@pytest.mark.parametrize("B,T,Hq,Hk,d,window,sinks,form", FORMS)
def test_backward_of_several_heads_a_workgroup(B, T, Hq, Hk, d, window, sinks, form):
    assert _form(B, T, Hq, Hk, d, window, sinks, B) == form
    x = _make(B, T, Hq, Hk, d, T + 1)
    _check_bwd(x, _grads(x, window, sinks)[2], window, sinks)


@pytest.mark.parametrize("window,sinks,form", [(70, 33, (4, "first keys")), (0, 0, (4, "direct"))])
@pytest.mark.parametrize("d", [64, 128])
def test_packed_backward_of_several_heads_a_workgroup(d, window, sinks, form):
    lens = np.random.default_rng(5).integers(0, 300, 120)
    lens[7], lens[60] = 0, 1
    cu = (3 + np.concatenate([[0], np.cumsum(lens)])).tolist()
    T = cu[-1] + 4
    # (the workspace serves a row with cu_seqlens and one without; here the former is the larger)
    assert _form(1, T, 20, 5, d, window, sinks, 120) == form
    x = _make(1, T, 20, 5, d, 17)
    _check_bwd(x, _grads(x, window, sinks, cu)[2], window, sinks, cu, slice(cu[0], cu[-1]))


@pytest.mark.parametrize("d", [64, 128])
def test_what_is_not_finite_in_one_of_several_heads(d):
    """An infinity in one query head's gradient of o: the keys that its row sees, of that key head, and no others."""
    B, T, Hq, Hk, window = 128, 130, 16, 4, 40
    x = _make(B, T, Hq, Hk, d, 23)
    clean = _grads(x, window, 0)[2]
    x["do"][5, 100, 6] = math.inf
    got = _grads(x, window, 0)[2]
    sees = torch.from_numpy(sa.visible([100], np.arange(T), window, 0)[0])
    for n in ("dk", "dv"):
        bad = ~torch.isfinite(got[n]).all(-1).cpu()
        want = torch.zeros_like(bad)
        want[5, :, 1] = sees
        assert torch.equal(bad, want), n
        assert torch.equal(got[n][(~want).cuda()], clean[n][(~want).cuda()])


@pytest.mark.parametrize("N,T,Hk,Hq,d,page,inter", [
    (600, 4, 4, 8, 128, 16, False), (520, 8, 6, 6, 128, 64, True), (1100, 1, 3, 15, 64, 32, True), (520, 8, 6, 12, 64, 16, False), (5, 1700, 5, 20, 128, 64, True),
    (9, 500, 3, 3, 128, 32, False), (6, 400, 2, 10, 64, 16, False), (3, 3000, 4, 28, 64, 128, False), (3, 3000, 4, 4, 128, 128, True)])
def test_append_of_several_heads_behind_the_same_angles(N, T, Hk, Hq, d, page, inter):
    lens = np.random.default_rng(N).integers(0, 60, N).tolist()
    lens[1] = -1
    pool = Pool(N, Hk, d, page, max(lens) + T, T + d)
    k, v, q = _tokens(N, T, Hk, d, 1), _tokens(N, T, Hk, d, 2), _tokens(N, T, Hq, d, 3)
    (q_out, k_out), q_ref, k_ref = _append_both(pool, k, v, lens, freqs=_freqs(d // 2), inter=inter, q=q, want_k=True)
    held = [n for n in range(N) if lens[n] >= 0]
    _turned_within(q_out[held], q_ref[held], q[held])
    _turned_within(k_out[held], k_ref[held], k[held])
    assert not bool(q_out[1].any()) and not bool(k_out[1].any())


@pytest.mark.parametrize("d,page,Hk,Hq,inter", [(128, 128, 4, 16, True), (128, 64, 8, 32, False), (64, 128, 6, 18, False)])
def test_packed_append_of_several_heads_behind_the_same_angles(d, page, Hk, Hq, inter):
    lens_new, held = [3000, 0, 2900, 1, 3100], [7, 0, 100, 63, 64]
    cu = (5 + np.concatenate([[0], np.cumsum(lens_new)])).tolist()
    T = cu[-1] + 6
    pool = Pool(5, Hk, d, page, max(h + n for h, n in zip(held, lens_new)), T)
    k, v, q = _tokens(1, T, Hk, d, 1), _tokens(1, T, Hk, d, 2), _tokens(1, T, Hq, d, 3)
    (q_out, k_out), q_ref, k_ref = _append_both(pool, k, v, held, cu=cu, freqs=_freqs(d // 2), inter=inter, q=q, want_k=True)
    rows = slice(cu[0], cu[-1])
    _turned_within(q_out[:, rows], q_ref[:, rows], q[:, rows])
    _turned_within(k_out[:, rows], k_ref[:, rows], k[:, rows])
    for t in (q_out, k_out):
        assert not bool(t[:, :cu[0]].any()) and not bool(t[:, cu[-1]:].any())


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("T,window", [(300, 0), (600, 0), (1000, 300), (600, 200)])
def test_long_walks_lose_to_the_rounding_of_o_in_dq_alone(T, window, d):
    """Where one key rules a row, d = do . o is as large as do . v, and o's rounding in it as large as that of dS.  dK has d from the
    unrounded terms: two independent roundings, of dS and of the result, 2.35e-3 in the mean square, and a tenth for the draw.  In dQ the
    error of d stays, delta_i scale sum_j P_ij k_j, with delta_i of a rounding (1.66e-3) of each o_ic and each term P_ij:
    1.66e-3 (sum_c (do_ic o_ic)^2 + sum_j (P_ij do_i . v_j)^2)^(1/2)."""
    x = _make(1, T, 4, 4, d, 71, q_std=4.0)
    got = _grads(x, window, 0)[2]
    n = {m: _np(t)[0] for m, t in x.items()}
    ref = sa.attention_backward(*(n[m][None] for m in ("q", "k", "v", "do")), window, 0)
    dk = _np(got["dk"])
    assert np.linalg.norm(dk - ref["dk"]) <= 2.6e-3 * np.linalg.norm(ref["dk"])
    scale, extra = d ** -0.5, 0.0
    for h in range(4):
        p, _ = sa.softmax_rows(scale * n["q"][:, h] @ n["k"][:, h].T, sa.visible(np.arange(T), np.arange(T), window, 0))
        o, dp = p @ n["v"][:, h], n["do"][:, h] @ n["v"][:, h].T
        delta2 = ((n["do"][:, h] * o) ** 2).sum(1) + ((p * dp) ** 2).sum(1)
        extra += (1.66e-3 * scale) ** 2 * (delta2 * ((p @ n["k"][:, h]) ** 2).sum(1)).sum()
    dq = np.linalg.norm(_np(got["dq"]) - ref["dq"])
    assert dq <= 1.1 * math.sqrt((2.35e-3 * np.linalg.norm(ref["dq"])) ** 2 + extra)


def test_gradients_of_keys_beyond_32_bits():
    """q, o and d_o of more than 2^31 elements, slices of one projection, 64 query heads a key head: the last keys' gradients."""
    import paper_2510_26692_amd as kda
    T, Hq, Hk, d, window = 132000, 128, 2, 128, 96
    g = torch.Generator(device="cuda").manual_seed(2)
    qkv = torch.empty(1, T, Hq + 2 * Hk, d, dtype=torch.bfloat16, device="cuda")
    for t in qkv[0].split(8192):
        t.copy_(torch.randn(t.shape, generator=g, device="cuda"))
    q, k, v = qkv[:, :, :Hq], qkv[:, :, Hq:Hq + Hk], qkv[:, :, Hq + Hk:]
    assert T * Hq * d > 1 << 31
    o, lse = kda.kda_window_attn_fwd(q, k, v, window=window, out_dtype=torch.bfloat16)
    do = torch.empty_like(o)
    for t in do[0].split(8192):
        t.copy_(torch.randn(t.shape, generator=g, device="cuda"))
    out = kda.kda_window_attn_bwd(q, k, v, o, lse, do, window=window)
    torch.cuda.synchronize()
    n = 300
    tail = {m: t[:, -n:].contiguous().cpu() for m, t in (("q", q[:, :, 64:]), ("k", k[:, :, 1:]), ("v", v[:, :, 1:]), ("do", do[:, :, 64:]))}
    far = slice(window, n)                                   # keys whose queries' whole windows are in the tail
    r = sa.attention_backward(*(_np(tail[m]) for m in ("q", "k", "v", "do")), window, rounding=TERMS)
    for m in ("dk", "dv"):
        _within(out[m][:, -n:, 1:][:, far], r[m][:, far], (r[m + "_bound"] * (1 + 2 * HALF) + HALF * np.abs(r[m]) + TINY)[:, far], m)


def test_gradients_with_entries_of_cu_seqlens_outside_the_batch():
    import paper_2510_26692_amd as kda
    x = {n: t.cuda() for n, t in _make(1, 200, 4, 2, 64, 5).items()}
    outs = []
    for cu in ([0, 100, 200], [-50, 100, 5000]):
        kw = dict(cu_seqlens=torch.tensor(cu, dtype=torch.int32, device="cuda"), window=30, sinks=2)
        o, lse = kda.kda_window_attn_fwd(x["q"], x["k"], x["v"], out_dtype=torch.bfloat16, **kw)
        outs.append(dict(kda.kda_window_attn_bwd(x["q"], x["k"], x["v"], o, lse, x["do"], **kw), o=o, lse=lse))
    assert all(torch.equal(outs[0][n], outs[1][n]) for n in outs[0])


def test_decreasing_cu_seqlens_give_an_empty_sequence():
    """Tokens of one sequence alone are right whatever the entries that decrease say of others."""
    import paper_2510_26692_amd as kda
    x = _make(1, 200, 2, 1, 64, 5)
    o, lse = Guarded((1, 200, 2, 64), torch.float32, fill=7), Guarded((1, 2, 200), torch.float32, fill=7)
    kda.kda_window_attn_fwd(*(x[n].cuda() for n in "qkv"), cu_seqlens=torch.tensor([0, 150, 90, 200], dtype=torch.int32, device="cuda"), o=o.tensor, lse=lse.tensor)
    o.assert_untouched("o")
    lse.assert_untouched("lse")
    for rows, cu in ((slice(0, 90), [0, 150, 200]), (slice(150, 200), [0, 90, 200])):
        ref = sa.attention(*(_np(x[n]) for n in "qkv"), cu=cu)
        _check_fwd(x, o.tensor[:, rows], lse.tensor[:, :, rows], {n: (t[:, :, rows] if n == "lse" else t[:, rows]) for n, t in ref.items()}, torch.float32)
