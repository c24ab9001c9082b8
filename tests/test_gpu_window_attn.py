"""Softmax attention with a window and sinks, forward and backward, against the fp64 oracle, element by element.

Tolerances.  The softmax's terms P (and their gradients dS) are rounded to bf16 ahead of the second product, half a step at most: 2^-8
relative each.  What else is computed is fp32: a logit of up to ~40 is formed by 128 products and rounded a few times, which moves a
term by less than 2^-11 relative at the sizes used here (128 * 2^-24 * sum |q k| scale, with sum |q k| scale up to 50).  TERMS bounds
both; the oracle carries it through the sums (``*_bound``).  A result in bf16 is rounded once more, 2^-8 relative."""
import math

import numpy as np
import pytest
import torch

from helpers import Guarded
from oracle import softmax_attention as sa

pytestmark = pytest.mark.gpu

TERMS = 2.0 ** -8 + 2.0 ** -11
HALF = 2.0 ** -8
TINY = 1e-30


def _make(B, T, Hq, Hk, d, seed, q_std=1.5):
    g = torch.Generator().manual_seed(seed)
    return {n: (torch.randn(B, T, h, d, generator=g) * s).to(torch.bfloat16) for n, h, s in (("q", Hq, q_std), ("k", Hk, 1.0), ("v", Hk, 1.0), ("do", Hq, 1.0))}


def _np(t):
    return t.detach().cpu().double().numpy()


def _within(got, ref, bound, what):
    got = _np(got)
    assert np.isfinite(got).all(), what
    off = np.abs(got - ref) - bound
    assert (off <= 0).all(), "%s: %g beyond its bound of %g at %s" % (what, off.max(), bound.flat[off.argmax()], np.unravel_index(off.argmax(), off.shape))


def _check_fwd(x, o, lse, ref, out_dtype):
    _within(o, ref["o"], (TERMS * ref["o_bound"]) * (1 + HALF) + (HALF if out_dtype == torch.bfloat16 else 2.0 ** -20) * np.abs(ref["o"]) + TINY, "o")
    if lse is not None:                                     # (a logit's error, and the logarithm's)
        _within(lse, ref["lse"], 2.0 ** -11 + 2.0 ** -21 * np.abs(ref["lse"]), "lse")


SHAPES = [  # B, T, Hq, Hk, d, window, sinks
    (1, 1, 1, 1, 128, 0, 0), (1, 1, 2, 1, 64, 1, 64), (3, 2, 3, 3, 64, 0, 0), (2, 31, 4, 2, 128, 0, 0), (1, 64, 2, 2, 64, 0, 0), (1, 65, 6, 2, 128, 7, 3),
    (2, 127, 2, 1, 128, 64, 0), (1, 128, 5, 1, 64, 63, 1), (1, 129, 2, 1, 128, 65, 64), (1, 191, 1, 1, 64, 1, 0), (1, 257, 8, 1, 128, 0, 0),
    (1, 333, 4, 2, 64, 333, 5), (1, 333, 4, 2, 128, 332, 5), (1, 520, 2, 1, 128, 128, 33), (1, 700, 2, 1, 64, 17, 64), (1, 900, 2, 2, 128, 200, 4),
    (1, 1500, 4, 2, 64, 90, 2), (1, 2100, 2, 1, 128, 40, 32),
]


@pytest.mark.parametrize("out_dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("B,T,Hq,Hk,d,window,sinks", SHAPES)
def test_forward(B, T, Hq, Hk, d, window, sinks, out_dtype):
    import paper_2510_26692_amd as kda
    x = _make(B, T, Hq, Hk, d, T)
    o, lse = Guarded((B, T, Hq, d), out_dtype, fill=7), Guarded((B, Hq, T), torch.float32, fill=7)
    kda.kda_window_attn_fwd(*(x[n].cuda() for n in "qkv"), window=window, sinks=sinks, o=o.tensor, lse=lse.tensor)
    o.assert_untouched("o")
    lse.assert_untouched("lse")
    _check_fwd(x, o.tensor, lse.tensor, sa.attention(*(_np(x[n]) for n in "qkv"), window, sinks), out_dtype)


def _grads(x, window, sinks, cu=None, scale=None, guard=True):
    """o, lse and gradients on the device; gradients and the workspace (of the exact size) between guard regions."""
    import paper_2510_26692_amd as kda
    c = {n: t.cuda() for n, t in x.items()}
    cud = None if cu is None else torch.tensor(cu, dtype=torch.int32, device="cuda")
    kw = dict(window=window, sinks=sinks, cu_seqlens=cud, scale=scale)
    o, lse = kda.kda_window_attn_fwd(c["q"], c["k"], c["v"], out_dtype=torch.bfloat16, **kw)
    g = {n: Guarded(x[n[1]].shape, torch.bfloat16, fill=7) for n in ("dq", "dk", "dv")}
    from paper_2510_26692_amd.attn import _attn_dims
    ws = Guarded((kda.kda_window_attn_bwd_workspace_size(_attn_dims(c["q"], c["k"], c["v"], window, sinks, cud, scale, torch.bfloat16)),), torch.uint8)
    out = {n: t.tensor for n, t in g.items()}
    kda.kda_window_attn_bwd(c["q"], c["k"], c["v"], o, lse, c["do"], workspace=ws.tensor, out=out, **kw)
    for n, t in list(g.items()) + [("workspace", ws)]:
        t.assert_untouched(n)
    return o, lse, out


def _check_bwd(x, out, window, sinks, cu=None, rows=None, scale=None):
    ref = sa.attention_backward(*(_np(x[n]) for n in ("q", "k", "v", "do")), window, sinks, cu, scale=scale, rounding=TERMS)
    for n in ("dq", "dk", "dv"):
        s = slice(None) if rows is None else rows
        _within(out[n][:, s], ref[n][:, s], (ref[n + "_bound"] * (1 + 2 * HALF) + HALF * np.abs(ref[n]) + TINY)[:, s], n)


@pytest.mark.parametrize("B,T,Hq,Hk,d,window,sinks", SHAPES)
def test_backward(B, T, Hq, Hk, d, window, sinks):
    x = _make(B, T, Hq, Hk, d, T + 1)
    _check_bwd(x, _grads(x, window, sinks)[2], window, sinks)


@pytest.mark.parametrize("out_dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("T,window,sinks", [(261, 70, 5), (200, 33, 0), (290, 200, 64), (190, 1, 1)])
def test_forward_of_many_rows_with_a_window(T, window, sinks, out_dtype):
    """More workgroups than the device has places for: tiles of 32 keys.  A value that is not finite reaches its own row's queries alone."""
    import paper_2510_26692_amd as kda
    x = _make(48, T, 12, 3, 128, T)
    c = {n: t.cuda() for n, t in x.items()}
    call = lambda: kda.kda_window_attn_fwd(c["q"], c["k"], c["v"], window=window, sinks=sinks, out_dtype=out_dtype)
    o, lse = call()
    _check_fwd(x, o, lse, sa.attention(*(_np(x[n]) for n in "qkv"), window, sinks), out_dtype)
    c["v"][7, 130, 1, 5] = math.inf
    bad = ~torch.isfinite(call()[0]).all(-1).cpu()
    want = torch.zeros_like(bad)
    want[7, :, 4:8] = torch.from_numpy(sa.visible(np.arange(T), [130], window, sinks))
    assert torch.equal(bad, want)


def test_forward_of_many_packed_sequences_with_a_window():
    lens = np.random.default_rng(3).integers(0, 90, 120)
    cu = np.concatenate([[0], np.cumsum(lens)]).tolist()
    import paper_2510_26692_amd as kda
    x = _make(1, cu[-1], 10, 2, 128, 11)
    o, lse = kda.kda_window_attn_fwd(*(x[n].cuda() for n in "qkv"), window=20, sinks=3, cu_seqlens=torch.tensor(cu, dtype=torch.int32, device="cuda"))
    _check_fwd(x, o, lse, sa.attention(*(_np(x[n]) for n in "qkv"), 20, 3, cu), torch.float32)


PACKED = [([5, 0, 300, 128, 1, 129, 700], 3, 6, 50, 3), ([1], 0, 0, 0, 0), ([0, 0, 64], 64, 200, 20, 64), ([256, 384], 0, 0, 0, 0), ([2000, 1, 130], 1, 0, 31, 40)]


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("lens,before,behind,window,sinks", PACKED)
def test_packed_batch_leaves_rows_of_no_sequence_alone(lens, before, behind, window, sinks, d):
    import paper_2510_26692_amd as kda
    T = before + sum(lens) + behind
    cu = (before + np.concatenate([[0], np.cumsum(lens)])).tolist()
    x = _make(1, T, 4, 2, d, T)
    for n in x:                                              # what stands there is not read
        x[n][:, :before] = float("nan")
        x[n][:, cu[-1]:] = float("nan")
    o, lse, out = _grads(x, window, sinks, cu)
    rows = slice(before, cu[-1])
    z = {n: torch.nan_to_num(t) for n, t in x.items()}
    ref = sa.attention(*(_np(z[n]) for n in "qkv"), window, sinks, cu)
    ref = {n: (t[:, :, rows] if n == "lse" else t[:, rows]) for n, t in ref.items()}
    _check_fwd(x, o[:, rows], lse[:, :, rows], ref, torch.bfloat16)
    _check_bwd(z, out, window, sinks, cu, rows)
    for t, fill in [(o, 0)] + [(out[n], 7) for n in out]:    # the binding clears what it allocates; the library writes owned rows only
        assert bool((t[:, :before] == fill).all()) and bool((t[:, cu[-1]:] == fill).all())
    c = {n: t.cuda() for n, t in x.items()}
    cud = torch.tensor(cu, dtype=torch.int32, device="cuda")
    fresh = kda.kda_window_attn_bwd(c["q"], c["k"], c["v"], o, lse, c["do"], window=window, sinks=sinks, cu_seqlens=cud)
    for n in fresh:
        assert torch.equal(fresh[n][:, rows], out[n][:, rows]) and not bool(fresh[n][:, :before].any()) and not bool(fresh[n][:, cu[-1]:].any())


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("lens", [[1500, 2, 0, 64, 65, 700], [3] * 50 + [600, 63], [127, 1]], ids=["long", "many short", "short"])
def test_packed_sinks_with_a_key_head_for_every_query_head(lens, d):
    """Nothing but the sinks' later queries is summed apart from the keys' own walks: few long sequences and many short ones."""
    cu = np.concatenate([[0], np.cumsum(lens)]).tolist()
    x = _make(1, cu[-1], 3, 3, d, len(lens))
    _check_bwd(x, _grads(x, 40, 33, cu)[2], 40, 33, cu)


def test_entries_of_cu_seqlens_outside_the_batch_are_clamped():
    import paper_2510_26692_amd as kda
    x = {n: t.cuda() for n, t in _make(1, 200, 2, 1, 64, 5).items()}
    good = torch.tensor([0, 100, 200], dtype=torch.int32, device="cuda")
    bad = torch.tensor([-50, 100, 5000], dtype=torch.int32, device="cuda")
    a, b = (kda.kda_window_attn_fwd(x["q"], x["k"], x["v"], cu_seqlens=cu)[0] for cu in (good, bad))
    assert torch.equal(a, b)
    back = torch.tensor([0, 150, 90, 200], dtype=torch.int32, device="cuda")         # decreasing: that sequence is empty
    kda.kda_window_attn_fwd(x["q"], x["k"], x["v"], cu_seqlens=back)
    torch.cuda.synchronize()


@pytest.mark.parametrize("d", [64, 128])
def test_slices_of_one_projection_give_the_same_bits(d):
    import paper_2510_26692_amd as kda
    g = torch.Generator().manual_seed(3)
    qkv = torch.randn(2, 150, 4 + 2 + 2 + 1, d, generator=g).to(torch.bfloat16).cuda()
    q, k, v = qkv[:, :, :4], qkv[:, :, 4:6], qkv[:, :, 6:8]
    kw = dict(window=40, sinks=2)
    o, lse = kda.kda_window_attn_fwd(q, k, v, out_dtype=torch.bfloat16, **kw)
    oc, lc = kda.kda_window_attn_fwd(q.contiguous(), k.contiguous(), v.contiguous(), out_dtype=torch.bfloat16, **kw)
    assert torch.equal(o, oc) and torch.equal(lse, lc)
    do = torch.randn(o.shape, generator=g).to(torch.bfloat16).cuda()
    a, b = kda.kda_window_attn_bwd(q, k, v, o, lse, do, **kw), kda.kda_window_attn_bwd(q.contiguous(), k.contiguous(), v.contiguous(), o, lse, do, **kw)
    for n in a:
        assert torch.equal(a[n], b[n])


@pytest.mark.parametrize("d", [64, 128])
def test_scale_and_large_logits(d):
    """Logits of some hundreds: one term rules, nothing overflows; and a scale of 1."""
    import paper_2510_26692_amd as kda
    x = _make(1, 150, 2, 1, d, 11, q_std=0.2)
    o, lse, out = _grads(x, 0, 0, scale=1.0)
    ref = sa.attention(*(_np(x[n]) for n in "qkv"), scale=1.0)
    _check_fwd(x, o, lse, ref, torch.bfloat16)
    _check_bwd(x, out, 0, 0, scale=1.0)
    big = _make(1, 150, 2, 1, d, 12, q_std=64.0)
    o, _ = kda.kda_window_attn_fwd(*(big[n].cuda() for n in "qkv"))
    # (terms move by 2^-24 * 128 * sum |q k| scale, about 2^-4 here, and sum to one)
    r = sa.attention(*(_np(big[n]) for n in "qkv"))
    _within(o, r["o"], (2.0 ** -3) * (r["o_bound"] + np.abs(r["o"])) + TINY, "o")


def _nonfinite_rows(t):
    return (~torch.isfinite(t).all(-1).all(-1)[0]).nonzero().flatten().tolist()


@pytest.mark.parametrize("window,sinks", [(0, 0), (50, 3)])
@pytest.mark.parametrize("d", [64, 128])
def test_what_is_not_finite_reaches_those_that_see_it_and_no_others(d, window, sinks):
    import paper_2510_26692_amd as kda
    T = 420
    x = {n: t.cuda() for n, t in _make(1, T, 4, 2, d, 21).items()}
    kw = dict(window=window, sinks=sinks)

    def run(y):
        o, lse = kda.kda_window_attn_fwd(y["q"], y["k"], y["v"], out_dtype=torch.bfloat16, **kw)
        return dict(kda.kda_window_attn_bwd(y["q"], y["k"], y["v"], o, lse, y["do"], **kw), o=o)

    clean = run(x)
    sees = lambda i, j: j <= i and (window == 0 or i - j < window or j < sinks)
    for n, row, value in (("v", 200, math.inf), ("v", 1, math.nan), ("k", 210, math.nan), ("q", 300, math.inf), ("do", 250, -math.inf)):
        y = dict(x, **{n: x[n].clone()})
        y[n][0, row] = value
        got = run(y)
        if n in "kv":
            hit = {"o": {i for i in range(T) if sees(i, row)}}
            hit["dq"] = hit["o"]
        else:
            hit = {"o": {row} if n == "q" else set(), "dq": {row}}
        touched = {j for i in hit["dq"] for j in range(T) if sees(i, j)}
        for m in ("o", "dq", "dk", "dv"):
            rows = hit[m] if m in hit else touched
            if n == "v" and m == "dv":                       # (dV does not depend on v)
                rows = set()
            bad = set(_nonfinite_rows(got[m]))
            assert bad == rows, (n, row, m, sorted(bad ^ rows)[:8])
            rest = [i for i in range(T) if i not in rows]
            assert torch.equal(got[m][0, rest], clean[m][0, rest]), (n, row, m)


def test_keys_of_the_lowest_value_hide_themselves():
    """A program that masks by the type's lowest value in k: those keys' terms are zero, and a row of nothing else is finite."""
    import paper_2510_26692_amd as kda
    x = _make(1, 200, 2, 2, 64, 31)
    x["q"] = x["q"].abs()
    low = torch.finfo(torch.bfloat16).min
    x["k"][0, 50:90] = low / 2 ** 12
    o, lse = kda.kda_window_attn_fwd(*(x[n].cuda() for n in "qkv"))
    ref = sa.attention(*(_np(x[n]) for n in "qkv"))
    _check_fwd(x, o, None, ref, torch.float32)
    x["k"][0, :] = -math.inf                                 # every visible key at minus infinity: as a row that sees nothing
    o, lse = kda.kda_window_attn_fwd(*(x[n].cuda() for n in "qkv"))
    assert not bool(o.any()) and bool((lse == -math.inf).all())


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("T,window", [(1, 0), (300, 1)])
def test_a_row_of_a_single_key_has_gradients_of_v_alone(d, T, window):
    """dS = P (do . v - d) with P = 1 and d = do . v: nothing is left but the fp32 roundings of lse and of the sums over d channels, less
    than 2^-15 of sum |do v| (lse below 2^5 at 2^-24 a rounding, and d products each way), whatever o was rounded to."""
    x = _make(1, T, 4, 2, d, T + 61)
    out = _grads(x, window, 0)[2]
    n = {m: _np(t) for m, t in x.items()}
    k, v = (np.repeat(n[m], 2, 2) for m in "kv")
    ds = 2.0 ** -15 * np.abs(n["do"] * v).sum(-1, keepdims=True) / math.sqrt(d)
    assert (np.abs(_np(out["dq"])) <= ds * np.abs(k)).all()
    assert (np.abs(_np(out["dk"])) <= (ds * np.abs(n["q"])).reshape(1, T, 2, 2, d).sum(3)).all()
    pairs = n["do"].reshape(1, T, 2, 2, d)
    assert (np.abs(_np(out["dv"]) - pairs.sum(3)) <= HALF * np.abs(pairs.sum(3)) + TERMS * np.abs(pairs).sum(3)).all()


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("T,window,sinks", [(64, 0, 0), (500, 3, 0), (500, 10, 2)])
def test_rows_of_few_keys_lose_nothing_to_the_rounding_of_o(d, T, window, sinks):
    """dQ is rounded twice, in dS and at the end.  A rounding to bf16 is uniform in half a step of 2^-8, 2^-8 / sqrt(3) * sqrt(3 / (8 ln 2)) =
    1.66e-3 of the value in the mean square over an octave; two independent ones 2.35e-3.  A tenth more covers the draw (2048 rows and more).
    With d from the rounded o there would be a third."""
    x = _make(4, T, 8, 8, d, 67)
    got = _np(_grads(x, window, sinks)[2]["dq"])
    ref = sa.attention_backward(*(_np(x[n]) for n in ("q", "k", "v", "do")), window, sinks)["dq"]
    assert np.linalg.norm(got - ref) <= 2.6e-3 * np.linalg.norm(ref)


def test_the_same_call_gives_the_same_bits():
    x = _make(2, 700, 8, 2, 128, 41)
    a, b = _grads(x, 300, 4), _grads(x, 300, 4)
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1]) and all(torch.equal(a[2][n], b[2][n]) for n in a[2])


def test_two_streams_at_once_and_a_graph_replayed():
    import paper_2510_26692_amd as kda
    kw = dict(window=100, sinks=4)
    xs = [{n: t.cuda() for n, t in _make(1, 600, 4, 2, 128, 50 + i).items()} for i in range(2)]

    def step(x):
        o, lse = kda.kda_window_attn_fwd(x["q"], x["k"], x["v"], out_dtype=torch.bfloat16, **kw)
        return dict(kda.kda_window_attn_bwd(x["q"], x["k"], x["v"], o, lse, x["do"], **kw), o=o, lse=lse)

    want = [step(x) for x in xs]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in xs]
    got = []
    for x, s in zip(xs, streams):
        with torch.cuda.stream(s):
            for _ in range(3):
                y = step(x)
            got.append(y)
    torch.cuda.synchronize()
    for w, y in zip(want, got):
        assert all(torch.equal(w[n], y[n]) for n in w)
    graph = torch.cuda.CUDAGraph()
    held = {n: t.clone() for n, t in xs[0].items()}
    step(held)
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        out = step(held)
    for rep in range(4):
        fresh = _make(1, 600, 4, 2, 128, 60 + rep)
        for n in held:
            held[n].copy_(fresh[n])
        eager = step(held)                                   # eager work of the program between the replays
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(out[n], eager[n]) for n in out), rep


def test_offsets_beyond_32_bits():
    """q and o of more than 2^31 elements, and a fused projection of as many: the last tokens against the oracle."""
    import paper_2510_26692_amd as kda
    T, Hq, Hk, d, window = 132000, 128, 2, 128, 96
    g = torch.Generator(device="cuda").manual_seed(1)
    qkv = torch.empty(1, T, Hq + 2 * Hk, d, dtype=torch.bfloat16, device="cuda")
    for t in qkv[0].split(8192):
        t.copy_(torch.randn(t.shape, generator=g, device="cuda"))
    q, k, v = qkv[:, :, :Hq], qkv[:, :, Hq:Hq + Hk], qkv[:, :, Hq + Hk:]
    assert T * Hq * d > 1 << 31
    o, lse = kda.kda_window_attn_fwd(q, k, v, window=window, out_dtype=torch.bfloat16)
    do = torch.ones_like(o)
    out = kda.kda_window_attn_bwd(q, k, v, o, lse, do, window=window)
    torch.cuda.synchronize()
    n = 400                                                  # (their gradients of q need no later token)
    tail = {m: t[:, -n:].contiguous().cpu() for m, t in (("q", q[:, :, -3:]), ("k", k[:, :, -1:]), ("v", v[:, :, -1:]), ("do", do[:, :, -3:]))}
    ref = sa.attention(*(_np(tail[m]) for m in "qkv"), window)
    far = slice(window, n)                                   # tokens whose whole window is in the tail
    _check_fwd(tail, o[:, -n:, -3:][:, far], lse[:, -3:, -n:][:, :, far], {m: (t[:, :, far] if m == "lse" else t[:, far]) for m, t in ref.items()}, torch.bfloat16)
    r = sa.attention_backward(*(_np(tail[m]) for m in ("q", "k", "v", "do")), window, rounding=TERMS)
    _within(out["dq"][:, -n:, -3:][:, far], r["dq"][:, far], (r["dq_bound"] * (1 + 2 * HALF) + HALF * np.abs(r["dq"]) + TINY)[:, far], "dq")
