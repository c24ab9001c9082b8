"""Rotation by positions of several axes against the fp64 oracle, its inverse and its gradient.

An angle's sine and cosine are off by at most 2^-23 (fp32 rounding of an angle up to pi / 4, and of the result), and by 2 pi 2^-51 of the revolutions
that were taken off; the two products and their sum are rounded to fp32, so with a and b the pair's values a result is off by less than
(|a| + |b|) (2^-22 + 2^-48 turns), and a bf16 one by half a step (2^-8) more."""
import numpy as np
import pytest
import torch

from oracle import softmax_attention as sa
from test_gpu_cache import HALF, _freqs, _np

pytestmark = pytest.mark.gpu


def _exact(x, positions, freqs, axes, inter, inverse):
    """x [B,T,H,d] in fp64; positions [A,B,T]."""
    out = x.copy()
    n = len(freqs)
    for b in range(x.shape[0]):
        for t in range(x.shape[1]):
            # (each frequency turned by its own axis: the oracle's rotation at position 1, by position times frequency)
            angle = np.array([np.longdouble(positions[axes[i], b, t]) * np.longdouble(freqs[i]) for i in range(n)])
            out[b, t] = sa.rotate(x[b, t][None], np.ones(1), -angle if inverse else angle, inter)[0]
    return out


def _bound(x, positions, freqs, n, inter, dtype, ref):
    a = np.abs(x)
    other = a.copy()
    if inter:
        other[..., 0:2 * n:2], other[..., 1:2 * n:2] = a[..., 1:2 * n:2], a[..., 0:2 * n:2]
    else:
        other[..., :n], other[..., n:2 * n] = a[..., n:2 * n], a[..., :n]
    other[..., 2 * n:] = 0
    turns = np.abs(positions.astype(np.float64)).max() * (np.abs(freqs).max() if n else 0)
    tol = (a + other) * (2.0 ** -22 + 2.0 ** -48 * turns)
    return tol + (HALF * (np.abs(ref) + tol) if dtype == torch.bfloat16 else 0)


CASES = [  # B, T, Hq, Hk, d, n, axes, interleaved, dtype
    (1, 1, 1, 1, 128, 64, 1, False, torch.bfloat16), (2, 37, 8, 2, 128, 64, 3, False, torch.bfloat16), (2, 37, 8, 2, 128, 64, 3, True, torch.bfloat16),
    (1, 300, 5, 1, 64, 32, 2, False, torch.float32), (3, 65, 7, 3, 64, 16, 4, True, torch.float32), (1, 33, 33, 0, 128, 24, 2, False, torch.bfloat16),
    (2, 9, 4, 4, 128, 8, 4, False, torch.float32), (1, 70, 3, 2, 64, 8, 1, True, torch.bfloat16), (4, 16, 40, 8, 128, 64, 1, False, torch.float32),
    (1, 5, 2, 1, 128, 0, 1, False, torch.bfloat16),
]


@pytest.mark.parametrize("B,T,Hq,Hk,d,n,A,inter,dtype", CASES)
@pytest.mark.parametrize("inverse", [False, True])
def test_rotate(B, T, Hq, Hk, d, n, A, inter, dtype, inverse):
    import paper_2510_26692_amd as kda
    g = torch.Generator().manual_seed(T)
    q, k = (torch.randn(B, T, H, d, generator=g).to(dtype) for H in (Hq, max(Hk, 1)))
    positions = np.random.default_rng(T).integers(-50, 200000, (A, B, T))
    freqs, axes = _freqs(n), [(5 * i + 1) % A for i in range(n)]
    pos = torch.tensor(positions if A > 1 or T % 2 else positions[0], dtype=torch.int32).cuda()
    qo, ko = kda.kda_rotate(q.cuda(), k.cuda() if Hk else None, pos, torch.from_numpy(freqs).cuda(), axes=axes if A > 1 else None, interleaved=inter,
                            inverse=inverse)
    assert (ko is None) == (Hk == 0)
    for x, got in ((q, qo),) + (((k, ko),) if Hk else ()):
        x = _np(x)
        ref = _exact(x, positions, freqs, axes, inter, inverse)
        assert (np.abs(_np(got) - ref) <= _bound(x, positions, freqs, n, inter, dtype, ref)).all()
        assert np.array_equal(_np(got)[..., 2 * n:], x[..., 2 * n:])


def test_rotate_far_positions():
    import paper_2510_26692_amd as kda
    x = torch.randn(1, 4, 2, 128, generator=torch.Generator().manual_seed(1))
    positions = np.array([[[2 ** 31 - 1, -2 ** 31, 2 ** 30 + 7, 123456789]]])
    freqs = _freqs(64)
    got, _ = kda.kda_rotate(x.cuda(), None, torch.tensor(positions, dtype=torch.int32).cuda(), torch.from_numpy(freqs).cuda())
    ref = _exact(_np(x), positions, freqs, [0] * 64, False, False)
    assert (np.abs(_np(got) - ref) <= _bound(_np(x), positions, freqs, 64, False, torch.float32, ref)).all()


def test_rotate_in_place_spaced_tokens_and_given_outputs():
    import paper_2510_26692_amd as kda
    fused = torch.randn(2, 50, 12 * 128, generator=torch.Generator().manual_seed(1)).to(torch.bfloat16).cuda()
    q, k = fused[..., :8 * 128].view(2, 50, 8, 128), fused[..., 8 * 128:10 * 128].view(2, 50, 2, 128)
    pos = torch.randint(0, 1000, (2, 50), dtype=torch.int32, generator=torch.Generator().manual_seed(2)).cuda()
    f = torch.from_numpy(_freqs(32)).cuda()
    want = kda.kda_rotate(q.contiguous(), k.contiguous(), pos, f)
    before = fused.clone()
    got = kda.kda_rotate(q, k, pos, f)
    assert all(torch.equal(a, b) for a, b in zip(got, want)) and torch.equal(fused, before)
    for inter in (False, True):
        qi, ki = q.contiguous(), k.contiguous()
        want = kda.kda_rotate(qi, ki, pos, f, interleaved=inter)
        out = kda.kda_rotate(qi, ki, pos, f, interleaved=inter, q_out=qi, k_out=ki)
        assert out[0] is qi and out[1] is ki and torch.equal(qi, want[0]) and torch.equal(ki, want[1])
    with pytest.raises(kda.KdaError):
        kda.kda_rotate(qi, qi, pos, f, q_out=qi)             # (what is read as k is written as q)


def test_rotate_what_is_not_finite_stays_in_its_pair():
    import paper_2510_26692_amd as kda
    x = torch.randn(1, 3, 2, 64, generator=torch.Generator().manual_seed(1)).cuda()
    pos = torch.tensor([[3, 4, 5]], dtype=torch.int32).cuda()
    f = torch.from_numpy(_freqs(32)).cuda()
    want, _ = kda.kda_rotate(x, None, pos, f)
    x[0, 1, 1, 7], x[0, 2, 0, 33] = float("nan"), float("inf")
    got, _ = kda.kda_rotate(x, None, pos, f)
    odd = torch.zeros_like(got, dtype=torch.bool)
    odd[0, 1, 1, [7, 39]] = odd[0, 2, 0, [1, 33]] = True
    assert not bool(torch.isfinite(got[odd]).any()) and torch.equal(got[~odd], want[~odd])


def test_rotate_gradient_is_the_inverse():
    """<g, R x> = <R^T g, x>, and the difference of the outputs along a direction, which is linear."""
    import paper_2510_26692_amd as kda
    gen = torch.Generator().manual_seed(3)
    x, g, e = (torch.randn(2, 40, 4, 128, generator=gen).cuda() for _ in range(3))
    pos = torch.randint(0, 5000, (3, 2, 40), dtype=torch.int32, generator=gen).cuda()
    f, axes = torch.from_numpy(_freqs(48)).cuda(), [i % 3 for i in range(48)]
    turn = lambda y, inverse=False: kda.kda_rotate(y, None, pos, f, axes=axes, inverse=inverse)[0].double()
    dx = turn(g, True)
    slope = ((turn(x + e) - turn(x - e)) * g.double()).sum() / 2
    exact = (dx * e.double()).sum()
    # (every one of the 2 40 4 128 products is off by a few 2^-22 of its factors)
    assert abs(float(slope - exact)) <= 2.0 ** -20 * float((g.double().abs() * (x.double().abs() + e.double().abs()) * 4).sum())
    back = turn(turn(x).float(), True)
    assert float((back - x.double()).abs().max()) <= 2.0 ** -20 * 8


def test_rotate_captured_beside_an_eager_graph():
    import paper_2510_26692_amd as kda
    x = torch.randn(2, 30, 4, 128, device="cuda").to(torch.bfloat16)
    pos = torch.arange(60, dtype=torch.int32, device="cuda").view(2, 30)
    f = torch.from_numpy(_freqs(64)).cuda()
    kda.kda_rotate(x, x, pos, f)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        a, _ = kda.kda_rotate(x, x, pos, f)
        b, _ = kda.kda_rotate(a, a, pos, f, inverse=True)
    for i in range(3):
        x.copy_(torch.randn(2, 30, 4, 128, device="cuda"))
        pos.add_(17)
        graph.replay()
        want, _ = kda.kda_rotate(x, x, pos, f)
        back, _ = kda.kda_rotate(want, want, pos, f, inverse=True)
        torch.cuda.synchronize()
        assert torch.equal(a, want) and torch.equal(b, back)
