"""Pins of the softmax-attention oracle (CPU): closed forms, finite differences, and torch's own e4m3 conversion."""
import numpy as np
import pytest
import torch

from oracle import softmax_attention as sa


def _inputs(B, T, Hq, Hk, d, seed=0):
    g = np.random.default_rng(seed)
    return tuple(g.standard_normal((B, T, h, d)) for h in (Hq, Hk, Hk, Hq))


def test_visible_keys_by_hand():
    seen = sa.visible(np.arange(6), np.arange(6), 2, 1)
    assert seen.astype(int).tolist() == [[1, 0, 0, 0, 0, 0], [1, 1, 0, 0, 0, 0], [1, 1, 1, 0, 0, 0], [1, 0, 1, 1, 0, 0], [1, 0, 0, 1, 1, 0],
                                         [1, 0, 0, 0, 1, 1]]
    assert sa.visible([3], np.arange(6), 0, 0).astype(int).tolist() == [[1, 1, 1, 1, 0, 0]]
    assert not sa.visible([-1], np.arange(6), 0, 0).any()


def test_equal_scores_average_the_visible_values():
    q, k, v, _ = _inputs(1, 9, 2, 1, 4)
    out = sa.attention(0 * q, k, v, window=3, sinks=1)
    for i in range(9):
        keys = [j for j in range(i + 1) if i - j < 3 or j < 1]
        np.testing.assert_allclose(out["o"][0, i, 1], v[0, keys, 0].mean(0), atol=1e-14)
        np.testing.assert_allclose(out["lse"][0, 1, i], np.log(len(keys)), atol=1e-14)


@pytest.mark.parametrize("window,sinks,cu", [(0, 0, None), (3, 2, None), (2, 0, [0, 4, 4, 7])])
def test_gradients_are_those_of_differences(window, sinks, cu):
    B = 2 if cu is None else 1
    q, k, v, do = _inputs(B, 7, 4, 2, 3, 1)
    kw = dict(window=window, sinks=sinks, cu=cu, scale=0.7)
    got = sa.attention_backward(q, k, v, do, **kw)
    g = np.random.default_rng(2)
    for name, x in (("dq", q), ("dk", k), ("dv", v)):
        for _ in range(6):
            at = tuple(g.integers(0, n) for n in x.shape)
            keep, e = x[at], 1e-5
            x[at] = keep + e
            up = (sa.attention(q, k, v, **kw)["o"] * do).sum()
            x[at] = keep - e
            down = (sa.attention(q, k, v, **kw)["o"] * do).sum()
            x[at] = keep
            assert abs((up - down) / (2 * e) - got[name][at]) < 1e-8


def test_rotation_is_one_of_pairs_and_relative():
    g = np.random.default_rng(3)
    x, y = g.standard_normal((2, 5, 2, 8))
    f = np.float32([1.0, 0.1, 0.01])
    for inter in (False, True):
        p = np.arange(5)
        a, b = sa.rotate(x, p, f, inter), sa.rotate(y, p, f, inter)
        c, d = sa.rotate(x, p + 1000, f, inter), sa.rotate(y, p + 1000, f, inter)
        np.testing.assert_allclose((a ** 2).sum(-1), (x ** 2).sum(-1))
        np.testing.assert_allclose(np.einsum("thc,shc->tsh", a, b), np.einsum("thc,shc->tsh", c, d), atol=1e-9)
        np.testing.assert_array_equal(a[..., 6:], x[..., 6:])
        np.testing.assert_array_equal(a[0], x[0])


def test_codes_are_those_of_torch():
    g = np.random.default_rng(4)
    x = np.concatenate([g.standard_normal(20000) * 10.0 ** g.integers(-4, 3, 20000), np.arange(-2 ** 12, 2 ** 12) * 2.0 ** -11, [0.0, -0.0, 448, 464, -464, 2.0 ** -10,
                                                                                                       3 * 2.0 ** -10]]).astype(np.float32)
    x = x[np.abs(x) <= 464]
    want = torch.from_numpy(x).to(torch.float8_e4m3fn)
    got = sa.e4m3_encode(x)
    np.testing.assert_array_equal(got, want.view(torch.uint8).numpy())
    np.testing.assert_array_equal(sa.E4M3[got], want.double().numpy())
    assert sa.e4m3_encode(np.array([np.nan, np.inf, -np.inf])).tolist() == [127, 127, 255]


def test_append_keeps_scales_and_rounds_again_only_where_they_grow():
    k = np.zeros((1, 1, 1, 64))
    kc, vc = np.zeros((2, 1, 16, 64), np.uint8), np.zeros((2, 1, 16, 64), np.uint8)
    ks, vs = np.ones((2, 1), np.float32), np.ones((2, 1), np.float32)
    table = np.array([[1]])
    k[0, 0, 0, 0] = 448.0
    sa.append(k, k, kc, vc, ks, vs, table, [0])
    assert ks[1, 0] == 1.0 and sa.E4M3[kc[1, 0, 0, 0]] == 448 and ks[0, 0] == 1.0
    k[0, 0, 0, 0] = 3.0
    sa.append(k, k, kc, vc, ks, vs, table, [1])
    assert ks[1, 0] == 1.0 and sa.E4M3[kc[1, 0, 1, 0]] == 3
    k[0, 0, 0, 0] = 449.0
    sa.append(k, k, kc, vc, ks, vs, table, [2])
    assert ks[1, 0] == 2.0 and [float(sa.E4M3[c]) for c in kc[1, 0, :3, 0]] == [224, 1.5, 224]
    assert vs[1, 0] == 2.0 and not kc[0].any()
