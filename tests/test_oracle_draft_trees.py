"""Pins of the fp64 oracle of draft trees and pages (oracle/draft_trees.py) against other definitions of the same things (CPU)."""
import numpy as np
import pytest

import oracle
from oracle import draft_trees as dt
from oracle import softmax_attention as sa


def test_lines():
    assert dt.lines([-1, 0, 0, 2, -1, 4]) == [[0], [0, 1], [0, 2], [0, 2, 3], [4], [4, 5]]
    assert dt.lines([-2, 0, -1, 1, 3, 9, 6]) == [[], [], [2], [], [], [], []]            # no token, and what follows it


def test_a_chain_is_causal_attention():
    g = np.random.default_rng(1)
    T, held = 6, 11
    q, k, v = g.standard_normal((T, 4, 8)), g.standard_normal((held + T, 2, 8)), g.standard_normal((held + T, 2, 8))
    full = np.concatenate([np.zeros((held, 4, 8)), q])
    for window, sinks in ((0, 0), (5, 2), (1, 0)):
        o, _ = dt.tree_attention(q, k, v, np.arange(-1, T - 1), held, window, sinks)
        want = sa.attention(full[None], k[None], v[None], window, sinks)["o"][0, held:]
        np.testing.assert_allclose(o, want, atol=1e-12)


def test_a_path_of_a_tree_is_that_path_alone():
    g = np.random.default_rng(2)
    held, parents = 5, [-1, 0, 0, 1, 2, 3]
    q, k, v = g.standard_normal((6, 2, 4)), g.standard_normal((11, 1, 4)), g.standard_normal((11, 1, 4))
    o, _ = dt.tree_attention(q, k, v, parents, held, 4, 1)
    path = [0, 1, 3, 5]
    keys = list(range(held)) + [held + t for t in path]
    alone, _ = dt.tree_attention(q[path], k[keys], v[keys], [-1, 0, 1, 2], held, 4, 1)
    np.testing.assert_allclose(o[path], alone, atol=1e-12)


def test_kda_over_a_tree_and_its_path_are_the_recurrence():
    g = np.random.default_rng(3)
    T, H, d = 5, 2, 64
    q, k, v = (g.standard_normal((T, H, d)) / 8 for _ in range(3))
    la, beta, S = -0.3 * g.random((T, H, d)), g.random((T, H)), g.standard_normal((H, d, d))
    path = [0, 2, 4]
    o, _ = dt.tree_steps(q, k, v, np.exp(la), beta, S, [-1, 0, 0, 1, 2], 0.5)
    state = S[None]
    for t in path:
        o1, state = oracle.kda_step(*(x[t][None].astype(np.float64) for x in (q, k, v, la, beta)), state, scale=0.5)
        np.testing.assert_allclose(o[t], o1[0], atol=1e-6)
    np.testing.assert_allclose(dt.commit(k, v, np.exp(la), beta, S, path + [-1]), state[0], atol=1e-6)
    np.testing.assert_allclose(dt.commit(k, v, np.exp(la), beta, S, [0, 2, 2, 4]), dt.commit(k, v, np.exp(la), beta, S, [0, 2]))


def test_written_out_form_of_the_tree_recurrence():
    """The form the kernel computes, u and o from the state before the tree, is the recurrence from state to state."""
    g = np.random.default_rng(4)
    T, d = 7, 64
    parents = [-1, 0, 0, 1, -1, 4, 2]
    q, k, v, a = (g.standard_normal((T, d)) / 8 for _ in range(4))
    a, beta, S = np.exp(-np.abs(a)), g.random(T), g.standard_normal((d, d))
    line = dt.lines(parents)
    u = np.zeros((T, d))
    for i in range(T):
        between = lambda j: np.prod([a[x] for x in line[i][line[i].index(j) + 1:]], axis=0) if j != i else np.ones(d)
        all_of = np.prod([a[x] for x in line[i]], axis=0)
        u[i] = beta[i] * (v[i] - (all_of * k[i]) @ S - sum((k[i] * between(j)) @ k[j] * u[j] for j in line[i][:-1]))
        o = (all_of * q[i]) @ S + sum((q[i] * between(j)) @ k[j] * u[j] for j in line[i])
        want, _ = dt.tree_steps(q[:, None], k[:, None], v[:, None], a[:, None], beta[:, None], S[None], parents, 1.0)
        np.testing.assert_allclose(o, want[i, 0], atol=1e-12)


def test_keep_moves_tokens_and_the_largest_scale_wins():
    g = np.random.default_rng(5)
    table, page = np.array([[2, 0, 1]]), 16
    cache = sa.e4m3_encode(g.standard_normal((3, 1, page, 8)) * 60)
    scale = np.float32([[0.5], [0.25], [1.0]])
    cache[2], scale[2] = cache[2], np.float32(0.125)
    before = [sa.E4M3[cache[table[0, t // page], 0, t % page]] * scale[table[0, t // page], 0] for t in range(48)]
    held, kept = 14, [0, 5, 20, 33]
    after, s = cache.copy(), scale.copy()
    dt.keep(after, s, table, [held], [kept + [-1]])
    assert s[2, 0] == 0.5 and s[0, 0] == 0.25 + 0.25 * (held + 20 < 32) or s[0, 0] in (0.25, 0.5)
    for i, t in enumerate(list(range(held)) + [held + x for x in kept]):
        at = i
        p = table[0, at // page]
        got = sa.E4M3[after[p, 0, at % page]] * s[p, 0]
        np.testing.assert_allclose(got, before[t], atol=2.0 ** -4 * np.abs(before[t]).max() + 2.0 ** -10 * s[p, 0])


def test_pages():
    table = np.array([[0, 1, 2, -1], [0, 3, -1, -1], [4, -1, -1, -1]], np.int32)
    refs = dt.count(table, 10)
    assert refs.tolist() == [2, 1, 1, 1, 1, 0, 0, 0, 0, 0]
    dt.fork(table, refs, [1, 1, -1])
    assert table.tolist() == [[0, 3, -1, -1], [0, 3, -1, -1], [-1] * 4] and refs.tolist() == [2, 0, 0, 2, 0, 0, 0, 0, 0, 0]
    copies, missing = dt.reserve(table, [20, 32, -1], [40, 33, 50], refs, 16)
    assert missing == 0 and copies.tolist() == [[3, 1], [-1, -1], [-1, -1]]
    assert table.tolist() == [[0, 1, 2, -1], [0, 3, 4, -1], [-1] * 4] and refs.tolist() == [2, 1, 1, 1, 1, 0, 0, 0, 0, 0]
    table[table == 1], refs[1], refs[8] = 8, 0, 1
    moves = dt.compact(table, refs)
    assert moves[:2].tolist() == [[8, 1], [-1, -1]] and table.tolist() == [[0, 1, 2, -1], [0, 3, 4, -1], [-1] * 4]
    assert refs.tolist() == dt.count(table, 10).tolist()
    full = np.array([[0, 0]], np.int32)
    refs = dt.count(full, 2)
    assert dt.reserve(full, [0], [32], refs, 16)[1] == 1 and full.tolist() == [[0, 0]] and refs.tolist() == [2, 0]


@pytest.mark.parametrize("kept,length", [([], 0), ([-1, 3], 0), ([3], 1), ([3, 2], 1), ([0, 1, 64], 3)])
def test_paths_end_where_they_do_not_rise(kept, length):
    table = np.arange(10)[None]
    g = np.random.default_rng(6)
    cache, scale = sa.e4m3_encode(g.standard_normal((10, 1, 16, 4)) * 60), np.ones((10, 1), np.float32)
    after = cache.copy()
    dt.keep(after, scale, table, [16], [kept + [-1]])
    for i in range(5):
        src = 16 + kept[i] if i < length else 16 + i
        assert np.array_equal(after[(16 + i) // 16, 0, (16 + i) % 16], cache[src // 16, 0, src % 16])
