"""KDA over draft trees where sums of finite inputs leave fp32's range: a row is what steps from state to state give, and no row is changed or lost for
another's sake.

Bound of a row, whatever the size of its keys.  Let M be the state that the recurrence has with every factor and term replaced by its absolute value,
M <- alpha M + beta |k| (|v| + |k|^T alpha M).  Every way of summing the recurrence's terms, from state to state or unrolled, adds up the same monomials, each of
which is in M's; a token's step puts less than 2 (d + 16) roundings of 2^-24 on a monomial, and 2^-22 (1 + |log alpha|) for its decay.  Products with the
state in larger trees leave out less than 2^-21 of a term.  So o is off by less than
scale |q|^T M ((depth + 1) (2 (d + 16) 2^-24 + 2^-22 (1 + max |log alpha|)) + 2^-21)."""
import math

import numpy as np
import pytest
import torch

from oracle import draft_trees as dt
from test_gpu_cache import HALF, _np
from test_gpu_draft_trees import _check_steps, _delta_tol, _inputs, int32, random_trees

pytestmark = pytest.mark.gpu

KINDS = [(8, 64, torch.float32), (16, 128, torch.bfloat16), (16, 128, torch.float32), (16, 64, torch.bfloat16), (20, 128, torch.bfloat16), (32, 64, torch.float32),
         (33, 64, torch.bfloat16), (48, 128, torch.float32), (64, 128, torch.bfloat16), (64, 64, torch.float32)]


def _steps(x, S, parents, scale=1.0, **kw):
    import paper_2510_26692_amd as kda
    return kda.kda_tree_steps(*(y.cuda() for y in x), S.cuda(), int32(parents), scale=scale, **kw)


def _exact(x, S, parents, scale, n, h):
    """Rows of one sequence and head in fp64, their bounds, and the largest number that steps from state to state meet on the way to each."""
    q, k, v, la, beta = (_np(y[n, :, h]) for y in x)
    la = np.broadcast_to(la[:, None], k.shape) if la.ndim == 1 else la
    T, d = k.shape
    o, tol, size = np.zeros(v.shape), np.zeros(v.shape), np.zeros(T)
    states, most, sizes = {-1: _np(S[n, h])}, {-1: np.abs(_np(S[n, h]))}, {-1: 0.0}
    for t, line in enumerate(dt.lines(parents[n])):
        if not line:
            continue
        up, a = int(parents[n][t]), np.exp(la[t])
        states[t] = dt.step(states[up], k[t], v[t], a, beta[t])
        m = most[up] * a[:, None]
        most[t] = m + np.abs(beta[t]) * np.outer(np.abs(k[t]), np.abs(v[t]) + np.abs(k[t]) @ m)
        s = np.abs(states[up]) * a[:, None]
        sizes[t] = max(sizes[up], s.max(), (np.abs(k[t]) @ s).max(), np.abs(states[t]).max())
        o[t] = scale * states[t].T @ q[t]
        size[t] = max(sizes[t], (np.abs(q[t]) @ np.abs(states[t])).max())
        tol[t] = abs(scale) * (np.abs(q[t]) @ most[t]) * ((len(line) + 1) * (2 * (d + 16) * 2.0 ** -24 + 2.0 ** -22 * (1 + np.abs(la).max())) + 2.0 ** -21)
    return o, tol, size


@pytest.mark.parametrize("T,d,dtype", KINDS)
@pytest.mark.parametrize("scalar", [False, True])
def test_products_of_keys_and_queries_beyond_fp32(T, d, dtype, scalar):
    """q . k = d 2^124 leaves fp32 ahead of u and the scale, which bring it back: powers of two, so exact.  Every third token has such vectors and follows the
    root; the others, ordinary ones, are as they are without them."""
    x = list(_inputs(2, T, 2, d, dtype, T))
    large = torch.arange(T) % 3 == 1
    parents = np.full((2, T), -1)
    for t in range(2, T):
        if not large[t]:
            parents[:, t] = t - 1 if not large[t - 1] else t - 2
    S = torch.zeros(2, 2, d, d)
    if scalar:
        x[3] = x[3][..., 0].contiguous()
    other = np.where(large.numpy()[None], -2, parents)
    want = _steps(x, S, other, 2.0 ** -7, scalar_gate=scalar)
    for i in (0, 1):
        x[i][0, large, 1] = 2.0 ** 62
    x[2][0, large, 1] = 2.0 ** (-40 - torch.arange(d) % 5).to(dtype)
    x[3][0, large, 1] = 0
    x[4][0, large, 1] = 1
    for out_dtype in (torch.float32, torch.bfloat16):
        got = _steps(x, S, parents, 2.0 ** -7, scalar_gate=scalar, out_dtype=out_dtype).cpu()
        exact = (2.0 ** (124 - 7 - 40) * d * 2.0 ** -(torch.arange(d) % 5).double())
        assert torch.equal(got[0, large, 1].double(), exact.expand(int(large.sum()), d))
        assert torch.equal(got[:, ~large], want.to(out_dtype).cpu()[:, ~large])


def test_a_correction_that_leaves_fp32():
    """Two tokens whose keys' product is 9e38: u of the second is -9e8 nevertheless, as the decode steps have it."""
    import paper_2510_26692_amd as kda
    d = 128
    x = [torch.zeros(1, 2, 1, d) for _ in range(4)] + [torch.ones(1, 2, 1)]
    x[0][..., 7], x[1][..., 7], x[2][..., 9] = 1.0, 3e19, 1e-30
    S = torch.zeros(1, 1, d, d)
    parents = np.array([[-1, 0]])
    got = _steps(x, S, parents).cpu()
    exact, tol, _ = _exact(x, S, parents, 1.0, 0, 0)
    assert abs(exact[1, 9] + 2.7e28) < 1e27
    assert (np.abs(_np(got[0, :, 0]) - exact) <= tol).all(), got[0, :, 0, 9]
    one = kda.kda_recurrent_steps_pooled(*(y.cuda() for y in x), S.cuda()).cpu()
    assert (np.abs(_np(one[0, :, 0]) - exact) <= tol).all()


@pytest.mark.parametrize("T,d,dtype", KINDS)
@pytest.mark.parametrize("scalar", [False, True])
def test_a_line_that_leaves_fp32_and_the_others_beside_it(T, d, dtype, scalar):
    """Every second token's key is 2^8 long in one channel, and follows the last of them: a step multiplies the state by 2^16, and the line leaves fp32 behind
    seven or eight.  Its rows are right up to there and not finite from there on, and the trees of the other tokens are right."""
    x = list(_inputs(2, T, 2, d, dtype, T + 1))
    S = torch.randn(2, 2, d, d, generator=torch.Generator().manual_seed(2)) * 0.3
    if scalar:
        x[3] = x[3][..., 0].contiguous()
    parents = np.full((2, T), -1)
    for t in range(2, T):
        parents[:, t] = t - 2
    parents[:, 5::6] = -1
    plain = parents.copy()
    want = _steps(x, S, plain, 0.1, scalar_gate=scalar).cpu()
    large = torch.arange(T) % 2 == 0
    x[1][1, large, 0] = 0
    x[1][1, large, 0, 3] = 2.0 ** 8
    x[4][1, large, 0] = 1
    got = _steps(x, S, parents, 0.1, scalar_gate=scalar).cpu()
    exact, tol, size = _exact(x, S, parents, 0.1, 1, 0)
    row = _np(got[1, :, 0])
    ended = 0
    for t in range(T):
        if not large[t] or size[t] < 2.0 ** 126:
            assert np.isfinite(row[t]).all() and (np.abs(row[t] - exact[t]) <= tol[t]).all(), (t, np.abs(row[t] - exact[t]).max(), tol[t].max())
        elif np.abs(exact[t]).min() > 2.0 ** 130:
            assert not np.isfinite(row[t]).any(), t
            ended += 1
    assert ended or T < 32
    # (the bound of unit keys is far narrower than the one of any keys)
    alone = parents.copy()
    alone[:, large.numpy()] = -2
    kept = got.clone()
    kept[:, large] = 0
    _check_steps(*[torch.nan_to_num(y) for y in x], S, None, alone, 0.1, torch.float32, kept, scalar)
    # the other heads and sequences
    assert torch.equal(got[0], want[0]) and torch.equal(got[1, :, 1], want[1, :, 1])


@pytest.mark.parametrize("T,d,dtype", KINDS)
def test_long_keys_in_a_chain_and_a_token_that_follows_the_root(T, d, dtype):
    """Keys of normal values with a standard deviation of 2: rows are finite as long as the steps are, and so is the last token's, which follows the root."""
    x = list(_inputs(1, T, 2, d, dtype, T))
    g = torch.Generator().manual_seed(T + d)
    x[1] = (torch.randn(1, T, 2, d, generator=g) * 2).to(dtype)
    x[4] = torch.ones_like(x[4])
    S = torch.randn(1, 2, d, d, generator=g) * 0.3
    parents = np.arange(-1, T - 1)[None]
    parents[0, T - 1] = -1
    got = _steps(x, S, parents, 0.1).cpu()
    for h in range(2):
        exact, tol, size = _exact(x, S, parents, 0.1, 0, h)
        row = _np(got[0, :, h])
        for t in range(T):
            if size[t] < 2.0 ** 126:
                assert np.isfinite(row[t]).all(), t
                assert (np.abs(row[t] - exact[t]) <= tol[t]).all(), t
            elif np.abs(exact[t]).min() > 2.0 ** 130:
                assert not np.isfinite(row[t]).any(), t


@pytest.mark.parametrize("T,d,dtype", KINDS)
def test_the_last_row_of_a_chain_alone(T, d, dtype):
    """The last token's query has a product with its own key beyond fp32, and none with the state: that row is worked through again, by itself."""
    x = list(_inputs(1, T, 1, d, dtype, T))
    x[2] = x[2] * 2.0 ** -10
    S = torch.randn(1, 1, d, d, generator=torch.Generator().manual_seed(2)) * 2.0 ** -10
    parents = np.arange(-1, T - 1)[None]
    want = _steps(x, S, parents, 2.0 ** -100).cpu()
    x[0][0, T - 1] = torch.copysign(torch.tensor(2.0 ** 126), x[1][0, T - 1].float()).to(dtype)
    assert float((x[0][0, T - 1].double() * x[1][0, T - 1].double()).sum()) > 2.0 ** 128
    got = _steps(x, S, parents, 2.0 ** -100).cpu()
    assert torch.equal(got[:, :-1], want[:, :-1])
    exact, _, size = _exact(x, S, parents, 2.0 ** -100, 0, 0)
    # (the bound of unit keys and queries, times the query's length)
    _, longest = dt.tree_steps(*(_np(y[0]) for y in x[:3]), np.exp(_np(x[3][0])), _np(x[4][0]), _np(S[0]), parents[0], 1.0)
    tol = _delta_tol(d, T, longest, _np(x[3]), 2.0 ** -100) * np.linalg.norm(_np(x[0][0, :, 0]), axis=1)
    assert size.max() < 2.0 ** 126 and (np.abs(_np(got[0, :, 0]) - exact) <= tol[:, None]).all()


@pytest.mark.parametrize("T,d,dtype", KINDS)
def test_a_bushy_tree_of_long_keys(T, d, dtype):
    """All of a tree's keys are long and it leaves fp32 on some lines, in one sequence of two that share a state; a bf16 result is rounded once more."""
    x = list(_inputs(2, T, 1, d, dtype, T))
    g = torch.Generator().manual_seed(T + d)
    x[1][1] = (torch.randn(T, 1, d, generator=g) * 2.0 ** 22).to(dtype)
    S = torch.randn(1, 1, d, d, generator=g) * 0.3
    parents = random_trees(2, T, 3, T, roots=True)
    both, idx = S.expand(2, 1, d, d), torch.zeros(2, dtype=torch.int32)
    for out_dtype in (torch.float32, torch.bfloat16):
        got = _steps(x, S, parents, 0.1, state_indices=idx.cuda(), out_dtype=out_dtype).cpu()
        _check_steps(*(y[:1] for y in x), S, None, parents[:1], 0.1, out_dtype, got[:1])
        exact, tol, size = _exact(x, both, parents, 0.1, 1, 0)
        row = _np(got[1, :, 0])
        for t in range(T):
            if size[t] < 2.0 ** 126:
                off = np.abs(row[t] - exact[t]) - tol[t] - (HALF * (np.abs(exact[t]) + tol[t]) if out_dtype == torch.bfloat16 else 0)
                assert np.isfinite(row[t]).all() and (off <= 0).all(), t
            elif np.abs(exact[t]).min() > 2.0 ** 130:
                assert not np.isfinite(row[t]).any(), t
    assert (size >= 2.0 ** 126).any() or T < 16


def test_a_captured_call_replays_where_lines_leave_fp32():
    """The rows that are worked through again, in a graph, with trees that need it and trees that do not in turn."""
    T, d = 64, 128
    fresh = lambda seed, size: [y.cuda() for y in _inputs(2, T, 2, d, torch.bfloat16, seed)][:1] + [
        (torch.randn(2, T, 2, d, generator=torch.Generator().manual_seed(seed)) * size).to(torch.bfloat16).cuda()] + [
        y.cuda() for y in _inputs(2, T, 2, d, torch.bfloat16, seed)][2:]
    import paper_2510_26692_amd as kda
    x, S, parents = fresh(1, 0.1), (torch.randn(2, 2, d, d, generator=torch.Generator().manual_seed(2)) * 0.3).cuda(), int32(random_trees(2, T, 3, 1))
    kda.kda_tree_steps(*x, S, parents)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        o = kda.kda_tree_steps(*x, S, parents)
    for seed, size in ((2, 4.0), (3, 0.1), (4, 2.0 ** 20), (5, 0.1)):
        for a, b in zip(x, fresh(seed, size)):
            a.copy_(b)
        graph.replay()
        torch.cuda.synchronize()
        again = kda.kda_tree_steps(*x, S, parents)
        assert torch.equal(o.view(torch.int32), again.view(torch.int32))
        assert bool(torch.isfinite(o).all()) == (size < 1), seed
