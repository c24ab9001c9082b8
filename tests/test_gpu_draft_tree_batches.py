"""Sequences of a batch in other places, among others and alone, and decays that are infinite or the same for all channels, over draft trees."""
import math

import numpy as np
import pytest
import torch

from oracle import draft_trees as dt
from test_gpu_cache import Pool, _tokens
from test_gpu_draft_trees import STEPS, _attend, _attend_refs, _check_steps, _inputs, _within, int32, random_trees

pytestmark = pytest.mark.gpu


def _rows(pool, n):
    """The same pool with some of its sequences, in that order."""
    some = Pool.__new__(Pool)
    some.__dict__.update(pool.__dict__, table=np.ascontiguousarray(pool.table[n]))
    return some


@pytest.mark.parametrize("d,N,Hk", [(64, 70, 8), (128, 33, 16), (128, 200, 3)])
@pytest.mark.parametrize("window,sinks", [(0, 0), (100, 4)])
@pytest.mark.parametrize("out_dtype", [torch.float32, torch.bfloat16])
def test_a_sequence_s_place_in_the_batch_changes_nothing(d, N, Hk, window, sinks, out_dtype):
    """More sequences and heads than a round of workgroups, none of them split: ranked by length, whatever their order in the batch, bit for bit; a sequence
    by itself, which is split, within the attention's rounding."""
    T, most = 24, 700
    pool = Pool(N, Hk, d, 16, most, 3)
    lens = np.random.default_rng(1).integers(0, most - T + 1, N)
    lens[7], lens[30] = -1, 0
    lens[[3, 11, 12]] = lens[4]                              # (of one length: ranked by their places)
    q, parents = _tokens(N, T, 2 * Hk, d, 3), random_trees(N, T, 4, 1, 10)
    call = lambda n: _attend(_rows(pool, n), q[torch.from_numpy(n)], lens[n], parents[n], window, sinks, out_dtype, max_kv_len=most)
    as_they_are = np.arange(N)
    got = call(as_they_are)
    assert torch.equal(got, call(as_they_are))
    for order in (as_they_are[::-1].copy(), np.random.default_rng(2).permutation(N), np.argsort(lens, kind="stable")):
        assert torch.equal(got[torch.from_numpy(order).cuda()], call(order))
    some = np.array([0, 3, 7, 30, int(np.argmax(lens))])
    ref = _attend_refs(_rows(pool, some), q[torch.from_numpy(some)], lens[some], parents[some], window, sinks)
    _within(got[torch.from_numpy(some).cuda()], *ref, out_dtype)
    for i, n in enumerate(some):
        _within(call(some[i:i + 1]), ref[0][i:i + 1], ref[1][i:i + 1], out_dtype)


@pytest.mark.parametrize("T,d,dtype", [(16, 128, torch.bfloat16), (40, 64, torch.float32), (64, 128, torch.float32), (64, 128, torch.bfloat16)])
@pytest.mark.parametrize("scalar", [False, True])
def test_a_decay_that_is_infinite_reaches_a_token_and_its_descendants(T, d, dtype, scalar):
    """log alpha of plus infinity: what the recurrence makes of it is not finite, in the token's row and its descendants'; no other row changes."""
    import paper_2510_26692_amd as kda
    x = list(_inputs(1, T, 2, d, dtype, T))
    if scalar:
        x[3] = x[3][..., 0].contiguous()
    S = (torch.randn(1, 2, d, d, generator=torch.Generator().manual_seed(2)) * 0.3).cuda()
    parents = random_trees(1, T, 3, T)
    line = dt.lines(parents[0])
    bad = next(t for t in range(T) if 1 < sum(t in y for y in line) < T - 2)
    run = lambda: kda.kda_tree_steps(*(y.cuda() for y in x), S, int32(parents), scale=0.1, scalar_gate=scalar).cpu()
    want = run()
    if scalar:
        x[3][0, bad, 1] = math.inf
    else:
        x[3][0, bad, 1, 5] = math.inf
    got = run()
    odd = torch.zeros(1, T, 2, d, dtype=torch.bool)
    odd[0, [t for t in range(T) if bad in line[t]], 1] = True
    assert torch.equal(got[~odd], want[~odd])
    assert not bool(torch.isfinite(got[odd]).any())


@pytest.mark.parametrize("N,T,H,d,dtype,spread,fewest", STEPS)
@pytest.mark.parametrize("out_dtype", [torch.float32, torch.bfloat16])
def test_tree_steps_with_one_decay_a_head(N, T, H, d, dtype, spread, fewest, out_dtype):
    import paper_2510_26692_amd as kda
    q, k, v, la, beta = _inputs(N, T, H, d, dtype, T + d)
    la = la[..., 0].contiguous()
    S = torch.randn(N + 2, H, d, d, generator=torch.Generator().manual_seed(2)) * 0.3
    parents = random_trees(N, T, spread, T, fewest, roots=True)
    idx = torch.arange(N + 1, 1, -1, dtype=torch.int32)
    Sd = S.cuda()
    o = kda.kda_tree_steps(*(x.cuda() for x in (q, k, v, la, beta)), Sd, int32(parents), state_indices=idx.cuda(), scale=d ** -0.5, out_dtype=out_dtype,
                           scalar_gate=True)
    assert o.dtype == out_dtype and torch.equal(Sd.cpu(), S)
    _check_steps(q, k, v, la, beta, S, idx, parents, d ** -0.5, out_dtype, o, True)
