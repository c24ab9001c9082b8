"""Pages that sequences share: whole numbers, equal to the oracle's."""
import numpy as np
import pytest
import torch

from oracle import draft_trees as dt

pytestmark = pytest.mark.gpu


def int32(x):
    return torch.tensor(np.asarray(x), dtype=torch.int32, device="cuda")


def _table(N, columns, P, seed, fill=0.7, shared=0.3):
    """A table whose rows hold some pages of their own and some of earlier rows, with entries that are no page, and its counts."""
    g = np.random.default_rng(seed)
    order, at = g.permutation(P), 0
    table = np.full((N, columns), -1, np.int64)
    for n in range(N):
        for c in range(int(columns * fill) if columns > 2 else columns):
            if n and g.random() < shared:
                table[n, c] = table[int(g.integers(0, n)), c]
            elif at < 0.8 * P and g.random() < 0.9:
                table[n, c] = order[at]
                at += 1
            else:
                table[n, c] = g.choice([-1, -5, P, 2 ** 31 - 1])
    return table.astype(np.int32), dt.count(table, P)


@pytest.mark.parametrize("N,columns,P", [(1, 1, 1), (5, 17, 60), (64, 3, 200), (200, 33, 5000), (8192, 2, 20000), (3, 1000, 900), (7, 16, 50)])
def test_fork(N, columns, P):
    import paper_2510_26692_amd as kda
    table, refs = _table(N, columns, P, N)
    g = np.random.default_rng(N + 1)
    for kind in range(3):
        source = [np.arange(N), g.integers(-1, N, N), np.where(g.random(N) < 0.5, g.integers(0, N, N), g.choice([N, N + 3, 2 ** 31 - 1, -9], N))][kind]
        td, rd = int32(table), int32(refs)
        assert kda.kda_pages_fork(td, rd, int32(source)) is None
        dt.fork(table, refs, source)
        assert np.array_equal(td.cpu().numpy(), table) and np.array_equal(rd.cpu().numpy(), refs)
        assert np.array_equal(refs, dt.count(table, P))


def test_fork_frees_everything():
    import paper_2510_26692_amd as kda
    table, refs = _table(9, 20, 100, 3)
    td, rd = int32(table), int32(refs)
    kda.kda_pages_fork(td, rd, int32([-1] * 9))
    assert bool((td == -1).all()) and not bool(rd.any())


@pytest.mark.parametrize("N,columns,P,page", [(1, 4, 6, 16), (6, 17, 90, 64), (128, 20, 4000, 32), (1500, 5, 20000, 128), (2, 3000, 40000, 16), (40, 40, 1700, 16),
                                              (8192, 3, 40000, 64)])
def test_reserve(N, columns, P, page):
    import paper_2510_26692_amd as kda
    g = np.random.default_rng(N)
    for kind in range(3):
        table, refs = _table(N, columns, P, 10 * N + kind, fill=0.5)
        lens = g.integers(0, columns * page * 3 // 4 + 1, N)
        after = lens + [g.integers(0, 3, N), g.integers(0, page * 3, N), g.integers(-5, columns * page, N)][kind]
        if kind == 1 and N > 3:
            lens[0], after[1], after[2] = -1, -3, 2 ** 31 - 1
        want_t, want_r = table.copy(), refs.copy()
        want_c, want_m = dt.reserve(want_t, lens, after, want_r, page)
        td, rd = int32(table), int32(refs)
        copies, missing = kda.kda_pages_reserve(td, int32(lens), int32(after), rd, page)
        assert int(missing) == want_m and np.array_equal(copies.cpu().numpy(), want_c)
        assert np.array_equal(td.cpu().numpy(), want_t) and np.array_equal(rd.cpu().numpy(), want_r)
        if want_m == 0:
            assert np.array_equal(want_r, dt.count(want_t, P)) or (refs != dt.count(table, P)).any()


def test_reserve_with_too_few_pages_changes_nothing():
    import paper_2510_26692_amd as kda
    table = np.array([[0, 1, -1, -1], [0, 2, -1, -1]], np.int32)
    refs = dt.count(table, 5)
    td, rd = int32(table), int32(refs)
    copies, missing = kda.kda_pages_reserve(td, int32([20, 20]), int32([60, 40]), rd, 16)          # 2 and 1 pages, two are free
    assert int(missing) == 1 and bool((copies == -1).all()) and np.array_equal(td.cpu().numpy(), table) and np.array_equal(rd.cpu().numpy(), refs)
    copies, missing = kda.kda_pages_reserve(td, int32([20, 20]), int32([48, 40]), rd, 16)
    assert int(missing) == 0 and td.tolist() == [[0, 1, 3, -1], [0, 2, 4, -1]] and rd.tolist() == [2, 1, 1, 1, 1]


@pytest.mark.parametrize("P,N,columns,used", [(1, 1, 1, 0.5), (2, 1, 2, 0.5), (17, 3, 4, 0.5), (100, 5, 20, 0.3), (5000, 64, 60, 0.5), (16385, 20, 500, 0.5), (40000, 100, 300, 0.9),
                                              (33000, 10, 100, 0.02), (64, 4, 16, 1.0), (64, 4, 16, 0.0)])
def test_compact(P, N, columns, used):
    import paper_2510_26692_amd as kda
    g = np.random.default_rng(P)
    pages = g.permutation(P)[:min(round(P * used), N * columns)]
    table = np.full((N, columns), -1, np.int64)
    table.reshape(-1)[g.permutation(N * columns)[:len(pages)]] = pages
    if N > 2 and columns > 1:
        table[1, 0] = table[0, 0]
        table[2, 1] = P + 3                                  # (no page, and not counted)
    refs = dt.count(table, P)
    td, rd = int32(table), int32(refs)
    moves = kda.kda_pages_compact(td, rd)
    want = dt.compact(table, refs)
    assert np.array_equal(moves.cpu().numpy(), want) and np.array_equal(td.cpu().numpy(), table) and np.array_equal(rd.cpu().numpy(), refs)
    n = int((refs > 0).sum())
    assert bool((rd[:n] > 0).all()) and not bool(rd[n:].any())
    assert bool((kda.kda_pages_compact(td, rd) == -1).all()) and np.array_equal(td.cpu().numpy(), table)


@pytest.mark.parametrize("L,P,Hk,page,d", [(1, 9, 2, 64, 128), (3, 20, 1, 16, 64), (2, 7, 8, 128, 128), (2, 12, 5, 32, 64)])
def test_copy_pages(L, P, Hk, page, d):
    import paper_2510_26692_amd as kda
    g = torch.Generator().manual_seed(P)
    codes = [torch.randint(0, 256, (L, P, Hk, page, d), dtype=torch.uint8, generator=g) for _ in range(2)]
    scales = [torch.rand(L, P, Hk, generator=g) for _ in range(2)]
    pairs = [[0, 3], [-1, -1], [1, 4], [P, 2], [1, P], [0, 5], [5, -1], [2 ** 31 - 1, 0], [6, 6]]
    dev = [x.cuda().view(torch.float8_e4m3fn) for x in codes] + [x.cuda() for x in scales]
    one = L == 1                                             # (a layer of its own, without the dimension of layers)
    assert kda.kda_cache_copy_pages(*((x[0] if one else x) for x in dev), int32(pairs)) is None
    for x in codes + scales:
        for a, b in ((0, 3), (1, 4), (0, 5)):
            x[:, b] = x[:, a]
    assert all(torch.equal(a.view(torch.uint8).cpu() if a.dtype == torch.float8_e4m3fn else a.cpu(), b) for a, b in zip(dev, codes + scales))
    kda.kda_cache_copy_pages(*dev, int32(np.zeros((0, 2))))


def test_a_step_of_beam_search():
    """Beams are doubled and dropped, the new token's page becomes each one's own, and what every beam holds is what it held."""
    import paper_2510_26692_amd as kda
    from test_gpu_cache import _tokens
    N, Hk, d, page, P, L = 6, 2, 64, 16, 60, 2
    g = torch.Generator().manual_seed(1)
    caches = [torch.zeros(L, P, Hk, page, d, dtype=torch.uint8).cuda().view(torch.float8_e4m3fn) for _ in range(2)] + [torch.ones(L, P, Hk).cuda() for _ in range(2)]
    table, refs = torch.full((N, 8), -1, dtype=torch.int32).cuda(), torch.zeros(P, dtype=torch.int32).cuda()
    lens = int32([0] * N)
    held = [[] for _ in range(N)]                            # what each beam should hold: its tokens' values
    rng = np.random.default_rng(5)
    for turn in range(40):
        source = rng.integers(0, 3, N) + np.array([0, 0, 0, 3, 3, 3])
        kda.kda_pages_fork(table, refs, int32(source))
        held = [list(held[s]) for s in source]
        copies, missing = kda.kda_pages_reserve(table, lens, lens + 1, refs, page)
        kda.kda_cache_copy_pages(*caches, copies)
        assert int(missing) == 0
        k = _tokens(N, 1, Hk, d, turn).cuda()
        for layer in range(L):
            kda.kda_cache_append(k, k + layer, *(x[layer] for x in caches), table, lens)
        lens += 1
        for n in range(N):
            held[n].append(k[n, 0].float())
        t = table.cpu().numpy()
        assert np.array_equal(refs.cpu().numpy(), dt.count(t, P))
        if turn % 13 == 12:                                  # (and the pool is made dense now and then)
            moves = kda.kda_pages_compact(table, refs)
            kda.kda_cache_copy_pages(*caches, moves)
            n = int((refs > 0).sum())
            assert not bool(refs[n:].any())
    for n in range(N):
        for i, want in enumerate(held[n]):
            p = int(table[n, i // page])
            got = caches[0].float()[0, p, :, i % page] * caches[2][0, p][:, None]
            # (rounded to e4m3 at most five times, as often as its page's scale can have grown)
            assert bool(((got - want).abs() <= 5 * (2.0 ** -4 * want.abs() + 2.0 ** -10 * caches[2][0, p][:, None])).all()), (n, i)


def test_captured_page_calls_replay():
    import paper_2510_26692_amd as kda
    N, columns, P, page = 12, 30, 700, 16
    make = lambda seed: _table(N, columns, P, seed, fill=0.5)
    t0, r0 = make(1)
    table, refs, source, lens = int32(t0), int32(r0), int32(np.arange(N)), int32(np.full(N, 100))

    def run(table, refs):
        kda.kda_pages_fork(table, refs, source)
        c, m = kda.kda_pages_reserve(table, lens, lens + 40, refs, page)
        return c, m, kda.kda_pages_compact(table, refs)

    run(int32(t0), int32(r0))
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = run(table, refs)
    for seed in (2, 3, 4):
        t, r = make(seed)
        table.copy_(int32(t)), refs.copy_(int32(r)), source.copy_(int32(np.random.default_rng(seed).integers(-1, N, N)))
        want_t, want_r = int32(t), int32(r)
        want = run(want_t, want_r)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip((*out, table, refs), (*want, want_t, want_r)))
