"""fp64 oracle of draft trees and of pages that sequences share: the definitions, one sequence, head and token at a time.

Independent of the kernels: numpy only.  KDA steps from state to state along the tree, where the kernel forms no token's state.
"""
import numpy as np

from .softmax_attention import E4M3, e4m3_encode, softmax_rows


def lines(parents):
    """For each token of one tree the tokens that it sees, from the root down to itself; [] where there is no such token."""
    out = []
    for t, up in enumerate(parents):
        if up == -1:
            out.append([t])
        elif 0 <= up < t and out[up]:
            out.append(out[up] + [t])
        else:
            out.append([])
    return out


def tree_mask(parents, held, window, sinks):
    """[T, held + T]: what each token sees of the sequence's own tokens and of the tree."""
    T = len(parents)
    seen = np.zeros((T, held + T), bool)
    line = lines(parents)
    for t in range(T):
        if not line[t]:
            continue
        pos = held + len(line[t]) - 1
        near = lambda p: not window or pos - p < window or p < sinks
        for j in range(held):
            seen[t, j] = near(j)
        for depth, j in enumerate(line[t]):
            seen[t, held + j] = near(held + depth)
    return seen


def tree_attention(q, k, v, parents, held, window=0, sinks=0, scale=None, there=None):
    """One sequence: q [T,Hq,d], k and v [held + T,Hk,d] in fp64; `there` [held + T]: whether a token has a page.  Returns o [T,Hq,d] and
    sum_j P_ij |v_j|."""
    T, Hq, d = q.shape
    G = Hq // k.shape[1]
    scale = d ** -0.5 if scale is None else scale
    seen = tree_mask(parents, held, window, sinks)
    if there is not None:
        seen &= np.asarray(there)[None, :]
    o, bound = np.zeros(q.shape), np.zeros(q.shape)
    for h in range(Hq):
        kh, vh = k[:, h // G], v[:, h // G]
        with np.errstate(invalid="ignore"):
            x = scale * q[:, h] @ kh.T
        p, _ = softmax_rows(np.where(seen, x, -np.inf), seen)
        for t in range(T):                                   # (what is not finite reaches those that see it alone)
            j = seen[t]
            o[t, h], bound[t, h] = p[t, j] @ vh[j], p[t, j] @ np.abs(vh[j])
    return o, bound


def keep(cache, scale, table, lens, kept):
    """Accepted tokens of one layer's keys or values move up: cache uint8 codes [P,H,page,d] and scale [P,H], in place."""
    P, H, page, _ = cache.shape
    old, old_scale = cache.copy(), scale.copy()
    at = lambda n, t: (int(table[n, t // page]) if t // page < table.shape[1] and 0 <= table[n, t // page] < P else -1, t % page)
    again = lambda codes, ratio: codes if ratio == 1 else e4m3_encode(np.float32(E4M3[codes]) * np.float32(ratio))
    for n, held in enumerate(lens):
        if held < 0:
            continue
        path = []
        for x in kept[n]:
            if x < 0 or (path and x <= path[-1]):
                break
            path.append(int(x))
        moves = [(at(n, held + x), at(n, held + i)) for i, x in enumerate(path)]
        moves = [(a, b) for a, b in moves if a[0] >= 0]
        older = held % page
        for p in sorted({b[0] for _, b in moves if b[0] >= 0}):
            for h in range(H):
                of = [old_scale[a[0], h] for a, b in moves if b[0] == p]
                own = p == at(n, held)[0] and older > 0
                new = np.float32(max(of + ([old_scale[p, h]] if own else [])))
                if own:
                    cache[p, h, :older] = again(old[p, h, :older], np.float32(old_scale[p, h]) / new)
                for a, b in moves:
                    if b[0] == p:
                        cache[p, h, b[1]] = again(old[a[0], h, a[1]], np.float32(old_scale[a[0], h]) / new)
                scale[p, h] = new


def fork(table, refs, source):
    """Rows become other rows, in place."""
    old, N = table.copy(), table.shape[0]
    for n, s in enumerate(source):
        if s != n and s < N:
            table[n] = old[s] if s >= 0 else -1
    refs[:] += count(table, len(refs)) - count(old, len(refs))


def count(table, pages):
    """Entries of the table that name each page."""
    e = table[(table >= 0) & (table < pages)]
    return np.bincount(e, minlength=pages).astype(np.int32)


def reserve(table, lens, after, refs, page):
    """Returns copies [N,2] and the pages that are missing; table and refs in place."""
    N, columns = table.shape
    P = len(refs)
    copies = np.full((N, 2), -1, np.int32)
    free = [p for p in range(P) if refs[p] == 0]
    want = []
    for n in range(N):
        if lens[n] < 0 or after[n] <= lens[n]:
            continue
        for c in range(lens[n] // page, min(columns, -(-int(after[n]) // page))):
            e = int(table[n, c])
            if not 0 <= e < P:
                want.append((n, c, -1))
            elif refs[e] > 1:
                want.append((n, c, e))
    if len(want) > len(free):
        return copies, len(want) - len(free)
    for (n, c, e), new in zip(want, free):
        table[n, c] = new
        refs[new] = 1
        if e >= 0:
            refs[e] -= 1
            if c == lens[n] // page and lens[n] % page:
                copies[n] = e, new
    return copies, 0


def compact(table, refs):
    """Returns moves [P // 2,2]; table and refs in place."""
    P = len(refs)
    used = int((refs > 0).sum())
    pairs = list(zip([p for p in range(used, P) if refs[p] > 0], [p for p in range(used) if refs[p] == 0]))
    moves = np.full((P // 2, 2), -1, np.int32)
    place = dict(pairs)
    for i, (a, b) in enumerate(pairs):
        moves[i] = a, b
        refs[b], refs[a] = refs[a], 0
    for i, e in np.ndenumerate(table):
        table[i] = place.get(int(e), e)
    return moves


def step(S, k, v, alpha, beta):
    """One token's step of one head's state [dk,dv]."""
    S = S * alpha[:, None]
    return S + beta * np.outer(k, v - S.T @ k)


def tree_steps(q, k, v, alpha, beta, S, parents, scale):
    """One sequence: q, k, alpha [T,H,dk], v [T,H,dv], beta [T,H], S [H,dk,dv].  Returns o [T,H,dv] and the largest length of a column of any
    state and of any value."""
    T, H, _ = q.shape
    o, size, line = np.zeros(v.shape), 0.0, lines(parents)
    for h in range(H):
        states = {-1: S[h]}
        for t in range(T):
            if not line[t]:
                continue
            states[t] = step(states[int(parents[t])], k[t, h], v[t, h], alpha[t, h], beta[t, h])
            o[t, h] = scale * states[t].T @ q[t, h]
            size = max(size, np.abs(v[t, h]).max())
        size = max([size] + [np.sqrt((x ** 2).sum(0)).max() for x in states.values()])
    return o, size


def commit(k, v, alpha, beta, S, kept):
    """One sequence's states [H,dk,dv] through the accepted tokens."""
    S, last = S.copy(), -1
    for t in kept:
        if t < 0 or t <= last or t >= k.shape[0]:
            break
        last = int(t)
        for h in range(S.shape[0]):
            S[h] = step(S[h], k[t, h], v[t, h], alpha[t, h], beta[t, h])
    return S
