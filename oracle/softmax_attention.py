"""fp64 oracle of the softmax-attention layers: the definitions, one sequence and head at a time, with every score in memory.

Independent of the kernels: numpy only, no tiling, no running statistics.  Next to each result stands what a rounding of the
softmax's terms can do to it (``*_bound``), from which the tests' tolerances follow.
"""
import numpy as np


def visible(queries, keys, window, sinks):
    """[q, k] truth values: key positions that query positions see."""
    i, j = np.asarray(queries)[:, None], np.asarray(keys)[None, :]
    ok = j <= i
    return ok & ((i - j < window) | (j < sinks)) if window else ok


def _rows(batch, tokens, cu):
    return [(b, 0, tokens) for b in range(batch)] if cu is None else [(0, int(a), int(e)) for a, e in zip(cu[:-1], cu[1:])]


def softmax_rows(x, seen):
    """exp(x - lse) over the seen entries of each row, and lse; rows that see nothing: zeros and -inf."""
    x = np.where(seen, x, -np.inf)
    m = x.max(1, keepdims=True)
    m = np.where(np.isfinite(m), m, 0.0)
    p = np.exp(x - m)
    z = p.sum(1, keepdims=True)
    with np.errstate(divide="ignore"):
        return p / np.where(z > 0, z, 1.0), (m + np.log(z))[:, 0]


def attention(q, k, v, window=0, sinks=0, cu=None, scale=None):
    """q [B,T,Hq,d], k, v [B,T,Hk,d] in fp64.  Returns a dict: o, lse [B,Hq,T], and o_bound = sum_j P_ij |v_j|."""
    B, T, Hq, d = q.shape
    G = Hq // k.shape[2]
    scale = d ** -0.5 if scale is None else scale
    out = {"o": np.zeros(q.shape), "lse": np.zeros((B, Hq, T)), "o_bound": np.zeros(q.shape)}
    for b, s, e in _rows(B, T, cu):
        seen = visible(np.arange(e - s), np.arange(e - s), window, sinks)
        for h in range(Hq):
            if e == s:
                continue
            p, lse = softmax_rows(scale * q[b, s:e, h] @ k[b, s:e, h // G].T, seen)
            out["o"][b, s:e, h], out["lse"][b, h, s:e] = p @ v[b, s:e, h // G], lse
            out["o_bound"][b, s:e, h] = p @ np.abs(v[b, s:e, h // G])
    return out


def attention_backward(q, k, v, do, window=0, sinks=0, cu=None, scale=None, rounding=2.0 ** -8):
    """Gradients of sum(o . do).  Returns dq, dk, dv and bounds on their errors where the terms P and dS are rounded by `rounding`
    relative before the products with do, k and q, and o before the row sums do . o:

        |err dV_j|  <= r sum_i P_ij |do_i|
        |err dS_ij| <= P_ij (r |do_i . v_j - d_i| + |err d_i|),   |err d_i| <= r sum_c |do_ic| (|o_ic| + sum_j P_ij |v_jc|)
        |err dQ_i|  <= scale sum_j |err dS_ij| |k_j|,             dK alike
    """
    B, T, Hq, d = q.shape
    G = Hq // k.shape[2]
    scale = d ** -0.5 if scale is None else scale
    r = rounding
    out = {n: np.zeros(x.shape) for n, x in (("dq", q), ("dk", k), ("dv", v), ("dq_bound", q), ("dk_bound", k), ("dv_bound", v))}
    for b, s, e in _rows(B, T, cu):
        seen = visible(np.arange(e - s), np.arange(e - s), window, sinks)
        for h in range(Hq):
            if e == s:
                continue
            Q, K, V, D = q[b, s:e, h], k[b, s:e, h // G], v[b, s:e, h // G], do[b, s:e, h]
            p, _ = softmax_rows(scale * Q @ K.T, seen)
            o = p @ V
            delta = (D * o).sum(1, keepdims=True)
            dp = D @ V.T
            ds = p * (dp - delta)
            err_delta = r * (np.abs(D) * (np.abs(o) + p @ np.abs(V))).sum(1, keepdims=True)
            err = p * (r * np.abs(dp - delta) + err_delta)
            out["dq"][b, s:e, h] = scale * ds @ K
            out["dk"][b, s:e, h // G] += scale * ds.T @ Q
            out["dv"][b, s:e, h // G] += p.T @ D
            out["dq_bound"][b, s:e, h] = scale * err @ np.abs(K)
            out["dk_bound"][b, s:e, h // G] += scale * err.T @ np.abs(Q)
            out["dv_bound"][b, s:e, h // G] += r * p.T @ np.abs(D)
    return out


def rotate(x, positions, inv_freq, interleaved=False):
    """x [T,H,d] turned at positions [T]; exact to fp64 (positions * inv_freq are formed in the longer type numpy has)."""
    x = np.asarray(x, dtype=np.float64).copy()
    n = len(inv_freq)
    angle = np.asarray(positions, dtype=np.longdouble)[:, None] * np.asarray(inv_freq, dtype=np.longdouble)[None, :]
    c, s = (f(angle).astype(np.float64)[:, None, :] for f in (np.cos, np.sin))
    ia, ib = (np.arange(0, 2 * n, 2), np.arange(1, 2 * n, 2)) if interleaved else (np.arange(n), np.arange(n, 2 * n))
    a, b = x[..., ia].copy(), x[..., ib].copy()
    x[..., ia], x[..., ib] = a * c - b * s, a * s + b * c
    return x


def _e4m3_values():
    codes = np.arange(256)
    e, m = (codes >> 3) & 15, codes & 7
    mag = np.where(e == 0, m * 2.0 ** -9, (1 + m / 8.0) * 2.0 ** (e - 7.0))
    mag = np.where((codes & 127) == 127, np.nan, mag)
    return np.where(codes & 128, -mag, mag)


E4M3 = _e4m3_values()


def e4m3_encode(x):
    """Codes of x, to nearest, ties to the even code; NaN (and anything beyond 464) becomes the NaN code of its sign."""
    x = np.asarray(x, dtype=np.float64)
    mag = E4M3[:127]
    a = np.abs(x)
    hi = np.clip(np.searchsorted(mag, np.nan_to_num(a, nan=0.0)), 1, 126)
    lo = hi - 1
    dl, dh = a - mag[lo], mag[hi] - a
    code = np.where((dl < dh) | ((dl == dh) & (lo % 2 == 0)), lo, hi)
    code = np.where(~(a <= 464), 127, code)
    return (code | np.where(np.signbit(x), 128, 0)).astype(np.uint8)


def scale_for(top):
    """The smallest power of two s >= 2^-100 with top <= 448 s."""
    s = 2.0 ** -100
    while top > 448 * s:
        s *= 2
    return s


def append(k, v, k_cache, v_cache, k_scale, v_scale, table, lens, cu=None):
    """New (already rotated) keys and values into the cache of codes, in place; k, v fp32-rounded values [N,T,Hk,d] or packed [1,T,Hk,d]."""
    P, H, page, _ = k_cache.shape
    for n, (b, s, e) in enumerate(_rows(k.shape[0], k.shape[1], cu)):
        if lens[n] < 0:
            continue
        for first in range(int(lens[n]), int(lens[n]) + e - s):
            if first != lens[n] and first % page:
                continue                                     # (once a page)
            p, a = first // page, first % page
            count = min(page - a, int(lens[n]) + e - s - first)
            if p >= table.shape[1] or not 0 <= table[n, p] < P:
                continue
            at, row = table[n, p], s + first - int(lens[n])
            for x, cache, scale in ((k, k_cache, k_scale), (v, v_cache, v_scale)):
                for h in range(H):
                    y = x[b, row:row + count, h].astype(np.float64)
                    finite = np.abs(y[np.isfinite(y)])
                    new = scale_for(finite.max() if finite.size else 0.0)
                    if a:
                        new = max(new, float(scale[at, h]))
                        if new > scale[at, h]:
                            cache[at, h, :a] = e4m3_encode(E4M3[cache[at, h, :a]] * (float(scale[at, h]) / new))
                    cache[at, h, a:a + count] = e4m3_encode(y / new)
                    scale[at, h] = new


def cache_attention(q, k_cache, v_cache, k_scale, v_scale, table, lens, window=0, sinks=0, scale=None):
    """q [N,Tq,Hq,d] over codes; returns o and o_bound = sum_j P_ij |v_j|."""
    N, Tq, Hq, d = q.shape
    P, Hk, page, _ = k_cache.shape
    scale = d ** -0.5 if scale is None else scale
    o, bound = np.zeros(q.shape), np.zeros(q.shape)
    for n in range(N):
        keys = [j for j in range(max(0, min(int(lens[n]), table.shape[1] * page))) if 0 <= table[n, j // page] < P]
        if not keys:
            continue
        at, off = np.array([table[n, j // page] for j in keys]), np.array(keys) % page
        seen = visible(int(lens[n]) - Tq + np.arange(Tq), keys, window, sinks)
        for h in range(Hq):
            g = h // (Hq // Hk)
            k = E4M3[k_cache[at, g, off]] * k_scale[at, g].astype(np.float64)[:, None]
            v = E4M3[v_cache[at, g, off]] * v_scale[at, g].astype(np.float64)[:, None]
            p, _ = softmax_rows(scale * q[n, :, h] @ k.T, seen)
            o[n, :, h], bound[n, :, h] = p @ v, p @ np.abs(v)
    return o, bound
