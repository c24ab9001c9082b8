"""Binding of libkda's entry points for draft trees and for pages that sequences share (see include/kda.h).

Argument marshalling only, like ``kda.py``: tensors are device-memory handles, the stream is torch's current HIP stream.  Block tables,
reference counts, ``kv_lens``, ``parents`` and ``kept`` are contiguous int32 tensors on the device, and no call waits for it.
"""
import ctypes

import torch

from .attn import KdaCache, KdaCacheQuery, _cache, _device, _native, _token_stride
from .kda import KdaDims, _DTYPE_CODE, _SCALAR_GATE, _call, _check_dev, _out_dtype, _ptr, load_library


class KdaRotation(ctypes.Structure):
    """Mirror of ``kda_rotation``."""
    _fields_ = [("batch", ctypes.c_int32), ("seqlen", ctypes.c_int64), ("heads_q", ctypes.c_int32), ("heads_k", ctypes.c_int32),
                ("dim", ctypes.c_int32), ("dtype", ctypes.c_int), ("q_stride", ctypes.c_int64), ("k_stride", ctypes.c_int64),
                ("axes", ctypes.c_int32), ("num_freqs", ctypes.c_int32), ("inv_freq", ctypes.c_void_p), ("axis_of_freq", ctypes.c_char_p),
                ("interleaved", ctypes.c_int32), ("inverse", ctypes.c_int32)]


def _int32(t, shape, name):
    if t.dtype != torch.int32 or tuple(t.shape) != tuple(shape):
        raise ValueError("%s must be int32 %s" % (name, list(shape)))


def kda_rotate(q, k, positions, inv_freq, axes=None, interleaved=False, inverse=False, q_out=None, k_out=None):
    """Queries and keys turned by their positions.  q [B,T,Hq,d], k [B,T,Hk,d] or None, bf16 or fp32 (d 64 or 128; tokens may be spaced);
    positions int32 [B,T], or [A,B,T] with 1 to 4 axes; inv_freq fp32 [n], n a multiple of 8 up to d / 2; axes: for each frequency the
    axis whose position it turns by (None: the first), a sequence of numbers on the host.  Channels (i, i + n) turn together, or interleaved
    (2 i, 2 i + 1); those from 2 n on stay as they are.  inverse=True turns back, which is the rotation's gradient too: dq, dk from those of
    the outputs.  Returns (q_out, k_out or None), contiguous, of the inputs' dtype; either may be given and be the (contiguous) input itself."""
    lib = load_library()
    if axes is not None:
        axes = bytes(list(axes))            # (numbers beyond a byte are refused here, those beyond the axes by the library)
    done = _native("rotate", q, k, positions, inv_freq, axes, interleaved, inverse, q_out, k_out)
    if done is not None:
        return done
    dev = _device(q, k, positions, inv_freq, q_out, k_out)
    if q.dim() != 4 or q.dtype not in _DTYPE_CODE:
        raise ValueError("q must be bf16 or fp32 [B,T,Hq,d]")
    B, T, Hq, d = q.shape
    Hk = 0
    if k is not None:
        if k.dim() != 4 or k.dtype != q.dtype or k.shape[:2] != (B, T) or k.shape[3] != d:
            raise ValueError("k must be [B,T,Hk,d] of q's dtype")
        Hk = k.shape[2]
    elif k_out is not None:
        raise ValueError("k_out without k")
    if positions.dtype != torch.int32 or positions.dim() not in (2, 3) or tuple(positions.shape[-2:]) != (B, T) or not positions.is_contiguous():
        raise ValueError("positions must be contiguous int32 [B,T] or [axes,B,T]")
    if inv_freq.dtype != torch.float32 or inv_freq.dim() != 1 or not inv_freq.is_contiguous():
        raise ValueError("inv_freq must be contiguous fp32 [n]")
    n, A = inv_freq.numel(), positions.shape[0] if positions.dim() == 3 else 1
    if axes is not None and len(axes) != n:
        raise ValueError("axes must hold a number for each of the %d frequencies" % n)
    for t, like, name in ((q_out, q, "q_out"), (k_out, k, "k_out")):
        if t is not None and (t.dtype != like.dtype or t.shape != like.shape or not t.is_contiguous()):
            raise ValueError("%s must be contiguous, of the shape and dtype of what is turned" % name)
    if q_out is None:
        q_out = torch.empty(q.shape, dtype=q.dtype, device=dev)
    if k is not None and k_out is None:
        k_out = torch.empty(k.shape, dtype=k.dtype, device=dev)
    r = KdaRotation(batch=B, seqlen=T, heads_q=Hq, heads_k=Hk, dim=d, dtype=_DTYPE_CODE[q.dtype], q_stride=_token_stride(q, "q"),
                    k_stride=0 if k is None else _token_stride(k, "k"), axes=A, num_freqs=n, inv_freq=inv_freq.data_ptr(), axis_of_freq=axes,
                    interleaved=int(bool(interleaved)), inverse=int(bool(inverse)))
    _call(dev, lib.kda_rotate, ctypes.byref(r), _ptr(q), _ptr(k), _ptr(positions), _ptr(q_out), _ptr(k_out))
    return q_out, k_out


def kda_cache_tree_attn(q, k_cache, v_cache, k_scale, v_scale, block_table, kv_lens, parents, window=0, sinks=0, scale=None, max_kv_len=0, o=None,
                        out_dtype=None, workspace=None):
    """Attention of each sequence's draft tree over the paged cache.  q bf16 [N,Tq,Hq,d], Tq up to 64; the cache as for kda_cache_attn, but
    kv_lens int32 [N] counts what a sequence holds WITHOUT the drafted tokens (negative: skip), whose keys and values stand behind it, token
    t's at place kv_lens + t; parents int32 [N,Tq]: the token that a token follows, -1: what the sequence holds, -2: there is no such
    token.  A token sees what is held (within window and sinks, from the position kv_lens + its depth), its ancestors and itself.
    max_kv_len: upper bound of kv_lens + Tq if known.  Returns o [N,Tq,Hq,d], fp32 unless out_dtype (or the `o` passed in) is
    torch.bfloat16, which holds the softmax's terms in bf16 and is faster; rows of tokens that are not there are zero."""
    lib = load_library()
    if workspace is None:
        done = _native("tree_attend", q, k_cache, v_cache, k_scale, v_scale, block_table, kv_lens, parents, window, sinks, scale, max_kv_len, o, out_dtype)
        if done is not None:
            return done
    dev = _device(q, k_cache, v_cache, k_scale, v_scale, block_table, kv_lens, parents, o, workspace)
    if q.dim() != 4 or q.dtype != torch.bfloat16:
        raise ValueError("q must be bf16 [N,Tq,Hq,d]")
    N, Tq, Hq, d = q.shape
    if k_cache.dim() != 4:
        raise ValueError("k_cache and v_cache must be float8_e4m3fn [P,Hk,page,d]")
    cache = _cache(k_cache, v_cache, k_scale, v_scale, block_table, kv_lens, Hq, k_cache.shape[1], d, N)
    _int32(parents, (N, Tq), "parents")
    _check_dev(parents)
    odt = _out_dtype(o, out_dtype)
    if o is None:
        o = torch.empty(N, Tq, Hq, d, dtype=odt, device=dev)
    elif o.shape != q.shape or not o.is_contiguous():
        raise ValueError("o must be contiguous [N,Tq,Hq,d]")
    query = KdaCacheQuery(tokens=Tq, q_stride=_token_stride(q, "q"), window=int(window), sinks=int(sinks),
                          scale=float(d ** -0.5 if scale is None else scale), max_kv_len=int(max_kv_len), out_dtype=_DTYPE_CODE[odt])
    if workspace is None:
        need = int(lib.kda_cache_tree_attn_workspace_size(ctypes.byref(cache), ctypes.byref(query)))
        workspace = torch.empty(need, dtype=torch.uint8, device=dev) if need else None
    else:
        _check_dev(workspace)
    _call(dev, lib.kda_cache_tree_attn, ctypes.byref(cache), ctypes.byref(query), _ptr(q), _ptr(parents), _ptr(o), _ptr(workspace),
          ctypes.c_size_t(0 if workspace is None else workspace.numel() * workspace.element_size()))
    return o


def _layers(k_cache, v_cache, k_scale, v_scale):
    """(layers, pages, heads, page size, dim) of one layer's cache or, with a dimension more in front, of a stack's."""
    if k_cache.dtype != torch.float8_e4m3fn or v_cache.dtype != torch.float8_e4m3fn or k_cache.dim() not in (4, 5) or k_cache.shape != v_cache.shape:
        raise ValueError("k_cache and v_cache must be float8_e4m3fn [P,Hk,page,d] or [layers,P,Hk,page,d]")
    for t in (k_scale, v_scale):
        if t.dtype != torch.float32 or t.shape != k_cache.shape[:-2]:
            raise ValueError("k_scale and v_scale must be fp32 [P,Hk] or [layers,P,Hk]")
    return (1, *k_cache.shape) if k_cache.dim() == 4 else tuple(k_cache.shape)


def kda_cache_keep(k_cache, v_cache, k_scale, v_scale, block_table, kv_lens, kept):
    """The accepted tokens of draft trees become the end of what their sequences hold, in place: codes at places kv_lens + kept[n][i] move to
    kv_lens + i, in one layer's cache (k_cache, v_cache float8_e4m3fn [P,Hk,page,d], k_scale, v_scale fp32 [P,Hk]) or in a whole stack's, with a
    dimension of layers in front of all four.  block_table int32 [N,pages] and kv_lens int32 [N] (without the drafted tokens; negative: skip;
    not changed here) are the layers' own in common; kept int32 [N,up to 64]: increasing indices of drafted tokens, ended by a negative one."""
    lib = load_library()
    if _native("keep", k_cache, v_cache, k_scale, v_scale, block_table, kv_lens, kept):
        return
    dev = _check_dev(k_cache, v_cache, k_scale, v_scale, block_table, kv_lens, kept)
    L, P, Hk, page, d = _layers(k_cache, v_cache, k_scale, v_scale)
    if block_table.dtype != torch.int32 or block_table.dim() != 2:
        raise ValueError("block_table must be int32 [N,pages]")
    N = block_table.shape[0]
    _int32(kv_lens, (N,), "kv_lens")
    if kept.dtype != torch.int32 or kept.dim() != 2 or kept.shape[0] != N:
        raise ValueError("kept must be int32 [N,up to 64]")
    cache = KdaCache(num_seqs=N, heads_q=Hk, heads_kv=Hk, dim=d, page_size=page, num_pages=P, max_pages=block_table.shape[1], k=k_cache.data_ptr(),
                     v=v_cache.data_ptr(), k_scale=k_scale.data_ptr(), v_scale=v_scale.data_ptr(), block_table=block_table.data_ptr(),
                     kv_lens=kv_lens.data_ptr())
    _call(dev, lib.kda_cache_keep, ctypes.byref(cache), L, _ptr(kept), kept.shape[1])


def kda_cache_copy_pages(k_cache, v_cache, k_scale, v_scale, pairs):
    """Copies pages, codes and scales, of one layer's cache or of a whole stack's (as for kda_cache_keep), in place.  pairs int32 [M,2]: (from,
    to); a pair with an entry that is no page, like (-1, -1), is skipped.  No page may be written by two pairs, or by one and read by another."""
    lib = load_library()
    if _native("copy_pages", k_cache, v_cache, k_scale, v_scale, pairs):
        return
    dev = _check_dev(k_cache, v_cache, k_scale, v_scale, pairs)
    L, P, Hk, page, d = _layers(k_cache, v_cache, k_scale, v_scale)
    if pairs.dtype != torch.int32 or pairs.dim() != 2 or pairs.shape[1] != 2:
        raise ValueError("pairs must be int32 [M,2]")
    cache = KdaCache(heads_kv=Hk, dim=d, page_size=page, num_pages=P, k=k_cache.data_ptr(), v=v_cache.data_ptr(), k_scale=k_scale.data_ptr(),
                     v_scale=v_scale.data_ptr())
    _call(dev, lib.kda_cache_copy_pages, ctypes.byref(cache), L, _ptr(pairs), pairs.shape[0])


def _pages(block_table, page_refs, *more):
    if block_table.dtype != torch.int32 or block_table.dim() != 2:
        raise ValueError("block_table must be int32 [N,pages]")
    if page_refs.dtype != torch.int32 or page_refs.dim() != 1:
        raise ValueError("page_refs must be int32 [P]")
    return _check_dev(block_table, page_refs, *more), block_table.shape[0], block_table.shape[1], page_refs.numel()


def kda_pages_fork(block_table, page_refs, source):
    """Rows of block_table int32 [N,pages] become what other rows were, in place, and page_refs int32 [P], how many entries name a page, follows:
    row n is row source[n] (source int32 [N]; n itself, or N and above: it stays), or empty where source[n] is negative, which frees the
    pages that no other row has.  A page with no reference is free."""
    lib = load_library()
    if _native("fork", block_table, page_refs, source):
        return
    dev, N, columns, P = _pages(block_table, page_refs, source)
    _int32(source, (N,), "source")
    _call(dev, lib.kda_pages_fork, _ptr(block_table), N, columns, _ptr(page_refs), P, _ptr(source))


def kda_pages_reserve(block_table, kv_lens, new_lens, page_refs, page_size, copies=None, missing=None, workspace=None):
    """Makes every sequence the only owner of the pages that it writes when it grows from kv_lens[n] to new_lens[n] tokens (int32 [N]): where
    block_table has none, or one that other rows have too, a free page takes its place, the lowest-numbered first.  Returns (copies int32
    [N,2], missing int32 [1]): copies for kda_cache_copy_pages, (-1, -1) where a sequence needs none; missing is how many pages were too few, and
    then nothing has changed."""
    lib = load_library()
    if workspace is None:
        done = _native("reserve", block_table, kv_lens, new_lens, page_refs, page_size, copies, missing)
        if done is not None:
            return done
    dev, N, columns, P = _pages(block_table, page_refs, kv_lens, new_lens, copies, missing, workspace)
    _int32(kv_lens, (N,), "kv_lens")
    _int32(new_lens, (N,), "new_lens")
    if copies is None:
        copies = torch.empty(N, 2, dtype=torch.int32, device=dev)
    if missing is None:
        missing = torch.empty(1, dtype=torch.int32, device=dev)
    _int32(copies, (N, 2), "copies")
    _int32(missing, (1,), "missing")
    if workspace is None:
        need = int(lib.kda_pages_reserve_workspace_size(N, columns, P))
        workspace = torch.empty(need, dtype=torch.uint8, device=dev) if need else None
    _call(dev, lib.kda_pages_reserve, _ptr(block_table), N, columns, int(page_size), _ptr(page_refs), P, _ptr(kv_lens), _ptr(new_lens), _ptr(copies),
          _ptr(missing), _ptr(workspace), ctypes.c_size_t(0 if workspace is None else workspace.numel() * workspace.element_size()))
    return copies, missing


def kda_pages_compact(block_table, page_refs, moves=None, workspace=None):
    """The pages in use move to the front of the pool: block_table and page_refs are changed in place, and the pages themselves are moved by
    kda_cache_copy_pages with what this returns, moves int32 [P // 2,2], (-1, -1) behind the last, before anything else writes them."""
    lib = load_library()
    dev, N, columns, P = _pages(block_table, page_refs, moves, workspace)
    if moves is None:
        moves = torch.empty(P // 2, 2, dtype=torch.int32, device=dev)
    _int32(moves, (P // 2, 2), "moves")
    if workspace is None:
        workspace = torch.empty(4 * P + 256, dtype=torch.uint8, device=dev)
    _call(dev, lib.kda_pages_compact, _ptr(block_table), N, columns, _ptr(page_refs), P, _ptr(moves), _ptr(workspace),
          ctypes.c_size_t(workspace.numel() * workspace.element_size()))
    return moves


def _delta(k, v, log_alpha, beta, S_pool, state_indices, scalar_gate):
    if k.dim() != 4 or v.dim() != 4 or k.dtype not in _DTYPE_CODE or not (k.dtype == v.dtype == log_alpha.dtype == beta.dtype):
        raise ValueError("k, v, log_alpha, beta must share a supported dtype, k and v be [N,Tq,H,d]")
    N, Tq, H, dk = k.shape
    dv = v.shape[3]
    if log_alpha.shape != ((N, Tq, H) if scalar_gate else k.shape) or v.shape[:3] != (N, Tq, H) or beta.shape != (N, Tq, H):
        raise ValueError("inconsistent input shapes")
    if S_pool.dtype != torch.float32 or S_pool.dim() != 4 or S_pool.shape[1:] != (H, dk, dv):
        raise ValueError("S_pool must be fp32 [P,H,dk,dv]")
    if state_indices is None:
        if S_pool.shape[0] < N:
            raise ValueError("S_pool holds fewer states than there are sequences")
    else:
        _int32(state_indices, (N,), "state_indices")
    return N, Tq, H, dk, dv


def kda_tree_steps(q, k, v, log_alpha, beta, S_pool, parents, state_indices=None, scale=1.0, o=None, out_dtype=None, scalar_gate=False):
    """KDA over a draft tree: token t steps from the state behind its parent, parents int32 [N,Tq] (-1: the sequence's own state; -2: there is no
    such token), and its output reads the state behind it.  q, k, log_alpha [N,Tq,H,dk], v [N,Tq,H,dv], beta [N,Tq,H] (Tq up to 64; bf16 or
    fp32); scalar_gate=True: log_alpha [N,Tq,H]; S_pool fp32 [P,H,dk,dv], read only; state_indices as for kda_recurrent_steps_pooled, but that
    sequences may share a state.  Returns o [N,Tq,H,dv], fp32 unless out_dtype (or the `o` passed in) is torch.bfloat16; rows of skipped
    sequences and of tokens that are not there are zero."""
    lib = load_library()
    done = _native("tree_steps", k, v, log_alpha, beta, S_pool, state_indices, q, parents, scale, o, out_dtype, scalar_gate)
    if done is not None:
        return done
    dev = _check_dev(q, k, v, log_alpha, beta, S_pool, parents, state_indices, o)
    N, Tq, H, dk, dv = _delta(k, v, log_alpha, beta, S_pool, state_indices, scalar_gate)
    if q.shape != k.shape or q.dtype != k.dtype:
        raise ValueError("q must be of k's shape and dtype")
    _int32(parents, (N, Tq), "parents")
    odt = _out_dtype(o, out_dtype)
    if o is None:
        o = torch.empty(v.shape, dtype=odt, device=dev)
    elif o.shape != v.shape:
        raise ValueError("o must have shape [N,Tq,H,dv]")
    dims = KdaDims(batch=N, seqlen=Tq, heads=H, dk=dk, dv=dv, chunk=64, num_seqs=N, in_dtype=_DTYPE_CODE[k.dtype], out_dtype=_DTYPE_CODE[odt],
                   scale=float(scale), max_seqlen=0)
    _call(dev, lib.kda_tree_steps, ctypes.byref(dims), _ptr(q), _ptr(k), _ptr(v), _ptr(log_alpha), _ptr(beta), _ptr(S_pool), _ptr(state_indices),
          _ptr(parents), _ptr(o), _SCALAR_GATE if scalar_gate else 0)
    return o


def kda_tree_commit(k, v, log_alpha, beta, S_pool, kept, state_indices=None, scalar_gate=False):
    """Takes the states of S_pool, in place, through the accepted tokens of the trees that kda_tree_steps had: kept int32 [N,up to 64],
    increasing indices ended by a negative one.  The other arguments are those of kda_tree_steps."""
    lib = load_library()
    if _native("tree_commit", k, v, log_alpha, beta, S_pool, state_indices, kept, scalar_gate):
        return
    dev = _check_dev(k, v, log_alpha, beta, S_pool, state_indices, kept)
    N, Tq, H, dk, dv = _delta(k, v, log_alpha, beta, S_pool, state_indices, scalar_gate)
    if kept.dtype != torch.int32 or kept.dim() != 2 or kept.shape[0] != N:
        raise ValueError("kept must be int32 [N,up to 64]")
    dims = KdaDims(batch=N, seqlen=Tq, heads=H, dk=dk, dv=dv, chunk=64, num_seqs=N, in_dtype=_DTYPE_CODE[k.dtype], out_dtype=0, scale=1.0,
                   max_seqlen=0)
    _call(dev, lib.kda_tree_commit, ctypes.byref(dims), _ptr(k), _ptr(v), _ptr(log_alpha), _ptr(beta), _ptr(S_pool), _ptr(state_indices), _ptr(kept),
          kept.shape[1], _SCALAR_GATE if scalar_gate else 0)
