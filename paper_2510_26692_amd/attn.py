"""Binding of libkda's softmax-attention entry points (see include/kda.h): the layers that a hybrid stack has beside KDA.

Argument marshalling only, like ``kda.py``: tensors are device-memory handles, the stream is torch's current HIP stream.
"""
import ctypes

import torch

from . import kda as _kda
from .kda import KdaError, _DTYPE_CODE, _call, _check_dev, _clear_unowned, _out_dtype, _ptr, kda_last_error, load_library


_APPEND_ZERO_Q, _APPEND_ZERO_K = 1, 2    # flags of kda_cache_append


class KdaAttnDims(ctypes.Structure):
    """Mirror of ``kda_attn_dims``."""
    _fields_ = [("batch", ctypes.c_int32), ("seqlen", ctypes.c_int64), ("heads_q", ctypes.c_int32), ("heads_kv", ctypes.c_int32),
                ("dim", ctypes.c_int32), ("num_seqs", ctypes.c_int32), ("in_dtype", ctypes.c_int), ("out_dtype", ctypes.c_int),
                ("scale", ctypes.c_float), ("window", ctypes.c_int64), ("sinks", ctypes.c_int32),
                ("q_stride", ctypes.c_int64), ("k_stride", ctypes.c_int64), ("v_stride", ctypes.c_int64)]


class KdaCache(ctypes.Structure):
    """Mirror of ``kda_cache``."""
    _fields_ = [("num_seqs", ctypes.c_int32), ("heads_q", ctypes.c_int32), ("heads_kv", ctypes.c_int32), ("dim", ctypes.c_int32),
                ("page_size", ctypes.c_int32), ("num_pages", ctypes.c_int64), ("max_pages", ctypes.c_int32),
                ("k", ctypes.c_void_p), ("v", ctypes.c_void_p), ("k_scale", ctypes.c_void_p), ("v_scale", ctypes.c_void_p),
                ("block_table", ctypes.c_void_p), ("kv_lens", ctypes.c_void_p)]


class KdaRope(ctypes.Structure):
    """Mirror of ``kda_rope``."""
    _fields_ = [("inv_freq", ctypes.c_void_p), ("num_freqs", ctypes.c_int32), ("interleaved", ctypes.c_int32)]


class KdaCacheQuery(ctypes.Structure):
    """Mirror of ``kda_cache_query``."""
    _fields_ = [("tokens", ctypes.c_int32), ("q_stride", ctypes.c_int64), ("window", ctypes.c_int64), ("sinks", ctypes.c_int32),
                ("scale", ctypes.c_float), ("max_kv_len", ctypes.c_int64), ("out_dtype", ctypes.c_int)]


def _native(name, *args):
    """What the native way (csrc/kda_host.cpp) returned, or None: not built, or a call it leaves to the general way."""
    if _kda._native is None:
        return None
    done = getattr(_kda._native, name)(*args)
    if type(done) is int:
        raise KdaError(done, kda_last_error())
    return done


def _token_stride(t, name):
    """Elements from a token of t [B,T,H,d] to the next: heads and channels contiguous, tokens evenly spaced over the whole batch.
    0: contiguous."""
    B, T, H, d = t.shape
    sb, st, sh, sd = t.stride()
    if t.numel() == 0 or t.is_contiguous():
        return 0
    step = st if T > 1 else sb if B > 1 else H * d
    if (d > 1 and sd != 1) or (H > 1 and sh != d) or (B > 1 and T > 1 and sb != T * st) or step < H * d:
        raise ValueError("%s: heads and channels must be contiguous, and tokens evenly spaced" % name)
    return step


def _device(*tensors):
    """The one device of the tensors, which need not be contiguous."""
    dev = None
    for t in tensors:
        if t is None:
            continue
        if not t.is_cuda:
            raise ValueError("libkda takes device tensors only")
        dev = dev or t.device
        if t.device != dev:
            raise ValueError("all tensors must live on one device")
    return dev


def _attn_dims(q, k, v, window, sinks, cu_seqlens, scale, out_dtype):
    if not (q.dim() == k.dim() == v.dim() == 4):
        raise ValueError("q, k and v must be [B,T,heads,dim]")
    B, T, Hq, d = q.shape
    if k.shape != v.shape or k.shape[:2] != (B, T) or k.shape[3] != d:
        raise ValueError("inconsistent input shapes")
    if not (q.dtype == k.dtype == v.dtype) or q.dtype not in _DTYPE_CODE:
        raise ValueError("q, k, v must share a supported dtype")
    if cu_seqlens is not None and (cu_seqlens.dtype != torch.int32 or cu_seqlens.dim() != 1 or not cu_seqlens.numel()
                                   or not cu_seqlens.is_contiguous()):
        raise ValueError("cu_seqlens must be contiguous int32 [N+1]")
    return KdaAttnDims(batch=B, seqlen=T, heads_q=Hq, heads_kv=k.shape[2], dim=d,
                       num_seqs=B if cu_seqlens is None else cu_seqlens.numel() - 1, in_dtype=_DTYPE_CODE[q.dtype],
                       out_dtype=_DTYPE_CODE[out_dtype], scale=float(d ** -0.5 if scale is None else scale), window=int(window),
                       sinks=int(sinks), q_stride=_token_stride(q, "q"), k_stride=_token_stride(k, "k"),
                       v_stride=_token_stride(v, "v"))


def kda_window_attn_fwd(q, k, v, window=0, sinks=0, cu_seqlens=None, scale=None, o=None, lse=None, want_lse=True, out_dtype=None):
    """Causal softmax attention.  q [B,T,Hq,d], k and v [B,T,Hk,d] bf16 (d 64 or 128, Hq a multiple of Hk; tokens may be spaced, as in
    slices of one projection's output); cu_seqlens int32 [N+1] on the device for a packed batch (B = 1), or None.  A query sees the
    `window` latest tokens (0: all earlier ones), itself among them, and the first `sinks` tokens of its sequence.  scale: d ** -0.5 unless
    given.  Returns (o [B,T,Hq,d], lse fp32 [B,Hq,T] or None); o is fp32 unless out_dtype (or the `o` passed in) is torch.bfloat16.
    Rows of tokens that belong to no sequence are zero in what this call allocates and untouched in what is passed in."""
    lib = load_library()
    if cu_seqlens is None:
        done = _native("window_fwd", q, k, v, window, sinks, scale, o, lse, want_lse, out_dtype)
        if done is not None:
            return done
    dev = _device(q, k, v, cu_seqlens, o, lse)
    odt = _out_dtype(o, out_dtype)
    dims = _attn_dims(q, k, v, window, sinks, cu_seqlens, scale, odt)
    B, T, Hq, d = q.shape
    fresh = []
    if o is None:
        o = torch.empty(B, T, Hq, d, dtype=odt, device=dev)
        fresh.append(o)
    elif o.shape != q.shape or not o.is_contiguous():
        raise ValueError("o must be contiguous [B,T,Hq,d]")
    if lse is not None:
        if lse.dtype != torch.float32 or lse.shape != (B, Hq, T) or not lse.is_contiguous():
            raise ValueError("lse must be contiguous fp32 [B,Hq,T]")
    elif want_lse:
        lse = (torch.empty if cu_seqlens is None else torch.zeros)(B, Hq, T, dtype=torch.float32, device=dev)
    _call(dev, lib.kda_window_attn_fwd, ctypes.byref(dims), _ptr(q), _ptr(k), _ptr(v), _ptr(cu_seqlens), _ptr(o), _ptr(lse))
    if cu_seqlens is not None and fresh:
        _clear_unowned(cu_seqlens, fresh)
    return o, lse


def kda_window_attn_bwd_workspace_size(dims):
    return int(load_library().kda_window_attn_bwd_workspace_size(ctypes.byref(dims)))


def kda_window_attn_bwd(q, k, v, o, lse, do, window=0, sinks=0, cu_seqlens=None, scale=None, workspace=None, out=None):
    """Backward pass of kda_window_attn_fwd: o (bf16) and lse are what it returned for the same inputs and options, do the gradient of o
    in bf16.  Returns a dict of bf16 tensors dq [B,T,Hq,d], dk and dv [B,T,Hk,d]; rows of tokens that belong to no sequence are zero (this
    wrapper clears them in the gradients it allocates).  `out`: the dict an earlier call returned, to be written in place."""
    lib = load_library()
    if cu_seqlens is None and workspace is None and out is None:
        done = _native("window_bwd", q, k, v, o, lse, do, window, sinks, scale)
        if done is not None:
            return dict(zip(("dq", "dk", "dv"), done))
    dev = _device(q, k, v, o, lse, do, cu_seqlens, workspace)
    if o.dtype != torch.bfloat16 or do.dtype != torch.bfloat16 or o.shape != q.shape or do.shape != q.shape:
        raise ValueError("o and do must be bf16 [B,T,Hq,d]")
    dims = _attn_dims(q, k, v, window, sinks, cu_seqlens, scale, torch.bfloat16)
    B, T, Hq, d = q.shape
    if lse.dtype != torch.float32 or lse.shape != (B, Hq, T):
        raise ValueError("lse must be fp32 [B,Hq,T]")
    _check_dev(o, lse, do, workspace)
    shapes = {"dq": q.shape, "dk": k.shape, "dv": v.shape}
    clear = None
    if out is None:
        out = {n: torch.empty(sh, dtype=torch.bfloat16, device=dev) for n, sh in shapes.items()}
        clear = list(out.values())
    else:
        for n, sh in shapes.items():
            t = out.get(n)
            if t is None or t.dtype != torch.bfloat16 or t.shape != sh:
                raise ValueError("out[%r] must be a contiguous bf16 tensor of shape %r" % (n, tuple(sh)))
        _check_dev(o, *out.values())
    if workspace is None:
        workspace = torch.empty(max(kda_window_attn_bwd_workspace_size(dims), 256), dtype=torch.uint8, device=dev)
    _call(dev, lib.kda_window_attn_bwd, ctypes.byref(dims), _ptr(q), _ptr(k), _ptr(v), _ptr(cu_seqlens), _ptr(o), _ptr(lse), _ptr(do),
          _ptr(out["dq"]), _ptr(out["dk"]), _ptr(out["dv"]), _ptr(workspace), ctypes.c_size_t(workspace.numel() * workspace.element_size()))
    if cu_seqlens is not None and clear:
        _clear_unowned(cu_seqlens, clear)
    return out


def _cache(k_cache, v_cache, k_scale, v_scale, block_table, kv_lens, heads_q, heads_kv, d, num_seqs):
    if k_cache.dtype != torch.float8_e4m3fn or v_cache.dtype != torch.float8_e4m3fn or k_cache.dim() != 4 or k_cache.shape != v_cache.shape \
            or k_cache.shape[1] != heads_kv or k_cache.shape[3] != d:
        raise ValueError("k_cache and v_cache must be float8_e4m3fn [P,Hk,page,d]")
    P, _, page, _ = k_cache.shape
    for t in (k_scale, v_scale):
        if t.dtype != torch.float32 or t.shape != (P, heads_kv):
            raise ValueError("k_scale and v_scale must be fp32 [P,Hk]")
    if block_table.dtype != torch.int32 or block_table.dim() != 2 or block_table.shape[0] != num_seqs:
        raise ValueError("block_table must be int32 [N,pages]")
    if kv_lens.dtype != torch.int32 or kv_lens.shape != (num_seqs,):
        raise ValueError("kv_lens must be int32 [N]")
    _check_dev(k_cache, v_cache, k_scale, v_scale, block_table, kv_lens)
    return KdaCache(num_seqs=num_seqs, heads_q=heads_q, heads_kv=heads_kv, dim=d, page_size=page, num_pages=P, max_pages=block_table.shape[1],
                    k=k_cache.data_ptr(), v=v_cache.data_ptr(), k_scale=k_scale.data_ptr(), v_scale=v_scale.data_ptr(),
                    block_table=block_table.data_ptr(), kv_lens=kv_lens.data_ptr())


def kda_cache_append(k, v, k_cache, v_cache, k_scale, v_scale, block_table, kv_lens, cu_seqlens=None, inv_freq=None, interleaved=False,
                     q=None, q_out=None, k_out=None, want_k=False):
    """Appends new tokens to the paged cache (kda_cache in kda.h), in place.  k, v bf16 [N,T,Hk,d], or packed [1,T,Hk,d] with cu_seqlens int32
    [N+1]; k_cache, v_cache float8_e4m3fn [P,Hk,page,d]; k_scale, v_scale fp32 [P,Hk]; block_table int32 [N,pages]; kv_lens int32 [N], the
    tokens held before the call (negative = skip; not changed here).  inv_freq fp32 [n]: keys are rotated by position * inv_freq, channels
    (i, i + n) or, interleaved, (2 i, 2 i + 1) together; None: no rotation.  q bf16 [..,Hq,d]: rotated too, into q_out if given.  want_k=True (or
    a k_out passed in): the rotated keys in bf16 as well.  Returns (q_out or None, k_out or None); rows of skipped sequences and of tokens that
    belong to none are zero in what this call allocates and untouched in what is passed in."""
    lib = load_library()
    done = _native("append", k, v, k_cache, v_cache, k_scale, v_scale, block_table, kv_lens, cu_seqlens, inv_freq, interleaved, q, q_out, k_out, want_k)
    if done is not None:
        return done
    dev = _device(k, v, q, k_cache, v_cache, k_scale, v_scale, block_table, kv_lens, cu_seqlens, inv_freq, q_out, k_out)
    if k.dim() != 4 or k.shape != v.shape or not (k.dtype == v.dtype == torch.bfloat16):
        raise ValueError("k and v must be bf16 [N,T,Hk,d]")
    B, T, Hk, d = k.shape
    Hq = Hk
    if q is not None:
        if q.dim() != 4 or q.dtype != torch.bfloat16 or q.shape[:2] != (B, T) or q.shape[3] != d:
            raise ValueError("q must be bf16 [N,T,Hq,d]")
        Hq = q.shape[2]
    elif q_out is not None:
        raise ValueError("q_out without q")
    N = B
    if cu_seqlens is not None:
        if cu_seqlens.dtype != torch.int32 or cu_seqlens.dim() != 1 or not cu_seqlens.numel() or not cu_seqlens.is_contiguous() or B != 1:
            raise ValueError("cu_seqlens must be contiguous int32 [N+1], with one row of packed tokens")
        N = cu_seqlens.numel() - 1
    cache = _cache(k_cache, v_cache, k_scale, v_scale, block_table, kv_lens, Hq, Hk, d, N)
    rope = None
    if inv_freq is not None:
        if inv_freq.dtype != torch.float32 or inv_freq.dim() != 1 or not inv_freq.is_contiguous():
            raise ValueError("inv_freq must be contiguous fp32 [n]")
        rope = KdaRope(inv_freq=inv_freq.data_ptr(), num_freqs=inv_freq.numel(), interleaved=int(bool(interleaved)))
    for t, like, name in ((q_out, q, "q_out"), (k_out, k, "k_out")):
        if t is not None and (t.dtype != torch.bfloat16 or t.shape != like.shape or not t.is_contiguous()):
            raise ValueError("%s must be contiguous bf16 of the shape of what is rotated" % name)
    flags = 0
    if q is not None and q_out is None:
        q_out = torch.empty(q.shape, dtype=torch.bfloat16, device=dev)
        flags |= _APPEND_ZERO_Q
    if want_k and k_out is None:
        k_out = torch.empty(k.shape, dtype=torch.bfloat16, device=dev)
        flags |= _APPEND_ZERO_K
    _call(dev, lib.kda_cache_append, ctypes.byref(cache), T, _ptr(k), _ptr(v), _token_stride(k, "k"), _token_stride(v, "v"), _ptr(cu_seqlens),
          None if rope is None else ctypes.byref(rope), _ptr(k_out), _ptr(q), 0 if q is None else _token_stride(q, "q"), _ptr(q_out), flags)
    return q_out, k_out


def kda_cache_attn(q, k_cache, v_cache, k_scale, v_scale, block_table, kv_lens, window=0, sinks=0, scale=None, max_kv_len=0, o=None,
                   out_dtype=None, workspace=None):
    """Attention of each sequence's 1-8 newest tokens over the paged cache.  q bf16 [N,Tq,Hq,d]; the cache as for kda_cache_append, kv_lens int32
    [N] counting the new tokens too; window and sinks as for kda_window_attn_fwd; max_kv_len: upper bound of kv_lens if known (it sets how far
    the work is split).  Returns o [N,Tq,Hq,d], fp32 unless out_dtype (or the `o` passed in) is torch.bfloat16; tokens that see nothing
    get zeros."""
    lib = load_library()
    if workspace is None:
        done = _native("attend", q, k_cache, v_cache, k_scale, v_scale, block_table, kv_lens, window, sinks, scale, max_kv_len, o, out_dtype)
        if done is not None:
            return done
    dev = _device(q, k_cache, v_cache, k_scale, v_scale, block_table, kv_lens, o, workspace)
    if q.dim() != 4 or q.dtype != torch.bfloat16:
        raise ValueError("q must be bf16 [N,Tq,Hq,d]")
    N, Tq, Hq, d = q.shape
    cache = _cache(k_cache, v_cache, k_scale, v_scale, block_table, kv_lens, Hq, k_cache.shape[1], d, N)
    odt = _out_dtype(o, out_dtype)
    if o is None:
        o = torch.empty(N, Tq, Hq, d, dtype=odt, device=dev)
    elif o.shape != q.shape or not o.is_contiguous():
        raise ValueError("o must be contiguous [N,Tq,Hq,d]")
    query = KdaCacheQuery(tokens=Tq, q_stride=_token_stride(q, "q"), window=int(window), sinks=int(sinks),
                          scale=float(d ** -0.5 if scale is None else scale), max_kv_len=int(max_kv_len), out_dtype=_DTYPE_CODE[odt])
    if workspace is None:
        need = int(lib.kda_cache_attn_workspace_size(ctypes.byref(cache), ctypes.byref(query)))
        workspace = torch.empty(need, dtype=torch.uint8, device=dev) if need else None
    else:
        _check_dev(workspace)
    _call(dev, lib.kda_cache_attn, ctypes.byref(cache), ctypes.byref(query), _ptr(q), _ptr(o), _ptr(workspace),
          ctypes.c_size_t(0 if workspace is None else workspace.numel() * workspace.element_size()))
    return o
