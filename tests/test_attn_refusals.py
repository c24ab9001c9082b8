"""What the softmax-attention entry points refuse (CPU): nothing is launched, the status and a description come back."""
import ctypes

import pytest
import torch

import paper_2510_26692_amd as kda

SOME = 1 << 20                       # (a 256-byte aligned address that no refused call looks at)
INVALID, UNSUPPORTED, WORKSPACE = 1, 2, 3


def _dims(**kw):
    d = dict(batch=2, seqlen=100, heads_q=4, heads_kv=2, dim=128, num_seqs=2, in_dtype=1, out_dtype=1, scale=0.1, window=0, sinks=0)
    d.update(kw)
    return kda.KdaAttnDims(**d)


def _fwd(d, q=SOME, k=SOME, v=SOME, cu=None, o=SOME, lse=None):
    return kda.load_library().kda_window_attn_fwd(None if d is None else ctypes.byref(d), q, k, v, cu, o, lse, None)


def _bwd(d, ws=SOME, ws_bytes=1 << 40, **kw):
    a = dict(q=SOME, k=SOME, v=SOME, cu=None, o=SOME, lse=SOME, do=SOME, dq=SOME, dk=SOME, dv=SOME)
    a.update(kw)
    return kda.load_library().kda_window_attn_bwd(ctypes.byref(d), *a.values(), ws, ctypes.c_size_t(ws_bytes), None)


BAD_DIMS = [(dict(batch=-1), INVALID), (dict(seqlen=-1), INVALID), (dict(heads_q=-4), INVALID), (dict(in_dtype=7), INVALID), (dict(out_dtype=-1), INVALID),
            (dict(in_dtype=0), UNSUPPORTED), (dict(dim=96), UNSUPPORTED), (dict(dim=0), UNSUPPORTED), (dict(heads_q=5), INVALID),
            (dict(heads_kv=0), INVALID), (dict(heads_q=65536, heads_kv=65536), UNSUPPORTED), (dict(window=-1), INVALID), (dict(sinks=-1), INVALID),
            (dict(sinks=65), UNSUPPORTED), (dict(scale=0.0), INVALID), (dict(scale=-1.0), INVALID), (dict(scale=float("nan")), INVALID),
            (dict(scale=float("inf")), INVALID), (dict(num_seqs=3), INVALID), (dict(q_stride=511), INVALID), (dict(q_stride=504), INVALID),
            (dict(k_stride=260), INVALID), (dict(v_stride=1 << 25), INVALID), (dict(batch=1, num_seqs=1, seqlen=1 << 40), UNSUPPORTED),
            (dict(batch=1 << 20, num_seqs=1 << 20, seqlen=4096), UNSUPPORTED),
            (dict(batch=1 << 27, num_seqs=1 << 27, seqlen=1 << 30, heads_q=32), UNSUPPORTED)]          # (2^64 threads)


@pytest.mark.parametrize("change,status", BAD_DIMS)
def test_window_attn_refuses_dims(change, status):
    assert _fwd(_dims(**change)) == status and kda.kda_last_error()
    assert _bwd(_dims(**change)) == status
    assert kda.kda_window_attn_bwd_workspace_size(_dims(**change)) == 0


def test_window_attn_refuses_pointers_and_packed_batches():
    assert _fwd(None) == INVALID
    for name in ("q", "k", "v", "o"):
        assert _fwd(_dims(), **{name: None}) == INVALID and _fwd(_dims(), **{name: SOME + 8}) == INVALID
    assert _fwd(_dims(), lse=SOME + 4) == INVALID
    assert _fwd(_dims(), cu=SOME) == INVALID                                       # packed: one row
    assert _fwd(_dims(batch=1, num_seqs=3), cu=SOME + 2) == INVALID
    assert _fwd(_dims(batch=1, num_seqs=3, seqlen=1 << 31), cu=SOME) == INVALID
    for name in ("q", "k", "v", "o", "lse", "do", "dq", "dk", "dv"):
        assert _bwd(_dims(), **{name: None}) == INVALID and _bwd(_dims(), **{name: SOME + 8}) == INVALID
    assert _bwd(_dims(out_dtype=0)) == UNSUPPORTED
    need = kda.kda_window_attn_bwd_workspace_size(_dims())
    assert need > 0 and _bwd(_dims(), ws=None) == WORKSPACE and _bwd(_dims(), ws=SOME + 128) == WORKSPACE and _bwd(_dims(), ws_bytes=need - 1) == WORKSPACE


def test_empty_calls_are_done_without_a_launch():
    for change in (dict(seqlen=0), dict(batch=0, num_seqs=0), dict(heads_q=0)):
        assert _fwd(_dims(**change), q=None, k=None, v=None, o=None) == 0
        assert _bwd(_dims(**change), ws=None, ws_bytes=0) == 0
    assert _fwd(_dims(batch=1, num_seqs=0), cu=SOME) == 0


def test_backward_workspace_serves_a_row_with_and_without_cu_seqlens():
    for T in (1, 127, 128, 129, 128 * 255, 128 * 256, 128 * 2047):
        for hq, hk in ((8, 1), (8, 8), (32, 4)):
            for window, sinks in ((0, 0), (64, 4)):
                n = kda.kda_window_attn_bwd_workspace_size(_dims(batch=1, num_seqs=1, seqlen=T, heads_q=hq, heads_kv=hk, window=window, sinks=sinks))
                assert n >= 8 * T * hq


def _cache(**kw):
    d = dict(num_seqs=2, heads_q=4, heads_kv=2, dim=128, page_size=64, num_pages=8, max_pages=3, k=SOME, v=SOME, k_scale=SOME, v_scale=SOME,
             block_table=SOME, kv_lens=SOME)
    d.update(kw)
    return kda.KdaCache(**d)


def _append(c, seqlen=4, rope=None, **kw):
    a = dict(k=SOME, v=SOME, ks=0, vs=0, cu=None)
    b = dict(k_out=None, q=None, qs=0, q_out=None, flags=0)
    for n, x in kw.items():
        (a if n in a else b)[n] = x
    return kda.load_library().kda_cache_append(None if c is None else ctypes.byref(c), seqlen, *a.values(), None if rope is None else ctypes.byref(rope),
                                               *b.values(), None)


def _attn(c, q=SOME, o=SOME, ws=SOME, ws_bytes=1 << 40, **kw):
    a = dict(tokens=1, q_stride=0, window=0, sinks=0, scale=0.1, max_kv_len=0, out_dtype=1)
    a.update(kw)
    return kda.load_library().kda_cache_attn(None if c is None else ctypes.byref(c), ctypes.byref(kda.KdaCacheQuery(**a)), q, o, ws, ctypes.c_size_t(ws_bytes),
                                             None)


BAD_CACHES = [(dict(num_seqs=-1), INVALID), (dict(num_pages=-1), INVALID), (dict(max_pages=-1), INVALID), (dict(dim=256), UNSUPPORTED),
              (dict(page_size=8), UNSUPPORTED), (dict(page_size=48), UNSUPPORTED), (dict(page_size=256), UNSUPPORTED), (dict(heads_q=3), INVALID),
              (dict(heads_kv=0), INVALID), (dict(heads_q=70000, heads_kv=70000), UNSUPPORTED), (dict(num_pages=1 << 31), INVALID), (dict(k=None), INVALID),
              (dict(v=SOME + 8), INVALID), (dict(k_scale=None), INVALID), (dict(v_scale=SOME + 2), INVALID), (dict(block_table=None), INVALID),
              (dict(kv_lens=None), INVALID), (dict(kv_lens=SOME + 1), INVALID)]


@pytest.mark.parametrize("change,status", BAD_CACHES)
def test_cache_calls_refuse_caches(change, status):
    assert _append(_cache(**change)) == status and kda.kda_last_error()
    assert _attn(_cache(**change)) == status


def test_cache_append_refuses():
    assert _append(None) == INVALID
    c = _cache()
    for kw in (dict(k=None), dict(v=None), dict(k=SOME + 8), dict(ks=250), dict(vs=128), dict(q=SOME), dict(q_out=SOME), dict(q=SOME, q_out=SOME + 8),
               dict(q=SOME, q_out=SOME, qs=100), dict(k_out=SOME + 8), dict(cu=SOME + 1), dict(seqlen=-1), dict(flags=4)):
        assert _append(c, **kw) == INVALID, kw
    for n in (-8, 4, 12, 72):
        assert _append(c, rope=kda.KdaRope(inv_freq=SOME, num_freqs=n)) == INVALID
    assert _append(c, rope=kda.KdaRope(inv_freq=None, num_freqs=64)) == INVALID
    assert _append(c, seqlen=1 << 40) == UNSUPPORTED and _append(_cache(num_seqs=1 << 27)) == UNSUPPORTED
    assert _append(_cache(num_seqs=1 << 22, heads_q=128), q=SOME, q_out=SOME) == UNSUPPORTED
    for page in (16, 32, 64, 128):                                                 # (2^64 tokens' heads, or pages')
        for n, hk in ((27, 64), (28, 32), (27, 128), (28, 64), (26, 128), (30, 16)):
            assert _append(_cache(num_seqs=1 << n, heads_q=hk, heads_kv=hk, page_size=page), seqlen=1 << 36) == UNSUPPORTED
    assert _append(c, seqlen=0, k=None, v=None) == 0 and _append(_cache(num_seqs=0)) == 0


def test_cache_attn_refuses():
    assert _attn(None) == INVALID
    c = _cache()
    for kw in (dict(tokens=-1), dict(window=-1), dict(sinks=-1), dict(max_kv_len=-1), dict(scale=0.0), dict(scale=float("nan")), dict(out_dtype=2),
               dict(q_stride=100), dict(q=None), dict(o=None), dict(q=SOME + 8), dict(o=SOME + 4)):
        assert _attn(c, **kw) == INVALID, kw
    for kw in (dict(tokens=9), dict(sinks=65)):
        assert _attn(c, **kw) == UNSUPPORTED, kw
    long = _cache(num_seqs=1, max_pages=1000, num_pages=1000)
    query = kda.KdaCacheQuery(tokens=1, scale=0.1, out_dtype=1)
    need = kda.load_library().kda_cache_attn_workspace_size(ctypes.byref(long), ctypes.byref(query))
    assert need > 0
    assert _attn(long, ws=None) == WORKSPACE and _attn(long, ws=SOME + 16) == WORKSPACE and _attn(long, ws_bytes=need - 1) == WORKSPACE
    assert _attn(_cache(max_pages=1 << 30)) == UNSUPPORTED and _attn(_cache(num_seqs=1 << 24)) == UNSUPPORTED
    assert _attn(c, tokens=0) == 0 and _attn(_cache(num_seqs=0)) == 0


def test_binding_refuses_before_it_calls():
    q, k = torch.zeros(1, 4, 2, 64, dtype=torch.bfloat16), torch.zeros(1, 4, 1, 64, dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="device tensors"):
        kda.kda_window_attn_fwd(q, k, k)
    with pytest.raises(ValueError, match="device tensors"):
        kda.kda_cache_append(k, k, *[torch.zeros(1)] * 6)
    with pytest.raises(ValueError, match="device tensors"):
        kda.kda_cache_attn(q, *[torch.zeros(1)] * 6)


def test_token_strides_the_binding_takes():
    from paper_2510_26692_amd.attn import _token_stride
    x = torch.zeros(2, 5, 12, 64)
    assert _token_stride(x, "x") == 0
    assert _token_stride(x[:, :, 4:6], "x") == 12 * 64                # a slice of one projection's output
    assert _token_stride(x[:1, :1, 4:6], "x") in (0, 2 * 64)          # one token: no distance to another
    assert _token_stride(x[:, :1, :2], "x") == 5 * 12 * 64            # one token of each row
    one = torch.zeros(1, 1, 12, 64)
    for bad in (x[:, :, ::2], x[..., ::2], x.transpose(1, 2), x[:, :4, :2], one.expand(1, 5, 12, 64), one.expand(3, 1, 12, 64), one.expand(3, 5, 12, 64),
                x[:, :, :1].expand(2, 5, 3, 64)):
        with pytest.raises(ValueError, match="evenly spaced"):
            _token_stride(bad, "x")
