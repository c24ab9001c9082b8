"""What the entry points for draft trees and shared pages refuse (CPU): nothing is launched, the status and a description come back."""
import ctypes

import pytest
import torch

import paper_2510_26692_amd as kda

SOME = 1 << 20                       # (a 256-byte aligned address that no refused call looks at)
FAR = 1 << 40                        # (another, behind whatever stands at the first)
INVALID, UNSUPPORTED, WORKSPACE = 1, 2, 3


def _lib():
    return kda.load_library()


def _rotate(q=SOME, k=SOME + (1 << 30), pos=SOME, qo=FAR, ko=2 * FAR, **kw):
    a = dict(batch=2, seqlen=10, heads_q=4, heads_k=2, dim=128, dtype=1, axes=1, num_freqs=64, inv_freq=SOME)
    a.update(kw)
    return _lib().kda_rotate(ctypes.byref(kda.KdaRotation(**a)), q, k, pos, qo, ko, None)


@pytest.mark.parametrize("change,status", [
    (dict(batch=-1), INVALID), (dict(seqlen=-1), INVALID), (dict(heads_q=-1), INVALID), (dict(heads_k=-1), INVALID), (dict(dim=96), UNSUPPORTED),
    (dict(dtype=5), INVALID), (dict(heads_q=65536), UNSUPPORTED), (dict(axes=0), UNSUPPORTED), (dict(axes=5), UNSUPPORTED), (dict(num_freqs=-8), INVALID),
    (dict(num_freqs=72), INVALID), (dict(num_freqs=12), INVALID), (dict(axes=2, axis_of_freq=bytes([0, 1] * 31 + [1, 2])), INVALID),
    (dict(q_stride=511), INVALID), (dict(q_stride=504), INVALID), (dict(k_stride=1 << 25), INVALID), (dict(seqlen=1 << 30), UNSUPPORTED),
    (dict(batch=1 << 30, seqlen=1 << 40), UNSUPPORTED), (dict(q=None), INVALID), (dict(q=SOME + 8), INVALID), (dict(k=None), INVALID),
    (dict(ko=None), INVALID), (dict(qo=None), INVALID), (dict(pos=None), INVALID), (dict(pos=SOME + 2), INVALID), (dict(inv_freq=None), INVALID),
    (dict(qo=FAR + 4), INVALID), (dict(qo=SOME + 16), INVALID), (dict(ko=SOME), INVALID), (dict(qo=FAR, ko=FAR + 512), INVALID),
    (dict(qo=SOME, q_stride=1024), INVALID), (dict(seqlen=1 << 28, heads_q=64, qo=1 << 45, ko=1 << 46, k=1 << 47), UNSUPPORTED)])
def test_rotate_refuses(change, status):
    assert _rotate(**change) == status and kda.kda_last_error()


def test_rotate_of_nothing():
    assert _lib().kda_rotate(None, SOME, SOME, SOME, FAR, FAR, None) == INVALID
    assert _rotate(batch=0) == 0 and _rotate(seqlen=0, q=None, k=None, qo=None, ko=None, pos=None) == 0 and _rotate(heads_q=0, heads_k=0) == 0


def _cache(**kw):
    a = dict(num_seqs=2, heads_q=4, heads_kv=2, dim=128, page_size=64, num_pages=10, max_pages=4, k=SOME, v=SOME, k_scale=SOME, v_scale=SOME,
             block_table=SOME, kv_lens=SOME)
    a.update(kw)
    return kda.KdaCache(**a)


def _attend(cache=None, q=SOME, parents=SOME, o=SOME, ws=SOME, ws_bytes=1 << 40, **kw):
    a = dict(tokens=8, scale=0.1, out_dtype=1)
    a.update(kw)
    query = kda.KdaCacheQuery(**a)
    cache = cache or _cache()
    return _lib().kda_cache_tree_attn(ctypes.byref(cache), ctypes.byref(query), q, parents, o, ws, ctypes.c_size_t(ws_bytes), None)


@pytest.mark.parametrize("change,status", [
    (dict(tokens=-1), INVALID), (dict(tokens=65), UNSUPPORTED), (dict(window=-1), INVALID), (dict(sinks=-1), INVALID), (dict(sinks=65), UNSUPPORTED),
    (dict(scale=0.0), INVALID), (dict(scale=float("nan")), INVALID), (dict(max_kv_len=-1), INVALID), (dict(out_dtype=3), INVALID),
    (dict(q_stride=500), INVALID), (dict(q=None), INVALID), (dict(q=SOME + 8), INVALID), (dict(o=None), INVALID), (dict(parents=None), INVALID),
    (dict(parents=SOME + 1), INVALID), (dict(ws=None), WORKSPACE), (dict(ws=SOME + 128), WORKSPACE), (dict(ws_bytes=1000), WORKSPACE)])
def test_tree_attention_refuses(change, status):
    assert _attend(cache=_cache(max_pages=400), **change) == status and kda.kda_last_error()


@pytest.mark.parametrize("change,status", [
    (dict(num_seqs=-1), INVALID), (dict(dim=80), UNSUPPORTED), (dict(page_size=48), UNSUPPORTED), (dict(heads_q=5), INVALID), (dict(heads_q=65536), UNSUPPORTED),
    (dict(max_pages=1 << 26), UNSUPPORTED), (dict(num_pages=1 << 31), INVALID), (dict(k=None), INVALID), (dict(v_scale=None), INVALID),
    (dict(block_table=None), INVALID), (dict(kv_lens=None), INVALID), (dict(v=SOME + 4), INVALID), (dict(kv_lens=SOME + 2), INVALID)])
def test_calls_over_the_cache_refuse(change, status):
    assert _attend(cache=_cache(**change)) == status
    assert _lib().kda_cache_keep(ctypes.byref(_cache(**change)), 1, SOME, 8, None) == status


def test_tree_attention_sizes():
    q = lambda **kw: kda.KdaCacheQuery(**dict(dict(tokens=8, scale=0.1, out_dtype=1), **kw))
    size = lambda c, x: _lib().kda_cache_tree_attn_workspace_size(ctypes.byref(c), ctypes.byref(x))
    assert size(_cache(max_pages=400), q()) > 0 and size(_cache(max_pages=1), q()) == 0 and size(_cache(), q(tokens=65)) == 0
    assert size(_cache(max_pages=4000), q(max_kv_len=64)) == 0
    assert _lib().kda_cache_tree_attn(ctypes.byref(_cache()), None, SOME, SOME, SOME, SOME, ctypes.c_size_t(1 << 40), None) == INVALID
    assert _attend(tokens=0) == 0 and _attend(cache=_cache(num_seqs=0)) == 0
    assert _attend(cache=_cache(num_seqs=1 << 22, heads_q=64, heads_kv=64)) == UNSUPPORTED


def test_keep_and_copy_refuse():
    keep = lambda layers=2, kept=SOME, most=8, **kw: _lib().kda_cache_keep(ctypes.byref(_cache(heads_q=2, **kw)), layers, kept, most, None)
    assert keep(layers=-1) == INVALID and keep(most=-1) == INVALID and keep(most=65) == UNSUPPORTED and keep(kept=None) == INVALID
    assert keep(kept=SOME + 2) == INVALID and keep(layers=1 << 30) == UNSUPPORTED and keep(num_seqs=1 << 24) == UNSUPPORTED
    assert keep(layers=0) == 0 and keep(most=0) == 0 and keep(num_seqs=0) == 0 and keep(num_pages=0) == 0
    copy = lambda layers=2, pairs=SOME, n=5, **kw: _lib().kda_cache_copy_pages(ctypes.byref(_cache(**kw)), layers, pairs, n, None)
    assert copy(layers=-1) == INVALID and copy(n=-1) == INVALID and copy(pairs=None) == INVALID and copy(pairs=SOME + 1) == INVALID
    assert copy(n=1 << 32) == UNSUPPORTED and copy(layers=65536) == UNSUPPORTED and copy(k=None) == INVALID and copy(k_scale=SOME + 2) == INVALID
    assert copy(dim=96) == UNSUPPORTED and copy(page_size=8) == UNSUPPORTED and copy(heads_kv=-1) == INVALID
    assert copy(layers=0) == 0 and copy(n=0) == 0 and copy(num_pages=0) == 0 and copy(heads_kv=0) == 0
    assert _lib().kda_cache_copy_pages(None, 1, SOME, 1, None) == INVALID and _lib().kda_cache_keep(None, 1, SOME, 1, None) == INVALID


def test_pages_refuse():
    fork = lambda table=SOME, n=4, cols=3, refs=SOME, pages=10, source=SOME: _lib().kda_pages_fork(table, n, cols, refs, pages, source, None)
    assert fork(n=-1) == INVALID and fork(cols=-1) == INVALID and fork(pages=-1) == INVALID and fork(pages=1 << 31) == INVALID
    assert fork(table=None) == INVALID and fork(refs=None) == INVALID and fork(source=None) == INVALID and fork(refs=SOME + 4) == INVALID
    assert fork(table=SOME + 1) == INVALID and fork(source=SOME + 3) == INVALID and fork(n=8193) == UNSUPPORTED
    assert fork(n=0) == 0 and fork(cols=0) == 0

    def reserve(table=SOME, n=4, cols=3, page=64, refs=SOME, pages=10, lens=SOME, after=SOME, copies=SOME, missing=SOME, ws=SOME, size=1 << 30):
        return _lib().kda_pages_reserve(table, n, cols, page, refs, pages, lens, after, copies, missing, ws, ctypes.c_size_t(size), None)
    assert reserve(page=20) == UNSUPPORTED and reserve(n=8193) == UNSUPPORTED and reserve(n=8192, cols=1 << 18, pages=0, refs=None) == UNSUPPORTED
    for name in ("table", "refs", "lens", "after", "copies", "missing"):
        assert reserve(**{name: None}) == INVALID and reserve(**{name: SOME + 2}) == INVALID
    need = _lib().kda_pages_reserve_workspace_size(4, 3, 10)
    assert need > 0 and reserve(ws=None) == WORKSPACE and reserve(ws=SOME + 64) == WORKSPACE and reserve(size=need - 1) == WORKSPACE
    assert _lib().kda_pages_reserve_workspace_size(-1, 3, 10) == 0

    def compact(table=SOME, n=4, cols=3, refs=SOME, pages=10, moves=SOME, ws=SOME, size=1 << 30):
        return _lib().kda_pages_compact(table, n, cols, refs, pages, moves, ws, ctypes.c_size_t(size), None)
    assert compact(moves=None) == INVALID and compact(moves=SOME + 2) == INVALID and compact(ws=None) == WORKSPACE and compact(size=295) == WORKSPACE
    assert compact(refs=None) == INVALID and compact(n=-1) == INVALID and compact(pages=0) == 0


def _dims(**kw):
    a = dict(batch=2, num_seqs=2, seqlen=8, heads=2, dk=128, dv=128, chunk=64, in_dtype=1, out_dtype=1, scale=1.0)
    a.update(kw)
    return kda.KdaDims(**a)


def _steps(d=None, flags=0, **kw):
    a = dict(q=SOME, k=SOME, v=SOME, la=SOME, beta=SOME, S=SOME, idx=None, parents=SOME, o=SOME)
    a.update(kw)
    return _lib().kda_tree_steps(ctypes.byref(d or _dims()), *a.values(), flags, None)


def _commit(d=None, flags=0, most=8, **kw):
    a = dict(k=SOME, v=SOME, la=SOME, beta=SOME, S=SOME, idx=None, kept=SOME)
    a.update(kw)
    return _lib().kda_tree_commit(ctypes.byref(d or _dims()), *a.values(), most, flags, None)


@pytest.mark.parametrize("change,status", [
    (dict(batch=-1), INVALID), (dict(seqlen=-1), INVALID), (dict(seqlen=65), UNSUPPORTED), (dict(heads=-1), INVALID), (dict(heads=65536), UNSUPPORTED),
    (dict(dk=64), UNSUPPORTED), (dict(dk=96, dv=96), UNSUPPORTED), (dict(in_dtype=2), INVALID), (dict(out_dtype=2), INVALID), (dict(num_seqs=3), INVALID),
    (dict(scale=float("nan")), INVALID), (dict(batch=1 << 20, num_seqs=1 << 20, heads=32), UNSUPPORTED)])
def test_tree_steps_and_commit_refuse_dims(change, status):
    assert _steps(_dims(**change)) == status and kda.kda_last_error()
    assert _commit(_dims(**change)) == status


def test_tree_steps_and_commit_refuse_pointers():
    for name in ("q", "k", "v", "la", "beta", "S", "parents", "o"):
        assert _steps(**{name: None}) == INVALID and _steps(**{name: SOME + 1}) == INVALID
    for name in ("k", "v", "la", "beta", "S", "kept"):
        assert _commit(**{name: None}) == INVALID and _commit(**{name: SOME + 1}) == INVALID
    assert _steps(idx=SOME + 2) == INVALID and _steps(flags=2) == INVALID and _steps(la=SOME + 2) == INVALID and _commit(flags=4) == INVALID
    assert _commit(most=65) == UNSUPPORTED and _commit(most=-1) == INVALID
    assert _lib().kda_tree_steps(None, *([SOME] * 9), 0, None) == INVALID and _lib().kda_tree_commit(None, *([SOME] * 7), 8, 0, None) == INVALID
    assert _steps(_dims(seqlen=0)) == 0 and _steps(_dims(heads=0)) == 0 and _commit(most=0) == 0 and _commit(_dims(batch=0, num_seqs=0)) == 0


def test_the_binding_refuses_what_is_not_on_a_device_or_of_another_kind():
    t = lambda *shape, dtype=torch.bfloat16: torch.zeros(*shape, dtype=dtype)
    i = lambda *shape: t(*shape, dtype=torch.int32)
    with pytest.raises(ValueError, match="device"):
        kda.kda_rotate(t(1, 2, 2, 64), None, i(1, 2), t(32, dtype=torch.float32))
    with pytest.raises(ValueError, match="device"):
        kda.kda_tree_steps(t(1, 2, 2, 64), t(1, 2, 2, 64), t(1, 2, 2, 64), t(1, 2, 2, 64), t(1, 2, 2), t(1, 2, 64, 64, dtype=torch.float32), i(1, 2))
    with pytest.raises(ValueError):
        kda.kda_pages_fork(i(2, 3), i(5).long(), i(2))
    with pytest.raises(ValueError):
        kda.kda_pages_reserve(i(2, 3).long(), i(2), i(2), i(5), 16)
    with pytest.raises(ValueError, match="device"):
        kda.kda_pages_compact(i(2, 3), i(5))


def test_tables_too_large_for_a_launch_are_refused():
    def reserve(n, cols):
        return _lib().kda_pages_reserve(SOME, n, cols, 64, SOME, 10, SOME, SOME, SOME, SOME, SOME, ctypes.c_size_t(0), None)
    # (one workgroup counts entries in steps of 1024, in 32 bits)
    assert reserve(1, 2 ** 31 - 1) == UNSUPPORTED and reserve(1, 2 ** 31 - 1024) == UNSUPPORTED and reserve(8192, 262144) == UNSUPPORTED
    assert reserve(1, 2 ** 31 - 1025) == WORKSPACE and reserve(8192, 262143) == WORKSPACE
    fork = lambda n, cols: _lib().kda_pages_fork(SOME, n, cols, SOME, 10, SOME, None)
    assert fork(1, 2 ** 31 - 1) == UNSUPPORTED and fork(8192, 1 << 24) == UNSUPPORTED and fork(1, 16 * (1 << 24) - 15) == UNSUPPORTED
    assert kda.kda_last_error()
