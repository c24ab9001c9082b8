"""The softmax-attention layer of a hybrid stack from prompt to answer, beside a KDA layer: a packed prefill, the prompt's keys into the paged
cache, then decode steps of one token and of drafts, as a serving program runs them; every step against the oracle on the same state."""
import numpy as np
import pytest
import torch

import oracle
import synth_inputs as si
from oracle import softmax_attention as sa
from test_gpu_cache import HALF, TERMS, Pool, _freqs, _np, _tokens

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("window,sinks", [(0, 0), (48, 4)])
def test_prompt_then_decode(window, sinks):
    import paper_2510_26692_amd as kda
    prompts, Hq, Hk, d, page = [70, 5, 130], 4, 2, 128, 32
    N, cu = len(prompts), np.concatenate([[0], np.cumsum(prompts)])
    pool, freqs = Pool(N, Hk, d, page, max(prompts) + 32, 1), _freqs(d // 2)
    kd, vd, ksd, vsd, table = pool.device()
    f = torch.from_numpy(freqs).cuda()
    cud = torch.tensor(cu, dtype=torch.int32, device="cuda")
    lens = torch.zeros(N, dtype=torch.int32, device="cuda")
    host_lens = [0] * N

    # ---- prompt: rotate, store, attend on the rotated bf16 keys ----
    q, k, v = (_tokens(1, int(cu[-1]), h, d, i) for i, h in enumerate((Hq, Hk, Hk)))
    q_rot, k_rot = kda.kda_cache_append(k.cuda(), v.cuda(), kd, vd, ksd, vsd, table, lens, cu_seqlens=cud, inv_freq=f, q=q.cuda(), want_k=True)
    o, _ = kda.kda_window_attn_fwd(q_rot, k_rot, v.cuda(), window=window, sinks=sinks, cu_seqlens=cud)
    ref = sa.attention(_np(q_rot), _np(k_rot), _np(v), window, sinks, cu)
    assert (np.abs(_np(o) - ref["o"]) <= TERMS * ref["o_bound"] * (1 + HALF) + 2.0 ** -20 * np.abs(ref["o"])).all()
    pos = np.concatenate([np.arange(n) for n in prompts])
    exact = sa.rotate(_np(k[0]), pos, freqs)[None]
    sa.append(exact.astype(np.float32), _np(v).astype(np.float32), pool.k, pool.v, pool.ks, pool.vs, pool.table, host_lens, cu)
    lens += torch.tensor(prompts, dtype=torch.int32, device="cuda")
    host_lens = list(prompts)

    # ---- the KDA layer beside it keeps its own states ----
    S = si.make_state(N, Hq, d, d, 0.02, 7)
    S_dev, S_ref = S.cuda().clone(), S.numpy().astype(np.float64)
    for step, Tq in enumerate((1, 1, 4, 1, 8)):
        tok = si.make_decode_tokens(N, Hq, d, d, "bf16", -2.0, 100, step)
        got = kda.kda_recurrent_step(*(tok[n].cuda() for n in ("q", "k", "v", "log_alpha", "beta")), S_dev)
        want, S_ref = oracle.kda_step(*(si.to_np32(tok[n]) for n in ("q", "k", "v", "log_alpha", "beta")), S_ref)
        assert np.abs(_np(got) - want).max() <= 1e-5 * np.abs(want).max()

        q, k, v = (_tokens(N, Tq, h, d, 50 + 3 * step + i) for i, h in enumerate((Hq, Hk, Hk)))
        q_rot, _ = kda.kda_cache_append(k.cuda(), v.cuda(), kd, vd, ksd, vsd, table, lens, inv_freq=f, q=q.cuda())
        lens += Tq
        o = kda.kda_cache_attn(q_rot, kd, vd, ksd, vsd, table, lens, window=window, sinks=sinks, max_kv_len=max(host_lens) + Tq)
        exact = np.stack([sa.rotate(_np(k[n]), host_lens[n] + np.arange(Tq), freqs) for n in range(N)])
        sa.append(exact.astype(np.float32), _np(v).astype(np.float32), pool.k, pool.v, pool.ks, pool.vs, pool.table, host_lens)
        host_lens = [n + Tq for n in host_lens]
        np.testing.assert_array_equal(kd.view(torch.uint8).cpu().numpy(), pool.k)
        np.testing.assert_array_equal(vsd.cpu().numpy(), pool.vs)
        ref, bound = sa.cache_attention(_np(q_rot), pool.k, pool.v, pool.ks, pool.vs, pool.table, host_lens, window, sinks)
        assert (np.abs(_np(o) - ref) <= TERMS * bound * (1 + HALF) + 2.0 ** -20 * np.abs(ref)).all(), step


def test_decode_over_the_cache_is_the_prefill_up_to_the_codes():
    """The last rows of a prefill against the same tokens attended over the cache: they differ by the codes' rounding alone.  With values that are
    codes already (small whole numbers, no rotation) nothing is lost, and both agree within their softmax terms' rounding."""
    import paper_2510_26692_amd as kda
    T, Tq, Hq, Hk, d = 300, 8, 8, 2, 64
    g = torch.Generator().manual_seed(1)
    k, v = (torch.randint(-8, 9, (1, T, Hk, d), generator=g).to(torch.bfloat16).cuda() for _ in range(2))
    q = (torch.randn(1, T, Hq, d, generator=g) * 0.2).to(torch.bfloat16).cuda()
    pool = Pool(1, Hk, d, 64, T, 2)
    kd, vd, ksd, vsd, table = pool.device()
    lens = torch.zeros(1, dtype=torch.int32, device="cuda")
    kda.kda_cache_append(k, v, kd, vd, ksd, vsd, table, lens)
    for window, sinks in ((0, 0), (100, 3)):
        full, _ = kda.kda_window_attn_fwd(q, k, v, window=window, sinks=sinks)
        tail = kda.kda_cache_attn(q[:, -Tq:], kd, vd, ksd, vsd, table, lens + T, window=window, sinks=sinks)
        bound = sa.attention(_np(q), _np(k), _np(v), window, sinks)["o_bound"][:, -Tq:]
        assert (np.abs(_np(full[:, -Tq:]) - _np(tail)) <= 2 * TERMS * bound * (1 + HALF)).all()


def test_training_step_descends():
    """Forward and backward of the layer as a step uses them: moving along the negative gradient changes the loss by minus the step times the
    gradient's square, to the first order."""
    import paper_2510_26692_amd as kda
    B, T, Hq, Hk, d = 2, 150, 4, 2, 64
    g = torch.Generator().manual_seed(3)
    x = {n: torch.randn(B, T, h, d, generator=g).to(torch.bfloat16).cuda() for n, h in (("q", Hq), ("k", Hk), ("v", Hk))}
    do = torch.randn(B, T, Hq, d, generator=g).to(torch.bfloat16).cuda()
    kw = dict(window=40, sinks=2)
    o, lse = kda.kda_window_attn_fwd(x["q"], x["k"], x["v"], out_dtype=torch.bfloat16, **kw)
    grad = kda.kda_window_attn_bwd(x["q"], x["k"], x["v"], o, lse, do, **kw)
    ref = sa.attention_backward(*(_np(t) for t in (x["q"], x["k"], x["v"], do)), **kw)
    for n in ("q", "k", "v"):
        # along u = the kernel's gradient, the exact slope (of the oracle's gradient) is the kernel's squared length, within their error
        u, exact = _np(grad["d" + n]), ref["d" + n]
        assert abs((u * exact).sum() / (u * u).sum() - 1) < 0.01
        e = 1e-3 / np.abs(u).max()
        loss = lambda s: (sa.attention(*(_np(x[m]) + (s * u if m == n else 0) for m in ("q", "k", "v")), **kw)["o"] * _np(do)).sum()
        assert abs((loss(e) - loss(-e)) / (2 * e) / (u * u).sum() - 1) < 0.01
