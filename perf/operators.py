"""The softmax-attention layers of a hybrid stack, next to Kimi Delta Attention: attention with a sliding window and sinks (training
and prefill), the rotated append to a paged 8-bit cache, and attention over that cache.

A case is a dict of plain values:

    op       "train"   kda_window_attn_fwd and kda_window_attn_bwd: o, lse and the gradients of q, k, v
             "prefill" kda_window_attn_fwd: o and lse
             "append"  kda_cache_append: keys and values of new tokens into the cache, keys and queries rotated on the way
             "attend"  kda_cache_attn: the newest tokens of every sequence over the cache
    rows     batch rows or sequences
    tokens   tokens of a row (train, prefill); new tokens per sequence (append, attend); the upper bound of a packed sequence's
    shortest, lengths_seed   with shortest > 0 the batch is packed, its lengths uniform in [shortest, tokens] from that seed
    heads, kv_heads, dim     query heads, key and value heads, head dimension
    window, sinks            visible tokens before a query, itself included (0: all); first tokens that stay visible
    cached, page             append, attend: sequences hold up to that many tokens (uniform from half of it on), in pages of `page`
    rope                     append: "half" (channels i and i + dim / 2 turn together) or "pairs" (2 i and 2 i + 1)
"""
import math
import random

import numpy as np
import torch

own = False
DEV = "cuda"
SINKS = 4
ROPE_BASE = 10000.0


def _case(name, op, rows, tokens, heads, kv_heads, dim=128, shortest=0, lengths_seed=0, window=0, sinks=0, cached=0, page=0, rope=""):
    c = dict(op=op, rows=rows, tokens=tokens, shortest=shortest, lengths_seed=lengths_seed, heads=heads, kv_heads=kv_heads, dim=dim,
             window=window, sinks=sinks, cached=cached, page=page, rope=rope)
    return dict(c, name=name) if name else c


def listed():
    return [
        # a small model's step on two short rows: latency counts
        _case("train_small", "train", 2, 200, 4, 4, dim=64),
        # four 4096-token rows, plain causal attention: the ordinary training step
        _case("train_rows", "train", 4, 4096, 16, 4),
        # documents of mixed lengths packed into one stream, local layers with sinks
        _case("train_packed_window", "train", 8, 4096, 32, 8, shortest=512, lengths_seed=1, window=1024, sinks=SINKS),
        # a short prompt of ragged length: the first answer waits for it
        _case("prefill_short_prompt", "prefill", 1, 333, 32, 8),
        # eight prompts of mixed lengths packed into one stream
        _case("prefill_packed", "prefill", 8, 4096, 32, 8, shortest=512, lengths_seed=2),
        # a long document through a local layer
        _case("prefill_long_window", "prefill", 1, 65536, 16, 2, window=1024, sinks=SINKS),
        # one user's chat turn being decoded: the new token's keys and values (latency counts)
        _case("append_one", "append", 1, 1, 32, 8, cached=2000, page=64, rope="half"),
        # a serving batch in speculative decoding: four draft tokens a sequence
        _case("append_drafts", "append", 256, 4, 32, 8, cached=4096, page=64, rope="half"),
        # prompts of a second turn behind what the cache holds of the first
        _case("append_prompts", "append", 16, 8192, 32, 8, shortest=512, lengths_seed=3, cached=512, page=64, rope="pairs"),
        # one user's chat turn being decoded: latency counts
        _case("attend_one", "attend", 1, 1, 32, 8, cached=2000, page=64),
        # a serving batch of ragged contexts
        _case("attend_batch", "attend", 256, 1, 32, 8, cached=8192, page=64),
        # long documents, four draft tokens each to verify
        _case("attend_long_drafts", "attend", 4, 4, 32, 8, cached=131072, page=128),
    ]


def _log_int(rng, low, high):
    return max(low, min(high, round(math.exp(rng.uniform(math.log(low), math.log(high))))))


def draw(rng):
    op = rng.choice(["train", "train", "prefill", "append", "attend", "attend"])
    kv_heads = rng.choice([1, 2, 4, 8])
    heads = kv_heads * rng.choice([1, 2, 4, 5, 8])
    heads = heads if heads <= 32 else kv_heads * 4
    dim = rng.choice([64, 128, 128])
    if op in ("train", "prefill"):
        window = rng.choice([0, _log_int(rng, 16, 4096)])
        sinks = rng.choice([0, 1, SINKS, 64]) if window else 0
        tokens = _log_int(rng, 17, 4096 if not window or window > 2048 else 16384)
        # (what the plain form holds of the scores: at most what the largest listed cases of the kind make it hold)
        width = tokens if not window or window >= tokens else 2 * window + sinks
        rows = _log_int(rng, 1, max(1, min(16, (1 << 30) // (heads * tokens * width))))
        shortest = rng.choice([0, max(1, tokens // 8)]) if rows > 1 else 0
        return _case("", op, rows, tokens, heads, kv_heads, dim=dim, shortest=shortest, lengths_seed=rng.randrange(1 << 20), window=window, sinks=sinks)
    page = rng.choice([16, 32, 64, 128])
    if op == "append":
        if rng.random() < 0.5:
            rows, tokens, shortest = _log_int(rng, 1, 512), rng.randint(1, 8), 0
        else:
            rows, tokens = _log_int(rng, 1, 16), _log_int(rng, 9, 8192)
            shortest = rng.choice([0, max(1, tokens // 16)])
        return _case("", op, rows, tokens, heads, kv_heads, dim=dim, shortest=shortest, lengths_seed=rng.randrange(1 << 20),
                     cached=_log_int(rng, 1, 2000), page=page, rope=rng.choice(["half", "pairs"]))
    cached = _log_int(rng, 1, 131072)
    rows = _log_int(rng, 1, max(1, min(256, (1 << 21) // cached)))
    window = rng.choice([0, 0, _log_int(rng, 16, 8192)])
    return _case("", op, rows, rng.choice([1, 1, 2, 4, 7, 8]), heads, kv_heads, dim=dim, lengths_seed=rng.randrange(1 << 20), cached=cached,
                 page=page, window=window, sinks=rng.choice([0, SINKS, 64]) if window else 0)


def _lengths(c):
    """New tokens of every sequence."""
    if not c["shortest"]:
        return [c["tokens"]] * c["rows"]
    r = random.Random(c["lengths_seed"])
    return [r.randint(c["shortest"], c["tokens"]) for _ in range(c["rows"])]


def _held(c):
    """Tokens that every sequence has in the cache before its new ones."""
    r = random.Random(c["lengths_seed"] + 1)
    return [r.randint((c["cached"] + 1) // 2, c["cached"]) for _ in range(c["rows"])]


def _visible(first, count, window, sinks):
    """Visible (query, key) pairs of the queries at positions first .. first + count - 1."""
    seen = np.arange(first + 1, first + count + 1, dtype=np.int64)
    if window:
        far = np.maximum(seen - window, 0)
        seen = np.minimum(seen, window) + np.minimum(far, sinks)
    return int(seen.sum())


def work(c):
    d, hq, hk, t = c["dim"], c["heads"], c["kv_heads"], sum(_lengths(c))
    if c["op"] in ("train", "prefill"):
        pairs = sum(_visible(0, n, c["window"], c["sinks"]) for n in _lengths(c))
        q, kv = 2 * t * hq * d, 2 * t * hk * d
        if c["op"] == "prefill":
            return {"bytes": 2 * q + 2 * kv + 4 * t * hq, "flops": 4 * d * hq * pairs}
        return {"bytes": 4 * q + 4 * kv + 4 * t * hq, "flops": 14 * d * hq * pairs}
    if c["op"] == "append":
        return {"bytes": 4 * t * hq * d + 2 * t * hk * d * (4 if c["shortest"] else 3), "flops": 6 * t * (hq + hk) * d}
    held = _held(c)
    n, w, s = c["tokens"], c["window"], c["sinks"]
    keys = sum(h + n if not w else min(h + n, w + n - 1 + s) for h in held)
    return {"bytes": 2 * keys * hk * d + 4 * len(held) * n * hq * d, "flops": 4 * d * hq * sum(_visible(h, n, w, s) for h in held)}


def _normal(g, *shape, std=1.0):
    return (torch.randn(*shape, generator=g, device=DEV) * std).to(torch.bfloat16)


def prepare(case, seed):
    c = case
    g = torch.Generator(device=DEV).manual_seed(seed)
    d, hq, hk, lens = c["dim"], c["heads"], c["kv_heads"], _lengths(c)
    packed = c["shortest"] > 0
    batch, tokens = (1, sum(lens)) if packed else (c["rows"], c["tokens"])
    cu = torch.tensor(np.concatenate([[0], np.cumsum(lens)]), dtype=torch.int32, device=DEV) if packed else None
    st = {"case": c, "cu_seqlens": cu, "q": _normal(g, batch, tokens, hq, d, std=1.5)}
    if c["op"] in ("train", "prefill"):
        st.update(k=_normal(g, batch, tokens, hk, d), v=_normal(g, batch, tokens, hk, d))
        if c["op"] == "train":
            st["do"] = _normal(g, batch, tokens, hq, d)
        return st
    held, page = _held(c), c["page"]
    ahead = max(h + n for h, n in zip(held, lens))
    columns = -(-ahead // page)
    need = [-(-(h + n) // page) for h, n in zip(held, lens)]
    pages = sum(need) + 3                                 # (a pool is never full)
    order = torch.randperm(pages, generator=g, device=DEV).to(torch.int32)
    starts = np.concatenate([[0], np.cumsum(need)])
    at = torch.tensor(starts[:-1, None] + np.minimum(np.arange(columns)[None, :], np.array(need)[:, None] - 1), device=DEV)
    table = torch.where(torch.arange(columns, device=DEV)[None, :] < torch.tensor(need, device=DEV)[:, None], order[at], -1).to(torch.int32)
    shape = (pages, hk, page, d)
    # (codes of normal values: a page's largest is 224 to 448)
    st.update(block_table=table.contiguous(),
              k_cache=(torch.randn(shape, generator=g, device=DEV) * 90).clamp_(-448, 448).to(torch.float8_e4m3fn),
              v_cache=(torch.randn(shape, generator=g, device=DEV) * 90).clamp_(-448, 448).to(torch.float8_e4m3fn),
              k_scale=torch.pow(2.0, torch.randint(-8, -5, (pages, hk), generator=g, device=DEV).float()),
              v_scale=torch.pow(2.0, torch.randint(-8, -5, (pages, hk), generator=g, device=DEV).float()))
    if c["op"] == "append":
        st.update(k=_normal(g, batch, tokens, hk, d), v=_normal(g, batch, tokens, hk, d),
                  kv_lens=torch.tensor(held, dtype=torch.int32, device=DEV),
                  inv_freq=(ROPE_BASE ** (-torch.arange(0, d, 2, device=DEV, dtype=torch.float64) / d)).float())
    else:
        st["kv_lens"] = torch.tensor([h + n for h, n in zip(held, lens)], dtype=torch.int32, device=DEV)
        st["max_kv_len"] = ahead
    return st


def run(state):
    s, c = state, state["case"]
    return {"train": _train, "prefill": _prefill, "append": _append, "attend": _attend}[c["op"]](s, c)


def _train(s, c):
    if own:
        import paper_2510_26692_amd as kda
        kw = dict(window=c["window"], sinks=c["sinks"], cu_seqlens=s["cu_seqlens"])
        o, lse = kda.kda_window_attn_fwd(s["q"], s["k"], s["v"], out_dtype=torch.bfloat16, **kw)
        g = kda.kda_window_attn_bwd(s["q"], s["k"], s["v"], o, lse, s["do"], **kw)
        return {"o": o, "lse": lse, "dq": g["dq"], "dk": g["dk"], "dv": g["dv"]}
    q, k, v = (_rows(s, c, s[n]).requires_grad_() for n in "qkv")
    o, lse = _softmax_attention(q, k, v, c["window"], c["sinks"])
    dq, dk, dv = torch.autograd.grad(o, (q, k, v), _rows(s, c, s["do"]))
    return {"o": _unrows(s, c, o.detach()).bfloat16(), "lse": _unrows_lse(s, c, lse.detach()), "dq": _unrows(s, c, dq).bfloat16(),
            "dk": _unrows(s, c, dk).bfloat16(), "dv": _unrows(s, c, dv).bfloat16()}


def _prefill(s, c):
    if own:
        import paper_2510_26692_amd as kda
        o, lse = kda.kda_window_attn_fwd(s["q"], s["k"], s["v"], window=c["window"], sinks=c["sinks"], cu_seqlens=s["cu_seqlens"],
                                         out_dtype=torch.bfloat16)
        return {"o": o, "lse": lse}
    o, lse = _softmax_attention(*(_rows(s, c, s[n]) for n in "qkv"), c["window"], c["sinks"])
    return {"o": _unrows(s, c, o).bfloat16(), "lse": _unrows_lse(s, c, lse)}


def _place(s, c):
    """Where a packed batch's tokens stand in padded rows: (sequence, index) of every token."""
    cu = s["cu_seqlens"].long()
    token = torch.arange(s["q"].shape[1], device=DEV)
    seq = torch.searchsorted(cu, token, right=True) - 1
    return seq, token - cu[seq]


def _rows(s, c, x):
    """[rows, H, tokens, d] in 32 bits; a packed batch is padded with zeros, which no query that counts sees."""
    x = x.float()
    if s["cu_seqlens"] is not None:
        full = x.new_zeros(c["rows"], c["tokens"], *x.shape[2:])
        full[_place(s, c)] = x[0]
        x = full
    return x.transpose(1, 2)


def _unrows(s, c, x):
    x = x.transpose(1, 2)
    return x[_place(s, c)][None] if s["cu_seqlens"] is not None else x


def _unrows_lse(s, c, lse):
    """[rows, H, tokens] -> [batch, H, tokens]"""
    if s["cu_seqlens"] is None:
        return lse
    return lse.transpose(1, 2)[_place(s, c)].T.contiguous()[None]


def _softmax_attention(q, k, v, window, sinks):
    """o and the log-sum-exp, q [N,Hq,T,d], k and v [N,Hk,T,d], every query over the keys of its own and earlier tokens."""
    n, hq, t, d = q.shape
    hk = k.shape[1]
    if window == 0 or window >= t:
        i = torch.arange(t, device=DEV)
        seen = (i[None, :] <= i[:, None]).repeat(hq // hk, 1)                     # rows: (head of the group, token)
        x = torch.matmul(q.reshape(n, hk, hq // hk * t, d), k.transpose(2, 3)) * d ** -0.5
        o, lse = _softmax(x.masked_fill_(~seen, -math.inf), v)
        return o.reshape(n, hq, t, d), lse.reshape(n, hq, t)
    # blocks of `window` queries, each with its own block of keys, the block before and the sinks
    blocks = -(-t // window)
    pad = lambda x: torch.nn.functional.pad(x, (0, 0, 0, blocks * window - t))
    q4 = pad(q).reshape(n, hk, hq // hk, blocks, window, d).transpose(2, 3).reshape(n, hk, blocks, hq // hk * window, d)

    def near(x):
        own_block = pad(x).reshape(n, hk, blocks, window, d)
        before = torch.cat([torch.zeros_like(own_block[:, :, :1]), own_block[:, :, :-1]], 2)
        return torch.cat([x[:, :, None, :sinks].expand(-1, -1, blocks, -1, -1), before, own_block], 3)

    b, r = torch.arange(blocks, device=DEV)[:, None, None], torch.arange(window, device=DEV)[None, :, None]
    i, j = b * window + r, (b - 1) * window + torch.arange(2 * window, device=DEV)[None, None, :]
    j0 = torch.arange(min(sinks, t), device=DEV)[None, None, :]
    seen = torch.cat([(i - j0) >= window, (j >= 0) & (j <= i) & (i - j < window)], 2).repeat(1, hq // hk, 1)
    x = torch.matmul(q4, near(k).transpose(3, 4)) * d ** -0.5
    o, lse = _softmax(x.masked_fill_(~seen, -math.inf), near(v))
    back = lambda y, *last: y.reshape(n, hk, blocks, hq // hk, window, *last).transpose(2, 3).reshape(n, hq, blocks * window, *last)[:, :, :t]
    return back(o, d), back(lse)


def _softmax(x, v):
    """softmax(x) v and the log-sum-exp; every row has a visible key."""
    m = x.detach().amax(-1, keepdim=True)
    p = torch.exp(x - m)
    z = p.sum(-1, keepdim=True)
    return torch.matmul(p / z, v), (m + torch.log(z)).squeeze(-1)


def _append(s, c):
    d, page = c["dim"], c["page"]
    if own:
        import paper_2510_26692_amd as kda
        q, k = kda.kda_cache_append(s["k"], s["v"], s["k_cache"], s["v_cache"], s["k_scale"], s["v_scale"], s["block_table"], s["kv_lens"],
                                    cu_seqlens=s["cu_seqlens"], inv_freq=s["inv_freq"], interleaved=c["rope"] == "pairs", q=s["q"],
                                    want_k=c["shortest"] > 0)
        return [x for x in (q, k, s["k_cache"], s["v_cache"], s["k_scale"], s["v_scale"]) if x is not None]
    if s["cu_seqlens"] is not None:
        seq, index = _place(s, c)
    else:
        t = torch.arange(c["rows"] * c["tokens"], device=DEV)
        seq, index = t // c["tokens"], t % c["tokens"]
    old = s["kv_lens"].long()
    pos = old[seq] + index
    angle = pos.double()[:, None] * s["inv_freq"].double()
    cos, sin = torch.cos(angle)[:, None], torch.sin(angle)[:, None]

    def turned(x):
        x = x.reshape(-1, *x.shape[2:]).double()
        if c["rope"] == "pairs":
            a, b = x[..., 0::2], x[..., 1::2]
            return torch.stack([a * cos - b * sin, a * sin + b * cos], -1).flatten(-2).float()
        a, b = x[..., :d // 2], x[..., d // 2:]
        return torch.cat([a * cos - b * sin, a * sin + b * cos], -1).float()

    k = turned(s["k"])
    number = s["block_table"][seq, pos // page].long()
    pages = s["k_cache"].shape[0]
    fresh = torch.full((pages,), 1 << 40, dtype=torch.int64, device=DEV).scatter_reduce(0, number, pos, "amin")      # first new token
    kept = torch.where(fresh < 1 << 40, fresh % page, 0)                                                              # older tokens of a page
    out = []
    for x, cache, scale in ((k, s["k_cache"], s["k_scale"]), (s["v"].reshape(k.shape).float(), s["v_cache"], s["v_scale"])):
        top = torch.zeros_like(scale).scatter_reduce(0, number[:, None].expand(-1, x.shape[1]), x.abs().amax(-1), "amax")
        m, e = torch.frexp(top)                            # the smallest power of two with top <= 448 of it
        least = torch.ldexp(torch.ones_like(m), torch.where(m <= 0.875, e - 9, e - 8))
        new = torch.where((kept > 0)[:, None], torch.maximum(scale, least), least)
        new = torch.where((fresh < 1 << 40)[:, None], new, scale)
        grown = torch.nonzero(((kept > 0)[:, None] & (new > scale)).any(1))[:, 0]
        if len(grown):
            again = (cache[grown].float() * (scale / new)[grown][:, :, None, None]).to(cache.dtype)
            older = torch.arange(page, device=DEV)[None, None, :, None] < kept[grown][:, None, None, None]
            cache.view(torch.uint8)[grown] = torch.where(older, again.view(torch.uint8), cache.view(torch.uint8)[grown])
        scale.copy_(new)
        cache.view(torch.uint8)[number, :, pos % page] = (x / new[number][..., None]).to(cache.dtype).view(torch.uint8)
        out += [cache]
    q = turned(s["q"]).bfloat16().reshape(s["q"].shape)
    return [q] + ([k.bfloat16().reshape(s["k"].shape)] if c["shortest"] else []) + [s["k_cache"], s["v_cache"], s["k_scale"], s["v_scale"]]


def _attend(s, c):
    if own:
        import paper_2510_26692_amd as kda
        return kda.kda_cache_attn(s["q"], s["k_cache"], s["v_cache"], s["k_scale"], s["v_scale"], s["block_table"], s["kv_lens"],
                                  window=c["window"], sinks=c["sinks"], max_kv_len=s["max_kv_len"], out_dtype=torch.bfloat16)
    n, t, hq, d = s["q"].shape
    hk, page = c["kv_heads"], c["page"]
    length = s["block_table"].shape[1] * page
    number = s["block_table"].long().clamp(min=0)

    def held(cache, scale):                                # [n, hk, length, d]
        x = cache[number].float() * scale[number][..., None, None]
        return x.transpose(1, 2).reshape(n, hk, length, d)

    q = s["q"].float().transpose(1, 2).reshape(n, hk, hq // hk * t, d)
    i = s["kv_lens"].long()[:, None] - t + torch.arange(t, device=DEV)
    i = i.repeat(1, hq // hk)[:, None, :, None]
    j = torch.arange(length, device=DEV)
    seen = j <= i
    if c["window"]:
        seen &= (i - j < c["window"]) | (j < c["sinks"])
    x = torch.matmul(q, held(s["k_cache"], s["k_scale"]).transpose(2, 3)) * d ** -0.5
    o, _ = _softmax(x.masked_fill_(~seen, -math.inf), held(s["v_cache"], s["v_scale"]))
    return o.reshape(n, hq, t, d).transpose(1, 2).bfloat16()


def exact(case, seed):
    """The definitions, in 64 bits: one sequence and a stretch of queries at a time, with every key."""
    c, s = case, prepare(case, seed)
    return {"train": _exact_attention, "prefill": _exact_attention, "append": _exact_append, "attend": _exact_attend}[c["op"]](s, c)


def _bounds(s, c):
    if s["cu_seqlens"] is None:
        return [(b, 0, c["tokens"]) for b in range(c["rows"])]
    cu = s["cu_seqlens"].tolist()
    return [(0, a, b) for a, b in zip(cu[:-1], cu[1:])]


def _allowed(i, j, window, sinks):
    ok = j <= i
    return ok & ((i - j < window) | (j < sinks)) if window else ok


def _exact_attention(s, c):
    flops = work(c)["flops"]
    dense = sum(4.0 * c["dim"] * c["heads"] * n * n for n in _lengths(c)) * (3 if c["op"] == "train" else 1)
    if dense > 6e13 and flops < dense / 4:
        return None                                        # (nearly all of it masked)
    group, scale = c["heads"] // c["kv_heads"], 1 / math.sqrt(c["dim"])
    out = {"o": torch.zeros(s["q"].shape, dtype=torch.float64, device=DEV),
           "lse": torch.zeros(s["q"].shape[0], c["heads"], s["q"].shape[1], dtype=torch.float64, device=DEV)}
    if c["op"] == "train":
        out.update({"d" + n: torch.zeros(s[n].shape, dtype=torch.float64, device=DEV) for n in "qkv"})
    for b, start, end in _bounds(s, c):
        n = end - start
        step = max(1, min(n, (1 << 28) // n))
        for h in range(c["heads"]):
            q, k, v = (s[x][b, start:end, h if x == "q" else h // group].double() for x in "qkv")
            for a in range(0, n, step):
                e = min(n, a + step)
                i, j = torch.arange(a, e, device=DEV)[:, None], torch.arange(e, device=DEV)[None, :]
                x = scale * (q[a:e] @ k[:e].T)
                x[~_allowed(i, j, c["window"], c["sinks"])] = -math.inf
                lse = torch.logsumexp(x, 1)
                p = torch.exp(x - lse[:, None])
                o = p @ v[:e]
                out["o"][b, start + a:start + e, h], out["lse"][b, h, start + a:start + e] = o, lse
                if c["op"] == "train":
                    do = s["do"][b, start + a:start + e, h].double()
                    ds = p * (do @ v[:e].T - (do * o).sum(1, keepdim=True)) * scale
                    out["dv"][b, start:start + e, h // group] += p.T @ do
                    out["dk"][b, start:start + e, h // group] += ds.T @ q[a:e]
                    out["dq"][b, start + a:start + e, h] = ds @ k[:e]
    return out


def _exact_append(s, c):
    page, table = c["page"], s["block_table"].cpu().numpy()
    inv = s["inv_freq"].double()
    pages = [s[x].double() for x in ("k_cache", "v_cache")]
    scales = [s[x].double() for x in ("k_scale", "v_scale")]
    turned = {x: torch.zeros(s[x].shape, dtype=torch.float64, device=DEV) for x in "qk"}
    held = s["kv_lens"].tolist()
    for n, (b, start, end) in enumerate(_bounds(s, c)):
        z = torch.exp(1j * (torch.arange(held[n], held[n] + end - start, device=DEV, dtype=torch.float64)[:, None] * inv))[:, None]
        for x in "qk":
            y = s[x][b, start:end].double()
            half = c["dim"] // 2
            w = (torch.complex(y[..., 0::2], y[..., 1::2]) if c["rope"] == "pairs" else torch.complex(y[..., :half], y[..., half:])) * z
            turned[x][b, start:end] = torch.view_as_real(w).flatten(-2) if c["rope"] == "pairs" else torch.cat([w.real, w.imag], -1)
        first, last = held[n], held[n] + end - start
        for p in range(first // page, (last - 1) // page + 1):
            a, e = max(first, p * page), min(last, (p + 1) * page)
            at, kept = int(table[n, p]), max(0, first - p * page)
            for x, cache, scale in zip((turned["k"], s["v"].double()), pages, scales):
                y = x[b, start + a - first:start + e - first]                    # [tokens, heads, d]
                least = 2.0 ** torch.ceil(torch.log2(y.abs().amax((0, 2)) / 448))
                new = torch.maximum(least, scale[at]) if kept else least
                cache[at, :, :kept] = (cache[at, :, :kept] * (scale[at] / new)[:, None, None]).float().to(torch.float8_e4m3fn).double()
                cache[at, :, a % page:a % page + e - a] = (y / new[:, None]).transpose(0, 1).float().to(torch.float8_e4m3fn).double()
                scale[at] = new
    return [turned["q"]] + ([turned["k"]] if c["shortest"] else []) + pages + scales


def _exact_attend(s, c):
    group, page = c["heads"] // c["kv_heads"], c["page"]
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device=DEV)
    for n, length in enumerate(s["kv_lens"].tolist()):
        at = s["block_table"][n, :-(-length // page)].long()
        i = torch.arange(length - c["tokens"], length, device=DEV)[:, None]
        seen = _allowed(i, torch.arange(length, device=DEV)[None, :], c["window"], c["sinks"])
        for h in range(c["kv_heads"]):
            k, v = ((s[x + "_cache"][at, h].double() * s[x + "_scale"][at, h].double()[:, None, None]).flatten(0, 1)[:length] for x in "kv")
            q = s["q"][n, :, h * group:(h + 1) * group].double().transpose(0, 1)                   # [group, t, d]
            x = (q.reshape(-1, c["dim"]) @ k.T).reshape(group, c["tokens"], length) / math.sqrt(c["dim"])
            p = torch.softmax(x.masked_fill(~seen, -math.inf), -1)
            out[n, :, h * group:(h + 1) * group] = (p.reshape(-1, length) @ v).reshape(group, c["tokens"], c["dim"]).transpose(0, 1)
    return out
