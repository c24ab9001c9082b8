"""Draft trees in a hybrid stack, and the pages behind them: rotation by positions of several axes, attention of drafted trees over a paged
8-bit cache, Kimi Delta Attention over the same trees, and the bookkeeping of accepted tokens and of shared pages.

A case is a dict of plain values:

    op       "rotate"  kda_rotate: queries and keys turned by their positions, with `grads` their gradients turned back too
             "attend"  kda_cache_tree_attn: the drafted tokens of every sequence over the cache
             "keep"    kda_cache_keep: the accepted tokens' codes move up to the end of what was there, in every layer
             "fork"    kda_pages_fork, kda_pages_reserve, kda_cache_copy_pages: a step of beam search, up to the new token's place
             "compact" kda_pages_compact, kda_cache_copy_pages: the pages in use move to the front of the pool
             "delta"   kda_tree_steps, kda_tree_commit: the drafted tokens over the recurrent states, then the accepted ones into them
    rows     sequences
    tokens   tokens of a row (rotate), drafted tokens of a sequence (attend, keep, delta), tokens to make room for (fork)
    spread   a drafted token's parent is one of the `spread` tokens before it (1: a chain)
    fewest   with 0 < fewest < tokens, sequences have between that and `tokens` drafted tokens
    sizes_seed                   where lengths, trees, accepted paths and tables come from
    heads, kv_heads, dim, dtype  query heads, key and value heads (delta: heads alone), head dimension, type of the inputs
    window, sinks                attend: visible tokens before a token, itself included (0: all); first tokens that stay visible
    cached, page, layers         sequences hold up to that many tokens (uniform from half of it on), in pages of `page`; layers of a cache
    axes, rope                   rotate: axes of a position; "half" (channels i and i + dim / 2 turn together) or "pairs" (2 i and 2 i + 1)
    beams, pool                  fork: beams of a request (rows are requests times beams); compact: pages of the pool
"""
import math
import random

import numpy as np
import torch

own = False
DEV = "cuda"
SINKS = 4
ROPE_BASE = 10000.0
_TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


def _case(name, op, rows, tokens, heads, kv_heads=0, dim=128, dtype="bf16", spread=0, fewest=0, sizes_seed=0, window=0, sinks=0, cached=0,
          page=0, layers=1, axes=1, rope="", grads=False, beams=1, pool=0):
    c = dict(op=op, rows=rows, tokens=tokens, spread=spread, fewest=fewest, sizes_seed=sizes_seed, heads=heads, kv_heads=kv_heads, dim=dim,
             dtype=dtype, window=window, sinks=sinks, cached=cached, page=page, layers=layers, axes=axes, rope=rope, grads=grads, beams=beams,
             pool=pool)
    return dict(c, name=name) if name else c


def listed():
    return [
        # one user's draft tree: its queries and keys at the positions of their depths (latency counts)
        _case("rotate_tree", "rotate", 1, 16, 32, 8, rope="half"),
        # a training step over text and images: time, height and width
        _case("rotate_train_axes", "rotate", 4, 4096, 32, 8, axes=3, rope="half", grads=True),
        # one user's draft tree over a chat's context (latency counts)
        _case("attend_tree_one", "attend", 1, 16, 32, 8, spread=4, sizes_seed=1, cached=2000, page=64),
        # a serving batch, ragged contexts and trees
        _case("attend_tree_batch", "attend", 64, 32, 32, 8, spread=8, fewest=20, sizes_seed=2, cached=8192, page=64),
        # long documents, the largest trees
        _case("attend_tree_long", "attend", 4, 64, 32, 8, spread=16, sizes_seed=3, cached=131072, page=128),
        # the accepted path of one user's tree, every attention layer of a stack
        _case("keep_one", "keep", 1, 16, 0, 8, spread=4, sizes_seed=17, cached=2000, page=64, layers=8),
        # the accepted paths of a serving batch
        _case("keep_batch", "keep", 64, 32, 0, 8, spread=8, sizes_seed=5, cached=256, page=64, layers=16),
        # a step of beam search, four beams to each of 32 requests
        _case("fork_beams", "fork", 128, 1, 0, 8, sizes_seed=6, cached=1024, page=64, layers=8, beams=4),
        # half of a pool is in use, all over it
        _case("compact_pool", "compact", 64, 0, 0, 8, sizes_seed=7, page=64, layers=4, pool=4000),
        # one user's draft tree over the recurrent states (latency counts)
        _case("delta_tree_one", "delta", 1, 16, 32, spread=4, sizes_seed=8),
        # a serving batch of small trees
        _case("delta_tree_batch", "delta", 256, 16, 32, spread=4, fewest=9, sizes_seed=9),
        # the largest trees
        _case("delta_tree_large", "delta", 64, 64, 32, spread=16, sizes_seed=10),
    ]


def _log_int(rng, low, high):
    return max(low, min(high, round(math.exp(rng.uniform(math.log(low), math.log(high))))))


def draw(rng):
    op = rng.choice(["rotate", "attend", "attend", "keep", "fork", "compact", "delta", "delta"])
    kv_heads = rng.choice([1, 2, 4, 8])
    heads = min(32, kv_heads * rng.choice([1, 2, 4, 5, 8]))
    heads = heads if heads % kv_heads == 0 else kv_heads
    dim, seed = rng.choice([64, 128, 128]), rng.randrange(1 << 20)
    if op == "rotate":
        tokens = _log_int(rng, 1, 16384)
        return _case("", op, _log_int(rng, 1, max(1, min(16, 16384 // tokens))), tokens, heads, kv_heads, dim=dim, sizes_seed=seed,
                     dtype=rng.choice(["bf16", "bf16", "f32"]), axes=rng.randint(1, 4), rope=rng.choice(["half", "pairs"]),
                     grads=rng.random() < 0.5)
    tokens = _log_int(rng, 2, 64)
    spread, fewest = rng.choice([1, 2, 4, 16, 64]), rng.choice([0, 0, (tokens + 1) // 2])
    if op == "delta":
        return _case("", op, _log_int(rng, 1, max(1, min(256, 4096 // tokens))), tokens, rng.choice([1, 4, 16, 32]), dim=dim, spread=spread,
                     fewest=fewest, sizes_seed=seed, dtype=rng.choice(["bf16", "bf16", "f32"]))
    page = rng.choice([16, 32, 64, 128])
    if op == "attend":
        cached = _log_int(rng, 1, 131072)
        rows = _log_int(rng, 1, max(1, min(64, (1 << 19) // cached)))
        window = rng.choice([0, 0, _log_int(rng, 4, 8192)])
        return _case("", op, rows, tokens, heads, kv_heads, dim=dim, spread=spread, fewest=fewest, sizes_seed=seed, cached=cached, page=page,
                     window=window, sinks=rng.choice([0, SINKS, 64]) if window else 0)
    layers = rng.randint(1, 16)
    if op == "keep":
        return _case("", op, _log_int(rng, 1, 64), tokens, 0, kv_heads, dim=dim, spread=spread, fewest=fewest, sizes_seed=seed,
                     cached=_log_int(rng, 1, 256), page=page, layers=layers)
    layers = rng.randint(1, 4)
    if op == "fork":
        beams = rng.randint(2, 8)
        return _case("", op, beams * _log_int(rng, 1, 32), rng.choice([1, 1, 4, 40]), 0, kv_heads, dim=dim, sizes_seed=seed,
                     cached=_log_int(rng, 1, 1024), page=page, layers=layers, beams=beams)
    return _case("", op, _log_int(rng, 1, 64), 0, 0, kv_heads, dim=dim, sizes_seed=seed, page=page, layers=layers,
                 pool=_log_int(rng, 64, 256000 // page))


def _sizes(c):
    """Drafted tokens of every sequence, and the tokens that it held before them."""
    r = random.Random(c["sizes_seed"])
    drafted = [r.randint(c["fewest"], c["tokens"]) if c["fewest"] else c["tokens"] for _ in range(c["rows"])]
    if c["op"] == "fork":                                  # (the beams of a request are of one length)
        held = [n for _ in range(c["rows"] // c["beams"]) for n in [r.randint((c["cached"] + 1) // 2, c["cached"])] * c["beams"]]
    else:
        held = [r.randint((c["cached"] + 1) // 2, c["cached"]) for _ in range(c["rows"])] if c["cached"] else [0] * c["rows"]
    return drafted, held


def _trees(c):
    """Parents [rows][tokens] (-1: the context, -2: no token), depths, and the accepted path of every tree (-1 behind its end)."""
    r = random.Random(c["sizes_seed"] + 1)
    drafted, _ = _sizes(c)
    parents, depths = np.full((c["rows"], c["tokens"]), -2), np.zeros((c["rows"], c["tokens"]), dtype=np.int64)
    kept = np.full((c["rows"], c["tokens"]), -1)
    for n, count in enumerate(drafted):
        for t in range(count):
            parents[n, t] = -1 if t == 0 else r.randint(max(0, t - c["spread"]), t - 1)
            depths[n, t] = 0 if t == 0 else depths[n, parents[n, t]] + 1
        path, t = [], r.randrange(count)
        while t >= 0:
            path, t = [t] + path, parents[n, t]
        kept[n, :len(path)] = path
    return parents, depths, kept


def work(c):
    d, hq, hk, n = c["dim"], c["heads"], c["kv_heads"], c["rows"]
    size = 2 if c["dtype"] == "bf16" else 4
    if c["op"] == "rotate":
        t, passes = n * c["tokens"], 2 if c["grads"] else 1
        return {"bytes": passes * (2 * size * t * (hq + hk) * d + 4 * t * c["axes"]), "flops": passes * 3 * t * (hq + hk) * d}
    drafted, held = _sizes(c)
    if c["op"] == "attend":
        _, depths, _ = _trees(c)
        keys, pairs = 0, 0
        for i, (m, h) in enumerate(zip(drafted, held)):
            at = depths[i, :m]
            if not c["window"]:
                keys, pairs = keys + h + m, pairs + m * h + int((at + 1).sum())
            else:                                          # (context keys of the window and the sinks behind it, then ancestors)
                inside = np.clip(c["window"] - 1 - at, 0, h)
                pairs += int((inside + np.minimum(h - inside, c["sinks"])).sum() + np.minimum(at + 1, c["window"]).sum())
                near = min(h, max(0, c["window"] - 1))
                keys += near + min(h - near, c["sinks"]) + m
        return {"bytes": 2 * keys * hk * d + 4 * sum(drafted) * hq * d, "flops": 4 * d * hq * pairs}
    if c["op"] == "delta":
        _, depths, kept = _trees(c)
        m, state, steps = sum(drafted), hq * d * d, int((kept >= 0).sum())
        pairs = sum(int((depths[i, :x] + 1).sum()) for i, x in enumerate(drafted))
        return {"bytes": 3 * 4 * n * state + m * hq * (4 * size * d + size + 2 * d), "flops": 4 * m * state + 8 * pairs * hq * d + 7 * steps * state}
    token = 2 * 2 * c["layers"] * hk * d                   # a token's codes of keys and values, read and written
    if c["op"] == "keep":
        _, _, kept = _trees(c)
        moved = int((kept > np.arange(c["tokens"])[None, :]).sum())
        return {"bytes": moved * token + 4 * kept.size, "flops": moved * token / 2}
    if c["op"] == "fork":
        _, _, table, _, _, source, lens, _ = _fork_tables(c)
        copied = int((lens % c["page"] > 0).sum())          # (at most: a beam that is carried on alone keeps its page)
        return {"bytes": 2 * 4 * table.size + copied * c["page"] * token, "flops": 0}
    table, refs = _compact_tables(c)
    used = int((refs > 0).sum())
    moved = int((refs[:used] == 0).sum())
    return {"bytes": 2 * 4 * (table.size + refs.size) + moved * c["page"] * token, "flops": 0}


def _fork_tables(c):
    """A pool after some steps of beam search: the beams of a request share the pages of its prompt, each has its own behind them."""
    page, beams, r = c["page"], c["beams"], random.Random(c["sizes_seed"] + 2)
    _, held = _sizes(c)
    columns = -(-(c["cached"] + c["tokens"]) // page) + 1
    table = np.full((c["rows"], columns), -1)
    count = 0
    for i in range(0, c["rows"], beams):
        pages = -(-held[i] // page)
        shared = r.randint(0, max(0, pages - 1))           # (the last page is each beam's own)
        for b in range(beams):
            table[i + b, :shared] = np.arange(count, count + shared)
        count += shared
        for b in range(beams):
            table[i + b, shared:pages] = np.arange(count, count + pages - shared)
            count += pages - shared
    pool = count + c["rows"] * (-(-c["tokens"] // page) + 1) + 5
    order = np.array(r.sample(range(pool), pool))
    table = np.where(table >= 0, order[np.maximum(table, 0)], -1)
    refs = np.bincount(table[table >= 0], minlength=pool)
    source = np.array([i + r.randrange(beams) for i in range(0, c["rows"], beams) for _ in range(beams)])
    lens = np.array(held)
    return pool, columns, table, refs, order, source, lens, lens + c["tokens"]


def _compact_tables(c):
    """Sequences whose pages stand all over the pool, about half of which is free; some share their first pages."""
    r = random.Random(c["sizes_seed"] + 3)
    pool, rows = c["pool"], c["rows"]
    used = r.sample(range(pool), max(1, min(pool - 1, round(pool * r.uniform(0.4, 0.6)))))
    cuts = sorted(r.randint(0, len(used)) for _ in range(rows - 1))
    parts = [used[a:b] for a, b in zip([0] + cuts, cuts + [len(used)])]
    table = np.full((rows, max(len(p) for p in parts)), -1)
    for n, p in enumerate(parts):
        table[n, :len(p)] = p
    for n in range(1, rows, 5):                            # (forked from the row before, its first two pages)
        both = (table[n, :2] >= 0) & (table[n - 1, :2] >= 0)
        table[n, :2] = np.where(both, table[n - 1, :2], table[n, :2])
    return table, np.bincount(table[table >= 0], minlength=pool)


def _normal(g, *shape, std=1.0, dtype=torch.bfloat16):
    return (torch.randn(*shape, generator=g, device=DEV) * std).to(dtype)


def _device(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


def _codes(g, *shape):
    """Codes of normal values: a page's largest is 224 to 448."""
    out = torch.empty(shape, dtype=torch.float8_e4m3fn, device=DEV)
    for i in range(shape[0]):
        out[i] = (torch.randn(shape[1:], generator=g, device=DEV) * 90).clamp_(-448, 448).to(torch.float8_e4m3fn)
    return out


def _pool(g, c, pages):
    shape = (c["layers"], pages, c["kv_heads"], c["page"], c["dim"])
    scale = lambda: torch.pow(2.0, torch.randint(-8, -5, shape[:3], generator=g, device=DEV).float())
    return dict(k_cache=_codes(g, *shape), v_cache=_codes(g, *shape), k_scale=scale(), v_scale=scale())


def prepare(case, seed):
    c = case
    g = torch.Generator(device=DEV).manual_seed(seed)
    n, t, hq, hk, d, dtype = c["rows"], c["tokens"], c["heads"], c["kv_heads"], c["dim"], _TYPES[c["dtype"]]
    st = {"case": c}
    if c["op"] == "rotate":
        names = ("q", "k", "dq", "dk") if c["grads"] else ("q", "k")
        st.update({x: _normal(g, n, t, hq if x[-1] == "q" else hk, d, std=1.5, dtype=dtype) for x in names})
        # (a position's axes: far along the first, inside a picture along the others)
        st["positions"] = torch.stack([torch.randint(0, 100000 if a == 0 else 256, (n, t), generator=g, device=DEV) for a in range(c["axes"])]).int()
        st["inv_freq"] = (ROPE_BASE ** (-torch.arange(0, d, 2, device=DEV, dtype=torch.float64) / d)).float()
        st["axes"] = [i % c["axes"] for i in range(d // 2)]
        return st
    if c["op"] == "delta":
        parents, _, kept = _trees(c)
        unit = lambda x: torch.nn.functional.normalize(x, dim=-1).to(dtype)
        st.update(q=unit(_normal(g, n, t, hq, d, dtype=torch.float32)), k=unit(_normal(g, n, t, hq, d, dtype=torch.float32)),
                  v=_normal(g, n, t, hq, d, dtype=dtype), beta=torch.rand(n, t, hq, generator=g, device=DEV).to(dtype),
                  log_alpha=(-0.2 * torch.rand(n, t, hq, d, generator=g, device=DEV)).to(dtype),
                  S=torch.randn(n + 2, hq, d, d, generator=g, device=DEV) * 0.1,
                  slots=torch.randperm(n + 2, generator=g, device=DEV)[:n].int(), parents=_device(parents), kept=_device(kept))
        return st
    if c["op"] == "fork":
        pool, _, table, refs, _, source, lens, after = _fork_tables(c)
        st.update(_pool(g, c, pool), table=_device(table), refs=_device(refs), source=_device(source), lens=_device(lens), after=_device(after))
        return st
    if c["op"] == "compact":
        table, refs = _compact_tables(c)
        st.update(_pool(g, c, c["pool"]), table=_device(table), refs=_device(refs))
        return st
    drafted, held = _sizes(c)
    parents, _, kept = _trees(c)
    need = [-(-(h + t) // c["page"]) for h in held]
    columns, pages = max(need), sum(need) + 3              # (a pool is never full)
    order = torch.randperm(pages, generator=g, device=DEV).to(torch.int32)
    starts = np.concatenate([[0], np.cumsum(need)])
    at = torch.tensor(starts[:-1, None] + np.minimum(np.arange(columns)[None, :], np.array(need)[:, None] - 1), device=DEV)
    table = torch.where(torch.arange(columns, device=DEV)[None, :] < torch.tensor(need, device=DEV)[:, None], order[at], -1).to(torch.int32)
    st.update(_pool(g, c, pages), table=table.contiguous(), lens=_device(held), parents=_device(parents), kept=_device(kept))
    if c["op"] == "attend":
        for x in ("k_cache", "v_cache", "k_scale", "v_scale"):
            st[x] = st[x][0]                               # (one layer's)
        st.update(q=_normal(g, n, t, hq, d, std=1.5), max_kv_len=max(held) + t)
    return st


def run(state):
    s, c = state, state["case"]
    return {"rotate": _rotate, "attend": _attend, "keep": _keep, "fork": _fork, "compact": _compact, "delta": _delta}[c["op"]](s, c)


def _rotate(s, c):
    if own:
        import paper_2510_26692_amd as kda
        kw = dict(axes=s["axes"], interleaved=c["rope"] == "pairs")
        out = kda.kda_rotate(s["q"], s["k"], s["positions"], s["inv_freq"], **kw)
        if c["grads"]:
            out = (*out, *kda.kda_rotate(s["dq"], s["dk"], s["positions"], s["inv_freq"], inverse=True, **kw))
        return list(out)
    d = c["dim"]
    angle = s["positions"].permute(1, 2, 0)[..., s["axes"]].double() * s["inv_freq"].double()
    cos, sin = torch.cos(angle).float()[:, :, None], torch.sin(angle).float()[:, :, None]

    def turned(x, sin):
        y = x.float()
        if c["rope"] == "pairs":
            a, b = y[..., 0::2], y[..., 1::2]
            return torch.stack([a * cos - b * sin, a * sin + b * cos], -1).flatten(-2).to(x.dtype)
        a, b = y[..., :d // 2], y[..., d // 2:]
        return torch.cat([a * cos - b * sin, a * sin + b * cos], -1).to(x.dtype)

    return [turned(s["q"], sin), turned(s["k"], sin)] + ([turned(s["dq"], -sin), turned(s["dk"], -sin)] if c["grads"] else [])


def _ancestors(parents):
    """seen [N,T,T]: token i sees token j (itself, and what it descends from), and depths [N,T]."""
    n, t = parents.shape
    seen = torch.zeros(n, t, t, dtype=torch.bool, device=DEV)
    row = torch.arange(n, device=DEV)
    for i in range(t):
        up = parents[:, i].long()
        seen[:, i] = seen[row, up.clamp(min=0)] & (up >= 0)[:, None]
        seen[:, i, i] = up >= -1
    return seen, (seen.sum(-1) - 1).clamp(min=0)


def _attend(s, c):
    if own:
        import paper_2510_26692_amd as kda
        return kda.kda_cache_tree_attn(s["q"], s["k_cache"], s["v_cache"], s["k_scale"], s["v_scale"], s["table"], s["lens"], s["parents"],
                                       window=c["window"], sinks=c["sinks"], max_kv_len=s["max_kv_len"], out_dtype=torch.bfloat16)
    n, t, hq, d = s["q"].shape
    hk, page = c["kv_heads"], c["page"]
    length = s["table"].shape[1] * page
    number = s["table"].long().clamp(min=0)

    def held(cache, scale):                                # [n, hk, length, d]
        x = cache[number].float() * scale[number][..., None, None]
        return x.transpose(1, 2).reshape(n, hk, length, d)

    tree, depth = _ancestors(s["parents"])
    lens = s["lens"].long()
    pos = lens[:, None] + depth
    j = torch.arange(length, device=DEV)
    node = j[None, :] - lens[:, None]                      # [n, length]: which drafted token stands there
    is_node = (node >= 0) & (node < t)
    at = torch.where(is_node, lens[:, None] + torch.gather(depth, 1, node.clamp(0, t - 1)), j[None, :])
    seen = torch.gather(tree, 2, node.clamp(0, t - 1)[:, None, :].expand(-1, t, -1)) & is_node[:, None, :]
    seen |= (node < 0)[:, None, :] & (s["parents"] >= -1)[:, :, None]
    if c["window"]:
        seen &= (pos[:, :, None] - at[:, None, :] < c["window"]) | (at < c["sinks"])[:, None, :]
    q = s["q"].float().transpose(1, 2).reshape(n, hk, hq // hk * t, d)
    x = torch.matmul(q, held(s["k_cache"], s["k_scale"]).transpose(2, 3)) * d ** -0.5
    x = x.masked_fill_(~seen.repeat(1, hq // hk, 1)[:, None], -math.inf)
    m = x.amax(-1, keepdim=True)
    p = torch.exp(x - torch.where(m > -math.inf, m, 0.0))
    p = p / p.sum(-1, keepdim=True).clamp(min=1e-30)
    o = torch.matmul(p, held(s["v_cache"], s["v_scale"]))
    return o.reshape(n, hq, t, d).transpose(1, 2).bfloat16()


def _keep(s, c):
    if own:
        import paper_2510_26692_amd as kda
        kda.kda_cache_keep(s["k_cache"], s["v_cache"], s["k_scale"], s["v_scale"], s["table"], s["lens"], s["kept"])
        return [s[x] for x in ("k_cache", "v_cache", "k_scale", "v_scale")]
    page, kept, lens = c["page"], s["kept"].long(), s["lens"].long()
    seq, index = torch.nonzero(kept >= 0, as_tuple=True)
    to, frm = lens[seq] + index, lens[seq] + kept[seq, index]
    to_page, from_page = s["table"][seq, to // page].long(), s["table"][seq, frm // page].long()
    head = lens % page                                     # older tokens of the page that the first kept one goes to
    first = s["table"][torch.arange(c["rows"], device=DEV), lens // page].long()
    some = (kept >= 0).any(1)
    for cache, scale in ((s["k_cache"], s["k_scale"]), (s["v_cache"], s["v_scale"])):
        moved = cache[:, from_page, :, frm % page].float()                       # [tokens, layers, heads, d]
        of = scale[:, from_page].transpose(0, 1)                                 # [tokens, layers, heads]
        top = torch.zeros_like(scale).scatter_reduce(1, to_page[None, :, None].expand(of.transpose(0, 1).shape), of.transpose(0, 1), "amax")
        older = first[some & (head > 0)]
        top[:, older] = torch.maximum(top[:, older], scale[:, older])
        new = torch.where(top > 0, top, scale)
        grown = some & (head > 0) & (new[:, first] > scale[:, first]).any(2).any(0)
        for i in torch.nonzero(grown)[:, 0].tolist():
            p, h = int(first[i]), int(head[i])
            again = cache[:, p, :, :h].float() * (scale[:, p] / new[:, p])[..., None, None]
            cache[:, p, :, :h] = again.to(cache.dtype)
        code = (moved * (of / new[:, to_page].transpose(0, 1))[..., None]).to(cache.dtype)
        cache.view(torch.uint8)[:, to_page, :, to % page] = code.view(torch.uint8)
        scale.copy_(new)
    return [s[x] for x in ("k_cache", "v_cache", "k_scale", "v_scale")]


def _copy_pages(s, pairs):
    pairs = pairs[pairs[:, 0] >= 0].long()
    for x in ("k_cache", "v_cache", "k_scale", "v_scale"):
        y = s[x].view(torch.uint8) if s[x].dtype == torch.float8_e4m3fn else s[x]
        y[:, pairs[:, 1]] = y[:, pairs[:, 0]]


def _fork(s, c):
    if own:
        import paper_2510_26692_amd as kda
        kda.kda_pages_fork(s["table"], s["refs"], s["source"])
        copies, missing = kda.kda_pages_reserve(s["table"], s["lens"], s["after"], s["refs"], c["page"])
        kda.kda_cache_copy_pages(s["k_cache"], s["v_cache"], s["k_scale"], s["v_scale"], copies)
        return [s["table"], s["refs"], copies, missing, s["k_cache"], s["v_cache"], s["k_scale"], s["v_scale"]]
    table, refs, page = s["table"], s["refs"], c["page"]
    table.copy_(table[s["source"].long()])
    refs.copy_(torch.bincount(table[table >= 0].long(), minlength=refs.numel()).int())
    # every page that a row is to write is its own: missing ones, and ones that others read too, are taken from the free ones
    column = torch.arange(table.shape[1], device=DEV)[None, :]
    written = (column >= s["lens"][:, None] // page) & (column < -(-s["after"] // page)[:, None])
    want = written & ((table < 0) | (refs[table.long().clamp(min=0)] > 1))
    row, at = torch.nonzero(want, as_tuple=True)
    free = torch.nonzero(refs == 0)[:, 0].int()
    missing = max(0, len(row) - len(free))
    copies = torch.full((table.shape[0], 2), -1, dtype=torch.int32, device=DEV)
    if not missing:
        old, new = table[row, at], free[:len(row)]
        older = (old >= 0) & (at == s["lens"][row] // page) & (s["lens"][row] % page > 0)
        copies[row[older]] = torch.stack([old, new], 1)[older]
        table[row, at] = new
        refs.copy_(torch.bincount(table[table >= 0].long(), minlength=refs.numel()).int())
    _copy_pages(s, copies)
    return [table, refs, copies, torch.tensor([missing], dtype=torch.int32, device=DEV), s["k_cache"], s["v_cache"], s["k_scale"], s["v_scale"]]


def _compact(s, c):
    # (the table and counts of before stay as they are: the pass can be made again)
    table, refs = s["table"].clone(), s["refs"].clone()
    if own:
        import paper_2510_26692_amd as kda
        moves = kda.kda_pages_compact(table, refs)
        kda.kda_cache_copy_pages(s["k_cache"], s["v_cache"], s["k_scale"], s["v_scale"], moves)
        return [table, refs, moves, s["k_cache"], s["v_cache"], s["k_scale"], s["v_scale"]]
    used = refs > 0
    count = int(used.sum())
    frm = torch.nonzero(used[count:])[:, 0] + count
    to = torch.nonzero(~used[:count])[:, 0]
    moves = torch.full((refs.numel() // 2, 2), -1, dtype=torch.int32, device=DEV)
    moves[:len(to)] = torch.stack([frm, to], 1).int()
    place = torch.arange(refs.numel(), dtype=torch.int32, device=DEV)
    place[frm] = to.int()
    table = torch.where(table >= 0, place[table.long().clamp(min=0)], table)
    refs[to] = refs[frm]
    refs[frm] = 0
    _copy_pages(s, moves)
    return [table, refs, moves, s["k_cache"], s["v_cache"], s["k_scale"], s["v_scale"]]


def _delta(s, c):
    scale = c["dim"] ** -0.5
    if own:
        import paper_2510_26692_amd as kda
        o = kda.kda_tree_steps(s["q"], s["k"], s["v"], s["log_alpha"], s["beta"], s["S"], s["parents"], state_indices=s["slots"], scale=scale,
                               out_dtype=torch.bfloat16)
        kda.kda_tree_commit(s["k"], s["v"], s["log_alpha"], s["beta"], s["S"], s["kept"], state_indices=s["slots"])
        return [o, s["S"]]
    q, k, v, beta = (s[x].float() for x in ("q", "k", "v", "beta"))
    alpha = torch.exp(s["log_alpha"].float())
    slots, parents, kept = s["slots"].long(), s["parents"].long(), s["kept"].long()
    n, t = parents.shape
    row = torch.arange(n, device=DEV)

    def step(state, at):                                   # [n,H,dk,dv] through the tokens `at` [n]
        kk = k[row, at][..., None]
        state = state * alpha[row, at][..., None]
        rest = v[row, at] - (kk * state).sum(2)
        return state + kk * (beta[row, at][..., None] * rest)[:, :, None, :]

    first = s["S"][slots]
    states = [None] * t
    o = torch.empty(s["v"].shape, dtype=torch.float32, device=DEV)
    used = parents.cpu()
    for i in range(t):
        before = first
        for j in sorted(set(used[:, i].tolist()) - {-1, -2}):
            before = torch.where((parents[:, i] == j)[:, None, None, None], states[j], before)
        states[i] = step(before, torch.full_like(row, i))
        there = (parents[:, i] >= -1)[:, None, None]
        o[:, i] = torch.where(there, scale * (q[:, i][..., None] * states[i]).sum(2), 0.0)
        for j in range(i):                                 # (a state that no token behind descends from goes)
            if states[j] is not None and not bool((used[:, i + 1:] == j).any()):
                states[j] = None
    for i in range(t):
        on = kept[:, i] >= 0
        if not bool(on.any()):
            break
        first = torch.where(on[:, None, None, None], step(first, kept[:, i].clamp(min=0)), first)
    s["S"][slots] = first
    return [o.bfloat16(), s["S"]]


def exact(case, seed):
    """The definitions, in 64 bits: one sequence at a time."""
    c, s = case, prepare(case, seed)
    return {"rotate": _exact_rotate, "attend": _exact_attend, "keep": _exact_keep, "fork": _exact_fork, "compact": _exact_compact,
            "delta": _exact_delta}[c["op"]](s, c)


def _exact_rotate(s, c):
    where = torch.zeros(*s["q"].shape[:2], c["dim"] // 2, dtype=torch.float64, device=DEV)
    for i, a in enumerate(s["axes"]):
        where[..., i] = s["positions"][a].double() * s["inv_freq"][i].double()
    out, half = [], c["dim"] // 2
    for x, sign in (("q", 1j), ("k", 1j), ("dq", -1j), ("dk", -1j))[:4 if c["grads"] else 2]:
        y = s[x].double()
        z = torch.complex(y[..., 0::2], y[..., 1::2]) if c["rope"] == "pairs" else torch.complex(y[..., :half], y[..., half:])
        z = z * torch.exp(sign * where)[:, :, None]
        out.append(torch.view_as_real(z).flatten(-2) if c["rope"] == "pairs" else torch.cat([z.real, z.imag], -1))
    return out


def _exact_attend(s, c):
    group, page, t = c["heads"] // c["kv_heads"], c["page"], c["tokens"]
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device=DEV)
    parents = s["parents"].tolist()
    for n, held in enumerate(s["lens"].tolist()):
        at = s["table"][n, :-(-(held + t) // page)].long()
        seen, depth = np.zeros((t, held + t), dtype=bool), [0] * t
        for i in range(t):
            up = parents[n][i]
            if up < -1:
                continue
            depth[i] = depth[up] + 1 if up >= 0 else 0
            j = i
            while j >= 0:
                seen[i, held + j] = not c["window"] or depth[i] - depth[j] < c["window"] or held + depth[j] < c["sinks"]
                j = parents[n][j]
            ctx = np.arange(held)
            seen[i, :held] = not c["window"] or (held + depth[i] - ctx < c["window"]) | (ctx < c["sinks"])
        rows = torch.tensor(seen.any(1), device=DEV)
        mask = torch.tensor(seen, device=DEV)
        for h in range(c["kv_heads"]):
            k, v = ((s[x + "_cache"][at, h].double() * s[x + "_scale"][at, h].double()[:, None, None]).flatten(0, 1)[:held + t] for x in "kv")
            for e in range(h * group, (h + 1) * group):
                x = (s["q"][n, :, e].double() @ k.T) / math.sqrt(c["dim"])
                p = torch.softmax(x.masked_fill(~mask, -math.inf), -1)
                out[n, :, e] = torch.where(rows[:, None], torch.nan_to_num(p) @ v, 0.0)
    return out


def _exact_keep(s, c):
    page, table, kept = c["page"], s["table"].cpu().numpy(), s["kept"].cpu().numpy()
    out = []
    for cache, scale in ((s["k_cache"], s["k_scale"]), (s["v_cache"], s["v_scale"])):
        y, old, new = cache.double(), scale.double(), scale.double()
        for n, held in enumerate(s["lens"].tolist()):
            path = [x for x in kept[n] if x >= 0]
            frm = [(int(table[n, (held + x) // page]), (held + int(x)) % page) for x in path]
            to = [(int(table[n, (held + i) // page]), (held + i) % page) for i in range(len(path))]
            for p in sorted(set(p for p, _ in to)):
                src = [i for i in range(len(path)) if to[i][0] == p]
                older = held % page if p == to[0][0] else 0
                stack = [old[:, frm[i][0]] for i in src] + ([old[:, p]] if older else [])
                new[:, p] = torch.stack(stack).amax(0)
                if older:
                    y[:, p, :, :older] = (cache[:, p, :, :older].double() * (old[:, p] / new[:, p])[..., None, None]).float().to(cache.dtype).double()
                for i in src:
                    q, at = frm[i]
                    y[:, p, :, to[i][1]] = (cache[:, q, :, at].double() * (old[:, q] / new[:, p])[..., None]).float().to(cache.dtype).double()
        out.append((y, new))
    return [out[0][0], out[1][0], out[0][1], out[1][1]]


def _exact_copies(s, pairs):
    out = []
    for x in ("k_cache", "v_cache", "k_scale", "v_scale"):
        y = s[x].double()
        for a, b in pairs:
            y[:, b] = s[x][:, a].double()
        out.append(y)
    return out


def _exact_fork(s, c):
    page, source = c["page"], s["source"].tolist()
    table = [list(r) for r in s["table"].tolist()]
    table = [list(table[i]) for i in source]
    count = [0] * s["refs"].numel()
    for r in table:
        for p in r:
            if p >= 0:
                count[p] += 1
    start, free, copies = list(count), [p for p, x in enumerate(count) if x == 0], []
    for n, (a, b) in enumerate(zip(s["lens"].tolist(), s["after"].tolist())):
        copies.append([-1, -1])
        for col in range(a // page, -(-b // page)):
            old = table[n][col]
            if old >= 0 and start[old] <= 1:
                continue
            new = free.pop(0)
            table[n][col], count[new] = new, 1
            if old >= 0:
                count[old] -= 1
                if col == a // page and a % page:
                    copies[n] = [old, new]
    return [_device(table), _device(count), _device(copies), _device([0])] + _exact_copies(s, [p for p in copies if p[0] >= 0])


def _exact_compact(s, c):
    table, count = s["table"].tolist(), s["refs"].tolist()
    used = sum(x > 0 for x in count)
    moves = list(zip([p for p in range(used, len(count)) if count[p]], [p for p in range(used) if not count[p]]))
    place = dict(moves)
    table = [[place.get(p, p) for p in r] for r in table]
    for a, b in moves:
        count[b], count[a] = count[a], 0
    listed_moves = [list(m) for m in moves] + [[-1, -1]] * (len(count) // 2 - len(moves))
    return [_device(table), _device(count), _device(listed_moves).reshape(-1, 2)] + _exact_copies(s, moves)


def _exact_delta(s, c):
    """Written out: every token's correction and output from the state before the tree and the corrections of its ancestors."""
    n, t, h, d = s["q"].shape
    parents, kept = s["parents"].cpu().numpy(), s["kept"].cpu().numpy()
    o = torch.zeros(s["q"].shape, dtype=torch.float64, device=DEV)
    S = s["S"].double()
    for b in range(n):
        slot, count = int(s["slots"][b]), int((parents[b] >= -1).sum())
        line = np.zeros((count, count))                    # ancestors, and the token itself
        for i in range(count):
            if parents[b, i] >= 0:
                line[i] = line[parents[b, i]]
            line[i, i] = 1
        line = torch.tensor(line, device=DEV)
        q, k, v, la = (s[x][b, :count].double().transpose(0, 1) for x in ("q", "k", "v", "log_alpha"))           # [h, count, d]
        beta = s["beta"][b, :count].double().T[..., None]                                                          # [h, count, 1]
        total = torch.matmul(line, la)                     # of all decays down to a token
        far = torch.matmul(k * torch.exp(total), S[slot])
        far_q = torch.matmul(q * torch.exp(total), S[slot])
        between = torch.exp((total[:, :, None] - total[:, None]).clamp(max=0.0))                                   # [h, i, j, d]
        kk = (between * k[:, :, None] * k[:, None]).sum(-1) * line
        qk = (between * q[:, :, None] * k[:, None]).sum(-1) * line
        lower = torch.eye(count, dtype=torch.float64, device=DEV) + beta * torch.tril(kk, -1)
        u = torch.linalg.solve_triangular(lower, beta * (v - far), upper=False)
        o[b, :count] = ((far_q + torch.matmul(qk, u)) * d ** -0.5).transpose(0, 1)
        path = [int(x) for x in kept[b] if x >= 0]
        if path:
            last = path[-1]
            left = torch.exp(total[:, last, None] - total[:, path])                                                # decays behind each token of the path
            S[slot] = torch.exp(total[:, last])[..., None] * S[slot] + torch.matmul((left * k[:, path]).transpose(1, 2), u[:, path])
    return [o, S]
