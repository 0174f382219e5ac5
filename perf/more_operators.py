"""A cache of latent vectors with the attentions that read it, in both of their forms, and the pages
under a cache: cases, their inputs, a plain form of every operator, its work and its 64-bit
result.

A latent cache holds, for each position, one vector of dc components that all heads share (keys and
values in one) and 64 more components of a key that is rotated to its position.  A case is a
dict of plain values.  Its `kind` names the operator:

  append    new tokens' latents, normalised, and rotated keys into the pages, the queries' rotated
            part beside them, and the same latents and keys side by side (`prepare_latent_append`)
  attend    attention over the pages in the absorbed form, every head against the latents
            themselves; `form`: "token" for the last position alone, "round" for the arbitrator's
            region of 2K + 3 queries, "chunk" for the last positions of a context
            (`prepare_latent_attention`), "tree" for a token tree's nodes
            (`prepare_latent_tree_attention`)
  expanded  the same attention over keys and values that were expanded for every head, not paged;
            `form`: "prefill" for whole inputs, "round" for the region alone
            (`prepare_expanded_attention`)
  fork      sequences that go on from others' positions share their pages, and get pages of their
            own for what comes next, with a copy of those that are partly filled
            (`prepare_pages_fork`, `prepare_pages_reserve`)
  compact   the ends of some sequences given back, and the pages in use moved to the front of the
            pool (`prepare_pages_release`, `prepare_pages_compact`)

`cache` is the latents' element type: "bf16", or "e4m3" (8 bits) with one power-of-two scale for
each position.  Rotated keys are bf16.  Lengths follow from the case alone; everything else is made
on the GPU from the seed.
"""
from __future__ import annotations

import math

import torch

own = False

_BF16, _E4M3 = "bf16", "e4m3"
_LOWEST = 2.0 ** -100          # scale of a position that holds nothing but zeros
_DR = 64                       # components of the rotated key
_EPS = 1e-6


def listed():
    return [
        # one user, one new token: latency is everything
        dict(name="append_token", kind="append", cache=_E4M3, B=1, n=1, start=2000, ragged=False, far=0, norm=True,
             interleaved=False, page=64, Hq=32, dc=512),
        # whole inputs into a bf16 cache, laid out side by side as well for the expanded form
        dict(name="append_prefill", kind="append", cache=_BF16, B=4, n=2065, start=0, ragged=True, far=0, norm=True,
             interleaved=True, page=64, Hq=32, dc=512),
        # one user's next token with few heads and short latents: latency
        dict(name="token_one", kind="attend", form="token", cache=_BF16, B=1, ctx=2000, K=0, page=32, Hq=16, dc=256),
        # plain decoding of a serving batch
        dict(name="token", kind="attend", form="token", cache=_E4M3, B=64, ctx=4096, K=0, page=64, Hq=32, dc=512),
        # one round of a serving batch (K = 7): the matrix cores bound it
        dict(name="round", kind="attend", form="round", cache=_E4M3, B=64, ctx=2048, K=7, page=64, Hq=32, dc=512),
        # trees of 60 nodes over a bf16 cache
        dict(name="tree_bf16", kind="attend", form="tree", cache=_BF16, B=16, ctx=2048, depth=6, page=64, Hq=32, dc=512),
        # the first pass over whole inputs, every head with keys and values of its own
        dict(name="prefill", kind="expanded", form="prefill", B=4, ctx=2048, K=7, H=32, D=128),
        # the region alone of a few short sequences, smaller heads
        dict(name="region", kind="expanded", form="round", B=8, ctx=317, K=5, H=16, D=64),
        # one prompt's branches, two layers
        dict(name="fork_one", kind="fork", store="latent", prompts=1, branches=4, ctx=1000, n=17, layers=2, page=64, dc=512,
             others=100, spare=100),
        # rollouts of a group of prompts, several layers: the copies count
        dict(name="fork_group", kind="fork", store="heads", prompts=8, branches=8, ctx=500, n=60, layers=8, page=64,
             Hkv=8, D=128, others=64, spare=200),
        # a pool of one small cache
        dict(name="compact_one", kind="compact", store="latent", B=4, ctx=700, layers=1, page=32, dc=256, spare=300),
        # a serving batch's pages in several layers
        dict(name="compact_batch", kind="compact", store="heads", B=32, ctx=500, layers=8, page=64, Hkv=8, D=128, spare=300),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["append", "attend", "attend", "attend", "expanded", "fork", "compact"])
    cache, dc = rng.choice([_E4M3, _E4M3, _BF16]), rng.choice([512, 512, 256])
    page = rng.choice([16, 32, 64, 128])
    if kind == "append":
        n = rng.choice([1, rng.randint(2, 60), _log_int(rng, 60, 2000)])
        B = max(1, min(_log_int(rng, 1, 96), 8000 // n))
        return dict(kind=kind, cache=cache, B=B, n=n, start=_log_int(rng, 1, 900), ragged=rng.random() < 0.5,
                    far=rng.choice([0, 0, 100003]), norm=rng.random() < 0.7, interleaved=rng.random() < 0.5, page=page,
                    Hq=rng.choice([8, 16, 32, 64, 128]), dc=dc)
    if kind == "attend":
        form = rng.choice(["token", "token", "round", "chunk", "tree"])
        Hq = rng.choice([8, 16, 20, 32, 64, 128])
        c = dict(kind=kind, form=form, cache=cache, ctx=_log_int(rng, 30, 20000), page=page, Hq=Hq, dc=dc)
        if form == "tree":
            c.update(depth=rng.randint(2, 8), ctx=min(c["ctx"], 8000))
            rows = _tree_nodes(c)
        elif form == "round":
            c["K"] = rng.choice([1, 4, 5, 7, 10, 15, 25])
            rows = 2 * c["K"] + 3
        else:
            rows = 1 if form == "token" else min(_log_int(rng, 2, 512), c["ctx"])
            c.update(K=0, n=rows)
        # no more than the serving batch's round: rows times positions, and positions
        c["B"] = max(1, min(_log_int(rng, 1, 64), 64 * 544 * 2000 // (rows * Hq * (c["ctx"] + rows)), 250000 // c["ctx"]))
        if rows * Hq * (c["ctx"] + rows) > 64 * 544 * 2000:
            c["ctx"] = 64 * 544 * 2000 // (rows * Hq) - rows
        return c
    if kind == "expanded":
        D, H = rng.choice([128, 128, 64]), rng.choice([8, 16, 20, 32])
        K = rng.choice([1, 4, 5, 7, 10, 15, 25])
        if rng.random() < 0.6:
            ctx = _log_int(rng, 60, 2000)
            return dict(kind=kind, form="prefill", B=max(1, min(_log_int(rng, 1, 12), int(3.5 * 2048.0 ** 2 / ctx ** 2))),
                        ctx=ctx, K=K, H=H, D=D)
        ctx = _log_int(rng, 30, 8000)
        return dict(kind=kind, form="round", B=max(1, min(_log_int(rng, 1, 32), 16000 // ctx)), ctx=ctx, K=K, H=H, D=D)
    layers = rng.choice([1, 2, 3, 5, 8])
    c = dict(kind=kind, store=rng.choice(["latent", "heads"]), layers=layers, page=page)
    c.update(dict(dc=dc) if c["store"] == "latent" else dict(Hkv=rng.choice([1, 4, 8]), D=rng.choice([64, 128])))
    if kind == "fork":
        c.update(prompts=_log_int(rng, 1, 8), branches=_log_int(rng, 1, 8), ctx=_log_int(rng, 1, 500), n=_log_int(rng, 1, 60),
                 others=rng.randint(0, 64), spare=rng.randint(0, 200))
    else:
        c.update(B=_log_int(rng, 1, 32), ctx=_log_int(rng, 8, 500), spare=rng.randint(0, 300))
    return c


# ------------------------------------------------------------------ lengths, from the case

def _ctx_len(c, b):
    return c["ctx"] - (b * 97) % (c["ctx"] // 4 + 1)


def _starts(c):
    return [c["start"] - (b * 37) % (c["start"] // 2 + 1) for b in range(c["B"])]


def _counts(c):
    cut = c["n"] // 2 + 1
    return [c["n"] - ((b * 5) % cut if c["ragged"] else 0) for b in range(c["B"])]


def _tree_nodes(c):
    # 4 children of the root, then 11 nodes a level
    return 1 + 4 + 11 * (c["depth"] - 1)


def _rows(c):
    """Query positions of a sequence."""
    region = 0 if c["form"] == "tree" else 2 * c["K"] + 3
    return {"token": 1, "tree": _tree_nodes(c) if c["form"] == "tree" else 0, "chunk": c.get("n", 0), "round": region,
            "prefill": c["ctx"] + region}[c["form"]]


def _kept(c, b):
    """Positions that a sequence of a compact case keeps: a third of them lose nothing."""
    return _ctx_len(c, b) if b % 3 == 0 else _ctx_len(c, b) * ((b * 5) % 8) // 8


def _pages(n, page):
    return -(-n // page)


# ------------------------------------------------------------------------------- inputs

def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(int(seed) * 1000003 + 31)


def _randn(g, *shape):
    return torch.randn(*shape, generator=g, device="cuda")


def _int32(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def _scale_of(amax):
    """The smallest power of two s with amax <= 448 s."""
    m, e = torch.frexp(amax)
    s = torch.ldexp(torch.ones_like(amax), torch.where(m > 0.875, e - 8, e - 9)).clamp(min=_LOWEST)
    return torch.where(amax > 0, s, _LOWEST)


def _to_pages(x, page, table):
    """Rows [B, L, d] into the pages of `table` [B, T]: [B T, page, d]."""
    B, L, d = x.shape
    T = table.shape[1]
    pages = torch.empty(B * T, page, d, dtype=x.dtype, device="cuda")
    pages[table.reshape(-1)] = torch.nn.functional.pad(x, (0, 0, 0, T * page - L)).reshape(B * T, page, d)
    return pages


def _weight(c, g):
    """A norm's weight: near one, with a few strong components."""
    w = 1 + 0.2 * _randn(g, c["dc"])
    w[torch.randperm(c["dc"], generator=g, device="cuda")[:c["dc"] // 64]] *= 3
    return w.bfloat16()


def _cache(c, g, lengths, room, along=None):
    """A latent cache that holds lengths[b] positions of sequence b, with room for `room`; `along`:
    where the first position's key [dc + 64] lies."""
    B, P, dc = c["B"], c["page"], c["dc"]
    L, T = max(max(lengths), 1), _pages(room, c["page"])
    live = (torch.arange(L, device="cuda")[None, :] < _int32(lengths)[:, None])[:, :, None]
    x = _randn(g, B, L, dc) * _weight(c, g).float()
    r = _randn(g, B, L, _DR)
    if along is not None:
        x[:, 0], r[:, 0] = along[:dc], along[dc:]
    x, r = (x * live).bfloat16(), (r * live).bfloat16()
    table = torch.randperm(B * T, generator=g, device="cuda").reshape(B, T)
    s = dict(table=table.int(), r=_to_pages(r, P, table), scale=None)
    if c["cache"] == _E4M3:
        scale = _scale_of(x.float().abs().amax(-1))
        x = (x.float() / scale[:, :, None]).to(torch.float8_e4m3fn)
        s["scale"] = _to_pages(scale[:, :, None], P, table)[:, :, 0].contiguous()
        x = x.view(torch.uint8)
    s["c"] = _to_pages(x, P, table)
    if c["cache"] == _E4M3:
        s["c"] = s["c"].view(torch.float8_e4m3fn)
    return s


def _parents(c, g):
    """Node 0, its 4 children, then levels of 11 nodes under random nodes of the level before."""
    B, parts = c["B"], [torch.full((c["B"], 1), -1), torch.zeros(c["B"], 4)]
    first, width = 1, 4
    for _ in range(c["depth"] - 1):
        parts.append(first + (torch.rand(B, 11, generator=g, device="cuda") * width).long().cpu())
        first, width = first + width, 11
    return torch.cat(parts, 1).int().cuda()


def _planes(c, g, n_pages):
    """Pages of every layer, as a cache of this kind keeps them: [layers, n_pages, ...] each."""
    L, P = c["layers"], c["page"]
    if c["store"] == "latent":
        return dict(c=_randn(g, L, n_pages, P, c["dc"]).bfloat16(), r=_randn(g, L, n_pages, P, _DR).bfloat16())
    H, D = c["Hkv"], c["D"]
    return dict(k=_randn(g, L, n_pages, H, P, D).bfloat16(), v=_randn(g, L, n_pages, H, D, P).bfloat16())


def _prepare_pages(c, g):
    """Tables and a pool whose free pages lie between those in use."""
    P = c["page"]
    if c["kind"] == "fork":
        B = c["prompts"]
        held = [_pages(_ctx_len(c, b), P) for b in range(B)]
        T = _pages(c["ctx"] + c["n"], P) + 1
        # the pages that the branches will need, and some more
        n_pages = sum(held) + c["others"] + B * c["branches"] * (_pages(c["n"], P) + 1) + c["spare"] + 1
        used = sum(held) + c["others"]
    else:
        B = c["B"]
        held = [_pages(_ctx_len(c, b), P) for b in range(B)]
        T = _pages(c["ctx"], P) + 1
        n_pages, used = sum(held) + c["spare"] + 1, sum(held)
    order = torch.randperm(n_pages, generator=g, device="cuda").int()
    s = dict(refs0=torch.zeros(n_pages, dtype=torch.int32, device="cuda"))
    s["refs0"][order[:used].long()] = 1
    first = [sum(held[:b]) for b in range(B)]
    at = torch.tensor([[first[b] + j if j < held[b] else 0 for j in range(T)] for b in range(B)], device="cuda")
    there = torch.tensor([[j < held[b] for j in range(T)] for b in range(B)], device="cuda")
    s["table0"] = torch.where(there, order[at], -1).int()
    s["refs"], s["table"] = s["refs0"].clone(), s["table0"].clone()
    s["planes"] = _planes(c, g, n_pages)
    if c["kind"] == "fork":
        rows = [b for b in range(B) for _ in range(c["branches"])]
        s["row"], s["len"] = _int32(rows), _int32([_ctx_len(c, b) for b in rows])
    else:
        s["keep"] = _int32([_kept(c, b) for b in range(B)])
    return s


def _prepare_attend(c, g):
    B, dc, Hq, n = c["B"], c["dc"], c["Hq"], _rows(c)
    ctx = [_ctx_len(c, b) for b in range(B)]
    if c["form"] == "chunk":
        ctx = [max(x, n) for x in ctx]
    more = n if c["form"] == "tree" else 2 * c["K"] + 3 if c["form"] == "round" else 0
    lengths = [x + more for x in ctx]
    # queries about a mean of each head's; the first key along the heads' mean
    mean = _randn(g, Hq, dc + _DR) * 0.4
    q = _randn(g, B, n, Hq, dc + _DR) * 0.5 + mean
    s = _cache(c, g, lengths, max(lengths), mean.mean(0) * (1.5 * Hq ** 0.5))
    s.update(q=q.bfloat16(), ctx=_int32(ctx), scale_qk=(128 + _DR) ** -0.5)
    if c["form"] == "tree":
        s["parent"] = _parents(c, g)
    else:
        s["q_start"] = _int32([x if c["form"] == "round" else x - n for x in ctx])
    return s


def _prepare_append(c, g):
    B, n, dc, Hq = c["B"], c["n"], c["dc"], c["Hq"]
    starts = _starts(c) if c["start"] else [0] * B
    s = _cache(c, g, starts, max(starts) + n)
    s["start"], s["count"] = _int32(starts), _int32(_counts(c))
    # one projection's output holds a token's latent and its key, another one the queries
    down = _randn(g, B, n, dc + _DR) * torch.exp(_randn(g, B, n, 1))
    down = down.bfloat16()
    s["new_c"], s["new_r"] = down[..., :dc], down[..., dc:]
    s["new_q"] = _randn(g, B, n, Hq, 128 + _DR).bfloat16()[..., 128:]
    s["weight"] = _weight(c, g) if c["norm"] else None
    s["inv_freq"] = (10000.0 ** (-torch.arange(0, _DR, 2, dtype=torch.float64, device="cuda") / _DR)).float()
    at = s["start"][:, None] + torch.arange(n, device="cuda", dtype=torch.int32)
    s["positions"] = (at + c["far"]).int() if c["far"] else None
    return s


def _prepare_expanded(c, g):
    B, H, D, n = c["B"], c["H"], c["D"], _rows(c)
    ctx = [_ctx_len(c, b) for b in range(B)]
    L = max(ctx) + 2 * c["K"] + 3
    mean = _randn(g, H, D + _DR) * 0.7
    s = dict(q=(_randn(g, B, n, H, D + _DR) + mean).bfloat16(), k_r=_randn(g, B, L, _DR).bfloat16())
    # one projection of the latents holds a head's key and value side by side
    kv = _randn(g, B, L, H, 2 * D)
    kv[:, 0, :, :D] = mean[:, :D] * 1.2
    kv = kv.bfloat16()
    s.update(k=kv[..., :D], v=kv[..., D:], ctx=_int32(ctx), scale_qk=(D + _DR) ** -0.5)
    s["q_start"] = _int32([0 if c["form"] == "prefill" else x for x in ctx])
    return s


def prepare(case, seed):
    c = dict(case)
    g = _gen(seed)
    kind = c["kind"]
    s = {"append": _prepare_append, "attend": _prepare_attend, "expanded": _prepare_expanded, "fork": _prepare_pages,
         "compact": _prepare_pages}[kind](c, g)
    s["case"] = c
    if own:
        s["calls"] = _calls(c, s)
    return s


def _calls(c, s):
    """The framework's calls, prepared as a serving loop keeps them."""
    import paper_2605_24793_amd as cs
    kind = c["kind"]
    if kind == "expanded":
        return [cs.prepare_expanded_attention(s["q"], s["k"], s["v"], s["k_r"], s["ctx"], s["q_start"], c["K"],
                                              s["scale_qk"])]
    if kind in ("fork", "compact"):
        pool, p = cs.PagePool(s["refs"], c["page"]), s["planes"]
        made = (lambda i: cs.LatentCache(p["c"][i], p["r"][i])) if c["store"] == "latent" else \
            (lambda i: cs.PagedCache(p["k"][i], p["v"][i]))
        caches = [made(i) for i in range(c["layers"])]
        if kind == "compact":
            return [cs.prepare_pages_release(pool, s["table"], s["keep"]),
                    cs.prepare_pages_compact(pool, s["table"], caches)]
        fork = cs.prepare_pages_fork(pool, s["table"], s["row"], s["len"])
        return [fork, cs.prepare_pages_reserve(pool, fork.outputs["table"], s["len"], c["n"], caches=caches)]
    cache = cs.LatentCache(s["c"], s["r"], s["scale"])
    if kind == "append":
        return [cs.prepare_latent_append(cache, s["table"], s["start"], s["new_c"], s["new_r"], weight=s["weight"], eps=_EPS,
                                         count=s["count"], inv_freq=s["inv_freq"], positions=s["positions"],
                                         interleaved=c["interleaved"], q=s["new_q"], dense=True)]
    if c["form"] == "tree":
        return [cs.prepare_latent_tree_attention(s["q"], cache, s["table"], s["ctx"], s["parent"], s["scale_qk"])]
    return [cs.prepare_latent_attention(s["q"], cache, s["table"], s["ctx"], s["q_start"], c["K"], s["scale_qk"])]


# ------------------------------------------------------------------------- the plain forms

def _rotated(x, positions, inv_freq, interleaved):
    """x [B, n, H, 64] rotated, in 64 bits: angles of far positions."""
    a = (positions.double()[:, :, None] * inv_freq.double())[:, :, None]
    cos, sin, half = a.cos(), a.sin(), inv_freq.numel()
    x = x.double()
    x1, x2 = (x[..., 0::2], x[..., 1::2]) if interleaved else (x[..., :half], x[..., half:])
    y1, y2 = x1 * cos - x2 * sin, x2 * cos + x1 * sin
    return torch.stack((y1, y2), -1).flatten(-2) if interleaved else torch.cat((y1, y2), -1)


def _raw(pages):
    return pages.view(torch.uint8) if pages.dtype == torch.float8_e4m3fn else pages


def _plain_append(s):
    c = s["case"]
    n, P = c["n"], c["page"]
    start, i = s["start"].long(), torch.arange(n, device="cuda")
    at = start[:, None] + i if s["positions"] is None else s["positions"]
    q = _rotated(s["new_q"], at, s["inv_freq"], c["interleaved"]).bfloat16()
    r = _rotated(s["new_r"][:, :, None], at, s["inv_freq"], c["interleaved"])[:, :, 0].bfloat16()
    # in 64 bits: values next to a border of the 8-bit type
    x = s["new_c"].double()
    if s["weight"] is not None:
        x = x * torch.rsqrt(x.square().mean(-1, keepdim=True) + _EPS) * s["weight"].double()
    # places past a sequence's count repeat its first token, so that they write what is written
    # there anyway
    tok = torch.where(i < s["count"][:, None], i, 0)
    place = start[:, None] + tok
    pid, slot = s["table"].long().gather(1, place // P), place % P
    b = torch.arange(c["B"], device="cuda")[:, None]
    s["r"][pid, slot] = r[b, tok]
    y = x
    if s["scale"] is not None:
        scale = _scale_of(x.abs().amax(-1)).float()
        s["scale"][pid, slot] = scale[b, tok]
        y = (x / scale[:, :, None]).float().to(torch.float8_e4m3fn).view(torch.uint8)
    else:
        y = x.bfloat16()
    _raw(s["c"])[pid, slot] = y[b, tok]
    return dict(q=q, dense_c=x.bfloat16(), dense_r=r)


def _softmax(score, mask):
    score = score.masked_fill(~mask, -math.inf)
    w = torch.exp(score - score.amax(-1, keepdim=True))
    return w / w.sum(-1, keepdim=True)


def _hybrid_seen(s, n, L):
    """Keys that a query sees [B, n, L] of the hybrid mask."""
    ctx, key = s["ctx"].long(), torch.arange(L, device="cuda")
    end = ctx + 2 * s["case"]["K"] + 3
    p = s["q_start"].long()[:, None] + torch.arange(n, device="cuda")
    return key < torch.where(p < ctx[:, None], p + 1, end[:, None])[:, :, None]


def _tree_seen(s, n, L):
    ctx, key = s["ctx"].long(), torch.arange(L, device="cuda")
    seen = _ancestors(torch.eye(n, dtype=torch.bool, device="cuda").expand(len(ctx), n, n),
                      s["parent"].long().clamp(min=0))
    own_key = (key - ctx[:, None]).clamp(0, n - 1)[:, None].expand(len(ctx), n, L)
    in_tree = (key >= ctx[:, None]) & (key < ctx[:, None] + n)
    return (key < ctx[:, None])[:, None] | (in_tree[:, None] & seen.gather(2, own_key))


def _ancestors(seen, up):
    # doubling the steps up: at most 128 nodes here, so seven reach the root from everywhere
    seen, up = _doubled(*_doubled(*_doubled(*_doubled(seen, up))))
    return _doubled(*_doubled(*_doubled(seen, up)))[0]


def _doubled(seen, up):
    return seen | seen.gather(1, up[:, :, None].expand_as(seen)), up.gather(1, up)


def _gathered(s):
    """Latents [B, L, dc] and rotated keys [B, L, 64] of every sequence in order, in 32 bits."""
    table = s["table"].long()
    x = s["c"][table] if s["scale"] is None else _raw(s["c"])[table].view(torch.float8_e4m3fn)
    x = x.float()
    if s["scale"] is not None:
        x = x * s["scale"][table][..., None]
    return x.flatten(1, 2), s["r"][table].float().flatten(1, 2)


def _plain_attend(s):
    c = s["case"]
    B, n, Hq, d = s["q"].shape
    x, r = _gathered(s)
    L = x.shape[1]
    keys = torch.cat((x, r), -1).transpose(1, 2).contiguous()
    score = torch.matmul(s["q"].float().reshape(B, n * Hq, d), keys).reshape(B, n, Hq, L) * s["scale_qk"]
    mask = _tree_seen(s, n, L) if c["form"] == "tree" else _hybrid_seen(s, n, L)
    w = _softmax(score, mask[:, :, None])
    return torch.matmul(w.reshape(B, n * Hq, L), x).reshape(B, n, Hq, c["dc"]).bfloat16()


def _plain_expanded(s):
    q, k, v, r = s["q"].float().transpose(1, 2), s["k"].float().transpose(1, 2), s["v"].float().transpose(1, 2), s["k_r"].float()
    D, L, n = k.shape[-1], k.shape[2], q.shape[2]
    score = torch.matmul(q[..., :D], k.transpose(2, 3).contiguous())
    score += torch.matmul(q[..., D:], r.transpose(1, 2)[:, None].contiguous())
    mask = _hybrid_seen(s, n, L)
    # positions past the sequence: rows of zeros
    p = s["q_start"].long()[:, None] + torch.arange(n, device="cuda")
    live = p < (s["ctx"].long() + 2 * s["case"]["K"] + 3)[:, None]
    out = torch.matmul(_softmax(score * s["scale_qk"], mask[:, None]), v.contiguous()).transpose(1, 2)
    return torch.where(live[:, :, None, None], out, 0).bfloat16()


def _shared(refs, pages, by):
    """refs[pages] += by where by is not 0 (pages of entries that name none: anything)."""
    refs.index_add_(0, pages.clamp(min=0).reshape(-1), by.to(refs.dtype).reshape(-1))


def _copied(s, source, target):
    for x in s["planes"].values():
        x[:, target] = x[:, source]


def _plain_fork(s):
    c = s["case"]
    P, n, refs = c["page"], c["n"], s["refs"]
    start, T, n_pages = s["len"].long(), s["table"].shape[1], len(refs)
    table = s["table"].long()[s["row"].long()]
    table = torch.where(torch.arange(T, device="cuda") * P < start[:, None], table, -1)
    _shared(refs, table, table >= 0)
    # pages of positions start .. start + n - 1: new ones where there is none or others hold it too;
    # the lowest free pages, in order of the sequences
    w = torch.arange(_pages(n - 1, P) + 1, device="cuda")
    j = start[:, None] // P + w
    here = j * P < start[:, None] + n
    j = j.clamp(max=T - 1)
    entry = table.gather(1, j)
    shared = here & (entry >= 0) & (refs[entry.clamp(min=0)] > 1)
    need = here & ((entry < 0) | shared)
    free = torch.argsort((refs != 0).int(), stable=True)
    rank = (need.reshape(-1).cumsum(0) - 1).reshape(need.shape).clamp(0, n_pages - 1)
    fresh = torch.where(need, free[rank], entry)
    short = (need.sum() - (refs == 0).sum()).clamp(min=0)
    given = (short == 0).long()
    _shared(refs, entry, -given * shared)
    _shared(refs, fresh, given * need)
    table = torch.where(here.new_zeros(len(start), T).scatter(1, j, here & (short == 0)),
                        table.scatter(1, torch.where(here, j, T - 1), torch.where(here, fresh, table[:, -1:])), table)
    part = (shared[:, 0] & (start % P > 0) & (short == 0))[:, None]
    copies = torch.where(part, torch.stack((entry[:, 0], fresh[:, 0]), 1), -1)
    kept = copies[part[:, 0]]
    _copied(s, kept[:, 0], kept[:, 1])
    return dict(table=table.int(), copies=copies.int(), short=short.int().reshape(1))


def _plain_compact(s):
    c = s["case"]
    refs, table = s["refs"], s["table"]
    T, n_pages = table.shape[1], len(s["refs"])
    entry = table.long()
    past = (torch.arange(T, device="cuda") * c["page"] >= s["keep"].long()[:, None]) & (entry >= 0)
    _shared(refs, entry, -past.int())
    entry = torch.where(past, -1, entry)
    used = refs > 0
    total, at = used.sum(), torch.arange(n_pages, device="cuda")
    source, target = (used & (at >= total)).nonzero()[:, 0], (~used & (at < total)).nonzero()[:, 0]
    to = at.clone()
    to[source] = target
    table.copy_(torch.where(entry >= 0, to[entry.clamp(min=0)], -1))
    refs[target] = refs[source]
    refs[source] = 0
    _copied(s, source, target)
    moves = torch.full((max(n_pages // 2, 1), 2), -1, dtype=torch.int32, device="cuda")
    moves[:len(source)] = torch.stack((source, target), 1).int()
    return dict(moves=moves, n_moves=torch.full((1,), len(source), dtype=torch.int32, device="cuda"))


def run(state):
    s = state
    kind = s["case"]["kind"]
    if kind in ("fork", "compact"):
        # a pass starts from the same tables and counts
        s["refs"].copy_(s["refs0"])
        if kind == "compact":
            s["table"].copy_(s["table0"])
    if own:
        out = {}
        for call in s["calls"]:
            call.launch()
            out.update(call.outputs)
        if kind == "append":
            out = dict(q=out["q"], dense_c=out["c"], dense_r=out["k_r"])
        elif kind == "fork":
            out["short"] = out.pop("lacking")
    elif kind == "append":
        out = _plain_append(s)
    elif kind == "attend":
        out = dict(out=_plain_attend(s))
    elif kind == "expanded":
        out = dict(out=_plain_expanded(s))
    else:
        out = _plain_fork(s) if kind == "fork" else _plain_compact(s)
    if kind == "append":
        out.update(c=s["c"], r=s["r"])
        if s["scale"] is not None:
            out["scale"] = s["scale"]
    elif kind == "fork":
        out.update(refs=s["refs"], **s["planes"])
    elif kind == "compact":
        out.update(refs=s["refs"], table=s["table"], **s["planes"])
    return out


# ----------------------------------------------------------------------- what a pass needs

def _page_bytes(c):
    width = c["dc"] + _DR if c["store"] == "latent" else 2 * c["Hkv"] * c["D"]
    return c["layers"] * c["page"] * width * 2


def work(case):
    c = case
    kind = c["kind"]
    if kind == "fork":
        # branches of a prompt that ends inside a page copy that page
        parted = sum(c["branches"] for b in range(c["prompts"]) if _ctx_len(c, b) % c["page"])
        branches = c["prompts"] * c["branches"]
        return {"bytes": 2 * parted * _page_bytes(c) + branches * (_pages(c["ctx"], c["page"]) + 2) * 8, "flops": 0}
    if kind == "compact":
        kept = sum(_pages(_kept(c, b), c["page"]) for b in range(c["B"]))
        n_pages = sum(_pages(_ctx_len(c, b), c["page"]) for b in range(c["B"])) + c["spare"] + 1
        # of pages in no order, a share of those in use lies behind
        moved = kept * (n_pages - kept) // n_pages
        return {"bytes": 2 * moved * _page_bytes(c) + 8 * n_pages, "flops": 0}
    if kind == "expanded":
        region, nbytes, flops = 2 * c["K"] + 3, 0, 0
        for b in range(c["B"]):
            ctx = _ctx_len(c, b)
            keys, rows = ctx + region, region + (ctx if c["form"] == "prefill" else 0)
            pairs = region * keys + (ctx * (ctx + 1) // 2 if c["form"] == "prefill" else 0)
            nbytes += 2 * keys * (2 * c["H"] * c["D"] + _DR) + 2 * rows * c["H"] * (2 * c["D"] + _DR)
            flops += 2 * pairs * c["H"] * (2 * c["D"] + _DR)
        return {"bytes": nbytes, "flops": flops}
    dc = c["dc"]
    held = dc + 4 + 2 * _DR if c["cache"] == _E4M3 else 2 * (dc + _DR)          # bytes of a position
    if kind == "append":
        new, every = sum(_counts(c)), c["B"] * c["n"]
        return {"bytes": new * held + every * (2 * (dc + _DR) * 2 + c["Hq"] * _DR * 4),
                "flops": every * (5 * dc + 3 * _DR * (c["Hq"] + 1))}
    nbytes = flops = 0
    rows = _rows(c)
    for b in range(c["B"]):
        ctx = max(_ctx_len(c, b), rows) if c["form"] == "chunk" else _ctx_len(c, b)
        if c["form"] == "tree":
            keys, pairs = ctx + rows, rows * ctx + rows * (c["depth"] + 1) // 2
        elif c["form"] == "round":
            keys, pairs = ctx + rows, rows * (ctx + rows)
        else:
            keys, pairs = ctx, rows * ctx - rows * (rows - 1) // 2
        nbytes += keys * held + 2 * rows * c["Hq"] * (2 * dc + _DR)
        flops += 2 * pairs * c["Hq"] * (2 * dc + _DR)
    return {"bytes": nbytes, "flops": flops}


# ---------------------------------------------------------------------------- 64-bit results

def exact(case, seed):
    global own
    if case["kind"] in ("fork", "compact"):
        return None                                          # nothing is computed there: bytes move
    asked, own = own, False
    try:
        s = prepare(case, seed)
    finally:
        own = asked
    if case["kind"] == "append":
        return _exact_append(case, s)
    return dict(out=_exact_expanded(case, s) if case["kind"] == "expanded" else _exact_attend(case, s))


def _power(amax):
    """The smallest power of two that brings amax [n] to 448 or less."""
    e = torch.ceil(torch.log2((amax / 448).clamp(min=_LOWEST))).clamp(min=-100)
    s = torch.exp2(e)
    s = torch.where(amax <= 224 * s, s / 2, s)
    return torch.where(amax > 448 * s, 2 * s, s).clamp(min=_LOWEST)


def _turns(x, positions, inv_freq, interleaved):
    """Tokens [n, H, 64], each rotated to its position, as complex numbers."""
    n, H, D = x.shape
    half = inv_freq.numel()
    x = x.double().reshape(n, H, *((half, 2) if interleaved else (2, half)))
    z = torch.complex(*(x.unbind(-1) if interleaved else x.unbind(-2)))
    a = torch.outer(positions.double(), inv_freq.double())
    z = z * torch.polar(torch.ones_like(a), a)[:, None]
    return torch.stack((z.real, z.imag), -1 if interleaved else -2).reshape(n, H, D)


def _exact_append(c, s):
    P, n, B = c["page"], c["n"], c["B"]
    pages, keys = s["c"].double(), s["r"].double()
    scales = None if s["scale"] is None else s["scale"].double()
    starts, counts, table = s["start"].tolist(), s["count"].tolist(), s["table"].tolist()
    q = torch.empty(B, n, c["Hq"], _DR, dtype=torch.float64, device="cuda")
    dense_c = torch.empty(B, n, c["dc"], dtype=torch.float64, device="cuda")
    dense_r = torch.empty(B, n, _DR, dtype=torch.float64, device="cuda")
    for b in range(B):
        at = torch.arange(starts[b], starts[b] + n, device="cuda") + c["far"]
        q[b] = _turns(s["new_q"][b], at, s["inv_freq"], c["interleaved"])
        dense_r[b] = _turns(s["new_r"][b][:, None], at, s["inv_freq"], c["interleaved"])[:, 0]
        x = s["new_c"][b].double()
        if c["norm"]:
            x = x / (torch.linalg.vector_norm(x, dim=-1, keepdim=True) ** 2 / c["dc"] + _EPS).sqrt()
            x = x * s["weight"].double()
        dense_c[b] = x
        power = _power(x.abs().amax(-1))
        for j in range(starts[b] // P, (starts[b] + counts[b] - 1) // P + 1):
            lo, hi = max(starts[b], j * P), min(starts[b] + counts[b], (j + 1) * P)
            new, at = slice(lo - starts[b], hi - starts[b]), slice(lo - j * P, hi - j * P)
            keys[table[b][j], at] = dense_r[b, new]
            pages[table[b][j], at] = x[new] if scales is None else x[new] / power[new, None]
            if scales is not None:
                scales[table[b][j], at] = power[new]
    out = dict(q=q, dense_c=dense_c, dense_r=dense_r, c=pages, r=keys)
    if scales is not None:
        out["scale"] = scales
    return out


def _sees(c, s, b, n, length):
    """Which of `length` keys each of the n queries of sequence b sees."""
    ctx = int(s["ctx"][b])
    sees = torch.zeros(n, length, dtype=torch.bool, device="cuda")
    if c["form"] == "tree":
        rows = []
        for i, p in enumerate(s["parent"][b].tolist()):
            rows.append(([False] * n if p < 0 else list(rows[p])))
            rows[i][i] = True
        sees[:, :ctx] = True
        sees[:, ctx:] = torch.tensor(rows, device="cuda")
        return sees
    p = torch.arange(n, device="cuda") + int(s["q_start"][b])
    at = torch.arange(length, device="cuda")
    sees |= (p[:, None] < ctx) & (at <= p[:, None])
    sees |= (p[:, None] >= ctx) & (p[:, None] < ctx + 2 * c["K"] + 3)
    return sees


def _exact_attend(c, s):
    B, n, Hq, d = s["q"].shape
    P, dc = c["page"], c["dc"]
    out = torch.zeros(B, n, Hq, dc, dtype=torch.float64, device="cuda")
    table = s["table"].long()
    for b in range(B):
        length = int(s["ctx"][b]) + (n if c["form"] in ("tree", "round") else 0)
        pages = table[b, :_pages(length, P)]
        x = _raw(s["c"])[pages].view(s["c"].dtype).double()
        if s["scale"] is not None:
            x = x * s["scale"][pages].double()[..., None]
        x = x.reshape(-1, dc)[:length]
        r = s["r"][pages].double().reshape(-1, _DR)[:length]
        q = s["q"][b].double().reshape(n * Hq, d)
        score = (q[:, :dc] @ x.t().contiguous() + q[:, dc:] @ r.t().contiguous()) * s["scale_qk"]
        sees = _sees(c, s, b, n, length).repeat_interleave(Hq, 0)
        out[b] = (torch.softmax(score.masked_fill(~sees, -math.inf), -1) @ x).reshape(n, Hq, dc)
    return out


def _exact_expanded(c, s):
    B, n, H, d = s["q"].shape
    D = c["D"]
    out = torch.zeros(B, n, H, D, dtype=torch.float64, device="cuda")
    for b in range(B):
        length = int(s["ctx"][b]) + 2 * c["K"] + 3
        sees = _sees(c, s, b, n, length)
        some = sees.any(1)
        for h in range(H):
            k = torch.cat((s["k"][b, :length, h], s["k_r"][b, :length]), -1).double()
            score = s["q"][b, :, h].double() @ k.t().contiguous() * s["scale_qk"]
            w = torch.softmax(score.masked_fill(~sees, -math.inf), -1)
            out[b, some, h] = (w @ s["v"][b, :length, h].double())[some]
    return out
