"""The paged key/value cache of a speculative round and the attentions that read it: cases,
their inputs, a plain form of every operator, its work and its 64-bit result.

A case is a dict of plain values.  Its `kind` names the operator:

  append  new keys (rotated to their positions) and values into the pages, the queries rotated
          beside them (`prepare_cache_append`)
  hybrid  the arbitrator's hybrid attention over the pages (`prepare_hybrid_attention_paged`);
          `form`: "round" for the region's 2K + 3 queries, "token" for the last position alone,
          "prefill" for every position
  tree    the attention of a token tree's nodes over the pages (`prepare_tree_attention`)
  keep    the accepted path of a tree moved to the front of the tree's places
          (`prepare_cache_keep`)

`cache` is the pages' element type: "bf16", or "e4m3" (8 bits) with one power-of-two scale for
each page and head.  A page's keys are [head][token][d], its values [head][d][token].

Keys are N(0, 1) with a few strong channels, as trained models have them, and the first
position's key lies along the mean query, so that part of the weight goes there; everything is
made on the GPU from the seed.  Lengths follow from the case alone.
"""
from __future__ import annotations

import math

import torch

own = False

_BF16, _E4M3 = "bf16", "e4m3"
_LOWEST = 2.0 ** -100          # scale of a page that holds nothing but zeros


def listed():
    return [
        # one user, one new token: latency is everything
        dict(name="append_token", kind="append", cache=_E4M3, B=1, n=1, start=2000, ragged=False, far=0, rot=128,
             interleaved=False, page=64, Hq=32, Hkv=8, D=128),
        # the arbitrator's region of a serving batch (K = 7), in place of the last round's
        dict(name="append_round", kind="append", cache=_E4M3, B=64, n=17, start=500, ragged=True, far=0, rot=128,
             interleaved=False, page=64, Hq=32, Hkv=8, D=128),
        # whole inputs into a bf16 cache
        dict(name="append_prefill_bf16", kind="append", cache=_BF16, B=4, n=2065, start=0, ragged=True, far=0, rot=128,
             interleaved=False, page=64, Hq=32, Hkv=8, D=128),
        # one round of a serving batch, the framework's attention benchmark with an 8-bit cache
        dict(name="round", kind="hybrid", form="round", cache=_E4M3, B=64, ctx=2048, K=7, page=64, Hq=32, Hkv=8, D=128),
        # a smaller batch with a bf16 cache in small pages
        dict(name="round_bf16", kind="hybrid", form="round", cache=_BF16, B=16, ctx=1024, K=5, page=16, Hq=32, Hkv=8,
             D=128),
        # two users with long contexts
        dict(name="long", kind="hybrid", form="round", cache=_E4M3, B=2, ctx=16384, K=7, page=64, Hq=32, Hkv=8, D=128),
        # plain decoding of a batch, one token each
        dict(name="token", kind="hybrid", form="token", cache=_E4M3, B=64, ctx=4096, K=0, page=64, Hq=32, Hkv=8, D=128),
        # the first pass over whole inputs: the matrix cores bound it
        dict(name="prefill", kind="hybrid", form="prefill", cache=_E4M3, B=4, ctx=2048, K=7, page=64, Hq=32, Hkv=8,
             D=128),
        # trees of 60 nodes of a serving batch
        dict(name="tree", kind="tree", cache=_E4M3, B=64, ctx=2048, depth=6, page=64, Hq=32, Hkv=8, D=128),
        # one user's tree, smaller heads, bf16
        dict(name="tree_one_bf16", kind="tree", cache=_BF16, B=1, ctx=1000, depth=4, page=32, Hq=16, Hkv=8, D=64),
        # the accepted paths of the same batch
        dict(name="keep", kind="keep", cache=_E4M3, B=64, ctx=500, depth=6, page=64, Hkv=8, D=128),
        # and of a small one
        dict(name="keep_bf16", kind="keep", cache=_BF16, B=8, ctx=300, depth=4, page=32, Hkv=8, D=64),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["append", "append", "hybrid", "hybrid", "hybrid", "tree", "keep"])
    cache = rng.choice([_E4M3, _E4M3, _BF16])
    Hq, Hkv = rng.choice([(32, 8), (32, 8), (16, 4), (16, 8), (28, 4), (8, 8)])
    D = rng.choice([128, 128, 64])
    page = rng.choice([16, 32, 64, 128])
    if kind == "append":
        n = rng.choice([1, rng.randint(2, 60), _log_int(rng, 60, 2000)])
        B = max(1, min(_log_int(rng, 1, 96), 8000 // n))
        return dict(kind=kind, cache=cache, B=B, n=n, start=_log_int(rng, 1, 900), ragged=rng.random() < 0.5,
                    far=rng.choice([0, 0, 100003]), rot=rng.choice([D, D, D // 2]), interleaved=rng.random() < 0.3,
                    page=page, Hq=Hq, Hkv=Hkv, D=D)
    if kind == "hybrid":
        form = rng.choice(["round", "round", "token", "prefill"])
        K = rng.choice([1, 4, 5, 7, 10, 15, 25])
        if form == "prefill":
            ctx = _log_int(rng, 60, 2000)
            B = max(1, min(_log_int(rng, 1, 12), int(3.5 * 2048.0 ** 2 / ctx ** 2)))
        elif form == "token":
            ctx = _log_int(rng, 30, 20000)
            B = max(1, min(_log_int(rng, 1, 64), 250000 // ctx))
        else:
            ctx = _log_int(rng, 100, 20000)
            B = max(1, min(_log_int(rng, 1, 64), 130000 // ctx))
        return dict(kind=kind, form=form, cache=cache, B=B, ctx=ctx, K=K, page=page, Hq=Hq, Hkv=Hkv, D=D)
    depth = rng.randint(2, 8)
    if kind == "tree":
        ctx = _log_int(rng, 40, 8000)
        return dict(kind=kind, cache=cache, B=max(1, min(_log_int(rng, 1, 48), 100000 // ctx)), ctx=ctx, depth=depth,
                    page=page, Hq=Hq, Hkv=Hkv, D=D)
    return dict(kind=kind, cache=cache, B=_log_int(rng, 1, 64), ctx=_log_int(rng, 1, 500), depth=depth, page=page,
                Hkv=Hkv, D=D)


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


def _path(c, b):
    """Node ids of the accepted path of tree b, root first: the draft's first choice, then a
    node of every level, none of them among the places the path moves to."""
    s = 2 + b % c["depth"]
    return [0, 1] + [max(s, 5 + 11 * (d - 2) + (7 * b + 3 * d) % 11) for d in range(2, s)]


# ------------------------------------------------------------------------------- inputs

def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(int(seed) * 1000003 + 29)


def _randn(g, *shape):
    return torch.randn(*shape, generator=g, device="cuda")


def _int32(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def _scale_of(amax):
    """The smallest power of two s with amax <= 448 s."""
    m, e = torch.frexp(amax)
    s = torch.ldexp(torch.ones_like(amax), torch.where(m > 0.875, e - 8, e - 9)).clamp(min=_LOWEST)
    return torch.where(amax > 0, s, _LOWEST)


def _to_pages(x, c, table):
    """Keys or values [B, L, H, D] into the pages of `table` [B, T]: pages [B T, H, page, D] and
    their scales [B T, H] (None for bf16)."""
    B, L, H, D = x.shape
    T, P = table.shape[1], c["page"]
    x = torch.nn.functional.pad(x, (0, 0, 0, 0, 0, T * P - L))
    x = x.reshape(B * T, P, H, D).permute(0, 2, 1, 3)
    pages = torch.empty(B * T, H, P, D, device="cuda")
    pages[table.reshape(-1)] = x
    if c["cache"] == _BF16:
        return pages.bfloat16(), None
    scale = _scale_of(pages.abs().amax((2, 3)))
    return (pages / scale[:, :, None, None]).to(torch.float8_e4m3fn), scale


def _cache(c, g, lengths, room, along=None):
    """A cache that holds lengths[b] positions of sequence b, with room for `room` positions;
    `along`: where the first key of every head [H, D] lies."""
    B, H, D, P = c["B"], c["Hkv"], c["D"], c["page"]
    L, T = max(max(lengths), 1), -(-room // P)
    live = (torch.arange(L, device="cuda")[None, :] < _int32(lengths)[:, None]).float()[:, :, None, None]
    strong = torch.ones(D, device="cuda")
    strong[torch.randperm(D, generator=g, device="cuda")[:D // 32]] = 4.0
    k = _randn(g, B, L, H, D).mul_(strong)
    if along is not None:
        k[:, 0] = along
    table = torch.randperm(B * T, generator=g, device="cuda").reshape(B, T)
    s = dict(table=table.int())
    s["k"], s["k_scale"] = _to_pages(k.mul_(live).bfloat16().float(), c, table)
    del k
    v, s["v_scale"] = _to_pages(_randn(g, B, L, H, D).mul_(live).bfloat16().float(), c, table)
    s["v"] = v.transpose(2, 3).contiguous()
    return s


def _queries(c, g, n):
    """Queries [B, n, Hq, D] about a mean of their head group's, and the first key along it."""
    B, Hq, Hkv, D = c["B"], c["Hq"], c["Hkv"], c["D"]
    mean = _randn(g, Hkv, D) * 0.7
    q = _randn(g, B, n, Hkv, Hq // Hkv, D) + mean[:, None]
    return q.reshape(B, n, Hq, D).bfloat16(), mean * 1.2


def _parents(c, g):
    """Node 0, its 4 children, then levels of 11 nodes under random nodes of the level before."""
    B, parts = c["B"], [torch.full((c["B"], 1), -1), torch.zeros(c["B"], 4)]
    first, width = 1, 4
    for _ in range(c["depth"] - 1):
        parts.append(first + (torch.rand(B, 11, generator=g, device="cuda") * width).long().cpu())
        first, width = first + width, 11
    return torch.cat(parts, 1).int().cuda()


def prepare(case, seed):
    c = dict(case)
    g = _gen(seed)
    kind, B = c["kind"], c["B"]
    if kind == "append":
        n, Hq, Hkv, D = c["n"], c["Hq"], c["Hkv"], c["D"]
        starts = _starts(c) if c["start"] else [0] * B
        s = _cache(c, g, starts, max(starts) + n)
        s["start"], s["count"] = _int32(starts), _int32(_counts(c))
        # one projection's output holds queries, keys and values side by side
        qkv = _randn(g, B, n, (Hq + 2 * Hkv) * D).bfloat16()
        s["new_q"] = qkv[:, :, :Hq * D].unflatten(2, (Hq, D))
        s["new_k"] = qkv[:, :, Hq * D:(Hq + Hkv) * D].unflatten(2, (Hkv, D))
        s["new_v"] = qkv[:, :, (Hq + Hkv) * D:].unflatten(2, (Hkv, D))
        s["inv_freq"] = (500000.0 ** (-torch.arange(0, c["rot"], 2, dtype=torch.float64, device="cuda")
                                      / c["rot"])).float()
        at = s["start"][:, None] + torch.arange(n, device="cuda", dtype=torch.int32)
        s["positions"] = (at + c["far"]).int() if c["far"] else None
    elif kind == "keep":
        lengths = [_ctx_len(c, b) for b in range(B)]
        N = _tree_nodes(c)
        s = _cache(c, g, [x + N for x in lengths], max(lengths) + N)
        s["ctx"] = _int32(lengths)
        paths = [_path(c, b) for b in range(B)]
        s["path"] = _int32([p + [-1] * (N - len(p)) for p in paths])
    else:
        ctx = [_ctx_len(c, b) for b in range(B)]
        if kind == "tree":
            n = _tree_nodes(c)
            lengths = [x + n for x in ctx]
        elif c["form"] == "token":
            n, lengths = 1, ctx
        else:
            region = 2 * c["K"] + 3
            n, lengths = region + (c["ctx"] if c["form"] == "prefill" else 0), [x + region for x in ctx]
        q, along = _queries(c, g, n)
        s = _cache(c, g, lengths, max(lengths), along)
        s["q"], s["ctx"], s["scale"] = q, _int32(ctx), c["D"] ** -0.5
        if kind == "tree":
            s["parent"] = _parents(c, g)
        else:
            s["q_start"] = _int32([0 if c["form"] == "prefill" else x - 1 if c["form"] == "token" else x for x in ctx])
    s["case"] = c
    if own:
        import paper_2605_24793_amd as cs
        cache = cs.PagedCache(s["k"], s["v"], s["k_scale"], s["v_scale"])
        if kind == "append":
            s["call"] = cs.prepare_cache_append(cache, s["table"], s["start"], s["new_k"], s["new_v"], count=s["count"],
                                                inv_freq=s["inv_freq"], positions=s["positions"],
                                                interleaved=c["interleaved"], q=s["new_q"])
        elif kind == "hybrid":
            s["call"] = cs.prepare_hybrid_attention_paged(s["q"], cache, s["table"], s["ctx"], s["q_start"], c["K"],
                                                          s["scale"])
        elif kind == "tree":
            s["call"] = cs.prepare_tree_attention(s["q"], cache, s["table"], s["ctx"], s["parent"], s["scale"])
        else:
            s["call"] = cs.prepare_cache_keep(cache, s["table"], s["ctx"], s["path"])
    return s


# ------------------------------------------------------------------------- the plain forms

def _rotated(x, positions, inv_freq, interleaved):
    """x [B, n, H, D] rotated, in 64 bits: angles of far positions, and values next to a border
    of the 8-bit type."""
    a = (positions.double()[:, :, None] * inv_freq.double())[:, :, None]
    cos, sin, half = a.cos(), a.sin(), inv_freq.numel()
    x = x.double()
    r = x[..., :2 * half]
    x1, x2 = (r[..., 0::2], r[..., 1::2]) if interleaved else (r[..., :half], r[..., half:])
    y1, y2 = x1 * cos - x2 * sin, x2 * cos + x1 * sin
    y = torch.stack((y1, y2), -1).flatten(-2) if interleaved else torch.cat((y1, y2), -1)
    return torch.cat((y, x[..., 2 * half:]), -1)


def _bytes(pages):
    return pages.view(torch.uint8) if pages.dtype == torch.float8_e4m3fn else pages


def _as(x, pages):
    """Values in the pages' type, as _bytes() has it."""
    return x.float().to(pages.dtype).view(torch.uint8) if pages.dtype == torch.float8_e4m3fn else x.to(pages.dtype)


def _write(pages, scale, x, dim, start, tok, pid, slot, table):
    """Writes tokens x [B, n, H, D] to slot `slot` of page `pid` [B, n]; `dim`: the pages' token
    dimension.  A sequence's places past its count repeat its first token, so that they write
    what is written there anyway."""
    b = torch.arange(x.shape[0], device="cuda")
    x = x[b[:, None], tok]
    raw = _bytes(pages)
    if scale is not None:
        H, P = scale.shape[1], pages.shape[dim]
        heads = torch.arange(H, device="cuda")
        flat = (pid[:, :, None] * H + heads).reshape(-1)
        amax = torch.zeros(scale.numel(), dtype=x.dtype, device="cuda").scatter_reduce(
            0, flat, x.abs().amax(-1).reshape(-1), "amax")
        need = _scale_of(amax).float().reshape(scale.shape)
        # the page that the first token goes to may hold earlier tokens: its scale only grows,
        # and they are rounded anew
        held = (start % P)[:, None, None, None]
        first = table[b, start // P]
        old = scale[first]
        fresh = scale.clone()
        fresh.view(-1)[flat] = need.view(-1)[flat]
        fresh[first] = torch.where(held[:, :, 0, 0] > 0, torch.maximum(need[first], old), need[first])
        scale.copy_(fresh)
        page = pages[first].float() * (old / fresh[first])[:, :, None, None]
        earlier = torch.arange(P, device="cuda")
        earlier = (earlier[:, None] if dim == 2 else earlier) < held
        raw[first] = torch.where(earlier, _as(page, pages), raw[first])
        x = x / fresh[pid][..., None]
    x = _as(x, pages)
    if dim == 2:
        raw[pid, :, slot] = x
    else:
        raw[pid, :, :, slot] = x


def _plain_append(s):
    c = s["case"]
    n, P = c["n"], c["page"]
    start = s["start"].long()
    i = torch.arange(n, device="cuda")
    at = start[:, None] + i if s["positions"] is None else s["positions"]
    q = _rotated(s["new_q"], at, s["inv_freq"], c["interleaved"]).bfloat16()
    k = _rotated(s["new_k"], at, s["inv_freq"], c["interleaved"])
    tok = torch.where(i < s["count"][:, None], i, 0)
    place = start[:, None] + tok
    table = s["table"].long()
    pid, slot = table.gather(1, place // P), place % P
    _write(s["k"], s["k_scale"], k, 2, start, tok, pid, slot, table)
    _write(s["v"], s["v_scale"], s["new_v"].float(), 3, start, tok, pid, slot, table)
    return q


def _gathered(pages, scale, table):
    """Pages [n, H, P, D] of every sequence in order, as 32-bit values [B, H, T P, D]."""
    x = pages[table].float()
    if scale is not None:
        x = x * scale[table][..., None, None]
    B, T, H, P, D = x.shape
    return x.transpose(1, 2).reshape(B, H, T * P, D)


def _plain_attention(s):
    c = s["case"]
    q, table, ctx = s["q"], s["table"].long(), s["ctx"].long()
    B, n, Hq, D = q.shape
    k = _gathered(s["k"], s["k_scale"], table)
    v = _gathered(s["v"].transpose(2, 3), s["v_scale"], table)
    H, L = k.shape[1], k.shape[2]
    x = q.float().reshape(B, n, H, Hq // H, D).permute(0, 2, 3, 1, 4).reshape(B, H, Hq // H * n, D)
    score = torch.matmul(x, k.transpose(2, 3).contiguous()).reshape(B, H, Hq // H, n, L) * s["scale"]
    key = torch.arange(L, device="cuda")
    if c["kind"] == "tree":
        seen = _ancestors(torch.eye(n, dtype=torch.bool, device="cuda").expand(B, n, n),
                          s["parent"].long().clamp(min=0))
        own_key = (key - ctx[:, None]).clamp(0, n - 1)[:, None].expand(B, n, L)
        in_tree = (key >= ctx[:, None]) & (key < ctx[:, None] + n)
        mask = (key < ctx[:, None])[:, None] | (in_tree[:, None] & seen.gather(2, own_key))
        live = torch.ones(B, n, dtype=torch.bool, device="cuda")
    else:
        end = (ctx + 2 * c["K"] + 3).clamp(max=L)
        p = s["q_start"].long()[:, None] + torch.arange(n, device="cuda")
        live = (p >= 0) & (p < end[:, None])
        mask = key < torch.where(p < ctx[:, None], p + 1, end[:, None])[:, :, None]
    score = score.masked_fill(~mask[:, None, None], -math.inf)
    w = torch.exp(score - score.amax(-1, keepdim=True))
    out = torch.matmul((w / w.sum(-1, keepdim=True)).reshape(B, H, -1, L), v).reshape(B, H, Hq // H, n, D)
    out = out.permute(0, 3, 1, 2, 4).reshape(B, n, Hq, D)
    return torch.where(live[:, :, None, None], out, 0).bfloat16()


def _ancestors(seen, up):
    # doubling the steps up: at most 128 nodes here, so seven reach the root from everywhere
    seen, up = _doubled(*_doubled(*_doubled(*_doubled(seen, up))))
    return _doubled(*_doubled(*_doubled(seen, up)))[0]


def _doubled(seen, up):
    return seen | seen.gather(1, up[:, :, None].expand_as(seen)), up.gather(1, up)


def _plain_keep(s):
    c = s["case"]
    P = c["page"]
    ctx, path, table = s["ctx"].long(), s["path"].long(), s["table"].long()
    B, N = path.shape
    i = torch.arange(N, device="cuda")
    # entries past a path's end move its root, which stays where it is
    to = torch.where(path >= 0, i, 0)
    place, source = ctx[:, None] + to, ctx[:, None] + path.gather(1, to)
    pid, slot, table_from = table.gather(1, place // P), place % P, table.gather(1, source // P)
    b = torch.arange(B, device="cuda")
    _move(s["k"], s["k_scale"], 2, ctx, b, pid, slot, table_from, source % P, table)
    _move(s["v"], s["v_scale"], 3, ctx, b, pid, slot, table_from, source % P, table)


def _move(pages, scale, dim, ctx, b, pid, slot, pid_from, slot_from, table):
    raw = _bytes(pages)
    old = raw[pid_from, :, slot_from] if dim == 2 else raw[pid_from, :, :, slot_from]
    if scale is not None:
        H, P = scale.shape[1], pages.shape[dim]
        value = old.view(pages.dtype).float() * scale[pid_from][..., None]
        flat = (pid[:, :, None] * H + torch.arange(H, device="cuda")).reshape(-1)
        need = torch.zeros(scale.numel(), device="cuda").scatter_reduce(
            0, flat, scale[pid_from].reshape(-1), "amax").reshape(scale.shape)
        held = (ctx % P)[:, None, None, None]
        first = table[b, ctx // P]
        before = scale[first]
        fresh = scale.clone()
        fresh.view(-1)[flat] = need.view(-1)[flat]
        fresh[first] = torch.where(held[:, :, 0, 0] > 0, torch.maximum(need[first], before), need[first])
        scale.copy_(fresh)
        page = pages[first].float() * (before / fresh[first])[:, :, None, None]
        earlier = torch.arange(P, device="cuda")
        earlier = (earlier[:, None] if dim == 2 else earlier) < held
        raw[first] = torch.where(earlier, _as(page, pages), raw[first])
        old = _as(value / fresh[pid][..., None], pages)
    if dim == 2:
        raw[pid, :, slot] = old
    else:
        raw[pid, :, :, slot] = old


def run(state):
    s = state
    kind = s["case"]["kind"]
    if own:
        s["call"].launch()
        out = s["call"].outputs
        q = out.get("q")
        attended = out.get("out")
    elif kind == "append":
        q = _plain_append(s)
    elif kind == "keep":
        _plain_keep(s)
    else:
        attended = _plain_attention(s)
    if kind in ("hybrid", "tree"):
        return dict(out=attended)
    held = dict(k=s["k"], v=s["v"])
    if s["k_scale"] is not None:
        held.update(k_scale=s["k_scale"], v_scale=s["v_scale"])
    if kind == "append":
        held.update(q=q)
    return held


# ----------------------------------------------------------------------- what a pass needs

def work(case):
    c = case
    kind, D, Hkv = c["kind"], c["D"], c["Hkv"]
    held = 1 if c["cache"] == _E4M3 else 2                   # bytes of a stored element
    if kind == "append":
        new = sum(_counts(c))
        pages = sum(-(-(s % c["page"] + k) // c["page"]) for s, k in zip(_starts(c) if c["start"] else [0] * c["B"],
                                                                        _counts(c)))
        nbytes = new * 2 * Hkv * D * (2 + held) + c["B"] * c["n"] * c["Hq"] * D * 4
        if held == 1:
            nbytes += pages * 2 * Hkv * 4 + c["B"] * 2 * Hkv * 4
        return {"bytes": nbytes, "flops": 3 * (new * Hkv + c["B"] * c["n"] * c["Hq"]) * c["rot"]}
    if kind == "keep":
        # the root, and the draft's first choice, stay where they are
        moved = sum(len(_path(c, b)) - 2 for b in range(c["B"]))
        return {"bytes": 2 * moved * 2 * Hkv * D * held + c["B"] * _tree_nodes(c) * 4, "flops": 0}
    nbytes = flops = 0
    for b in range(c["B"]):
        ctx = _ctx_len(c, b)
        if kind == "tree":
            rows = _tree_nodes(c)
            keys, pairs = ctx + rows, rows * ctx + rows * (c["depth"] + 1) // 2
        elif c["form"] == "token":
            rows, keys, pairs = 1, ctx, ctx
        else:
            region = 2 * c["K"] + 3
            rows, keys, pairs = region, ctx + region, region * (ctx + region)
            if c["form"] == "prefill":
                rows, pairs = c["ctx"] + region, pairs + ctx * (ctx + 1) // 2
        nbytes += 2 * keys * Hkv * D * held + 2 * rows * c["Hq"] * D * 2
        if held == 1:
            nbytes += 2 * -(-keys // c["page"]) * Hkv * 4
        flops += 4 * pairs * c["Hq"] * D
    return {"bytes": nbytes, "flops": flops}


# ---------------------------------------------------------------------------- 64-bit results

def exact(case, seed):
    global own
    asked, own = own, False
    try:
        s = prepare(case, seed)
    finally:
        own = asked
    kind = case["kind"]
    if kind == "append":
        return _exact_append(case, s)
    if kind == "keep":
        return _exact_keep(case, s)
    return dict(out=_exact_attention(case, s))


def _power(amax):
    """The smallest power of two that brings amax [H] to 448 or less."""
    e = torch.ceil(torch.log2((amax / 448).clamp(min=_LOWEST))).clamp(min=-100)
    s = torch.exp2(e)
    s = torch.where(amax <= 224 * s, s / 2, s)
    return torch.where(amax > 448 * s, 2 * s, s).clamp(min=_LOWEST)


def _turns(x, positions, inv_freq, interleaved):
    """Tokens [n, H, D], each rotated to its position, as complex numbers."""
    n, H, D = x.shape
    half = inv_freq.numel()
    out = x.double().clone()
    r = out[..., :2 * half].reshape(n, H, *((half, 2) if interleaved else (2, half)))
    z = torch.complex(*(r.unbind(-1) if interleaved else r.unbind(-2)))
    a = torch.outer(positions.double(), inv_freq.double())
    z = z * torch.polar(torch.ones_like(a), a)[:, None]
    out[..., :2 * half] = torch.stack((z.real, z.imag), -1 if interleaved else -2).reshape(n, H, 2 * half)
    return out


def _exact_append(c, s):
    P, n = c["page"], c["n"]
    k, v = s["k"].double(), s["v"].double().transpose(2, 3).contiguous()
    ks, vs = (None, None) if s["k_scale"] is None else (s["k_scale"].double(), s["v_scale"].double())
    starts, counts, table = s["start"].tolist(), s["count"].tolist(), s["table"].tolist()
    q = torch.empty(c["B"], n, c["Hq"], c["D"], dtype=torch.float64, device="cuda")
    for b in range(c["B"]):
        at = torch.arange(starts[b], starts[b] + n, device="cuda") + c["far"]
        q[b] = _turns(s["new_q"][b], at, s["inv_freq"], c["interleaved"])
        news = (_turns(s["new_k"][b], at, s["inv_freq"], c["interleaved"]), s["new_v"][b].double())
        for x, pages, scales in zip(news, (k, v), (ks, vs)):
            for j in range(starts[b] // P, (starts[b] + counts[b] - 1) // P + 1):
                lo, hi = max(starts[b], j * P), min(starts[b] + counts[b], (j + 1) * P)
                part = x[lo - starts[b]:hi - starts[b]].transpose(0, 1)          # [H, tokens, D]
                page = pages[table[b][j]]
                if scales is not None:
                    new = _power(part.abs().amax((1, 2)))
                    kept = lo - j * P
                    if kept:
                        new = torch.maximum(new, scales[table[b][j]])
                        page[:, :kept] *= (scales[table[b][j]] / new)[:, None, None]
                    scales[table[b][j]] = new
                    part = part / new[:, None, None]
                page[:, lo - j * P:hi - j * P] = part
    out = dict(k=k, v=v.transpose(2, 3).contiguous(), q=q)
    if ks is not None:
        out.update(k_scale=ks, v_scale=vs)
    return out


def _exact_keep(c, s):
    P = c["page"]
    ctx, table = s["ctx"].tolist(), s["table"].tolist()
    out = {}
    for name in ("k", "v"):
        pages, scales = s[name].double(), s[name + "_scale"]
        pages = pages if name == "k" else pages.transpose(2, 3).contiguous()
        scales = None if scales is None else scales.double()
        for b in range(c["B"]):
            path, page_of = _path(c, b), table[b]
            # values and scales as they were
            moved = []
            for i, node in enumerate(path):
                pid = page_of[(ctx[b] + node) // P]
                x = pages[pid][:, (ctx[b] + node) % P].clone()
                moved.append((x, torch.ones(x.shape[0], dtype=x.dtype, device="cuda") if scales is None else scales[pid].clone()))
            for j in range(ctx[b] // P, (ctx[b] + len(path) - 1) // P + 1):
                places = [i for i in range(len(path)) if (ctx[b] + i) // P == j]
                new = torch.stack([moved[i][1] for i in places]).amax(0)
                page = pages[page_of[j]]
                kept = (ctx[b] + places[0]) % P
                if scales is not None:
                    if kept:
                        new = torch.maximum(new, scales[page_of[j]])
                        page[:, :kept] *= (scales[page_of[j]] / new)[:, None, None]
                    scales[page_of[j]] = new
                for i in places:
                    page[:, (ctx[b] + i) % P] = moved[i][0] * (moved[i][1] / new)[:, None]
        out[name] = pages if name == "k" else pages.transpose(2, 3).contiguous()
        if scales is not None:
            out[name + "_scale"] = scales
    return out


def _exact_attention(c, s):
    B, n, Hq, D = s["q"].shape
    P, H = c["page"], c["Hkv"]
    out = torch.zeros(B, n, Hq, D, dtype=torch.float64, device="cuda")
    ctx, table = s["ctx"].tolist(), s["table"].long()
    for b in range(B):
        length = ctx[b] + (n if c["kind"] == "tree" else 2 * c["K"] + 3)
        pages = table[b, :-(-length // P)]
        k, v = s["k"][pages].double(), s["v"][pages].double().transpose(2, 3)
        if s["k_scale"] is not None:
            k, v = k * s["k_scale"][pages].double()[..., None, None], v * s["v_scale"][pages].double()[..., None, None]
        k, v = (x.transpose(0, 1).reshape(H, -1, D)[:, :length] for x in (k, v))
        length = k.shape[1]
        sees = torch.zeros(n, length, dtype=torch.bool, device="cuda")
        if c["kind"] == "tree":
            rows = []
            for i, p in enumerate(s["parent"][b].tolist()):
                rows.append(([False] * n if p < 0 else list(rows[p])))
                rows[i][i] = True
            sees[:, :ctx[b]] = True
            sees[:, ctx[b]:] = torch.tensor(rows, device="cuda")
        else:
            p = torch.arange(n, device="cuda") + int(s["q_start"][b])
            at = torch.arange(length, device="cuda")
            sees |= (p[:, None] < ctx[b]) & (at <= p[:, None])
            sees |= (p[:, None] >= ctx[b]) & (p[:, None] < length)
        some = sees.any(1)
        for h in range(Hq):
            x = s["q"][b, :, h].double() @ k[h // (Hq // H)].t().contiguous() * s["scale"]
            w = torch.softmax(x.masked_fill(~sees, -math.inf), -1)
            out[b, some, h] = (w @ v[h // (Hq // H)])[some]
    return out
