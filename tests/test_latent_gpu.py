"""The paged cache of latent vectors and its attentions on the GPU against plain 64-bit
implementations (tests/latent_reference.py)."""
import math

import pytest
import torch

import latent_reference as ref
import paper_2605_24793_amd as cs

pytestmark = pytest.mark.gpu
DEV = torch.device("cuda:0")
F8, BF16 = torch.float8_e4m3fn, torch.bfloat16


def _gen(seed):
    return torch.Generator().manual_seed(seed)


def _table(B, T, seed, extra=3):
    n_pages = B * T + extra
    return torch.randperm(n_pages, generator=_gen(seed))[:B * T].reshape(B, T).int(), n_pages


def _filled(table, n_pages, dc, P, dtype, lengths, seed, junk=True, size=1.0):
    """A cache whose sequences hold `lengths[b]` random positions; every other place holds NaN (or zeros)."""
    g = _gen(seed)
    c, r = torch.randn(n_pages, P, dc, generator=g) * size, torch.randn(n_pages, P, 64, generator=g)
    live = torch.zeros(n_pages, P, dtype=torch.bool)
    for b, length in enumerate(lengths):
        for p in range(length):
            pid = int(table[b, p // P])
            if 0 <= pid < n_pages:
                live[pid, p % P] = True
    fill = math.nan if junk else 0.0
    scale = None
    if dtype == F8:
        # |x| < 6 here: 448 * 2^-6 holds it
        scale = 2.0 ** torch.randint(-6, -2, (n_pages, P), generator=g).float() * size
        c = c / scale[:, :, None]
        scale = torch.where(live, scale, fill).to(DEV)
    c = c.masked_fill(~live[:, :, None], fill).to(dtype).to(DEV)
    return cs.LatentCache(c, r.masked_fill(~live[:, :, None], fill).to(BF16).to(DEV), scale)


def _int(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


def _check(out, cache, table, q, sees_of, scale, rows=None):
    """out [B, n, Hq, dc] against the reference, each element within its own bound; `rows`: query positions that
    are looked at (None: all)."""
    host = ref.Latents(cache)
    out = out.double().cpu()
    room = table.shape[1] * cache.page
    for b in range(q.shape[0]):
        c, r, there = host.sequence(table[b])
        sees = sees_of(b, room) & there
        want, off = ref.attend(q[b].cpu(), c, r, sees, scale)
        err = (out[b] - want).abs()
        at = range(q.shape[1]) if rows is None else rows
        for i in at:
            assert torch.isfinite(out[b, i]).all(), (b, i)
            assert bool((err[i] <= off[i]).all()), (b, i, float((err[i] / off[i]).max()))


def _run_hybrid(dtype, dc, P, Hq, ctx, q_start, K, n, seed=0, T=None, scale=0.07, table=None, n_pages=None, q=None, cache=None):
    B = len(ctx)
    ends = [max(c, 0) + 2 * K + 3 for c in ctx]
    T = T or -(-max(max(ends), 1) // P)
    if table is None:
        table, n_pages = _table(B, T, seed)
    if cache is None:
        cache = _filled(table, n_pages, dc, P, dtype, [min(e, T * P) for e in ends], seed)
    if q is None:
        q = (torch.randn(B, n, Hq, dc + 64, generator=_gen(seed + 1)) * 0.6).to(BF16).to(DEV)
    out = cs.latent_attention(q, cache, table.to(DEV), _int(ctx), _int(q_start), K, scale)
    assert tuple(out.shape) == (B, n, Hq, dc)
    _check(out, cache, table, q, lambda b, room: ref.hybrid_sees(ctx[b], q_start[b], K, n, room), scale)
    return out


@pytest.mark.parametrize("dtype", [BF16, F8])
@pytest.mark.parametrize("dc", [512, 256])
@pytest.mark.parametrize("Hq,n,ctx,P", [
    (1, 1, [1, 2, 40], 16), (16, 1, [700, 3, 64, 65], 64), (8, 1, [129], 32), (32, 1, [333, 64], 128), (33, 1, [200, 77], 64),
    (128, 1, [150, 64], 64), (20, 3, [90, 33], 16),
])
def test_the_last_positions_of_a_context(dtype, dc, Hq, n, ctx, P):
    ctx = [max(c, n) for c in ctx]
    _run_hybrid(dtype, dc, P, Hq, ctx, [c - n for c in ctx], 0, n, seed=Hq + n)


@pytest.mark.parametrize("dtype", [BF16, F8])
@pytest.mark.parametrize("dc,Hq,K,ctx,P", [
    (512, 16, 7, [100, 0, 31], 64), (256, 8, 1, [64, 61, 0], 16), (512, 5, 25, [10, 130], 32), (256, 32, 4, [53, 1], 128),
])
def test_the_region(dtype, dc, Hq, K, ctx, P):
    _run_hybrid(dtype, dc, P, Hq, ctx, ctx, K, 2 * K + 3, seed=K)


@pytest.mark.parametrize("dtype", [BF16, F8])
@pytest.mark.parametrize("Hq,n,ctx", [(4, 70, [70, 61, 90]), (16, 40, [33, 0, 200]), (1, 130, [120])])
def test_whole_inputs_and_queries_outside(dtype, Hq, n, ctx):
    # positions from 0 on, the region, and padding behind it; negative starts as well
    _run_hybrid(dtype, 512, 16, Hq, ctx, [0] * len(ctx), 2, n, seed=n)
    _run_hybrid(dtype, 256, 32, Hq, ctx, [-5, 3, 50][:len(ctx)], 2, n, seed=n)


@pytest.mark.parametrize("dtype", [BF16, F8])
def test_odd_lengths_of_context_and_a_short_table(dtype):
    # negative contexts act as 0; the table ends inside the region
    _run_hybrid(dtype, 512, 16, 3, [-4, 0, 13], [0, 0, 13], 5, 13, T=1, seed=5)


@pytest.mark.parametrize("dtype", [BF16, F8])
def test_no_queries_and_no_sequences(dtype):
    cache = cs.LatentCache.empty(4, 512, 16, dtype)
    for B, n in ((0, 3), (2, 0)):
        q = torch.empty(B, n, 4, 576, dtype=BF16, device=DEV)
        out = cs.latent_attention(q, cache, _int([[0]] * B).reshape(B, 1), _int([5] * B), _int([4] * B), 0, 0.1)
        assert tuple(out.shape) == (B, n, 4, 512)


@pytest.mark.parametrize("dtype", [BF16, F8])
@pytest.mark.parametrize("Hq,n,dc", [(16, 1, 512), (32, 5, 512), (64, 1, 256)])
def test_many_pieces_and_segments_of_pages(dtype, Hq, n, dc):
    # 4500 positions in pages of 16: more than are looked up at a time; few rows: cut into pieces
    _run_hybrid(dtype, dc, 16, Hq, [4500, 1100], [4500 - n, 1100 - n], 0, n, seed=3)


def test_a_table_longer_than_the_sequences():
    _run_hybrid(F8, 512, 64, 16, [70, 1, 500], [69, 0, 499], 0, 1, T=60, seed=8)
    _run_hybrid(BF16, 256, 64, 48, [70, 1, 500], [69, 0, 499], 0, 1, T=60, seed=9)


def test_one_workgroup_for_all_keys():
    # as many sequences as CUs: not cut, several segments
    ctx = [20 + 7 * b for b in range(256)] + [4200]
    _run_hybrid(BF16, 256, 16, 1, ctx, [c - 1 for c in ctx], 0, 1, seed=4)


@pytest.mark.parametrize("dtype", [BF16, F8])
def test_missing_pages(dtype):
    P, T = 16, 12
    table, n_pages = _table(3, T, 1)
    cache = _filled(table, n_pages, 512, P, dtype, [180, 180, 180], 2)
    table[0, 3], table[0, 11], table[1, 0], table[1, 1:5] = -1, n_pages, -7, 2 ** 30
    table[2] = -1                                            # nothing at all: zeros
    for n, Hq in ((1, 8), (9, 8)):
        ctx = [177, 150, 100]
        q = (torch.randn(3, n, Hq, 576, generator=_gen(n)) * 0.6).to(BF16).to(DEV)
        qs = [c - n for c in ctx]
        out = cs.latent_attention(q, cache, table.to(DEV), _int(ctx), _int(qs), 0, 0.07)
        _check(out, cache, table, q, lambda b, room: ref.hybrid_sees(ctx[b], qs[b], 0, n, room), 0.07)
        assert bool((out[2] == 0).all())


@pytest.mark.parametrize("scale", [-0.07, 0.0, 1e-30])
def test_scales_of_scores(scale):
    _run_hybrid(F8, 512, 64, 4, [90], [89], 0, 1, scale=scale, seed=1)
    _run_hybrid(BF16, 256, 64, 40, [90], [88], 0, 2, scale=scale, seed=2)


@pytest.mark.parametrize("dtype", [BF16, F8])
@pytest.mark.parametrize("Hq,n,q_start", [(5, 9, -4), (3, 70, 50), (7, 10, 58), (4, 5, -2), (5, 4, 61)])
def test_negative_scales_and_rows_that_see_nothing(dtype, Hq, n, q_start):
    """Queries before the first position and behind the last one, in blocks that are not full, of few rows and of many."""
    _run_hybrid(dtype, 512, 32, Hq, [60, 61], [q_start, q_start], 1, n, seed=n, scale=-0.07)


@pytest.mark.parametrize("dtype", [BF16, F8])
@pytest.mark.parametrize("Hq,n", [(8, 1), (40, 2)])
def test_scores_that_rise_far(dtype, Hq, n):
    # later keys' scores lie far above the first turn's, for some rows: its sums would overflow
    P, T, ctx = 64, 6, 380
    table, n_pages = _table(1, T, 6)
    cache = _filled(table, n_pages, 512, P, dtype, [ctx], 6)
    q = (torch.randn(1, n, Hq, 576, generator=_gen(7)) * 0.6).to(BF16)
    for pos, far in ((100, 30.0), (200, 90.0), (350, 300.0)):
        page = int(table[0, pos // P])
        cache.r[page, pos % P] = (q[0, 0, pos % Hq, 512:].float() * far).to(BF16).to(DEV)
    out = cs.latent_attention(q.to(DEV), cache, table.to(DEV), _int([ctx]), _int([ctx - n]), 0, 0.07)
    _check(out, cache, table, q, lambda b, room: ref.hybrid_sees(ctx, ctx - n, 0, n, room), 0.07)


@pytest.mark.parametrize("dtype", [BF16, F8])
@pytest.mark.parametrize("where", ["latent", "key", "scale"])
@pytest.mark.parametrize("value", [math.nan, math.inf, -math.inf])
def test_what_is_not_finite_stays_with_those_who_see_it(dtype, where, value):
    if where == "scale" and dtype == BF16:
        pytest.skip("bf16 latents have no scales")
    P, n, Hq, ctx, bad = 16, 70, 3, 70, 40
    table, n_pages = _table(1, 5, 9)
    cache = _filled(table, n_pages, 512, P, dtype, [ctx], 9)
    page, slot = int(table[0, bad // P]), bad % P
    q = (torch.randn(1, n, Hq, 576, generator=_gen(9)) * 0.6).to(BF16).to(DEV)
    if where == "latent":
        cache.c[page, slot, 17] = torch.tensor(math.nan if dtype == F8 else value).to(dtype)
    elif where == "key":
        cache.r[page, slot, 5] = value
    else:
        cache.scale[page, slot] = value
    out = cs.latent_attention(q, cache, table.to(DEV), _int([ctx]), _int([0]), 0, 0.07)
    # queries before it: as if it held nothing
    _check(out, cache, table, q, lambda b, room: ref.hybrid_sees(ctx, 0, 0, n, room) & (torch.arange(room) != bad), 0.07,
           rows=range(bad))
    seen = out[0, bad:ctx].float()
    if where == "key" and value != value or where != "key":
        assert bool(torch.isnan(seen).any(-1).all())
    else:
        # an infinite key component: plus infinity (NaN) or minus infinity (weight zero) of a score, by the query's sign
        up = (q[0, bad:ctx, :, 512 + 5].float() * value) > 0
        assert bool(torch.isnan(seen).all(-1)[up].all())
        assert bool(torch.isfinite(seen[~up]).all())


def test_a_query_that_is_not_finite_stays_alone():
    P, n, Hq, ctx = 16, 6, 8, 70
    table, n_pages = _table(1, 5, 9)
    cache = _filled(table, n_pages, 256, P, BF16, [ctx], 9)
    q = (torch.randn(1, n, Hq, 320, generator=_gen(9)) * 0.6).to(BF16)
    bad = q.clone()
    bad[0, 2, 3, 7] = math.nan
    args = (cache, table.to(DEV), _int([ctx]), _int([ctx - n]), 0, 0.07)
    good, out = cs.latent_attention(q.to(DEV), *args), cs.latent_attention(bad.to(DEV), *args)
    assert bool(torch.isnan(out[0, 2, 3]).all())
    out[0, 2, 3] = good[0, 2, 3]
    assert torch.equal(good, out)


def _cut(q, cache, table, ctx, q_start, scale=0.07):
    """cs.latent_attention, of calls whose keys are cut into pieces that are joined."""
    call = cs.prepare_latent_attention(q.to(DEV), cache, table.to(DEV), _int(ctx), _int(q_start), 0, scale)
    assert call.workspace is not None
    call.launch()
    return call.outputs["out"]


@pytest.mark.parametrize("dtype", [BF16, F8])
@pytest.mark.parametrize("dc,n,Hq,ctx", [(256, 1, 8, 300), (512, 1, 32, 2000), (512, 6, 8, 700), (256, 6, 8, 140)])
def test_a_query_that_is_not_finite_stays_alone_over_pieces(dtype, dc, n, Hq, ctx):
    P = 16
    table, n_pages = _table(2, -(-ctx // P), 9)
    cache = _filled(table, n_pages, dc, P, dtype, [ctx, ctx - 9], 9)
    q = (torch.randn(2, n, Hq, dc + 64, generator=_gen(9)) * 0.6).to(BF16)
    bad = q.clone()
    bad[0, n // 2, 3, 7] = math.nan
    args = (cache, table, [ctx, ctx - 9], [ctx - n, ctx - 9 - n])
    good, out = _cut(q, *args), _cut(bad, *args)
    assert bool(torch.isfinite(good).all())
    assert bool(torch.isnan(out[0, n // 2, 3]).all())
    out[0, n // 2, 3] = good[0, n // 2, 3]
    assert torch.equal(good, out)


@pytest.mark.parametrize("dtype", [BF16, F8])
@pytest.mark.parametrize("where", ["latent", "key", "scale"])
@pytest.mark.parametrize("value", [math.nan, math.inf, -math.inf])
@pytest.mark.parametrize("n,Hq,ctx", [(1, 8, 129), (1, 40, 257), (14, 3, 140), (14, 20, 268)])
def test_what_is_not_finite_alone_in_a_piece(dtype, where, value, n, Hq, ctx):
    """The first position of the last piece: a query there sees nothing else in it."""
    if where == "scale" and dtype == BF16:
        pytest.skip("bf16 latents have no scales")
    P, dc = 16, 256
    bad = (ctx - 1) // 128 * 128
    table, n_pages = _table(1, -(-ctx // P), 9)
    cache = _filled(table, n_pages, dc, P, dtype, [ctx], 9)
    page, slot = int(table[0, bad // P]), bad % P
    q = (torch.randn(1, n, Hq, dc + 64, generator=_gen(9)) * 0.6).to(BF16).to(DEV)
    if where == "latent":
        cache.c[page, slot, 17] = torch.tensor(math.nan if dtype == F8 else value).to(dtype)
    elif where == "key":
        cache.r[page, slot, 5] = value
    else:
        cache.scale[page, slot] = value
    first = ctx - n
    out = _cut(q, cache, table, [ctx], [first])
    # queries before it: as if it held nothing
    _check(out, cache, table, q, lambda b, room: ref.hybrid_sees(ctx, first, 0, n, room) & (torch.arange(room) != bad), 0.07,
           rows=range(bad - first))
    seen = out[0, bad - first:].float()
    if where == "key" and value == value:
        # plus infinity (NaN) or minus infinity (weight zero) of a score, by the query's sign
        up = (q[0, bad - first:, :, dc + 5].float() * value) > 0
        assert bool(torch.isnan(seen).all(-1)[up].all())
        assert bool(torch.isfinite(seen[~up]).all())
    else:
        assert bool(torch.isnan(seen).any(-1).all())


@pytest.mark.parametrize("dtype", [BF16, F8])
@pytest.mark.parametrize("n,Hq,ctx", [(1, 8, 64), (1, 40, 128), (1, 8, 256), (3, 20, 640), (1, 8, 300)])
def test_infinite_latents_where_no_score_is_above_minus_infinity(dtype, n, Hq, ctx):
    """Every latent that a query sees is infinite, and every score minus infinity: in one piece and in several."""
    P, dc = 16, 256
    table, n_pages = _table(2, -(-ctx // P), 9)
    cache = _filled(table, n_pages, dc, P, dtype, [ctx, ctx], 9)
    pages = table[0].long().to(DEV)
    if dtype == BF16:
        cache.c[pages, :, 17] = math.inf
    else:
        cache.c[pages] = torch.ones(1, device=DEV).to(F8)
        cache.scale[pages] = math.inf
    q = (torch.rand(2, n, Hq, dc + 64, generator=_gen(9)) * -0.6 - 0.1).to(BF16).to(DEV)
    out = cs.latent_attention(q, cache, table.to(DEV), _int([ctx, ctx]), _int([ctx - n, ctx - n]), 0, 0.07)
    assert bool((~torch.isfinite(out[0])).any(-1).all())
    assert bool(torch.isfinite(out[1]).all())                # (the other sequence)


def _parents(B, N, seed, kind="random"):
    g = _gen(seed)
    p = torch.full((B, N), -1, dtype=torch.int32)
    for b in range(B):
        for i in range(1, N):
            p[b, i] = i - 1 if kind == "path" else 0 if kind == "star" else int(torch.randint(0, i, (1,), generator=g))
    return p


@pytest.mark.parametrize("dtype", [BF16, F8])
@pytest.mark.parametrize("dc,Hq,N,ctx,P,kind", [
    (512, 16, 60, [130, 0, 61], 64, "random"), (256, 4, 256, [77], 16, "random"), (512, 3, 70, [5, 64], 32, "path"),
    (256, 1, 33, [40, 1], 128, "star"), (512, 32, 1, [100], 64, "path"), (512, 1, 17, [700], 16, "random"),
])
def test_trees(dtype, dc, Hq, N, ctx, P, kind):
    B = len(ctx)
    T = -(-(max(ctx) + N) // P)
    table, n_pages = _table(B, T, N)
    cache = _filled(table, n_pages, dc, P, dtype, [c + N for c in ctx], N)
    parent = _parents(B, N, N, kind)
    q = (torch.randn(B, N, Hq, dc + 64, generator=_gen(N)) * 0.6).to(BF16).to(DEV)
    out = cs.latent_tree_attention(q, cache, table.to(DEV), _int(ctx), parent.to(DEV), 0.07)
    _check(out, cache, table, q, lambda b, room: ref.tree_sees(ctx[b], parent[b], room), 0.07)


def test_trees_with_broken_parents_and_no_room():
    N, P, T = 20, 16, 2
    table, n_pages = _table(2, T, 3)
    cache = _filled(table, n_pages, 512, P, BF16, [32, 32], 3)
    parent = _parents(2, N, 3)
    parent[0, 4], parent[0, 7], parent[0, 9], parent[1, 0] = 4, 300, -9, 5
    ctx = [3, 21]                                            # nodes 11 .. 19 of the second have no place
    q = (torch.randn(2, N, 2, 576, generator=_gen(3)) * 0.6).to(BF16).to(DEV)
    out = cs.latent_tree_attention(q, cache, table.to(DEV), _int(ctx), parent.to(DEV), 0.07)
    _check(out, cache, table, q, lambda b, room: ref.tree_sees(ctx[b], parent[b], room), 0.07)
    assert bool((out[1, 11:] == 0).all())


def test_the_hybrid_attention_agrees_where_both_forms_are_one():
    """With latents as keys and values of one head, the absorbed form is the paged attention's, up to roundings: the same
    rows through both."""
    P, d, ctx, n = 64, 128, [200, 64], 3
    table, n_pages = _table(2, 4, 11)
    lat = _filled(table, n_pages, 256, P, BF16, ctx, 11, junk=False)
    lat.c[:, :, d:] = 0
    lat.r.zero_()
    k = lat.c[:, :, :d].reshape(n_pages, 1, P, d).contiguous()
    paged = cs.PagedCache(k, k.transpose(2, 3).contiguous())
    q = (torch.randn(2, n, 4, d, generator=_gen(11)) * 0.6).to(BF16).to(DEV)
    wide = torch.zeros(2, n, 4, 320, dtype=BF16, device=DEV)
    wide[..., :d] = q
    args = (table.to(DEV), _int(ctx), _int([c - n for c in ctx]), 0, 0.1)
    a, b = cs.hybrid_attention_paged(q, paged, *args), cs.latent_attention(wide, lat, *args)
    # each within its own rounding (2^-8) and its weights' (2^-8 of a mean of |v|, at most 6)
    assert bool(((a.float() - b[..., :d].float()).abs() <= 2 * 2.0 ** -8 * (a.float().abs() + 6)).all())
    assert bool((b[..., d:] == 0).all())


# ------------------------------------------------------------------------------- append

def _half_step(x, dtype, scale=None):
    """Half a step of the stored type about x (64 bits), with what 32-bit products add."""
    if dtype == BF16:
        return x.abs() * (2.0 ** -8 + 2.0 ** -20) + 1e-38
    return (x.abs() * 2.0 ** -4).clamp(min=scale * 2.0 ** -10) * (1 + 2.0 ** -16)   # normal, and below 2^-6


def _run_append(dtype, dc, P, n, start, count=None, Hq=0, rot=64, interleaved=False, positions=None, norm=True, seed=0,
                T=None, size=1.0, strided=True, table=None, special=None, dense=True):
    B, g = len(start), _gen(seed)
    T = T or max(-(-(max(max(start), 0) + n) // P), 1)
    if table is None:
        table, n_pages = _table(B, T, seed)
    else:
        n_pages = 4 + B * T
    cache = _filled(table, n_pages, dc, P, dtype, [min(max(s, 0), T * P) for s in start], seed, junk=False)
    before = ref.Latents(cache)
    down = torch.randn(B, n, dc + 64 + (16 if strided else 0), generator=g) * size
    down = down.to(BF16)
    if special:
        special(down)
    dev = down.to(DEV)
    c, k_r = dev[..., :dc], dev[..., dc:dc + 64]
    if not strided:
        c, k_r = c.contiguous(), k_r.contiguous()
    weight = (1 + 0.3 * torch.randn(dc, generator=g)).to(BF16) if norm else None
    inv = (10000.0 ** (-torch.arange(0, rot, 2, dtype=torch.float64) / max(rot, 1))).float() if rot else None
    q = torch.randn(B, n, Hq, 192, generator=g).to(BF16).to(DEV) if Hq else None
    full = torch.full((B, n, Hq, dc + 64), 7.0, dtype=BF16, device=DEV) if Hq else None
    pos = None if positions is None else torch.tensor(positions, dtype=torch.int32)
    outs = cs.latent_append(cache, table.to(DEV), _int(start), c, k_r, None if weight is None else weight.to(DEV), 1e-6,
                            None if count is None else _int(count), None if inv is None else inv.to(DEV),
                            None if pos is None else pos.to(DEV), interleaved, None if q is None else q[..., 128:],
                            None if full is None else full[..., dc:], dense)
    where = pos if pos is not None else torch.tensor(start)[:, None] + torch.arange(n)
    x = ref.normalised(down[..., :dc], weight, 1e-6)
    turned = (lambda t: ref.rotated(t, where, inv, interleaved)) if rot else (lambda t: t.double())
    keys = turned(down[..., dc:dc + 64])
    after = ref.Latents(cache)
    if dense:
        ok = torch.isfinite(x)
        got = outs["c"].double().cpu()
        assert bool(((got - x).abs() <= _half_step(x, BF16))[ok].all())
        assert bool(((outs["k_r"].double().cpu() - keys).abs() <= keys.abs() * 2.0 ** -8 + _angle(keys)).all())
    if Hq:
        want = turned(q[..., 128:].cpu())
        assert bool(((full[..., dc:].double().cpu() - want).abs() <= want.abs() * 2.0 ** -8 + _angle(want)).all())
        assert bool((full[..., :dc] == 7.0).all())
    # what the pages hold now: new places the new values, all others their bytes
    c_want, r_want = before.c.clone(), before.r.clone()
    s_want = None if before.scale is None else before.scale.clone()
    new = torch.zeros(n_pages, P, dtype=torch.bool)
    for b in range(B):
        cnt = n if count is None else min(max(count[b], 0), n)
        for i in range(cnt):
            p = start[b] + i
            if not 0 <= p < T * P:
                continue
            pid = int(table[b, p // P])
            if not 0 <= pid < n_pages:
                continue
            new[pid, p % P] = True
            s = ref.power_for(x[b, i].float().double()) if s_want is not None else 1.0
            if s_want is not None:
                assert float(after.scale[pid, p % P]) == s, (b, i)
            got, want = after.c[pid, p % P] * s, x[b, i]
            ok = torch.isfinite(want)
            assert bool(((got - want).abs() <= _half_step(want, dtype, s))[ok].all()), (b, i)
            if dtype == F8:
                assert bool(torch.isnan(got[~ok]).all())
            assert bool(((after.r[pid, p % P] - keys[b, i]).abs() <= keys[b, i].abs() * 2.0 ** -8 + _angle(keys[b, i])).all())
    assert torch.equal(torch.nan_to_num(after.c[~new]), torch.nan_to_num(before.c[~new]))
    assert torch.equal(after.r[~new], before.r[~new])
    if s_want is not None:
        assert torch.equal(after.scale[~new], before.scale[~new])


def _angle(x):
    """What 32-bit sines and products leave: of values of a few units, 1e-6 each."""
    return 4e-6 * (1 + x.abs().amax())


@pytest.mark.parametrize("dtype", [BF16, F8])
@pytest.mark.parametrize("dc", [512, 256])
@pytest.mark.parametrize("P,n,start,Hq", [
    (16, 1, [0], 1), (64, 1, [63, 64, 5], 16), (32, 5, [30, 0], 33), (128, 7, [125], 4), (16, 40, [9, 70], 0), (64, 3, [1], 128),
])
def test_append(dtype, dc, P, n, start, Hq):
    _run_append(dtype, dc, P, n, start, Hq=Hq, seed=n + Hq)


@pytest.mark.parametrize("dtype", [BF16, F8])
@pytest.mark.parametrize("kw", [
    dict(interleaved=True, Hq=5), dict(rot=32, Hq=3), dict(rot=16, interleaved=True, Hq=3), dict(rot=0, Hq=2), dict(norm=False),
    dict(norm=False, size=1e30), dict(norm=False, size=1e-33), dict(count=[3, 0, 9], Hq=2), dict(count=[-2, 5, 1 << 30]),
    dict(strided=False, dense=False), dict(positions=[[5, 2000000, 0, 7, 2147483647]] * 3, Hq=2),
])
def test_append_forms(dtype, kw):
    _run_append(dtype, 512, 32, 5, [0, 30, 64], seed=3, **kw)


@pytest.mark.parametrize("B,n", [(1, 1), (1, 7), (3, 1), (2, 5)])
def test_one_heads_queries_into_the_attentions(B, n):
    dc, P, g = 256, 16, _gen(B * n)
    table, n_pages = _table(B, 2, 3)
    cache = cs.LatentCache.empty(n_pages, dc, P)
    x = torch.randn(B, n, dc + 64, generator=g).to(BF16).to(DEV)
    q = torch.randn(B, n, 1, 64, generator=g).to(BF16).to(DEV)
    inv_freq = (10000.0 ** (-torch.arange(32) / 32)).to(DEV)
    args = (cache, table.to(DEV), _int([4] * B), x[..., :dc], x[..., dc:])
    want = cs.latent_append(*args, inv_freq=inv_freq, q=q)["q"]
    whole = torch.full((B, n, 1, dc + 64), 7.0, dtype=BF16, device=DEV)
    out = cs.latent_append(*args, inv_freq=inv_freq, q=q, q_out=whole[..., dc:])["q"]
    assert torch.equal(out, want) and torch.equal(whole[..., dc:], want)
    assert bool((whole[..., :dc] == 7).all())


@pytest.mark.parametrize("dtype", [BF16, F8])
def test_append_where_there_is_no_place(dtype):
    # before the first position, behind the last one, on no page
    _run_append(dtype, 256, 16, 6, [-3, 45, -2147483648], T=3, seed=1)
    table, _ = _table(2, 3, 5)
    table[0, 1], table[1, 2] = -1, 1000
    _run_append(dtype, 512, 16, 40, [3, 5], T=3, table=table, seed=2)


def test_append_of_values_that_are_not_finite():
    def special(x):
        x[0, 0, 3], x[0, 1, 200], x[1, 0, 511] = math.inf, math.nan, -math.inf
        x[1, 2, :512] = 0
    _run_append(F8, 512, 16, 3, [0, 5], norm=False, special=special)
    _run_append(BF16, 512, 16, 3, [0, 5], norm=False, special=special)


@pytest.mark.parametrize("dtype", [BF16, F8])
def test_keep(dtype):
    P, N, dc = 16, 60, 512
    ctx = [5, 0, 33, 14, -3]
    table, n_pages = _table(5, 7, 2)
    cache = _filled(table, n_pages, dc, P, dtype, [112] * 5, 2, junk=False)
    paths = [[0, 1, 2], [0, 4, 9, 30, 59], list(range(60)), [0], [0, 3, 60, 5]]
    path = torch.full((5, N), -1, dtype=torch.int32)
    for b, p in enumerate(paths):
        path[b, :len(p)] = torch.tensor(p)
    before = ref.Latents(cache)
    cs.latent_keep(cache, table.to(DEV), _int(ctx), path.to(DEV))
    after = ref.Latents(cache)
    for name in ("c", "r", "scale"):
        old, got = getattr(before, name), getattr(after, name)
        if old is None:
            continue
        want = old.clone()
        for b, p in enumerate(paths):
            for i, node in enumerate(p):
                if node >= N:
                    break
                a, t = max(ctx[b], 0) + node, max(ctx[b], 0) + i
                want[int(table[b, t // P]), t % P] = old[int(table[b, a // P]), a % P]
        assert torch.equal(got, want), name


# ------------------------------------------------------------------------ the expanded form

def _run_expanded(d, H, ctx, q_start, K, n, L=None, seed=0, scale=0.08, apart=False, special=None):
    B, g = len(ctx), _gen(seed)
    L = L or max(max(ctx), 0) + 2 * K + 3
    q = (torch.randn(B, n, H, d + 64, generator=g)).to(BF16)
    kv = torch.randn(B, L, H, 2 * d, generator=g).to(BF16)
    k_r = torch.randn(B, L, 80, generator=g).to(BF16)
    if special:
        special(kv, k_r)
    dev = kv.to(DEV)
    k, v = (dev[..., :d], dev[..., d:]) if not apart else (dev[..., :d].contiguous(), dev[..., d:].contiguous())
    out = cs.expanded_attention(q.to(DEV), k, v, k_r.to(DEV)[..., 8:72], _int(ctx), _int(q_start), K, scale)
    got = out.double().cpu()
    for b in range(B):
        sees = ref.hybrid_sees(ctx[b], q_start[b], K, n, L)
        for h in range(H):
            want, off = _attend_kv(q[b, :, h], kv[b, :, h, :d], k_r[b, :, 8:72], kv[b, :, h, d:], sees, scale)
            assert bool(((got[b, :, h] - want).abs() <= off).all()), (b, h)
    return got


def _attend_kv(q, k, r, v, sees, scale):
    q, key, v = q.double(), torch.cat((k, r), 1).double(), v.double()
    some = sees.any(1)
    s = (q @ key.t() * scale).masked_fill(~sees, -math.inf)
    w = torch.zeros_like(s)
    w[some] = torch.softmax(s[some], -1)
    rough = (q.abs() @ key.abs().t() * abs(scale)).masked_fill(~sees, 0).amax(-1, keepdim=True)
    slack = (q.shape[1] + 2) * ref.F32_HALF_STEP * rough * 2 + 1e-6
    out = w @ v
    return out, 1.1 * (2.0 ** -8 * out.abs() + (2.0 ** -8 + 2 * slack) * (w @ v.abs())) + 1e-30


@pytest.mark.parametrize("d", [128, 64])
@pytest.mark.parametrize("H,ctx,K,n,start", [
    (3, [100, 61], 2, None, 0), (1, [300], 7, None, 0), (5, [40, 0, 7], 5, 13, None), (2, [200, 130], 1, 5, None), (9, [64], 0, 1, 63),
    (2, [1, 0], 0, 3, 0), (4, [127, 129, 128], 0, 260, -3),
])
def test_expanded(d, H, ctx, K, n, start):
    n = n or max(ctx) + 2 * K + 3
    _run_expanded(d, H, ctx, ctx if start is None else [start] * len(ctx), K, n, seed=n)


def test_expanded_with_arrays_of_their_own_and_short_ones():
    _run_expanded(128, 4, [50, 30], [0, 0], 3, 59, apart=True, seed=1)
    _run_expanded(64, 2, [50, 30], [0, 0], 3, 59, L=40, seed=2)          # l is cut to L
    _run_expanded(128, 2, [-5], [0], 2, 9, seed=3)
    _run_expanded(128, 2, [90], [0], 2, 97, scale=-0.08, seed=4)


@pytest.mark.parametrize("n", [97, 200])
def test_expanded_values_that_are_not_finite(n):
    """Queries before it do not notice."""
    ctx, bad, d = n - 7, 50, 128
    g = _gen(5)
    q = torch.randn(1, n, 2, d + 64, generator=g).to(BF16).to(DEV)
    kv = torch.randn(1, n, 2, 2 * d, generator=g).to(BF16).to(DEV)
    k_r = torch.randn(1, n, 64, generator=g).to(BF16).to(DEV)
    args = (k_r, _int([ctx]), _int([0]), 2, 0.08)
    good = cs.expanded_attention(q, kv[..., :d], kv[..., d:], *args)
    for part, value in ((d + 3, math.nan), (d + 3, math.inf), (4, math.nan)):
        x = kv.clone()
        x[0, bad, 1, part] = value
        out = cs.expanded_attention(q, x[..., :d], x[..., d:], *args)
        assert torch.equal(out[0, :bad], good[0, :bad])
        assert torch.equal(out[0, :, 0], good[0, :, 0])
        assert bool((~torch.isfinite(out[0, bad:, 1])).any(-1).all())


@pytest.mark.parametrize("d", [128, 64])
@pytest.mark.parametrize("ctx,n", [(64, 1), (64, 9), (256, 130)])
def test_expanded_values_that_are_not_finite_where_no_score_is_above_minus_infinity(d, ctx, n):
    g = _gen(5)
    q = -torch.rand(1, n, 2, d + 64, generator=g).to(BF16).to(DEV) - 0.1
    kv = torch.randn(1, ctx, 2, 2 * d, generator=g).to(BF16).to(DEV)
    k_r = torch.randn(1, ctx, 64, generator=g).to(BF16).to(DEV)
    args = (k_r, _int([ctx]), _int([ctx - n]), 0, 0.08)
    good = cs.expanded_attention(q, kv[..., :d], kv[..., d:], *args)
    kv[0, :, 1, 4] = math.inf                               # a component of every key
    kv[0, 3, 1, d + 10] = math.nan                          # one of a value that all queries see
    out = cs.expanded_attention(q, kv[..., :d], kv[..., d:], *args)
    assert bool(torch.isnan(out[0, :, 1, 10]).all())
    assert torch.equal(out[0, :, 0], good[0, :, 0])


@pytest.mark.parametrize("d", [128, 64])
@pytest.mark.parametrize("layout", ["heads first", "one key for all", "wide"])
def test_expanded_strides(d, layout):
    """Heads before positions, one position's key and value for every position, and rows of 2^24 bytes and more."""
    L, H, ctx, K, n = 150, 2, 140, 2, 150
    g = _gen(8)
    q = torch.randn(1, n, H, d + 64, generator=g).to(BF16)
    k, v = (torch.randn(1, L, H, d, generator=g).to(BF16) for _ in range(2))
    k_r = torch.randn(1, L, 64, generator=g).to(BF16)
    if layout == "heads first":
        dk, dv = (x.to(DEV).transpose(1, 2).contiguous().transpose(1, 2) for x in (k, v))
    elif layout == "one key for all":
        k, v = (x[:, :1].expand(1, L, H, d) for x in (k, v))
        dk, dv = (x[:, :1].contiguous().to(DEV).expand(1, L, H, d) for x in (k, v))
    else:
        room = torch.empty(1, L, 2 ** 23 + 1024, dtype=BF16, device=DEV)
        wide = room[..., :2 * H * d].view(1, L, 2 * H, d)
        wide.copy_(torch.cat((k, v), 2).to(DEV))
        dk, dv = wide[:, :, :H], wide[:, :, H:]
    got = cs.expanded_attention(q.to(DEV), dk, dv, k_r.to(DEV), _int([ctx]), _int([0]), K, 0.08).double().cpu()
    sees = ref.hybrid_sees(ctx, 0, K, n, L)
    for h in range(H):
        want, off = _attend_kv(q[0, :, h], k[0, :, h], k_r[0], v[0, :, h], sees, 0.08)
        assert bool(((got[0, :, h] - want).abs() <= off).all()), h


def test_expanded_scores_that_rise():
    def special(kv, k_r):
        for j, far in ((70, 8.0), (150, 40.0)):
            kv[:, j, :, :128] = (kv[:, j, :, :128].float() * far).to(BF16)
    _run_expanded(128, 2, [180], [0], 1, 185, seed=6, special=special)


# --------------------------------------------------------------------------- a large cache

@pytest.mark.parametrize("dtype", [BF16, F8])
def test_places_past_32_bits(dtype):
    """The last pages of a cache whose latents, and then some, lie past 2^32 bytes, against the same in a small cache."""
    P, dc, T, n = 64, 512, 8, 250
    n_pages = 2 ** 32 // (P * dc * (2 if dtype == BF16 else 1)) + 40
    near, g = torch.tensor([[3, 1, 2, 0]]), _gen(31)
    tables = [near.int().to(DEV), (n_pages - T + near).int().to(DEV)]
    caches = [cs.LatentCache.empty(T, dc, P, dtype), cs.LatentCache.empty(n_pages, dc, P, dtype)]
    down = torch.randn(1, n, dc + 64, generator=g).to(BF16).to(DEV)
    queries = [(torch.randn(1, m, Hq, dc + 64, generator=g) * 0.6).to(BF16).to(DEV) for m, Hq in ((1, 16), (5, 32))]
    path = _int([[0, 2, 4] + [-1] * 5])
    outs = []
    for cache, table in zip(caches, tables):
        cs.latent_append(cache, table, _int([0]), down[..., :dc], down[..., dc:])
        outs.append([cs.latent_attention(q, cache, table, _int([n - 7]), _int([n - 9]), 2, 0.07) for q in queries])
        outs[-1].append(cs.latent_tree_attention(queries[1], cache, table, _int([n - 5]), _int([[-1, 0, 0, 1, 2]]), 0.07))
        cs.latent_keep(cache, table, _int([n - 8]), path)
        cs.pages_copy(cs.PagePool.empty(cache.n_pages, P), [cache], table.view(2, 2) + _int([0, 4]))
    for a, b in zip(*outs):
        assert torch.isfinite(a).all() and torch.equal(a, b)
    for small, large in zip(caches[0]._planes(), caches[1]._planes()):
        small, large = (x.view(torch.uint8) for x in (small, large[-T:]))
        # pages 3 and 2 went to places 1 + 4 and 0 + 4; page 0 has places that nothing was written to
        assert torch.equal(small[[1, 2, 3, 4, 5]], large[[1, 2, 3, 4, 5]]) and torch.equal(small[0, :n % P], large[0, :n % P])
        assert torch.equal(large[5], large[3]) and torch.equal(large[4], large[2])


# ----------------------------------------------------------------- as a serving loop uses them

def test_a_round_of_a_latent_layer():
    """Whole inputs into the cache and through the expanded form; the same through the absorbed form agree, as W_h and
    U_h are the heads' expansions; a tree appended, attended, and its path kept; the next token."""
    g = _gen(21)
    B, P, dc, H, d = 2, 64, 512, 4, 128
    ctx = [90, 57]
    n = max(ctx)
    pool_pages, T = 8, 3
    table = torch.randperm(pool_pages, generator=g)[:B * T].reshape(B, T).int().to(DEV)
    cache = cs.LatentCache.empty(pool_pages, dc, P, F8)
    weight = (1 + 0.2 * torch.randn(dc, generator=g)).to(BF16).to(DEV)
    inv = (10000.0 ** (-torch.arange(0, 64, 2, dtype=torch.float64) / 64)).float().to(DEV)
    up = (torch.randn(H, dc, 2 * d, generator=g) * dc ** -0.5).to(DEV)     # [head][latent][key, value]
    down = torch.randn(B, n, dc + 64, generator=g).to(BF16).to(DEV)
    q = torch.randn(B, n, H, d + 64, generator=g).to(BF16).to(DEV)
    absorbed = torch.empty(B, n, H, dc + 64, dtype=BF16, device=DEV)
    absorbed[..., :dc] = torch.stack([q[:, :, h, :d].float() @ up[h, :, :d].t().contiguous() for h in range(H)], 2).to(BF16)
    out = cs.latent_append(cache, table, _int([0, 0]), down[..., :dc], down[..., dc:], weight, count=_int(ctx), inv_freq=inv,
                           q=q[..., d:], q_out=absorbed[..., dc:], dense=True)
    kv = torch.stack([out["c"].float() @ up[h] for h in range(H)], 2).to(BF16)
    full = torch.cat((q[..., :d], absorbed[..., dc:]), -1).contiguous()
    scale = (d + 64) ** -0.5
    # (K = 0: three positions of a region after the context, which no query asks for)
    a = cs.expanded_attention(full, kv[..., :d], kv[..., d:], out["k_r"], _int(ctx), _int([0, 0]), 0, scale)
    o = cs.latent_attention(absorbed, cache, table, _int(ctx), _int([0, 0]), 0, scale)
    b = torch.stack([o[:, :, h].float() @ up[h, :, d:] for h in range(H)], 2)
    for s in range(B):
        x, y = a[s, :ctx[s]].float(), b[s, :ctx[s]]
        # e4m3 latents: 2^-4 at most each, 2^-5.6 of their size in the mean square, of sums of many
        assert float((x - y).norm() / x.norm()) < 0.06
    # a tree of 5 nodes
    N = 5
    parent = _int([[-1, 0, 0, 1, 3]] * B)
    depth = torch.tensor([0, 1, 1, 2, 3], dtype=torch.int32, device=DEV)
    positions = (_int(ctx)[:, None] + depth).contiguous()
    node = torch.randn(B, N, dc + 64, generator=g).to(BF16).to(DEV)
    tq = (torch.randn(B, N, H, dc + 64, generator=g) * 0.5).to(BF16).to(DEV)
    cs.latent_append(cache, table, _int(ctx), node[..., :dc], node[..., dc:], weight, inv_freq=inv, positions=positions)
    out = cs.latent_tree_attention(tq, cache, table, _int(ctx), parent, scale)
    _check(out, cache, table.cpu(), tq, lambda s, room: ref.tree_sees(ctx[s], parent[s].cpu(), room), scale)
    # nodes 0, 1, 3 were accepted: the path as a sequence of its own gives the same
    kept = out[:, 3].clone()
    path = torch.full((B, N), -1, dtype=torch.int32)
    path[:, :3] = torch.tensor([0, 1, 3], dtype=torch.int32)
    cs.latent_keep(cache, table, _int(ctx), path.to(DEV))
    last = [c + 3 for c in ctx]
    again = cs.latent_attention(tq[:, 3:4].contiguous(), cache, table, _int(last), _int([x - 1 for x in last]), 0, scale)
    assert bool(((again[:, 0].float() - kept.float()).abs() <= 2 * 2.0 ** -8 * (kept.float().abs() + 4)).all())


def test_prepared_calls_read_their_tensors_anew_and_on_other_streams():
    P, ctx = 16, [100, 37]
    table, n_pages = _table(2, 7, 1)
    cache = _filled(table, n_pages, 512, P, F8, [112, 112], 1, junk=False)
    q = (torch.randn(2, 1, 16, 576, generator=_gen(1)) * 0.6).to(BF16).to(DEV)
    length, start = _int(ctx), _int([c - 1 for c in ctx])
    call = cs.prepare_latent_attention(q, cache, table.to(DEV), length, start, 0, 0.07)
    call.launch()
    first = call.outputs["out"].clone()
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        length.copy_(_int([60, 90]))
        start.copy_(_int([59, 89]))
        call.launch()
    torch.cuda.current_stream().wait_stream(s)
    _check(call.outputs["out"], cache, table, q, lambda b, room: ref.hybrid_sees([60, 90][b], [59, 89][b], 0, 1, room), 0.07)
    assert not torch.equal(first, call.outputs["out"])


def test_captured_calls():
    """Append, both attentions and keep in one graph, replayed with other lengths between eager calls."""
    P, B, N, dc, H = 32, 3, 9, 256, 8
    table, n_pages = _table(B, 8, 2)
    dev = table.to(DEV)

    def fresh():
        return _filled(table, n_pages, dc, P, F8, [256] * B, 2, junk=False)

    g = _gen(4)
    new = torch.randn(B, N, dc + 64, generator=g).to(BF16).to(DEV)
    q = (torch.randn(B, N, H, dc + 64, generator=g) * 0.6).to(BF16).to(DEV)
    kv = torch.randn(B, 40, H, 256, generator=g).to(BF16).to(DEV)
    qe = torch.randn(B, N, H, 192, generator=g).to(BF16).to(DEV)
    inv = (10000.0 ** (-torch.arange(0, 64, 2, dtype=torch.float64) / 64)).float().to(DEV)
    parent, path = _parents(B, N, 1).to(DEV), torch.full((B, N), -1, dtype=torch.int32, device=DEV)
    path[:, :3] = _int([0, 2, 5])
    ctx, rows = _int([0] * B), _int([0] * B)

    def calls(cache):
        return [cs.prepare_latent_append(cache, dev, ctx, new[..., :dc], new[..., dc:], inv_freq=inv),
                cs.prepare_latent_tree_attention(q, cache, dev, ctx, parent, 0.07),
                cs.prepare_latent_attention(q, cache, dev, ctx, rows, 3, 0.07),
                cs.prepare_expanded_attention(qe, kv[..., :128], kv[..., 128:], new[:, :1, :64].expand(B, 40, 64).contiguous(), ctx,
                                              rows, 3, 0.08),
                cs.prepare_latent_keep(cache, dev, ctx, path)]

    caches = [fresh(), fresh()]
    eager, held = calls(caches[0]), calls(caches[1])
    for c in held:
        c.launch()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        for c in held:
            c.launch()
    for lengths in ([3, 40, 100], [0, 1, 200], [64, 31, 95], [3, 40, 100]):
        ctx.copy_(_int(lengths))
        rows.copy_(_int(lengths))
        for cache in caches:
            again = fresh()
            cache.c.view(torch.uint8).copy_(again.c.view(torch.uint8))
            cache.r.copy_(again.r)
            cache.scale.copy_(again.scale)
        for c in eager:
            c.launch()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(eager, held):
            for name in a.outputs:
                assert torch.equal(a.outputs[name], b.outputs[name]), name
        assert torch.equal(caches[0].c.view(torch.uint8), caches[1].c.view(torch.uint8))
        assert torch.equal(caches[0].r, caches[1].r) and torch.equal(caches[0].scale, caches[1].scale)


def test_the_same_bits_every_time():
    q = (torch.randn(2, 5, 32, 576, generator=_gen(1)) * 0.6).to(BF16).to(DEV)
    table, n_pages = _table(2, 40, 1)
    cache = _filled(table, n_pages, 512, 64, F8, [2560, 2560], 1)
    args = (q, cache, table.to(DEV), _int([2500, 1777]), _int([2495, 1772]), 0, 0.07)
    first = cs.latent_attention(*args)
    for _ in range(5):
        assert torch.equal(first, cs.latent_attention(*args))


def test_the_binding_refuses():
    cache = cs.LatentCache.empty(4, 512, 16, F8)
    q = torch.zeros(1, 1, 4, 576, dtype=BF16, device=DEV)
    t, one = _int([[0, 1]]), _int([1])
    bad = [lambda: cs.latent_attention(q[..., :512], cache, t, one, one, 0, 0.1),
           lambda: cs.latent_attention(q.float(), cache, t, one, one, 0, 0.1),
           lambda: cs.latent_attention(q, cache, t.long(), one, one, 0, 0.1),
           lambda: cs.latent_attention(q, cache, t, one.long(), one, 0, 0.1),
           lambda: cs.latent_tree_attention(q, cache, t, one, _int([[0, 1]]), 0.1),
           lambda: cs.latent_append(cache, t, one, q[:, :, 0, :512].float(), q[:, :, 0, 512:]),
           lambda: cs.latent_append(cache, t, one, q[:, :, 0, :512], q[:, :, 0, 512:], q_out=q[..., :64]),
           lambda: cs.latent_append(cache, t, one, q[:, :, 0, :512], q[:, :, 0, 512:], torch.ones(512, device=DEV)),
           lambda: cs.LatentCache(cache.c, cache.r), lambda: cs.LatentCache(cache.c.to(BF16), cache.r, cache.scale),
           lambda: cs.LatentCache(cache.c, cache.r.float(), cache.scale),
           lambda: cs.expanded_attention(q, q[..., :128], q[..., :128], q[:, :, 0, :64], one, one, 0, 0.1)]
    for call in bad:
        with pytest.raises((ValueError, TypeError, cs.CospecError)):
            call()
