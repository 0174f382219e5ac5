"""The paged key/value cache and its attentions on the GPU against plain 64-bit
implementations (tests/cache_reference.py)."""
import math

import pytest
import torch

import cache_reference as ref
import paper_2605_24793_amd as cs

pytestmark = pytest.mark.gpu
DEV = torch.device("cuda:0")
F8, BF16 = torch.float8_e4m3fn, torch.bfloat16


def _gen(seed):
    return torch.Generator().manual_seed(seed)


def _filled(table, n_pages, H, D, P, dtype, lengths, seed, junk=True):
    """A cache whose sequences hold `lengths[b]` random positions; every other place, and the
    scales of unused pages, hold NaN (`junk`) or zeros."""
    g = _gen(seed)
    k = torch.randn(n_pages, H, P, D, generator=g)
    v = torch.randn(n_pages, H, P, D, generator=g)
    live = torch.zeros(n_pages, P, dtype=torch.bool)
    for b, length in enumerate(lengths):
        for p in range(length):
            pid = int(table[b, p // P])
            if 0 <= pid < n_pages:
                live[pid, p % P] = True
    scales = [None, None]
    if dtype == F8:
        # |x| < 6 here: 448 * 2^-6 holds it
        scales = [2.0 ** torch.randint(-6, -2, (n_pages, H), generator=g).float() for _ in range(2)]
        k, v = k / scales[0][:, :, None, None], v / scales[1][:, :, None, None]
        scales = [torch.where(live.any(1)[:, None], s, math.nan if junk else 1.0) for s in scales]
    dead = ~live[:, None, :, None]
    k, v = (x.masked_fill(dead, math.nan if junk else 0.0).to(dtype) for x in (k, v))
    dev = [k.to(DEV), v.transpose(2, 3).contiguous().to(DEV)] + [None if s is None else s.to(DEV) for s in scales]
    return cs.PagedCache(*dev)


def _host(cache):
    return ref.Pages(cache.k, cache.v, cache.k_scale, cache.v_scale)


def _bits(x):
    return x.contiguous().view(torch.uint8)


def _same(a, b):
    """The same bits, but that e4m3 has two codes for NaN, which differ in the sign."""
    x, y = _bits(a), _bits(b)
    if a.dtype == F8:
        x, y = (torch.where((t & 127) == 127, 127, t) for t in (x, y))
    return bool((x == y).all())


# ------------------------------------------------------------------------------- append

def _check_append(dtype, D, P, H, n, start, count=None, rot=None, interleaved=False, Hq=0, positions=None, seed=0,
                  T=None, strided=False, size=1.0, table=None, special=None):
    B = len(start)
    g = _gen(seed)
    T = T or (max(max(start), 0) + n + P - 1) // P
    if table is None:
        table, n_pages = ref.make_table(B, T, seed)
    else:
        n_pages = int(table.max()) + 3
    cache = _filled(table, n_pages, H, D, P, dtype, [min(max(s, 0), T * P) for s in start], seed, junk=False)
    heads = Hq + 2 * H
    wide = torch.randn(B, n, heads * D + (24 if strided else 0), generator=g) * size
    wide = wide.to(BF16)
    if special:
        special(wide)
    dev = wide.to(DEV)
    at = [0, Hq * D, (Hq + H) * D, heads * D]
    parts = [wide[:, :, at[i]:at[i + 1]].reshape(B, n, -1, D) for i in range(3)]
    views = [dev[:, :, at[i]:at[i + 1]].unflatten(2, ((at[i + 1] - at[i]) // D, D)) if at[i + 1] > at[i] else None
             for i in range(3)]
    rot = D if rot is None else rot
    inv_freq = (10000.0 ** (-torch.arange(0, rot, 2).double() / rot)).float() if rot else None
    i32 = lambda x: None if x is None else torch.tensor(x, dtype=torch.int32)  # noqa: E731
    pos, cnt = i32(positions), i32(count)
    host = _host(cache)
    before = _host(cache)
    news = ref.append(host, table, start, parts[1], parts[2], count, inv_freq, pos, interleaved)
    on = lambda t: None if t is None else t.to(DEV)  # noqa: E731
    got_q = cs.cache_append(cache, on(table), on(i32(start)), views[1], views[2], count=on(cnt), inv_freq=on(inv_freq),
                            positions=on(pos), interleaved=interleaved, q=views[0])
    torch.cuda.synchronize()
    got = _host(cache)
    for side in ("k", "v"):
        if dtype == F8:
            assert torch.equal(got.scale[side], host.scale[side]), side
        want = host.raw[side].clone()
        for pid, place, x in news[side]:
            # the largest pair bounds the rotation's fp32 error (three roundings and the angle's)
            fp32 = 2.0 ** -21 * float(x[torch.isfinite(x)].abs().max()) if torch.isfinite(x).any() else 0.0
            y = got.raw[side][pid, :, place].double()
            s = host.scale[side][pid].double()[:, None] if dtype == F8 else torch.ones(H, 1, dtype=torch.float64)
            real = torch.isfinite(x)
            if dtype == F8:
                assert torch.isnan(y[~real]).all()
                # half a step of e4m3: relative 2^-4, or 2^-10 among the subnormals
                tol = torch.maximum(2.0 ** -4 * x.abs(), 2.0 ** -10 * s) + fp32
            else:
                tol = 2.0 ** -8 * x.abs() + fp32
                assert torch.equal(torch.isnan(y[~real]), torch.isnan(x[~real]))
            assert ((y * s - x).abs() <= tol)[real].all(), (side, pid, place)
            want[pid, :, place] = got.raw[side][pid, :, place]
        # nothing else has changed, but for the earlier values of pages whose scale grew
        assert _same(got.raw[side], want), side
    if Hq:
        p0 = torch.tensor(start)[:, None] + torch.arange(n) if pos is None else pos
        for b in range(B):
            for i in range(n):
                x = ref.rotate(parts[0][b, i], int(p0[b, i]), inv_freq, interleaved) if rot else parts[0][b, i].double()
                tol = 2.0 ** -8 * x.abs() + 2.0 ** -21 * float(x.abs().max())
                assert ((got_q[b, i].cpu().double() - x).abs() <= tol).all()
    return before, got


@pytest.mark.parametrize("dtype", [F8, BF16])
@pytest.mark.parametrize("D,P,H,n,start", [
    (128, 64, 2, 1, [0]), (128, 64, 2, 1, [63, 64, 65]), (64, 16, 3, 5, [14, 0, 16]), (128, 128, 1, 130, [126, 7]),
    (64, 32, 2, 37, [31, 95]), (128, 16, 2, 70, [3, 33]),
])
def test_append(dtype, D, P, H, n, start):
    _check_append(dtype, D, P, H, n, start, Hq=2 * H, seed=n)


@pytest.mark.parametrize("dtype", [F8, BF16])
@pytest.mark.parametrize("rot,interleaved", [(0, False), (16, False), (32, True), (64, True), (48, False)])
def test_append_rotations(dtype, rot, interleaved):
    _check_append(dtype, 64, 32, 2, 9, [29, 4], rot=rot, interleaved=interleaved, Hq=3, strided=True, seed=rot)


@pytest.mark.parametrize("dtype", [F8, BF16])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("rot,P,n,start", [(128, 128, 117, [9, 100]), (64, 128, 130, [0, 77]), (48, 16, 20, [5, 16]),
                                           (128, 32, 1, [31, 32]), (112, 64, 70, [60, 1])])
def test_append_rotations_of_wide_heads(dtype, interleaved, rot, P, n, start):
    # d = 128: eight units a token, up to four of a thread; all of the components rotated, or the first ones
    _check_append(dtype, 128, P, 2, n, start, rot=rot, interleaved=interleaved, Hq=3, strided=True, seed=rot + n)


@pytest.mark.parametrize("dtype", [F8, BF16])
def test_append_positions_and_counts(dtype):
    # tree nodes rotated to their depth, far positions, counts of nothing, too many, too few
    n, start = 6, [10, 61, 0, 5, 40]
    positions = [[s + 1000003 + (i + 1) // 2 for i in range(n)] for s in start]
    _check_append(dtype, 128, 64, 2, n, start, count=[0, 6, 99, -4, 3], positions=positions, Hq=2, T=2)


@pytest.mark.parametrize("dtype", [F8, BF16])
def test_append_outside_the_room(dtype):
    # before position 0, past the table, on entries that name no page
    table = torch.tensor([[4, 1], [-1, 6], [2, 9], [7, 3]], dtype=torch.int32)
    table[2, 1] = 10 ** 9
    n_pages_table = table.clone()
    cache_pages = 12
    B, H, D, P, n = 4, 2, 64, 16, 20
    start = [-7, 10, 10, 30]
    safe = torch.where((table < 0) | (table >= cache_pages), torch.full_like(table, -1), table)
    cache = _filled(safe, cache_pages, H, D, P, dtype, [0, 10, 10, 30], 3, junk=False)
    g = _gen(5)
    k, v = (torch.randn(B, n, H, D, generator=g).to(BF16) for _ in range(2))
    host = _host(cache)
    news = ref.append(host, n_pages_table, start, k, v, None, None, None, False)
    cs.cache_append(cache, table.to(DEV), torch.tensor(start, dtype=torch.int32, device=DEV), k.to(DEV), v.to(DEV))
    torch.cuda.synchronize()
    got = _host(cache)
    # 13 of the first (seven lie before position 0), 14 on the second's real page, 6 on the third's, 2 of the last
    assert len(news["k"]) == 13 + 14 + 6 + 2
    for side in ("k", "v"):
        want = host.raw[side].clone()
        for pid, place, x in news[side]:
            want[pid, :, place] = got.raw[side][pid, :, place]
            s = host.scale[side][pid].double()[:, None] if dtype == F8 else 1.0
            assert ((got.raw[side][pid, :, place].double() * s - x).abs() <= 2.0 ** -4 * x.abs() + 2.0 ** -10).all()
        assert _same(got.raw[side], want)


@pytest.mark.parametrize("dtype", [F8, BF16])
@pytest.mark.parametrize("n", [2, 17, 200])
@pytest.mark.parametrize("count", [None, 0, 1])
def test_append_far_outside_writes_nothing(dtype, n, count):
    # the lowest and the highest position that a start can name, and tokens that end before position 0
    low, high = -(1 << 31), (1 << 31) - 1
    start = [low, low + 1, low + n, high, high - n, -n]
    B = len(start)
    table, n_pages = ref.make_table(B, 16, 2)
    cache = _filled(table, n_pages, 2, 128, 64, dtype, [1000] * B, 2, junk=False)
    before = [t.clone() for t in (cache.k, cache.v, cache.k_scale, cache.v_scale) if t is not None]
    g = _gen(3)
    k, v, q = (torch.randn(B, n, h, 128, generator=g).to(BF16).to(DEV) for h in (2, 2, 4))
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device=DEV)  # noqa: E731
    got = cs.cache_append(cache, table.to(DEV), i32(start), k, v, count=None if count is None else i32([count] * B), q=q)
    torch.cuda.synchronize()
    for a, b in zip(before, (t for t in (cache.k, cache.v, cache.k_scale, cache.v_scale) if t is not None)):
        assert _same(a, b)
    assert torch.equal(got, q)


@pytest.mark.parametrize("size", [300.0, 1e-3, 3e38, 1e-36])
def test_append_scales_grow_and_keep(size):
    # far larger values: earlier ones are rounded anew; far smaller ones: the scale stays
    _check_append(F8, 128, 64, 2, 3, [40, 62, 0], rot=0, size=size, seed=7)


def test_append_values_without_a_number():
    def special(x):
        x[0, 0, 3], x[0, 1, 200], x[1, 2, 70] = math.inf, math.nan, -math.inf
        x[1, 0] = 0.0
    for dtype in (F8, BF16):
        _check_append(dtype, 64, 32, 2, 3, [5, 31], rot=0, special=special)


def test_append_after_values_without_a_number():
    """Earlier values of a page whose scale grows: NaN stays NaN, the others are rounded anew."""
    table, n_pages = ref.make_table(1, 1, 1)
    cache = _filled(table, n_pages, 2, 64, 32, F8, [20], 1, junk=False)
    for x in (cache.k, cache.v):
        _bits(x)[:, :, 3:9] |= 127
    k, v = (torch.randn(1, 2, 2, 64, generator=_gen(i)).mul(1000).to(BF16) for i in range(2))
    host = _host(cache)
    news = ref.append(host, table, [20], k, v, None, None, None, False)
    cs.cache_append(cache, table.to(DEV), torch.tensor([20], dtype=torch.int32, device=DEV), k.to(DEV), v.to(DEV))
    torch.cuda.synchronize()
    got = _host(cache)
    pid = int(table[0, 0])
    for side in ("k", "v"):
        assert len(news[side]) == 2 and bool(torch.isnan(host.raw[side][pid, :, :20].float()).any())
        assert _same(got.raw[side][pid, :, :20], host.raw[side][pid, :, :20])


def test_append_again_changes_nothing_more():
    table, n_pages = ref.make_table(2, 2, 1)
    cache = _filled(table, n_pages, 2, 128, 64, F8, [50, 3], 1, junk=False)
    g = _gen(2)
    k, v = (torch.randn(2, 20, 2, 128, generator=g).to(BF16).to(DEV) for _ in range(2))
    call = cs.prepare_cache_append(cache, table.to(DEV), torch.tensor([50, 3], dtype=torch.int32, device=DEV), k, v)
    call.launch()
    once = [t.clone() for t in (cache.k, cache.v, cache.k_scale, cache.v_scale)]
    call.launch()
    for a, b in zip(once, (cache.k, cache.v, cache.k_scale, cache.v_scale)):
        assert _same(a, b)


# ----------------------------------------------------------------------------- attention

def _tolerance(out, size):
    # with weights off by e_j, |e_j| <= 2^-8 (half a bf16 step), in the product and in their sum alike,
    # out is off by sum(w_j e_j (v_j - out)) / (1 + sum(w_j e_j)) <= 2^-8 (size + |out|) to first order,
    # size = sum(w |v|); the result is stored off by at most 2^-8 of it.  Scores in fp32: D + 4
    # roundings of at most sum |q k| scale < 20, on both sides of the quotient, below 4e-4.
    return (2.0 ** -8 + 4e-4) * (size + out.abs()) + 2.0 ** -8 * out.abs() + 1e-30


def _check_rows(got, out, size):
    err = (got.double().cpu() - out).abs()
    worst = float((err / _tolerance(out, size)).max()) if err.numel() else 0.0
    print(f"worst error {worst:.3f} of the tolerance", flush=True)
    assert not torch.isnan(got.float()).any()
    assert (err <= _tolerance(out, size)).all()


def _longer(table, columns):
    """The table with more entries behind, which name no page: room for long sequences, which the
    kernels' work split goes by as long as it does not know better."""
    return torch.cat([table, torch.full((table.shape[0], columns), -1, dtype=torch.int32)], 1)


def _check_hybrid(dtype, D, P, Hq, H, ctx, q_start, n_q, K, T=None, scale=None, seed=0, spoil=None,
                  only=None, more=0):
    B = len(ctx)
    need = max(max(c, 0) for c in ctx) + 2 * K + 3
    T = T or (need + P - 1) // P
    table, n_pages = ref.make_table(B, T, seed)
    lengths = [min(max(c, 0) + 2 * K + 3, T * P) for c in ctx]
    if spoil:
        spoil(table)
    table = _longer(table, more)
    room = table.shape[1] * P
    cache = _filled(table, n_pages, H, D, P, dtype, lengths, seed)
    g = _gen(seed + 1)
    q = torch.randn(B, n_q, Hq, D, generator=g).to(BF16)
    scale = D ** -0.5 if scale is None else scale
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device=DEV)  # noqa: E731
    got = cs.hybrid_attention_paged(q.to(DEV), cache, table.to(DEV), i32(ctx), i32(q_start), K, scale)
    torch.cuda.synchronize()
    host = _host(cache)
    for b in only or range(B):
        sees = torch.tensor(ref.hybrid_sees(ctx[b], q_start[b], n_q, K, room))
        mask = torch.arange(lengths[b]) < sees[:, None]
        out, size = ref.attention(q[b], host.of("k", table[b], lengths[b]), host.of("v", table[b], lengths[b]), mask,
                                  scale)
        _check_rows(got[b], out, size)


@pytest.mark.parametrize("dtype", [F8, BF16])
@pytest.mark.parametrize("D,P,Hq,H,ctx,n_q,K", [
    (128, 64, 8, 2, [100, 61, 0], 9, 3),          # the region's queries
    (64, 16, 6, 2, [1, 15, 33], 3, 0),            # groups of three heads
    (128, 16, 4, 4, [250, 777], 17, 7),           # one head a group
    (128, 128, 14, 2, [130, 5], 5, 1),            # groups of seven
    (64, 32, 16, 2, [64, 200], 13, 5),            # 104 rows a group
    (128, 32, 8, 1, [40, 321], 23, 10),           # 184 rows
])
@pytest.mark.parametrize("more", [0, 3000])
def test_hybrid_region(dtype, D, P, Hq, H, ctx, n_q, K, more):
    _check_hybrid(dtype, D, P, Hq, H, ctx, ctx, n_q, K, seed=n_q, more=more)


@pytest.mark.parametrize("dtype", [F8, BF16])
@pytest.mark.parametrize("D,ctx", [(128, [1, 2, 64, 65, 255, 256, 257, 1030]), (64, [63, 500, 3, 129])])
def test_hybrid_single_token(dtype, D, ctx):
    _check_hybrid(dtype, D, 64, 8, 2, ctx, [c - 1 for c in ctx], 1, 0, seed=ctx[0])


@pytest.mark.parametrize("dtype", [F8, BF16])
@pytest.mark.parametrize("more", [0, 3000])
@pytest.mark.parametrize("D,P", [(128, 32), (64, 128)])
def test_hybrid_whole_input(dtype, D, P, more):
    # every position, and padding rows behind the shorter sequence
    _check_hybrid(dtype, D, P, 4, 2, [70, 23], [0, 0], 79, 3, seed=3, more=more)
    _check_hybrid(dtype, D, P, 4, 2, [330, 140], [0, 0], 345, 6, seed=4, more=more)


@pytest.mark.parametrize("dtype", [F8, BF16])
@pytest.mark.parametrize("n_q,Hq,more", [(8, 4, 0), (8, 24, 3000), (60, 8, 3000)])
def test_hybrid_queries_outside(dtype, n_q, Hq, more):
    # before position 0, across its border, past the end, a negative context, nothing at all; few rows a
    # group, 96 and 240
    _check_hybrid(dtype, 128, 16, Hq, 2, [40, 40, 40, -5, 12], [-9, -3, 45, 0, 1000], n_q, 2, seed=4, more=more)


@pytest.mark.parametrize("dtype", [F8, BF16])
@pytest.mark.parametrize("D", [64, 128])
def test_hybrid_padding_beside_long_rows(dtype, D):
    # padding rows in workgroups whose other rows see whole turns of keys, cut and uncut
    for more in (0, 3000):
        _check_hybrid(dtype, D, 32, 2, 2, [300, 150], [270, 120], 80, 4, seed=12, more=more)
        _check_hybrid(dtype, D, 32, 1, 1, [900], [880], 90, 4, seed=13, more=more)
        _check_hybrid(dtype, D, 32, 2, 1, [900, 333], [880, 200], 150, 4, seed=14, more=more)


def test_hybrid_room_cuts_the_input():
    _check_hybrid(F8, 64, 16, 4, 2, [60, 64, 90], [58, 60, 55], 12, 5, T=4, seed=5)


@pytest.mark.parametrize("dtype", [F8, BF16])
def test_hybrid_long_in_pieces(dtype):
    # cut over the keys, lengths that end inside a piece, one far shorter sequence
    _check_hybrid(dtype, 128, 64, 8, 2, [3001, 40, 2047], [3001, 40, 2047], 9, 3, seed=6)


def test_hybrid_of_the_longest_sequence():
    """2^31 - 65664 positions in pages that repeat: no piece of them is left out.  With keys of zeros every weight is
    one, and the values are 0 in the first three fifths, then 1 and 2: all sums are whole numbers (up to 2^24 in a wave,
    multiples of 64 above), so that only the quotient and the result's rounding are off."""
    P, D = 128, 64
    T = ((1 << 31) - 1 - 65536) // P
    v = torch.zeros(2, 1, D, P)
    v[1] = torch.arange(D)[:, None] % 2 + 1.0
    cache = cs.PagedCache(torch.zeros(2, 1, P, D, dtype=BF16, device=DEV), v.to(BF16).to(DEV))
    table = (torch.arange(T) >= T * 3 // 5).int()[None].to(DEV)
    ctx = torch.tensor([T * P], dtype=torch.int32, device=DEV)
    q = torch.ones(1, 1, 2, D, dtype=BF16, device=DEV)
    got = cs.hybrid_attention_paged(q, cache, table, ctx, ctx - 1, 0, 0.125).double().cpu()
    want = (T - T * 3 // 5) / T * (torch.arange(D) % 2 + 1.0).double()
    assert ((got - want).abs() <= (2.0 ** -8 + 2.0 ** -20) * want).all()


@pytest.mark.parametrize("dtype", [F8, BF16])
@pytest.mark.parametrize("n_q,Hq,more", [(3, 4, 0), (60, 8, 3000)])
def test_hybrid_far_positions_of_queries(dtype, n_q, Hq, more):
    # the lowest and the highest position and length that 32 bits name
    low, high = -(1 << 31), (1 << 31) - 1
    _check_hybrid(dtype, 128, 32, Hq, 2, [70, 70, low, 70], [low, high, high - n_q, low + 1], n_q, 2, seed=5, more=more)
    _check_hybrid(dtype, 128, 32, Hq, 2, [high, high], [high, 90], n_q, 2, T=4, seed=6)


@pytest.mark.parametrize("dtype", [F8, BF16])
@pytest.mark.parametrize("B,n_q,Hq", [(17, 1, 8), (32, 13, 32), (32, 17, 32), (17, 25, 32)])
def test_hybrid_more_pages_than_are_looked_up_at_once(dtype, B, n_q, Hq):
    # groups enough that nothing is cut, more than 252 pages each: few rows, 52, 68 and 100 of a group
    ctx = [4100 - 31 * (b % 5) for b in range(B)]
    _check_hybrid(dtype, 64, 16, Hq, 8, ctx, ctx, n_q, 3, seed=B, only=[0, B - 1])


@pytest.mark.parametrize("dtype", [F8, BF16])
@pytest.mark.parametrize("n_q,Hq", [(3, 2), (40, 8), (140, 2)])
@pytest.mark.parametrize("more", [0, 3000])
def test_hybrid_pieces_of_many_rows(dtype, n_q, Hq, more):
    # cut over the keys with few rows, 160 of a group, and context queries that see some pieces only
    _check_hybrid(dtype, 128, 32, Hq, 2, [1900, 700], [1850, 640], n_q, 7, seed=n_q, more=more)


@pytest.mark.parametrize("dtype", [F8, BF16])
@pytest.mark.parametrize("D,P,n_q,K", [(128, 64, 13, 5), (128, 16, 17, 7), (64, 32, 24, 2), (128, 128, 22, 0),
                                       (128, 64, 33, 15), (64, 16, 41, 19), (128, 32, 48, 20), (128, 128, 68, 30)])
def test_hybrid_of_many_groups(dtype, D, P, n_q, K):
    # 256 groups of 52 to 272 rows: waves that share their keys, padding and context queries among the rows
    B = 32
    ctx = [30 + 67 * (b % 4) for b in range(B)]
    start = [c - 3 * (b % 3) for b, c in enumerate(ctx)]
    _check_hybrid(dtype, D, P, 32, 8, ctx, start, n_q, K, seed=n_q, only=[0, 1, 2, 7], more=40)


@pytest.mark.parametrize("dtype", [F8, BF16])
@pytest.mark.parametrize("scale", [-0.1, 0.0, 0.9])
@pytest.mark.parametrize("n_q", [5, 70])
def test_hybrid_scales(dtype, scale, n_q):
    _check_hybrid(dtype, 64, 32, 4, 2, [90, 33], [50, 13], n_q, 1, scale=scale, seed=7, more=3000)


@pytest.mark.parametrize("dtype", [F8, BF16])
def test_hybrid_entries_that_name_no_page(dtype):
    def spoil(table):
        table[0, 1], table[1, 0], table[2, :] = -1, 2 ** 30, -7
    for n_q, Hq, more in ((13, 4, 0), (13, 12, 3000), (70, 6, 3000)):
        _check_hybrid(dtype, 128, 16, Hq, 2, [60, 10, 30, 50], [60, 0, 30, 50], n_q, 5, seed=8, spoil=spoil, more=more)


def test_scales_count_by_their_power_of_two():
    table, n_pages = ref.make_table(2, 3, 4)
    cache = _filled(table, n_pages, 2, 64, 32, F8, [90, 40], 4)
    q = torch.randn(2, 5, 4, 64, generator=_gen(5)).to(BF16).to(DEV)
    ctx = torch.tensor([85, 35], dtype=torch.int32, device=DEV)
    want = cs.hybrid_attention_paged(q, cache, table.to(DEV), ctx, ctx, 1, 0.125)
    cache.k_scale.mul_(1.75)
    cache.v_scale.mul_(1.25)
    assert _same(cs.hybrid_attention_paged(q, cache, table.to(DEV), ctx, ctx, 1, 0.125), want)


@pytest.mark.parametrize("B,H,Hq,more", [(1, 2, 4, 0), (32, 8, 416, 40), (1, 1, 256, 3000)])
def test_the_largest_scale_is_read_as_it_was_written(B, H, Hq, more):
    """Values that need the scale 2^120: those up to 240 times it are finite in bf16 and come back; one query per
    head that sees one position, in every kernel, with others behind it that it does not see."""
    D, P, n = 64, 16, 3
    table, n_pages = ref.make_table(B, 1, 3)
    cache = cs.PagedCache.empty(n_pages, H, D, P, F8, DEV)
    v = torch.tensor([1.796875, 1.875, -1.796875, -1.9296875, 1.75, -1.0, 2.0 ** -8, 0.0]).double() * 2.0 ** 127
    v = v.to(BF16).repeat(D // 8).expand(B, n, H, D).contiguous()
    k = torch.zeros(B, n, H, D, dtype=BF16)
    i32 = lambda x: torch.tensor([x] * B, dtype=torch.int32, device=DEV)  # noqa: E731
    cs.cache_append(cache, table.to(DEV), i32(0), k.to(DEV), v.to(DEV))
    assert (cache.v_scale[table[:, 0].long().to(DEV)] == 2.0 ** 120).all()
    _bits(cache.v)[:, :, :, 2] = 126                        # 448: what nobody sees, were it read
    q = torch.zeros(B, 1, Hq, D, dtype=BF16, device=DEV)
    got = cs.hybrid_attention_paged(q, cache, _longer(table, more).to(DEV), i32(1), i32(0), 0, 0.125).cpu().double()
    want = v[:, :1, :1].double().expand_as(got)
    # half a step of e4m3 (subnormals: 2^-10 of the scale); what it gives is exact in bf16
    assert ((got - want).abs() <= torch.maximum(2.0 ** -4 * want.abs(), torch.tensor(2.0 ** 110).double())).all()
    # two of the three positions seen, by a tree's node, beside another that sees the third
    parent = torch.tensor([[-1, 0, 0]] * B, dtype=torch.int32, device=DEV)
    q = torch.zeros(B, n, Hq, D, dtype=BF16, device=DEV)
    got = cs.tree_attention(q, cache, _longer(table, more).to(DEV), i32(0), parent, 0.125)[:, :1].cpu().double()
    assert ((got - want).abs() <= torch.maximum(2.0 ** -4 * want.abs(), torch.tensor(2.0 ** 110).double())).all()


def _check_tree(dtype, D, P, Hq, H, ctx, parent, T=None, seed=0, more=0, only=None):
    B, N = len(ctx), len(parent[0])
    T = T or (max(max(c, 0) for c in ctx) + N + P - 1) // P
    table, n_pages = ref.make_table(B, T, seed)
    room = (T + more) * P
    lengths = [min(max(c, 0) + N, room) for c in ctx]
    cache = _filled(table, n_pages, H, D, P, dtype, lengths, seed)
    table = _longer(table, more)
    q = torch.randn(B, N, Hq, D, generator=_gen(seed + 1)).to(BF16)
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device=DEV)  # noqa: E731
    got = cs.tree_attention(q.to(DEV), cache, table.to(DEV), i32(ctx), i32(parent), D ** -0.5)
    torch.cuda.synchronize()
    host = _host(cache)
    for b in only or range(B):
        lc = max(ctx[b], 0)
        mask = torch.zeros(N, lengths[b], dtype=torch.bool)
        mask[:, :min(lc, room)] = True
        inside = max(lengths[b] - lc, 0)
        mask[:, lc:] = ref.ancestors(parent[b])[:, :inside]
        mask[inside:] = False
        out, size = ref.attention(q[b], host.of("k", table[b], lengths[b]), host.of("v", table[b], lengths[b]), mask,
                                  D ** -0.5)
        _check_rows(got[b], out, size)


def _random_tree(N, seed, near=None):
    g = _gen(seed)
    return [-1] + [int(torch.randint(max(0, n - (near or n)), n, (1,), generator=g)) for n in range(1, N)]


@pytest.mark.parametrize("dtype", [F8, BF16])
@pytest.mark.parametrize("D,P,Hq,H,ctx,N", [(128, 64, 8, 2, [50, 0, 333], 33), (64, 16, 3, 3, [7, 16], 60),
                                            (128, 128, 4, 1, [700], 256), (64, 32, 8, 2, [5], 1)])
@pytest.mark.parametrize("more", [0, 3000])
def test_tree(dtype, D, P, Hq, H, ctx, N, more):
    _check_tree(dtype, D, P, Hq, H, ctx, [_random_tree(N, b, near=6) for b in range(len(ctx))], seed=N, more=more)


@pytest.mark.parametrize("dtype", [F8, BF16])
@pytest.mark.parametrize("D,N", [(128, 13), (64, 24), (128, 60), (128, 33), (64, 68)])
def test_tree_of_many_groups(dtype, D, N):
    # 256 groups of 52, 96, 240, 132 and 272 rows
    ctx = [25 + 41 * (b % 5) for b in range(32)]
    _check_tree(dtype, D, 32, 32, 8, ctx, [_random_tree(N, b, near=5) for b in range(32)], seed=N, more=40, only=[1, 4, 31])


@pytest.mark.parametrize("N", [2, 65, 256])
def test_tree_shapes(N):
    # a path, a star, and parents that break the rule (the node itself, later ones, none)
    bad = [n - 1 if n % 5 else (n, n + 3, -4, 10 ** 6)[n % 4] for n in range(N)]
    for more in (0, 3000):
        _check_tree(F8, 64, 32, 4, 2, [20, 61, 90], [list(range(-1, N - 1)), [-1] + [0] * (N - 1), bad], seed=N, more=more)


@pytest.mark.parametrize("dtype", [F8, BF16])
def test_tree_room_cuts_the_nodes(dtype):
    _check_tree(dtype, 128, 16, 4, 2, [40, 48, 70], [_random_tree(20, b) for b in range(3)], T=3, seed=9)


# ---------------------------------------------------------------------------------- keep

# What a query does not see is not to reach it, whatever it holds: bit by bit the result with good values there.

def _spoil(cache, table, b, positions, how):
    """Bad keys and values at positions of sequence b, and for "scales" a bad scale of their pages as well
    (whose every position must be among them, or past the sequence)."""
    nan = {"nan": math.nan, "inf": math.inf, "scales": 1.0}[how]
    for p in positions:
        pid, place = int(table[b, p // cache.page]), p % cache.page
        for x, at in ((cache.k, (pid, slice(None), place)), (cache.v, (pid, slice(None), slice(None), place))):
            good = x[at].float()
            good[..., 3::7] = nan
            x[at] = good.to(x.dtype)
        if how == "scales":
            cache.k_scale[pid], cache.v_scale[pid] = math.inf, math.inf


def _check_unseen(attend, cache, table, masks, bad, how):
    """masks[b] [n, length]: what the queries see; bad[b]: positions to spoil."""
    want = attend()
    for b, positions in enumerate(bad):
        _spoil(cache, table, b, positions, how)
    got = attend()
    torch.cuda.synchronize()
    for b, positions in enumerate(bad):
        hit = masks[b][:, positions].any(1)
        assert 0 < int((~hit).sum()), "some query sees none of them"
        assert torch.equal(got[b][~hit].float(), want[b][~hit].float())


def _hows(dtype):
    return ("nan", "scales") if dtype == F8 else ("nan", "inf")


# few rows, spread out; 58 and 90 rows in many groups; up to 45 in some; over 200 in one group, and in some;
# 116 and 180 of many
_ROWS = [(1, 4, 2, 1, 0), (1, 8, 2, 3, 0), (32, 16, 8, 1, 40), (4, 8, 8, 1, 3000), (1, 8, 1, 1, 3000), (4, 16, 8, 5, 3000),
         (32, 32, 8, 1, 40)]


@pytest.mark.parametrize("dtype", [F8, BF16])
@pytest.mark.parametrize("D,P", [(128, 32), (64, 16), (128, 128)])
@pytest.mark.parametrize("B,Hq,H,times,more", _ROWS)
@pytest.mark.parametrize("how", [0, 1])
def test_tree_nodes_not_seen(dtype, D, P, B, Hq, H, times, more, how):
    # the nodes behind the first 20, at the start of a page, and some before them, hold nothing good
    N = 20 * times + 9
    ctx = [3 * P - 20 * times] * B if 3 * P > 20 * times else [7 * P - 20 * times] * B
    T = (max(ctx) + N + P - 1) // P
    table, n_pages = ref.make_table(B, T, 5)
    cache = _filled(table, n_pages, H, D, P, dtype, [c + N for c in ctx], 5)
    parent = [_random_tree(20 * times, b, near=4) + [0] * 9 for b in range(B)]
    q = torch.randn(B, N, Hq, D, generator=_gen(6)).to(BF16).to(DEV)
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device=DEV)  # noqa: E731
    args = (q, cache, _longer(table, more).to(DEV), i32(ctx), i32(parent), D ** -0.5)
    masks, bad = [], []
    for b in range(B):
        mask = torch.zeros(N, ctx[b] + N, dtype=torch.bool)
        mask[:, :ctx[b]] = True
        mask[:, ctx[b]:] = ref.ancestors(parent[b])
        masks.append(mask)
        bad.append(list(range(ctx[b] + 20 * times, ctx[b] + N)) + ([ctx[b] + 9, ctx[b] + 13] if how == 0 else []))
    _check_unseen(lambda: cs.tree_attention(*args), cache, table, masks, bad, _hows(dtype)[how])


@pytest.mark.parametrize("dtype", [F8, BF16])
@pytest.mark.parametrize("D,P", [(128, 32), (64, 16), (128, 128)])
@pytest.mark.parametrize("B,Hq,H,times,more", _ROWS)
@pytest.mark.parametrize("how", [0, 1])
def test_hybrid_positions_not_seen(dtype, D, P, B, Hq, H, times, more, how):
    # context queries, padding behind them, and positions after the first of them that hold nothing good
    n_q, K = 20 * times + 25, 3
    ctx = [2 * P + 20 * times] * B
    T = (max(ctx) + 2 * K + 3 + P - 1) // P
    table, n_pages = ref.make_table(B, T, 7)
    lengths = [c + 2 * K + 3 for c in ctx]
    cache = _filled(table, n_pages, H, D, P, dtype, lengths, 7)
    start = [2 * P - 3] * B
    q = torch.randn(B, n_q, Hq, D, generator=_gen(8)).to(BF16).to(DEV)
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device=DEV)  # noqa: E731
    args = (q, cache, _longer(table, more).to(DEV), i32(ctx), i32(start), K, D ** -0.5)
    sees = torch.tensor(ref.hybrid_sees(ctx[0], start[0], n_q, K, T * P))
    masks = [torch.arange(lengths[0]) < sees[:, None]] * B
    first = [2 * P + (0 if how else 7 + b % 5) for b in range(B)]
    bad = [list(range(f, lengths[b])) if how else [f, f + 5] for b, f in enumerate(first)]
    _check_unseen(lambda: cs.hybrid_attention_paged(*args), cache, table, masks, bad, _hows(dtype)[how])


@pytest.mark.parametrize("dtype", [F8, BF16])
@pytest.mark.parametrize("more", [0, 3000])
def test_hybrid_not_seen_where_pages_are_looked_up_anew(dtype, more):
    # positions on both sides of the 252nd page, which waves share (52 rows a group) or not
    for B in (1, 32):
        ctx, K, n_q, P = [252 * 16 + 9] * B, 2, 13, 16
        T = (ctx[0] + 2 * K + 3 + P - 1) // P
        table, n_pages = ref.make_table(B, T, 9)
        lengths = [c + 2 * K + 3 for c in ctx]
        cache = _filled(table, n_pages, 8, 64, P, dtype, lengths, 9)
        q = torch.randn(B, n_q, 32, 64, generator=_gen(10)).to(BF16).to(DEV)
        start = [252 * 16 - 6] * B
        i32 = lambda x: torch.tensor(x, dtype=torch.int32, device=DEV)  # noqa: E731
        args = (q, cache, _longer(table, more).to(DEV), i32(ctx), i32(start), K, 0.125)
        sees = torch.tensor(ref.hybrid_sees(ctx[0], start[0], n_q, K, T * P))
        masks = [torch.arange(lengths[0]) < sees[:, None]] * B
        bad = [[252 * 16 - 4 + b % 3, 252 * 16 + 2 + b % 2] for b in range(B)]
        _check_unseen(lambda: cs.hybrid_attention_paged(*args), cache, table, masks, bad, "nan")


@pytest.mark.parametrize("dtype", [F8, BF16])
@pytest.mark.parametrize("Hq,n_q,more", [(8, 9, 0), (8, 9, 3000), (16, 60, 3000)])
def test_padding_beside_bad_values_gets_zeros(dtype, Hq, n_q, more):
    table, n_pages = ref.make_table(1, 8, 3)
    cache = _filled(table, n_pages, 2, 64, 64, dtype, [409], 3)
    _spoil(cache, table, 0, [5, 70, 200, 405], "nan")
    q = torch.randn(1, n_q, Hq, 64, generator=_gen(4)).to(BF16).to(DEV)
    at = torch.tensor([400], dtype=torch.int32, device=DEV)
    got = cs.hybrid_attention_paged(q, cache, _longer(table, more).to(DEV), at, at + 5, 3, 0.125)
    assert not got[0, 4:].float().ne(0).any()


def _check_seen(attend, cache, table, masks, bad, side, what):
    """A bad key or value shows in the results of the queries that see it, and in no other's.  masks as for
    _check_unseen; bad[b]: positions that get `what` in one component."""
    want = attend()
    for b, positions in enumerate(bad):
        for p in positions:
            pid, place = int(table[b, p // cache.page]), p % cache.page
            x, at = (cache.k, (pid, slice(None), place, 5)) if side == "k" else (cache.v, (pid, slice(None), 5, place))
            x[at] = torch.full((cache.heads,), what).to(x.dtype).to(DEV)
    got = attend()
    torch.cuda.synchronize()
    for b, positions in enumerate(bad):
        hit = masks[b][:, positions].any(1)
        assert 0 < int(hit.sum()) < hit.numel()
        assert torch.equal(got[b][~hit].float(), want[b][~hit].float())
        assert not torch.isfinite(got[b][hit][..., 5].float()).any()


_SEEN = [("v", math.nan), ("v", math.inf), ("k", math.nan), ("k", math.inf)]


def _positive_there(q):
    """Queries whose product with an infinity of _check_seen is plus infinity."""
    q[..., 5] = q[..., 5].abs() + 0.1
    return q.to(BF16).to(DEV)


@pytest.mark.parametrize("dtype", [F8, BF16])
@pytest.mark.parametrize("D,P", [(128, 32), (64, 16), (128, 128)])
@pytest.mark.parametrize("B,Hq,H,times,more", _ROWS)
@pytest.mark.parametrize("side,what", _SEEN)
def test_tree_bad_nodes_show(dtype, D, P, B, Hq, H, times, more, side, what):
    # two nodes, in different pages where trees are large
    N = 20 * times
    ctx = [3 * P + 11] * B
    T = (max(ctx) + N + P - 1) // P
    table, n_pages = ref.make_table(B, T, 5)
    cache = _filled(table, n_pages, H, D, P, dtype, [c + N for c in ctx], 5)
    parent = [_random_tree(N, b, near=4) for b in range(B)]
    q = _positive_there(torch.randn(B, N, Hq, D, generator=_gen(6)))
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device=DEV)  # noqa: E731
    args = (q, cache, _longer(table, more).to(DEV), i32(ctx), i32(parent), D ** -0.5)
    masks, bad = [], []
    for b in range(B):
        mask = torch.ones(N, ctx[b] + N, dtype=torch.bool)
        mask[:, ctx[b]:] = ref.ancestors(parent[b])
        masks.append(mask)
        bad.append([ctx[b] + 3 + b % 3, ctx[b] + N - 1])
    _check_seen(lambda: cs.tree_attention(*args), cache, table, masks, bad, side, what)


@pytest.mark.parametrize("dtype", [F8, BF16])
@pytest.mark.parametrize("D,P", [(128, 32), (64, 16), (128, 128)])
@pytest.mark.parametrize("B,Hq,H,times,more", _ROWS)
@pytest.mark.parametrize("side,what", _SEEN)
def test_hybrid_bad_positions_show(dtype, D, P, B, Hq, H, times, more, side, what):
    # context queries on both sides of a bad position, and padding
    n_q, K = 20 * times + 25, 3
    ctx = [2 * P + 20 * times] * B
    lengths = [c + 2 * K + 3 for c in ctx]
    table, n_pages = ref.make_table(B, (lengths[0] + P - 1) // P, 7)
    cache = _filled(table, n_pages, H, D, P, dtype, lengths, 7)
    start = [2 * P - 3] * B
    q = _positive_there(torch.randn(B, n_q, Hq, D, generator=_gen(8)))
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device=DEV)  # noqa: E731
    args = (q, cache, _longer(table, more).to(DEV), i32(ctx), i32(start), K, D ** -0.5)
    sees = torch.tensor(ref.hybrid_sees(ctx[0], start[0], n_q, K, lengths[0]))
    masks = [torch.arange(lengths[0]) < sees[:, None]] * B
    bad = [[2 * P + 2 + b % 7] for b in range(B)]
    _check_seen(lambda: cs.hybrid_attention_paged(*args), cache, table, masks, bad, side, what)


@pytest.mark.parametrize("dtype", [F8, BF16])
@pytest.mark.parametrize("more", [0, 3000])
def test_bad_values_show_where_pages_are_looked_up_anew(dtype, more):
    # in the last turn before the 253rd page and the first one behind it, which waves share (52 rows a group) or
    # not; many rows, cut over the keys and not
    for B, n_q, Hq in ((1, 13, 32), (32, 13, 32), (4, 70, 32), (8, 70, 32)):
        for at in (252 * 16 - 2, 252 * 16, 252 * 16 + 70):
            ctx, K, P = [252 * 16 + 90] * B, 2, 16
            lengths = [c + 2 * K + 3 for c in ctx]
            table, n_pages = ref.make_table(B, (lengths[0] + P - 1) // P, 9)
            cache = _filled(table, n_pages, 8, 64, P, dtype, lengths, 9)
            q = torch.randn(B, n_q, Hq, 64, generator=_gen(10)).to(BF16).to(DEV)
            start = [at - 6] * B
            i32 = lambda x: torch.tensor(x, dtype=torch.int32, device=DEV)  # noqa: E731
            args = (q, cache, _longer(table, more).to(DEV), i32(ctx), i32(start), K, 0.125)
            sees = torch.tensor(ref.hybrid_sees(ctx[0], start[0], n_q, K, lengths[0]))
            masks = [torch.arange(lengths[0]) < sees[:, None]] * B
            _check_seen(lambda: cs.hybrid_attention_paged(*args), cache, table, masks, [[at]] * B, "v", math.nan)


def _check_keep(dtype, D, P, H, ctx, path, N, T=None, seed=0):
    B = len(ctx)
    T = T or (max(max(c, 0) for c in ctx) + N + P - 1) // P
    table, n_pages = ref.make_table(B, T, seed)
    cache = _filled(table, n_pages, H, D, P, dtype, [min(max(c, 0) + N, T * P) for c in ctx], seed, junk=False)
    full = torch.tensor([p + [-1] * (N - len(p)) for p in path], dtype=torch.int32)
    host = _host(cache)
    ref.keep(host, table, ctx, full)
    cs.cache_keep(cache, table.to(DEV), torch.tensor(ctx, dtype=torch.int32, device=DEV), full.to(DEV))
    torch.cuda.synchronize()
    got = _host(cache)
    for side in ("k", "v"):
        if dtype == F8:
            assert torch.equal(got.scale[side], host.scale[side])
        assert _same(got.raw[side], host.raw[side])


@pytest.mark.parametrize("dtype", [F8, BF16])
@pytest.mark.parametrize("D,P,H,ctx,N,seed", [(128, 64, 2, [60, 0, 130], 60, 1), (64, 16, 3, [15, 16, 1], 33, 2),
                                              (128, 32, 1, [5, 31], 256, 3), (64, 128, 2, [127], 7, 4)])
def test_keep(dtype, D, P, H, ctx, N, seed):
    g = _gen(seed)
    paths = []
    for _ in ctx:
        s = int(torch.randint(1, N + 1, (1,), generator=g))
        paths.append([0] + sorted((torch.randperm(N - 1, generator=g)[:s - 1] + 1).tolist()))
    _check_keep(dtype, D, P, H, ctx, paths, N, seed=seed)


@pytest.mark.parametrize("dtype", [F8, BF16])
def test_keep_nothing_everything_and_beyond(dtype):
    # an empty path, one that stays, ends at an id too large, runs out of the room, a negative context
    _check_keep(dtype, 64, 16, 2, [20, 20, 20, 40, -3], [[], [0, 1, 2], [0, 2, 30, 4], [0, 3, 8, 9, 19], [0, 2, 5]], 20,
                T=3, seed=6)


# ------------------------------------------------------------------------------ together

def _round_trip(dtype, seed):
    """A token tree under the target's attention, its accepted path kept, and the arbitrator's
    region over the result, with the cache's contents checked against values that never were in one."""
    B, H, Hq, D, P, N, V = 3, 2, 8, 64, 16, 13, 211
    g = _gen(seed)
    T = 8
    table, n_pages = ref.make_table(B, T, seed)
    cache = cs.PagedCache.empty(n_pages, H, D, P, dtype, DEV)
    tab = table.to(DEV)
    inv = (10000.0 ** (-torch.arange(0, D, 2).double() / D)).float().to(DEV)
    draw = lambda n, h: torch.randn(B, n, h, D, generator=g).to(BF16).to(DEV)  # noqa: E731
    ctx = torch.tensor([30, 17, 5], dtype=torch.int32, device=DEV)
    zero = torch.zeros_like(ctx)
    pk, pv = draw(30, H), draw(30, H)
    cs.cache_append(cache, tab, zero, pk, pv, count=ctx, inv_freq=inv)
    parent = torch.tensor([_random_tree(N, b, near=4) for b in range(B)], dtype=torch.int32)
    depth = torch.zeros(B, N, dtype=torch.int32)
    for n in range(1, N):
        depth[:, n] = depth.gather(1, parent[:, n:n + 1].long())[:, 0] + 1
    tk, tv, tq = draw(N, H), draw(N, H), draw(N, Hq)
    positions = ctx[:, None] + depth.to(DEV)
    q = cs.cache_append(cache, tab, ctx, tk, tv, inv_freq=inv, positions=positions, q=tq)
    att = cs.tree_attention(q, cache, tab, ctx, parent.to(DEV), D ** -0.5)
    # logits of a made-up head over the attention's result
    w = torch.randn(Hq * D, V, generator=g).to(DEV) / 8
    logits = torch.nn.functional.pad((att.float().reshape(B, N, -1) @ w).to(BF16), (0, 5))[:, :, :V]
    tokens = logits.float().argmax(-1).int().gather(1, parent.clamp(min=0).long().to(DEV)).contiguous()
    tokens[:, 5::3] = (tokens[:, 5::3] + 1) % V
    from paper_2605_24793_amd.workloads import Head
    head = Head((torch.randn(64, 64, generator=g) / 8).to(BF16).to(DEV), None,
                (torch.randn(64, generator=g) / 8).to(BF16).to(DEV), 0.0)
    hidden = torch.randn(B, N, 64, generator=g).to(BF16).to(DEV)
    step = cs.verify_tree(logits, logits, parent.to(DEV), tokens, hidden, head, 2.0)
    cs.cache_keep(cache, tab, ctx, step["path"])
    new_ctx = ctx + step["accept_len"]
    K = 2
    rk, rv, rq = draw(2 * K + 3, H), draw(2 * K + 3, H), draw(2 * K + 3, Hq)
    rq2 = cs.cache_append(cache, tab, new_ctx, rk, rv, inv_freq=inv, q=rq)
    out = cs.hybrid_attention_paged(rq2, cache, tab, new_ctx, new_ctx, K, D ** -0.5)
    torch.cuda.synchronize()
    assert int(step["accept_len"].max()) > 1
    for b in range(B):
        c, s = int(ctx[b]), int(step["accept_len"][b])
        path = step["path"][b, :s].tolist()
        rows = [(pk[b, i], pv[b, i], i) for i in range(c)]
        rows += [(tk[b, n], tv[b, n], c + int(depth[b, n])) for n in path]
        rows += [(rk[b, i], rv[b, i], c + s + i) for i in range(2 * K + 3)]
        assert [r[2] for r in rows] == list(range(len(rows)))
        keys = torch.stack([ref.rotate(k.cpu(), p, inv.cpu(), False) for k, _, p in rows], 1)
        values = torch.stack([v.cpu().double() for _, v, _ in rows], 1)
        host = _host(cache)
        held = {"k": host.of("k", table[b], len(rows)), "v": host.of("v", table[b], len(rows))}
        half = 2.0 ** -4 if dtype == F8 else 2.0 ** -8
        for side, x in (("k", keys), ("v", values)):
            # one rounding to the stored type, and in 8 bits one more where a scale grew later;
            # among the subnormals 2^-10 of a scale, no more than 2^-6 here (|x| < 7)
            tol = half * x.abs() + (2 * 2.0 ** -16 if dtype == F8 else 2.0 ** -20)
            assert ((held[side] - x).abs() <= tol).all(), side
        m = torch.ones(2 * K + 3, len(rows), dtype=torch.bool)
        want, size = ref.attention(rq2[b].cpu(), held["k"], held["v"], m, D ** -0.5)
        _check_rows(out[b], want, size)


@pytest.mark.parametrize("dtype", [F8, BF16])
def test_a_round_on_the_cache(dtype):
    _round_trip(dtype, 11)


def test_calls_replay_from_a_hip_graph():
    """Append and attention captured once; every replay sees the inputs of its moment."""
    B, H, Hq, D, P, n = 2, 2, 8, 128, 64, 7
    table, n_pages = ref.make_table(B, 30, 3)
    cache = _filled(table, n_pages, H, D, P, F8, [1700, 70], 3, junk=False)
    tab = table.to(DEV)
    g = _gen(4)
    start = torch.tensor([1700, 70], dtype=torch.int32, device=DEV)
    k, v, q = (torch.randn(B, n, h, D, generator=g).to(BF16).to(DEV) for h in (H, H, Hq))
    inv = (10000.0 ** (-torch.arange(0, D, 2).double() / D)).float().to(DEV)
    app = cs.prepare_cache_append(cache, tab, start, k, v, inv_freq=inv, q=q)
    att = cs.prepare_hybrid_attention_paged(app.outputs["q"], cache, tab, start, start, 2, D ** -0.5)
    assert att.workspace is not None                        # cut: both kernels are in the graph
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        app.launch()
        att.launch()
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        app.launch()
        att.launch()
    for i in range(4):
        k.copy_(torch.randn(B, n, H, D, generator=g).to(BF16))
        q.copy_(torch.randn(B, n, Hq, D, generator=g).to(BF16))
        start.copy_(torch.tensor([1700 - i, 70 + i], dtype=torch.int32))
        graph.replay()
        torch.cuda.synchronize()
        first = att.outputs["out"].clone()
        app.launch()
        att.launch()
        torch.cuda.synchronize()
        assert _same(first, att.outputs["out"])


def test_two_calls_on_two_streams():
    B, H, Hq, D, P = 2, 2, 8, 128, 32
    calls, wants = [], []
    for i in range(2):
        table, n_pages = ref.make_table(B, 80, i)
        cache = _filled(table, n_pages, H, D, P, F8, [2500, 900], i, junk=False)
        q = torch.randn(B, 9, Hq, D, generator=_gen(i)).to(BF16).to(DEV)
        ctx = torch.tensor([2400, 800], dtype=torch.int32, device=DEV)
        calls.append(cs.prepare_hybrid_attention_paged(q, cache, table.to(DEV), ctx, ctx, 3, D ** -0.5))
        wants.append(cs.hybrid_attention_paged(q, cache, table.to(DEV), ctx, ctx, 3, D ** -0.5).clone())
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in calls]
    for _ in range(5):
        for c, s in zip(calls, streams):
            with torch.cuda.stream(s):
                c.launch()
    torch.cuda.synchronize()
    for c, w in zip(calls, wants):
        assert _same(c.outputs["out"], w)


def test_pages_past_four_gigabytes():
    """Pages whose memory lies past 2^32 bytes of the array."""
    H, D, P = 8, 128, 128
    n_pages = (1 << 32) // (H * D * P * 2) + 40
    cache = cs.PagedCache.empty(n_pages, H, D, P, BF16, DEV)
    table = torch.tensor([[n_pages - 1, n_pages - 17], [n_pages - 30, 0]], dtype=torch.int32)
    g = _gen(1)
    k, v = (torch.randn(2, 150, H, D, generator=g).to(BF16) for _ in range(2))
    zero = torch.zeros(2, dtype=torch.int32, device=DEV)
    cs.cache_append(cache, table.to(DEV), zero, k.to(DEV), v.to(DEV))
    q = torch.randn(2, 2, H, D, generator=g).to(BF16)
    ctx = torch.full((2,), 150, dtype=torch.int32, device=DEV)
    got = cs.hybrid_attention_paged(q.to(DEV), cache, table.to(DEV), ctx, ctx - 2, 0, D ** -0.5)
    torch.cuda.synchronize()
    for b in range(2):
        mask = torch.arange(150) < torch.tensor([149, 150])[:, None]
        out, size = ref.attention(q[b], k[b].double().transpose(0, 1), v[b].double().transpose(0, 1), mask, D ** -0.5)
        _check_rows(got[b], out, size)


def test_nothing_to_do():
    table, n_pages = ref.make_table(2, 2, 0)
    cache = _filled(table, n_pages, 2, 64, 16, BF16, [4, 4], 0, junk=False)
    before = _host(cache)
    tab, z = table.to(DEV), torch.zeros(2, dtype=torch.int32, device=DEV)
    empty = torch.empty(2, 0, 2, 64, dtype=BF16, device=DEV)
    cs.cache_append(cache, tab, z, empty, empty)
    assert cs.hybrid_attention_paged(torch.empty(2, 0, 4, 64, dtype=BF16, device=DEV), cache, tab, z, z, 1, 0.1).numel() == 0
    none = torch.empty(0, 3, 4, 64, dtype=BF16, device=DEV)
    assert cs.hybrid_attention_paged(none, cache, tab[:0], z[:0], z[:0], 1, 0.1).shape == (0, 3, 4, 64)
    cs.cache_keep(cache, tab[:0], z[:0], torch.empty(0, 3, dtype=torch.int32, device=DEV))
    torch.cuda.synchronize()
    after = _host(cache)
    assert torch.equal(before.raw["k"], after.raw["k"]) and torch.equal(before.raw["v"], after.raw["v"])
