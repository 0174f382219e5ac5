"""The pages under the caches on the GPU against lists that follow the rules
(tests/latent_reference.py)."""
import random

import pytest
import torch

import latent_reference as ref
import paper_2605_24793_amd as cs

pytestmark = pytest.mark.gpu
DEV = torch.device("cuda:0")
BF16, F8 = torch.bfloat16, torch.float8_e4m3fn


def _int(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


def _state(n_pages, B, T, page, seed, fill=0.6, holes=0.1, share=0.3):
    """Tables and counts that agree, with entries that name no page among them."""
    rng = random.Random(seed)
    free = list(range(n_pages))
    rng.shuffle(free)
    refs, table = [0] * n_pages, []
    for b in range(B):
        row = []
        for j in range(T):
            if rng.random() > fill or (not free and not any(refs)):
                row.append(rng.choice([-1, -1, n_pages, -5]) if rng.random() < 0.5 else -1)
            elif rng.random() < share and any(refs):
                row.append(rng.choice([p for p in range(n_pages) if refs[p]]))
                refs[row[-1]] += 1
            elif free and rng.random() > holes:
                row.append(free.pop())
                refs[row[-1]] += 1
            else:
                row.append(-1)
        table.append(row)
    return refs, table


def _same(pool, table, host, rows):
    assert pool.refs.tolist() == host.refs
    assert table.tolist() == rows


SIZES = [(1, 1, 1, 16), (7, 2, 3, 16), (100, 5, 8, 64), (3000, 40, 30, 32), (9000, 300, 17, 128), (5000, 3, 1000, 16)]


@pytest.mark.parametrize("n_pages,B,T,P", SIZES)
def test_fork(n_pages, B, T, P):
    refs, rows = _state(n_pages, B, T, P, n_pages)
    rng = random.Random(3)
    row = [rng.choice([-1, B, rng.randrange(B), rng.randrange(B)]) for _ in range(B + 4)]
    length = [rng.choice([-3, 0, 1, P, P + 1, T * P, T * P + 9, rng.randrange(T * P + 1)]) for _ in row]
    host, pool, table = ref.Pool(refs, P), cs.PagePool(_int(refs), P), _int(rows)
    out = cs.pages_fork(pool, table, _int(row), _int(length))
    want = host.fork(rows, row, length)
    _same(pool, out, host, want)
    assert table.tolist() == rows


@pytest.mark.parametrize("n_pages,B,T,P", SIZES)
@pytest.mark.parametrize("n", [1, 5, 40, 200])
def test_reserve(n_pages, B, T, P, n):
    refs, rows = _state(n_pages, B, T, P, n_pages + n)
    rng = random.Random(n)
    start = [rng.choice([-7, 0, rng.randrange(T * P), T * P - 1, T * P + 3, 2 ** 31 - 1]) for _ in range(B)]
    count = [rng.choice([0, -1, n, n, rng.randrange(n + 1), n + 100]) for _ in range(B)]
    host, pool, table = ref.Pool(refs, P), cs.PagePool(_int(refs), P), _int(rows)
    for given in (count, None):
        out = cs.pages_reserve(pool, table, _int(start), n, None if given is None else _int(given))
        copies, lacking = host.reserve(rows, start, [min(max(c, 0), n) for c in given] if given else [n] * B)
        assert int(out["lacking"]) == lacking
        assert out["copies"].tolist() == [list(c) for c in copies]
        _same(pool, table, host, rows)


def test_reserve_takes_the_last_page_and_not_one_more():
    pool, table = cs.PagePool.empty(5, 16), _int([[-1] * 4, [-1] * 4])
    assert int(cs.pages_reserve(pool, table, _int([0, 0]), 33)["lacking"]) == 1
    assert table.tolist() == [[-1] * 4] * 2 and pool.refs.tolist() == [0] * 5
    assert int(cs.pages_reserve(pool, table, _int([0, 0]), 33, _int([33, 32]))["lacking"]) == 0
    assert table.tolist() == [[0, 1, 2, -1], [3, 4, -1, -1]] and pool.refs.tolist() == [1] * 5
    # again: they have them
    assert int(cs.pages_reserve(pool, table, _int([0, 0]), 33, _int([33, 32]))["lacking"]) == 0
    assert table.tolist() == [[0, 1, 2, -1], [3, 4, -1, -1]]


def test_reserve_for_nobody():
    pool = cs.PagePool.empty(5, 16)
    out = cs.pages_reserve(pool, torch.empty(0, 3, dtype=torch.int32, device=DEV), torch.empty(0, dtype=torch.int32, device=DEV), 4)
    assert int(out["lacking"]) == 0 and pool.refs.tolist() == [0] * 5
    table = _int([[-1, -1]])
    out = cs.pages_reserve(pool, table, _int([3]), 0)
    assert int(out["lacking"]) == 0 and out["copies"].tolist() == [[-1, -1]] and table.tolist() == [[-1, -1]]


@pytest.mark.parametrize("n_pages,B,T,P", SIZES)
def test_release_and_compact(n_pages, B, T, P):
    refs, rows = _state(n_pages, B, T, P, n_pages)
    rng = random.Random(5)
    keep = [rng.choice([-3, 0, 1, P, P + 1, T * P, T * P + 9, rng.randrange(T * P + 1)]) for _ in range(B)]
    host, pool, table = ref.Pool(refs, P), cs.PagePool(_int(refs), P), _int(rows)
    cs.pages_release(pool, table, _int(keep))
    host.release(rows, keep)
    _same(pool, table, host, rows)
    for _ in range(2):                                       # the second time nothing moves
        out = cs.pages_compact(pool, table)
        moves = host.compact(rows)
        _same(pool, table, host, rows)
        assert int(out["n_moves"]) == len(moves)
        got = out["moves"].tolist()
        assert got[:len(moves)] == [list(m) for m in moves] and all(m == [-1, -1] for m in got[len(moves):])
    used = sum(n > 0 for n in host.refs)
    assert all(n > 0 for n in host.refs[:used])


def _caches(n_pages, P, g):
    def bits(t):
        raw = t.view(torch.uint8)
        raw.copy_(torch.randint(0, 256, raw.shape, generator=g, dtype=torch.uint8))
        return t
    out = []
    for dtype in (BF16, F8):
        p = cs.PagedCache.empty(n_pages, 3, 64, P, dtype)
        lat = cs.LatentCache.empty(n_pages, 256, P, dtype)
        out += [p, lat]
    for c in out:
        for t in c._planes():
            bits(t)
    return out


def _raw(caches):
    return [t.view(torch.uint8).reshape(t.shape[0], -1).clone() for c in caches for t in c._planes()]


@pytest.mark.parametrize("P", [16, 128])
@pytest.mark.parametrize("layers", [1, 25])
def test_copy(P, layers):
    n_pages = 40
    g = torch.Generator().manual_seed(P)
    caches = [c for _ in range(layers) for c in _caches(n_pages, P, g)]      # 25: more planes than a launch takes
    pool = cs.PagePool.empty(n_pages, P)
    pairs = [[3, 7], [-1, -1], [3, 39], [40, 2], [5, -2], [6, 6], [11, 0], [12, 1], [13, 14]]
    before = _raw(caches)
    cs.pages_copy(pool, caches, _int(pairs), _int([8]))
    for old, now in zip(before, _raw(caches)):
        want = old.clone()
        for a, b in pairs[:8]:
            if 0 <= a < n_pages and 0 <= b < n_pages:
                want[b] = old[a]
        assert torch.equal(now, want)
    for count in (0, -4):
        before = _raw(caches)
        cs.pages_copy(pool, caches, _int(pairs), _int([count]))
        assert all(torch.equal(a, b) for a, b in zip(before, _raw(caches)))


def test_branches_of_a_prompt():
    """A prompt's branches: they read the same, write pages of their own, and give them back; the pool is compacted, and
    every sequence still reads what it did."""
    g = torch.Generator().manual_seed(1)
    P, dc, Hq, n_pages, T = 16, 256, 4, 40, 6
    pool, layers = cs.PagePool.empty(n_pages, P), [cs.LatentCache.empty(n_pages, dc, P, d) for d in (BF16, F8)]
    table = torch.full((2, T), -1, dtype=torch.int32, device=DEV)
    lens = _int([37, 48])
    assert int(cs.pages_reserve(pool, table, _int([0, 0]), 48, lens, layers)["lacking"]) == 0
    x = torch.randn(2, 48, dc + 64, generator=g).to(BF16).to(DEV)
    for cache in layers:
        cs.latent_append(cache, table, _int([0, 0]), x[..., :dc], x[..., dc:], count=lens)
    q = (torch.randn(5, 1, Hq, dc + 64, generator=g) * 0.6).to(BF16).to(DEV)

    def reads(t, at, rows):
        return [cs.latent_attention(q[rows], cache, t, at, at - 1, 0, 0.07) for cache in layers]

    row = _int([0, 0, 1, 1, 0])
    at = lens[row.long()].contiguous()
    fork = cs.pages_fork(pool, table, row, at)
    for a, b in zip(reads(fork, at, slice(None)), reads(table, lens, slice(0, 2))):
        assert torch.equal(a[0], b[0])                       # the same query over the same pages
    alone = reads(table, lens, slice(0, 2))
    assert int(cs.pages_reserve(pool, fork, at, 3, caches=layers)["lacking"]) == 0
    y = torch.randn(5, 3, dc + 64, generator=g).to(BF16).to(DEV)
    for cache in layers:
        cs.latent_append(cache, fork, at, y[..., :dc], y[..., dc:])
    assert all(torch.equal(a, b) for a, b in zip(alone, reads(table, lens, slice(0, 2))))   # the prompts have not changed
    longer = (at + 3).contiguous()
    ahead = reads(fork, longer, slice(None))
    # each branch reads as a sequence that was appended whole
    whole = torch.cat((x[row.long()], torch.zeros(5, 3, dc + 64, dtype=BF16, device=DEV)), 1)
    for b in range(5):
        whole[b, int(at[b]):int(at[b]) + 3] = y[b]
    other, own = cs.PagePool.empty(n_pages, P), torch.full((5, T), -1, dtype=torch.int32, device=DEV)
    cs.pages_reserve(other, own, _int([0] * 5), 51, longer)
    for cache, got in zip(layers, ahead):
        fresh = cs.LatentCache.empty(n_pages, dc, P, cache.c.dtype)
        cs.latent_append(fresh, own, _int([0] * 5), whole[..., :dc], whole[..., dc:], count=longer)
        assert torch.equal(got, cs.latent_attention(q, fresh, own, longer, longer - 1, 0, 0.07))
    # two branches end, and the pool is compacted
    both = torch.cat((table, fork))
    keep = torch.cat((lens, longer))
    keep[2], keep[5] = 0, 0
    cs.pages_release(pool, both, keep)
    cs.pages_compact(pool, both, layers)
    refs = pool.refs.tolist()
    used = sum(r > 0 for r in refs)
    assert all(r > 0 for r in refs[:used]) and used < n_pages
    counted = [0] * n_pages
    for e in both.reshape(-1).tolist():
        if e >= 0:
            counted[e] += 1
    assert counted == refs
    kept = [1, 2, 4]
    now = [cs.latent_attention(q, cache, both[2:].contiguous(), longer, longer - 1, 0, 0.07) for cache in layers]
    assert all(torch.equal(a[b], c[b]) for a, c in zip(ahead, now) for b in kept)
    assert all(torch.equal(a, b) for a, b in zip(alone, reads(both[:2].contiguous(), lens, slice(0, 2))))


@pytest.mark.parametrize("dtype", [BF16, F8])
def test_all_holders_of_a_page_leave_it_at_once(dtype):
    """The page that they share is free then, and still holds what their copies take; the next reserve hands it out."""
    g = torch.Generator().manual_seed(4)
    P, n_pages, dc = 16, 8, 256
    pool, cache = cs.PagePool.empty(n_pages, P), cs.LatentCache.empty(n_pages, dc, P, dtype)
    prompt = torch.full((1, 3), -1, dtype=torch.int32, device=DEV)
    cs.pages_reserve(pool, prompt, _int([0]), 20)
    x = torch.randn(1, 20, dc + 64, generator=g).to(BF16).to(DEV)
    cs.latent_append(cache, prompt, _int([0]), x[..., :dc], x[..., dc:])
    fork = cs.pages_fork(pool, prompt, _int([0, 0, 0]), _int([20, 20, 20]))
    cs.pages_release(pool, prompt, _int([0]))
    assert pool.refs.tolist() == [3, 3] + [0] * 6
    before = [t[1].view(torch.uint8).clone() for t in cache._planes()]
    out = cs.pages_reserve(pool, fork, _int([20, 20, 20]), 4, caches=[cache])
    assert int(out["lacking"]) == 0 and out["copies"].tolist() == [[1, 2], [1, 3], [1, 4]]
    assert fork.tolist() == [[0, 2, -1], [0, 3, -1], [0, 4, -1]]
    assert pool.refs.tolist() == [3, 0, 1, 1, 1, 0, 0, 0]
    for t, old in zip(cache._planes(), before):
        assert all(torch.equal(t[p].view(torch.uint8), old) for p in (1, 2, 3, 4))
    other = torch.full((1, 3), -1, dtype=torch.int32, device=DEV)
    cs.pages_reserve(pool, other, _int([0]), 1)
    assert other.tolist() == [[1, -1, -1]]


def test_captured_turns_of_a_pool():
    """Fork, reserve with copies, release and compact in one graph, replayed."""
    P, n_pages, T = 16, 64, 6
    g = torch.Generator().manual_seed(2)
    refs, rows = _state(n_pages, 4, T, P, 9, holes=0.0, share=0.0)
    cache = cs.LatentCache.empty(n_pages, 256, P, BF16)
    cache.c.copy_(torch.randn(cache.c.shape, generator=g).to(BF16))
    cache.r.copy_(torch.randn(cache.r.shape, generator=g).to(BF16))
    first = (cache.c.clone(), cache.r.clone())
    pool, table = cs.PagePool(_int(refs), P), _int(rows)
    row, at, n = _int([0, 1, 1, 3]), _int([20, 33, 16, 90]), 9
    fork = cs.prepare_pages_fork(pool, table, row, at)
    reserve = cs.prepare_pages_reserve(pool, fork.outputs["table"], at, n, caches=[cache])
    release = cs.prepare_pages_release(pool, table, _int([0, 40, 40, 0]))
    both = torch.empty(8, T, dtype=torch.int32, device=DEV)
    compact = cs.prepare_pages_compact(pool, both, [cache])

    def turn():
        fork.launch()
        reserve.launch()
        release.launch()
        both[:4] = table
        both[4:] = fork.outputs["table"]
        compact.launch()

    def restore():
        pool.refs.copy_(_int(refs))
        table.copy_(_int(rows))
        cache.c.copy_(first[0])
        cache.r.copy_(first[1])

    turn()
    torch.cuda.synchronize()
    want = [t.clone() for t in (pool.refs, both, reserve.outputs["copies"], compact.outputs["moves"], cache.c, cache.r)]
    restore()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        turn()
    for _ in range(3):
        restore()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        now = (pool.refs, both, reserve.outputs["copies"], compact.outputs["moves"], cache.c, cache.r)
        assert all(torch.equal(a, b) for a, b in zip(want, now))


def test_the_binding_refuses():
    pool = cs.PagePool.empty(8, 16)
    table, one = _int([[0, 1]]), _int([0])
    cache = cs.LatentCache.empty(9, 256, 16)
    bad = [lambda: cs.pages_fork(pool, table.long(), one, one), lambda: cs.pages_fork(pool, table, one, _int([1, 2])),
           lambda: cs.pages_reserve(pool, table, _int([1, 2]), 3), lambda: cs.pages_reserve(pool, table, one, 3, caches=[cache]),
           lambda: cs.pages_reserve(pool, table, one, -1), lambda: cs.pages_release(pool, table[:, :1], _int([1, 1])),
           lambda: cs.pages_compact(pool, table, [cache]), lambda: cs.pages_copy(pool, [], _int([[1, 2, 3]])),
           lambda: cs.pages_copy(pool, [cs.LatentCache.empty(8, 256, 32)], _int([[1, 2]])), lambda: cs.PagePool(pool.refs.long(), 16),
           lambda: cs.pages_release(cs.PagePool(pool.refs, 20), table, one)]
    for call in bad:
        with pytest.raises((ValueError, TypeError, cs.CospecError)):
            call()
