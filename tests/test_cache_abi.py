"""The paged cache's entry points without a GPU: what they refuse before anything is enqueued."""
import ctypes
import math

import pytest
import torch

import paper_2605_24793_amd as cs
from paper_2605_24793_amd import binding

OK, INVALID, UNSUPPORTED, WORKSPACE = 0, -1, -2, -3
FAKE = 0x10000          # an aligned address; validation never dereferences device pointers
BF16, F8 = 1, 2


def _cache(dtype=F8, page=64, heads=8, d=128, n_pages=100, k=FAKE, v=FAKE, k_scale=FAKE, v_scale=FAKE, table=FAKE,
           max_pages=20):
    return binding._Cache(dtype, page, heads, d, n_pages, k, v, k_scale, v_scale, table, max_pages)


def _append(L, cache=None, start=FAKE, count=None, k=FAKE, ld_k=1024, v=FAKE, ld_v=1024, rope=None, positions=None, B=2,
            n=3, q=None, ld_q=0, Hq=0, q_out=None):
    return L.cospec_cache_append(ctypes.byref(cache or _cache()), start, count, k, ld_k, v, ld_v,
                                 None if rope is None else ctypes.byref(binding._Rope(*rope)), positions, B, n, q, ld_q,
                                 Hq, q_out, None)


def _keep(L, cache=None, ctx=FAKE, path=FAKE, B=2, N=9):
    return L.cospec_cache_keep(ctypes.byref(cache or _cache()), ctx, path, B, N, None)


def _hybrid(L, cache=None, q=FAKE, ctx=FAKE, qs=FAKE, B=2, n=17, Hq=32, K=7, scale=0.1, out=FAKE, ws=FAKE, wsb=1 << 40):
    return L.cospec_hybrid_attention_paged(q, ctypes.byref(cache or _cache()), ctx, qs, B, n, Hq, K, scale, out, ws, wsb,
                                           None)


def _tree(L, cache=None, q=FAKE, ctx=FAKE, parent=FAKE, B=2, N=60, Hq=32, scale=0.1, out=FAKE, ws=FAKE, wsb=1 << 40):
    return L.cospec_tree_attention(q, ctypes.byref(cache or _cache()), ctx, parent, B, N, Hq, scale, out, ws, wsb, None)


CACHES = [
    (dict(dtype=0), UNSUPPORTED), (dict(dtype=3), UNSUPPORTED), (dict(page=8), UNSUPPORTED), (dict(page=48), UNSUPPORTED),
    (dict(page=256), UNSUPPORTED), (dict(d=96), UNSUPPORTED), (dict(heads=0), INVALID), (dict(n_pages=-1), INVALID),
    (dict(n_pages=0), INVALID), (dict(max_pages=0), INVALID), (dict(max_pages=-3), INVALID),
    (dict(max_pages=(1 << 31) // 64 + 1), UNSUPPORTED), (dict(n_pages=1 << 31), UNSUPPORTED), (dict(k=None), INVALID),
    (dict(v=FAKE + 8), INVALID), (dict(k_scale=None), INVALID), (dict(v_scale=FAKE + 2), INVALID),
    (dict(table=None), INVALID), (dict(table=FAKE + 2), INVALID),
]


@pytest.mark.parametrize("kw,code", CACHES)
def test_every_call_checks_the_cache(kw, code):
    L = cs.lib()
    bad = _cache(**kw)
    for call in (_append, _keep, _hybrid, _tree):
        assert call(L, cache=bad) == code, call.__name__


def test_no_cache_at_all():
    L = cs.lib()
    assert L.cospec_cache_append(None, FAKE, None, FAKE, 1024, FAKE, 1024, None, None, 1, 1, None, 0, 0, None, None) == INVALID
    assert L.cospec_cache_keep(None, FAKE, FAKE, 1, 1, None) == INVALID
    assert L.cospec_hybrid_attention_paged(FAKE, None, FAKE, FAKE, 1, 1, 8, 0, 0.1, FAKE, None, 0, None) == INVALID
    assert L.cospec_tree_attention(FAKE, None, FAKE, FAKE, 1, 1, 8, 0.1, FAKE, None, 0, None) == INVALID
    assert L.cospec_paged_attention_workspace_size(None, 1, 1, 8) == 0


@pytest.mark.parametrize("kw,code", [
    (dict(B=-1), INVALID), (dict(n=-1), INVALID), (dict(start=None), INVALID), (dict(start=FAKE + 2), INVALID),
    (dict(count=FAKE + 1), INVALID), (dict(k=None), INVALID), (dict(k=FAKE + 8), INVALID), (dict(v=None), INVALID),
    (dict(ld_k=1016), INVALID), (dict(ld_v=1028), INVALID), (dict(positions=FAKE + 2), INVALID),
    (dict(rope=(130, 0, FAKE)), INVALID), (dict(rope=(-16, 0, FAKE)), INVALID), (dict(rope=(24, 0, FAKE)), UNSUPPORTED),
    (dict(rope=(64, 0, None)), INVALID), (dict(rope=(64, 1, FAKE + 2)), INVALID),
    (dict(q=FAKE, Hq=0, ld_q=4096, q_out=FAKE), INVALID), (dict(q=FAKE, Hq=32, ld_q=4088, q_out=FAKE), INVALID),
    (dict(q=FAKE, Hq=32, ld_q=4096, q_out=None), INVALID), (dict(q=FAKE + 4, Hq=32, ld_q=4096, q_out=FAKE), INVALID),
    (dict(B=1 << 20, n=1 << 20), UNSUPPORTED), (dict(B=1 << 28, n=1), UNSUPPORTED), (dict(B=0), OK), (dict(n=0), OK),
    (dict(B=0, k=None, v=None, start=None), OK),
])
def test_append_refuses(kw, code):
    assert _append(cs.lib(), **kw) == code


@pytest.mark.parametrize("kw,code", [
    (dict(B=-1), INVALID), (dict(N=0), INVALID), (dict(N=257), UNSUPPORTED), (dict(ctx=None), INVALID),
    (dict(path=FAKE + 2), INVALID), (dict(B=1 << 29), UNSUPPORTED), (dict(B=0, ctx=None, path=None), OK),
])
def test_keep_refuses(kw, code):
    assert _keep(cs.lib(), **kw) == code


@pytest.mark.parametrize("call,kw,code", [
    (_hybrid, dict(Hq=12), INVALID), (_hybrid, dict(Hq=0), INVALID), (_hybrid, dict(K=-1), INVALID),
    (_hybrid, dict(scale=math.nan), INVALID), (_hybrid, dict(scale=math.inf), INVALID), (_hybrid, dict(q=None), INVALID),
    (_hybrid, dict(q=FAKE + 8), INVALID), (_hybrid, dict(out=FAKE + 2), INVALID), (_hybrid, dict(ctx=None), INVALID),
    (_hybrid, dict(qs=FAKE + 2), INVALID), (_hybrid, dict(B=-2), INVALID), (_hybrid, dict(n=-2), INVALID),
    (_hybrid, dict(B=1 << 20, n=1 << 20), UNSUPPORTED), (_hybrid, dict(n=0, q=None), OK), (_hybrid, dict(B=0, q=None), OK),
    (_hybrid, dict(ws=None), WORKSPACE), (_hybrid, dict(ws=FAKE + 16), WORKSPACE), (_hybrid, dict(wsb=1000), WORKSPACE),
    (_tree, dict(Hq=12), INVALID), (_tree, dict(N=0), INVALID), (_tree, dict(N=257), UNSUPPORTED),
    (_tree, dict(parent=None), INVALID), (_tree, dict(parent=FAKE + 2), INVALID), (_tree, dict(scale=-math.inf), INVALID),
    (_tree, dict(q=FAKE + 4), INVALID), (_tree, dict(B=0, q=None, parent=None), OK),
    (_tree, dict(N=1, ws=None), WORKSPACE),
])
def test_attention_refuses(call, kw, code):
    assert call(cs.lib(), **kw) == code


@pytest.mark.parametrize("call,kw", [
    (_append, dict(B=1 << 21, n=1)), (_append, dict(B=1 << 18, n=129, cache=_cache(page=16))),
    (_append, dict(cache=_cache(heads=1), B=1 << 24, n=8, q=FAKE, Hq=1, ld_q=128, q_out=FAKE)),
    (_keep, dict(B=1 << 20)), (_hybrid, dict(B=1 << 21, n=1)), (_tree, dict(B=1 << 21, N=5)),
])
def test_more_workgroups_than_a_launch_holds(call, kw):
    # 2^24 workgroups of 256 threads and more: refused, not left to the launch
    assert call(cs.lib(), **kw) == UNSUPPORTED


def test_workspace_size():
    L = cs.lib()

    def size(B, n, Hq, **kw):
        return L.cospec_paged_attention_workspace_size(ctypes.byref(_cache(**kw)), B, n, Hq)
    rows = 2 * 17 * 32
    need = size(2, 17, 32)
    assert need % 256 == 0 and need >= 2 * rows * (128 * 4 + 8)     # two pieces at least
    assert size(64, 17, 32) == 0                                      # groups enough without cutting
    assert size(2, 17, 32, max_pages=1) == 0                          # too few keys to cut
    # a size, and no memory, is all it looks at
    assert size(2, 17, 32, k=None, table=None) == need
    for bad in ((-1, 17, 32), (2, -1, 32), (2, 17, 12)):
        assert size(*bad) == 0
    assert size(0, 17, 32) == 0 and size(2, 0, 32) == 0
    assert _hybrid(L, wsb=need - 1) == WORKSPACE


def test_other_entries_refuse_the_cache_type():
    # e4m3 is a type of cache pages only
    hd = binding._Head(512, 128, F8, FAKE, None, FAKE, 0.0)
    L = cs.lib()
    assert L.cospec_arbitrate_workspace_size(10, ctypes.byref(hd)) == 0
    assert L.cospec_verify_block_sps(FAKE, FAKE, F8, 151936, FAKE, FAKE, 4, 7, 151936, FAKE, FAKE, None, None, FAKE,
                                     1 << 40, None) == INVALID


class _Fake(torch.Tensor):
    """A CPU tensor that says it is on the GPU, so that the binding's own checks can be met here."""
    is_cuda = True


def _pages(n=4, heads=2, page=16, d=64, dtype=torch.bfloat16):
    k, v = torch.zeros(n, heads, page, d, dtype=dtype), torch.zeros(n, heads, d, page, dtype=dtype)
    return k.as_subclass(_Fake), v.as_subclass(_Fake)


def test_paged_cache_checks_its_tensors():
    k, v = _pages()
    c = cs.PagedCache(k, v)
    assert (c.n_pages, c.heads, c.page, c.d) == (4, 2, 16, 64)
    k8, v8 = _pages(dtype=torch.float8_e4m3fn)
    s = torch.ones(4, 2).as_subclass(_Fake)
    assert cs.PagedCache(k8, v8, s, s).dtype == F8
    with pytest.raises(ValueError):
        cs.PagedCache(k8, v8)                                       # no scales
    with pytest.raises(ValueError):
        cs.PagedCache(k8, v8, s, s.double())
    with pytest.raises(ValueError):
        cs.PagedCache(k, v, s, s)                                   # scales that mean nothing
    with pytest.raises(ValueError):
        cs.PagedCache(k, k)                                         # values not transposed
    with pytest.raises(ValueError):
        cs.PagedCache(k, v8)
    with pytest.raises(ValueError):
        cs.PagedCache(k[:, :, :, ::2], v)
    with pytest.raises(TypeError):
        cs.PagedCache(k.half(), v.half())
    with pytest.raises(ValueError):
        cs.PagedCache(torch.zeros(4, 2, 16, 64, dtype=torch.bfloat16), v)     # not on the GPU


def test_binding_checks_shapes_before_the_library():
    cache = cs.PagedCache(*_pages())
    fake = lambda *s, dtype=torch.bfloat16: torch.zeros(*s, dtype=dtype).as_subclass(_Fake)  # noqa: E731
    table, z = fake(3, 5, dtype=torch.int32), fake(3, dtype=torch.int32)
    k, q = fake(3, 4, 2, 64), fake(3, 4, 8, 64)
    bad = [
        lambda: cs.cache_append(cache, table[:2], z, k, k),                          # a table of another batch
        lambda: cs.cache_append(cache, table.long(), z, k, k),
        lambda: cs.cache_append(cache, table, z.long(), k, k),
        lambda: cs.cache_append(cache, table, z, k[:, :, :1], k),                    # another head count
        lambda: cs.cache_append(cache, table, z, k.float(), k),
        lambda: cs.cache_append(cache, table, z, k, k[:, :3]),
        lambda: cs.cache_append(cache, table, z, k.transpose(1, 2).contiguous().transpose(1, 2), k),
        lambda: cs.cache_append(cache, table, z, k, k, count=z[:2]),
        lambda: cs.cache_append(cache, table, fake(6, dtype=torch.int32)[::2], k, k),  # every launch reads it anew
        lambda: cs.cache_append(cache, table, z, k, k, positions=z),
        lambda: cs.cache_append(cache, table, z, k, k, inv_freq=fake(32)),
        lambda: cs.cache_append(cache, table, z, k, k, q=q[..., :32]),
        lambda: cs.cache_keep(cache, table, z, fake(3, 4)),
        lambda: cs.cache_keep(cache, table, z[:2], fake(3, 4, dtype=torch.int32)),
        lambda: cs.hybrid_attention_paged(q.float(), cache, table, z, z, 1, 0.1),
        lambda: cs.hybrid_attention_paged(q[:, ::2], cache, table, z, z, 1, 0.1),
        lambda: cs.hybrid_attention_paged(q, cache, table, z, z[:2], 1, 0.1),
        lambda: cs.tree_attention(q, cache, table, z, fake(3, 5, dtype=torch.int32), 0.1),
        lambda: cs.tree_attention(q, cache, table, z, fake(3, 4), 0.1),
    ]
    for f in bad:
        with pytest.raises(ValueError):
            f()


def test_tokens_of_a_projection_are_taken_as_they_are():
    qkv = torch.zeros(3, 5, 12 * 64, dtype=torch.bfloat16).as_subclass(_Fake)
    assert binding._tokens(qkv[:, :, :512].unflatten(2, (8, 64)), 3, 5, 64, "q") == 768
    assert binding._tokens(qkv[:1, :, 512:640].unflatten(2, (2, 64)), 1, 5, 64, "k") == 768
    assert binding._tokens(qkv[:, :1, 512:640].unflatten(2, (2, 64)), 3, 1, 64, "k") == 5 * 768
    assert binding._tokens(qkv[:1, :1, 512:640].unflatten(2, (2, 64)), 1, 1, 64, "k") == 128
