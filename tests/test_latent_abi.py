"""The latent cache's and the pages' entry points without a GPU: what they refuse before anything is
enqueued."""
import ctypes
import math

import pytest
import torch

import paper_2605_24793_amd as cs
from paper_2605_24793_amd import binding

OK, INVALID, UNSUPPORTED, WORKSPACE = 0, -1, -2, -3
FAKE = 0x10000          # an aligned address; validation never dereferences device pointers
BF16, F8 = 1, 2


def _cache(dtype=F8, page=64, d_c=512, n_pages=100, c=FAKE, r=FAKE, scale=FAKE, table=FAKE, max_pages=20):
    return binding._LatentCache(dtype, page, d_c, n_pages, c, r, scale, table, max_pages)


def _append(L, cache=None, start=FAKE, count=None, c=FAKE, ld_c=576, k_r=FAKE, ld_r=576, weight=None, eps=1e-6, rope=None,
            positions=None, B=2, n=3, q=None, ld_q=0, head_q=0, Hq=0, q_out=None, head_out=0, c_out=None, k_out=None):
    return L.cospec_latent_append(ctypes.byref(cache or _cache()), start, count, c, ld_c, k_r, ld_r, weight, eps,
                                  None if rope is None else ctypes.byref(binding._Rope(*rope)), positions, B, n, q, ld_q,
                                  head_q, Hq, q_out, head_out, c_out, k_out, None)


def _keep(L, cache=None, ctx=FAKE, path=FAKE, B=2, N=9):
    return L.cospec_latent_keep(ctypes.byref(cache or _cache()), ctx, path, B, N, None)


def _attend(L, cache=None, q=FAKE, ctx=FAKE, qs=FAKE, B=2, n=17, Hq=16, K=7, scale=0.1, out=FAKE, ws=FAKE, wsb=1 << 40):
    return L.cospec_latent_attention(q, ctypes.byref(cache or _cache()), ctx, qs, B, n, Hq, K, scale, out, ws, wsb, None)


def _tree(L, cache=None, q=FAKE, ctx=FAKE, parent=FAKE, B=2, N=60, Hq=16, scale=0.1, out=FAKE, ws=FAKE, wsb=1 << 40):
    return L.cospec_latent_tree_attention(q, ctypes.byref(cache or _cache()), ctx, parent, B, N, Hq, scale, out, ws, wsb, None)


@pytest.mark.parametrize("kw,code", [
    (dict(dtype=0), UNSUPPORTED), (dict(dtype=3), UNSUPPORTED), (dict(page=8), UNSUPPORTED), (dict(page=48), UNSUPPORTED),
    (dict(page=256), UNSUPPORTED), (dict(d_c=128), UNSUPPORTED), (dict(d_c=384), UNSUPPORTED), (dict(n_pages=-1), INVALID),
    (dict(n_pages=0), INVALID), (dict(max_pages=0), INVALID), (dict(max_pages=-3), INVALID),
    (dict(max_pages=(1 << 31) // 64 + 1), UNSUPPORTED), (dict(n_pages=1 << 31), UNSUPPORTED), (dict(c=None), INVALID),
    (dict(c=FAKE + 8), INVALID), (dict(r=FAKE + 8), INVALID), (dict(r=None), INVALID), (dict(scale=None), INVALID),
    (dict(scale=FAKE + 2), INVALID), (dict(table=None), INVALID), (dict(table=FAKE + 2), INVALID),
])
def test_every_call_checks_the_cache(kw, code):
    L = cs.lib()
    bad = _cache(**kw)
    for call in (_append, _keep, _attend, _tree):
        assert call(L, cache=bad) == code, call.__name__


def test_no_cache_at_all():
    L = cs.lib()
    assert L.cospec_latent_attention(FAKE, None, FAKE, FAKE, 1, 1, 8, 0, 0.1, FAKE, None, 0, None) == INVALID
    assert L.cospec_latent_tree_attention(FAKE, None, FAKE, FAKE, 1, 1, 8, 0.1, FAKE, None, 0, None) == INVALID
    assert L.cospec_latent_keep(None, FAKE, FAKE, 1, 1, None) == INVALID
    assert L.cospec_latent_append(None, FAKE, None, FAKE, 576, FAKE, 576, None, 0.0, None, None, 1, 1, None, 0, 0, 0, None,
                                  0, None, None, None) == INVALID
    assert L.cospec_latent_attention_workspace_size(None, 1, 1, 8) == 0


Q = dict(q=FAKE, ld_q=16 * 192, head_q=192, Hq=16, q_out=FAKE, head_out=576)


@pytest.mark.parametrize("kw,code", [
    (dict(B=-1), INVALID), (dict(n=-1), INVALID), (dict(start=None), INVALID), (dict(start=FAKE + 2), INVALID),
    (dict(count=FAKE + 1), INVALID), (dict(c=None), INVALID), (dict(c=FAKE + 8), INVALID), (dict(k_r=None), INVALID),
    (dict(k_r=FAKE + 4), INVALID), (dict(ld_c=504), INVALID), (dict(ld_c=516), INVALID), (dict(ld_r=56), INVALID),
    (dict(ld_r=68), INVALID), (dict(weight=FAKE + 8), INVALID), (dict(eps=-1e-6), INVALID), (dict(eps=math.nan), INVALID),
    (dict(eps=math.inf), INVALID), (dict(positions=FAKE + 2), INVALID), (dict(rope=(80, 0, FAKE)), INVALID),
    (dict(rope=(-16, 0, FAKE)), INVALID), (dict(rope=(24, 0, FAKE)), UNSUPPORTED), (dict(rope=(64, 0, None)), INVALID),
    (dict(rope=(64, 1, FAKE + 2)), INVALID), (dict(Q, Hq=0), INVALID), (dict(Q, head_q=56), INVALID),
    (dict(Q, head_q=196), INVALID), (dict(Q, ld_q=100), INVALID), (dict(Q, ld_q=-8), INVALID), (dict(Q, head_out=60), INVALID),
    (dict(Q, q_out=None), INVALID), (dict(Q, q=FAKE + 4), INVALID), (dict(Q, q_out=FAKE + 8), INVALID),
    (dict(c_out=FAKE + 8), INVALID), (dict(k_out=FAKE + 8), INVALID), (dict(B=1 << 20, n=1 << 20), UNSUPPORTED),
    (dict(B=1 << 24, n=1), UNSUPPORTED), (dict(B=0), OK), (dict(n=0), OK), (dict(B=0, c=None, k_r=None, start=None), OK),
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
    (_attend, dict(Hq=0), INVALID), (_attend, dict(K=-1), INVALID), (_attend, dict(scale=math.nan), INVALID),
    (_attend, dict(scale=math.inf), INVALID), (_attend, dict(q=None), INVALID), (_attend, dict(q=FAKE + 8), INVALID),
    (_attend, dict(out=FAKE + 2), INVALID), (_attend, dict(ctx=None), INVALID), (_attend, dict(qs=FAKE + 2), INVALID),
    (_attend, dict(B=-2), INVALID), (_attend, dict(n=-2), INVALID), (_attend, dict(B=1 << 20, n=1 << 20), UNSUPPORTED),
    (_attend, dict(B=1 << 25, n=1, Hq=1), UNSUPPORTED), (_attend, dict(n=0, q=None), OK), (_attend, dict(B=0, q=None), OK),
    (_attend, dict(ws=None), WORKSPACE), (_attend, dict(ws=FAKE + 16), WORKSPACE), (_attend, dict(wsb=1000), WORKSPACE),
    (_tree, dict(N=0), INVALID), (_tree, dict(N=257), UNSUPPORTED), (_tree, dict(parent=None), INVALID),
    (_tree, dict(parent=FAKE + 2), INVALID), (_tree, dict(scale=-math.inf), INVALID), (_tree, dict(q=FAKE + 4), INVALID),
    (_tree, dict(B=0, q=None, parent=None), OK), (_tree, dict(N=1, ws=None), WORKSPACE),
])
def test_attention_refuses(call, kw, code):
    assert call(cs.lib(), **kw) == code


def test_attention_workspace_size():
    L = cs.lib()

    def size(B, n, Hq, **kw):
        return L.cospec_latent_attention_workspace_size(ctypes.byref(_cache(**kw)), B, n, Hq)

    assert size(1, 1, 16) > 0 and size(1, 1, 16) % 256 == 0
    assert size(1024, 1, 16) == 0                            # a workgroup for every CU: not cut
    assert size(1, 1, 16, d_c=256) < size(1, 1, 16)
    assert size(-1, 1, 16) == 0 and size(1, 1, 0) == 0 and size(1, 1, 16, page=20) == 0


def _expanded(L, q=FAKE, k=FAKE, ld_k=4096, head_k=256, v=FAKE, ld_v=4096, head_v=256, k_r=FAKE, ld_r=64, ctx=FAKE, qs=FAKE,
              B=2, n=17, length=100, H=16, d=128, K=7, scale=0.1, out=FAKE):
    return L.cospec_expanded_attention(q, k, ld_k, head_k, v, ld_v, head_v, k_r, ld_r, ctx, qs, B, n, length, H, d, K, scale,
                                       out, None)


@pytest.mark.parametrize("kw,code", [
    (dict(d=96), UNSUPPORTED), (dict(H=0), INVALID), (dict(B=-1), INVALID), (dict(n=-1), INVALID), (dict(length=-1), INVALID),
    (dict(K=-1), INVALID), (dict(scale=math.nan), INVALID), (dict(head_k=120), INVALID), (dict(head_v=132), INVALID),
    (dict(ld_k=-8), INVALID), (dict(ld_v=4), INVALID), (dict(ld_r=56), INVALID), (dict(q=None), INVALID),
    (dict(k=FAKE + 8), INVALID), (dict(v=None), INVALID), (dict(k_r=FAKE + 4), INVALID), (dict(ctx=None), INVALID),
    (dict(qs=None), INVALID), (dict(out=FAKE + 8), INVALID), (dict(B=1 << 22, H=16), UNSUPPORTED),
    (dict(B=1 << 10, H=16, n=1 << 20), UNSUPPORTED), (dict(B=0, q=None), OK), (dict(n=0, q=None), OK),
])
def test_expanded_refuses(kw, code):
    assert _expanded(cs.lib(), **kw) == code


def _pool(refs=FAKE, n_pages=100, page=64):
    return binding._Pool(refs, n_pages, page)


def _fork(L, pool=None, table=FAKE, rows=3, row=FAKE, length=FAKE, B=2, T=10, to=FAKE):
    return L.cospec_pages_fork(ctypes.byref(pool or _pool()), table, rows, row, length, B, T, to, None)


def _reserve(L, pool=None, table=FAKE, T=10, start=FAKE, count=None, B=2, n=5, copies=FAKE, lacking=FAKE, ws=FAKE, wsb=1 << 30):
    return L.cospec_pages_reserve(ctypes.byref(pool or _pool()), table, T, start, count, B, n, copies, lacking, ws, wsb, None)


def _release(L, pool=None, table=FAKE, T=10, keep=FAKE, B=2):
    return L.cospec_pages_release(ctypes.byref(pool or _pool()), table, T, keep, B, None)


def _compact(L, pool=None, table=FAKE, T=10, B=2, moves=FAKE, n_moves=FAKE, ws=FAKE, wsb=1 << 30):
    return L.cospec_pages_compact(ctypes.byref(pool or _pool()), table, T, B, moves, n_moves, ws, wsb, None)


@pytest.mark.parametrize("kw,code", [
    (dict(refs=None), INVALID), (dict(refs=FAKE + 2), INVALID), (dict(n_pages=0), INVALID), (dict(n_pages=-1), INVALID),
    (dict(n_pages=1 << 30), UNSUPPORTED), (dict(page=20), UNSUPPORTED),
])
def test_every_call_checks_the_pool(kw, code):
    L = cs.lib()
    for call in (_fork, _reserve, _release, _compact):
        assert call(L, pool=_pool(**kw)) == code, call.__name__


@pytest.mark.parametrize("call,kw,code", [
    (_fork, dict(B=-1), INVALID), (_fork, dict(rows=-1), INVALID), (_fork, dict(T=0), INVALID), (_fork, dict(table=None), INVALID),
    (_fork, dict(row=None), INVALID), (_fork, dict(length=FAKE + 2), INVALID), (_fork, dict(to=None), INVALID),
    (_fork, dict(B=1 << 28), UNSUPPORTED), (_fork, dict(B=0, table=None, row=None, to=None), OK),
    (_reserve, dict(B=-1), INVALID), (_reserve, dict(n=-1), INVALID), (_reserve, dict(T=0), INVALID),
    (_reserve, dict(table=None), INVALID), (_reserve, dict(start=None), INVALID), (_reserve, dict(copies=FAKE + 4), INVALID),
    (_reserve, dict(lacking=None), INVALID), (_reserve, dict(count=FAKE + 2), INVALID), (_reserve, dict(ws=None), WORKSPACE),
    (_reserve, dict(wsb=256), WORKSPACE), (_reserve, dict(ws=FAKE + 8), WORKSPACE), (_reserve, dict(B=1 << 20, n=1 << 20), UNSUPPORTED),
    (_release, dict(B=-1), INVALID), (_release, dict(table=None), INVALID), (_release, dict(keep=FAKE + 2), INVALID),
    (_release, dict(B=0, table=None), OK),
    (_compact, dict(B=-1), INVALID), (_compact, dict(table=None), INVALID), (_compact, dict(moves=FAKE + 4), INVALID),
    (_compact, dict(n_moves=None), INVALID), (_compact, dict(ws=None), WORKSPACE), (_compact, dict(wsb=256), WORKSPACE),
])
def test_pages_refuse(call, kw, code):
    assert call(cs.lib(), **kw) == code


@pytest.mark.parametrize("kw,code", [
    (dict(data=None), INVALID), (dict(data=FAKE + 2), INVALID), (dict(size=0), INVALID), (dict(size=6), INVALID),
    (dict(size=-4), INVALID), (dict(size=(1 << 32) + 4), UNSUPPORTED), (dict(n_planes=-1), INVALID), (dict(n_pairs=-1), INVALID),
    (dict(n_pages=0), INVALID), (dict(n_pages=1 << 30), UNSUPPORTED), (dict(pairs=None), INVALID), (dict(pairs=FAKE + 4), INVALID),
    (dict(count=FAKE + 2), INVALID), (dict(n_planes=0), OK), (dict(n_pairs=0, pairs=None), OK),
])
def test_copy_refuses(kw, code):
    a = dict(dict(data=FAKE, size=64, n_planes=1, n_pages=10, pairs=FAKE, n_pairs=2, count=None), **kw)
    planes = (binding._Plane * 1)(binding._Plane(a["data"], a["size"]))
    assert cs.lib().cospec_pages_copy(planes, a["n_planes"], a["n_pages"], a["pairs"], a["n_pairs"], a["count"], None) == code


def test_the_binding_refuses_tensors_of_the_host():
    with pytest.raises(ValueError):
        cs.LatentCache(torch.zeros(2, 16, 512, dtype=torch.bfloat16), torch.zeros(2, 16, 64, dtype=torch.bfloat16))
    with pytest.raises(ValueError):
        cs.PagePool(torch.zeros(4, dtype=torch.int32), 64)
    with pytest.raises(TypeError):
        cs.LatentCache(torch.zeros(2, 16, 512), torch.zeros(2, 16, 64, dtype=torch.bfloat16))
