"""The C entry points of the experts' rows and of the paged cache on the CPU:
workspace sizes and the refusals that return before any HIP call, with no pointer
read; and the bindings' own checks, which need no device."""
import ctypes
import math

import pytest

import paper_2608_06912_amd as L
import paper_2608_06912_amd.experts as E
import paper_2608_06912_amd.paged as G

pytestmark = pytest.mark.skipif(not __import__("os").path.exists(L.LIB_PATH), reason="library not built")

INVALID, WORKSPACE = 1, 2
P = 256          # a pointer that is never read


@pytest.mark.parametrize("kw", [
    dict(indices=0), dict(order=0), dict(place=0), dict(offsets=0), dict(count=-1), dict(count=(1 << 30) + 1),
    dict(experts=0), dict(experts=2049)])
def test_order_refuses(kw):
    a = dict(indices=P, count=10, experts=4, order=P, place=P, offsets=P, ws=0, nbytes=0)
    a.update(kw)
    assert E._load().lapsum_expert_order(*a.values(), None) == INVALID


def test_order_workspace():
    lib = E._load()
    assert L.lapsum_expert_order_workspace_size(0, 4) == L.lapsum_expert_order_workspace_size(8192, 2048) == 0
    need = L.lapsum_expert_order_workspace_size(100000, 64)
    assert need > 0 and need % 256 == 0
    for ws, n in ((0, need), (P, need - 1), (P + 8, need)):
        assert lib.lapsum_expert_order(P, 100000, 64, P, P, P, ws, n, None) == WORKSPACE


def _strides(*s):
    return (ctypes.c_int64 * 3)(*s)


PRODUCT = dict(x=P, dtype=1, x_rows=10, x_stride=8, order=0, top_k=1, offsets=P, experts=3, rows=10, n_in=8,
               n_out=16)
BAD_PRODUCT = [
    dict(x=0), dict(dtype=3), dict(dtype=-1), dict(x_rows=-1), dict(x_rows=9), dict(x_stride=7), dict(top_k=0),
    dict(offsets=0), dict(experts=0), dict(experts=2049), dict(rows=-1), dict(rows=(1 << 30) + 1, order=P),
    dict(n_in=0), dict(n_out=0), dict(n_in=1 << 25, x_stride=1 << 25), dict(n_out=1 << 25)]


@pytest.mark.parametrize("kw", BAD_PRODUCT + [
    dict(w=0), dict(y=0), dict(y_dtype=2), dict(y_dtype=3), dict(strides=None), dict(strides=(128, 17, 2)),
    dict(strides=(128, 15, 1)), dict(strides=(128, 1, 7)), dict(strides=(-1, 16, 1))])
def test_matmul_refuses(kw):
    a = dict(PRODUCT, w=P, strides=(128, 16, 1), y=P, y_dtype=1)
    a.update(kw)
    if a["strides"] is not None:
        a["strides"] = _strides(*a["strides"])
    assert E._load().lapsum_expert_matmul(*a.values(), None) == INVALID


@pytest.mark.parametrize("kw", BAD_PRODUCT + [
    dict(g=0), dict(g_stride=15), dict(grad=0), dict(strides=(127, 16, 1)), dict(strides=(128, 2, 16)),
    dict(strides=(100, 1, 8))])
def test_matmul_weights_refuses(kw):
    a = dict(PRODUCT, g=P, g_stride=16, grad=P, strides=(128, 16, 1), ws=0, nbytes=0)
    a.update(kw)
    a["strides"] = _strides(*a["strides"])
    assert E._load().lapsum_expert_matmul_weights(*a.values(), None) == INVALID


@pytest.mark.parametrize("kw", [
    dict(rows=1 << 29, x_rows=1 << 29, n_out=1 << 10), dict(experts=512, rows=512, x_rows=512, n_out=1 << 24)])
def test_matmul_refuses_launches_of_too_many_threads(kw):
    a = {**PRODUCT, **kw, "w": P}
    strides = _strides(a["n_in"] * a["n_out"], a["n_out"], 1)
    assert E._load().lapsum_expert_matmul(*a.values(), strides, P, 1, None) == INVALID


def test_matmul_weights_refuses_launches_of_too_many_threads():
    a = {**PRODUCT, "experts": 2048, "x_stride": 1 << 14, "n_in": 1 << 14, "n_out": 1 << 13}
    strides = _strides(1 << 27, 1 << 13, 1)
    assert E._load().lapsum_expert_matmul_weights(*a.values(), P, 1 << 13, P, strides, 0, 0, None) == INVALID


def test_matmul_weights_workspace():
    lib = E._load()
    assert L.lapsum_expert_matmul_weights_workspace_size(64, 10000, 2048, 1024) == 0
    need = L.lapsum_expert_matmul_weights_workspace_size(2, 20000, 64, 72)
    assert need > 0 and need % 256 == 0
    for ws, n in ((0, need), (P, need - 1), (P + 8, need)):
        assert lib.lapsum_expert_matmul_weights(P, 1, 20000, 64, 0, 1, P, 2, 20000, 64, 72, P, 72, P,
                                                _strides(64 * 72, 72, 1), ws, n, None) == WORKSPACE


@pytest.mark.parametrize("kw", [
    dict(y=0), dict(dtype=3), dict(rows=-1), dict(dim=0), dict(dim=(1 << 24) + 1), dict(place=0), dict(tokens=-1),
    dict(top_k=0), dict(out=0), dict(out_dtype=2), dict(tokens=1 << 30, top_k=1 << 12)])
def test_combine_refuses(kw):
    a = dict(y=P, dtype=1, rows=8, dim=16, weights=0, place=P, tokens=4, top_k=2, out=P, out_dtype=1)
    a.update(kw)
    assert E._load().lapsum_expert_combine(*a.values(), None) == INVALID


@pytest.mark.parametrize("kw", [
    dict(grad=0), dict(y=0), dict(dtype=4), dict(rows=-1), dict(dim=0), dict(weights=0), dict(place=0),
    dict(offsets=0), dict(experts=0), dict(experts=2049), dict(tokens=-1), dict(top_k=0), dict(gy=0), dict(gw=0)])
def test_combine_backward_refuses(kw):
    a = dict(grad=P, y=P, dtype=1, rows=8, dim=16, weights=P, place=P, offsets=P, experts=4, tokens=4, top_k=2,
             gy=P, gw=P)
    a.update(kw)
    assert E._load().lapsum_expert_combine_backward(*a.values(), None) == INVALID


CACHE = dict(data=P, scale=P, pages=6, slots=16, page=16 * 64 * 2, head=16 * 64, slot=64, sp=32, sh=16)


def _cache(**kw):
    return ctypes.byref(G._Paged(*{**CACHE, **kw}.values()))


BAD_CACHE = [dict(pages=0), dict(slots=0), dict(slots=(1 << 30) + 1), dict(page=-1), dict(head=-1), dict(slot=-1),
             dict(scale=None), dict(sp=-1), dict(sh=-1)]


def _append(cache={}, **kw):
    a = dict(kn=P, ks=_strides(128, 64, 64), vn=P, vs=_strides(128, 64, 64), dtype=1, batch=2, kv=2, fresh=1, dim=64,
             seen=P, count=0, k=_cache(**cache), v=_cache(**{"data": P + 4096, "scale": P + 8192, **cache}), kind=3,
             table=P, width=3)
    a.update(kw)
    return G._load().lapsum_cache_append(*a.values(), None)


@pytest.mark.parametrize("cache", BAD_CACHE + [dict(slot=63), dict(head=0), dict(page=0), dict(sh=15), dict(sp=0)])
def test_append_refuses_caches(cache):
    assert _append(cache) == INVALID


@pytest.mark.parametrize("kw", [
    dict(kn=0), dict(vn=0), dict(ks=None), dict(vs=_strides(-1, 64, 64)), dict(dtype=3), dict(batch=-1), dict(kv=0),
    dict(fresh=-1), dict(dim=0), dict(dim=257), dict(seen=0), dict(kind=2), dict(kind=5), dict(kind=-1),
    dict(v=_cache(pages=5)), dict(v=_cache(slots=8)), dict(width=-1), dict(width=(1 << 30) // 16 + 1),
    dict(table=0, batch=7), dict(batch=1 << 20, fresh=1 << 20), dict(batch=1 << 27, fresh=1),
    dict(v=_cache(scale=P + 8192)), dict(v=_cache(data=P + 4096)), dict(v=_cache(), vn=P + 64),
    dict(v=_cache(), vs=_strides(128, 0, 64)), dict(v=_cache(slot=128)), dict(v=_cache(scale=None), kind=1, vn=P + 64)])
def test_append_refuses(kw):
    assert _append(**kw) == INVALID


@pytest.mark.parametrize("cache", BAD_CACHE)
def test_read_refuses_caches(cache):
    assert G._load().lapsum_cache_read(_cache(**cache), 3, 2, 2, 48, 64, P, P, 3, P, 1, None) == INVALID


@pytest.mark.parametrize("kw", [
    dict(kind=5), dict(kind=0), dict(batch=-1), dict(kv=0), dict(room=-1), dict(dim=0), dict(dim=257), dict(lens=0),
    dict(table=0, batch=7), dict(width=-1), dict(out=0), dict(dtype=3), dict(batch=1 << 20, room=1 << 20),
    dict(batch=1 << 25, room=4)])
def test_read_refuses(kw):
    a = dict(cache=_cache(), kind=3, batch=2, kv=2, room=48, dim=64, lens=P, table=P, width=3, out=P, dtype=1)
    a.update(kw)
    assert G._load().lapsum_cache_read(*a.values(), None) == INVALID


ATTEND = dict(q=P, qb=256, qh=64, dtype=1, k=None, v=None, kind=3, batch=2, heads=4, kv=2, dim=64, lens=P, table=P,
              width=3, scale=0.125, window=0, out=P, lse=0, weights=0, ws=0, nbytes=0)


def _attend(**kw):
    return G._load().lapsum_cache_attend(*{**ATTEND, "k": _cache(), "v": _cache(), **kw}.values(), None)


@pytest.mark.parametrize("kw", [
    dict(q=0), dict(qb=-1), dict(qh=-1), dict(dtype=3), dict(kind=2), dict(batch=-1), dict(heads=0), dict(heads=5),
    dict(kv=0), dict(dim=0), dict(dim=257), dict(lens=0), dict(table=0, batch=7), dict(width=-1),
    dict(scale=math.inf), dict(scale=math.nan), dict(window=-1), dict(window=1 << 31), dict(out=0), dict(weights=P),
    dict(batch=1 << 22, heads=4), dict(v=_cache(pages=5))] + [dict(k=_cache(**c)) for c in BAD_CACHE])
def test_attend_refuses(kw):
    assert _attend(**kw) == INVALID


def test_attend_workspace():
    assert L.lapsum_cache_attend_workspace_size(0, 4, 2, 64, 48) == 0
    need = L.lapsum_cache_attend_workspace_size(2, 4, 2, 64, 100000)
    assert need > 0 and need % 256 == 0
    wide = dict(width=100000 // 16 + 1)
    assert _attend(**wide) == WORKSPACE
    need = L.lapsum_cache_attend_workspace_size(2, 4, 2, 64, wide["width"] * 16)
    for ws, n in ((P, need - 1), (P + 8, need)):
        assert _attend(**wide, ws=ws, nbytes=n) == WORKSPACE


def test_bindings_refuse_what_is_not_on_a_device():
    import torch
    x, i = torch.zeros(2, 2, 8, 64), torch.zeros(2, dtype=torch.int32)
    for call in (lambda: L.lapsum_expert_order(i, 3), lambda: L.lapsum_expert_matmul(x[0, 0], x[0], i),
                 lambda: L.lapsum_expert_combine(x[0, 0], i[:, None]),
                 lambda: L.lapsum_expert_combine_backward(x[0, 0], x[0, 0], i[:, None], x[0, 0], i),
                 lambda: L.lapsum_expert_matmul_weights(x[0, 0], x[0, 0], i, x[0]),
                 lambda: L.lapsum_cache_append(x, x, i, x, x), lambda: L.lapsum_cache_read(x, i, 3),
                 lambda: L.lapsum_cache_attend(x[:, :, 0], x, x, i)):
        with pytest.raises(ValueError):
            call()
