"""The hard selections' C entry points on the CPU: workspace sizes and the
refusals that return before any HIP call, with no pointer read; and the Python
binding's own checks, which need no device."""
import ctypes

import pytest

import paper_2608_06912_amd as L
import paper_2608_06912_amd.selection as S

pytestmark = pytest.mark.skipif(not __import__("os").path.exists(L.LIB_PATH), reason="library not built")

INVALID, WORKSPACE = 1, 2
P = 256          # a pointer that is never read


@pytest.fixture(scope="module")
def lib():
    return S._load()


def _route(lib, **kw):
    a = dict(logits=P, dtype=0, tokens=4, experts=16, stride=16, score=0, bias=0, groups=1,
             topk_groups=1, group_top=1, top_k=2, renorm=0, scale=1.0, weights=P, indices=P, counts=0,
             ws=0, nbytes=0)
    assert set(kw) <= set(a)
    a.update(kw)
    return lib.lapsum_route_forward(*a.values(), None)


@pytest.mark.parametrize("kw", [
    dict(logits=0), dict(weights=0), dict(indices=0), dict(dtype=3), dict(dtype=-1), dict(tokens=-1),
    dict(experts=0), dict(experts=2049, stride=4096), dict(stride=15), dict(score=2), dict(score=-1),
    dict(groups=0), dict(groups=3), dict(groups=65), dict(groups=4, topk_groups=0),
    dict(groups=4, topk_groups=5), dict(group_top=0), dict(group_top=3),
    dict(groups=16, topk_groups=4, group_top=2), dict(top_k=0), dict(top_k=17),
    dict(groups=8, topk_groups=1, top_k=3), dict(scale=float("inf")), dict(scale=float("nan")),
    dict(experts=128, stride=128, top_k=65)])
def test_route_forward_refuses(lib, kw):
    assert _route(lib, **kw) == INVALID


def test_route_workspace(lib):
    assert L.lapsum_route_forward_workspace_size(10 ** 6, 256, 8) == 0
    assert L.lapsum_route_forward_workspace_size(16, 256, 8, 1, True) == 0
    need = L.lapsum_route_forward_workspace_size(10 ** 6, 256, 8, 1, True)
    assert need > 0 and need % 256 == 0
    assert _route(lib, tokens=10 ** 6, experts=256, stride=256, counts=P) == WORKSPACE
    assert _route(lib, tokens=10 ** 6, experts=256, stride=256, counts=P, ws=P, nbytes=need - 1) == WORKSPACE
    assert _route(lib, tokens=10 ** 6, experts=256, stride=256, counts=P, ws=P + 8, nbytes=need) == WORKSPACE


@pytest.mark.parametrize("kw", [
    dict(grad=0), dict(logits=0), dict(indices=0), dict(out=0), dict(dtype=9), dict(tokens=-3),
    dict(experts=0), dict(stride=3), dict(score=5), dict(top_k=0), dict(top_k=99), dict(scale=float("nan"))])
def test_route_backward_refuses(lib, kw):
    a = dict(grad=P, logits=P, dtype=0, tokens=4, experts=16, stride=16, indices=P, score=0, top_k=2,
             renorm=0, scale=1.0, out=P)
    a.update(kw)
    assert lib.lapsum_route_backward(*a.values(), None) == INVALID


@pytest.mark.parametrize("kw", [
    dict(logits=0), dict(cum=0), dict(scores=0), dict(tokens=0), dict(parents=0), dict(dtype=4),
    dict(batch=-1), dict(beams=0), dict(beams=33), dict(batch=65535), dict(vocab=0),
    dict(vocab=2 ** 31 // 2, stride=2 ** 31), dict(stride=99), dict(num=0), dict(num=33)])
def test_beam_select_refuses(lib, kw):
    a = dict(logits=P, dtype=1, batch=2, beams=4, vocab=100, stride=100, cum=P, num=8, scores=P, tokens=P,
             parents=P, ws=0, nbytes=0)
    a.update(kw)
    assert lib.lapsum_beam_select(*a.values(), None) == INVALID


def test_beam_workspace(lib):
    need = L.lapsum_beam_select_workspace_size(2, 4, 32000, 8)
    assert need > 0 and need % 256 == 0
    assert L.lapsum_beam_select_workspace_size(0, 4, 32000, 8) == 0
    args = (P, 1, 2, 4, 32000, 32000, P, 8, P, P, P)
    assert lib.lapsum_beam_select(*args, None, 0, None) == WORKSPACE
    assert lib.lapsum_beam_select(*args, P, need - 1, None) == WORKSPACE
    assert lib.lapsum_beam_select(*args, P + 4, need, None) == WORKSPACE


@pytest.mark.parametrize("kw", [
    dict(src=0), dict(dst=0), dict(row_bytes=100), dict(outer=-1), dict(live_bytes=-1),
    dict(outer_stride=10), dict(row_bytes=-4), dict(outer=2 ** 62), dict(live_bytes=2 ** 62),
    dict(outer_stride=2 ** 62)])
def test_beam_reorder_refuses_states(lib, kw):
    a = dict(src=P, dst=P, row_bytes=256, outer=4, outer_stride=64, live_bytes=32)
    a.update(kw)
    s = S._BeamState(**a)
    assert lib.lapsum_beam_reorder(ctypes.addressof(s), 1, P, 4, 2, 4, None) == INVALID


def test_beam_reorder_refuses(lib):
    for args in ((None, 1, P, 4, 2, 4), (None, -1, P, 4, 2, 4), (None, 0, None, 4, 2, 4),
                 (None, 0, P, 3, 2, 4), (None, 0, P, 4, -1, 4), (None, 0, P, 4, 65536, 4),
                 (None, 0, P, 4, 2, 0), (None, 0, P, 64, 2, 33)):
        assert lib.lapsum_beam_reorder(*args, None) == INVALID


@pytest.mark.parametrize("kw", [
    dict(weights=0), dict(acc=0), dict(dtype=3), dict(batch=-1), dict(heads=0), dict(heads=7), dict(kv=0),
    dict(queries=-1), dict(keys=-1), dict(keys=2 ** 31), dict(sb=-1), dict(sh=-1), dict(sq=-1),
    dict(batch=2 ** 30, keys=2 ** 20)])
def test_cache_accumulate_refuses(lib, kw):
    a = dict(weights=P, dtype=0, batch=2, heads=8, kv=4, queries=3, keys=50, sb=1200, sh=150, sq=50, seen=0,
             acc_in=0, acc=P)
    a.update(kw)
    assert lib.lapsum_cache_accumulate(*a.values(), None) == INVALID


STRIDES = (ctypes.c_int64 * 3)(4000, 1000, 10)
NEGATIVE = (ctypes.c_int64 * 3)(4000, -1000, 10)


@pytest.mark.parametrize("kw", [
    dict(k=0), dict(ks=None), dict(v=0), dict(vs=None), dict(ks=NEGATIVE), dict(vs=NEGATIVE),
    dict(row_bytes=0), dict(row_bytes=2 ** 31), dict(acc=0), dict(seen=0), dict(batch=-1), dict(kv=0),
    dict(slots=0), dict(slots=2 ** 31), dict(budget=0), dict(budget=2 ** 31), dict(sink=-1),
    dict(recent=-1), dict(sink=6, recent=5), dict(k_out=0), dict(v_out=0), dict(acc_out=0),
    dict(pos_out=0), dict(batch=2 ** 22, kv=4)])
def test_cache_evict_refuses(lib, kw):
    a = dict(k=P, ks=STRIDES, v=P, vs=STRIDES, row_bytes=10, acc=P, pos=0, seen=P, batch=2, kv=4, slots=100,
             budget=10, sink=2, recent=3, k_out=P, v_out=P, acc_out=P, pos_out=P, ws=0, nbytes=0)
    a.update(kw)
    assert lib.lapsum_cache_evict(*a.values(), None) == INVALID


def test_cache_evict_workspace(lib):
    need = L.lapsum_cache_evict_workspace_size(2, 4, 100, 10)
    assert need >= 2 * 4 * 10 * 4 and need % 256 == 0
    args = (P, STRIDES, P, STRIDES, 10, P, 0, P, 2, 4, 100, 10, 2, 3, P, P, P, P)
    for ws, nbytes in ((None, 0), (P, need - 1), (P + 16, need)):
        assert lib.lapsum_cache_evict(*args, ws, nbytes, None) == WORKSPACE


@pytest.mark.parametrize("kw", [
    dict(weights=0), dict(dtype=7), dict(sb=-1), dict(sh=-1), dict(k_new=0), dict(v_new=0), dict(seen=0),
    dict(k=0), dict(ks=None), dict(v=0), dict(vs=None), dict(ks=NEGATIVE), dict(row_bytes=0), dict(acc=0),
    dict(pos=0), dict(batch=-2), dict(heads=6), dict(heads=0), dict(kv=0), dict(slots=0), dict(sink=-1),
    dict(recent=0), dict(sink=97, recent=4), dict(slot=0)])
def test_cache_step_refuses(lib, kw):
    a = dict(weights=P, dtype=0, sb=800, sh=100, k_new=P, v_new=P, seen=P, k=P, ks=STRIDES, v=P, vs=STRIDES,
             row_bytes=10, acc=P, pos=P, batch=2, heads=8, kv=4, slots=100, sink=2, recent=3, slot=P)
    a.update(kw)
    assert lib.lapsum_cache_step(*a.values(), None) == INVALID


def test_the_binding_refuses_host_tensors():
    import torch
    x, f = torch.zeros(4, 8), torch.zeros(2, 2)
    i = torch.zeros(2, 2, dtype=torch.int32)
    c = torch.zeros(2, 2, 4, 8)
    for call in (lambda: L.lapsum_route_forward(x, 2), lambda: L.lapsum_beam_select(x, f, 2),
                 lambda: L.lapsum_route_backward(f, x, i), lambda: L.lapsum_beam_reorder([x], i),
                 lambda: L.lapsum_cache_accumulate(c, 2), lambda: L.lapsum_cache_evict(c, c, c, i, 2),
                 lambda: L.lapsum_cache_step(c, c, c, i, c, c, c, i)):
        with pytest.raises(ValueError):
            call()


def test_cache_accumulate_refuses_more_rows_than_it_counts(lib):
    for heads, kv, queries in ((8, 4, 2 ** 29 + 1), (4, 4, 2 ** 31), (4, 1, 2 ** 28 + 1), (2 ** 31, 1, 1)):
        assert lib.lapsum_cache_accumulate(P, 0, 1, heads, kv, queries, 1, 0, 0, 0, 0, 0, P, None) == INVALID
