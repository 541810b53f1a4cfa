"""The paged cache has no gradients: asking for one is an error, and never a gradient that is silently
without the cache's part."""
import pytest

from test_gpu_products_binding import _inputs, way  # noqa: F401  (both ways into the library)

pytestmark = pytest.mark.gpu


def _cache(r, kind):
    import torch
    if kind == "same":
        return r(2, 2, 16, 64), None
    return torch.randint(-9, 9, (2, 2, 16, 64), device="cuda", dtype=torch.int8), r(2, 2, 16).abs()


@pytest.mark.parametrize("kind", ["same", "int8"])
def test_attention_has_no_gradient(lib, way, kind):  # noqa: F811
    torch, gen, r = _inputs(4)
    (k, ks), (v, vs) = _cache(r, kind), _cache(r, kind)
    lens = torch.tensor([16, 5], dtype=torch.int32, device="cuda")
    q = r(2, 4, 64)
    want = lib.lapsum_cache_attend(q, k, v, lens, k_scale=ks, v_scale=vs, lse=True, weights=True)
    assert not any(t.requires_grad for t in want)
    leaves = [{"q": q.clone().requires_grad_()}]
    leaves += [{n: t.clone().requires_grad_()} for n, t in
               ((("k", k), ("v", v)) if kind == "same" else (("k_scale", ks), ("v_scale", vs)))]
    for leaf in leaves:
        (x,) = leaf.values()
        args = {"q": q, "k": k, "v": v, "lens": lens, "k_scale": ks, "v_scale": vs, **leaf}
        for more in ({}, {"lse": True}, {"lse": True, "weights": True}, {"weights": True}):
            got = lib.lapsum_cache_attend(**args, **more)
            got = got if isinstance(got, tuple) else (got,)
            assert bool(torch.equal(got[0], want[0]))
            for y in got:
                with pytest.raises(RuntimeError, match="lapsum_cache_attend"):
                    (y.sum() + x.sum()).backward()
            x.grad = None
        with torch.no_grad():
            y = lib.lapsum_cache_attend(**args)
        assert not y.requires_grad
        (y.sum() + x.sum()).backward()
        assert bool((x.grad == 1.0).all())


@pytest.mark.parametrize("kind", ["same", "int8"])
def test_reading_back_has_no_gradient(lib, way, kind):  # noqa: F811
    torch, gen, r = _inputs(4)
    x, s = _cache(r, kind)
    lens = torch.tensor([16, 5], dtype=torch.int32, device="cuda")
    want = lib.lapsum_cache_read(x, lens, 16, scale=s)
    leaf = (x if s is None else s).clone().requires_grad_()
    args = {"x": leaf, "scale": None} if s is None else {"x": x, "scale": leaf}
    got = lib.lapsum_cache_read(lens=lens, room=16, **args)
    assert bool(torch.equal(got, want)) and not want.requires_grad
    with pytest.raises(RuntimeError, match="lapsum_cache_read"):
        (got.sum() + leaf.sum()).backward()
    with torch.no_grad():
        assert not lib.lapsum_cache_read(lens=lens, room=16, **args).requires_grad
