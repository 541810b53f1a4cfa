"""What autograd is told by the selections: derivatives in forward mode are
refused and not dropped, and what a call writes in place is known as changed."""
import pytest

from test_gpu_selection_binding import way  # noqa: F401  (both ways into the library)

pytestmark = pytest.mark.gpu


def test_forward_mode_is_refused(lib, way):  # noqa: F811
    import torch
    import torch.autograd.forward_ad as fw
    import paper_2608_06912_amd.autograd as A
    x = torch.randn(5, 12, device="cuda")
    want = A.route_topk(x, 3, counts=True)
    with fw.dual_level():
        dual = fw.make_dual(x, torch.ones_like(x))
        for kw in ({}, dict(score="sigmoid", renormalise=True), dict(counts=True)):
            with pytest.raises(RuntimeError):
                A.route_topk(dual, 3, **kw)
            with torch.no_grad(), pytest.raises(RuntimeError):
                A.route_topk(dual, 3, **kw)
        # what has no tangent goes on as it does elsewhere
        for a, b in zip(A.route_topk(x, 3, counts=True), want):
            assert torch.equal(a, b)
    with pytest.raises(RuntimeError):
        torch.func.jvp(lambda t: A.route_topk(t, 3)[0], (x,), (torch.ones_like(x),))


def _cache(torch, batch=2, kv=2, slots=10, dim=4):
    k, v = torch.randn(batch, kv, slots, dim, device="cuda"), torch.randn(batch, kv, slots, dim, device="cuda")
    acc = torch.rand(batch, kv, slots, device="cuda")
    pos = torch.arange(slots, dtype=torch.int32, device="cuda").expand(batch, kv, slots).contiguous()
    seen = torch.full((batch,), slots, dtype=torch.int32, device="cuda")
    return k, v, acc, pos, seen


def test_what_is_written_in_place_is_known_as_changed(lib, way):  # noqa: F811
    """Version counters of what a call writes go up, of what it reads not, and a
    backward through what it wrote over is an error, as after torch's own in-place calls."""
    import torch
    k, v, acc, pos, seen = _cache(torch)
    w, new = torch.rand(2, 4, 10, device="cuda"), torch.randn(2, 2, 4, device="cuda")
    states = [torch.randn(4, 3, 6, 2, device="cuda") for _ in range(2)]
    other = [torch.empty_like(t) for t in states]
    parents = torch.tensor([[1, 0], [1, 1]], dtype=torch.int32, device="cuda")
    window = torch.rand(2, 4, 3, 10, device="cuda")
    calls = [
        (lambda: lib.lapsum_cache_step(w, new, new, seen, k, v, acc, pos), [k, v, acc, pos], [w, new, seen]),
        (lambda: lib.lapsum_beam_reorder(states, parents, length=3), states, [parents]),
        (lambda: lib.lapsum_beam_reorder(states, parents, out=other), other, [parents, *states]),
        (lambda: lib.lapsum_cache_accumulate(window, 2, seen=seen, acc=acc), [acc], [window, seen]),
        (lambda: lib.lapsum_cache_accumulate(window, 2, seen=seen), [], [window, seen, acc]),
        (lambda: lib.lapsum_cache_evict(k, v, acc, seen, 4, pos=pos), [], [k, v, acc, seen, pos]),
    ]
    for call, written, read in calls:
        leaf = torch.ones((), device="cuda", requires_grad=True)
        products = [leaf * t for t in written if t.is_floating_point()]
        before = [t._version for t in written], [t._version for t in read]
        call()
        assert all(t._version > n for t, n in zip(written, before[0]))
        assert [t._version for t in read] == before[1]
        for y in products:
            with pytest.raises(RuntimeError, match="modified by an inplace operation"):
                y.sum().backward()


def test_a_view_that_is_written_changes_its_base(lib, way):  # noqa: F811
    import torch
    k, v, acc, pos, seen = _cache(torch)
    both = torch.stack([k, v])
    n = both._version
    lib.lapsum_cache_step(torch.rand(2, 4, 10, device="cuda"), torch.randn(2, 2, 4, device="cuda"),
                          torch.randn(2, 2, 4, device="cuda"), seen, both[0], both[1], acc, pos)
    assert both._version > n


def test_tensors_that_require_grad_are_not_written(lib, way):  # noqa: F811
    import torch
    w, new = torch.rand(2, 4, 10, device="cuda"), torch.randn(2, 2, 4, device="cuda")
    parents = torch.tensor([[1, 0], [1, 1]], dtype=torch.int32, device="cuda")
    window = torch.rand(2, 4, 3, 10, device="cuda")
    for which in range(3):
        for leaf in (True, False):
            parts = list(_cache(torch))
            parts[which].requires_grad_()
            if not leaf:
                parts[which] = parts[which] * 1.0
            was = [t.detach().clone() for t in parts]
            k, v, acc, pos, seen = parts
            with pytest.raises(RuntimeError, match="requires grad"):
                lib.lapsum_cache_step(w, new, new, seen, k, v, acc, pos)
            if which == 2:
                with pytest.raises(RuntimeError, match="requires grad"):
                    lib.lapsum_cache_accumulate(window, 2, acc=acc)
            assert all(torch.equal(a, b) for a, b in zip(parts, was))
            with torch.no_grad():
                lib.lapsum_cache_step(w, new, new, seen, k, v, acc, pos)
            assert not torch.equal(parts[which], was[which])
    plain, grad = torch.randn(4, 6, device="cuda"), torch.randn(4, 6, device="cuda", requires_grad=True)
    was = grad.detach().clone()
    with pytest.raises(RuntimeError, match="requires grad"):
        lib.lapsum_beam_reorder([grad], parents)
    with pytest.raises(RuntimeError, match="requires grad"):
        lib.lapsum_beam_reorder([plain], parents, out=[grad])
    assert torch.equal(grad, was)
    # read, it may: the result is one without a gradient
    out = torch.empty_like(plain)
    lib.lapsum_beam_reorder([grad], parents, out=[out])
    assert torch.equal(out, grad.detach()[[1, 0, 3, 3]])
    with torch.no_grad():
        lib.lapsum_beam_reorder([grad], parents)
    assert torch.equal(grad, was[[1, 0, 3, 3]])


def test_inference_tensors_are_written(lib, way):  # noqa: F811
    """They have no version and nothing saves them: inside inference mode and after it."""
    import torch
    with torch.inference_mode():
        k, v, acc, pos, seen = _cache(torch)
        w, new = torch.rand(2, 4, 10, device="cuda"), torch.randn(2, 2, 4, device="cuda")
        lib.lapsum_cache_step(w, new, new, seen, k, v, acc, pos)
        plain = acc.clone()
    lib.lapsum_cache_step(w, new, new, seen + 1, k, v, acc, pos)
    lib.lapsum_cache_accumulate(w[:, :, None], 2, acc=acc)
    lib.lapsum_beam_reorder([k, v], torch.tensor([[1, 0]], dtype=torch.int32, device="cuda"))
    assert not torch.equal(acc, plain)
