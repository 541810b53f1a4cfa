"""What autograd is told by the selections: derivatives in forward mode are
refused and not dropped."""
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
