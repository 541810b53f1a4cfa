"""What the routing compares where a softmax has a bias, to the last bit.

c = s + bias in float32, from s = e / float32(sum of e) with e = exp(x - max),
the sum formed in 64 bits.  The bias is large beside the scores, so that c holds few of their
bits: many experts are equal or a spacing apart, and a bit of s decides."""
import pytest

pytestmark = pytest.mark.gpu


def _best(value, k):
    """The k largest of float32 values, equal ones by the lowest index."""
    import torch
    bits = (value + 0.0).view(torch.int32)
    order = (bits ^ ((bits >> 31) & 0x7FFFFFFF)).long() << 32
    key = order + torch.arange(value.shape[-1] - 1, -1, -1, device=value.device)
    return torch.topk(key, k).indices


def _inputs(experts, seed, tokens=20_000):
    import torch
    gen = torch.Generator(device="cuda").manual_seed(seed)
    x = (2.0 * torch.randn(tokens, experts, generator=gen, device="cuda")).bfloat16()
    return x, 1.0 + 0.002 * torch.rand(experts, generator=gen, device="cuda")


@pytest.mark.parametrize("experts", [64, 160, 256, 500])
def test_softmax_choice_does_not_depend_on_the_variant(lib, experts):
    """As many experts as a row of lanes takes and one more, groups that make
    no difference, two types of the same logits, strided rows."""
    import torch
    x, bias = _inputs(experts, experts)
    w, idx = lib.lapsum_route_forward(x, 8, bias=bias)
    more = lib.lapsum_route_forward(x, 9, bias=bias)
    assert torch.equal(idx, more[1][:, :8]) and torch.equal(w, more[0][:, :8])
    wide = lib.lapsum_route_forward(x.float(), 8, bias=bias)
    assert torch.equal(idx, wide[1]) and torch.equal(w, wide[0])
    assert torch.equal(idx, lib.lapsum_route_forward(x.float(), 9, bias=bias)[1][:, :8])
    part = torch.cat([x, x[:, :3]], 1)[:, :experts]
    assert torch.equal(idx, lib.lapsum_route_forward(part, 8, bias=bias)[1])


@pytest.mark.parametrize("experts,k", [(64, 8), (256, 8), (256, 12), (500, 4), (1000, 8)])
def test_softmax_choice_is_that_of_the_rounded_sum(lib, experts, k):
    import torch
    for kind in (torch.bfloat16, torch.float32):
        x, bias = _inputs(experts, experts + k)
        x = x.to(kind)
        f = x.float()
        e = torch.exp(f - f.amax(-1, keepdim=True))
        s = e / e.sum(-1, keepdim=True, dtype=torch.float64).float()
        want = _best(s + bias, k)
        w, idx = lib.lapsum_route_forward(x, k, bias=bias)
        assert torch.equal(idx.long(), want)
        assert torch.equal(w, s.gather(1, want))
