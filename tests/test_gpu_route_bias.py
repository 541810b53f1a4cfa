"""What the routing compares where a bias takes part, to the last bit: the
softmax's denominator, and groups whose experts' biases have opposite signs.

c = s + bias in float32, from s = e / float32(sum of e) with e = exp(x - max)
for a softmax (the sum formed in 64 bits), s = 1 / (1 + exp(-x)) for a
sigmoid.  The bias is large beside the scores, so that c holds few of their
bits: many experts are equal or a spacing apart, and a bit of s decides."""
import pytest

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True, scope="module")
def _leave_no_large_blocks():
    """Tests that count on what the allocator holds follow these."""
    yield
    import torch
    torch.cuda.empty_cache()


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


@pytest.mark.parametrize("size,masked", [(2, 0), (8, 6), (400, 398)])
@pytest.mark.parametrize("high", [4.0, 64.0, 1000.0])
def test_groups_with_biases_of_opposite_signs(lib, size, masked, high):
    """Two groups, the sum of two experts each, one bias +high and one -high:
    the sum is small, its terms' spacing is not.  In a row of four the second
    group's score is the higher by less than a spacing, mostly the same one (the
    groups are then equal and the first stays); in the others it is clearly lower."""
    import torch
    tokens = 60_000
    gen = torch.Generator(device="cuda").manual_seed(int(high) + size)
    # logits whose scores lie just below the middle of two values that c can have
    step = torch.tensor(high, device="cuda").nextafter(torch.tensor(1e9, device="cuda")) - high
    cells = torch.randint(int(0.15 / float(step)) + 1, int(0.85 / float(step)) + 2, (tokens,), generator=gen,
                          device="cuda")
    middle = (cells.double() + 0.5) * step.double()
    close = torch.rand(tokens, generator=gen, device="cuda").double() * 4e-7
    second = torch.logit(middle - close).float()
    first = torch.logit(middle - 0.25 * step.double()).float()
    # the other three rows: tokens that share a wave are not all looked at again
    second[torch.arange(tokens, device="cuda") % 4 != 1] -= 1.0
    x = torch.full((tokens, 2, size), -float("inf"), device="cuda")
    x[:, 0, masked], x[:, 1, masked] = first, second
    x[:, :, masked + 1] = torch.randn(tokens, 1, generator=gen, device="cuda")
    bias = torch.zeros(2, size, device="cuda")
    bias[:, masked], bias[:, masked + 1] = high, -high
    s = 1.0 / (1.0 + torch.exp(-x))
    c = (s + bias)[:, :, masked:masked + 2]
    score = c.sum(-1)
    stays = (score[:, 1] > score[:, 0]).int()             # the first where they are equal
    assert 0.05 < float((score[:, 0] == score[:, 1]).float().mean())
    w, idx = lib.lapsum_route_forward(x.flatten(1), 2, score="sigmoid", bias=bias.flatten(), groups=2,
                                      topk_groups=1, group_top=2)
    assert torch.equal(idx[:, 0] // size, stays) and torch.equal(idx[:, 1] // size, stays)


@pytest.mark.parametrize("dtype", ["float32", "bfloat16", "float16"])
def test_sigmoid_scores_are_torchs_on_every_value(lib, dtype):
    """The exact score of a routing is 1 / (1 + exp(-x)) as torch rounds it, for
    every float of the type (those of float32 in parts)."""
    import torch
    kind = getattr(torch, dtype)
    bits = 32 if dtype == "float32" else 16
    part = 1 << min(bits, 26)
    for start in range(0, 1 << bits, part):
        raw = torch.arange(start, start + part, device="cuda")
        x = (raw.to(torch.int32).view(kind) if bits == 32 else raw.to(torch.int16).view(kind))
        x = x[x > -float("inf")].clamp_max(torch.finfo(torch.float32).max)
        if not x.numel():
            continue
        w, idx = lib.lapsum_route_forward(x[:, None], 1, score="sigmoid")
        assert bool((idx == 0).all())
        assert torch.equal(w[:, 0], 1.0 / (1.0 + torch.exp(-x.float()))), hex(start)
