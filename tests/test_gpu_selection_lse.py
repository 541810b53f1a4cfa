"""The log-sum-exp that a beam search's step compares by: rows whose largest
logit stands far above what comes before it, rows that are log-probabilities
already, and one request alone against the same request among others.

The definition rounds lse = log sum e^x to float32 and then each step of
cum + (x - lse), so from lse in float64 the scores follow in float32.  lse's
own error before it is rounded is far below a rounding, so an lse within it of
the middle of two floats may take the other one: a score one spacing off,
and a choice among continuations that a spacing holds."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True, scope="module")
def _leave_no_large_blocks():
    """Tests that count on what the allocator holds follow these."""
    yield
    import torch
    torch.cuda.empty_cache()


REQUESTS, BEAMS, VOCAB = 32, 8, 128_000   # rows enough for parts of several steps


def _rows(kind):
    import torch
    gen = torch.Generator(device="cuda").manual_seed(17)
    rows = REQUESTS * BEAMS
    x = 2.5 * torch.randn(rows, VOCAB, generator=gen, device="cuda")
    at = torch.randint(0, VOCAB, (rows,), generator=gen, device="cuda")
    here = torch.arange(rows, device="cuda")
    if kind == "peaks":            # 20 to 55 above the others' size
        x[here, at] = 20.0 + 35.0 * torch.rand(rows, generator=gen, device="cuda")
    elif kind == "several":        # some of about the same size, at different places
        for q in range(6):
            x[here, (at + 20_011 * q) % VOCAB] = 28.0 + torch.rand(rows, generator=gen, device="cuda")
    elif kind == "far":            # below what a float32 exponential holds, and above it
        x[:, : VOCAB // 2] -= 400.0
        x[here[::2], at[::2]] = 900.0
    elif kind == "logprobs":       # one near 0, the rest near -40
        x = x - 40.0
        x[here, at] = -0.05 * torch.rand(rows, generator=gen, device="cuda")
    elif kind == "normalised":     # what a log-softmax leaves: lse is 0 but for its roundings
        x = torch.log_softmax(4.0 * x.double(), -1).float()
    return x, -20.0 * torch.rand(REQUESTS, BEAMS, generator=gen, device="cuda")


def _values(x, cum):
    """s of every continuation, float32 [requests, beams * vocabulary]."""
    import torch
    lse = torch.cat([torch.logsumexp(r.double(), -1) for r in x.split(16)]).float()
    return (cum.reshape(-1, 1) + (x.float() - lse[:, None])).view(cum.shape[0], -1)


KINDS = ["normal", "peaks", "several", "far", "logprobs", "normalised"]


@pytest.mark.parametrize("dtype", ["float32", "bfloat16", "float16"])
@pytest.mark.parametrize("kind", KINDS)
def test_scores_are_those_of_the_rounded_lse(lib, kind, dtype):
    import torch
    x, cum = _rows(kind)
    x = x.to(getattr(torch, dtype))
    for c in (cum, torch.zeros_like(cum)):
        scores, tokens, parents = lib.lapsum_beam_select(x, c, 16)
        value = _values(x, c)
        want = torch.topk(value, 16).values.cpu().numpy()
        flat = parents.long() * VOCAB + tokens
        got = value.gather(1, flat).cpu().numpy()
        spacing = np.spacing(np.maximum(np.abs(want), np.abs(got)))
        assert np.all(np.abs(scores.cpu().numpy() - got) <= spacing)
        assert np.all(np.abs(got - want) <= spacing)
        off = np.mean(scores.cpu().numpy() != want)
        # one lse in a hundred at the middle of two floats is far more than its error makes
        assert off <= 0.01, off


@pytest.mark.parametrize("kind", KINDS)
def test_a_request_alone_is_the_request_among_others(lib, kind):
    """The rows' parts depend on how many there are; the results do not."""
    import torch
    x, cum = _rows(kind)
    every = lib.lapsum_beam_select(x, cum, 16)
    for b in range(REQUESTS):
        alone = lib.lapsum_beam_select(x[b * BEAMS:(b + 1) * BEAMS], cum[b:b + 1], 16)
        for one, some in zip(alone, every):
            assert torch.equal(one[0], some[b]), b


def test_a_beam_with_infinity_or_nan_offers_nothing_at_any_place(lib):
    """In a part's first step or a later one, beside masked logits."""
    import torch
    x, cum = _rows("normal")
    x[:, 1000:1100] = -float("inf")
    for r, (place, bad) in enumerate([(0, "inf"), (3000, "inf"), (127_999, "inf"), (0, "nan"), (3000, "nan"),
                                      (127_999, "nan"), (5000, "inf"), (9000, "nan")]):
        x[r, place] = float(bad)
    x[7] = -float("inf")
    x[7, 9000] = float("nan")
    scores, tokens, parents = lib.lapsum_beam_select(x, cum, 16)
    assert parents[0].tolist() == [-1] * 16 and tokens[0].tolist() == [-1] * 16
    assert bool((scores[0] == -float("inf")).all()) and bool((parents[1:] >= 0).all())
    half = x.half()
    assert bool((lib.lapsum_beam_select(half, cum, 16)[2][0] == -1).all())
