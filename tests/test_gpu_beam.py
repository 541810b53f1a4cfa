"""A beam search's step against the float64 oracle: sizes from one token to a
large vocabulary, types, odd strides, masks, beams that offer nothing, ties
within and across beams, and the reordering of states.

Tolerance of a score: three float32 roundings of numbers of the size of
cum, x and lse, 2^-24 each, and lse's own (below 2^-24 of it): 4e-7 of their sum."""
import numpy as np
import pytest

import oracle.selection_oracle as S

pytestmark = pytest.mark.gpu

DTYPES = ["float32", "bfloat16", "float16"]


def _np64(t):
    return t.detach().double().cpu().numpy()


def _logits(seed, rows, vocab, dtype, spread=2.5):
    import torch
    gen = torch.Generator(device="cuda").manual_seed(seed)
    return (spread * torch.randn(rows, vocab, generator=gen, device="cuda")).to(getattr(torch, dtype))


def _check(x, cum, num, out):
    scores, tokens, parents = (t.cpu().numpy() for t in out)
    cums = cum.cpu().numpy()
    batch, beams = cums.shape
    xs = _np64(x).reshape(batch, beams, -1)
    for b in range(batch):
        s = S.beam_scores(xs[b], cums[b])
        ref = S.best(s.reshape(-1), num)
        n = len(ref)
        assert np.all(tokens[b, n:] == -1) and np.all(parents[b, n:] == -1)
        assert np.all(scores[b, n:] == -np.inf)
        pairs = list(zip(parents[b, :n].tolist(), tokens[b, :n].tolist()))
        assert len(set(pairs)) == n
        got = np.array([s[w, v] for w, v in pairs])
        want = s.reshape(-1)[ref]
        size = np.array([abs(cums[b][w]) + 2 * abs(xs[b][w, v]) + abs(s[w, v]) for w, v in pairs])
        tol = 4e-7 * (size + 1.0)
        assert np.all(np.abs(scores[b, :n] - got) <= tol), (b, scores[b], got)
        assert np.all(np.abs(got - want) <= 2 * tol), (b, got, want)


@pytest.mark.parametrize("vocab", [1, 2, 5, 63, 64, 65, 1000, 2048, 2049, 8191, 32001, 100_003])
@pytest.mark.parametrize("dtype", DTYPES)
def test_beam_select_sizes(lib, vocab, dtype):
    import torch
    for batch, beams, num in ((1, 1, 1), (1, 4, 8), (3, 5, 5), (2, 16, 32)):
        if batch * beams * vocab > 2_000_000:
            continue
        x = _logits(vocab + beams, batch * beams, vocab, dtype)
        cum = -10.0 * torch.rand(batch, beams, device="cuda")
        _check(x, cum, num, lib.lapsum_beam_select(x, cum, num))


@pytest.mark.parametrize("dtype", DTYPES)
def test_beam_select_many_rows_and_three_dimensions(lib, dtype):
    import torch
    x = _logits(1, 40 * 7, 3001, dtype)
    cum = -30.0 * torch.rand(40, 7, device="cuda") - 50.0
    out = lib.lapsum_beam_select(x, cum, 14)
    _check(x, cum, 14, out)
    for a, b in zip(out, lib.lapsum_beam_select(x.view(40, 7, 3001), cum, 14)):
        assert torch.equal(a, b)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("vocab,pad", [(4000, 96), (4001, 7), (333, 1)])
def test_beam_select_strided_rows(lib, dtype, vocab, pad):
    """Padded vocabularies at any alignment: what lies past a row is not read."""
    import torch
    wide = _logits(pad, 12, vocab + pad, dtype)
    wide[:, vocab:] = 1000.0
    view = wide[:, :vocab]
    cum = -torch.rand(3, 4, device="cuda")
    out = lib.lapsum_beam_select(view, cum, 8)
    for a, b in zip(out, lib.lapsum_beam_select(view.contiguous(), cum, 8)):
        assert torch.equal(a, b)
    shifted = wide[:, pad:]
    for a, b in zip(lib.lapsum_beam_select(shifted, cum, 8),
                    lib.lapsum_beam_select(shifted.contiguous(), cum, 8)):
        assert torch.equal(a, b)
    _check(view, cum, 8, out)


@pytest.mark.parametrize("vocab", [7, 2500, 20_000])
def test_beam_select_first_step_masks_and_dead_beams(lib, vocab):
    import torch
    inf, nan = float("inf"), float("nan")
    x = _logits(2, 8 * 4, vocab, "float32")
    x[:, 1] = -inf
    cum = -5.0 * torch.rand(8, 4, device="cuda")
    cum[0] = torch.tensor([0.0, -inf, -inf, -inf])       # the first step
    cum[1, 2] = nan
    x[2 * 4 + 1] = -inf                                   # a beam with every token masked
    x[3 * 4 + 1, 3] = nan                                 # and beams that offer nothing
    x[3 * 4 + 2, 0] = inf
    x[4 * 4:5 * 4, 2:] = -inf                             # one token left each
    x[5 * 4:6 * 4] = -inf                                 # a request without any
    cum[6] = torch.tensor([-inf] * 4)
    x[7 * 4] = torch.finfo(torch.float32).min             # masked by the lowest value
    _check(x, cum, 8, lib.lapsum_beam_select(x, cum, 8))
    out = lib.lapsum_beam_select(x, cum, 8)
    assert out[2][0].unique().tolist() == ([0] if vocab > 9 else [-1, 0])
    for b in (5, 6):
        assert (out[0][b] == -inf).all() and (out[1][b] == -1).all() and (out[2][b] == -1).all()
    assert sorted(out[2][4, :4].tolist()) == [0, 1, 2, 3] and (out[1][4, :4] == 0).all()


@pytest.mark.parametrize("vocab", [40, 3000, 50_001])
@pytest.mark.parametrize("dtype", DTYPES)
def test_beam_select_ties_go_to_the_lowest_index(lib, vocab, dtype):
    """Equal logits in equal beams: the order is that of beam * vocab + token."""
    import torch
    one = torch.zeros(4, vocab, device="cuda", dtype=getattr(torch, dtype))
    cum = torch.full((1, 4), -2.0, device="cuda")
    s, t, p = lib.lapsum_beam_select(one, cum, 16)
    assert t.tolist() == [list(range(16))] and p.tolist() == [[0] * 16]
    row = torch.randint(0, 3, (vocab,), device="cuda").to(one.dtype)
    s, t, p = lib.lapsum_beam_select(row.expand(4, vocab).contiguous(), cum, 32)
    top = torch.nonzero(row == row.max()).reshape(-1)
    flat = torch.cat([top + w * vocab for w in range(4)])[:32]
    n = flat.numel()
    assert (p.long() * vocab + t)[0, :n].tolist() == flat.tolist()


@pytest.mark.parametrize("vocab", [300, 5000, 30_000])
def test_beam_select_scores_that_round_to_one_value(lib, vocab):
    """A score far from 0 holds few bits: many continuations are equal in
    float32, and the index decides among them, in beams at the lowest float too."""
    import torch
    low = torch.finfo(torch.float32).min
    for cums in ([-1e8, -1e8, -1e8], [-3e7, -2.9e7, -1e8], [low, low, low], [low, -1e8, low],
                 [low, -float("inf"), low]):
        x = _logits(vocab, 3, vocab, "float32")
        cum = torch.tensor([cums], device="cuda")
        s, t, p = lib.lapsum_beam_select(x, cum, 12)
        lse = np.array([np.log(np.exp(r).sum()) for r in _np64(x)]).astype(np.float32)
        xs = x.cpu().numpy()
        value = np.array(cums, np.float32)[:, None] + (xs - lse[:, None])
        ref = S.best(value.astype(np.float64).reshape(-1), 12)
        assert (p.long() * vocab + t)[0].tolist() == ref, cums
        assert s[0].tolist() == value.reshape(-1)[ref].tolist()
    # fewer candidates in the live beam than wanted: the dead ones follow
    x = _logits(1, 2, 3, "float32")
    cum = torch.tensor([[low, -1.0]], device="cuda")
    s, t, p = lib.lapsum_beam_select(x, cum, 5)
    assert p.tolist() == [[1, 1, 1, 0, 0]] and t[0, 3:].tolist() == [0, 1]


def test_beam_select_rising_and_extreme_logits(lib):
    """Every logit above all before it, steps of the reference exponent, and
    sums of one term."""
    import torch
    v = 20_000
    up = torch.arange(v, device="cuda", dtype=torch.float32)
    x = torch.stack([up, 0.01 * up, -up, 1000.0 * (up == 5000) - 500.0, up * 1e30, up.flip(0) * 0.3])
    cum = torch.zeros(6, 1, device="cuda")
    out = lib.lapsum_beam_select(x, cum, 10)
    _check(x, cum, 10, out)
    assert out[1][0].tolist() == list(range(v - 1, v - 11, -1))


@pytest.mark.parametrize("dtype", DTYPES)
def test_beam_select_references_that_move(lib, dtype):
    """Parts of a row that are masked, far below or far above the rest, at the
    types' ends, in every order."""
    import torch
    v = 12_000
    big = 6e4 if dtype == "float16" else 3e38
    x = _logits(9, 12, v, dtype, 1.0)
    x[0, :5000] = -float("inf")
    x[0, 5000:] -= 500.0
    x[1, 4096:] -= 300.0
    x[2, :4096] -= 300.0
    x[3, :6000] = -big
    x[4, 6000:] = -big
    x[5, 7000] = 300.0
    x[6, :] = -big
    x[6, 9000] = -big / 2
    x[7, 2047:2049] = 200.0
    x[8, :] = -float("inf")
    x[8, 11_999] = -700.0
    x[9, ::2048] += 90.0
    x[10] *= 1000.0
    x[11, 100] = big
    cum = -torch.rand(12, 1, device="cuda")
    for num in (1, 7, 32):
        _check(x, cum, num, lib.lapsum_beam_select(x, cum, num))


def test_beam_select_of_a_long_row(lib):
    """Steps of more than one turn of the finish, in several beams."""
    import torch
    v = 3_000_001
    x = _logits(4, 2, v, "bfloat16")
    cum = torch.tensor([[-1.0, -1.5]], device="cuda")
    _check(x, cum, 16, lib.lapsum_beam_select(x, cum, 16))
    flat = torch.zeros(2, v, dtype=torch.bfloat16, device="cuda")
    flat[1, 2_999_000] = 1.0
    s, t, p = lib.lapsum_beam_select(flat, torch.zeros(1, 2, device="cuda"), 20)
    assert t[0].tolist() == [2_999_000, *range(19)] and p[0].tolist() == [1] + [0] * 19


def test_beam_select_under_graph_capture(lib):
    import torch
    x = _logits(3, 8, 10_001, "float16")
    cum = -torch.rand(2, 4, device="cuda")
    states = [torch.randn(8, 2, 50, 16, device="cuda")]
    outs = [torch.empty_like(states[0])]
    ws = torch.empty(lib.lapsum_beam_select_workspace_size(2, 4, 10_001, 8), dtype=torch.uint8,
                     device="cuda")
    lib.lapsum_beam_select(x, cum, 8, workspace=ws)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = lib.lapsum_beam_select(x, cum, 8, workspace=ws)
        lib.lapsum_beam_reorder(states, out[2][:, :4], length=37, out=outs)
    for i in range(4):
        x.copy_(_logits(30 + i, 8, 10_001, "float16"))
        outs[0].zero_()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        want = lib.lapsum_beam_select(x, cum, 8)
        for a, b in zip(out, want):
            assert torch.equal(a, b)
        row = (want[2][:, :4] + 4 * torch.arange(2, device="cuda")[:, None]).reshape(-1).long()
        assert torch.equal(outs[0][:, :, :37], states[0][row][:, :, :37])
        assert bool((outs[0][:, :, 37:] == 0).all())


def test_beam_select_refusals(lib):
    import torch
    x, cum = torch.zeros(8, 20, device="cuda"), torch.zeros(2, 4, device="cuda")
    for num in (0, 33, -1):
        with pytest.raises(lib.LapsumError):
            lib.lapsum_beam_select(x, cum, num)
    with pytest.raises(lib.LapsumError):
        lib.lapsum_beam_select(torch.zeros(33, 4, device="cuda"), torch.zeros(1, 33, device="cuda"), 2)
    for a, c in ((x.cpu(), cum), (x, cum.double()), (x[:7], cum), (x.double(), cum), (x, cum[0]),
                 (x, cum.t().contiguous().t())):
        with pytest.raises(ValueError):
            lib.lapsum_beam_select(a, c, 2)
    s, t, p = lib.lapsum_beam_select(x[:0], cum[:0], 3)
    assert s.shape == (0, 3)


# ---------------------------------------------------------------- reorder ----
@pytest.mark.parametrize("beams", [1, 2, 4, 7, 16, 31, 32])
@pytest.mark.parametrize("dtype,dim", [("bfloat16", 64), ("float32", 3), ("float16", 5), ("uint8", 7),
                                       ("bfloat16", 80), ("float64", 4)])
def test_beam_reorder(lib, beams, dtype, dim):
    import torch
    batch, heads, room = 3, 2, 21
    gen = torch.Generator(device="cuda").manual_seed(beams)
    dt = getattr(torch, dtype)
    base = [torch.randint(0, 200, (batch * beams, heads, room, dim), generator=gen, device="cuda").to(dt)
            for _ in range(3)]
    parents = torch.randint(0, beams, (batch, beams), generator=gen, device="cuda", dtype=torch.int32)
    parents[1] = torch.arange(beams, dtype=torch.int32).flip(0)       # a permutation
    parents[2] = torch.arange(beams, dtype=torch.int32)               # nothing moves
    row = (parents + beams * torch.arange(batch, device="cuda")[:, None]).reshape(-1).long()
    for length in (None, 0, 1, 13, 21):
        n = room if length is None else length
        want = []
        for t in base:
            w = t.clone()
            w[:, :, :n] = t[row][:, :, :n]
            want.append(w)
        inplace = [t.clone() for t in base]
        assert lib.lapsum_beam_reorder(inplace, parents, length=length)[0] is inplace[0]
        other = [torch.full_like(t, 9) for t in base]
        lib.lapsum_beam_reorder(base, parents, length=length, out=other)
        for a, b, w, t in zip(inplace, other, want, base):
            assert torch.equal(a, w)
            assert torch.equal(b[:, :, :n], w[:, :, :n]) and bool((b[:, :, n:] == 9).all())


def test_beam_reorder_of_many_states_and_plain_rows(lib):
    """More states than a launch takes, of different shapes, with parents out
    of a wider tensor; parents that are none leave a row."""
    import torch
    batch, beams = 2, 4
    states = [torch.randn(8, 5 + i, device="cuda") for i in range(37)] + [torch.randn(8, device="cuda")]
    wide = torch.tensor([[3, -1, 0, 0, 7], [1, 1, 9, 2, 7]], device="cuda", dtype=torch.int32)
    src = torch.tensor([3, 1, 0, 0, 5, 5, 6, 6], device="cuda")
    want = [t[src] for t in states]
    lib.lapsum_beam_reorder(states, wide[:, :4])
    for a, b in zip(states, want):
        assert torch.equal(a, b)


def test_beam_reorder_refusals(lib):
    import torch
    p = torch.zeros(2, 3, dtype=torch.int32, device="cuda")
    s = torch.zeros(6, 4, 5, device="cuda")
    for states, parents, kw in (([s[:5]], p, {}), ([s], p.long(), {}), ([s], p, dict(length=5)),
                                ([s[:, 0]], p, dict(length=1)), ([s.cpu()], p, {}),
                                ([s.transpose(1, 2)], p, {}), ([s], p, dict(out=[])),
                                ([s], p, dict(out=[torch.zeros(6, 4, 6, device="cuda")])),
                                ([s], p.t().contiguous().t(), {})):
        with pytest.raises(ValueError):
            lib.lapsum_beam_reorder(states, parents, **kw)
    with pytest.raises(lib.LapsumError):
        lib.lapsum_beam_reorder([torch.zeros(33, 2, device="cuda")],
                                torch.zeros(1, 33, dtype=torch.int32, device="cuda"))
    assert lib.lapsum_beam_reorder([], p) == []
