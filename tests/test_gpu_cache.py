"""A key-value cache of bounded size against the float64 oracle: accumulated
attention weights, what an eviction keeps, and the single-token step.

acc is the float64 sum rounded once, so it is the oracle's to one rounding
(2^-24 relative, and as much again where the oracle's own sum rounds);
selections are made on float32 values that both sides share, so they are equal."""
import numpy as np
import pytest

import oracle.selection_oracle as S

pytestmark = pytest.mark.gpu

DTYPES = ["float32", "bfloat16", "float16"]


def _np64(t):
    return t.detach().double().cpu().numpy()


# ------------------------------------------------------------- accumulate ----
@pytest.mark.parametrize("keys", [1, 3, 64, 255, 511, 513, 1000, 4097, 20_001])
@pytest.mark.parametrize("dtype", DTYPES)
def test_accumulate(lib, keys, dtype):
    import torch
    for batch, heads, kv, queries in ((1, 1, 1, 1), (2, 6, 2, 5), (3, 8, 8, 17), (1, 32, 4, 33)):
        gen = torch.Generator(device="cuda").manual_seed(keys + heads)
        w = torch.rand(batch, heads, queries, keys, generator=gen, device="cuda").pow(4)
        w = w.to(getattr(torch, dtype))
        seen = torch.randint(0, keys + 1, (batch,), generator=gen, device="cuda", dtype=torch.int32)
        seen[0] = keys
        got = lib.lapsum_cache_accumulate(w, kv, seen=seen)
        want = S.accumulate(_np64(w), kv, seen.tolist())
        np.testing.assert_allclose(_np64(got), want, rtol=2.0 ** -23, atol=0)
        old = torch.rand(batch, kv, keys, generator=gen, device="cuda")
        acc = old.clone()
        assert lib.lapsum_cache_accumulate(w, kv, seen=seen, acc=acc) is acc
        np.testing.assert_allclose(_np64(acc), S.accumulate(_np64(w), kv, seen.tolist(), _np64(old)),
                                   rtol=2.0 ** -23, atol=0)
        np.testing.assert_allclose(_np64(lib.lapsum_cache_accumulate(w, kv)),
                                   S.accumulate(_np64(w), kv), rtol=2.0 ** -23, atol=0)


def test_accumulate_reads_nothing_past_the_live_columns(lib):
    """NaN and infinities in the columns after the last, lengths of 0 and past the
    end, and strides of every dimension."""
    import torch
    w = torch.rand(4, 6, 9, 130, device="cuda")
    seen = torch.tensor([0, 1, 77, 500], device="cuda", dtype=torch.int32)
    clean = lib.lapsum_cache_accumulate(w, 3, seen=seen)
    bad = w.clone()
    for b, n in enumerate(seen.tolist()):
        bad[b, :, :, n:] = float("nan") if b % 2 else float("inf")
    assert torch.equal(lib.lapsum_cache_accumulate(bad, 3, seen=seen), clean)
    assert bool((clean[0] == 0).all()) and bool((clean[1, :, 1:] == 0).all())
    acc = torch.full((4, 3, 130), 2.0, device="cuda")
    lib.lapsum_cache_accumulate(bad, 3, seen=seen, acc=acc)
    assert torch.equal(acc, clean + 2.0) or float((acc - clean - 2.0).abs().max()) < 1e-5
    assert bool((acc[0] == 2).all())
    # by other strides: [queries, batch, heads, keys], and a part of a wider row
    turned = w.permute(2, 0, 1, 3).contiguous().permute(1, 2, 0, 3)
    assert torch.equal(lib.lapsum_cache_accumulate(turned, 3, seen=seen), clean)
    wide = torch.rand(4, 6, 9, 137, device="cuda").to(torch.bfloat16)
    part = wide[..., 3:133]
    assert torch.equal(lib.lapsum_cache_accumulate(part, 3), lib.lapsum_cache_accumulate(part.contiguous(), 3))
    last = w.transpose(2, 3).contiguous().transpose(2, 3)       # no dense last dimension
    assert torch.equal(lib.lapsum_cache_accumulate(last, 3, seen=seen), clean)
    one = w[:, :, :1].expand(4, 6, 9, 130)                       # a broadcast of queries
    assert torch.equal(lib.lapsum_cache_accumulate(one, 3), lib.lapsum_cache_accumulate(one.contiguous(), 3))


def test_accumulate_empty(lib):
    import torch
    assert lib.lapsum_cache_accumulate(torch.zeros(0, 4, 3, 5, device="cuda"), 2).shape == (0, 2, 5)
    assert lib.lapsum_cache_accumulate(torch.zeros(2, 4, 3, 0, device="cuda"), 2).shape == (2, 2, 0)
    none = lib.lapsum_cache_accumulate(torch.zeros(2, 4, 0, 5, device="cuda"), 2)
    assert bool((none == 0).all())


# ------------------------------------------------------------------ evict ----
def _cache(seed, batch, kv, slots, dim, dtype="bfloat16"):
    import torch
    gen = torch.Generator(device="cuda").manual_seed(seed)
    dt = getattr(torch, dtype)
    k, v = (torch.randint(-100, 100, (batch, kv, slots, dim), generator=gen, device="cuda").to(dt)
            for _ in range(2))
    acc = torch.rand(batch, kv, slots, generator=gen, device="cuda").pow(6)
    return k, v, acc


def _check_evict(lib, k, v, acc, seen, budget, sink, recent, pos=None):
    import torch
    out = lib.lapsum_cache_evict(k, v, acc, seen, budget, sink=sink, recent=recent, pos=pos)
    batch, kv, slots, dim = k.shape
    accs, seens = acc.cpu().numpy(), seen.tolist()
    at = np.arange(slots)
    for b in range(batch):
        for h in range(kv):
            ps = np.where(at < seens[b], at, -1) if pos is None else pos[b, h].cpu().numpy()
            keep = S.kept_slots(accs[b, h].astype(np.float64), ps, max(0, seens[b]), budget, sink, recent)
            n = len(keep)
            where = (b, h, budget, sink, recent)
            assert out[3][b, h].tolist() == [int(ps[i]) for i in keep] + [-1] * (budget - n), where
            idx = torch.tensor(keep, device="cuda", dtype=torch.long)
            assert torch.equal(out[0][b, h, :n], k[b, h][idx]), where
            assert torch.equal(out[1][b, h, :n], v[b, h][idx]), where
            assert np.array_equal(out[2][b, h, :n].cpu().numpy(), accs[b, h][keep], equal_nan=True)
            assert not out[0][b, h, n:].any() and not out[1][b, h, n:].any() and not out[2][b, h, n:].any()
    return out


@pytest.mark.parametrize("slots", [1, 2, 63, 64, 100, 1024, 1025, 5000, 33_000, 140_001])
def test_evict_sizes(lib, slots):
    import torch
    batch = 3 if slots < 10_000 else 1
    k, v, acc = _cache(slots, batch, 2, slots, 8)
    seen = torch.tensor([slots, slots // 2, 0][:batch], dtype=torch.int32, device="cuda")
    for budget, sink, recent in ((1, 0, 0), (1, 0, 1), (slots // 3 + 2, 1, 1), (slots, 0, 0),
                                 (slots + 5, 4, 1), (slots // 2 + 40, 4, 32)):
        _check_evict(lib, k, v, acc, seen, budget, sink, recent)


@pytest.mark.parametrize("slots", [50, 3000, 40_000])
def test_evict_ties_and_values_that_are_none(lib, slots):
    """Equal sums by the lowest slot; NaN first out, then -inf; both zeros equal."""
    import torch
    k, v, acc = _cache(1, 2, 3, slots, 4)
    gen = torch.Generator(device="cuda").manual_seed(slots)
    acc = torch.randint(0, 3, acc.shape, generator=gen, device="cuda").float()
    acc[0, 0] = 0.0
    acc[0, 1, ::2] = -0.0
    acc[0, 1, 1::2] = 0.0
    acc[0, 2, torch.rand(slots, generator=gen, device="cuda") < 0.5] = float("nan")
    acc[1, 0, ::3] = float("inf")
    acc[1, 0, 1::3] = -float("inf")
    acc[1, 1, ::2] = -float("nan")
    acc[1, 1, 1::2] = torch.finfo(torch.float32).min
    acc[1, 2] = float("nan")
    seen = torch.tensor([slots, slots - 3], dtype=torch.int32, device="cuda")
    for budget, sink, recent in ((7, 2, 3), (slots // 2, 0, 0), (slots - 5, 3, 1), (slots, 0, slots)):
        _check_evict(lib, k, v, acc, seen, budget, sink, recent)


@pytest.mark.parametrize("slots", [32_769, 100_000, 262_144, 300_007])
def test_evict_long_rows_that_a_sample_misleads(lib, slots):
    """Values that the sample's stride meets or misses, sorted rows, rows of few
    values and of one, and budgets from nearly none to nearly all."""
    import torch
    k, v, _ = _cache(7, 1, 8, slots, 2)
    gen = torch.Generator(device="cuda").manual_seed(slots)
    acc = torch.rand(1, 8, slots, generator=gen, device="cuda")
    acc[0, 1] = acc[0, 1].sort()[0]
    acc[0, 2] = acc[0, 2].sort(descending=True)[0]
    acc[0, 3, :] = 0.5
    acc[0, 4] = (acc[0, 4] * 3).floor()
    acc[0, 5, ::slots // 4096] = 10.0 + acc[0, 5, ::slots // 4096]
    acc[0, 6] = acc[0, 6].pow(40)
    acc[0, 7] = -acc[0, 7]
    acc[0, 7, ::5] = float("nan")
    seen = torch.tensor([slots], dtype=torch.int32, device="cuda")
    for budget, sink, recent in ((1, 0, 0), (100, 4, 64), (slots // 30, 4, 64), (slots // 2, 0, 1),
                                 (slots - 7, 3, 4), (slots // 2, slots // 4, slots // 4)):
        _check_evict(lib, k, v, acc, seen, budget, sink, recent)


def test_evict_long_rows_whose_window_ends_between_numbers(lib):
    """The last kept entry among NaN ones, below every number, and among the
    smallest negative numbers, next to zeros: the ends of the sample's bins are
    then no number's key."""
    import torch
    slots = 40_000
    k, v, _ = _cache(8, 1, 4, slots, 2)
    gen = torch.Generator(device="cuda").manual_seed(17)
    order = torch.stack([torch.randperm(slots, generator=gen, device="cuda") for _ in range(4)])
    seen = torch.tensor([slots], dtype=torch.int32, device="cuda")

    # 12000 entries are there, 9000 of them NaN
    acc = torch.rand(1, 4, slots, generator=gen, device="cuda")
    pos = torch.full((1, 4, slots), -1, dtype=torch.int32, device="cuda")
    for h in range(4):
        pos[0, h, order[h, :12_000]] = order[h, :12_000].to(torch.int32)
        acc[0, h, order[h, :9000]] = float("nan")
    acc[0, 1] = -acc[0, 1]
    acc[0, 2, order[2, 9000:9100]] = -float("inf")
    for budget in (11_100, 11_500, 11_990):
        _check_evict(lib, k, v, acc, seen, budget, 0, 0, pos)
    _check_evict(lib, k, v, acc, seen, 11_500, 3, 40, pos)

    # a range whose bins, 2^20 keys wide, end at zero
    low = np.uint32(0xbfffffff).view(np.float32)
    acc[:] = float(low)
    for h in range(4):
        acc[0, h, order[h, 0]] = 1.0
        acc[0, h, order[h, 1:9000]] = torch.rand(8999, generator=gen, device="cuda")
        acc[0, h, order[h, 9000:10_000]] = 0.0
        tiny = torch.randint(1, 1 << 20, (9000,), generator=gen, device="cuda", dtype=torch.int64)
        acc[0, h, order[h, 10_000:19_000]] = (tiny - (1 << 31)).to(torch.int32).view(torch.float32)
    for budget in (12_000, 15_000, 18_000):
        _check_evict(lib, k, v, acc, seen, budget, 0, 0)


@pytest.mark.parametrize("slots", [40, 2000, 36_000])
def test_evict_by_positions(lib, slots):
    """Slots that earlier steps left in any order, with empty ones between."""
    import torch
    k, v, acc = _cache(2, 2, 2, slots, 4)
    gen = torch.Generator(device="cuda").manual_seed(slots)
    pos = torch.stack([torch.randperm(2 * slots, generator=gen, device="cuda")[:slots]
                       for _ in range(4)]).view(2, 2, slots).to(torch.int32)
    pos[:, :, torch.rand(slots, generator=gen, device="cuda") < 0.2] = -1
    seen = torch.full((2,), 2 * slots, dtype=torch.int32, device="cuda")
    for budget, sink, recent in ((10, 3, 4), (slots // 2, 2, slots // 4), (slots, 0, 1)):
        out = _check_evict(lib, k, v, acc, seen, budget, sink, recent, pos)
    pos[:] = -1
    _check_evict(lib, k, v, acc, seen, 9, 1, 1, pos)


@pytest.mark.parametrize("dtype,dim", [("bfloat16", 128), ("float16", 5), ("float32", 80), ("uint8", 3),
                                       ("float32", 1), ("float64", 6), ("bfloat16", 1024)])
def test_evict_types_and_strides(lib, dtype, dim):
    import torch
    k, v, acc = _cache(3, 2, 3, 150, dim, dtype)
    seen = torch.tensor([150, 90], dtype=torch.int32, device="cuda")
    want = _check_evict(lib, k, v, acc, seen, 33, 2, 8)
    k2 = k.permute(0, 2, 1, 3).contiguous().permute(0, 2, 1, 3)       # [batch, slots, heads, dim]
    wide = torch.zeros(2, 3, 200, dim + 1, dtype=v.dtype, device="cuda")
    wide[:, :, 7:157, 1:] = v
    got = lib.lapsum_cache_evict(k2, wide[:, :, 7:157, 1:], acc, seen, 33, sink=2, recent=8)
    for a, b in zip(got, want):
        assert torch.equal(a, b)


def test_evict_offsets_past_32_bits(lib):
    """A cache of more than 2^32 bytes, its kept rows at both ends."""
    import torch
    slots, dim = 70_000, 128
    k = torch.zeros(1, 280, slots, dim, dtype=torch.bfloat16, device="cuda")   # 5 GB
    acc = torch.zeros(1, 280, slots, device="cuda")
    for h in (0, 279):
        acc[0, h, slots - 9] = 1.0
        k[0, h, slots - 9] = h + 1.0
    seen = torch.tensor([slots], dtype=torch.int32, device="cuda")
    out = lib.lapsum_cache_evict(k, k, acc, seen, 2)
    assert out[3][0, 279].tolist() == [0, slots - 9] and bool((out[0][0, 279, 1] == 280).all())
    assert bool((out[1][0, 0, 1] == 1).all()) and bool((out[1][0, 1] == 0).all())


def test_evict_refusals(lib):
    import torch
    k, v, acc = _cache(4, 2, 2, 20, 4)
    seen = torch.tensor([20, 20], dtype=torch.int32, device="cuda")
    for budget, sink, recent in ((0, 0, 0), (-1, 0, 0), (5, 3, 3), (5, -1, 0), (5, 0, -1)):
        with pytest.raises(lib.LapsumError):
            lib.lapsum_cache_evict(k, v, acc, seen, budget, sink=sink, recent=recent)
    for args in ((k.cpu(), v, acc, seen), (k, v[:, :1], acc, seen), (k, v.float(), acc, seen),
                 (k, v, acc.double(), seen), (k, v, acc[:, :, :5], seen), (k, v, acc, seen.long()),
                 (k.transpose(2, 3), v.transpose(2, 3), acc, seen), (k, v, acc, seen[:1])):
        with pytest.raises(ValueError):
            lib.lapsum_cache_evict(*args, 5)
    with pytest.raises(ValueError):
        lib.lapsum_cache_accumulate(torch.zeros(2, 4, 5, device="cuda"), 2)
    with pytest.raises(lib.LapsumError):
        lib.lapsum_cache_accumulate(torch.zeros(2, 4, 1, 5, device="cuda"), 3)
    none = lib.lapsum_cache_evict(k[:0], v[:0], acc[:0], seen[:0], 5)
    assert none[0].shape == (0, 2, 5, 4)


# ------------------------------------------------------------------- step ----
@pytest.mark.parametrize("slots", [1, 2, 5, 64, 130, 1023, 1024, 1025, 4100])
@pytest.mark.parametrize("dtype", DTYPES)
def test_step_by_step(lib, slots, dtype):
    """A cache from empty past full: every token's slot, sum, entry and
    position."""
    import torch
    batch, heads, kv, dim = 2, 6, 2, 5
    gen = torch.Generator(device="cuda").manual_seed(slots)
    dt = getattr(torch, dtype)
    sink, recent = min(2, max(0, slots - 1)), max(1, min(3, slots - 2))
    k = torch.zeros(batch, kv, slots, dim, dtype=dt, device="cuda")
    v = torch.zeros_like(k)
    acc = torch.zeros(batch, kv, slots, device="cuda")
    pos = torch.full((batch, kv, slots), -1, dtype=torch.int32, device="cuda")
    start = 0
    if slots > 200:            # most of it filled beforehand
        start = slots - 3
        pos[:, :, :start] = torch.arange(start, dtype=torch.int32)
        acc[:, :, :start] = torch.rand(start, generator=gen, device="cuda")
    for t in range(start, slots + 6 if slots > 200 else 2 * slots + 3):
        w = torch.rand(batch, heads, slots, generator=gen, device="cuda").to(dt)
        k1, v1 = (torch.randn(batch, kv, dim, generator=gen, device="cuda").to(dt) for _ in range(2))
        seen = torch.full((batch,), t, dtype=torch.int32, device="cuda")
        old = [x.clone() for x in (k, v, acc, pos)]
        if t % 2:              # what empty slots hold of weights is not read
            w.masked_fill_((old[3] < 0).repeat_interleave(heads // kv, 1), float("nan"))
        got = lib.lapsum_cache_step(w, k1, v1, seen, k, v, acc, pos, sink=sink, recent=recent)
        ws, olds = _np64(w), _np64(old[2])
        for b in range(batch):
            for h in range(kv):
                ps = old[3][b, h].cpu().numpy()
                add = np.where(ps >= 0, ws[b].reshape(kv, -1, slots)[h].sum(0), 0.0)
                a = (olds[b, h] + add).astype(np.float32)
                slot = S.step_slot(a.astype(np.float64), ps, t, sink, recent)
                assert int(got[b, h]) == slot, (t, b, h)
                a[slot] = 0.0
                ps = ps.copy()
                ps[slot] = t
                assert np.array_equal(acc[b, h].cpu().numpy(), a)
                assert np.array_equal(pos[b, h].cpu().numpy(), ps)
                old[0][b, h, slot], old[1][b, h, slot] = k1[b, h], v1[b, h]
        assert torch.equal(k, old[0]) and torch.equal(v, old[1])


@pytest.mark.parametrize("slots", [37, 2050])
def test_step_ties_nan_and_strides(lib, slots):
    import torch
    batch, kv, dim = 2, 3, 8
    pos = torch.arange(slots, dtype=torch.int32, device="cuda").repeat(batch, kv, 1)
    acc = torch.ones(batch, kv, slots, device="cuda")
    acc[0, 1, 9], acc[0, 2, 11], acc[0, 2, 8] = float("nan"), -float("inf"), -float("inf")
    acc[1, 0, 20:25] = 0.0
    acc[1, 1, slots - 1] = float("nan")                     # among the last: stays
    acc[1, 2, :4] = -5.0                                    # among the first: stay
    seen = torch.full((batch,), slots, dtype=torch.int32, device="cuda")
    k = torch.zeros(batch, slots, kv, dim, device="cuda").permute(0, 2, 1, 3)
    v = torch.zeros(batch, kv, slots + 9, dim + 3, device="cuda")[:, :, 4:4 + slots, 1:1 + dim]
    w = torch.zeros(batch, kv, 1, slots + 1, device="cuda")[..., 1:]
    k1 = torch.ones(batch, kv, 1, dim, device="cuda")
    got = lib.lapsum_cache_step(w, k1, k1 * 2, seen, k, v, acc, pos, sink=4, recent=5)
    assert got.tolist() == [[4, 9, 8], [20, 4, 4]]
    for b in range(batch):
        for h in range(kv):
            s = int(got[b, h])
            assert bool((k[b, h, s] == 1).all()) and bool((v[b, h, s] == 2).all())
            assert int(pos[b, h, s]) == slots and float(acc[b, h, s]) == 0.0
    assert float(k.sum()) == batch * kv * dim and float(v.sum()) == 2 * batch * kv * dim


def test_step_after_evict_under_graph_capture(lib):
    import torch
    batch, heads, kv, slots, budget, dim = 3, 8, 4, 700, 128, 16
    k, v, acc = _cache(5, batch, kv, slots, dim)
    seen = torch.tensor([700, 60, 500], dtype=torch.int32, device="cuda")
    k, v, acc, pos = lib.lapsum_cache_evict(k, v, acc, seen, budget, sink=4, recent=16)
    w = torch.rand(batch, heads, budget, device="cuda").to(torch.bfloat16)
    k1, v1 = torch.randn(2, batch, kv, dim, device="cuda").to(torch.bfloat16)
    first = [x.clone() for x in (seen, k, v, acc, pos)]
    eager = [x.clone() for x in first]
    slots_of = []
    for _ in range(5):
        slots_of.append(lib.lapsum_cache_step(w, k1, v1, *eager, sink=4, recent=16))
        eager[0] += 1
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        slot = lib.lapsum_cache_step(w, k1, v1, seen, k, v, acc, pos, sink=4, recent=16)
        seen += 1
    for x, y in zip((seen, k, v, acc, pos), first):
        x.copy_(y)
    for i in range(5):
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(slot, slots_of[i])
    for x, y in zip((seen, k, v, acc, pos), eager):
        assert torch.equal(x, y)


def test_step_refusals(lib):
    import torch
    k, v, acc = _cache(6, 2, 2, 10, 4)
    pos = torch.zeros(2, 2, 10, dtype=torch.int32, device="cuda")
    seen = torch.zeros(2, dtype=torch.int32, device="cuda")
    w = torch.zeros(2, 4, 10, device="cuda")
    one = k[:, :, 0].contiguous()
    for sink, recent in ((0, 0), (8, 3), (-1, 1), (0, 11)):
        with pytest.raises(lib.LapsumError):
            lib.lapsum_cache_step(w, one, one, seen, k, v, acc, pos, sink=sink, recent=recent)
    with pytest.raises(lib.LapsumError):
        lib.lapsum_cache_step(w[:, :3], one, one, seen, k, v, acc, pos)
    same = k[:, :, :1].expand(2, 2, 10, 4)
    for args in ((w[:, :, :9], one, one, seen, k, v, acc, pos), (w, one.float(), one, seen, k, v, acc, pos),
                 (w, one, one[:1], seen, k, v, acc, pos), (w, one, one, seen.long(), k, v, acc, pos),
                 (w, one, one, seen, k, v, acc.half(), pos), (w, one, one, seen, k, v, acc, pos.long()),
                 (w.cpu(), one, one, seen, k, v, acc, pos), (w, one, one, seen, same, v, acc, pos)):
        with pytest.raises(ValueError):
            lib.lapsum_cache_step(*args)
