"""The paged cache against plain float64: entries written, read back, attended to."""
import math

import pytest

pytestmark = pytest.mark.gpu

TYPES = ["float32", "bfloat16", "float16"]
KINDS = ["same", "int8", "float8_e4m3fn"]
MOST = {"int8": 127.0, "float8_e4m3fn": 448.0}


def _torch():
    import torch
    return torch


def _gen(seed):
    return _torch().Generator(device="cuda").manual_seed(seed)


def _bits(x):
    torch = _torch()
    return x.view({1: torch.int8, 2: torch.int16, 4: torch.int32}[x.element_size()])


def _pages(batch, width, slots, seed, spare=2):
    """(pages, table): every page of every sequence, in any order, and some more."""
    torch = _torch()
    pages = batch * width + spare
    table = torch.randperm(pages, generator=_gen(seed), device="cuda")[:batch * width]
    return pages, table.view(batch, width).int().contiguous()


def _quantised(x, kind):
    """Codes and scales by their definition, in float32 on the CPU."""
    torch = _torch()
    x = x.float().cpu()
    most = x.abs().amax(-1)
    odd = ~torch.isfinite(x).all(-1)
    unit = torch.tensor(1.0 / MOST[kind], dtype=torch.float32)
    scale = (most * unit).clamp(min=2.0 ** -126)
    scale[odd] = float("nan")
    y = torch.where(odd[..., None], 0.0, x / scale[..., None])
    code = y.round().to(torch.int8) if kind == "int8" else y.to(torch.float8_e4m3fn)
    return code, scale


def _empty(shape, kind, dtype, fill=7):
    torch = _torch()
    t = torch.full(shape, fill, device="cuda", dtype=torch.int8)
    if kind == "int8":
        return t, torch.full(shape[:3], 0.25, device="cuda")
    if kind == "float8_e4m3fn":
        return t.view(torch.float8_e4m3fn), torch.full(shape[:3], 0.25, device="cuda")
    return t.to(getattr(torch, dtype)), None


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("batch,kv,new,dim,slots,paged", [
    (1, 1, 1, 1, 1, True), (3, 2, 1, 128, 16, True), (2, 3, 37, 80, 24, True), (4, 1, 5, 33, 7, True),
    (2, 2, 300, 256, 64, True), (2, 4, 19, 136, 40, False), (5, 2, 1, 64, 9, False)])
def test_append_and_read(lib, batch, kv, new, dim, slots, paged, dtype, kind):
    torch = _torch()
    gen = _gen(batch + new + dim)
    room = slots if not paged else -(-(new + 20) // slots) * slots
    pages, table = _pages(batch, room // slots, slots, 5) if paged else (batch, None)
    x = [torch.randn(batch, kv, new, dim, generator=gen, device="cuda").to(getattr(torch, dtype)) for _ in "kv"]
    x[0][0, 0, 0] = 0.0
    x[1][-1, -1, -1] *= 2.0 ** -20
    seen = torch.randint(0, 20, (batch,), generator=gen, device="cuda", dtype=torch.int32)
    count = torch.randint(0, new + 1, (batch,), generator=gen, device="cuda", dtype=torch.int32)
    for counts in (None, count):
        cache = [_empty((pages, kv, slots, dim), kind, dtype) for _ in "kv"]
        want = [(c.clone().cpu(), None if s is None else s.clone().cpu()) for c, s in cache]
        lib.lapsum_cache_append(x[0], x[1], seen, cache[0][0], cache[1][0], table=table, count=counts,
                                k_scale=cache[0][1], v_scale=cache[1][1])
        for n in range(2):
            rows = x[n].cpu() if kind == "same" else _quantised(x[n], kind)[0]
            scales = None if kind == "same" else _quantised(x[n], kind)[1]
            for b in range(batch):
                for i in range(new if counts is None else int(counts[b])):
                    at = int(seen[b]) + i
                    if at >= room:
                        continue
                    page = b if table is None else int(table[b, at // slots])
                    _bits(want[n][0])[page, :, at % slots] = _bits(rows)[b, :, i]
                    if scales is not None:
                        want[n][1][page, :, at % slots] = scales[b, :, i]
            assert bool(torch.equal(_bits(cache[n][0].cpu()), _bits(want[n][0])))
            assert scales is None or bool(torch.equal(_bits(cache[n][1].cpu()), _bits(want[n][1])))
        lens = torch.randint(0, room + 1, (batch,), generator=gen, device="cuda", dtype=torch.int32)
        for to in ([dtype] if kind == "same" else TYPES):
            got = lib.lapsum_cache_read(cache[0][0], lens, room + 3, table=table, scale=cache[0][1],
                                        dtype=getattr(torch, to))
            c, s = want[0]
            full = c.float() if s is None else c.float() * s[..., None]
            for b in range(batch):
                line = full[b] if table is None else torch.cat([full[int(p)] for p in table[b]], 1)
                line = torch.nn.functional.pad(line, (0, 0, 0, 3))
                line[:, int(lens[b]):] = 0
                assert bool(torch.equal(_bits(got[b].cpu()), _bits(line.to(getattr(torch, to)))))


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("dim", [40, 128, 200])
def test_many_entries(lib, dim, dtype, kind):
    """Rows in whole workgroups, and every rounding of a few hundred thousand elements."""
    torch = _torch()
    gen = _gen(dim)
    batch, kv, new, slots = 4, 4, 4500, 16
    pages, table = _pages(batch, 282, slots, 1)
    x = torch.randn(2, batch, kv, new, dim, generator=gen, device="cuda").to(getattr(torch, dtype))
    seen = torch.tensor([0, 3, 12, 11], dtype=torch.int32, device="cuda")
    k, ks = _empty((pages, kv, slots, dim), kind, dtype)
    v, vs = _empty((pages, kv, slots, dim), kind, dtype)
    lib.lapsum_cache_append(x[0], x[1], seen, k, v, table=table, k_scale=ks, v_scale=vs)
    for c, s, rows in ((k, ks, x[0]), (v, vs, x[1])):
        want, scale = (rows.cpu(), None) if kind == "same" else _quantised(rows, kind)
        back = lib.lapsum_cache_read(c, seen + new, 4512, table=table, scale=s)
        value = want if scale is None else want.float() * scale[..., None]
        for b in range(batch):
            at = int(seen[b])
            assert bool(torch.equal(_bits(back[b, :, at:at + new].cpu()), _bits(value[b])))
            assert not back[b, :, at + new:].any()


@pytest.mark.parametrize("kind", ["int8", "float8_e4m3fn"])
def test_rows_at_the_ends_of_the_range(lib, kind):
    torch = _torch()
    dim = 72
    x = torch.randn(1, 1, 12, dim, generator=_gen(1), device="cuda")
    x[0, 0, 0] = 0.0
    x[0, 0, 1] = 1e-41
    x[0, 0, 2] *= 1e-38
    x[0, 0, 3] = 3.4e38
    x[0, 0, 4, 5] = float("inf")
    x[0, 0, 5, 71] = float("nan")
    x[0, 0, 6, 0] = -float("inf")
    x[0, 0, 7] = torch.arange(dim, device="cuda") * 0.5 - 17.25      # ties
    x[0, 0, 7, 0] = MOST[kind]
    x[0, 0, 8] = -1.0
    k, ks = _empty((1, 1, 12, dim), kind, None)
    v, vs = _empty((1, 1, 12, dim), kind, None)
    zero = torch.zeros(1, dtype=torch.int32, device="cuda")
    lib.lapsum_cache_append(x, x, zero, k, v, k_scale=ks, v_scale=vs)
    code, scale = _quantised(x, kind)
    assert bool(torch.equal(_bits(k.cpu()), _bits(code))) and bool(torch.equal(_bits(v.cpu()), _bits(code)))
    odd = torch.isnan(scale)
    assert odd[0, 0].tolist() == [i in (4, 5, 6) for i in range(12)]
    assert bool(torch.isnan(ks.cpu()[odd]).all()) and bool(torch.equal(ks.cpu()[~odd], scale[~odd]))
    back = lib.lapsum_cache_read(k, zero + 12, 12, scale=ks)
    assert bool(torch.isnan(back.cpu()[odd]).all()) and bool(torch.isfinite(back.cpu()[~odd]).all())


def test_positions_that_are_not_there(lib):
    """Pages out of range, positions before 0 and past the room: nothing is written, zeros are read."""
    torch = _torch()
    k, v = (torch.zeros(4, 1, 4, 8, device="cuda") for _ in "kv")
    table = torch.tensor([[0, -1, 3], [4, 2, 1 << 30], [1, -7, 1 << 20]], dtype=torch.int32, device="cuda")
    new = torch.ones(3, 1, 40, 8, device="cuda")
    seen = torch.tensor([0, 2, -6], dtype=torch.int32, device="cuda")
    lib.lapsum_cache_append(new, new, seen, k, v, table=table)
    here = k[:, 0, :, 0]
    assert here.tolist() == [[1.0] * 4, [1.0] * 4, [1.0] * 4, [1.0] * 4]
    lib.lapsum_cache_append(new * 0, new * 0, seen + (1 << 30), k, v, table=table)
    lib.lapsum_cache_append(new * 0, new * 0, torch.full_like(seen, 2147483600), k, v, table=table)
    assert bool(k.all()) and bool(v.all())
    lens = torch.tensor([100, 100, -3], dtype=torch.int32, device="cuda")
    got = lib.lapsum_cache_read(k, lens, 15, table=table)[:, 0, :, 0]
    assert got.tolist() == [[1.0] * 4 + [0.0] * 4 + [1.0] * 4 + [0.0] * 3, [0.0] * 4 + [1.0] * 4 + [0.0] * 7,
                            [0.0] * 15]


def _attend(q, k, v, scale, keep):
    """float64 attention [batch, heads, dim] over [batch, kv, room, dim]: outputs, lse,
    weights; and the scores' largest sum of magnitudes."""
    torch = _torch()
    group = q.shape[1] // k.shape[1]
    keep = keep[:, None]
    k = torch.where(keep[..., None], k, 0.0).repeat_interleave(group, 1)
    v = torch.where(keep[..., None], v, 0.0).repeat_interleave(group, 1)
    s = scale * (q[:, :, None] * k).sum(-1)
    size = abs(scale) * (q[:, :, None] * k).abs().sum(-1)
    s = s.masked_fill(~keep, -math.inf)
    lse = torch.logsumexp(s, -1)
    w = torch.exp(s - torch.where(lse == -math.inf, 0.0, lse)[..., None])
    return (w[..., None] * v).sum(2), lse, w, size.amax(-1), (w[..., None] * v.abs()).sum(2)


CASES = [  # batch, heads, kv, dim, slots, width, window
    (1, 1, 1, 1, 1, 1, 0), (1, 4, 4, 64, 16, 3, 0), (3, 8, 2, 128, 16, 20, 0), (2, 6, 2, 80, 24, 9, 0),
    (2, 7, 1, 96, 5, 30, 0), (2, 40, 2, 128, 32, 12, 0), (2, 3, 3, 33, 7, 11, 0), (1, 16, 1, 256, 64, 40, 0),
    (2, 4, 2, 130, 8, 10, 0), (3, 4, 1, 64, 16, 40, 100), (2, 2, 2, 128, 1, 150, 33), (2, 8, 2, 128, 700, 0, 0),
    (3, 4, 2, 48, 37, 0, 5), (1, 2, 1, 128, 128, 40, 0),
]


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("case", CASES)
def test_attend(lib, case, dtype, kind):
    torch = _torch()
    batch, heads, kv, dim, slots, width, window = case
    gen = _gen(sum(case))
    q = (1.5 * torch.randn(batch, heads, dim, generator=gen, device="cuda")).to(getattr(torch, dtype))
    pages, table = _pages(batch, width, slots, 3) if width else (batch, None)
    room = slots * width if width else slots
    lens = torch.randint(1, room + 1, (batch,), generator=gen, device="cuda", dtype=torch.int32)
    lens[0] = room
    if batch > 1:
        lens[-1] = 0 if batch > 2 else 1
    cache = []
    for _ in "kv":
        x = torch.randn(pages, kv, slots, dim, generator=gen, device="cuda")
        if kind == "same":
            cache.append((x.to(q.dtype), None))
        else:
            code, scale = _quantised(x, kind)
            cache.append((code.cuda(), scale.cuda()))
    if table is not None and width > 4:   # a page that is not there, masked like the end
        table[0, 2] = -1
    at = torch.arange(room, device="cuda")
    keep = at < lens[:, None]
    if window:
        keep &= at >= lens[:, None] - window
    flat = []
    for c, s in cache:
        x = c.double() if s is None else c.double() * s.double()[..., None]
        if table is not None:
            x = torch.stack([torch.cat([x[int(p)] for p in row.clamp(min=0)], 1) for row in table])
        flat.append(x)
    if table is not None:
        keep &= (table >= 0).repeat_interleave(slots, 1)
    scale = 0.3 if dim == 64 else None
    by = scale or dim ** -0.5
    want, lse, w, size, sums = _attend(q.double(), *flat, by, keep)
    # what nobody may read into the results: every slot that is no position's holds NaN
    used = torch.zeros(pages, slots, dtype=torch.bool, device="cuda")
    for b in range(batch):
        for p in torch.nonzero(keep[b])[:, 0].tolist():
            used[b if table is None else int(table[b, p // slots]), p % slots] = True
    for n, (c, s) in enumerate(cache):
        if s is None:
            cache[n] = (torch.where(used[:, None, :, None], c, float("nan")), None)
        else:
            cache[n] = (c, torch.where(used[:, None], s, float("nan")))
    got = lib.lapsum_cache_attend(q, cache[0][0], cache[1][0], lens, table=table, k_scale=cache[0][1],
                                  v_scale=cache[1][1], scale=scale, window=window, lse=True, weights=True)
    y, total, weights = got
    assert y.dtype is q.dtype and total.dtype is weights.dtype is torch.float32
    # a score is off by dim + 6 roundings of its magnitudes (products, two scales, powers of two), a
    # weight by that relative and the exponential's; sums of room terms; the weights' own terms
    off = (dim + 6) * 2.0 ** -24 * size + 2.0 ** -22 * (1 + lse.abs().nan_to_num(posinf=0.0, neginf=0.0))
    n = int(lens.clamp(max=room).max())
    assert bool(((total.double() - lse).abs() <= off + n * 2.0 ** -24 + 2.0 ** -22).logical_or(total == lse).all())
    assert bool(((weights.double() - w).abs() <= (2 * off[..., None] + n * 2.0 ** -23) * w + 2.0 ** -126).all())
    terms = 2.0 ** -23 if dtype == "float32" else 2.0 ** -16
    half = torch.finfo(q.dtype).eps / 2
    room_y = (2 * off[..., None] + 2 * n * 2.0 ** -24 + terms) * sums + half * want.abs() + 2.0 ** -25
    assert bool(((y.double() - want).abs() <= room_y).all()), float(((y.double() - want).abs() / room_y).max())
    empty = ~keep.any(-1)
    assert not y[empty].any() and bool((total[empty] == -math.inf).all())
    alone = lib.lapsum_cache_attend(q[:, :, None], cache[0][0], cache[1][0], lens, table=table,
                                    k_scale=cache[0][1], v_scale=cache[1][1], scale=scale, window=window)
    assert alone.shape == (batch, heads, 1, dim) and bool(torch.equal(alone[:, :, 0], y))


@pytest.mark.parametrize("kind", KINDS)
def test_attend_through_strides(lib, kind):
    """A cache stored [pages, slots, kv, dim], queries cut from a larger array."""
    torch = _torch()
    gen = _gen(4)
    x = torch.randn(6, 32, 3, 64, generator=gen, device="cuda")
    base = torch.randn(2, 9, 3, 64, generator=gen, device="cuda").half()
    q = base[:, :, 1]
    c, s = (x.half(), None) if kind == "same" else [t.cuda() for t in _quantised(x, kind)]
    view, dense = c.transpose(1, 2), c.transpose(1, 2).contiguous()
    scale = None if s is None else s.transpose(1, 2).contiguous()
    table = torch.tensor([[3, 1], [5, 0]], dtype=torch.int32, device="cuda")
    lens = torch.tensor([64, 33], dtype=torch.int32, device="cuda")
    kw = {"table": table, "k_scale": scale, "v_scale": scale}
    a = lib.lapsum_cache_attend(q, view, view, lens, **kw)
    b = lib.lapsum_cache_attend(q.contiguous(), dense, dense, lens, **kw)
    assert bool(torch.equal(a, b))
    new = torch.randn(2, 3, 5, 64, generator=gen, device="cuda").half()
    seen = torch.tensor([60, 0], dtype=torch.int32, device="cuda")
    scales = [None if scale is None else scale.clone() for _ in range(2)]
    for x, sc, n in ((view, scales[0], new), (dense, scales[1], new.transpose(1, 2).contiguous().transpose(1, 2))):
        lib.lapsum_cache_append(n, n, seen, x, x, table=table, k_scale=sc, v_scale=sc)
    assert bool(torch.equal(_bits(view.contiguous()), _bits(dense)))
    rows = [lib.lapsum_cache_read(x, lens, 64, table=table, scale=sc) for x, sc in ((view, scales[0]), (dense, scales[1]))]
    assert bool(torch.equal(*rows))


def test_attend_values_that_are_not_numbers(lib):
    """NaN in a key or value that counts reaches the outputs of its head; infinite scores, too."""
    torch = _torch()
    k, v = torch.randn(1, 2, 50, 64, device="cuda"), torch.randn(1, 2, 50, 64, device="cuda")
    q = torch.randn(1, 4, 64, device="cuda")
    lens = torch.tensor([50], dtype=torch.int32, device="cuda")
    v[0, 1, 7, 3] = float("nan")
    y = lib.lapsum_cache_attend(q, k, v, lens)
    assert torch.isnan(y).nonzero().tolist() == [[0, 2, 3], [0, 3, 3]]
    k[0, 0, 49] = float("nan")
    y, lse = lib.lapsum_cache_attend(q, k, v, lens, lse=True)
    assert bool(torch.isnan(y[0, :2]).all()) and torch.isnan(lse).tolist() == [[True, True, False, False]]


def test_attend_large_scores(lib):
    """Scores far apart and far from zero: the running maximum moves in every step."""
    torch = _torch()
    n = 1000
    k = torch.zeros(1, 1, n, 64, device="cuda")
    k[0, 0, :, 0] = torch.arange(n, device="cuda") * 3.0 - 1500.0
    v = torch.randn(1, 1, n, 64, device="cuda")
    q = torch.zeros(1, 3, 64, device="cuda")
    q[0, 0, 0], q[0, 1, 0], q[0, 2, 0] = 8.0, -8.0, 1e-3
    lens = torch.tensor([n], dtype=torch.int32, device="cuda")
    for dtype in (torch.float32, torch.bfloat16, torch.float16):
        kk, vv, qq = k.to(dtype), v.to(dtype), q.to(dtype)
        got, lse, w = lib.lapsum_cache_attend(qq, kk, vv, lens, lse=True, weights=True)
        want, total, ws, _, _ = _attend(qq.double(), kk.double(), vv.double(), 0.125, torch.ones(1, n, dtype=torch.bool,
                                                                                                 device="cuda"))
        # scores up to 1.5e3 in float32: 2^-24 of that, three times
        assert float((lse.double() - total).abs().max()) < 1500 * 3 * 2.0 ** -24 + 1e-5
        assert float((w.double() - ws).abs().max()) < 1500 * 6 * 2.0 ** -24 + 1e-5
        assert float((got.double() - want).abs().max()) < 4 * (1500 * 6 * 2.0 ** -24 + torch.finfo(dtype).eps)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("scale", [-0.4, 0.0, 1e-30])
def test_attend_scales(lib, scale, kind):
    """Scores that fall as the products grow, and scores that are all the same."""
    torch = _torch()
    gen = _gen(6)
    q = torch.randn(2, 6, 96, generator=gen, device="cuda")
    lens = torch.tensor([70, 3], dtype=torch.int32, device="cuda")
    x = torch.randn(2, 2, 70, 96, generator=gen, device="cuda")
    c, s = (x, None) if kind == "same" else [t.cuda() for t in _quantised(x, kind)]
    full = c.double() if s is None else c.double() * s.double()[..., None]
    got, lse, w = lib.lapsum_cache_attend(q, c, c, lens, k_scale=s, v_scale=s, scale=scale, lse=True, weights=True)
    keep = torch.arange(70, device="cuda") < lens[:, None]
    want, total, ws, _, _ = _attend(q.double(), full, full, scale, keep)
    # scores below 50 in float32, sums of 96 products: 200 roundings of it at most
    for a, b in ((got, want), (lse, total), (w, ws)):
        assert float((a.double() - b).abs().max()) < 50 * 200 * 2.0 ** -24


def test_weights_feed_the_bounded_cache(lib):
    """evict, attend with weights, step: as the plain sums have it."""
    torch = _torch()
    gen = _gen(8)
    r = lambda *s: torch.randn(*s, generator=gen, device="cuda")  # noqa: E731
    k, v, acc = r(2, 2, 60, 64).half(), r(2, 2, 60, 64).half(), torch.rand(2, 2, 60, generator=gen, device="cuda")
    seen = torch.tensor([60, 13], dtype=torch.int32, device="cuda")
    k, v, acc, pos = lib.lapsum_cache_evict(k, v, acc, seen, 20, sink=2, recent=4)
    live = torch.minimum(seen, torch.full_like(seen, 20))
    for _ in range(9):
        q = r(2, 4, 64).half()
        y, w = lib.lapsum_cache_attend(q, k, v, live, weights=True)
        before = acc.clone()
        slot = lib.lapsum_cache_step(w, r(2, 2, 64).half(), r(2, 2, 64).half(), seen, k, v, acc, pos, sink=2, recent=4)
        want = before.double() + w.double().view(2, 2, 2, 20).sum(2)
        want.scatter_(-1, slot.long()[..., None], 0.0)
        assert float((acc.double() - want).abs().max()) < 1e-6
        seen += 1
        live = torch.minimum(live + 1, torch.full_like(live, 20))
        assert bool(((pos >= 0).sum(-1) == live[:, None]).all())


def test_long_cache_past_32_bits(lib):
    """A cache of more than 2^32 elements: the last pages are found."""
    torch = _torch()
    pages, slots, dim = 132, 1 << 18, 128
    k = torch.zeros(pages, 1, slots, dim, dtype=torch.int8, device="cuda")
    scale = torch.ones(pages, 1, slots, device="cuda")
    table = torch.tensor([[131, 130]], dtype=torch.int32, device="cuda")
    new = torch.randn(1, 1, 3, dim, device="cuda").bfloat16()
    seen = torch.tensor([slots - 1], dtype=torch.int32, device="cuda")
    lib.lapsum_cache_append(new, new, seen, k, k, table=table, k_scale=scale, v_scale=scale)
    code, s = _quantised(new, "int8")
    assert bool(torch.equal(k[131, 0, -1].cpu(), code[0, 0, 0])) and bool(torch.equal(k[130, 0, :2].cpu(), code[0, 0, 1:]))
    q = torch.randn(1, 2, dim, device="cuda").bfloat16()
    lens = torch.tensor([slots + 2], dtype=torch.int32, device="cuda")
    y = lib.lapsum_cache_attend(q, k, k, lens, table=table, k_scale=scale, v_scale=scale, window=3)
    x = (code.double() * s.double()[..., None]).cuda()
    want = _attend(q.double(), x, x, dim ** -0.5, torch.ones(1, 3, dtype=torch.bool, device="cuda"))[0]
    assert float((y.double() - want).abs().max()) < 0.01
    got = lib.lapsum_cache_read(k, lens, slots + 2, table=table, scale=scale, dtype=torch.bfloat16)
    assert bool(torch.equal(got[0, 0, -3:], x[0, 0].float().bfloat16()))


def test_captured_and_replayed(lib):
    """Two graphs of the decode step, replayed in turn with eager work between."""
    torch = _torch()
    gen = _gen(2)
    r = lambda *s: torch.randn(*s, generator=gen, device="cuda")  # noqa: E731
    pages, table = _pages(3, 20, 16, 9)
    states = []
    for n in range(2):
        k, v = (torch.zeros(pages, 2, 16, 128, dtype=torch.int8, device="cuda") for _ in "kv")
        ks, vs = (torch.ones(pages, 2, 16, device="cuda") for _ in "kv")
        states.append({"k": k, "v": v, "ks": ks, "vs": vs, "q": r(3, 8, 128).bfloat16(), "new": r(3, 2, 128).bfloat16(),
                       "seen": torch.tensor([0, 100, 250], dtype=torch.int32, device="cuda")})

    def step(s):
        lib.lapsum_cache_append(s["new"], s["new"] * 0.5, s["seen"], s["k"], s["v"], table=table, k_scale=s["ks"],
                                v_scale=s["vs"])
        s["seen"] += 1
        return lib.lapsum_cache_attend(s["q"], s["k"], s["v"], s["seen"], table=table, k_scale=s["ks"],
                                       v_scale=s["vs"], lse=True)

    spare = [{n: t.clone() for n, t in s.items()} for s in states]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step({n: t.clone() for n, t in states[0].items()})
    torch.cuda.current_stream().wait_stream(side)
    graphs = []
    for s in states:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            held = step(s)
        graphs.append((g, held))
    for turn in range(5):
        for n in (0, 1, 1):
            for name in ("q", "new"):
                states[n][name].copy_(r(*states[n][name].shape))
                spare[n][name].copy_(states[n][name])
            graphs[n][0].replay()
            torch.cuda.synchronize()
            for a, b in zip(graphs[n][1], step(spare[n])):
                assert bool(torch.equal(a, b))


def test_refusals(lib):
    torch = _torch()
    k, v = (torch.zeros(4, 2, 8, 64, device="cuda") for _ in "kv")
    new = torch.zeros(2, 2, 1, 64, device="cuda")
    seen = torch.zeros(2, dtype=torch.int32, device="cuda")
    table = torch.zeros(2, 2, dtype=torch.int32, device="cuda")
    scale = torch.ones(4, 2, 8, device="cuda")
    q = torch.zeros(2, 4, 64, device="cuda")
    one = {"k_new": new, "v_new": new, "seen": seen, "k": k, "v": v, "table": table}
    for bad in (dict(k_new=new.half()), dict(k_new=new.half(), v_new=new.half()), dict(seen=seen.long()),
                dict(table=table[:1]), dict(table=table.long()), dict(k=k[..., ::2]), dict(k=k[:3]),
                dict(k_scale=scale), dict(k=k.to(torch.int8), v=v.to(torch.int8)), dict(count=seen[:1]),
                dict(k=k[:1].expand(4, 2, 8, 64)), dict(k_new=new[:, :1]), dict(seen=seen.cpu()),
                dict(k=torch.zeros(4, 2, 8, 64, device="cuda", requires_grad=True))):
        with pytest.raises((ValueError, RuntimeError)):
            lib.lapsum_cache_append(**{**one, **bad})
    with pytest.raises(lib.LapsumError):      # more sequences than rows of a cache without a table
        lib.lapsum_cache_append(torch.zeros(5, 2, 1, 64, device="cuda"), torch.zeros(5, 2, 1, 64, device="cuda"),
                                torch.zeros(5, dtype=torch.int32, device="cuda"), k, v)
    wide = torch.zeros(4, 2, 8, 264, device="cuda")
    with pytest.raises(lib.LapsumError):
        lib.lapsum_cache_read(wide, seen, 8)
    with pytest.raises(lib.LapsumError):
        lib.lapsum_cache_read(k, seen, -1)
    with pytest.raises(ValueError):
        lib.lapsum_cache_read(k, seen, 8, dtype=torch.float16)
    two = {"q": q, "k": k, "v": v, "lens": seen, "table": table}
    for bad in (dict(q=q.half()), dict(q=q[:, :3]), dict(q=q[..., :32]), dict(lens=seen[:1]), dict(scale=math.inf),
                dict(scale=math.nan), dict(v=v.half()), dict(v=v[:, :, :4]), dict(q=q.double()), dict(window=-1)):
        with pytest.raises((ValueError, RuntimeError)):
            lib.lapsum_cache_attend(**{**two, **bad})


def test_lengths_and_sizes_of_zero(lib):
    torch = _torch()
    k, v = (torch.full((2, 2, 8, 64), float("nan"), device="cuda") for _ in "kv")
    none = torch.zeros(0, dtype=torch.int32, device="cuda")
    zero = torch.zeros(2, dtype=torch.int32, device="cuda")
    q = torch.randn(2, 4, 64, device="cuda")
    y, lse, w = lib.lapsum_cache_attend(q, k, v, zero, lse=True, weights=True)
    assert not y.any() and not w.any() and bool((lse == -math.inf).all())
    y = lib.lapsum_cache_attend(q, k, v, zero + 8, table=torch.zeros(2, 0, dtype=torch.int32, device="cuda"))
    assert not y.any()
    assert lib.lapsum_cache_attend(q[:0], k, v, none).shape == (0, 4, 64)
    assert lib.lapsum_cache_read(k, none, 5).shape == (0, 2, 5, 64)
    assert lib.lapsum_cache_read(k, zero + 8, 0).shape == (2, 2, 0, 64)
    lib.lapsum_cache_append(q[:0, :2], q[:0, :2], none, k, v)
    lib.lapsum_cache_append(q[:, :2, None][:, :, :0], q[:, :2, None][:, :, :0], zero, k, v)
    assert bool(torch.isnan(k).all())
