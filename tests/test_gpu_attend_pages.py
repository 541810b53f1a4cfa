"""Attention over a cache with pages that are not there: their positions count as masked, and
no others, whatever the size of a page, wherever the pages are missing."""
import math

import pytest

from test_gpu_paged import KINDS, TYPES, _attend, _gen, _pages, _quantised

pytestmark = pytest.mark.gpu


def _inputs(batch, heads, kv, dim, slots, width, dtype, kind, seed):
    """Queries, [codes or entries, scales] of keys and values, the table, and both caches
    as float64 arrays by position."""
    import torch
    gen = _gen(seed)
    q = torch.randn(batch, heads, dim, generator=gen, device="cuda").to(getattr(torch, dtype))
    pages, table = _pages(batch, width, slots, seed)
    caches, lines = [], []
    for _ in "kv":
        x = torch.randn(pages, kv, slots, dim, generator=gen, device="cuda")
        c, s = (x.to(q.dtype), None) if kind == "same" else [t.cuda() for t in _quantised(x, kind)]
        x = c.double() if s is None else c.double() * s.double()[..., None]
        lines.append(torch.stack([torch.cat([x[int(p)] for p in row], 1) for row in table]))
        caches.append((c, s))
    return q, caches, table, lines


def _check(lib, q, caches, table, lens, window, lines, keep):
    import torch
    dim, dtype = q.shape[-1], q.dtype
    y, total, weights = lib.lapsum_cache_attend(q, caches[0][0], caches[1][0], lens, table=table, window=window,
                                                k_scale=caches[0][1], v_scale=caches[1][1], lse=True, weights=True)
    want, lse, w, size, sums = _attend(q.double(), *lines, dim ** -0.5, keep)
    # a score is off by dim + 6 roundings of its magnitudes (products, two scales, powers of two), a
    # weight by that relative and the exponential's; sums of n terms; the weights' own terms
    off = (dim + 6) * 2.0 ** -24 * size + 2.0 ** -22 * (1 + lse.abs().nan_to_num(posinf=0.0, neginf=0.0))
    n = keep.shape[1]
    assert bool(((total.double() - lse).abs() <= off + n * 2.0 ** -24 + 2.0 ** -22).logical_or(total == lse).all())
    assert bool(((weights.double() - w).abs() <= (2 * off[..., None] + n * 2.0 ** -23) * w + 2.0 ** -126).all())
    terms = 2.0 ** -23 if dtype is torch.float32 else 2.0 ** -16
    half = torch.finfo(dtype).eps / 2
    room = (2 * off[..., None] + 2 * n * 2.0 ** -24 + terms) * sums + half * want.abs() + 2.0 ** -25
    assert bool(((y.double() - want).abs() <= room).all()), float(((y.double() - want).abs() / room).max())
    empty = ~keep.any(-1)
    assert not y[empty].any() and bool((total[empty] == -math.inf).all())


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("slots", [8, 16, 24, 32, 48, 64, 80, 96, 112, 144])
def test_pages_that_are_not_there(lib, slots, dtype, kind):
    """Every other page missing, the first or the second on; one in the middle; the last; all but one."""
    import torch
    width = 8
    q, caches, table, lines = _inputs(5, 4, 2, 64, slots, width, dtype, kind, slots)
    table[0, 0::2] = -1
    table[1, 1::2] = 1 << 20
    table[2, 4] = -7
    table[3, -1] = -1
    table[4, :] = -1
    table[4, 5] = 0
    for line, c in zip(lines, caches):     # (the one page of the last sequence is another's)
        x = c[0][0].double() if c[1] is None else c[0][0].double() * c[1][0].double()[..., None]
        line[4, :, 5 * slots:6 * slots] = x
    there = ((table >= 0) & (table < caches[0][0].shape[0])).repeat_interleave(slots, 1)
    at = torch.arange(slots * width, device="cuda")
    for short in (0, 1, slots // 2 + 1):
        lens = torch.full((5,), slots * width - short, dtype=torch.int32, device="cuda")
        _check(lib, q, caches, table, lens, 0, lines, there & (at < lens[:, None]))


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("slots", [16, 32, 48, 80, 112, 144])
def test_window_behind_pages_given_back(lib, slots, dtype, kind):
    """Pages wholly before the window are -1: none of the window's positions is lost with them."""
    import torch
    width, window = 7, 2 * slots + 5
    ends = sorted({window + slots + d for d in (0, 1, 15, 16, 17, 31, 32, 47)} | {7 * slots, 7 * slots - 3, window})
    q, caches, table, lines = _inputs(len(ends), 4, 1, 128, slots, width, dtype, kind, 3 * slots)
    lens = torch.tensor([min(e, slots * width) for e in ends], dtype=torch.int32, device="cuda")
    for b, e in enumerate(lens.tolist()):
        table[b, :max(e - window, 0) // slots] = -1
    at = torch.arange(slots * width, device="cuda")
    keep = (at < lens[:, None]) & (at >= lens[:, None] - window)
    _check(lib, q, caches, table, lens, window, lines, keep)
