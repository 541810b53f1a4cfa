"""Attention where entries or queries are infinite: what the definition gives in float32, for every
type, length of a row and alignment."""
import math

import pytest

from test_gpu_paged import TYPES, _attend, _gen

pytestmark = pytest.mark.gpu


def _close(got, want, lse, size, sums, dim, n, dtype):
    """Finite results within the roundings that test_attend counts, the others equal."""
    import torch
    off = (dim + 6) * 2.0 ** -24 * size + 2.0 ** -22 * (1 + lse.abs())
    terms = 2.0 ** -23 if dtype is torch.float32 else 2.0 ** -16
    room = (2 * off[..., None] + 2 * n * 2.0 ** -24 + terms) * sums + torch.finfo(dtype).eps / 2 * want.abs() + 2.0 ** -25
    finite = torch.isfinite(want)
    assert bool(((got.double() - want).abs() <= room)[finite].all())
    assert got.double()[~finite].nan_to_num(nan=7.0).tolist() == want[~finite].nan_to_num(nan=7.0).tolist()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("dim", [8, 16, 33, 40, 48, 64, 72, 80, 96, 104, 128, 136, 200, 248, 256])
def test_keys_of_score_minus_infinity(lib, dim, dtype):
    """An infinity in the last elements of a key: the key has weight 0, and no other is touched."""
    import torch
    n = 90
    gen = _gen(dim)
    q = torch.randn(2, 4, dim, generator=gen, device="cuda")
    q[..., -3:] = q[..., -3:].abs() + 0.25
    q = q.to(getattr(torch, dtype))
    k, v = (torch.randn(2, 2, n, dim, generator=gen, device="cuda").to(q.dtype) for _ in "kv")
    keep = torch.ones(2, n, dtype=torch.bool, device="cuda")
    for b, at, d in ((0, 0, -1), (0, 17, -2), (0, 89, -3), (1, 40, -1), (1, 63, -1), (1, 64, -2)):
        k[b, :, at, d] = -math.inf
        keep[b, at] = False
    lens = torch.tensor([n, n], dtype=torch.int32, device="cuda")
    want, lse, w, size, sums = _attend(q.double(), k.double(), v.double(), dim ** -0.5, keep)
    y, total, weights = lib.lapsum_cache_attend(q, k, v, lens, lse=True, weights=True)
    _close(y, want, lse, size, sums, dim, n, q.dtype)
    off = (dim + 6) * 2.0 ** -24 * size + 2.0 ** -22 * (1 + lse.abs())
    assert bool(((total.double() - lse).abs() <= off + n * 2.0 ** -24 + 2.0 ** -22).all())
    assert bool(((weights.double() - w).abs() <= (2 * off[..., None] + n * 2.0 ** -23) * w + 2.0 ** -126).all())
    assert not weights[~keep[:, None].expand(2, 4, n)].any()
    k[1, :, :, -1] = -math.inf
    y, total = lib.lapsum_cache_attend(q, k, v, lens, lse=True)
    assert not y[1].any() and bool((total[1] == -math.inf).all()) and bool(torch.isfinite(total[0]).all())


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("dim,n,paged", [(64, 1, False), (64, 50, False), (128, 700, True), (80, 5000, True),
                                         (33, 300, False), (256, 90, True), (8, 40, False), (200, 2100, False)])
def test_infinite_values(lib, dim, n, paged, dtype):
    """A value of weight above 0 gives infinity of its sign, two of both signs NaN, and the other
    dims are what they are without."""
    import torch
    gen = _gen(dim + n)
    q = torch.randn(2, 4, dim, generator=gen, device="cuda").to(getattr(torch, dtype))
    k, v = (torch.randn(2, 2, n, dim, generator=gen, device="cuda").to(q.dtype) for _ in "kv")
    lens = torch.tensor([n, (n + 1) // 2], dtype=torch.int32, device="cuda")
    keep = torch.arange(n, device="cuda") < lens[:, None]
    best = _attend(q.double(), k.double(), v.double(), dim ** -0.5, keep)[2].argmax(-1)
    for b in range(2):
        last = int(lens[b]) - 1
        v[b, 0, int(best[b, 0]), 1] = math.inf          # (the largest weight of a head, a power of two)
        v[b, 0, last, dim - 1] = -math.inf
        v[b, 0, last // 3, 3] = math.inf
        v[b, 1, 0, 0], v[b, 1, last, 0] = math.inf, -math.inf
        v[b, 1, last // 2, 5] = math.nan
        v[b, 1, int(lens[b]):] = math.inf               # (past the length)
    want, lse, _, size, sums = _attend(q.double(), k.double(), torch.where(keep[:, None, :, None], v, 0.0).double(),
                                       dim ** -0.5, keep)
    kw = {}
    if paged:
        slots = 32
        width = -(-n // slots)
        pad = [torch.nn.functional.pad(x, (0, 0, 0, width * slots - n)) for x in (k, v)]
        k, v = (x.view(2, 2, width, slots, dim).transpose(1, 2).reshape(2 * width, 2, slots, dim) for x in pad)
        kw["table"] = torch.arange(2 * width, dtype=torch.int32, device="cuda").view(2, width)
    y, total = lib.lapsum_cache_attend(q, k, v, lens, lse=True, **kw)
    assert bool(torch.isfinite(total).all())
    assert int((want == math.inf).sum()) >= 4 and bool(torch.isnan(want[:, 2:, 5]).all())
    _close(y, want, lse, size, sums, dim, n, q.dtype)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("apart", [5.0, 12.0, 25.0, 60.0])
def test_infinite_values_of_little_weight(lib, apart, dtype):
    """Weights down to e^-60 are numbers above 0 in float32."""
    import torch
    n, dim = 200, 64
    q = torch.zeros(1, 1, dim, device="cuda", dtype=getattr(torch, dtype))
    k, v = (torch.zeros(1, 1, n, dim, device="cuda", dtype=q.dtype) for _ in "kv")
    q[..., 0] = 8.0
    k[0, 0, 137, 0] = apart
    v[0, 0, :, 4] = 2.0
    v[0, 0, 20, 9], v[0, 0, 180, 10] = math.inf, -math.inf
    lens = torch.tensor([n], dtype=torch.int32, device="cuda")
    y = lib.lapsum_cache_attend(q, k, v, lens)[0, 0].float()
    assert y[9] == math.inf and y[10] == -math.inf and abs(float(y[4]) - 2.0) <= 2.0 ** -7
    y[9] = y[10] = y[4] = 0.0
    assert not y.any()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("heads", [2, 16, 20])
def test_infinities_beside_numbers_that_are_none(lib, heads, dtype):
    """One head's query is NaN, one dim's values are NaN, two are infinite now and then, and all of
    the longest sequence: each shows where it belongs."""
    import torch
    n, dim = 900, 96
    gen = _gen(heads)
    q = torch.randn(3, heads, dim, generator=gen, device="cuda").to(getattr(torch, dtype))
    k, v = (torch.randn(3, 1, n, dim, generator=gen, device="cuda").to(q.dtype) for _ in "kv")
    q[:, 1, 7] = math.nan
    v[0, 0, ::50, 2] = math.nan
    v[0, 0, 7::70, 64], v[0, 0, 8::90, 95] = math.inf, -math.inf
    v[0, 0, 33, 10], v[0, 0, 877, 10] = math.inf, -math.inf
    v[1] = math.inf
    lens = torch.tensor([n, n - 1, n - 2], dtype=torch.int32, device="cuda")
    keep = torch.arange(n, device="cuda") < lens[:, None]
    want, lse, _, size, sums = _attend(q.double(), k.double(), v.double(), dim ** -0.5, keep)
    y, total = lib.lapsum_cache_attend(q, k, v, lens, lse=True)
    assert bool(torch.isnan(y[:, 1]).all()) and bool(torch.isnan(total[:, 1]).all())
    rest = [r for r in range(heads) if r != 1]
    _close(y[:, rest], want[:, rest], lse[:, rest], size[:, rest], sums[:, rest], dim, n, q.dtype)


@pytest.mark.parametrize("kind", ["int8", "float8_e4m3fn"])
@pytest.mark.parametrize("dtype", TYPES)
def test_infinite_queries_of_a_cache_in_8_bits(lib, dtype, kind):
    """Scores of -inf all of them give 0 and -inf; the largest finite queries stay finite."""
    import torch
    n, dim = 70, 64
    gen = _gen(1)
    q = torch.randn(1, 3, dim, generator=gen, device="cuda").to(getattr(torch, dtype))
    code = torch.randint(1, 100, (1, 1, n, dim), generator=gen, device="cuda").float()
    scale = torch.full((1, 1, n), 2.0 ** -9, device="cuda")
    q[0, 0, 5] = -math.inf
    q[0, 1], code[..., 7] = 0.0, 1.0       # (its one product, before the scales, is a number)
    q[0, 1, 7] = torch.finfo(q.dtype).max
    code = code.to(getattr(torch, kind))
    lens = torch.tensor([n], dtype=torch.int32, device="cuda")
    y, total, w = lib.lapsum_cache_attend(q, code, code, lens, k_scale=scale, v_scale=scale, scale=2.0 ** -12, lse=True,
                                          weights=True)
    assert not y[0, 0].any() and not w[0, 0].any() and float(total[0, 0]) == -math.inf
    assert bool(torch.isfinite(y[0, 1:]).all()) and bool(torch.isfinite(total[0, 1:]).all())
    x = code.double() * scale.double()[..., None]
    keep = torch.ones(1, n, dtype=torch.bool, device="cuda")
    want, lse, _, size, sums = _attend(q[:, 2:].double(), x, x, 2.0 ** -12, keep)
    _close(y[:, 2:], want, lse, size, sums, dim, n, q.dtype)
