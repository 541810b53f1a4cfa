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
