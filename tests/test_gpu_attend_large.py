"""Attention of many sequences over one cache of many slots: shares past 32 bits."""
import pytest

from test_gpu_paged import _attend, _gen

pytestmark = pytest.mark.gpu


def test_many_sequences_on_one_long_cache(lib):
    import torch
    batch, slots, dim, most = 1 << 15, 1 << 26, 8, 300
    gen = _gen(1)
    q = torch.randn(batch, 1, dim, generator=gen, device="cuda").bfloat16()
    k, v = (torch.zeros(1, 1, slots, dim, device="cuda", dtype=torch.bfloat16) for _ in "kv")
    k[..., :most, :], v[..., :most, :] = (torch.randn(most, dim, generator=gen, device="cuda") for _ in "kv")
    lens = torch.randint(0, most + 1, (batch,), generator=gen, device="cuda", dtype=torch.int32)
    y, lse = lib.lapsum_cache_attend(q, k.expand(batch, -1, -1, -1), v.expand(batch, -1, -1, -1), lens, lse=True)
    for b0 in range(0, batch, 4096):
        at = slice(b0, b0 + 4096)
        keep = torch.arange(most, device="cuda") < lens[at, None]
        kk, vv = (x[:, :, :most].double().expand(4096, -1, -1, -1) for x in (k, v))
        want, total, _, size, sums = _attend(q[at].double(), kk, vv, dim ** -0.5, keep)
        off = (dim + 6) * 2.0 ** -24 * size + 2.0 ** -22 * (1 + total.abs().nan_to_num(neginf=0.0))
        room = (2 * off[..., None] + 2 * most * 2.0 ** -24 + 2.0 ** -16) * sums + 2.0 ** -8 * want.abs() + 2.0 ** -25
        assert bool(((y[at].double() - want).abs() <= room).all())
        assert bool(((lse[at].double() - total).abs() <= off + most * 2.0 ** -24 + 2.0 ** -22).logical_or(
            lse[at] == total).all())
