"""How the library divides its launches, for sizes up to the largest that its entry points take."""
import ctypes
import itertools
import os

import pytest

import paper_2608_06912_amd as L

pytestmark = pytest.mark.skipif(not os.path.exists(L.LIB_PATH), reason="library not built")


def _attend_plan(batch, heads, kv, room, window):
    """lapsum::attend_plan: (splits of a sequence, keys of a split)."""
    plan = ctypes.CDLL(L.LIB_PATH)["_ZN6lapsum11attend_planElllllPiS0_"]
    plan.argtypes, plan.restype = [ctypes.c_int64] * 5 + [ctypes.POINTER(ctypes.c_int)] * 2, None
    splits, chunk = ctypes.c_int(), ctypes.c_int()
    plan(batch, heads, kv, room, window, ctypes.byref(splits), ctypes.byref(chunk))
    return splits.value, chunk.value


ROOMS = [0, 1, 31, 128, 129, 5000, 1 << 17, (1 << 26) - 1, 1 << 26, (1 << 26) + 1, 1 << 28, (1 << 30) - 7, 1 << 30]


@pytest.mark.parametrize("batch,heads,kv", [(1, 1, 1), (1, 40, 1), (3, 8, 2), (512, 64, 64), (32768, 1, 1),
                                            (65536, 1, 1), (1 << 18, 32, 8), (1 << 23, 1, 1), (1, 1 << 23, 1 << 23),
                                            (1, 1 << 23, 1)])
def test_every_key_is_some_split_s(batch, heads, kv):
    """The splits of a sequence take in its keys, however many there are; in whole steps, in the 32
    bits that they are passed in."""
    for room, window in itertools.product(ROOMS, (0, 1, 100, 4096, 1 << 30, 2147483647)):
        splits, chunk = _attend_plan(batch, heads, kv, room, window)
        assert splits >= 1 and chunk >= 128 and chunk % 128 == 0
        # (a window begins within a step of 32, which belongs to it)
        keys = min(room, window + 31) if window else room
        assert splits * chunk >= keys
        rows = batch * kv * -(-(heads // kv) // 16)
        assert splits == 1 or splits * rows <= 1024 + rows
        assert (L.lapsum_cache_attend_workspace_size(batch, heads, kv, 64, room, window) > 0) == (splits > 1)


# Launches of 2^32 threads or more are refused, by the tiles that would be launched: P is a pointer
# that is never read, as the refusal comes before any HIP call.
INVALID, P = 1, 256


def _strides(*s):
    return (ctypes.c_int64 * 3)(*s)


@pytest.mark.parametrize("dtype,rows,experts,n_in,out,strides", [
    # float32 off the direct way to LDS: tiles of 64 x 64
    (0, 1 << 30, 1, 8, 1, (8, 1, 1)), (0, 1 << 29, 3, 8, 75, (600, 75, 1)),
    (0, 40000, 2048, 3, 405000, (3 * 405000, 405000, 1)), (0, 1 << 28, 1, 7, 200, (1400, 1, 7)),
    # tiles of 128 x 128 and 256 x 256
    (1, 1 << 29, 3, 8, 1 << 10, (1 << 13, 1 << 10, 1)), (2, 1 << 30, 1, 7, 130 * 128, (7 * 130 * 128, 1, 7))])
def test_products_of_too_many_threads(dtype, rows, experts, n_in, out, strides):
    import paper_2608_06912_amd.experts as E
    call = E._load().lapsum_expert_matmul
    assert call(P, dtype, rows, n_in, 0, 1, P, experts, rows, n_in, out, P, _strides(*strides), P, dtype, None) == INVALID


@pytest.mark.parametrize("dtype,experts,n_in,out,strides", [
    # matrices stored the other way round: their lines in memory are tiled as rows, four lines of tiles at once
    (1, 127, 1 << 24, 2, (1 << 25, 1, 1 << 24)), (0, 127, 1 << 24, 3, (3 << 24, 1, 1 << 24)),
    (1, 2048, 1 << 14, 1 << 13, (1 << 27, 1 << 13, 1))])
def test_gradients_of_too_many_threads(dtype, experts, n_in, out, strides):
    import paper_2608_06912_amd.experts as E
    call = E._load().lapsum_expert_matmul_weights
    assert call(P, dtype, 10, n_in, 0, 1, P, experts, 10, n_in, out, P, out, P, _strides(*strides), 0, 0, None) == INVALID
