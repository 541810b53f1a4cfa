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
