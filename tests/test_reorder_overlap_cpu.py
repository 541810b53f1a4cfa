"""Which states lapsum_beam_reorder takes together: what a call writes must be
nothing else that it reads or writes.  On the CPU, from addresses alone: a call that
is taken ends at the device check, with nothing read or enqueued."""
import ctypes
import random

import pytest
import torch

import paper_2608_06912_amd as L
import paper_2608_06912_amd.selection as S

pytestmark = [
    pytest.mark.skipif(not __import__("os").path.exists(L.LIB_PATH), reason="library not built"),
    pytest.mark.skipif(torch.cuda.is_available(), reason="the addresses are no memory: no device may be there")]

INVALID = 1
P = 1 << 40          # the states' addresses, never read
PARENTS = 1 << 30


def _taken(states, batch=2, beams=4, parents=PARENTS, stride=None):
    """states: (in, out, row_bytes, outer, outer_stride, live_bytes)."""
    array = (S._BeamState * len(states))(*[S._BeamState(*s) for s in states])
    status = S._load().lapsum_beam_reorder(ctypes.addressof(array), len(states), parents,
                                           beams if stride is None else stride, batch, beams, None)
    assert status != 0
    return status != INVALID


def _plain(src, dst, row=64):
    return (src, dst, row, 1, 0, row)


def test_states_apart_are_taken():
    a, b, c, d = P, P + 512, P + 1024, P + 1536       # eight rows of 64 bytes each
    assert _taken([_plain(a, a)])
    assert _taken([_plain(a, a), _plain(b, b)])
    assert _taken([_plain(b, b), _plain(a, a)])
    assert _taken([_plain(a, b), _plain(c, d)])
    assert _taken([_plain(a, b), _plain(a, c)])       # the same memory read twice


@pytest.mark.parametrize("states", [
    [_plain(P, P), _plain(P, P)],                     # listed twice, in place
    [_plain(P, P + 512), _plain(P + 512, P)],         # two states swapped
    [_plain(P, P + 512), _plain(P + 1024, P + 512)],  # one out for two
    [_plain(P, P + 512), _plain(P + 512, P + 1024)],  # an out that is another's in
    [_plain(P, P), _plain(P, P + 512)],               # in place and read as well
    [_plain(P, P + 64)],                              # an out a row further
    [_plain(P, P + 32)],
    [_plain(P, P), _plain(P + 511, P + 511)],         # the last byte
    [_plain(P + 511, P + 511), _plain(P, P)],
    [_plain(P + 64 * i, P + 64 * i, 1024) for i in (0, 1, 17)]])
def test_shared_states_are_refused(states):
    assert not _taken(states)
    apart = [_plain(P + (1 << 20) * (i + 1), P + (1 << 20) * (i + 1)) for i in range(20)]
    assert not _taken(apart + states) and not _taken(states + apart)
    assert _taken(apart)


def test_an_empty_state_shares_nothing():
    assert _taken([_plain(P, P), (P, P, 64, 0, 0, 64), (P, P, 64, 1, 0, 0)])


def test_parents_that_are_written_are_refused():
    assert not _taken([_plain(PARENTS, PARENTS)])
    assert not _taken([_plain(PARENTS + 28, PARENTS + 28)])
    assert _taken([_plain(PARENTS + 32, PARENTS + 32)])
    assert not _taken([_plain(PARENTS + 32, PARENTS + 32)], stride=7)     # rows 7 apart: 44 bytes
    assert _taken([_plain(PARENTS + 44, PARENTS + 44)], stride=7)


def test_states_side_by_side_in_one_buffer_are_taken():
    """Keys and values of every layer in one row, or in one head."""
    rows = [(P + 64 * i, P + 64 * i, 64 * 6, 1, 0, 64) for i in range(6)]
    assert _taken(rows) and not _taken(rows + rows[:1])
    heads = [(P + 32 * i, P + 32 * i, 4 * 96, 4, 96, 32) for i in range(3)]
    assert _taken(heads)
    assert not _taken(heads + [(P + 31, P + 31, 4 * 96, 1, 0, 2)])
    half = [(P + 32 * i, P + 32 * i, 4 * 96, 4, 96, 40) for i in range(2)]
    assert not _taken(half)
    assert _taken([(P, P, 400, 4, 100, 60), (P + 60, P + 60, 400, 4, 100, 40)], batch=1, beams=1)


def _bytes(address, rows, state):
    row, outer, stride, live = state[2:]
    return {address + r * row + o * stride + i for r in range(rows) for o in range(outer) for i in range(live)}


def test_no_sharing_is_missed():
    """Random small states against their bytes: shared ones are never taken, and ones that
    end before the others begin always are."""
    rng = random.Random(5)
    shared = taken = 0
    for _ in range(4000):
        batch, beams = rng.choice([(1, 1), (1, 3), (2, 2)])
        row = rng.choice([12, 24, 48])
        states, sets = [], []
        for _ in range(rng.randint(1, 3)):
            r = row if rng.random() < 0.8 else rng.choice([12, 24, 48])
            outer = rng.choice([1, 1, 2, 3])
            stride = r // outer if outer > 1 else 0
            live = rng.randint(1, stride or r)
            src = P + rng.randint(0, 60) * rng.choice([1, 4, 12])
            dst = src if rng.random() < 0.5 else P + rng.randint(0, 200)
            s = (src, dst, r, outer, stride, live)
            states.append(s)
            sets.append((_bytes(dst, batch * beams, s), None if src == dst else _bytes(src, batch * beams, s)))
        every = [(w, True) for w, _ in sets] + [(r, False) for _, r in sets if r is not None]
        bad = any((every[i][1] or every[j][1]) and every[i][0] & every[j][0]
                  for i in range(len(every)) for j in range(i))
        ends = sorted((min(b), max(b)) for b, _ in every)
        got = _taken(states, batch, beams)
        shared += bad
        taken += got
        assert not (bad and got), states
        if all(a[1] < b[0] for a, b in zip(ends, ends[1:])):
            assert got, states
    assert shared > 500 and taken > 500
