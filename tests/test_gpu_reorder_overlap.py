"""States of one reorder that share memory: refused where one is written, moved
where all of it is only read or lies side by side."""
import ctypes

import pytest

from test_gpu_selection_binding import way  # noqa: F401  (both ways into the library)

pytestmark = pytest.mark.gpu


def test_states_that_share_what_is_written_are_refused(lib, way):  # noqa: F811
    import torch
    k, v = torch.randn(8, 3, 5, 4, device="cuda"), torch.randn(8, 3, 5, 4, device="cuda")
    wide = torch.randn(12, 3, 5, 4, device="cuda")
    parents = torch.randint(0, 4, (2, 4), dtype=torch.int32, device="cuda")
    was = [t.clone() for t in (k, v, wide)]
    for states, kw in (([k, v, k], {}), ([k, k.view(8, 15, 4)], {}), ([k, v], dict(out=[v, k])),
                       ([k, v], dict(out=[torch.empty_like(k)] * 2)), ([wide[:8], wide[4:]], {}),
                       ([wide[:8]], dict(out=[wide[4:]])), ([k, v], dict(out=[k, k])),
                       ([k, k], dict(length=2))):
        with pytest.raises(lib.LapsumError):
            lib.lapsum_beam_reorder(states, parents, **kw)
    with pytest.raises(lib.LapsumError):
        lib.lapsum_beam_reorder([parents.view(8)], parents)
    assert all(torch.equal(a, b) for a, b in zip((k, v, wide), was))


def test_states_that_share_what_is_read_are_moved(lib, way):  # noqa: F811
    import torch
    k = torch.randn(8, 3, 5, 4, device="cuda")
    parents = torch.tensor([[3, 3, 0, 1], [2, 0, 0, 2]], dtype=torch.int32, device="cuda")
    row = [3, 3, 0, 1, 6, 4, 4, 6]
    one, two = torch.empty_like(k), torch.empty_like(k)
    lib.lapsum_beam_reorder([k, k], parents, out=[one, two])
    assert torch.equal(one, k[row]) and torch.equal(two, k[row])
    # one in place, the other out of place
    other = torch.randn(8, 6, device="cuda")
    want = [other[row], k[row]]
    lib.lapsum_beam_reorder([other, k], parents, out=[other, one])
    assert torch.equal(other, want[0]) and torch.equal(one, want[1])


def test_keys_and_values_in_one_buffer_are_moved(lib):
    """Through the C entry: [rows, heads, 2, room, dim], a state a half of each head."""
    import torch
    import paper_2608_06912_amd.selection as S
    both = torch.randn(8, 3, 2, 5, 4, device="cuda")
    parents = torch.tensor([[3, 3, 0, 1], [2, 0, 0, 2]], dtype=torch.int32, device="cuda")
    want = both.clone()
    want[:, :, 0, :2] = both[[3, 3, 0, 1, 6, 4, 4, 6]][:, :, 0, :2]
    want[:, :, 1] = both[[3, 3, 0, 1, 6, 4, 4, 6]][:, :, 1]
    at = both.data_ptr()
    array = (S._BeamState * 2)(S._BeamState(at, at, 480, 3, 160, 32), S._BeamState(at + 80, at + 80, 480, 3, 160, 80))
    stream = torch.cuda.current_stream().cuda_stream
    status = S._load().lapsum_beam_reorder(ctypes.addressof(array), 2, parents.data_ptr(), 4, 2, 4, stream)
    assert status == 0 and torch.equal(both, want)
