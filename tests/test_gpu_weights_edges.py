"""Calls of the attention weights that the documentation allows or refuses and that lie at its edges, against plain statements in 64 bits (tolerances: see
test_gpu_evict)."""
import pytest
import torch

pytestmark = pytest.mark.gpu

siso = pytest.importorskip("paper_2508_18736_b200")
I32 = dict(dtype=torch.int32, device="cuda")


def i32(x):
    return torch.tensor(x, **I32)


def status_of(call, *args, **kwargs):
    """The status that a call is refused with (0: it is not).  Unlike a kept exception, this leaves no cycle through the caller's frame."""
    try:
        call(*args, **kwargs)
    except siso.SisoError as e:
        return e.status
    return 0


@pytest.mark.parametrize("heads,n", [(4, 1), (8, 100)])
@pytest.mark.parametrize("decay", [0.0, 1.0])
def test_weights_that_begin_off_a_boundary_of_16_bytes_are_refused(heads, n, decay):
    # nothing is launched: they are read 16 bytes at a time
    kv = siso.PagedKV.allocate(1, 16, 16, 2, 64)
    q, lse = torch.zeros((n, heads, 64), dtype=torch.bfloat16, device="cuda"), torch.zeros((n, heads), device="cuda")
    room = torch.zeros(kv.new_weights().numel() + 4, device="cuda")
    for first, status in ((1, 2), (2, 2), (3, 2), (4, 0)):
        w = room[first:first + 16 * 2 * 16].view(1, 16, 2, 16)
        assert w.is_contiguous() and w.data_ptr() % 16 == 4 * first % 16
        room.zero_()
        assert status_of(kv.add_weights, w, q, lse, i32([0, n]), i32([200]), torch.arange(16, **I32)[None], n, decay=decay) == status
        assert (room != 0).any() == (status == 0)
    kv.check_status()
    kv.close()
