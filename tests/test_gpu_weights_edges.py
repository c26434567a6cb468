"""Calls of the attention weights that the documentation allows or refuses and that lie at its edges, against plain statements in 64 bits (tolerances: see
test_gpu_evict)."""
import math

import pytest
import torch

import paged_ref as ref
import tree_ref as tree

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


@pytest.mark.parametrize("kind", ["bf16", "e4m3", "i8"])
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("heads,n", [(2, 1), (4, 5), (8, 8), (8, 30), (8, 70), (6, 300)])       # rows of every kernel
@pytest.mark.parametrize("causal", [True, False])
def test_queries_without_statistics_give_nothing_whatever_they_hold(kind, dim, heads, n, causal):
    # queries whose lse is -infinity: a padded batch's, say, with anything in them
    kv_heads, page, lens = 2, 16, [500, 340]
    g = torch.Generator(device="cuda").manual_seed(31)
    kv = siso.PagedKV(*ref.make_pages(kind, 1, 64, page, kv_heads, dim))
    table = torch.randperm(64, device="cuda", generator=g).to(torch.int32).view(2, 32)
    slots = [table[b].long()[torch.arange(m, device="cuda") // page] * page + torch.arange(m, device="cuda") % page for b, m in enumerate(lens)]
    rows = [torch.randn((m, kv_heads, dim), device="cuda", generator=g) for m in lens]
    for x, at in zip(rows, slots):
        kv.write(x, x, at)
    truth = [x.to(torch.bfloat16).double() if kind == "bf16" else ref.values(*ref.quantised(x, kind)) for x in rows]
    q = torch.randn((2 * n, heads, dim), device="cuda", generator=g).to(torch.bfloat16)
    lse = torch.cat([ref.attention(q[b * n:(b + 1) * n], truth[b], truth[b], n, causal)[1].float() for b in range(2)])
    dead = torch.rand((2 * n, heads), device="cuda", generator=g) < 0.3
    dead[0] = True
    lse[dead] = -math.inf
    held = q.clone()
    held[dead] = torch.tensor([math.nan, math.inf, -math.inf, 3e38], device="cuda").to(torch.bfloat16).repeat(dim // 4)
    zero = q.masked_fill(dead[:, :, None], 0)
    got, want = (torch.full_like(kv.new_weights(), 2.0) for _ in range(2))
    for w, x in ((got, held), (want, zero)):
        kv.add_weights(w, x, lse, i32([0, n, 2 * n]), i32(lens), table, n, causal=causal, decay=0.5)
    assert torch.equal(got.view(torch.int32), want.view(torch.int32))
    for b, m in enumerate(lens):
        given, top, ab = tree.weights(zero[b * n:(b + 1) * n], truth[b], lse[b * n:(b + 1) * n], causal)
        before = torch.where(torch.arange(m, device="cuda")[:, None] < m - n, 1.0, 0.0).double()
        most = float(lse[b * n:(b + 1) * n].masked_fill(dead[b * n:(b + 1) * n], 0).abs().max())
        tol = given * (2 * (dim + 8) * 2.0 ** -24 * ab + 2.0 ** -22 * (top + most) + 2.0 ** -20 + n * heads // kv_heads * 2.0 ** -24) + 2.0 ** -22 * (before + given) + 1e-37
        w = got[0].transpose(1, 2).reshape(-1, kv_heads)[slots[b]].double()
        assert ((w - before - given).abs() <= tol).all()
    kv.check_status()
    kv.close()
