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


def filled(kind, lens, page, kv_heads, dim, g, room=0):
    """A cache with rows of every sequence, NaN in every other place: (kv, table, places of each sequence's tokens and of `room` more, true rows)."""
    held = [-(-(m + room) // page) for m in lens]
    kv = siso.PagedKV(*ref.make_pages(kind, 1, sum(held) + 1, page, kv_heads, dim, fill="nan"))
    order = torch.randperm(sum(held) + 1, device="cuda", generator=g).to(torch.int32)
    table = torch.full((len(lens), max(held)), -1, **I32)
    slots, truth = [], []
    for b, m in enumerate(lens):
        table[b, :held[b]] = order[sum(held[:b]):sum(held[:b + 1])]
        at = torch.arange(m + room, device="cuda")
        slots.append(table[b].long()[at // page] * page + at % page)
        x = torch.randn((m, kv_heads, dim), device="cuda", generator=g)
        kv.write(x, x, slots[b][:m])
        truth.append(true_rows(x, kind))
    return kv, table, slots, truth


def true_rows(x, kind):
    return x.to(torch.bfloat16).double() if kind == "bf16" else ref.values(*ref.quantised(x, kind))


def by_place(w, layer=0):
    """weights [layers, pages, kv heads, tokens] as [places, kv heads]; a view's copy."""
    return w[layer].transpose(1, 2).reshape(-1, w.shape[2])


def check_weights(got, q, truth, lse, before, heads, kv_heads, dim):
    """got [n, kv heads] against what the queries give and `before`; tolerance: see test_gpu_evict."""
    given, top, ab = tree.weights(q, truth, lse)
    most = float(lse[lse > -math.inf].abs().max())
    tol = given * (2 * (dim + 8) * 2.0 ** -24 * ab + 2.0 ** -22 * (top + most) + 2.0 ** -20 + q.shape[0] * heads // kv_heads * 2.0 ** -24) + 2.0 ** -22 * (before + given) + 1e-37
    assert torch.isfinite(got).all() and ((got.double() - before - given).abs() <= tol).all()


@pytest.mark.parametrize("kind", ["bf16", "e4m3", "i8"])
@pytest.mark.parametrize("heads,n,dim", [(2, 1, 64), (4, 4, 128), (8, 4, 64), (8, 7, 128), (8, 30, 128), (8, 70, 64), (32, 200, 128)])       # rows of every kernel
def test_tokens_are_new_by_their_number_and_not_by_the_queries(kind, heads, n, dim):
    # the last n queries of longer chunks, or of no chunk at all; the places of new tokens hold NaN, as if left by others
    kv_heads, page, lens = 2, 16, [700, 450, 300, 333, n]
    fresh = [n + 137, 0, 300, n, 2 ** 31 - 1]
    g = torch.Generator(device="cuda").manual_seed(37)
    kv, table, slots, truth = filled(kind, lens, page, kv_heads, dim, g)
    q = torch.randn((len(lens) * n, heads, dim), device="cuda", generator=g).to(torch.bfloat16)
    part = lambda t, b: t[b * n:(b + 1) * n]
    lse = torch.cat([ref.attention(part(q, b), x, x, n)[1].float() for b, x in enumerate(truth)])
    w = kv.new_weights().fill_(math.nan)
    old = []
    for b, m in enumerate(lens):
        old.append(torch.where(torch.arange(m, device="cuda")[:, None] < m - min(fresh[b], m), torch.rand((m, kv_heads), device="cuda", generator=g) * 3, math.nan))
        w[0, slots[b] // page, :, slots[b] % page] = old[b]
    cu = i32([b * n for b in range(len(lens) + 1)])
    start = w.clone()
    kv.add_weights(w, q, lse, cu, i32(lens), table, n, decay=0.75, n_new=i32(fresh))
    for b, m in enumerate(lens):
        check_weights(by_place(w)[slots[b]], part(q, b), truth[b], part(lse, b), torch.nan_to_num(0.75 * old[b].double(), nan=0.0), heads, kv_heads, dim)
    # below zero is none; as many as there are queries is what a call without the number takes
    for x, y in ((i32([-5] * len(lens)), i32([0] * len(lens))), (i32([n] * len(lens)), None)):
        a, b = start.nan_to_num(nan=1.0), start.nan_to_num(nan=1.0)
        for t, new in ((a, x), (b, y)):
            kv.add_weights(t, q, lse, cu, i32(lens), table, n, decay=0.75, n_new=new)
        assert torch.equal(a, b)
    kv.check_status()
    for bad in (i32(fresh).long(), i32(fresh)[:4], torch.tensor(fresh, dtype=torch.int32), i32(fresh)[None]):
        with pytest.raises(ValueError):
            kv.add_weights(w, q, lse, cu, i32(lens), table, n, n_new=bad)
    kv.close()


@pytest.mark.parametrize("kind", ["bf16", "i8"])
def test_a_cache_is_evicted_from_drafted_into_and_weighed_on(kind):
    # eviction in place leaves weights in the places it vacates; a chunk comes to lie there of which the last queries alone are given, then a tree of drafts, whose
    # path is weighed once with its own queries and once by the next token's alone
    heads, kv_heads, dim, page, total, budget, recent = 8, 2, 64, 16, 400, 100, 20
    g = torch.Generator(device="cuda").manual_seed(41)
    kv, table, slots, truth = filled(kind, [total], page, kv_heads, dim, g, room=64)
    slots, truth = slots[0], truth[0]
    new_q = lambda n: torch.randn((n, heads, dim), device="cuda", generator=g).to(torch.bfloat16)

    def append(n):
        nonlocal truth
        x = torch.randn((n, kv_heads, dim), device="cuda", generator=g)
        kv.write(x, x, slots[truth.shape[0]:truth.shape[0] + n])
        truth = torch.cat([truth, true_rows(x, kind)])
        return i32([truth.shape[0]])

    w = kv.new_weights()
    q = new_q(total)
    _, lse = kv.attention(q, i32([0, total]), i32([total]), table, total, want_lse=True)
    kv.add_weights(w, q, lse, i32([0, total]), i32([total]), table, total)
    lens, kept = kv.evict(w, i32([total]), table, budget, recent)
    truth = torch.stack([truth[kept[0, 0, h].long(), h] for h in range(kv_heads)], 1)
    stale = by_place(w)[slots[budget:total]]
    assert (stale > 0).all()                                       # what the places vacated still hold
    before = by_place(w)[slots[:budget]].double()
    # a chunk of 50, its last 6 queries
    lens = append(50)
    q = new_q(50)
    _, lse = kv.attention(q, i32([0, 50]), lens, table, 50, want_lse=True)
    kv.add_weights(w, q[-6:], lse[-6:], i32([0, 6]), lens, table, 6, decay=0.5, n_new=i32([50]))
    before = torch.cat([0.5 * before, torch.zeros((50, kv_heads), dtype=torch.float64, device="cuda")])
    check_weights(by_place(w)[slots[:150]], q[-6:], truth, lse[-6:], before, heads, kv_heads, dim)
    # a tree of 8 nodes, three of them accepted
    before = by_place(w)[slots[:150]].double()
    lens = append(8)
    q = new_q(8)
    cu = i32([0, 8])
    mask, _ = siso.tree_mask(i32([-1, 0, 0, 2, 1, 3, 5, 0]), cu, 8)
    _, lse = kv.tree_attention(q, cu, lens, table, mask, 8, want_lse=True)
    lens = kv.keep_path(i32([[2, 3, 5]]), i32([3]), cu, lens, table)
    assert lens.tolist() == [154]
    truth = torch.cat([truth[:151], truth[[152, 153, 155]]])
    path = torch.tensor([0, 2, 3, 5], device="cuda")
    one, two = w.clone(), w.clone()
    kv.add_weights(one, q[path], lse[path], i32([0, 4]), lens, table, 4, decay=0.5)
    none = torch.zeros((4, kv_heads), dtype=torch.float64, device="cuda")
    check_weights(by_place(one)[slots[:154]], q[path], truth, lse[path], torch.cat([0.5 * before, none]), heads, kv_heads, dim)
    # or the next token, five of them new
    lens = append(1)
    q = new_q(1)
    _, lse = kv.attention(q, i32([0, 1]), lens, table, 1, want_lse=True)
    kv.add_weights(two, q, lse, i32([0, 1]), lens, table, 1, decay=0.5, n_new=i32([5]))
    check_weights(by_place(two)[slots[:155]], q, truth, lse, torch.cat([0.5 * before, none, none[:1]]), heads, kv_heads, dim)
    kv.check_status()
    kv.close()
