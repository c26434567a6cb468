"""The weight that attention gives to cached tokens, and the eviction by it, against plain statements in 64 bits.

Tolerances.  Eviction is exact.  A weight: the score is off by at most d = (dim + 8) 2^-24 max sum |q||k| scale, its difference from lse in powers of two is
rounded to fp32 twice (2^-23 of |score| + |lse| together, times log2 e), the exponential adds less than 2^-20, and a sum of m positive terms in any order at most
m 2^-24 of itself:
    |w - exact| <= W (2 d + 2^-22 (max |score| + max |lse|) + 2^-20 + m 2^-24) + 2^-22 (decay |old| + W),   W = sum of the weights given, m = queries x heads of a kv head
"""
import math

import pytest
import torch

import paged_ref as ref
import tree_ref as tree

pytestmark = pytest.mark.gpu

siso = pytest.importorskip("paper_2508_18736_b200")
I32 = dict(dtype=torch.int32, device="cuda")
NAN = math.nan


def i32(x):
    return torch.tensor(x, **I32)


def status_of(call, *args, **kwargs):
    """The status that a call is refused with (0: it is not).  Unlike a kept exception, this leaves no cycle through the caller's frame, whose tensors would
    stay until a collection at some later time."""
    try:
        call(*args, **kwargs)
    except siso.SisoError as e:
        return e.status
    return 0


def held_pages(lens, page, spare=2, seed=1):
    held = [-(-max(n, 0) // page) for n in lens]
    order = torch.randperm(sum(held) + spare, device="cuda", generator=torch.Generator(device="cuda").manual_seed(seed)).to(torch.int32)
    table = torch.full((len(lens), max(held) + 1), -1, **I32)
    for b, h in enumerate(held):
        table[b, :h] = order[sum(held[:b]):sum(held[:b]) + h]
    return table, sum(held) + spare


def run_weights(kind, dim, heads, kv_heads, page, lens, q_lens, causal=True, decay=1.0, head_major=False, hint=None, gain=1.0, scale=None, strided=False,
                last=None):
    """Every place beyond a sequence's tokens is NaN, and so are the weights that must not be read.  last: only so many of a sequence's queries are given."""
    g = torch.Generator(device="cuda").manual_seed(23)
    table, pages = held_pages(lens, page)
    k, v, ke, ve = ref.make_pages(kind, 2, pages, page, kv_heads, dim, head_major, fill="nan")
    kv = siso.PagedKV(k, v, ke, ve)
    w = kv.new_weights().fill_(NAN)
    truth, old, slots = [], [], []
    cu = [sum(q_lens[:i]) for i in range(len(lens) + 1)]
    for b, n in enumerate(lens):
        i = torch.arange(n, device="cuda")
        p, t = table[b].long()[i // page], i % page
        x = torch.randn((n, kv_heads, dim), device="cuda", generator=g)
        kv.write(x, x, p * page + t, layer=1)
        truth.append(x.to(torch.bfloat16).double() if kind == "bf16" else ref.values(*ref.quantised(x, kind)))
        x = torch.rand((n, kv_heads), device="cuda", generator=g) * 3
        if decay == 0:
            x.fill_(NAN)
        x[max(0, n - q_lens[b]):] = NAN                       # new tokens: nothing is there yet
        if q_lens[b] == 0:
            x.fill_(2.5)
        w[1, p, :, t] = x
        old.append(x)
        slots.append((p, t))
    q = torch.full((cu[-1] + 3, heads, dim), NAN, device="cuda")                  # rows that no sequence covers
    q[:cu[-1]] = gain * torch.randn((cu[-1], heads, dim), device="cuda", generator=g)
    q = q.to(torch.bfloat16)
    if strided:
        wide = torch.full((q.shape[0], heads + 2, dim + 8), NAN, dtype=torch.bfloat16, device="cuda")
        wide[:, 1:1 + heads, :dim] = q
        q = wide[:, 1:1 + heads, :dim]
    lse = torch.full((q.shape[0], heads), NAN, device="cuda")
    for b, n in enumerate(lens):
        lo, hi = cu[b], cu[b + 1]
        if hi > lo:
            lse[lo:hi] = ref.attention(q[lo:hi], truth[b], truth[b], hi - lo, causal, 0, scale)[1].float()
    start = w.clone()
    args = (q, lse, i32(cu), i32(lens), table, max(q_lens) if hint is None else hint)
    kv.add_weights(w, *args, layer=1, scale=scale, causal=causal, decay=decay)
    assert kv.sync_status() == 0
    again = start.clone()
    kv.add_weights(again, *args, layer=1, scale=scale, causal=causal, decay=decay)
    assert torch.equal(w.view(torch.int32), again.view(torch.int32)), "two calls differ"
    untouched = torch.ones_like(w, dtype=torch.bool)
    for b, n in enumerate(lens):
        lo, hi = cu[b], cu[b + 1]
        p, t = slots[b]
        if hi == lo or n == 0:
            continue
        untouched[1, p, :, t] = False
        got = w[1, p, :, t].double()
        given, top, ab = tree.weights(q[lo:hi], truth[b], lse[lo:hi], causal, scale)
        before = torch.where(torch.arange(n, device="cuda")[:, None] < n - (hi - lo), decay * old[b].double(), 0.0) if decay else torch.zeros_like(given)
        d = (dim + 8) * 2.0 ** -24 * ab
        m = (hi - lo) * heads // kv_heads
        finite = lse[lo:hi][lse[lo:hi] > -math.inf]
        most = float(finite.abs().max()) if finite.numel() else 0.0
        tol = given * (2 * d + 2.0 ** -22 * (top + most) + 2.0 ** -20 + m * 2.0 ** -24) + 2.0 ** -22 * (before + given) + 1e-37
        assert torch.isfinite(got).all()
        assert ((got - before - given).abs() <= tol).all(), float(((got - before - given).abs() / tol).max())
    assert torch.equal(w.view(torch.int32)[untouched], start.view(torch.int32)[untouched]), "a weight of no token changed"
    kv.close()


@pytest.mark.parametrize("kind", ["bf16", "e4m3", "i8"])
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("heads,kv_heads,page", [(8, 2, 16), (7, 1, 48), (4, 4, 8), (24, 2, 128)])
def test_single_tokens(kind, dim, heads, kv_heads, page):
    run_weights(kind, dim, heads, kv_heads, page, [1, 2, 17, 63, 64, 65, 127, 128, 129, 700, 0, 1999, 40], [1] * 12 + [0], head_major=page == 16)


@pytest.mark.parametrize("kind", ["bf16", "e4m3", "i8"])
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("heads,kv_heads,page,q_lens,decay", [(8, 2, 32, [5, 2, 7, 0, 16, 3, 11], 0.5), (7, 1, 24, [30, 9, 18, 19, 0, 3, 1], 0.0),
                                                              (3, 3, 64, [5, 9, 128, 129, 64, 3, 127], 1.0), (32, 2, 16, [4, 8, 9, 16, 7, 3, 17], 0.9)])
def test_short_chunks(kind, dim, heads, kv_heads, page, q_lens, decay):
    run_weights(kind, dim, heads, kv_heads, page, [5, 9, 300, 257, 64, 3, 1030], q_lens, decay=decay)


@pytest.mark.parametrize("kind", ["bf16", "e4m3", "i8"])
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("heads,kv_heads,page,lens,q_lens", [
    (4, 1, 64, [130, 511], [130, 257]), (8, 2, 16, [1025, 640, 90], [300, 1, 90]), (5, 1, 48, [777], [401]), (2, 2, 8, [1300], [1300]), (40, 1, 32, [500, 31], [33, 31]),
    (200, 1, 16, [300, 600], [7, 2]), (9, 1, 16, [3000, 100, 257], [3000, 57, 200])])
def test_long_chunks(kind, dim, heads, kv_heads, page, lens, q_lens):
    run_weights(kind, dim, heads, kv_heads, page, lens, q_lens, head_major=page in (16, 48))


@pytest.mark.parametrize("q_len,n", [(1, 70), (6, 333), (200, 1024)])
@pytest.mark.parametrize("kind", ["bf16", "i8"])
def test_without_causality_with_strides_and_any_hint(kind, q_len, n):
    run_weights(kind, 128, 8, 2, 32, [n, n // 2], [q_len, q_len], causal=False, strided=True, decay=0.25)
    for hint in (0, 1, 1 << 20):
        run_weights(kind, 64, 8, 2, 32, [n, n // 2], [q_len, q_len], hint=hint)


@pytest.mark.parametrize("q_len", [1, 8, 260])
def test_queries_that_see_nothing(q_len):
    run_weights("bf16", 128, 8, 2, 16, [q_len // 2, 0, 700], [q_len, q_len, q_len])
    run_weights("e4m3", 64, 4, 4, 16, [q_len // 2, 0, 700], [q_len, q_len, q_len], decay=0.0)


@pytest.mark.parametrize("q_len", [1, 190])
def test_steep_flat_and_reversed_scores(q_len):
    run_weights("bf16", 128, 8, 2, 32, [900, 1300], [q_len, q_len], gain=40.0)
    run_weights("bf16", 64, 8, 2, 32, [900, 1300], [q_len, q_len], scale=0.0)
    run_weights("e4m3", 128, 8, 2, 32, [900, 1300], [q_len, q_len], scale=-0.2)


@pytest.mark.parametrize("kind", ["bf16", "e4m3"])
def test_many_row_tiles_for_few_keys_are_split_and_joined(kind):
    run_weights(kind, 64, 16, 1, 64, [1500], [1500])
    run_weights(kind, 128, 8, 1, 64, [20011, 3], [9, 3])


@pytest.mark.parametrize("kind", ["bf16", "e4m3", "i8"])
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("q_len,heads", [(1, 8), (4, 32), (7, 32), (20, 32)])
def test_many_units_for_each_sm(kind, dim, q_len, heads):
    # 8 kv heads x 30,000 tokens: every ring goes round more than once
    run_weights(kind, dim, heads, 8, 64, [29003, 1500], [q_len, q_len], decay=0.5)


@pytest.mark.parametrize("n_q", [1, 20, 100])
def test_pages_outside_the_pool_and_long_lengths(n_q):
    page, heads, dim = 16, 2, 128
    k, v, _, _ = ref.make_pages("bf16", 1, 10, page, heads, dim)
    kv = siso.PagedKV(k, v)
    q = torch.randn((n_q, 8, dim), device="cuda").to(torch.bfloat16)
    lse = torch.full((n_q, 8), 4.0, device="cuda")
    for bad in (-1, 10, 2 ** 31 - 1):
        w = kv.new_weights()
        table = i32([[3, 4, bad, 5, 0, 1, 2]])
        kv.add_weights(w, q, lse, i32([0, n_q]), i32([7 * page]), table, n_q, causal=False)
        assert kv.sync_status() == 1 and kv.sync_status() == 0
        kept = [3, 4, 5, 0, 1, 2]
        given, _, _ = tree.weights(q, k[0, kept].reshape(-1, heads, dim).double(), lse, causal=False)
        got = w[0, kept].transpose(1, 2).reshape(-1, heads).double()
        assert ((got - given).abs() <= 1e-4 * given).all() and (w[0, 6:] == 0).all()
    w = kv.new_weights()
    kv.add_weights(w, q, lse, i32([0, n_q]), i32([7 * page]), i32([[3, 4]]), n_q, causal=False)          # cut to what the table can hold
    assert kv.sync_status() == 0 and (w[0, [0, 1, 2, 5, 6, 7, 8, 9]] == 0).all() and (w[0, 3:5] > 0).all()
    kv.close()


def test_infinite_and_missing_statistics():
    kv = siso.PagedKV.allocate(1, 4, 16, 1, 64)
    q = torch.ones((3, 2, 64), dtype=torch.bfloat16, device="cuda")
    lse = torch.tensor([[-math.inf, 0.0], [math.inf, 0.0], [0.0, math.log(4.0)]], device="cuda")
    w = kv.new_weights()
    kv.add_weights(w, q, lse, i32([0, 3]), i32([40]), i32([[0, 1, 2, 3]]), 3)             # keys are zero: every score is 0
    got = w[0].reshape(-1)
    assert torch.allclose(got[:38], torch.full((38,), 3.25, device="cuda")) and torch.allclose(got[38:40], torch.tensor([2.25, 1.25], device="cuda")) and (got[40:] == 0).all()
    kv.close()


def test_a_long_pool_is_addressed_beyond_32_bits():
    page, heads, dim = 64, 8, 128
    pages = (1 << 31) // (page * heads * dim) + 40
    k = torch.zeros((1, pages, page, heads, dim), dtype=torch.int8, device="cuda")
    exps = [torch.full((1, pages, heads, page), 127, dtype=torch.uint8, device="cuda") for _ in range(2)]
    v = torch.zeros_like(k)
    kv = siso.PagedKV(k, v, *exps)
    g = torch.Generator(device="cuda").manual_seed(3)
    n = 3 * page + 5
    table = i32([[pages - 1, 2, pages - 7, pages - 2]])
    i = torch.arange(n, device="cuda")
    p, t = table[0].long()[i // page], i % page
    rows = torch.randn((n, heads, dim), device="cuda", generator=g)
    kv.write(rows, rows, p * page + t)
    truth = ref.values(*ref.quantised(rows, "i8"))
    for n_q in (1, 150):
        w = kv.new_weights()
        q = torch.randn((n_q, 4 * heads, dim), device="cuda", generator=g).to(torch.bfloat16)
        lse = ref.attention(q, truth, truth, n_q)[1].float().contiguous()
        kv.add_weights(w, q, lse, i32([0, n_q]), i32([n]), table, n_q)
        given, _, _ = tree.weights(q, truth, lse)
        assert ((w[0, p, :, t].double() - given).abs() <= 1e-4 * given).all()
        assert (w[0, p, :, t].sum() - 4 * heads * n_q).abs() <= 1e-3 * heads * n_q       # each query gives 1 in all
    codes = k[0, p, t].clone()
    new, kept = kv.evict(w, i32([n]), table, 70, 5)
    assert new.tolist() == [70]
    for h in range(heads):
        assert torch.equal(k[0, p[:70], t[:70], h], codes[kept[0, 0, h].long(), h])
    kv.close()


# ---- eviction ------------------------------------------------------------------------------------------------------------------
def check_evict(kind, dim, heads, page, lens, budget, recent, layers=2, head_major=False, where="in place", fill="random", seed=7):
    g = torch.Generator(device="cuda").manual_seed(seed)
    table, used = held_pages(lens, page, spare=0)
    goal = [min(max(n, 0), budget) for n in lens]
    held = [-(-n // page) for n in goal]
    pages = used + sum(held) + 1
    k, v, ke, ve = ref.make_pages(kind, layers, pages, page, heads, dim, head_major, seed=seed)
    kv = siso.PagedKV(k, v, ke, ve)
    w = torch.rand((layers, pages, heads, page), device="cuda", generator=g)
    if fill == "ties":
        w = (w * 6).floor()
    elif fill == "odd":
        pick = torch.randint(0, 12, w.shape, device="cuda", generator=g)
        for i, x in enumerate((NAN, math.inf, -math.inf, 0.0, -0.0, 1e-42, -1e-42, -1.0, 3e38)):
            w[pick == i] = x
    elif fill == "equal":
        w.fill_(0.25)
    out = table
    if where != "in place":
        out = torch.full((len(lens), max(max(held), 1) + 1), -1, **I32)
        for b, h in enumerate(held):
            out[b, :h] = used + sum(held[:b]) + torch.arange(h, **I32)
            if where == "both" and h:
                out[b, ::2] = torch.where(torch.arange(out.shape[1], device="cuda")[::2] < h, table[b, :out.shape[1]][::2] if table.shape[1] >= out.shape[1] else out[b, ::2], out[b, ::2])
    bits = lambda t: t.view(torch.int32 if t.dtype == torch.float32 else torch.int8) if t.dtype != torch.bfloat16 else t.view(torch.int16)
    now = [t for t in (w, k, v, ke, ve) if t is not None]
    old = [bits(t).clone() for t in now]
    want = [t.clone() for t in old]
    weights = w.clone().cpu()
    new, kept = kv.evict(w, i32(lens), table, budget, recent, out_pages=None if where == "in place" else out)
    assert kv.sync_status() == 0 and new.tolist() == goal
    for b, n in enumerate(lens):
        n = max(n, 0)
        j = torch.arange(n, device="cuda")
        p, t = table[b].long()[j // page], j % page
        for layer in range(layers):
            for h in range(heads):
                stay = tree.kept(weights[layer, p.cpu(), h, t.cpu()], budget, recent)
                assert kept[layer, b, h].tolist() == stay + [-1] * (budget - len(stay))
                s = torch.tensor(stay, dtype=torch.long, device="cuda")
                to = torch.arange(len(stay), device="cuda")
                p1, t1 = out[b].long()[to // page], to % page
                for x, y in zip(want, old):
                    if x.dim() == 5:
                        x[layer, p1, t1, h] = y[layer, p[s], t[s], h]
                    else:
                        x[layer, p1, h, t1] = y[layer, p[s], h, t[s]]
    for a, b in zip(now, want):
        assert torch.equal(bits(a), b)
    kv.close()


@pytest.mark.parametrize("kind", ["bf16", "e4m3", "i8"])
@pytest.mark.parametrize("dim,heads,page,head_major", [(128, 2, 16, False), (64, 3, 48, True), (8, 1, 8, False), (72, 2, 8, True), (256, 1, 32, False)])
@pytest.mark.parametrize("where", ["in place", "new pages", "both"])
def test_rows_are_chosen_and_moved(kind, dim, heads, page, head_major, where):
    check_evict(kind, dim, heads, page, [700, 1, 0, 130, 129, 128, 1500], 128, 17, head_major=head_major, where=where)


@pytest.mark.parametrize("budget,recent", [(1, 0), (1, 1), (64, 0), (64, 64), (63, 62), (511, 3), (512, 100), (513, 7), (5000, 10)])
@pytest.mark.parametrize("fill", ["random", "ties", "odd", "equal"])
def test_budgets_and_weights_of_every_kind(budget, recent, fill):
    check_evict("bf16", 64, 2, 16, [512, 513, 1025, 3000], budget, recent, layers=1, fill=fill)


@pytest.mark.parametrize("lens,budget,heads", [([40_000], 5000, 1), ([33_000, 20_001, 12], 3001, 2), ([9000] * 40, 100, 4)])
def test_long_sequences_and_many(lens, budget, heads):
    check_evict("e4m3", 16, heads, 64, lens, budget, 100, layers=1)


def test_more_weights_than_shared_memory_holds():
    # 700,000 places of one head: more than the CTAs of a cluster keep
    n, page, budget, recent = 700_000, 64, 3000, 50
    pages = -(-n // page)
    k = torch.zeros((1, pages, page, 1, 8), dtype=torch.bfloat16, device="cuda")
    k[0, :, :, 0, 0] = (torch.arange(pages * page, device="cuda") % 251).view(pages, page).to(torch.bfloat16)
    kv = siso.PagedKV(k, k.clone())
    w = torch.rand((1, pages, 1, page), device="cuda", generator=torch.Generator(device="cuda").manual_seed(2))
    flat = w.reshape(-1).clone()
    new, kept = kv.evict(w, i32([n]), torch.arange(pages, **I32)[None], budget, recent)
    want = torch.cat([torch.sort(flat[:n - recent], descending=True, stable=True).indices[:budget - recent].sort().values, torch.arange(n - recent, n, device="cuda")])
    assert torch.equal(kept[0, 0, 0].long(), want) and torch.equal(k.reshape(-1, 8)[:budget, 0].long(), want % 251)
    assert torch.equal(w.reshape(-1)[:budget], flat[want])
    kv.close()


def test_pages_outside_the_pool_are_reported_and_left_out():
    k, v, _, _ = ref.make_pages("bf16", 1, 10, 16, 1, 64)
    kv = siso.PagedKV(k, v)
    w = torch.rand((1, 10, 1, 16), device="cuda")
    for bad in (-1, 10, 2 ** 31 - 1):
        weights, old = w.clone(), w.clone()
        table = i32([[3, 4, bad, 5]])
        new, kept = kv.evict(weights, i32([64]), table, 20, 4)
        assert kv.sync_status() == 1 and kv.sync_status() == 0
        places = old[0, [3, 4], 0].reshape(-1).tolist() + [NAN] * 16 + old[0, 5, 0].tolist()
        assert kept[0, 0, 0].tolist() == tree.kept(torch.tensor(places), 20, 4)
    kv.evict(w, i32([64]), i32([[3, 4, 6, 5]]), 40, 4, out_pages=i32([[0]]))               # too few pages for what stays
    assert kv.sync_status() == 1
    kv.close()


def test_evicted_caches_are_attended_over_as_what_stayed():
    # weights from a prompt's last queries, eviction, then the next token attends: as if over the rows that stayed of each head
    for kind in ("bf16", "i8"):
        n, page, heads, kv_heads, dim, budget, recent = 900, 16, 8, 2, 64, 200, 32
        table, pages = held_pages([n], page)
        kv = siso.PagedKV(*ref.make_pages(kind, 1, pages, page, kv_heads, dim, fill="nan"))
        j = torch.arange(n, device="cuda")
        slots = table[0].long()[j // page] * page + j % page
        g = torch.Generator(device="cuda").manual_seed(6)
        k, v = (torch.randn((n, kv_heads, dim), device="cuda", generator=g) for _ in range(2))
        kv.write(k, v, slots)
        k, v = (x.to(torch.bfloat16).double() if kind == "bf16" else ref.values(*ref.quantised(x, kind)) for x in (k, v))
        q = torch.randn((n, heads, dim), device="cuda", generator=g).to(torch.bfloat16)
        out, lse = kv.attention(q, i32([0, n]), i32([n]), table, n, want_lse=True)
        w = kv.new_weights().fill_(NAN)
        kv.add_weights(w, q[-40:], lse[-40:], i32([0, 40]), i32([n]), table, 40, decay=0.0)
        new, kept = kv.evict(w, i32([n]), table, budget, recent)
        q1 = torch.randn((1, heads, dim), device="cuda", generator=g).to(torch.bfloat16)
        got = kv.attention(q1, i32([0, 1]), new, table, 1, causal=False)
        idx = kept[0, 0].long()
        k1, v1 = (torch.stack([x[idx[h], h] for h in range(kv_heads)], 1) for x in (k, v))
        o, _, mass, _ = ref.attention(q1, k1, v1, 1, causal=False)
        assert ((got.double() - o).abs() <= 2.0 ** -8 * o.abs() + 1.02 * mass * 2.0 ** -8 + 1e-4 * mass).all()
        assert kv.sync_status() == 0
        kv.close()


def test_streams_and_graphs():
    k, v, ke, ve = ref.make_pages("i8", 1, 64, 16, 2, 128)
    kv = siso.PagedKV(k, v, ke, ve)
    q = torch.randn((300, 8, 128), device="cuda").to(torch.bfloat16)
    cu, lens, table = i32([0, 299, 300]), i32([400, 300]), torch.randperm(64, device="cuda").to(torch.int32).view(2, 32)
    lse = torch.full((300, 8), 5.0, device="cuda")
    state = [t.clone() for t in (k, v, ke, ve)]
    w = kv.new_weights()

    def calls(stream):
        for t, s in zip((k, v, ke, ve), state):
            t.copy_(s)
        w.zero_()
        kv.add_weights(w, q, lse, cu, lens, table, 299, stream=stream)
        return [*kv.evict(w, lens, table, 100, 10, stream=stream)]

    want = [t.clone() for t in calls(None)] + [t.clone() for t in (w, k, v, ke, ve)]
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        got = calls(s)
    s.synchronize()
    for a, b in zip(want, got + [w, k, v, ke, ve]):
        assert torch.equal(a, b)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured = calls(None)
    for _ in range(2):
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(want, captured + [w, k, v, ke, ve]):
            assert torch.equal(a, b)
    kv.close()


def test_a_captured_call_keeps_its_scratch_when_later_calls_need_theirs():
    k, v, _, _ = ref.make_pages("bf16", 1, 64, 16, 2, 128)
    kv = siso.PagedKV(k, v)
    q = torch.randn((300, 8, 128), device="cuda").to(torch.bfloat16)
    cu, lens, table = i32([0, 300]), i32([1000]), torch.arange(64, **I32)[None]
    lse = torch.full((300, 8), 5.0, device="cuda")
    w = kv.new_weights()
    kv.add_weights(w, q, lse, cu, lens, table, 300, decay=0.0)
    want, blocks = w.clone(), dict(kv._blocks)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        kv.add_weights(w, q, lse, cu, lens, table, 300, decay=0.0)
    for n in (1, 300):
        kv.attention(q[:n], i32([0, n]), lens, table, n)
    assert dict(kv._blocks).keys() == blocks.keys()
    w.zero_()
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(w, want)
    kv.close()


def test_empty_calls_and_refusals():
    kv = siso.PagedKV.allocate(1, 4, 16, 2, 128)
    w = kv.new_weights()
    q = torch.zeros((1, 4, 128), dtype=torch.bfloat16, device="cuda")
    lse = torch.zeros((1, 4), device="cuda")
    cu, lens, table = i32([0, 1]), i32([5]), torch.zeros((1, 4), **I32)
    good = dict(weights=w, q=q, lse=lse, cu_q=cu, kv_len=lens, pages=table, max_q=1)
    kv.add_weights(**good)
    kv.add_weights(**(good | dict(q=q[:0], lse=lse[:0])))
    assert [t.numel() for t in kv.evict(w, lens[:0], table[:0], 4, 1)] == [0, 0]
    for bad in (dict(weights=w.double()), dict(weights=w[0]), dict(weights=w.transpose(2, 3)), dict(q=q.float()), dict(lse=lse[0]), dict(lse=lse.double()), dict(cu_q=cu[:1]),
                dict(kv_len=lens.long()), dict(pages=table[0])):
        with pytest.raises(ValueError):
            kv.add_weights(**(good | bad))
    for bad in (dict(layer=1), dict(scale=NAN), dict(decay=-0.5), dict(decay=NAN), dict(decay=math.inf), dict(max_q=-1)):
        assert status_of(kv.add_weights, **(good | bad)) == 1
    assert status_of(kv.add_weights, **(good | dict(q=q[:, :3].contiguous(), lse=lse[:, :3].contiguous()))) == 1      # 3 heads over 2
    for budget, recent in ((0, 0), (4, 5), (4, -1), (-2, -3)):
        with pytest.raises(ValueError):
            kv.evict(w, lens, table, budget, recent)
    for bad in (dict(weights=w[:, :2]), dict(kv_len=lens.long()), dict(out_pages=table.long()), dict(out_pages=torch.zeros((2, 4), **I32))):
        with pytest.raises(ValueError):
            kv.evict(**(dict(weights=w, kv_len=lens, pages=table, budget=4, recent=1) | bad))
    kv.close()
    wide = siso.PagedKV.allocate(1, 4, 16, 2, 96)                 # evicted from, but not attended over
    assert status_of(wide.add_weights, wide.new_weights(), torch.zeros((1, 4, 96), dtype=torch.bfloat16, device="cuda"), lse, cu, lens, table, 1) == 2
    wide.close()
