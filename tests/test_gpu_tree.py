"""Trees of drafted tokens: ancestors, attention over the paged cache, verification and the accepted path, against plain statements in 64 bits.
Ancestors, verification and the path are exact; the attention's tolerance is that of test_gpu_paged, derived there (the mask changes which tokens are
summed over, not how)."""
import gc
import math

import pytest
import torch

import paged_ref as ref
import tree_ref as tree
from test_gpu_paged import check_attention
from test_gpu_paged_edges import filled

pytestmark = pytest.mark.gpu

siso = pytest.importorskip("paper_2508_18736_b200")
I32 = dict(dtype=torch.int32, device="cuda")


def some_tree(n, seed, kind="random"):
    g = torch.Generator().manual_seed(seed)
    if kind == "chain":
        return list(range(-1, n - 1))
    if kind == "star":
        return [-1] + [0] * (n - 1)
    return [-1] + [int(torch.randint(0, i, (1,), generator=g)) for i in range(1, n)]


def i32(x):
    return torch.tensor(x, **I32)


@pytest.fixture(scope="module", autouse=True)
def nothing_left_behind():
    """Tests of refusals that keep an exception leave tensors to the cycle collector; those that compare the allocator's figures come after this module."""
    yield
    gc.collect()


def status_of(call, *args, **kwargs):
    """The status that a call is refused with (0: it is not).  Unlike a kept exception, this leaves no cycle through the caller's frame, whose tensors would
    stay until a collection at some later time."""
    try:
        call(*args, **kwargs)
    except siso.SisoError as e:
        return e.status
    return 0


# ---- ancestors -----------------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("sizes,words", [([1], 1), ([9, 0, 33, 64, 2], 2), ([65, 200], 7), ([40, 70], 1), ([5000], 157), ([300] * 40, 12)])
@pytest.mark.parametrize("kind", ["random", "chain", "star"])
def test_ancestors(sizes, words, kind):
    if kind == "chain" and max(sizes) > 4000:
        sizes, words = [4200], 132
    parents = [some_tree(n, i, kind) if n else [] for i, n in enumerate(sizes)]
    if kind == "random":
        parents[0][0] = 7                                     # no earlier node: none
        if len(parents[-1]) > 40:
            parents[-1][40], parents[-1][33] = -5, 33
    cu = [sum(sizes[:i]) for i in range(len(sizes) + 1)]
    flat = i32(sum(parents, []))
    mask, depth = siso.tree_mask(flat, i32(cu), 32 * words)
    assert mask.shape == (cu[-1], words)
    for p, lo, hi in zip(parents, cu, cu[1:]):
        if hi > lo:
            up, d = tree.ancestors(p)
            assert torch.equal(depth[lo:hi].cpu(), d.to(torch.int32))
            assert torch.equal(mask[lo:hi].cpu(), tree.words_of(up, words))


def test_ancestors_of_strided_and_uncovered_rows():
    flat = i32([9, -1, 0, 0, 2, 9, 9])[::1]
    wide = torch.stack([flat, flat], 1)[:, 0]                  # stride 2
    mask, depth = siso.tree_mask(wide, i32([1, 5]), 4)
    assert mask[1:5, 0].tolist() == [1, 3, 5, 13] and depth[1:5].tolist() == [0, 1, 1, 2]
    assert siso.tree_mask(flat[:0], i32([0, 0]), 4)[0].shape == (0, 1) and siso.tree_mask(flat, i32([0]), 4)[0].shape == (7, 1)


# ---- attention -----------------------------------------------------------------------------------------------------------
def run_tree(kind, dim, heads, kv_heads, page, lens, sizes, window=0, rows="tree", head_major=False, hint=None, words=None, wide=False, scale=None, gain=1.0):
    """Every place beyond a sequence's tokens is NaN.  rows: what the new tokens see: their ancestors, or random bits with some rows empty."""
    g = torch.Generator(device="cuda").manual_seed(11)
    held = [-(-max(n, 0) // page) for n in lens]
    pages = sum(held) + 2
    k, v, ke, ve = ref.make_pages(kind, 2, pages, page, kv_heads, dim, head_major, fill="nan")
    kv = siso.PagedKV(k, v, ke, ve)
    order = torch.randperm(pages, device="cuda", generator=g).to(torch.int32)
    table = torch.full((len(lens), max(held) + 1), -1, **I32)
    at, truth = 0, []
    for b, n in enumerate(lens):
        table[b, :held[b]] = order[at:at + held[b]]
        at += held[b]
        new = [torch.randn((n, kv_heads, dim), device="cuda", generator=g) for _ in range(2)]
        i = torch.arange(n, device="cuda")
        kv.write(new[0], new[1], table[b].long()[i // page] * page + i % page, layer=1)
        truth.append([r.to(torch.bfloat16).double() if kind == "bf16" else ref.values(*ref.quantised(r, kind)) for r in new])
    cu = [sum(sizes[:i]) for i in range(len(sizes) + 1)]
    q = (gain * torch.randn((cu[-1], heads, dim), device="cuda", generator=g)).to(torch.bfloat16)
    parents = [some_tree(n, b, ("random", "chain", "star")[b % 3]) if n else [] for b, n in enumerate(sizes)]
    words = words or max(1, -(-max(sizes) // 32))
    sees = [tree.ancestors(p)[0] if p else torch.zeros((0, 0), dtype=torch.bool) for p in parents]
    if rows == "bits":
        gc = torch.Generator().manual_seed(5)
        sees = [torch.rand((n, n), generator=gc) < torch.rand((n, 1), generator=gc) for n in sizes]
        for s in sees:
            s[::3] = False
        mask = torch.cat([tree.words_of(torch.cat([s, torch.ones((s.shape[0], 32 * words), dtype=torch.bool)], 1), words) for s in sees]).cuda()   # bits of no node too
    else:
        mask, depth = siso.tree_mask(i32(sum(parents, [])), i32(cu), 32 * words)
    if wide:
        mask = torch.cat([mask, torch.full((cu[-1], 3), -1, **I32)], 1)[:, :words]
    for s in sees:
        s[:, 32 * words:] = False
    args = (q, i32(cu), i32(lens), table, mask, max(sizes) if hint is None else hint)
    got, lse = kv.tree_attention(*args, layer=1, window=window, want_lse=True, scale=scale)
    assert kv.sync_status() == 0
    again, lse2 = kv.tree_attention(*args, layer=1, window=window, want_lse=True, scale=scale)
    assert torch.equal(got, again) and torch.equal(lse, lse2), "two calls differ"
    for b, n in enumerate(lens):
        lo, hi = cu[b], cu[b + 1]
        if hi > lo:
            want = tree.attention(q[lo:hi], truth[b][0], truth[b][1], tree.seen_of(sees[b], n, window), scale)
            check_attention(got[lo:hi], lse[lo:hi], want, dim)
    kv.close()


@pytest.mark.parametrize("kind", ["bf16", "e4m3", "i8"])
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("heads,kv_heads,page,sizes", [
    (8, 2, 16, [1, 2, 1, 2]), (8, 4, 48, [4, 3, 1, 0]), (4, 1, 8, [8, 5, 1, 7]), (8, 2, 32, [16, 9, 2, 13]),          # 8, 8, 32 and 64 rows
    (7, 1, 24, [31, 33, 18, 1]), (4, 4, 64, [64, 65, 129, 32]), (24, 2, 128, [40, 100, 22, 0]), (2, 2, 16, [257, 300, 40, 129])])
def test_trees(kind, dim, heads, kv_heads, page, sizes):
    run_tree(kind, dim, heads, kv_heads, page, [sizes[0] + 130, sizes[1], sizes[2] + 127, sizes[3] + 700], sizes, head_major=page in (32, 64))


@pytest.mark.parametrize("kind", ["bf16", "i8"])
@pytest.mark.parametrize("sizes", [[5, 8, 1], [30, 17, 64], [150, 260, 33]])
@pytest.mark.parametrize("window", [0, 3, 130])
def test_any_bits_and_rows_that_see_nothing(kind, sizes, window):
    # the second sequence has no tokens before the new ones: rows without bits see nothing there
    run_tree(kind, 128, 8, 2, 16, [sizes[0] + 200, sizes[1], sizes[2] + 61], sizes, window=window, rows="bits", wide=True)
    run_tree(kind, 64, 4, 2, 32, [sizes[0] + 200, sizes[1], sizes[2] + 61], sizes, window=window, rows="bits")


@pytest.mark.parametrize("kind", ["bf16", "e4m3"])
@pytest.mark.parametrize("sizes", [[6, 8, 7], [50, 64, 33], [130, 257, 90]])
@pytest.mark.parametrize("window", [1, 40, 2000, 2 ** 31 - 1])
def test_windows(kind, sizes, window):
    run_tree(kind, 128, 8, 2, 48, [sizes[0] + 300, sizes[1] + 1, sizes[2] + 1200], sizes, window=window)


@pytest.mark.parametrize("hint", [0, 1, 1 << 20])
def test_any_hint(hint):
    run_tree("bf16", 128, 8, 2, 32, [900, 130, 40], [70, 1, 13], hint=hint)
    run_tree("i8", 64, 8, 2, 32, [900, 130, 40], [70, 1, 13], hint=hint, window=33)


@pytest.mark.parametrize("sizes", [[7, 3], [40, 3], [200, 3]])
def test_long_sequences_are_split_and_joined(sizes):
    run_tree("bf16", 128, 4, 1, 64, [20011, 3], sizes)
    run_tree("e4m3", 64, 4, 1, 64, [30001, 3], sizes, window=9000)


@pytest.mark.parametrize("sizes", [[20, 8], [60, 70]])
def test_nodes_beyond_the_masks_columns_are_not_seen_and_more_nodes_than_tokens(sizes):
    run_tree("bf16", 128, 8, 2, 16, [500, 90], [max(sizes[0], 40), sizes[1]], words=1)
    # the first nodes stand before the sequence's start
    run_tree("bf16", 64, 8, 2, 16, [sizes[0] // 2, 90], sizes)
    run_tree("i8", 128, 4, 2, 16, [sizes[0] // 2, 0], sizes, window=5)


@pytest.mark.parametrize("sizes", [[9, 4], [48, 30]])
def test_steep_flat_and_reversed_scores(sizes):
    run_tree("bf16", 128, 8, 2, 32, [900, 130], sizes, gain=40.0)
    run_tree("bf16", 64, 8, 2, 32, [900, 130], sizes, scale=0.0)
    run_tree("e4m3", 128, 8, 2, 32, [900, 130], sizes, scale=-0.2)


@pytest.mark.parametrize("n", [3, 12, 40, 150])
def test_a_chain_is_a_causal_chunk(n):
    kv, table, k, v = filled("bf16", 700, 16, 2, 128)
    q = torch.randn((n, 8, 128), device="cuda").to(torch.bfloat16)
    cu, lens = i32([0, n]), i32([700])
    mask, depth = siso.tree_mask(i32(some_tree(n, 0, "chain")), cu, n)
    assert torch.equal(depth, torch.arange(n, **I32))
    for window in (0, 90):
        a, b = kv.attention(q, cu, lens, table, n, want_lse=True, window=window)
        c, d = kv.tree_attention(q, cu, lens, table, mask, n, want_lse=True, window=window)
        want = ref.attention(q, k, v, n, True, window) if not window or n <= window else None
        if want:
            check_attention(c, d, want, 128)
            assert (a.float() - c.float()).abs().max() <= 2.0 ** -7 * a.float().abs().max()
    kv.close()


@pytest.mark.parametrize("n", [6, 90])
def test_pages_before_the_window_are_not_looked_up_and_bad_ones_are_reported(n):
    page, total = 16, 600
    kv, table, k, v = filled("bf16", total, page, 2, 128)
    q = torch.randn((n, 8, 128), device="cuda").to(torch.bfloat16)
    parents = some_tree(n, 3)
    mask, _ = siso.tree_mask(i32(parents), i32([0, n]), n)
    window = 100
    gone = (total - n - window + 1) // page
    given_back = table.clone()
    given_back[0, :gone] = -1
    up = tree.ancestors(parents)[0]
    for t, ok in ((given_back, True), (table, True)):
        out, lse = kv.tree_attention(q, i32([0, n]), i32([total]), t, mask, n, window=window, want_lse=True)
        assert kv.sync_status() == 0
        check_attention(out, lse, tree.attention(q, k, v, tree.seen_of(up, total, window)), 128)
    given_back[0, gone + 1] = 10 ** 6
    kv.tree_attention(q, i32([0, n]), i32([total]), given_back, mask, n, window=window)
    assert kv.sync_status() == 1
    kv.close()


@pytest.mark.parametrize("n", [4, 20, 90])
def test_rows_that_no_sequence_covers_and_strided_outputs(n):
    kv, table, k, v = filled("e4m3", 300, 16, 2, 64)
    q = torch.randn((n + 5, 8, 64), device="cuda").to(torch.bfloat16)
    q[:2], q[n + 2:] = math.nan, math.nan
    cu = i32([2, n + 2])
    mask, _ = siso.tree_mask(i32([9, 9] + some_tree(n, 1) + [9] * 3), cu, n)
    wide = torch.full((8, n + 5, 72), 7.0, dtype=torch.bfloat16, device="cuda")
    out = wide.transpose(0, 1)[:, :, :64]
    got = kv.tree_attention(q, cu, i32([300]), table, mask, n, out=out)
    assert got is out and (wide[:, :2] == 7).all() and (wide[:, n + 2:] == 7).all() and (wide[:, :, 64:] == 7).all()
    o, _, mass, _ = tree.attention(q[2:n + 2], k, v, tree.seen_of(tree.ancestors(some_tree(n, 1))[0], 300, 0))
    assert ((got[2:n + 2].double() - o).abs() <= 2.0 ** -8 * o.abs() + 1.02 * mass * 2.0 ** -8 + 1e-4 * mass).all()
    kv.close()


# ---- verification ----------------------------------------------------------------------------------------------------------
def drafted(sizes, vocab, dtype, probs, seed, kinds=("random", "chain", "star")):
    g = torch.Generator(device="cuda").manual_seed(seed)
    n = sum(sizes)
    cu = [sum(sizes[:i]) for i in range(len(sizes) + 1)]
    parents = sum((some_tree(m, seed + b, kinds[b % len(kinds)]) if m else [] for b, m in enumerate(sizes)), [])
    logits = 2.0 * torch.randn((n, vocab), device="cuda", generator=g)
    target = torch.softmax(logits, -1)
    draft = torch.softmax(logits + 0.4 * torch.randn((n, vocab), device="cuda", generator=g), -1) if probs else None
    pick = draft if probs else target ** 2 + 1e-30
    rows = torch.tensor([lo + max(p, 0) for lo, hi in zip(cu, cu[1:]) for p in parents[lo:hi]], device="cuda")
    tokens = torch.multinomial(pick[rows], 1, generator=g)[:, 0].to(torch.int32)
    u = torch.rand(n, device="cuda", generator=g)
    return (target.to(dtype), None if draft is None else draft.to(dtype), tokens, i32(parents), i32(cu), u, torch.rand(len(sizes), device="cuda", generator=g)), cu


def check_verified(args, cu, max_path):
    target, draft, tokens, parents, c, u, us = args
    got = siso.verify_tree(target, draft, tokens, parents, c, max_path, u, us)
    want = tree.verify_tree(target, draft, tokens, parents, cu, max_path, u, us)
    for a, b in zip(got, want):
        assert torch.equal(a.cpu(), b)
    return got


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("probs", [True, False])
@pytest.mark.parametrize("sizes,vocab,max_path", [([1], 1, 1), ([3, 1, 0, 5], 17, 2), ([9, 30, 2, 64, 13], 1000, 12), ([40] * 20, 333, 5), ([7, 12], 50257, 6),
                                                  ([16, 31], 128256, 8), ([25], 262144, 8), ([700, 20], 64, 40)])
def test_verification_is_exact(dtype, probs, sizes, vocab, max_path):
    for seed in range(3):
        args, cu = drafted(sizes, vocab, dtype, probs, 10 * seed + vocab)
        if seed == 1:
            args[5].mul_(0.4)                 # longer paths
        if seed == 2:
            args[5].fill_(1 - 2.0 ** -24)     # nearly every draft falls
            args[6][-1] = 1 - 2.0 ** -24
        check_verified(args, cu, max_path)


def test_verification_at_its_edges():
    for probs in (True, False):
        args, cu = drafted([6, 9, 12, 5, 8], 40, torch.float32, probs, 3)
        target, draft, tokens, parents, c, u, us = args
        tokens[7], tokens[9] = -1, 40                    # outside the vocabulary
        parents[16:20] = i32([0, -3, 99, 2])             # without a parent, or one that does not come before it
        tokens[28:31] = tokens[27]                       # the same token several times
        parents[27:31] = 0
        target[0] = 0.0                                  # nothing to draw from
        target[6, 3] = math.nan
        if probs:
            draft[6, 4] = math.nan
        target[15, ::2] = 0.0
        us[1], us[2] = 0.0, 1 - 2.0 ** -24
        for longest in (0, 1, 3, 8, 20):
            check_verified(args, cu, longest)
        u.fill_(0.999)
        check_verified(args, cu, 8)
        u.zero_()
        check_verified(args, cu, 8)
    none = siso.verify_tree(target[:0], None, tokens[:0], parents[:0], i32([0, 0]), 2, u[:0], us[:1])
    assert none[0].tolist() == [[-1, -1, -1]] and none[1].tolist() == [0] and none[2].tolist() == [[-1, -1]]
    assert siso.verify_tree(target, None, tokens, parents, i32([0]), 2, u, us[:0])[0].shape == (0, 3)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("probs", [True, False])
def test_a_chain_gives_what_the_verification_of_a_chain_gives(dtype, probs):
    seqs, n, vocab = 50, 5, 1003
    args, cu = drafted([n + 1] * seqs, vocab, dtype, probs, 9, kinds=("chain",))
    target, draft, tokens, parents, c, u, us = args
    u.mul_(0.7)
    out, accepted, path = siso.verify_tree(target, draft, tokens, parents, c, n, u, us)
    by = lambda t: t.view(seqs, n + 1, *t.shape[1:])
    out2, accepted2 = siso.verify_drafts(by(target), None if draft is None else by(draft)[:, :n].contiguous(), by(tokens)[:, 1:].contiguous(), None,
                                         by(u)[:, 1:].contiguous(), us)
    assert torch.equal(out, out2) and torch.equal(accepted, accepted2)
    assert torch.equal(path, torch.where(torch.arange(n, device="cuda") < accepted[:, None], torch.arange(1, n + 1, device="cuda"), -1).to(torch.int32))


@pytest.mark.parametrize("probs", [True, False])
def test_verified_tokens_are_distributed_as_the_target(probs):
    # root with three children drawn from q (or certain and distinct): the first token out must follow p whatever they are.  100,000 sequences: the share of a
    # token has a standard deviation of at most sqrt(0.25 / 100000) = 0.0016; five of them
    g = torch.Generator(device="cuda").manual_seed(4)
    vocab, seqs = 10, 100_000
    p, q = (torch.softmax(torch.randn(vocab, device="cuda", generator=g), -1) for _ in range(2))
    tokens = torch.multinomial(q, 3 * seqs, replacement=True, generator=g).view(seqs, 3) if probs else torch.rand((seqs, vocab), device="cuda", generator=g).argsort(-1)[:, :3]
    tokens = torch.cat([torch.zeros((seqs, 1), device="cuda"), tokens], 1).to(torch.int32).reshape(-1)
    parents = i32([-1, 0, 0, 0]).repeat(seqs)
    cu = torch.arange(seqs + 1, **I32) * 4
    rows = lambda x: x.expand(4 * seqs, vocab).contiguous()
    out, n, path = siso.verify_tree(rows(p), rows(q) if probs else None, tokens, parents, cu, 2, torch.rand(4 * seqs, device="cuda", generator=g),
                                    torch.rand(seqs, device="cuda", generator=g))
    share = torch.bincount(out[:, 0].long(), minlength=vocab).double() / seqs
    assert (share - p.double()).abs().max() < 0.008 and int(n.max()) == 1 and int(path.max()) == 3


# ---- the accepted path -------------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("kind", ["bf16", "e4m3", "i8"])
@pytest.mark.parametrize("dim,heads,page,layers,head_major", [(128, 8, 16, 3, False), (64, 2, 48, 1, True), (8, 3, 8, 2, False), (72, 1, 8, 2, True), (256, 2, 32, 2, False)])
def test_the_path_moves_to_its_place(kind, dim, heads, page, layers, head_major):
    sizes, lens = [1, 9, 40, 0, 130, 6, 3], [5, 9, 100, 30, 300, 77, 2]          # (the last: more nodes than tokens, refused)
    paths = [[], [1, 2, 5, 8], [7, 8, 9, 39], [], list(range(3, 130, 1)), [5], [1]]
    longest = 130
    held = [-(-n // page) for n in lens]
    k, v, ke, ve = ref.make_pages(kind, layers, sum(held) + 2, page, heads, dim, head_major, seed=3)
    kv = siso.PagedKV(k, v, ke, ve)
    order = torch.randperm(sum(held) + 2, device="cuda").to(torch.int32)
    table = torch.full((len(lens), max(held)), -1, **I32)
    for b, h in enumerate(held):
        table[b, :h] = order[sum(held[:b]):sum(held[:b]) + h]
    before = [t.clone() if t is not None else None for t in (k, v, ke, ve)]
    path = torch.full((len(lens), longest), -1, **I32)
    for b, p in enumerate(paths):
        path[b, :len(p)] = i32(p)
    accepted = i32([len(p) for p in paths])
    cu = i32([sum(sizes[:i]) for i in range(len(sizes) + 1)])
    new = kv.keep_path(path, accepted, cu, i32(lens), table)
    assert kv.sync_status() == 1 and kv.sync_status() == 0                        # the last sequence
    assert new.tolist() == [5, 5, 65, 30, 298, 73, 2]
    for x, old, exps in ((k, before[0], False), (v, before[1], False), (ke, before[2], True), (ve, before[3], True)):
        if x is None:
            continue
        want = old.clone().view(torch.int8 if x.dtype != torch.bfloat16 else x.dtype)
        old = old.view(want.dtype)
        for b, p in enumerate(paths[:-1]):
            for t, node in enumerate(p):
                (p0, t0), (p1, t1) = ((int(table[b, j // page]), j % page) for j in (lens[b] - sizes[b] + node, lens[b] - sizes[b] + 1 + t))
                if exps:
                    want[:, p1, :, t1] = old[:, p0, :, t0]
                else:
                    want[:, p1, t1] = old[:, p0, t0]
        assert torch.equal(x.view(want.dtype), want)
    kv.close()


def test_paths_that_do_not_ascend_end_and_are_reported():
    k, v, _, _ = ref.make_pages("bf16", 1, 8, 16, 2, 64, seed=3)
    kv = siso.PagedKV(k, v)
    table, cu, lens = torch.arange(8, **I32).view(2, 4), i32([0, 20, 40]), i32([40, 50])
    for path, accepted, want in (([[3, 2, 5], [1, 2, 3]], [3, 3], [22, 34]), ([[3, 20, 5], [1, 1, 3]], [3, 2], [22, 32]), ([[0, 2, 5], [-1, 2, 3]], [3, 1], [21, 31]),
                                 ([[3, 5, 0], [4, 2 ** 31 - 1, 3]], [3, 2], [23, 32]), ([[-2 ** 31, -2 ** 31 + 1, -5], [-9, -8, 1]], [3, 3], [21, 31])):
        assert kv.keep_path(i32(path), i32(accepted), cu, lens, table).tolist() == want and kv.sync_status() == 1
    assert kv.keep_path(i32([[2, 3, 4], [1, 2, 3]]), i32([-4, 99]), cu, lens, table).tolist() == [21, 34] and kv.sync_status() == 0
    bad = table.clone()
    bad[0, 1] = 8                                          # the path's rows lie there
    old = k.clone()
    assert kv.keep_path(i32([[2, 3, 4], [1, 2, 3]]), i32([3, 0]), cu, lens, bad).tolist() == [24, 31] and kv.sync_status() == 1
    assert torch.equal(k, old)
    assert kv.keep_path(torch.empty((2, 0), **I32), i32([0, 5]), cu, lens, table).tolist() == [21, 31] and kv.sync_status() == 0
    kv.close()


# ---- streams, graphs, refusals -------------------------------------------------------------------------------------------------
def test_calls_run_on_the_stream_they_are_given_and_can_be_captured():
    k, v, ke, ve = ref.make_pages("e4m3", 2, 40, 32, 2, 128)
    kv = siso.PagedKV(k, v, ke, ve)
    n = 48
    args, cu = drafted([20, 28], 5003, torch.float32, True, 5)
    target, draft, tokens, parents, c, u, us = args
    q = torch.randn((n, 8, 128), device="cuda").to(torch.bfloat16)
    lens, table = i32([500, 600]), torch.arange(40, **I32).view(2, 20)
    state = [t.clone() for t in (k.view(torch.int8), v.view(torch.int8), ke, ve)]

    def calls(stream):
        for t, s in zip((k.view(torch.int8), v.view(torch.int8), ke, ve), state):
            t.copy_(s)
        mask, depth = siso.tree_mask(parents, c, 28, stream=stream)
        out = kv.tree_attention(q, c, lens, table, mask, 28, layer=1, stream=stream)
        got = siso.verify_tree(target, draft, tokens, parents, c, 8, u, us, stream=stream)
        return [mask, depth, out, *got, kv.keep_path(got[2], got[1], c, lens, table, stream=stream)]

    want = [t.clone() for t in calls(None)] + [k.view(torch.int8).clone(), ke.clone()]
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        got = calls(s)
    s.synchronize()
    for a, b in zip(want, got + [k.view(torch.int8), ke]):
        assert torch.equal(a, b)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured = calls(None)
    for _ in range(2):
        for t in captured:
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(want, captured + [k.view(torch.int8), ke]):
            assert torch.equal(a, b)
    kv.close()


def test_refusals():
    kv = siso.PagedKV.allocate(1, 4, 16, 2, 128)
    q = torch.zeros((2, 4, 128), dtype=torch.bfloat16, device="cuda")
    cu, lens, table, mask = i32([0, 2]), i32([9]), torch.zeros((1, 4), **I32), i32([[1], [3]])
    for bad in (mask.long(), mask[:1], mask[:, 0], mask[:, :0], mask.cpu()):
        with pytest.raises(ValueError):
            kv.tree_attention(q, cu, lens, table, bad, 2)
    for kwargs in (dict(layer=1), dict(window=-1), dict(scale=math.nan)):
        assert status_of(kv.tree_attention, q, cu, lens, table, mask, 2, **kwargs) == 1
    path, accepted = i32([[1]]), i32([1])
    for bad in (dict(path=path.long()), dict(path=path[0]), dict(accepted=i32([1, 1])), dict(kv_len=lens.long()), dict(cu_q=cu[:1]), dict(pages=table[0])):
        with pytest.raises(ValueError):
            kv.keep_path(**(dict(path=path, accepted=accepted, cu_q=cu, kv_len=lens, pages=table) | bad))
    kv.close()
    good = dict(target=torch.ones((2, 8), device="cuda"), draft=None, tokens=i32([0, 1]), parents=i32([-1, 0]), cu_q=cu, max_path=1, u_accept=torch.zeros(2, device="cuda"),
                u_sample=torch.zeros(1, device="cuda"))
    siso.verify_tree(**good)
    for bad in (dict(target=good["target"].double()), dict(draft=torch.ones((1, 8), device="cuda")), dict(tokens=i32([0])), dict(parents=i32([0, 0]).long()), dict(cu_q=i32([0])),
                dict(max_path=-1), dict(u_sample=torch.zeros(2, device="cuda")), dict(u_accept=torch.zeros(2))):
        with pytest.raises(ValueError):
            siso.verify_tree(**(good | bad))
    assert status_of(siso.verify_tree, **(good | dict(target=torch.empty((2, (1 << 18) + 1), device="cuda")))) == 2
    for bad in (dict(parents=good["parents"].long()), dict(cu_q=cu.cpu()), dict(parents=good["parents"].view(1, 2))):
        with pytest.raises(ValueError):
            siso.tree_mask(**(dict(parents=good["parents"], cu_q=cu, max_nodes=2) | bad))
