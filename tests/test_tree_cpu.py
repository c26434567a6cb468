"""What of the trees of drafts and of the eviction needs no GPU: the definitions that the GPU tests compare with, and the refusals."""
import ctypes
import math

import pytest
import torch

import paged_ref as ref
import tree_ref as tree


def test_ancestors_and_their_words():
    up, depth = tree.ancestors([-1, 0, 0, 2, 7, 4])
    assert depth.tolist() == [0, 1, 1, 2, 0, 1]
    assert tree.words_of(up, 2).tolist() == [[1, 0], [3, 0], [5, 0], [13, 0], [16, 0], [48, 0]]
    assert tree.words_of(torch.ones((1, 40), dtype=torch.bool), 1).tolist() == [[-1]]


def test_a_chain_is_verified_as_drafts_are():
    g = torch.Generator().manual_seed(3)
    seqs, n, vocab = 30, 4, 50
    logits = 2 * torch.randn((seqs, n + 1, vocab), generator=g)
    target, guess = torch.softmax(logits, -1), torch.softmax(logits + torch.randn(logits.shape, generator=g), -1)
    tokens = torch.multinomial(guess[:, :n].reshape(-1, vocab), 1, generator=g).view(seqs, n).to(torch.int32)
    u, us = torch.rand((seqs, n), generator=g) * 0.7, torch.rand(seqs, generator=g)
    pad = lambda x: torch.cat([torch.zeros_like(x[:, :1]), x], 1).reshape(-1)
    for draft in (guess, None):
        want = ref.verify(target, None if draft is None else draft[:, :n], tokens, None, u, us)
        got = tree.verify_tree(target.view(-1, vocab), None if draft is None else draft.reshape(-1, vocab), pad(tokens), torch.arange(-1, n).repeat(seqs),
                               list(range(0, seqs * (n + 1) + 1, n + 1)), n, pad(u), us)
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


def test_a_verified_tree_follows_the_target():
    # a root with two children, drawn from q by themselves: over all pairs of children and a grid of uniform numbers the first token out follows p
    p, q, n = torch.tensor([0.5, 0.25, 0.125, 0.125]), torch.tensor([0.25, 0.5, 0.125, 0.125]), 12
    grid = (torch.arange(n) + 0.5) / n
    a, b, s = (x.reshape(-1) for x in torch.meshgrid(grid, grid, grid, indexing="ij"))
    share = torch.zeros(4, dtype=torch.float64)
    rows = n ** 3
    for x in range(4):
        for y in range(4):
            out, _, _ = tree.verify_tree(p.repeat(3 * rows, 1), q.repeat(3 * rows, 1), torch.tensor([0, x, y]).repeat(rows), torch.tensor([-1, 0, 0]).repeat(rows),
                                         list(range(0, 3 * rows + 1, 3)), 1, torch.stack([a, a, b], 1).reshape(-1), s)
            share += float(q[x] * q[y]) * torch.bincount(out[:, 0].long(), minlength=4).double() / rows
    assert (share - p.double()).abs().max() <= 3.0 / n


def test_which_tokens_stay():
    w = torch.tensor([3.0, math.nan, 1.0, 3.0, -math.inf, 2.0, 9.0])
    assert tree.kept(w, 7, 2) == list(range(7)) and tree.kept(w, 4, 2) == [0, 3, 5, 6] and tree.kept(w, 3, 2) == [0, 5, 6]
    assert tree.kept(w, 6, 1) == [0, 2, 3, 4, 5, 6] and tree.kept(w, 2, 2) == [5, 6] and tree.kept(w, 1, 0) == [6]


def test_tensors_on_the_cpu_are_refused():
    siso = pytest.importorskip("paper_2508_18736_b200")
    i = torch.zeros(2, dtype=torch.int32)
    with pytest.raises(ValueError):
        siso.tree_mask(i, i, 4)
    with pytest.raises(ValueError):
        siso.verify_tree(torch.zeros((2, 8)), None, i, i, i, 1, torch.zeros(2), torch.zeros(1))


def test_the_c_entry_points_refuse_bad_arguments_before_any_launch():
    siso = pytest.importorskip("paper_2508_18736_b200")
    lib = siso.load_library()
    big = ctypes.c_void_p(256)
    assert lib.siso_tree_mask(None, None, 1, 1, 1, None, None, None) == 1 and lib.siso_tree_mask(big, big, 1, 1, 0, big, None, None) == 1
    assert lib.siso_tree_mask(big, big, -1, 1, 1, big, None, None) == 1 and lib.siso_tree_mask(None, None, 0, 1, 1, None, None, None) == 0
    assert lib.siso_tree_mask(big, big, 1 << 31, 1, 1, big, None, None) == 2
    assert lib.siso_kv_tree_attention(None, None, None, 1, 1, None) == 1
    args = [big, None, 0, 4, 1, 8, big, big, big, 2, big, big, big, big, big, None]

    def verify(**change):
        a = list(args)
        for k, x in change.items():
            a[int(k[1:])] = x
        return lib.siso_verify_tree(*a)
    for change in (dict(a2=2), dict(a3=-1), dict(a4=-1), dict(a5=0), dict(a9=-1), dict(a0=None), dict(a6=None), dict(a7=None), dict(a8=None), dict(a10=None), dict(a11=None),
                   dict(a12=None), dict(a13=None)):
        assert verify(**change) == 1, change
    assert verify(a5=(1 << 18) + 1) == 2 and verify(a3=1 << 31) == 2 and verify(a4=0) == 0
    assert lib.siso_kv_keep_path(None, big, big, 1, big, big, big, 1, 1, 1, big, None) == 1
    assert lib.siso_kv_add_weights(None, None, None) == 1
    assert lib.siso_kv_evict(None, big, big, big, 1, 1, big, 1, 1, 1, 4, 1, big, big, None) == 1


def test_no_run_within_an_item_is_without_a_unit():
    # how units are dealt to CTAs, as a model: an item cut at runs' borders has a part in every run from its first unit's to its last one's, which is what the kernels that join parts
    # count on.  Trees over bf16: tiles of 6 (5 where no sequence has more), 20 more for an item; weights: a unit each and one more for an item
    import bisect
    import random
    rng = random.Random(1)

    def holds(starts, total, ctas):
        borders = [total * c // ctas for c in range(ctas + 1)]
        return all(set(range(o[0], o[-1] + 1)) == set(o) for o in ([bisect.bisect_right(borders, s) - 1 for s in item] for item in starts))

    for _ in range(4000):
        grid = rng.choice([3, 17, 148])
        only_half = rng.random() < 0.3
        at, starts, most = 0, [], 5
        for _ in range(rng.randint(1, 12)):
            cost, tiles = (5 if only_half or rng.random() < 0.5 else 6), rng.randint(1, rng.choice([3, 20, 60]))
            most = max(most, cost)
            starts.append([at + 20 + cost * k for k in range(tiles)])
            at += 20 + cost * tiles
        assert holds(starts, at, min(grid, max(at // most, 1)))
        at, starts = 0, []
        for _ in range(rng.randint(1, 12)):
            n = rng.randint(1, rng.choice([2, 9, 200]))
            starts.append([at] + [at + k + 1 for k in range(1, n)])
            at += n + 1
        assert holds(starts, at, min(grid, (at + 1) // 2))
