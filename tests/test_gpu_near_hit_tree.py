"""The semantic cache, a tree of several near hits' stored answers, its attention, verification and accepted path, and the eviction from the prompt's cache run
together (examples/near_hit_tree.py)."""
import importlib.util
import os

import pytest
import torch

import paged_ref as ref
import tree_ref as tree

pytestmark = pytest.mark.gpu

siso = pytest.importorskip("paper_2508_18736_b200")
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def example():
    spec = importlib.util.spec_from_file_location("near_hit_tree", os.path.join(ROOT, "examples", "near_hit_tree.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


@pytest.mark.parametrize("kind", ["bf16", "e4m3", "i8"])
@pytest.mark.parametrize("budget", [None, 12])
def test_near_hits_save_passes(kind, budget):
    model, near, alone, passes, drafted = example().main(kind, length=32, budget=budget, verbose=False)
    assert len(near) == 2 and alone == 32 and passes < alone and drafted.shape == (32,)
    model.kv.close()


def test_a_node_has_the_probabilities_of_its_path():
    # a tree below a prompt against each node's path by itself as a causal chunk over plain attention in 64 bits.  Rounding of the layers' bf16 values, 2^-8 each, is
    # what separates them; probabilities agree within 3 % of the largest
    m = example()
    model = m.TreeDecoder(kind="bf16")
    g = torch.Generator(device="cuda").manual_seed(5)
    prompt = torch.randint(0, 512, (41,), device="cuda", generator=g)
    model.start(prompt)
    parents = [-1, 0, 1, 1, 0, 4, 2, 6, 0, 8]
    tokens = torch.cat([prompt[-1:], torch.randint(0, 512, (9,), device="cuda", generator=g)])
    got = model.nodes(tokens, parents)

    def plain(layer, q, k, v):
        return ref.attention(q, k.double(), v.double(), q.shape[0])[0].to(torch.bfloat16)

    up, depth = tree.ancestors(parents)
    for node in range(10):
        path = torch.cat([prompt[:-1], tokens[up[node].cuda()]])
        want = model.probabilities(path, 0, attend=plain)[-1]
        assert (got[node] - want).abs().max() < 0.03 * want.max()
    model.kv.check_status()
    model.kv.close()


def test_shared_beginnings_are_in_the_tree_once():
    tokens, parents = example().tree_of([[5, 6, 7, 8], [5, 6, 9], [4]], 3)
    assert tokens == [5, 6, 7, 9, 4] and parents == [0, 1, 2, 2, 0]
