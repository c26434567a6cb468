"""The semantic cache, the paged key/value cache, the attention over it and the verification run together (examples/near_hit_drafts.py)."""
import importlib.util
import os

import pytest
import torch

import paged_ref as ref

pytestmark = pytest.mark.gpu

siso = pytest.importorskip("paper_2508_18736_b200")
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def example():
    spec = importlib.util.spec_from_file_location("near_hit_drafts", os.path.join(ROOT, "examples", "near_hit_drafts.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


@pytest.mark.parametrize("kind", ["bf16", "e4m3", "i8"])
def test_a_near_hit_saves_passes(kind):
    model, near, alone, passes, drafted = example().main(kind, length=32, verbose=False)
    assert near and alone == 32 and passes < alone and drafted.shape == (32,)
    model.kv.close()


def test_the_model_over_the_paged_cache_agrees_with_plain_attention():
    # one pass over all tokens with plain attention in 64 bits (bf16 in and out, as the kernel has) against prompt, drafts and single tokens over
    # the cache.  Rounding of the layers' bf16 values, 2^-8 each, is what separates them; probabilities agree within 3 % of the largest
    m = example()
    model = m.Decoder(kind="bf16")
    tokens = torch.randint(0, 512, (75,), device="cuda", generator=torch.Generator(device="cuda").manual_seed(5))
    parts, seen = [], 0
    for n in (50, 1, 5, 1, 18):
        parts.append(model.probabilities(tokens[seen:seen + n], seen))
        seen += n

    def plain(layer, q, k, v):
        return ref.attention(q, k.double(), v.double(), q.shape[0])[0].to(torch.bfloat16)

    want = model.probabilities(tokens, 0, attend=plain)
    assert (torch.cat(parts) - want).abs().max() < 0.03 * want.max()
    model.kv.check_status()
    model.kv.close()
