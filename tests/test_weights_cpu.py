"""What of the attention weights and of the tree's dealing of work needs no GPU: refusals of the C entry points before any launch, and that the model of the dealing
goes by the kernels' numbers."""
import os
import re

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2508_18736_b200", "csrc")


def test_the_entry_points_refuse_a_call_without_a_handle():
    siso = pytest.importorskip("paper_2508_18736_b200")
    lib = siso.load_library()
    assert lib.siso_kv_add_weights_new(None, None, None, None) == 1 and lib.siso_kv_add_weights(None, None, None) == 1


def test_the_model_of_the_dealing_goes_by_the_kernels_numbers():
    # test_tree_cpu's test_no_run_within_an_item_is_without_a_unit models how units are dealt, with 6 or 5 for a tile and 20 for an item's beginning and end (trees over
    # bf16), and a unit each and one more for an item (weights).  Here they are read from the kernels' sources
    read = lambda name: re.sub(r"\s+", " ", open(os.path.join(CSRC, name)).read())
    tc, shared, weights = read("kv_attention_tc.cu"), read("kv_attention.cuh"), read("kv_weights.cu")
    w, more = re.search(r"constexpr int W = HALF \? (\d+) : 1, MORE = HALF \? (\d+) : EXTRA;", tc).groups()
    part = re.search(r"return HALF && rows <= MR / 2 \? W - W / (\d+) : W;", shared).group(1)
    assert int(w) == 6 and int(w) - int(w) // int(part) == 5 and int(more) == 20
    assert "const int most = __any_sync(0xFFFFFFFFu, __syncthreads_or(full) != 0) ? W : W - W / 6;" in shared and "max(run.total / most, 1ll)" in shared
    assert "return tiles - first_tile(g, kb) + 1;" in weights and "(total + 1) / 2" in weights and "full) * (tiles + 1);" in weights
