"""What of the attention weights needs no GPU: refusals of the C entry points before any launch."""
import pytest


def test_the_entry_points_refuse_a_call_without_a_handle():
    siso = pytest.importorskip("paper_2508_18736_b200")
    lib = siso.load_library()
    assert lib.siso_kv_add_weights_new(None, None, None, None) == 1 and lib.siso_kv_add_weights(None, None, None) == 1
