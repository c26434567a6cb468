"""What of the paged key/value cache and the verification needs no GPU: the definitions that the GPU tests compare with, and the refusals."""
import math

import pytest
import torch

import paged_ref as ref


@pytest.mark.parametrize("kind", ["e4m3", "i8"])
def test_a_row_keeps_its_largest_value_within_its_type_and_rounds_once(kind):
    g = torch.Generator().manual_seed(2)
    x = torch.randn((400, 64), generator=g) * torch.exp2(torch.randint(-100, 100, (400, 1), generator=g).float())
    x[0] = 0
    codes, exps = ref.quantised(x, kind)
    y = ref.values(codes, exps)
    top = x.double().abs().amax(-1)
    scale = torch.exp2(exps.double() - 127)
    assert (top <= ref.TOP[kind] * scale).all() and (top > ref.TOP[kind] * scale / 2)[1:].all() and exps[0] == 0
    step = scale[:, None] if kind == "i8" else torch.maximum(torch.exp2(torch.floor(torch.log2(x.double().abs().clamp(min=1e-300)))) / 8, scale[:, None] * 2.0 ** -9)
    assert ((y - x.double()).abs() <= step / 2 * (1 + 1e-12)).all()
    assert torch.equal(y.to(torch.bfloat16).double(), y), "a stored value is a bf16 value"


def test_a_row_that_is_not_finite_is_marked():
    x = torch.ones((3, 16))
    x[1, 3], x[2, 0] = math.inf, math.nan
    codes, exps = ref.quantised(x, "i8")
    assert exps.tolist() == [127 - 6, 255, 255] and torch.isnan(ref.values(codes, exps)[1:]).all()


def test_verified_drafts_follow_the_target():
    # one draft drawn from q, verified against p: the first token out follows p exactly when summed over every draft and every uniform number
    # on a grid (the acceptance and the draw are piecewise constant in them)
    p, q = torch.tensor([0.5, 0.25, 0.125, 0.125]), torch.tensor([0.25, 0.25, 0.25, 0.25])
    n = 64
    u = (torch.arange(n) + 0.5) / n
    share = torch.zeros(4, dtype=torch.float64)
    for x in range(4):
        a, s = torch.meshgrid(u, u, indexing="ij")
        rows = n * n
        out, _ = ref.verify(p.expand(rows, 2, 4), q.expand(rows, 1, 4), torch.full((rows, 1), x), None, a.reshape(-1, 1), s.reshape(-1))
        share += 0.25 * torch.bincount(out[:, 0].long(), minlength=4).double() / rows
    assert (share - p.double()).abs().max() <= 2.0 / n


def test_pages_on_the_cpu_are_refused():
    siso = pytest.importorskip("paper_2508_18736_b200")
    k = torch.zeros((1, 2, 8, 1, 64), dtype=torch.bfloat16)
    with pytest.raises(RuntimeError):
        siso.PagedKV(k, k)
    with pytest.raises(ValueError):
        siso.PagedKV(k.float(), k.float())
    with pytest.raises(ValueError):
        siso.PagedKV(k[0], k[0])
    with pytest.raises(ValueError):
        siso.PagedKV(k, k, torch.zeros((1, 2, 1, 8), dtype=torch.uint8), None)
    with pytest.raises(ValueError):
        siso.verify_drafts(torch.zeros((1, 2, 4)), None, torch.zeros((1, 1), dtype=torch.int32), None, torch.zeros((1, 1)), torch.zeros(1))


def test_the_c_entry_points_refuse_bad_arguments_before_any_launch():
    import ctypes
    siso = pytest.importorskip("paper_2508_18736_b200")
    lib = siso.load_library()
    out = ctypes.c_void_p()
    assert lib.siso_kv_create(ctypes.byref(out), None) == 1 and not out.value
    assert lib.siso_kv_destroy(None) == 1 and lib.siso_kv_sync_status(None, None) == 1
    assert lib.siso_kv_write(None, 0, None, None, 0, 1, 64, 64, None, None) == 1
    assert lib.siso_kv_read(None, 0, None, None, 0, 1, 64, 64, None, None) == 1
    assert lib.siso_kv_attention(None, None, None) == 1
    none = [None] * 6
    assert lib.siso_verify_drafts(None, None, 0, 1, 1, 8, *none, None) == 1           # NULL pointers
    assert lib.siso_verify_drafts(None, None, 2, 1, 1, 8, *none, None) == 1           # probabilities in 8 bits
    assert lib.siso_verify_drafts(None, None, 0, 1, -1, 8, *none, None) == 1
    assert lib.siso_verify_drafts(None, None, 0, 0, 1, 8, *none, None) == 0           # no sequences: nothing to do
    big = ctypes.c_void_p(256)
    assert lib.siso_verify_drafts(big, None, 0, 1, 1, (1 << 24) + 1, big, None, big, big, big, big, None) == 2
