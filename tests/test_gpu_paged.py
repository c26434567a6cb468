"""The paged key/value cache, attention over it and draft verification against plain statements in 64 bits.

Tolerances.  Writing, reading and verification are exact.  Attention: a probability is rounded once to bf16 (unit roundoff 2^-8) before
it meets the values and the result is rounded once to bf16; a score's fp32 sum of dim products is off by at most
dim 2^-24 sum |q||k| scale, which moves exp by that much relatively, in numerator and denominator; the exponential and the
sums add less than 2^-18.  With A = sum p |v|:
    |out - exact| <= 2^-8 |exact| + (1 + 2^-7) A (2^-8 + 2 d + 2^-18),   |lse - exact| <= d + 2^-20 (1 + |exact|),   d = (dim + 8) 2^-24 max sum |q||k| scale
"""
import math

import pytest
import torch

import paged_ref as ref

pytestmark = pytest.mark.gpu

siso = pytest.importorskip("paper_2508_18736_b200")
NAN = math.nan


def check_attention(out, lse, want, dim):
    o, l, mass, ab = want
    d = (dim + 8) * 2.0 ** -24 * ab
    tol = 2.0 ** -8 * o.abs() + (1 + 2.0 ** -7) * mass * (2.0 ** -8 + 2 * d + 2.0 ** -18) + 1e-30
    assert torch.isfinite(out).all()
    assert ((out.double() - o).abs() <= tol).all(), float(((out.double() - o).abs() / tol).max())
    none = l == -math.inf
    assert torch.equal(lse == -math.inf, none) and (out[none] == 0).all()
    assert ((lse.double() - l).abs()[~none] <= d + 2.0 ** -20 * (1 + l.abs()[~none])).all()


def run_case(kind, dim, heads, kv_heads, page, lens, q_lens, causal=True, window=0, head_major=False, layers=1, gain=1.0, scale=None, hint=None,
             strided=False):
    """Builds pages in which every place beyond a sequence's tokens is NaN, runs the attention and compares it."""
    g = torch.Generator(device="cuda").manual_seed(7)
    held = [-(-max(n, 0) // page) for n in lens]
    pages = sum(held) + 2
    layer = layers - 1
    k, v, ke, ve = ref.make_pages(kind, layers, pages, page, kv_heads, dim, head_major, fill="nan")
    kv = siso.PagedKV(k, v, ke, ve)
    order = torch.randperm(pages, device="cuda", generator=g).to(torch.int32)
    table = torch.full((len(lens), max(held) + 1), -1, dtype=torch.int32, device="cuda")
    at, n_q = 0, sum(q_lens)
    truth = []
    for b, n in enumerate(lens):
        table[b, :held[b]] = order[at:at + held[b]]
        at += held[b]
        rows = [torch.randn((n, kv_heads, dim), device="cuda", generator=g) for _ in range(2)]
        i = torch.arange(n, device="cuda")
        slots = table[b].long()[i // page] * page + i % page
        kv.write(rows[0], rows[1], slots, layer=layer)
        if kind == "bf16":
            truth.append([r.to(torch.bfloat16).double() for r in rows])
        else:
            truth.append([ref.values(*ref.quantised(r, kind)) for r in rows])
    q = (gain * torch.randn((n_q, heads, dim), device="cuda", generator=g)).to(torch.bfloat16)
    out = None
    if strided:
        wide = torch.randn((n_q, heads + 3, dim + 16), device="cuda", generator=g).to(torch.bfloat16)
        wide[:, 1:1 + heads, 8:8 + dim] = q
        q = wide[:, 1:1 + heads, 8:8 + dim]
        out = torch.full((heads, n_q, dim + 8), 7.0, dtype=torch.bfloat16, device="cuda").transpose(0, 1)[:, :, :dim]
    cu = torch.tensor([sum(q_lens[:i]) for i in range(len(lens) + 1)], dtype=torch.int32, device="cuda")
    kv_len = torch.tensor(lens, dtype=torch.int32, device="cuda")
    args = (q, cu, kv_len, table, max(q_lens) if hint is None else hint)
    more = dict(layer=layer, scale=scale, causal=causal, window=window, want_lse=True)
    got, lse = kv.attention(*args, out=out, **more)
    assert kv.sync_status() == 0
    again, lse2 = kv.attention(*args, **more)
    assert torch.equal(got, again) and torch.equal(lse, lse2), "two calls differ"
    for b, n in enumerate(lens):
        lo, hi = int(cu[b]), int(cu[b + 1])
        if hi > lo:
            want = ref.attention(q[lo:hi], truth[b][0], truth[b][1], hi - lo, causal, window, scale)
            check_attention(got[lo:hi], lse[lo:hi], want, dim)
    kv.close()


# ---- the cache -----------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("kind", ["bf16", "e4m3", "i8"])
@pytest.mark.parametrize("source", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("dim,heads,page,n,head_major", [(128, 8, 16, 1, False), (64, 1, 8, 77, True), (96, 3, 24, 130, False), (256, 2, 64, 33, True),
                                                         (8, 5, 8, 19, False)])
def test_rows_are_quantised_as_defined_and_read_back(kind, source, dim, heads, page, n, head_major):
    g = torch.Generator(device="cuda").manual_seed(n)
    pages = -(-n // page) + 2
    k, v, ke, ve = ref.make_pages(kind, 2, pages, page, heads, dim, head_major, seed=1)
    before = [t.clone() for t in (k, v)]
    kv = siso.PagedKV(k, v, ke, ve)
    fused = (torch.randn((n, 3 * heads * dim), device="cuda", generator=g) * torch.exp2(torch.randint(-40, 40, (n, 1), device="cuda", generator=g).float())).to(source)
    kr, vr = (fused[:, i * heads * dim:(i + 1) * heads * dim].view(n, heads, dim) for i in (1, 2))
    kr[n // 2, 0], vr[n // 3, heads - 1] = 0, 1e-42               # rows of zeros and of values below the normal range
    slots = torch.randperm(pages * page, device="cuda", generator=g)[:n]
    skipped = torch.rand(n, device="cuda", generator=g) < 0.2
    skipped[0] = False
    used = torch.where(skipped, torch.where(slots % 2 == 0, torch.full_like(slots, -1), pages * page + slots), slots)
    kv.write(kr, vr, used, layer=1)
    for rows, codes, exps, old in ((kr, k, ke, before[0]), (vr, v, ve, before[1])):
        p, t = slots // page, slots % page
        if kind == "bf16":
            assert torch.equal(codes[1][p, t][~skipped], rows.to(torch.bfloat16)[~skipped])
        else:
            c, e = ref.quantised(rows, kind)
            assert torch.equal(codes.view(torch.int8)[1][p, t][~skipped], c.view(torch.int8)[~skipped])
            assert torch.equal(exps[1].transpose(1, 2)[p, t][~skipped], e[~skipped])
        as_bytes = (lambda x: x.view(torch.int8) if kind != "bf16" else x.view(torch.int16))
        assert torch.equal(as_bytes(codes)[0], as_bytes(old)[0]), "another layer changed"
        touched = torch.zeros((pages, page), dtype=torch.bool, device="cuda")
        touched[p[~skipped], t[~skipped]] = True
        assert torch.equal(as_bytes(codes)[1][~touched], as_bytes(old)[1][~touched]), "a place outside the slots changed"
    for dtype in (torch.float32, torch.bfloat16):
        for rows, got in zip((kr, vr), kv.read(used, layer=1, dtype=dtype)):
            want = rows.to(torch.bfloat16).double() if kind == "bf16" else ref.values(*ref.quantised(rows, kind))
            if dtype == torch.float32 or kind == "bf16":
                assert torch.equal(got[~skipped].double(), want[~skipped])
            else:
                assert torch.equal(got[~skipped], want[~skipped].to(torch.bfloat16))
            assert (got[skipped] == 0).all()
    kv.close()


@pytest.mark.parametrize("kind", ["e4m3", "i8"])
def test_rows_that_are_not_finite_read_back_as_nan_and_largest_values_fit(kind):
    kv = siso.PagedKV.allocate(1, 2, 8, 1, 64, ref.TYPES[kind])
    x = torch.randn((6, 1, 64), device="cuda")
    x[0, 0, 5], x[1, 0, 63], x[2, 0, 0] = math.inf, NAN, -math.inf
    x[3] = 3.0e38 * torch.linspace(-1, 1, 64, device="cuda")
    x[4] = ref.TOP[kind] * 2.0 ** -3
    x[5] = torch.nextafter(torch.tensor(ref.TOP[kind], device="cuda"), torch.tensor(1e9, device="cuda"))
    slots = torch.arange(6, device="cuda")
    kv.write(x, x, slots)
    got = kv.read(slots, dtype=torch.float32)[0]
    assert torch.isnan(got[:3]).all() and torch.isfinite(got[3:]).all()
    assert torch.equal(got[3:].double(), ref.values(*ref.quantised(x[3:], kind)))
    assert torch.equal(got[4], x[4]) and kv.k_exp[0, 0, 0, 5] == 128
    kv.close()


def test_a_long_pool_is_addressed_beyond_32_bits():
    page, heads, dim = 64, 8, 128
    pages = (1 << 31) // (page * heads * dim) + 40                # over 2^31 elements of one layer
    k = torch.empty((1, pages, page, heads, dim), dtype=torch.int8, device="cuda")
    exps = [torch.full((1, pages, heads, page), 255, dtype=torch.uint8, device="cuda") for _ in range(2)]
    kv = siso.PagedKV(k, torch.empty_like(k), *exps)
    g = torch.Generator(device="cuda").manual_seed(3)
    n = 3 * page + 5
    table = torch.tensor([[pages - 1, 2, pages - 7, pages - 2]], dtype=torch.int32, device="cuda")
    i = torch.arange(n, device="cuda")
    slots = table[0].long()[i // page] * page + i % page
    rows = [torch.randn((n, heads, dim), device="cuda", generator=g) for _ in range(2)]
    kv.write(*rows, slots)
    want = [ref.values(*ref.quantised(r, "i8")) for r in rows]
    for a, b in zip(kv.read(slots, dtype=torch.float32), want):
        assert torch.equal(a.double(), b)
    for n_q in (1, 150):
        q = torch.randn((n_q, 4 * heads, dim), device="cuda", generator=g).to(torch.bfloat16)
        cu, lens = (torch.tensor(x, dtype=torch.int32, device="cuda") for x in ([0, n_q], [n]))
        out, lse = kv.attention(q, cu, lens, table, n_q, want_lse=True)
        check_attention(out, lse, ref.attention(q, *want, n_q), dim)
    kv.close()


# ---- attention -----------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("kind", ["bf16", "e4m3", "i8"])
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("heads,kv_heads,page", [(8, 2, 16), (7, 1, 48), (4, 4, 8), (24, 2, 128)])
def test_single_tokens(kind, dim, heads, kv_heads, page):
    run_case(kind, dim, heads, kv_heads, page, [1, 2, 17, 63, 64, 65, 127, 128, 129, 700, 0, 1999], [1] * 10 + [1, 1])


@pytest.mark.parametrize("kind", ["bf16", "e4m3", "i8"])
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("heads,kv_heads,page,window", [(8, 2, 32, 0), (7, 1, 24, 100), (3, 3, 64, 0), (16, 1, 16, 1)])
def test_short_chunks(kind, dim, heads, kv_heads, page, window):
    run_case(kind, dim, heads, kv_heads, page, [5, 9, 300, 257, 64, 3, 1030], [5, 2, 7, 0, 16, 3, 11], window=window, head_major=page == 32)


@pytest.mark.parametrize("kind", ["bf16", "e4m3", "i8"])
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("heads,kv_heads,page,lens,q_lens,window", [
    (4, 1, 64, [130, 511], [130, 257], 0),
    (8, 2, 16, [1025, 640, 90], [300, 1, 90], 0),
    (5, 1, 48, [777], [401], 0),
    (6, 2, 128, [1500, 400], [256, 380], 200),
    (2, 2, 8, [1300], [1300], 0),
    (40, 1, 32, [500, 31], [33, 31], 64),
])
def test_long_chunks(kind, dim, heads, kv_heads, page, lens, q_lens, window):
    run_case(kind, dim, heads, kv_heads, page, lens, q_lens, window=window, head_major=page in (16, 128), layers=2)


@pytest.mark.parametrize("q_len,n", [(1, 70), (6, 333), (200, 1024)])
@pytest.mark.parametrize("kind", ["bf16", "i8"])
def test_without_causality_and_with_strides(kind, q_len, n):
    run_case(kind, 128, 8, 2, 32, [n, n // 2], [q_len, q_len], causal=False, strided=True)
    run_case(kind, 64, 8, 2, 32, [n, n // 2], [q_len, q_len], causal=False, window=50, strided=True)


@pytest.mark.parametrize("q_len", [1, 8, 260])
def test_rows_that_see_nothing(q_len):
    # more new tokens than the cache holds: the first ones stand before its start; and no tokens at all
    run_case("bf16", 128, 8, 2, 16, [q_len // 2, 0, 700], [q_len, q_len, q_len])
    run_case("e4m3", 64, 4, 4, 16, [q_len // 2, 0, 700], [q_len, q_len, q_len], window=3)


@pytest.mark.parametrize("q_len", [1, 190])
def test_steep_and_flat_scores(q_len):
    run_case("bf16", 128, 8, 2, 32, [900, 1300], [q_len, q_len], gain=40.0)            # scores up to several hundred
    run_case("bf16", 64, 8, 2, 32, [900, 1300], [q_len, q_len], scale=0.0)             # all alike
    run_case("e4m3", 128, 8, 2, 32, [900, 1300], [q_len, q_len], scale=-0.2)


@pytest.mark.parametrize("hint", [0, 1, 1 << 20])
def test_any_hint_gives_the_result(hint):
    run_case("bf16", 128, 8, 2, 32, [900, 130, 40], [150, 1, 13], hint=hint)
    run_case("i8", 64, 8, 2, 32, [900, 130, 40], [150, 1, 13], hint=hint)


@pytest.mark.parametrize("q_len", [1, 9, 140])
def test_long_sequences_are_split_and_joined(q_len):
    run_case("bf16", 128, 4, 1, 64, [20011, 3], [q_len, min(q_len, 3)])
    run_case("e4m3", 64, 4, 1, 64, [30001, 3], [q_len, min(q_len, 3)])


@pytest.mark.parametrize("kind,heads,window", [("bf16", 8, 0), ("e4m3", 8, 700)])
def test_a_prompt_of_many_row_tiles(kind, heads, window):
    # 21,000 tokens x 8 heads: more row tiles than the kernel has threads.  Rows at the start, in the middle and at the end are compared
    n, page, dim = 21_000, 64, 64
    held = -(-n // page)
    k, v, ke, ve = ref.make_pages(kind, 1, held, page, 1, dim, seed=9)
    kv = siso.PagedKV(k, v, ke, ve)
    table = torch.randperm(held, device="cuda").to(torch.int32)[None]
    slots = (table[0].long()[:, None] * page + torch.arange(page, device="cuda")).reshape(-1)[:n]
    rows = [r.double() for r in kv.read(slots, dtype=torch.float32)]
    q = torch.randn((n, heads, dim), device="cuda").to(torch.bfloat16)
    cu, lens = (torch.tensor(x, dtype=torch.int32, device="cuda") for x in ([0, n], [n]))
    out, lse = kv.attention(q, cu, lens, table, n, window=window, want_lse=True)
    for lo in (0, 63, 10_441, n - 40):
        hi = lo + 40
        want = ref.attention(q[lo:hi], rows[0][:hi], rows[1][:hi], 40, window=window)
        check_attention(out[lo:hi], lse[lo:hi], want, dim)
    assert kv.sync_status() == 0
    kv.close()


@pytest.mark.parametrize("n_q", [1, 100])
def test_page_outside_the_pool_is_reported_and_left_out(n_q):
    page = 16
    k, v, _, _ = ref.make_pages("bf16", 1, 10, page, 2, 128)
    kv = siso.PagedKV(k, v)
    q = torch.randn((n_q, 8, 128), device="cuda").to(torch.bfloat16)
    cu, lens = (torch.tensor(x, dtype=torch.int32, device="cuda") for x in ([0, n_q], [7 * page]))
    for bad in (-1, 10, 2 ** 31 - 1):
        table = torch.tensor([[3, 4, bad, 5, 0, 1, 2]], dtype=torch.int32, device="cuda")
        out, lse = kv.attention(q, cu, lens, table, n_q, causal=False, want_lse=True)
        assert kv.sync_status() == 1 and kv.sync_status() == 0
        kept = [3, 4, 5, 0, 1, 2]
        want = ref.attention(q, k[0, kept].reshape(-1, 2, 128).double(), v[0, kept].reshape(-1, 2, 128).double(), n_q, causal=False)
        check_attention(out, lse, want, 128)
    # a length beyond what the table can hold is cut to it
    table = torch.tensor([[3, 4]], dtype=torch.int32, device="cuda")
    out, lse = kv.attention(q, cu, lens, table, n_q, causal=False, want_lse=True)
    check_attention(out, lse, ref.attention(q, k[0, 3:5].reshape(-1, 2, 128).double(), v[0, 3:5].reshape(-1, 2, 128).double(), n_q, causal=False), 128)
    assert kv.sync_status() == 0
    kv.close()


def test_calls_run_on_the_stream_they_are_given():
    k, v, ke, ve = ref.make_pages("e4m3", 1, 40, 32, 2, 128)
    kv = siso.PagedKV(k, v, ke, ve)
    rows = torch.randn((64, 2, 128), device="cuda")
    slots = torch.arange(64, device="cuda")
    q = torch.randn((64, 8, 128), device="cuda").to(torch.bfloat16)
    cu, lens = (torch.tensor(x, dtype=torch.int32, device="cuda") for x in ([0, 64], [1000]))
    table = torch.arange(40, dtype=torch.int32, device="cuda")[None]
    target = torch.softmax(torch.randn((3, 3, 500), device="cuda"), -1)
    tokens = torch.zeros((3, 2), dtype=torch.int32, device="cuda")
    u = torch.rand((3, 3), device="cuda")

    def calls(stream):
        kv.write(rows, rows, slots, stream=stream)
        return [kv.attention(q, cu, lens, table, 64, stream=stream), *kv.read(slots, stream=stream),
                *siso.verify_drafts(target, None, tokens, None, u[:, :2].contiguous(), u[:, 2].contiguous(), stream=stream)]

    want = calls(None)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    got = calls(s)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):              # a warmed handle takes no memory, so the calls can be captured
        captured = calls(None)
    for t in captured:
        t.zero_()
    graph.replay()
    torch.cuda.synchronize()
    for a, b, c in zip(want, got, captured):
        assert torch.equal(a, b) and torch.equal(a, c)
    kv.close()


def test_empty_calls_and_refusals():
    kv = siso.PagedKV.allocate(1, 4, 16, 2, 128)
    none = torch.empty((0, 2, 128), device="cuda")
    slots = torch.empty(0, dtype=torch.int64, device="cuda")
    kv.write(none, none, slots)
    assert kv.read(slots)[0].shape == (0, 2, 128)
    i32 = dict(dtype=torch.int32, device="cuda")
    cu, lens, table = torch.zeros(2, **i32), torch.zeros(1, **i32), torch.zeros((1, 4), **i32)
    assert kv.attention(torch.empty((0, 4, 128), dtype=torch.bfloat16, device="cuda"), cu, lens, table, 0).shape == (0, 4, 128)
    q = torch.zeros((1, 4, 128), dtype=torch.bfloat16, device="cuda")
    for bad in (q.float(), q[..., :64], q[0]):
        with pytest.raises(ValueError):
            kv.attention(bad, cu, lens, table, 1)
    with pytest.raises(ValueError):
        kv.attention(q, cu.long(), lens, table, 1)
    with pytest.raises(ValueError):
        kv.attention(q, cu, torch.zeros(2, **i32), table, 1)
    for kwargs in (dict(layer=1), dict(layer=-1), dict(window=-1), dict(scale=NAN)):
        with pytest.raises(siso.SisoError) as e:
            kv.attention(q, cu, lens, table, 1, **kwargs)
        assert e.value.status == 1
    with pytest.raises(siso.SisoError) as e:                       # 3 heads over 2
        kv.attention(q[:, :3].contiguous(), cu, lens, table, 1)
    assert e.value.status == 1
    odd = torch.zeros(1 * 4 * 128 + 1, dtype=torch.bfloat16, device="cuda")[1:].view(1, 4, 128)
    with pytest.raises(siso.SisoError) as e:                       # rows off a 16-byte boundary
        kv.attention(odd, cu, lens, table, 1)
    assert e.value.status == 2
    row = torch.zeros((1, 2, 128), device="cuda")
    with pytest.raises(ValueError):
        kv.write(row, row, torch.zeros(1, **i32))
    with pytest.raises(ValueError):
        kv.write(row, row.to(torch.bfloat16), torch.zeros(1, dtype=torch.int64, device="cuda"))
    kv.close()
    wide = siso.PagedKV.allocate(1, 4, 16, 2, 96)                  # stored, but not attended over
    with pytest.raises(siso.SisoError) as e:
        wide.attention(torch.zeros((1, 4, 96), dtype=torch.bfloat16, device="cuda"), cu, lens, table, 1)
    assert e.value.status == 2
    wide.close()
    for page, dim in ((12, 128), (16, 100), (16, 264)):
        with pytest.raises(siso.SisoError) as e:
            siso.PagedKV.allocate(1, 4, page, 2, dim)
        assert e.value.status == 2
    k = torch.zeros((1, 4, 16, 2, 128), dtype=torch.int8, device="cuda")
    with pytest.raises(ValueError):
        siso.PagedKV(k, k)


# ---- verification --------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("probs", [True, False])
@pytest.mark.parametrize("seqs,n_max,vocab", [(1, 1, 1), (3, 5, 17), (70, 3, 1000), (9, 40, 333), (130, 2, 4097), (300, 1, 511), (2, 8, 50257), (1, 3, 160001)])
def test_verification_is_exact(dtype, probs, seqs, n_max, vocab):
    g = torch.Generator(device="cuda").manual_seed(vocab + n_max)
    logits = 2.0 * torch.randn((seqs, n_max + 1, vocab), device="cuda", generator=g)
    target = torch.softmax(logits, -1).to(dtype)
    draft = torch.softmax(logits[:, :n_max] + 0.4 * torch.randn((seqs, n_max, vocab), device="cuda", generator=g), -1).to(dtype) if probs else None
    pick = draft.float() if probs else target[:, :n_max].float() ** 3
    tokens = torch.multinomial(pick.reshape(-1, vocab) + 1e-30, 1, generator=g).view(seqs, n_max).to(torch.int32)
    n_drafts = torch.randint(0, n_max + 1, (seqs,), device="cuda", generator=g, dtype=torch.int32)
    n_drafts[0] = n_max
    u_accept = torch.rand((seqs, n_max), device="cuda", generator=g) * (0.3 if vocab > 100 else 1.0)
    u_sample = torch.rand((seqs,), device="cuda", generator=g)
    u_sample[-1] = 1 - 2.0 ** -24
    for limits in (n_drafts, None):
        out, n = siso.verify_drafts(target, draft, tokens, limits, u_accept, u_sample)
        want, taken = ref.verify(target, draft, tokens, limits, u_accept, u_sample)
        assert torch.equal(n.cpu(), taken) and torch.equal(out.cpu(), want)


def test_verification_at_its_edges():
    f = dict(device="cuda")
    target = torch.tensor([[[0.5, 0.5, 0.0, 0.0], [0.0, 0.0, 0.0, 1.0]]] * 7, **f)
    draft = target[:, :1].clone()
    draft[3] = torch.tensor([0.25, 0.75, 0.0, 0.0])
    target[4, 1] = 0.0                       # nothing to draw from
    target[5, 0, 0] = NAN
    tokens = torch.tensor([[0], [2], [-1], [1], [0], [0], [9]], dtype=torch.int32, **f)
    n_drafts = torch.tensor([1, 1, 1, 1, 1, 1, -3], dtype=torch.int32, **f)
    u_accept = torch.tensor([[0.999]] * 7, **f)
    u_sample = torch.tensor([0.0, 0.6, 0.4, 0.9, 0.5, 0.5, 0.99], **f)
    for d in (draft, None):
        out, n = siso.verify_drafts(target, d, tokens, n_drafts, u_accept, u_sample)
        want, taken = ref.verify(target, d, tokens, n_drafts, u_accept, u_sample)
        assert torch.equal(n.cpu(), taken) and torch.equal(out.cpu(), want)
    assert out[4].tolist() == [-1, -1] or n[4] == 0
    none, n = siso.verify_drafts(target[:, :1], None, tokens[:, :0], None, u_accept[:, :0], u_sample)      # no drafts: a plain draw
    assert torch.equal(none.cpu(), ref.verify(target[:, :1], None, tokens[:, :0], None, u_accept[:, :0], u_sample)[0]) and (n == 0).all()
    assert siso.verify_drafts(target[:0], None, tokens[:0], None, u_accept[:0], u_sample[:0])[0].shape == (0, 2)
    for bad in (dict(target=target.double()), dict(draft=draft.to(torch.bfloat16)), dict(tokens=tokens.long()), dict(u_sample=u_sample[:3])):
        args = dict(target=target, draft=draft, tokens=tokens, n_drafts=n_drafts, u_accept=u_accept, u_sample=u_sample) | bad
        with pytest.raises(ValueError):
            siso.verify_drafts(**args)


def test_verified_tokens_are_distributed_as_the_target():
    # drafts drawn from q, verified against p: the first token out must follow p.  200,000 draws, bins of at least 1 %: the share of a bin
    # has a standard deviation of at most sqrt(0.25 / 200000) = 0.0011; five of them
    g = torch.Generator(device="cuda").manual_seed(11)
    vocab, n = 12, 200_000
    p = torch.softmax(torch.randn(vocab, device="cuda", generator=g), -1)
    q = torch.softmax(torch.randn(vocab, device="cuda", generator=g), -1)
    tokens = torch.multinomial(q, n, replacement=True, generator=g).to(torch.int32)[:, None]
    target, draft = p.expand(n, 2, vocab).contiguous(), q.expand(n, 1, vocab).contiguous()
    out, _ = siso.verify_drafts(target, draft, tokens, None, torch.rand((n, 1), device="cuda", generator=g), torch.rand(n, device="cuda", generator=g))
    share = torch.bincount(out[:, 0].long(), minlength=vocab).double() / n
    assert (share - p.double()).abs().max() < 0.0056
