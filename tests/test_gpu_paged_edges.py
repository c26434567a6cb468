"""The paged key/value cache and what reads it at the edges of their arguments, against the 64-bit statements of paged_ref.  Tolerances are
those of test_gpu_paged, derived there."""
import math

import pytest
import torch

import paged_ref as ref
from test_gpu_paged import check_attention

pytestmark = pytest.mark.gpu

siso = pytest.importorskip("paper_2508_18736_b200")
I32 = dict(dtype=torch.int32, device="cuda")


def filled(kind, n, page, kv_heads, dim, scale=None, holes=False, seed=3, spare=1):
    """A cache that holds n tokens in shuffled pages, whose value rows are `scale` [n] times as large, every second value of large rows zero if
    `holes`: (kv, table [1, pages], keys, values as the cache holds them, in 64 bits)."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    held = -(-n // page)
    kv = siso.PagedKV(*ref.make_pages(kind, 1, held + spare, page, kv_heads, dim, fill="nan"))
    table = torch.randperm(held + spare, device="cuda", generator=g)[:held].to(torch.int32)[None]
    i = torch.arange(n, device="cuda")
    slots = table[0].long()[i // page] * page + i % page
    k, v = (torch.randn((n, kv_heads, dim), device="cuda", generator=g) for _ in range(2))
    if scale is not None:
        v *= scale[:, None, None]
        if holes:
            v[scale > 1, :, ::2] = 0.0
    kv.write(k, v, slots)
    if kind == "bf16":
        return kv, table, k.to(torch.bfloat16).double(), v.to(torch.bfloat16).double()
    return kv, table, ref.values(*ref.quantised(k, kind)), ref.values(*ref.quantised(v, kind))


def attend(kv, table, n, n_q, heads, dim, k, v, gain=1.0, causal=True, window=0, hint=None, seed=4):
    """Attention of the last n_q of n tokens (more than n: the first ones stand before the start) is compared with its statement."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    q = (gain * torch.randn((n_q, heads, dim), device="cuda", generator=g)).to(torch.bfloat16)
    cu, lens = (torch.tensor(x, **I32) for x in ([0, n_q], [n]))
    out, lse = kv.attention(q, cu, lens, table, n_q if hint is None else hint, causal=causal, window=window, want_lse=True)
    assert kv.sync_status() == 0
    check_attention(out, lse, ref.attention(q, k, v, n_q, causal, window), dim)


# ---- value rows of unlike size ------------------------------------------------------------------------------------------------
ROWS = [1, 2, 4, 6, 9]              # queries of 4 heads per kv head: 4, 8, 16, 24 and 36 rows, every kernel and shape


@pytest.mark.parametrize("kind", ["e4m3", "i8"])
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("n_q", ROWS)
@pytest.mark.parametrize("holes", [False, True])
def test_value_rows_of_unlike_size(kind, dim, n_q, holes):
    n = 700
    steps = torch.randint(-40, 41, (n,), device="cuda", generator=torch.Generator(device="cuda").manual_seed(n_q)).float()
    for scale in (torch.exp2(steps), torch.exp2(steps.abs().neg()), torch.exp2(torch.linspace(-60, 60, n, device="cuda").round())):
        kv, table, k, v = filled(kind, n, 16, 2, dim, scale, holes)
        attend(kv, table, n, n_q, 8, dim, k, v)
        kv.close()


@pytest.mark.parametrize("n_q", ROWS)
def test_e4m3_codes_below_the_normal_range(n_q):
    # one large value a row, in the first place; the others are codes of 2^-9 to 7 x 2^-9
    n, dim = 150, 128
    g = torch.Generator(device="cuda").manual_seed(n_q)
    kv = siso.PagedKV.allocate(1, 10, 16, 1, dim, torch.float8_e4m3fn)
    k = torch.randn((n, 1, dim), device="cuda", generator=g)
    v = torch.randint(1, 8, (n, 1, dim), device="cuda", generator=g) * 2.0 ** -9 * torch.where(torch.rand((n, 1, dim), device="cuda", generator=g) < 0.5, -1.0, 1.0)
    v[:, :, 0] = 448.0
    kv.write(k, v, torch.arange(n, device="cuda"))
    assert torch.equal(kv.read(torch.arange(n, device="cuda"), dtype=torch.float32)[1], v)
    attend(kv, torch.arange(10, **I32)[None], n, n_q, 4, dim, ref.values(*ref.quantised(k, "e4m3")), v.double())
    kv.close()


@pytest.mark.parametrize("kind", ["e4m3", "i8"])
@pytest.mark.parametrize("n_q,window", [(2, 1), (8, 3), (9, 0), (9, 5), (60, 40)])
def test_large_value_rows_that_a_query_does_not_see(kind, n_q, window):
    # the first token of all, the one before the window of the last query, and the last token, which only the last query sees
    n, dim = 300, 128
    scale = torch.ones(n, device="cuda")
    scale[[0, n - 1 - (window or 1), n - 1]] = 2.0 ** 40
    kv, table, k, v = filled(kind, n, 16, 1, dim, scale)
    attend(kv, table, n, n_q, 4, dim, k, v, window=window)
    kv.close()


@pytest.mark.parametrize("kind", ["bf16", "e4m3", "i8"])
@pytest.mark.parametrize("n_q", ROWS)
def test_small_probabilities_where_the_large_ones_meet_zeros(kind, n_q):
    # every second value of the heavy rows is zero: what the light ones give stands alone there, however small it is
    n, dim, kv_heads = 200, 128, 2
    g = torch.Generator(device="cuda").manual_seed(1)
    kv = siso.PagedKV.allocate(1, -(-n // 16), 16, kv_heads, dim, ref.TYPES[kind])
    k, v = (torch.randn((n, kv_heads, dim), device="cuda", generator=g) for _ in range(2))
    k[::7] += 2.0
    v[::7, :, ::2] = 0.0
    slots = torch.arange(n, device="cuda")
    kv.write(k, v, slots)
    table = torch.arange(-(-n // 16), **I32)[None]
    k, v = (x.to(torch.bfloat16).double() if kind == "bf16" else ref.values(*ref.quantised(x, kind)) for x in (k, v))
    q = torch.full((n_q, 8, dim), 1.5, dtype=torch.bfloat16, device="cuda")        # heavy rows: scores higher by about 34
    cu, lens = (torch.tensor(x, **I32) for x in ([0, n_q], [n]))
    out, lse = kv.attention(q, cu, lens, table, n_q, want_lse=True)
    check_attention(out, lse, ref.attention(q, k, v, n_q), dim)
    kv.close()


# ---- windows ---------------------------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("kind", ["bf16", "i8"])
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("window", [2 ** 31 - 1, 2 ** 31 - 700, 1500, 1300, 1299])
@pytest.mark.parametrize("n,n_q", [(1300, 1), (1300, 6), (1300, 150), (1300, 1300), (5, 8), (100, 260)])
def test_windows_as_long_as_the_sequence_and_longer(kind, causal, window, n, n_q):
    kv, table, k, v = filled(kind, n, 32, 2, 64)
    attend(kv, table, n, n_q, 8, 64, k, v, causal=causal, window=window)
    kv.close()


@pytest.mark.parametrize("kind", ["bf16", "e4m3", "i8"])
@pytest.mark.parametrize("page", [8, 48, 64, 128])
@pytest.mark.parametrize("n_q,window", [(1, 100), (1, 1), (7, 300), (20, 77), (300, 50)])
def test_pages_before_the_window_may_be_gone(kind, page, n_q, window):
    # pages that end before the first query's window: every other one released, the others in other hands (all NaN); and NaN in the
    # places of the window's first page that lie before it
    n, dim = 1000, 128
    kv, table, k, v = filled(kind, n, page, 2, dim, spare=2)
    lo = n - n_q - window + 1
    kv.write(torch.full((lo, 2, dim), math.nan, device="cuda"), torch.full((lo, 2, dim), math.nan, device="cuda"),
             (table[0].long()[:, None] * page + torch.arange(page, device="cuda")).reshape(-1)[:lo])
    table[0, :lo // page:2] = -1
    attend(kv, table, n, n_q, 8, dim, k, v, window=window)
    kv.close()


# ---- verification ----------------------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("seqs", [1, 3, 17, 70, 300, 600])          # clusters of 8, 8, 8, 4, 2 and 1 CTAs
@pytest.mark.parametrize("n_max,vocab", [(0, 1), (0, 40), (1, 1), (2, 9)])
def test_short_rows_are_shared_by_ctas_that_have_all_started(seqs, n_max, vocab):
    # almost nothing stands between a CTA's start and what it writes to its neighbours; many calls, one close behind the other
    g = torch.Generator(device="cuda").manual_seed(seqs + vocab)
    target = torch.softmax(torch.randn((seqs, n_max + 1, vocab), device="cuda", generator=g), -1)
    tokens = torch.randint(0, vocab, (seqs, n_max), device="cuda", generator=g, dtype=torch.int32)
    u_accept, u_sample = torch.rand((seqs, n_max), device="cuda", generator=g), torch.rand(seqs, device="cuda", generator=g)
    calls = [siso.verify_drafts(target, None, tokens, None, u_accept, u_sample) for _ in range(50)]
    want, taken = ref.verify(target, None, tokens, None, u_accept, u_sample)
    for out, n in calls:
        assert torch.equal(out.cpu(), want) and torch.equal(n.cpu(), taken)


# ---- streams ---------------------------------------------------------------------------------------------------------------------
def spread(t):
    """The same values, not contiguous."""
    wide = torch.zeros((*t.shape, 2), dtype=t.dtype, device=t.device)
    wide[..., 0] = t
    return wide[..., 0]


@pytest.mark.parametrize("what", ["rows", "queries", "lengths", "drafts"])
@pytest.mark.parametrize("busy", ["the current stream", "the given stream"])
def test_arguments_that_are_copied_belong_to_the_given_stream(what, busy):
    # the current stream busy: the copies must not wait there while the kernel runs; the given one busy: the copies must not be given back to
    # the current stream, which writes over what it can get, before the kernel has run
    g = torch.Generator(device="cuda").manual_seed(5)
    n, n_q, heads, dim, page = 400, 7, 8, 128, 16
    kv, table, k, v = filled("bf16", n, page, 2, dim)
    s = torch.cuda.Stream()
    rows = [torch.randn((n, 2, dim), device="cuda", generator=g) for _ in range(2)]
    i = torch.arange(n, device="cuda")
    slots = table[0].long()[i // page] * page + i % page
    q = torch.randn((n_q, heads, dim), device="cuda", generator=g).to(torch.bfloat16)
    cu, lens = (torch.tensor(x, **I32) for x in ([0, 3, n_q], [n, n - 50]))
    tables = table.repeat(2, 1)
    target = torch.softmax(torch.randn((5, 4, 2000), device="cuda", generator=g), -1)
    draft = torch.softmax(torch.randn((5, 3, 2000), device="cuda", generator=g), -1)
    tokens = torch.randint(0, 2000, (5, 3), device="cuda", generator=g, dtype=torch.int32)
    n_drafts, u, u_sample = torch.tensor([3, 2, 0, 3, 1], **I32), torch.rand((5, 3), device="cuda", generator=g), torch.rand(5, device="cuda", generator=g)

    def call(f, stream):
        if what == "rows":
            kv.write(f(rows[0]), f(rows[1]), f(slots), stream=stream)
            return kv.read(f(slots), stream=stream)
        if what == "queries":
            return kv.attention(f(q), cu, lens, tables, 4, want_lse=True, stream=stream)
        if what == "lengths":
            return kv.attention(q, f(cu), f(lens), f(tables), 4, want_lse=True, stream=stream)
        return siso.verify_drafts(f(target), f(draft), f(tokens), f(n_drafts), f(u), f(u_sample), stream=stream)

    want = [t.clone() for t in call(lambda t: t, None)]
    for _ in range(3):
        ready = {}                                    # the arguments are there, not contiguous, before the streams become busy
        call(lambda t: ready.setdefault(id(t), spread(t)), None)
        if what == "rows":
            kv.write(torch.zeros_like(rows[0]), torch.zeros_like(rows[1]), slots)
        torch.cuda.synchronize()
        with torch.cuda.stream(torch.cuda.current_stream() if busy == "the current stream" else s):
            torch.cuda._sleep(40_000_000)             # about 20 ms
        got = call(lambda t: ready[id(t)], s)
        if busy == "the given stream":                # what the call gave back is overwritten
            over = [torch.full((m,), 0x7F, dtype=torch.uint8, device="cuda") for m in (1 << 9, 1 << 12, 1 << 14, 1 << 16, 200_000, 1 << 18, 1 << 20) for _ in range(6)]
        s.synchronize()
        for a, b in zip(got, want):
            assert torch.equal(a, b)
        torch.cuda.synchronize()
        over = None
    kv.close()


def test_a_stream_of_another_device_is_refused():
    kv = siso.PagedKV.allocate(1, 4, 16, 2, 128)
    other = torch.cuda.ExternalStream(torch.cuda.Stream().cuda_stream, device=torch.device("cuda", 0))
    kv.read(torch.zeros(1, dtype=torch.int64, device="cuda"), stream=other)

    class Elsewhere:
        device_index, cuda_stream = 1, 0

    with pytest.raises(ValueError):
        kv.read(torch.zeros(1, dtype=torch.int64, device="cuda"), stream=Elsewhere())
    kv.close()


# ---- waits -----------------------------------------------------------------------------------------------------------------------
def test_a_wait_that_runs_out_is_reported_and_the_handle_goes_on():
    kv, table, k, v = filled("i8", 300, 16, 2, 128)
    kv.selftest_wait_timeout()
    assert kv.sync_status() == 6 and kv.sync_status() == 0          # SISO_ERR_TIMEOUT, once
    attend(kv, table, 300, 2, 8, 128, k, v)
    attend(kv, table, 300, 60, 8, 128, k, v)
    kv.close()


# ---- devices ---------------------------------------------------------------------------------------------------------------------
@pytest.mark.skipif(torch.cuda.device_count() < 2, reason="needs two GPUs")
def test_calls_leave_the_current_device_as_it_was():
    kv = siso.PagedKV.allocate(1, 4, 16, 2, 128, device=1)
    here = dict(device="cuda:1")
    slots, row = torch.zeros(1, dtype=torch.int64, **here), torch.randn((1, 2, 128), **here)
    q, one = torch.zeros((1, 4, 128), dtype=torch.bfloat16, **here), torch.ones(1, dtype=torch.int32, **here)
    for call in (lambda: kv.write(row, row, slots), lambda: kv.read(slots),
                 lambda: kv.attention(q, torch.cat([one - 1, one]), one, (one - 1)[None], 1), lambda: kv.sync_status(), lambda: kv.close()):
        call()
        assert torch.cuda.current_device() == 0


# ---- strides ---------------------------------------------------------------------------------------------------------------------
def test_pages_whose_entries_share_a_place_are_refused():
    one = torch.zeros((2, 4, 16, 2, 64), dtype=torch.bfloat16, device="cuda")
    for dim in range(4):
        shared = one.narrow(dim, 0, 1).expand(one.shape)
        with pytest.raises(siso.SisoError) as e:
            siso.PagedKV(shared, shared.clone().narrow(dim, 0, 1).expand(one.shape))
        assert e.value.status == 2
        siso.PagedKV(one.narrow(dim, 0, 1 if dim != 2 else 8), one.clone().narrow(dim, 0, 1 if dim != 2 else 8)).close()


def any_stride(t, dim, stride):
    """t, whose dimension `dim` has one entry, with another stride there."""
    assert t.shape[dim] == 1
    s = list(t.stride())
    s[dim] = stride
    return t.as_strided(t.shape, s)


@pytest.mark.parametrize("kind", ["bf16", "e4m3"])
@pytest.mark.parametrize("stride", [0, 1, 83])
def test_strides_of_one_entry_count_for_nothing(kind, stride):
    # one layer, one kv head, one token: a row of a projection whose width is odd, pages turned out of another order
    n, dim, page = 20, 64, 32
    k, v, ke, ve = ref.make_pages(kind, 1, 1, page, 1, dim, fill="nan")
    for d in (0, 1, 3):
        k, v = any_stride(k, d, stride), any_stride(v, d, stride)
    kv = siso.PagedKV(k, v, ke, ve)
    rows = [torch.randn((n, 1, dim), device="cuda") for _ in range(2)]
    slots = torch.arange(n, device="cuda")
    kv.write(*(any_stride(r[:-1], 1, stride) for r in rows), slots[:-1])
    kv.write(*(any_stride(any_stride(r[-1:], 1, stride), 0, stride) for r in rows), slots[-1:])
    k, v = ([r.to(torch.bfloat16).double() if kind == "bf16" else ref.values(*ref.quantised(r, kind)) for r in rows])
    got = torch.full((1, 1, dim), 7.0, device="cuda")
    kv.read(slots[-1:], out=(any_stride(got, 0, stride), any_stride(torch.empty_like(got), 0, stride)))
    assert torch.equal(got.double(), k[-1:])
    for heads in (1, 4):
        q = any_stride(torch.randn((1, heads, dim), device="cuda").to(torch.bfloat16), 0, stride)
        q = any_stride(q, 1, stride) if heads == 1 else q
        cu, lens, table = torch.tensor([0, 1], **I32), torch.tensor([n], **I32), torch.zeros((1, 1), **I32)
        out, lse = kv.attention(q, cu, lens, table, 1, want_lse=True, out=any_stride(torch.empty((1, heads, dim), dtype=torch.bfloat16, device="cuda"), 0, stride))
        check_attention(out, lse, ref.attention(q, k, v, 1), dim)
    kv.close()


# ---- size ------------------------------------------------------------------------------------------------------------------------
def test_more_units_of_work_than_32_bits_count():
    # 140,000 queries of 8 heads over 2 M tokens, sent to the kernel for few rows: 2.3 G units for the one kv head.  All queries are alike, so all
    # outputs are
    n, n_q, heads, dim, page = 1 << 21, 140_000, 8, 64, 4096
    g = torch.Generator(device="cuda").manual_seed(2)
    kv = siso.PagedKV.allocate(1, n // page, page, 1, dim, torch.int8)
    for t in (kv.k, kv.v):
        t.copy_(torch.randint(-127, 128, t.shape, device="cuda", generator=g, dtype=torch.int8))
    kv.k_exp.fill_(127 - 9)
    kv.v_exp.fill_(127 - 7)
    table = torch.randperm(n // page, device="cuda", generator=g).to(torch.int32)[None]
    q = torch.randn((1, heads, dim), device="cuda", generator=g).to(torch.bfloat16)
    cu, lens = torch.tensor([0, n_q], **I32), torch.tensor([n], **I32)
    out, lse = kv.attention(q.expand(n_q, heads, dim), cu, lens, table, 1, causal=False, want_lse=True)
    assert kv.sync_status() == 0
    k, v = kv.k.double().view(n, dim) * 2.0 ** -9, kv.v.double().view(n, dim) * 2.0 ** -7
    x = q[0].double() @ k.T * dim ** -0.5
    p = torch.softmax(x, -1)
    want = ((p @ v)[None], torch.logsumexp(x, -1)[None], (p @ v.abs())[None], float((q[0].double().abs() @ k.abs().T).max()) * dim ** -0.5)
    for i in range(0, n_q, 20_000):
        m = min(20_000, n_q - i)
        check_attention(out[i:i + m], lse[i:i + m], [w if isinstance(w, float) else w.expand(m, *w.shape[1:]) for w in want], dim)
    kv.close()


# ---- rows that no sequence covers ------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("n_q", [2, 90])
def test_rows_that_no_sequence_covers_are_left_alone(n_q):
    n, heads, dim = 200, 8, 128
    kv, table, k, v = filled("bf16", n, 16, 2, dim)
    q = torch.randn((n_q + 7, heads, dim), device="cuda").to(torch.bfloat16)
    cu, lens = torch.tensor([3, 3 + n_q], **I32), torch.tensor([n], **I32)
    out = torch.full_like(q, 7.0)
    kv.attention(q, cu, lens, table, n_q, out=out)
    assert (out[:3] == 7).all() and (out[3 + n_q:] == 7).all()
    _, lse = kv.attention(q, cu, lens, table, n_q, want_lse=True)
    check_attention(out[3:3 + n_q], lse[3:3 + n_q], ref.attention(q[3:3 + n_q], k, v, n_q), dim)
    kv.attention(q, cu[:1], lens[:0], table[:0], n_q, out=out.fill_(7.0))         # no sequences at all
    assert (out == 7).all()
    kv.close()


# ---- queries that are not finite -------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("kind", ["bf16", "e4m3"])
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("n,n_q", [(100, 1), (100, 4), (20_011, 1), (20_011, 7), (300, 12), (300, 150), (20_011, 20), (20_011, 100)])
@pytest.mark.parametrize("bad", [math.nan, math.inf])
def test_a_query_that_is_not_finite_gives_nan_and_no_other_row_does(kind, dim, n, n_q, bad):
    # in one part and in several, in every kernel: not a zero that looks like a row that sees nothing
    kv, table, k, v = filled(kind, n, 64, 1, dim)
    q = torch.randn((n_q, 4, dim), device="cuda").to(torch.bfloat16)
    q[n_q // 2, 2, dim // 3] = bad
    cu, lens = torch.tensor([0, n_q], **I32), torch.tensor([n], **I32)
    out, lse = kv.attention(q, cu, lens, table, n_q, want_lse=True)
    assert kv.sync_status() == 0
    hurt = torch.zeros((n_q, 4), dtype=torch.bool, device="cuda")
    hurt[n_q // 2, 2] = True
    assert out[hurt].isnan().all() and lse[hurt].isnan().all()
    want = ref.attention(q.masked_fill(hurt[:, :, None], 0), k, v, n_q)
    check_attention(out.masked_fill(hurt[:, :, None], 0)[:, [0, 1, 3]], lse[:, [0, 1, 3]], [w if isinstance(w, float) else w[:, [0, 1, 3]] for w in want], dim)
    rest = [i for i in range(n_q) if i != n_q // 2]
    check_attention(out[rest], lse[rest], [w if isinstance(w, float) else w[rest] for w in want], dim)
    kv.close()
