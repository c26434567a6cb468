// Shared by the two attention kernels over the paged key/value cache: arguments, the cut of a call into units of work, the
// partial results and their join.
//
// The queries of one sequence that share a key/value head form its rows: row r is token r / group, query head
// kv_head * group + r % group.  An item is (sequence, key/value head, tile of MR rows); its keys are taken in tiles of TK, and
// one tile of one item is a unit of work.  The units of a call, in the order (sequence, head, row tile, key tile), are dealt to the
// CTAs in equal contiguous runs, so CTAs are equally loaded whatever the lengths are, and one long sequence spreads over
// all of them.  A tile may count more than one unit, and an item counts some more for its beginning and end.  A CTA that holds all units of an item writes its output; otherwise it writes a partial result
// (unnormalised output, maximum, sum), and a second small kernel joins the parts of an item in a fixed order.
#pragma once

#include "kv.cuh"
#include "umma_pair.cuh"

namespace siso {
namespace kva {

constexpr int TC_ROWS = 256;           // rows of a row tile of the tcgen05 kernel

// n / d for 0 <= n < 2^31 and 1 <= d < 2^31, by a multiplication: m = floor(2^(31 + s) / d) + 1 with s = ceil(log2 d)
struct FastDiv {
    uint32_t d, m, s;
    __host__ void set(uint32_t divisor) {
        d = divisor;
        s = 0;
        while ((1ull << s) < divisor) ++s;
        m = static_cast<uint32_t>((1ull << (31 + s)) / divisor + 1);
        if (divisor == 1) m = 0x80000001u;
    }
    __device__ __forceinline__ uint32_t div(uint32_t n) const {
        return static_cast<uint32_t>((static_cast<unsigned long long>(n) * m) >> (31 + s));
    }
};

struct Record {                        // an item that several CTAs share, kept at the first of them
    int valid, b, head, row_tile, n_parts;
};

struct Args {
    KvView kv;
    siso_attention_t a;
    FastDiv by_page, by_group;
    int group;
    float scale_log2;                  // scale * log2(e)
    int box;                           // tokens of one TMA box: they lie in one page
    int grid;                          // CTAs that share the units
    float *part_o, *part_ml;           // [2 grid][MR][D], [2 grid][MR][2]
    Record *records;                   // [grid]
    int *status;
};

#ifdef __CUDACC__
// the row tile `rt` of a sequence: positions of its first and last row's token and the key tiles it has to see
struct Span {
    int first_pos, last_pos, hi, tile0, tiles;
};
__device__ __forceinline__ int seq_len(const Args &g, int b) {
    const long long cap = static_cast<long long>(g.a.max_pages) * g.kv.page_size;
    return static_cast<int>(min(static_cast<long long>(max(g.a.d_kv_len[b], 0)), cap));
}
// queries of sequence b, cut to the tokens that the call has: q0 is its first row of d_q
__device__ __forceinline__ int seq_queries(const Args &g, int b, int &q0) {
    const int n = static_cast<int>(g.a.n_tokens);
    q0 = min(max(g.a.d_cu_q[b], 0), n);
    return max(0, min(g.a.d_cu_q[b + 1], n) - q0);
}
// Position of query i of a sequence.  Queries that stand before the sequence's start all count as standing at -1: they see the same there, and
// differences of positions and windows, both up to 2^31 - 1, stay inside 32 bits
__device__ __forceinline__ int position(int len, int n_q, int i) { return max(len - n_q + i, -1); }
__device__ __forceinline__ int first_seen(const Args &g, int first_pos) { return g.a.window > 0 ? max(0, first_pos - g.a.window + 1) : 0; }
template <int MR, int TK> __device__ __forceinline__ Span span_of(const Args &g, int len, int n_q, int rt) {
    Span s;
    const int rows = n_q * g.group;
    s.first_pos = position(len, n_q, static_cast<int>(g.by_group.div(static_cast<uint32_t>(rt * MR))));
    s.last_pos = position(len, n_q, static_cast<int>(g.by_group.div(static_cast<uint32_t>(min(rows, (rt + 1) * MR) - 1))));
    s.hi = (g.a.flags & SISO_ATTN_CAUSAL) ? max(0, min(len, s.last_pos + 1)) : len;
    const int lo = first_seen(g, s.first_pos);
    s.tile0 = lo / TK;
    s.tiles = max(1, (s.hi + TK - 1) / TK - s.tile0);       // a row tile that sees nothing is one unit that writes zeros
    return s;
}
// Whether the TMA box of token j of a row tile's keys holds tokens that some row may see, and j is not beyond the last.  What lies wholly before
// the window is not looked up: its pages may have been given back
__device__ __forceinline__ bool holds_seen(const Args &g, int lo, int hi, int j) { return j < hi && (j | (g.box - 1)) >= lo; }
// units of one key/value head of sequence b: a key tile counts W, and an item EXTRA more, for its beginning and end
template <int MR, int TK, int EXTRA, int W> __device__ __forceinline__ long long seq_units(const Args &g, int b) {
    int q0;
    const int n_q = seq_queries(g, b, q0), len = seq_len(g, b);
    long long units = 0;
    for (int rt = 0; rt * MR < n_q * g.group; ++rt) units += W * span_of<MR, TK>(g, len, n_q, rt).tiles + EXTRA;
    return units;
}

// A place in this CTA's run of units: an item and a key tile of it.
template <int MR, int TK, int EXTRA, int W> struct Cursor {
    int b, head, rt, q0, n_q, len, tile;
    int left;                                                  // units from this tile's first to the run's end
    Span s;
    __device__ __forceinline__ void load_seq(const Args &g) {
        n_q = seq_queries(g, b, q0);
        len = seq_len(g, b);
    }
    __device__ __forceinline__ void load_span(const Args &g) { s = span_of<MR, TK>(g, len, n_q, rt); }
    __device__ __forceinline__ void next_item(const Args &g) {
        tile = 0;
        if ((rt + 1) * MR < n_q * g.group) ++rt;
        else {
            rt = 0;
            if (++head == g.kv.n_kv_heads) {
                head = 0;
                do { ++b; load_seq(g); } while (n_q == 0);     // only called while units are left
            }
        }
        load_span(g);
    }
    // from the item `rt` of its head, `x` units into it, to the first tile that begins there or later: a tile belongs to the run that
    // its first unit lies in
    __device__ __forceinline__ void enter(const Args &g, int x) {
        tile = max(x - EXTRA + W - 1, 0) / W;
        left -= EXTRA + W * tile - x;
        if (left > 0 && tile == s.tiles) {
            left -= EXTRA;
            if (left > 0) next_item(g);
        }
    }
    // key tiles of this item that belong to the run
    __device__ __forceinline__ int tiles_here() const { return min(s.tiles - tile, (left + W - 1) / W); }
    // the first key that a row of this item sees (worked out again where it is needed: kept, it costs registers)
    __device__ __forceinline__ int lo(const Args &g) const { return g.a.window > 0 && tile == 0 ? first_seen(g, position(len, n_q, static_cast<int>(g.by_group.div(static_cast<uint32_t>(rt * MR))))) : 0; }
    // n <= tiles_here() tiles further; false: the run is over
    __device__ __forceinline__ bool step(const Args &g, int n = 1) {
        tile += n;
        left -= W * n;
        if (left > 0 && tile == s.tiles) {
            left -= EXTRA;
            if (left > 0) next_item(g);
        }
        return left > 0;
    }
};

// inclusive sum over the CTA's threads; `all`: the total.  Two barriers
template <int THREADS>
__device__ __forceinline__ unsigned long long cta_scan(unsigned long long x, unsigned long long &all, unsigned long long *buf) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const unsigned long long y = __shfl_up_sync(0xFFFFFFFFu, x, o);
        if (lane >= o) x += y;
    }
    __syncthreads();
    if (lane == 31) buf[warp] = x;
    __syncthreads();
    unsigned long long before = 0ull;
    all = 0ull;
    for (int w = 0; w < THREADS / 32; ++w) {
        if (w < warp) before += buf[w];
        all += buf[w];
    }
    return before + x;
}

// The run of this CTA among the call's units: it ends before unit `end` of `total`, which `ctas` CTAs share.
struct Run {
    long long end, total;
    int ctas;
};
constexpr int FEW_TILES = 16;          // row tiles that one thread goes through alone; the CTA takes more of them together

// units of one head of the sequences b0 .. b0 + THREADS - 1 that the call has, one per thread
template <int MR, int TK, int EXTRA, int W, int THREADS>
__device__ __forceinline__ long long chunk_units(const Args &g, int b0, unsigned long long *buf) {
    const int n = min(g.a.n_seqs - b0, THREADS);
    // a thread per sequence, unless there are a few long ones: then a thread per row tile (six prompts of 4 to 15 row tiles: 108 us and 111 us)
    if (MR < TC_ROWS || n > 16 || static_cast<long long>(g.a.max_q) * g.group <= 32 * MR) return static_cast<int>(threadIdx.x) < n ? seq_units<MR, TK, EXTRA, W>(g, b0 + threadIdx.x) : 0;
    long long mine = 0;
    for (int i = 0; i < n; ++i) {
        int q0;
        const int n_q = seq_queries(g, b0 + i, q0), len = seq_len(g, b0 + i), tiles = (n_q * g.group + MR - 1) / MR;
        unsigned long long x = 0ull, all;
        for (int rt = threadIdx.x; rt < tiles; rt += THREADS) x += W * span_of<MR, TK>(g, len, n_q, rt).tiles + EXTRA;
        cta_scan<THREADS>(x, all, buf);
        if (static_cast<int>(threadIdx.x) == i) mine = static_cast<long long>(all);
    }
    return mine;
}
// This CTA's run and the cursor at its start; every thread of the CTA gets the same.  False: nothing to do.  The CTA's record
// is cleared.  `buf`: THREADS / 32 + 3 words of shared memory.  A run is counted in 32 bits: a call of 2^31 units a CTA (more than ten
// minutes of work) is reported and not done.
template <int MR, int TK, int EXTRA, int W, int THREADS>
__device__ __forceinline__ bool locate(const Args &g, Run &run, Cursor<MR, TK, EXTRA, W> &cur, unsigned long long *buf) {
    constexpr int WARPS = THREADS / 32;
    const int cta = blockIdx.x;
    if (threadIdx.x == 0) g.records[cta].valid = 0;
    unsigned long long mine = 0ull, upto = 0ull, all;          // units of this thread's sequence of the first chunk, and up to them
    long long per_head = 0;
    run.total = 0;
    for (int c0 = 0; c0 < g.a.n_seqs; c0 += THREADS) {
        const long long ph = chunk_units<MR, TK, EXTRA, W, THREADS>(g, c0, buf);
        const unsigned long long x = static_cast<unsigned long long>(ph) * g.kv.n_kv_heads, s = cta_scan<THREADS>(x, all, buf);
        if (c0 == 0) { mine = x; upto = s; per_head = ph; }
        run.total += static_cast<long long>(all);
    }
    run.ctas = static_cast<int>(min(static_cast<long long>(g.grid), (run.total + W - 1) / W));      // (so that every run within an item has a tile)
    if (cta >= run.ctas) return false;
    if (run.total / run.ctas >= 0x7FFFFFFFll - EXTRA) {
        set_status(g.status, SISO_ERR_UNSUPPORTED);
        return false;
    }
    const unsigned long long want = static_cast<unsigned long long>(run.total * cta / run.ctas);
    run.end = run.total * (cta + 1) / run.ctas;
    cur.left = static_cast<int>(run.end - static_cast<long long>(want));
    // buf[WARPS] and the two after it: what the one thread that finds it says
    auto found = [&](bool here, unsigned long long a, unsigned long long b, unsigned long long c) {
        __syncthreads();
        if (threadIdx.x == 0) buf[WARPS] = ~0ull;
        __syncthreads();
        if (here) { buf[WARPS] = a; buf[WARPS + 1] = b; buf[WARPS + 2] = c; }
        __syncthreads();
        return buf[WARPS] != ~0ull;
    };
    // the sequence that the first unit belongs to
    unsigned long long base = 0ull;
    for (int c0 = 0;; c0 += THREADS) {
        if (c0 > 0) {
            per_head = chunk_units<MR, TK, EXTRA, W, THREADS>(g, c0, buf);
            mine = static_cast<unsigned long long>(per_head) * g.kv.n_kv_heads;
            upto = base + cta_scan<THREADS>(mine, all, buf);
        }
        if (found(want < upto && want >= upto - mine, static_cast<unsigned long long>(c0 + threadIdx.x), upto - mine, static_cast<unsigned long long>(per_head))) break;
        __syncthreads();
        if (threadIdx.x == THREADS - 1) buf[0] = upto;
        __syncthreads();
        base = buf[0];
    }
    cur.b = static_cast<int>(buf[WARPS]);
    cur.load_seq(g);
    const unsigned long long within = want - buf[WARPS + 1], head_units = buf[WARPS + 2];
    const int tiles = (cur.n_q * g.group + MR - 1) / MR;
    cur.head = static_cast<int>(within / head_units);
    unsigned long long x = within - static_cast<unsigned long long>(cur.head) * head_units;
    cur.rt = 0;
    if (tiles <= FEW_TILES) {
        for (cur.load_span(g); x >= static_cast<unsigned long long>(W * cur.s.tiles + EXTRA); cur.load_span(g)) {
            x -= W * cur.s.tiles + EXTRA;
            ++cur.rt;
        }
    } else {
        unsigned long long before = 0ull;
        for (int c0 = 0;; c0 += THREADS) {
            const int rt = c0 + static_cast<int>(threadIdx.x);
            const unsigned long long n = rt < tiles ? W * span_of<MR, TK>(g, cur.len, cur.n_q, rt).tiles + EXTRA : 0;
            const unsigned long long s = before + cta_scan<THREADS>(n, all, buf);
            if (found(x < s && x >= s - n, static_cast<unsigned long long>(rt), s - n, 0ull)) break;
            before += all;
        }
        cur.rt = static_cast<int>(buf[WARPS]);
        x -= buf[WARPS + 1];
        cur.load_span(g);
    }
    cur.enter(g, static_cast<int>(x));
    return cur.left > 0;
}
// the CTA that unit u is dealt to: the last c with floor(total c / ctas) <= u
__device__ __forceinline__ int cta_of(long long u, long long total, int ctas) {
    return static_cast<int>(((u + 1) * ctas - 1) / total);
}
// what is noted of an item whose first part ends this CTA's run; tile `tile` of it begins `left` units before the run's end
template <int W>
__device__ __forceinline__ Record record_of(const Run &run, int left, int b, int head, int row_tile, int tiles, int tile) {
    return Record{1, b, head, row_tile, cta_of(run.end - left + W * (tiles - 1 - tile), run.total, run.ctas) - static_cast<int>(blockIdx.x) + 1};
}
// Where a part goes: a CTA's run has at most one item that began before it (place 0) and one that goes on after it (place 1).
__device__ __forceinline__ long long part_place(int cta, bool began_before) { return 2ll * cta + (began_before ? 0 : 1); }

__device__ __forceinline__ float ex2(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

// From a row's maximum (in powers of two) and sum: a sum of zero means that nothing is seen; NaN stays NaN
__device__ __forceinline__ float inverse_of(float l) { return l == 0.f ? 0.f : 1.f / l; }
__device__ __forceinline__ float lse_of(float m, float l) { return l == 0.f ? -INFINITY : (m + log2f(l)) * 0.6931471805599453f; }

constexpr unsigned long long WAIT_NS = 1000000000ull;       // a wait gives up after a second

// byte offset of a 16-byte chunk in a tile of TK rows as TMA writes it: lines of 128 bytes with the chunk's place xor-ed with the
// row's lowest bits (rows of 256 bytes are two such tiles), or of 64 bytes
template <int RB, int TK> __device__ __forceinline__ int chunk_at(int row, int chunk) {
    if constexpr (RB == 64) return row * 64 + ((chunk ^ ((row >> 1) & 3)) << 4);
    else return (chunk >> 3) * (TK * 128) + row * 128 + (((chunk & 7) ^ (row & 7)) << 4);
}
__device__ __forceinline__ uint32_t pack(float lo, float hi, bool half) {
    uint32_t r;
    if (half) asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    else asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}
__device__ __forceinline__ void load_box(uint32_t dst, const CUtensorMap *map, int d, int head, int token, int page, int layer, uint64_t *bar) {
    asm volatile("cp.async.bulk.tensor.5d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4, %5, %6}], [%7];"
                 ::"r"(dst), "l"(reinterpret_cast<uint64_t>(map)), "r"(d), "r"(head), "r"(token), "r"(page), "r"(layer), "r"(umma2::smem_u32(bar))
                 : "memory");
}
// A wait for this CTA's own copies or warps, bounded; one that gives up says so in the status word, whichever warp it belongs to.  Once any
// has given up, none waits any more: the loops run to their ends on whatever the ring holds, so every barrier of the CTA is still met.
__device__ __forceinline__ void wait_bar(uint64_t *bar, uint32_t parity, volatile int *gave_up, int *status) {
    if (umma2::mbar_try_wait_cta(bar, parity)) return;
    unsigned long long t0, t;
    asm volatile("mov.u64 %0, %%globaltimer;" : "=l"(t0));
    for (uint32_t it = 1; it < umma2::SPIN_LIMIT; ++it) {
        if (umma2::mbar_try_wait_cta(bar, parity)) return;
        if ((it & 63u) == 0u) {
            if (*gave_up) return;
            asm volatile("mov.u64 %0, %%globaltimer;" : "=l"(t));
            if (t - t0 > WAIT_NS) break;
        }
    }
    *gave_up = 1;
    set_status(status, SISO_ERR_TIMEOUT);
}
// after a wait has given up: copies in flight land before the shared memory is handed back
__device__ __forceinline__ void let_copies_land(const volatile int *gave_up) {
    if (*gave_up) for (int i = 0; i < 64; ++i) __nanosleep(1000);
}

#endif  // __CUDACC__

// joins the parts of every item that was cut; MR = rows of a row tile, D = head_dim
siso_status_t launch_join(const Args &g, int mr, int dim, cudaStream_t s);
// many rows per key/value head (tcgen05)
siso_status_t launch_many_rows(Kv *h, Args &g, cudaStream_t s);
siso_status_t kv_scratch(Kv *h, size_t bytes, cudaStream_t s);

}  // namespace kva
}  // namespace siso
