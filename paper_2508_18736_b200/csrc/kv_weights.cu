// The weight that attention gives to each cached token, accumulated: for the eviction by it.
//
// Query i of a sequence (head g of the kv head's group) gives token j, if it sees it, exp(scale q.k_j - lse): its probability.  For each token and
// kv head the call takes w_j <- decay w_j + sum over queries and heads (from 0 where the token has no weight yet).  The statistics (lse) are the attention's, so one pass over the keys is all.
//
// Scores are taken transposed, S^T = K Q^T by tcgen05: keys are the 128 lanes of TMEM and query rows its columns.  A thread then owns a key: the sum over
// queries stays in one register, a scale of an 8-bit row is one factor, causality is one first column, and keys that are not there spoil their own thread only.
// A step's few rows make few columns (32 at least) instead of a mostly empty tile of 128 rows.
// An item is (sequence, kv head, block of 256 keys = two tiles), a unit is an item with one tile of up to 128 query rows: whole tokens with all their heads of
// the group (groups above 128: the largest part that divides them).  Units are dealt to one CTA per SM in equal runs, as in the attention; items that were cut are
// joined by a second kernel in a fixed order.  With one row tile an item is one unit and nothing is cut (FEW).
//   the first warps (FEW: 8, a thread per key; else 16, two threads per key, which share the columns): scores from TMEM (two buffers), exponentials, sum
//   one warp         issues the products
//   one warp         fills the ring of key tiles by TMA, one box per run of tokens in one page
//   one warp         fills the ring of query tiles by TMA, and their -lse log2 e beside them
//   one warp         brings what else belongs to the keys: their weights so far and where they lie, exponents
//   8 warps          8-bit caches only: turn codes into bf16 tiles (without the scale, exactly)
// Bounds: few rows read every key once: HBM.  A chunk's 256 x 128 scores take 1024 cycles of tcgen05.mma (d = 128) and 2048 of the SM's 16 exponentials a
// cycle: the exponentials, of which some are taken on the FMA pipe.
// Measured (8 kv heads x 128 with 4 query heads each, bf16, the kernel and its join): 4096 queries over 8193 tokens 250 to 254 us in runs of seconds (222 us in short ones), the
// exponentials' pipe 72 % busy; 32 query tokens (128 rows a kv head) of each of 64 sequences over 4096 tokens 119 us, 16 of them 97 us.
#include "kv_attention.cuh"

namespace siso {
namespace kvw {

using namespace umma2;
using kva::FastDiv;
using kva::wait_bar;

constexpr int TK = 128, KB = 2 * TK, ROWS = 128;

struct Record {                        // an item that several CTAs share, kept at the first of them
    int valid, b, head, kb, n_parts;
};
struct Args {
    KvView kv;
    siso_weights_t a;
    const int32_t *fresh;
    FastDiv by_page;
    int group, hb, tb, chunks;         // a row tile: hb heads of tb tokens; chunks = group / hb
    int box, grid;
    float scale_log2;
    float *part;                       // [2 grid][KB]
    Record *records;                   // [grid]
    int *status;
};

#ifdef __CUDACC__
// ---- units ------------------------------------------------------------------------------------------------------------------
__device__ __forceinline__ int seq_len(const Args &g, int b) {
    return static_cast<int>(min(static_cast<long long>(max(g.a.d_kv_len[b], 0)), static_cast<long long>(g.a.max_pages) * g.kv.page_size));
}
__device__ __forceinline__ int seq_queries(const Args &g, int b, int &q0) {
    const int n = static_cast<int>(g.a.n_tokens);
    q0 = min(max(g.a.d_cu_q[b], 0), n);
    return max(0, min(g.a.d_cu_q[b + 1], n) - q0);
}
// tokens of a sequence that have a weight already
__device__ __forceinline__ int old_tokens(const Args &g, int b, int len, int n_q) { return len - (g.fresh ? min(max(g.fresh[b], 0), len) : n_q); }
// What the items of a sequence cost: `tiles` row tiles and one more, for the beginning and end, as long as all of them see the block (`full` blocks), fewer tiles then
struct Seq {
    int q0, n_q, len, tiles, blocks, full;
    __device__ __forceinline__ void load(const Args &g, int b) {
        n_q = seq_queries(g, b, q0);
        len = n_q > 0 ? seq_len(g, b) : 0;
        tiles = (n_q + g.tb - 1) / g.tb * g.chunks;
        blocks = (len + KB - 1) / KB;
        full = !(g.a.flags & SISO_ATTN_CAUSAL) ? blocks : len >= n_q ? min(blocks, (len - n_q) / KB + 1) : 0;
    }
    // the first row tile that sees a key of the block
    __device__ __forceinline__ int first_tile(const Args &g, int kb) const {
        return kb < full ? 0 : (kb * KB - (len - n_q)) / g.tb * g.chunks;
    }
    __device__ __forceinline__ int cost(const Args &g, int kb) const { return tiles - first_tile(g, kb) + 1; }
    __device__ __forceinline__ long long head_cost(const Args &g) const {
        long long c = static_cast<long long>(full) * (tiles + 1);
        for (int kb = full; kb < blocks; ++kb) c += cost(g, kb);
        return c;
    }
};
// A place in this CTA's run
template <bool FEW> struct Cursor {
    Seq s;
    int b, head, kb, tile, tile0;
    long long left;                                     // cost from this unit to the run's end
    __device__ __forceinline__ void next_item(const Args &g) {
        if (++kb == s.blocks) {
            kb = 0;
            if (++head == g.kv.n_kv_heads) {
                head = 0;
                do { ++b; s.load(g, b); } while (s.blocks == 0);       // only called while some are left
            }
        }
        tile = tile0 = s.first_tile(g, kb);
    }
    // units of this item that belong to the run: FEW: all of them, where the run holds the first
    __device__ __forceinline__ int units_here() const {
        const int n = s.tiles - tile;
        return FEW ? n : static_cast<int>(min(static_cast<long long>(n), tile == tile0 ? (left <= 2 ? 1 : left - 1) : left));
    }
    // all units of units_here() further; false: the run is over
    __device__ __forceinline__ bool step(const Args &g) {
        const int n = units_here();
        left -= n + (tile == tile0 ? 1 : 0);
        tile += n;
        if (left <= 0) return false;
        next_item(g);
        return true;
    }
    __device__ __forceinline__ bool whole(int n) const { return tile == tile0 && tile + n == s.tiles; }
};
constexpr int MAX_THREADS = 896;
struct Find {
    unsigned long long buf[MAX_THREADS / 32], found[3];
};
// This CTA's run and the cursor at its start, the same in every thread.  False: nothing to do
template <bool FEW, int THREADS>
__device__ __forceinline__ bool locate(const Args &g, Cursor<FEW> &cur, long long &end, long long &total, int &ctas, Find &f) {
    if (threadIdx.x == 0) g.records[blockIdx.x].valid = 0;
    Seq s;
    unsigned long long mine = 0ull, upto = 0ull, all;
    auto chunk = [&](int c0) {
        const int b = c0 + static_cast<int>(threadIdx.x);
        if (b >= g.a.n_seqs) return 0ull;
        s.load(g, b);
        return static_cast<unsigned long long>(s.head_cost(g));
    };
    total = 0;
    unsigned long long per_head = 0ull;
    for (int c0 = 0; c0 < g.a.n_seqs; c0 += THREADS) {
        const unsigned long long ph = chunk(c0), x = ph * g.kv.n_kv_heads, to = kva::cta_scan<THREADS>(x, all, f.buf);
        if (c0 == 0) { per_head = ph; mine = x; upto = to; }
        total += static_cast<long long>(all);
    }
    ctas = static_cast<int>(min(static_cast<long long>(g.grid), (total + 1) / 2));
    if (static_cast<int>(blockIdx.x) >= ctas) return false;
    const unsigned long long want = kva::quotient(static_cast<unsigned long long>(total) * blockIdx.x, ctas);
    end = static_cast<long long>(kva::quotient(static_cast<unsigned long long>(total) * (blockIdx.x + 1), ctas));
    unsigned long long base = 0ull;
    for (int c0 = 0;; c0 += THREADS) {
        if (c0 > 0) {
            per_head = chunk(c0);
            mine = per_head * g.kv.n_kv_heads;
            upto = base + kva::cta_scan<THREADS>(mine, all, f.buf);
        }
        __syncthreads();
        if (threadIdx.x == 0) f.found[0] = ~0ull;
        __syncthreads();
        if (want < upto && want >= upto - mine) { f.found[0] = static_cast<unsigned long long>(c0 + threadIdx.x); f.found[1] = upto - mine; f.found[2] = per_head; }
        __syncthreads();
        if (f.found[0] != ~0ull) break;
        if (threadIdx.x == THREADS - 1) f.buf[0] = upto;
        __syncthreads();
        base = f.buf[0];
        __syncthreads();
    }
    cur.b = static_cast<int>(f.found[0]);
    cur.s.load(g, cur.b);
    const unsigned long long within = want - f.found[1];
    cur.head = static_cast<int>(kva::quotient(within, f.found[2]));
    long long x = static_cast<long long>(within - static_cast<unsigned long long>(cur.head) * f.found[2]);
    const int full_cost = cur.s.tiles + 1;
    cur.kb = static_cast<int>(min(static_cast<long long>(kva::quotient(static_cast<unsigned long long>(x), full_cost)), static_cast<long long>(cur.s.full)));
    x -= static_cast<long long>(cur.kb) * full_cost;
    while (cur.kb >= cur.s.full && x >= cur.s.cost(g, cur.kb)) x -= cur.s.cost(g, cur.kb++);
    cur.tile0 = cur.s.first_tile(g, cur.kb);
    cur.tile = cur.tile0;
    cur.left = end - static_cast<long long>(want);
    if (x > 0) {                                        // the first unit that begins at x or later: units begin at 0, 2, 3, ..
        const int n = FEW ? cur.s.tiles - cur.tile0 : static_cast<int>(max(x - 1, 1ll));
        cur.left -= (FEW ? n + 1 : max(x, 2ll)) - x;
        cur.tile += n;
        if (cur.left <= 0) return false;
        if (cur.tile >= cur.s.tiles) cur.next_item(g);
    }
    return true;
}

// ---- the kernel ---------------------------------------------------------------------------------------------------------------
constexpr int SHIFTS = 8;              // their ring: they are needed until the sums are done, the queries only until the products are
constexpr int METAS = 4;               // items whose keys' small things are there or on their way
struct Bars {
    uint64_t s_full[2][2], s_empty[2][2], k_full[8], k_empty[8], q_full[3], q_empty[3], sh_full[SHIFTS], sh_empty[SHIFTS], raw_full[8], raw_empty[8], meta_full[METAS], meta_empty[METAS];
    uint32_t tmem;
    int gave_up;
    int dead[3];                       // of a query tile that has rows whose lse is -infinity: where its statistics lie among the SHIFTS, and 1; else 0
    union {
        Find find;
        float peer[2][TK];             // a key's sum on its way to the other thread of the key
    };
};
// What belongs to an item's keys: where their weights lie (of blocks of 8, -1: nowhere), the weights so far, the exponents; how many of the sequence's tokens have weights
struct Meta {
    long long place[KB / 8];
    int n_old, pad[3];
    float old[KB];
    uint8_t exp[KB];
};
template <int KIND, int D, bool FEW> struct Shape {
    static constexpr bool EIGHT = KIND != SISO_BF16;
    static constexpr int PER_KEY = FEW ? 1 : 2, SUM_WARPS = 8 * PER_KEY;    // threads of a key
    static constexpr int THREADS = 32 * (SUM_WARPS + 4 + (EIGHT ? 8 : 0));
    // of 16 pairs of exponentials so many are taken on the FMA pipe (chunk of 4096 queries over 8193 tokens: none 282 us, two 280 us, three 274 us, five 287 us, before other steps)
    static constexpr int POLY = FEW ? 0 : 3;
    static constexpr int TILE = TK * D * 2, Q_TILE = ROWS * D * 2, RAW = EIGHT ? TK * D : 0;
    static constexpr int STAGES = D == 64 ? (EIGHT ? 4 : FEW ? 8 : 6) : (EIGHT ? 3 : 4);
    static constexpr int Q_STAGES = 2;
    static constexpr int RAWS = !EIGHT ? 0 : D == 64 ? 8 : 3;
    static constexpr int SMEM = STAGES * TILE + Q_STAGES * Q_TILE + RAWS * RAW + SHIFTS * ROWS * 4 + METAS * static_cast<int>(sizeof(Meta)) + static_cast<int>(sizeof(Bars));
    static_assert(SMEM <= 232448, "shared memory");
    // registers: what the CTA has at launch, moved to the sums
    static constexpr int AT_LAUNCH = 65536 / THREADS / 8 * 8 > 168 ? 168 : 65536 / THREADS / 8 * 8;
    static constexpr int SUM_REGS = PER_KEY == 1 ? (EIGHT ? 144 : 216) : (EIGHT ? 96 : 104);
    static constexpr int OTHER_REGS = PER_KEY == 1 ? (EIGHT ? 64 : 72) : (EIGHT ? 40 : 64), CONVERT_REGS = PER_KEY == 1 ? 64 : 40;
    static_assert(2 * PER_KEY * SUM_REGS + OTHER_REGS + (EIGHT ? 2 * CONVERT_REGS : 0) == THREADS / 128 * AT_LAUNCH, "register split");
};
__device__ __forceinline__ bool elect_one() {
    uint32_t one;
    asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xFFFFFFFF;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(one));
    return one != 0u;
}
__device__ __forceinline__ float2 fma2(float2 a, float2 b, float2 c) {
    float2 d;
    asm("fma.rn.f32x2 %0, %1, %2, %3;"
        : "=l"(reinterpret_cast<unsigned long long &>(d))
        : "l"(reinterpret_cast<unsigned long long &>(a)), "l"(reinterpret_cast<unsigned long long &>(b)), "l"(reinterpret_cast<unsigned long long &>(c)));
    return d;
}
__device__ __forceinline__ float2 add2(float2 a, float2 b) {
    float2 d;
    asm("add.rn.f32x2 %0, %1, %2;"
        : "=l"(reinterpret_cast<unsigned long long &>(d)) : "l"(reinterpret_cast<unsigned long long &>(a)), "l"(reinterpret_cast<unsigned long long &>(b)));
    return d;
}
// 2^x for x up to 127 on the FMA pipe, 0 below -127: x = n + f with n whole and f in [-1/2, 1/2], a polynomial of degree 5 for 2^f (largest relative
// error on the interval minimised numerically: 1.5e-7), times 2^n, whose bits are n + 127 moved up
__device__ __forceinline__ float2 ex2_poly(float2 x) {
    asm("max.NaN.f32 %0, %0, %1;" : "+f"(x.x) : "f"(-127.f));
    asm("max.NaN.f32 %0, %0, %1;" : "+f"(x.y) : "f"(-127.f));
    const float big = 12583039.f;                     // 1.5 2^23 + 127: adding it leaves n + 127 in the low bits
    const float2 t = add2(x, make_float2(big, big));
    const float2 f = add2(x, fma2(t, make_float2(-1.f, -1.f), make_float2(big, big)));
    float2 y = make_float2(0.0013276468962430954f, 0.0013276468962430954f);
    y = fma2(y, f, make_float2(0.009675541892647743f, 0.009675541892647743f));
    y = fma2(y, f, make_float2(0.05550713464617729f, 0.05550713464617729f));
    y = fma2(y, f, make_float2(0.24022120237350464f, 0.24022120237350464f));
    y = fma2(y, f, make_float2(0.6931469440460205f, 0.6931469440460205f));
    y = fma2(y, f, make_float2(1.0000001192092896f, 1.0000001192092896f));
    y.x *= __uint_as_float(__float_as_uint(t.x) << 23);
    y.y *= __uint_as_float(__float_as_uint(t.y) << 23);
    return y;
}
// bits first .. last of 32, as far as there are such
__device__ __forceinline__ uint32_t bits_between(int first, int last) {
    const uint32_t from = first <= 0 ? 0xFFFFFFFFu : first > 31 ? 0u : 0xFFFFFFFFu << first;
    return from & (last >= 31 ? 0xFFFFFFFFu : last < 0 ? 0u : 0xFFFFFFFFu >> (31 - last));
}
__device__ __forceinline__ void load_q_box(uint32_t dst, const CUtensorMap *map, int d, int head, int token, uint64_t *bar) {
    asm volatile("cp.async.bulk.tensor.3d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];"
                 ::"r"(dst), "l"(reinterpret_cast<uint64_t>(map)), "r"(d), "r"(head), "r"(token), "r"(smem_u32(bar)) : "memory");
}
struct Yes { static constexpr bool value = true; };
struct No { static constexpr bool value = false; };
// D fp32, A and B bf16 from shared memory, both K-major; N columns
__device__ __forceinline__ uint32_t idesc(int n) {
    return (1u << 4) | (1u << 7) | (1u << 10) | (static_cast<uint32_t>(n >> 3) << 17) | (static_cast<uint32_t>(128 >> 4) << 24);
}
// codes of a word as bf16, in order
template <int KIND> __device__ __forceinline__ void widen(uint32_t w, uint32_t &a, uint32_t &b) {
    uint32_t even, odd;
    if constexpr (KIND == SISO_E4M3) CodeScale<KIND>(127).widen(w, even, odd);
    else {
        const uint32_t x = w >> 8;
        even = sub2_bf16((w & 0x007F007Fu) | 0x43004300u, (w & 0x00800080u) | 0x43004300u);
        odd = sub2_bf16((x & 0x007F007Fu) | 0x43004300u, (x & 0x00800080u) | 0x43004300u);
    }
    a = __byte_perm(even, odd, 0x5410);
    b = __byte_perm(even, odd, 0x7632);
}

// Rows of a query tile that has come whose lse is -infinity (their `shift` too) may hold anything, and a NaN less infinity is one: zeros, for the products.  Not inlined,
// and by the warp that issues the products: in the sums it cost every chunk of 4096 queries 1 to 2 %, inlined with the queries' loads 64 rows over 8 bits 8 %.  2048 queries over 4097 tokens,
// none of the rows such, one in a hundred, half of them: 69, 79, 98 us
template <int D> __device__ __noinline__ void clear_rows(uint8_t *tile, const float *shift, int rows, int lane) {
    for (int r = lane; r < rows; r += 32)                       // a row a lane, its pieces in an order of the lane's own, so that lanes write to different banks
        if (shift[r] == -INFINITY) {
#pragma unroll 4
            for (int c = 0; c < D / 8; ++c) *reinterpret_cast<uint4 *>(tile + (c >> 3) * (ROWS * 128) + r * 128 + ((c + lane) & 7) * 16) = make_uint4(0u, 0u, 0u, 0u);
        }
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    __syncwarp();
}

template <int KIND, int D, bool FEW>
__global__ void __launch_bounds__(Shape<KIND, D, FEW>::THREADS, 1)
weights_kernel(const __grid_constant__ Args g, const __grid_constant__ CUtensorMap map_k, const __grid_constant__ CUtensorMap map_q) {
    using S = Shape<KIND, D, FEW>;
    constexpr bool EIGHT = S::EIGHT;
    constexpr int SUM_WARPS = S::SUM_WARPS, PER_KEY = S::PER_KEY;
    constexpr int RB = D * (EIGHT ? 1 : 2), LINE = RB < 128 ? RB : 128;
    extern __shared__ __align__(1024) uint8_t smem[];           // all of it: nothing static, so that it begins on a boundary of the swizzle
    uint8_t *tiles = smem, *q_tiles = tiles + S::STAGES * S::TILE, *raws = q_tiles + S::Q_STAGES * S::Q_TILE;
    float *shifts = reinterpret_cast<float *>(raws + S::RAWS * S::RAW);              // -lse log2 e of a query tile's rows
    Meta *metas = reinterpret_cast<Meta *>(shifts + SHIFTS * ROWS);
    Bars &bars = *reinterpret_cast<Bars *>(metas + METAS);

    wait_for_earlier();
    dependents_may_start();
    const int lane = threadIdx.x & 31, warp = __shfl_sync(0xFFFFFFFFu, static_cast<int>(threadIdx.x >> 5), 0);      // (uniform)
    if (threadIdx.x == 0) {
        for (int i = 0; i < 4; ++i) { mbar_init(&bars.s_full[0][0] + i, 1); mbar_init(&bars.s_empty[0][0] + i, SUM_WARPS / 2); }
        for (int i = 0; i < S::STAGES; ++i) { mbar_init(&bars.k_full[i], EIGHT ? 8 : 1); mbar_init(&bars.k_empty[i], 1); }
        for (int i = 0; i < S::Q_STAGES; ++i) { mbar_init(&bars.q_full[i], 1); mbar_init(&bars.q_empty[i], 1); }
        for (int i = 0; i < SHIFTS; ++i) { mbar_init(&bars.sh_full[i], 1); mbar_init(&bars.sh_empty[i], SUM_WARPS); }
        for (int i = 0; i < S::RAWS; ++i) { mbar_init(&bars.raw_full[i], 1); mbar_init(&bars.raw_empty[i], 8); }
        for (int i = 0; i < METAS; ++i) { mbar_init(&bars.meta_full[i], 33); mbar_init(&bars.meta_empty[i], SUM_WARPS); }      // 33: the copies, and the places
        bars.gave_up = 0;
        for (int i = 0; i < S::Q_STAGES; ++i) bars.dead[i] = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    const int rows = g.hb * g.tb;                                // of a full row tile
    const int n_cols = FEW && rows <= 64 ? 64 : ROWS;
    // rows behind a full tile's: zeros, or what stands there would reach the scores as NaN
    for (int i = threadIdx.x; i < S::Q_STAGES * (D / 64) * (n_cols - rows) * 8; i += S::THREADS) {
        const int line = i / 8, part = line / (n_cols - rows), row = rows + line % (n_cols - rows);
        *reinterpret_cast<uint4 *>(q_tiles + part * (ROWS * 128) + row * 128 + (i & 7) * 16) = make_uint4(0u, 0u, 0u, 0u);
    }
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    __syncthreads();
    Cursor<FEW> cur;
    long long run_end, total;
    int ctas;
    if (warp == SUM_WARPS) {                       // (while the others look for their run)
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&bars.tmem)), "r"(512u) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    if (!locate<FEW, S::THREADS>(g, cur, run_end, total, ctas, bars.find)) {
        if (warp == SUM_WARPS) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(*const_cast<volatile uint32_t *>(&bars.tmem)), "r"(512u) : "memory");
        return;
    }
    tcgen05_fence_before();
    __syncthreads();
    tcgen05_fence_after();
    const uint32_t tmem = bars.tmem;
    volatile int *gave_up = &bars.gave_up;

    if (warp >= SUM_WARPS + 4) {
        if constexpr (EIGHT) {
            // ---- codes -> bf16 tiles.  8 (4) lanes share a row of 128 (64) bytes; each writes two chunks of 8 values, lanes of the upper half of a
            // row the second one first
            asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(S::CONVERT_REGS));
            constexpr int CH = RB / 16, PER = 32 / CH, MINE = TK / 8;     // chunks of a row, rows of a warp's step, rows of a warp
            const int chunk = lane % CH, r0 = (warp - SUM_WARPS - 4) * MINE + lane / CH, flip = CH == 8 ? chunk >> 2 : 0;
            int stage = 0, raw = 0;
            uint32_t phase = 0, raw_phase = 0;
            do {
                for (int t = 0; t < 2; ++t) {
                    wait_bar(&bars.raw_full[raw], raw_phase, gave_up, g.status);
                    wait_bar(&bars.k_empty[stage], phase ^ 1u, gave_up, g.status);
                    const uint8_t *src = raws + raw * S::RAW;
                    uint8_t *dst = tiles + stage * S::TILE;
#pragma unroll
                    for (int i = 0; i < MINE / PER; ++i) {
                        const int row = r0 + i * PER;
                        const uint4 w = *reinterpret_cast<const uint4 *>(src + kva::chunk_at<RB, TK>(row, chunk));
                        uint4 a, b;
                        widen<KIND>(w.x, a.x, a.y);
                        widen<KIND>(w.y, a.z, a.w);
                        widen<KIND>(w.z, b.x, b.y);
                        widen<KIND>(w.w, b.z, b.w);
                        *reinterpret_cast<uint4 *>(dst + kva::chunk_at<2 * D, TK>(row, 2 * chunk + flip)) = flip ? b : a;
                        *reinterpret_cast<uint4 *>(dst + kva::chunk_at<2 * D, TK>(row, 2 * chunk + 1 - flip)) = flip ? a : b;
                    }
                    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                    __syncwarp();
                    if (lane == 0) { mbar_arrive(&bars.k_full[stage]); mbar_arrive(&bars.raw_empty[raw]); }
                    if (++stage == S::STAGES) { stage = 0; phase ^= 1u; }
                    if (++raw == S::RAWS) { raw = 0; raw_phase ^= 1u; }
                }
            } while (cur.step(g));
        }
    } else if (warp >= SUM_WARPS) {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(S::OTHER_REGS));
        if (warp == SUM_WARPS + 1) {
            // ---- keys: lanes 0-15 own the runs of 8 tokens of an item's first tile, lanes 16-31 of its second.  Pages are asked for one item ahead
            constexpr int RING = EIGHT ? S::RAWS : S::STAGES;
            const int box_blocks = g.box / 8;
            int stage = 0;
            uint32_t phase = 0;
            struct Place { int head, tok, page; bool wanted; } at;
            auto look_up = [&](Place &p) {
                const int j = cur.kb * KB + lane * 8, i = static_cast<int>(g.by_page.div(static_cast<uint32_t>(j)));
                p.head = cur.head;
                p.tok = j - i * g.kv.page_size;
                p.wanted = j < cur.s.len;
                p.page = p.wanted ? g.a.d_pages[cur.b * g.a.pages_stride + i] : -1;
            };
            look_up(at);
            for (bool more = true; more;) {
                Place ahead = at;
                more = cur.step(g);
                if (more) look_up(ahead);
                const bool in_pool = at.wanted && at.page >= 0 && at.page < g.kv.n_pages;
                if (at.wanted && !in_pool) set_status(g.status, SISO_ERR_INVALID_ARG);
                const bool first = in_pool && lane % box_blocks == 0;
                const uint32_t boxes = __ballot_sync(0xFFFFFFFFu, first);
                for (int t = 0; t < 2; ++t) {
                    uint64_t *full = EIGHT ? &bars.raw_full[stage] : &bars.k_full[stage];
                    wait_bar(EIGHT ? &bars.raw_empty[stage] : &bars.k_empty[stage], phase ^ 1u, gave_up, g.status);
                    uint8_t *dst = EIGHT ? raws + stage * S::RAW : tiles + stage * S::TILE;
                    if (*gave_up == 0) {
                        if (lane == 0) mbar_arrive_expect_tx(full, __popc(boxes & (0xFFFFu << (16 * t))) * (g.box * RB));
                        __syncwarp();
                        if (first && lane >> 4 == t) {
#pragma unroll
                            for (int half = 0; half < RB / LINE; ++half)
                                kva::load_box(smem_u32(dst) + half * (TK * 128) + (lane & 15) * 8 * LINE, &map_k, half * 64, at.head, at.tok, at.page, g.a.layer, full);
                        }
                    }
                    if (++stage == RING) { stage = 0; phase ^= 1u; }
                }
                at = ahead;
            }
        } else if (warp == SUM_WARPS + 2) {
            // ---- queries and their statistics, which are asked for one tile ahead
            int stage = 0, sh = 0;
            uint32_t phase = 0, sh_phase = 0;
            const uint32_t bytes = rows * (D * 2);
            struct Tile { int token, head, here; } at;         // first token (row of d_q), first head, tokens of the sequence from there on
            float shift[ROWS / 32];
            auto statistics = [&](const Tile &x, float (&s)[ROWS / 32]) {
#pragma unroll
                for (int i = 0; i < ROWS / 32; ++i) {
                    const int r = i * 32 + lane, tok = r / g.hb;
                    s[i] = INFINITY;
                    if (r < rows && tok < x.here) s[i] = g.a.d_lse[static_cast<long long>(x.token + tok) * g.a.n_heads + x.head + r - tok * g.hb];
                }
            };
            int tile = cur.tile, left = cur.units_here();
            auto place = [&](Tile &x) {
                const int block = g.chunks == 1 ? tile : tile / g.chunks, part = tile - block * g.chunks;
                x.token = cur.s.q0 + block * g.tb;
                x.here = cur.s.n_q - block * g.tb;
                x.head = cur.head * g.group + part * g.hb;
            };
            place(at);
            statistics(at, shift);
            for (bool more = true; more;) {
                Tile ahead = at;
                float ahead_shift[ROWS / 32];
                ++tile;
                if (--left == 0) {
                    more = cur.step(g);
                    if (more) { tile = cur.tile; left = cur.units_here(); }
                }
                if (more) {
                    place(ahead);
                    statistics(ahead, ahead_shift);
                }
                const int mine = sh;
                wait_bar(&bars.sh_empty[sh], sh_phase ^ 1u, gave_up, g.status);
#pragma unroll
                for (int i = 0; i < ROWS / 32; ++i)             // nothing seen (-infinity), or no row: exponentials are zero
                    shifts[sh * ROWS + i * 32 + lane] = shift[i] == -INFINITY ? -INFINITY : shift[i] * -1.4426950408889634f;
                __syncwarp();
                if (lane == 0) mbar_arrive(&bars.sh_full[sh]);
                if (++sh == SHIFTS) { sh = 0; sh_phase ^= 1u; }
                bool dead = false;
#pragma unroll
                for (int i = 0; i < ROWS / 32; ++i) dead = dead || shift[i] == -INFINITY;
                const int some = __any_sync(0xFFFFFFFFu, dead) ? mine + 1 : 0;
                wait_bar(&bars.q_empty[stage], phase ^ 1u, gave_up, g.status);
                if (*gave_up == 0 && lane == 0) {
                    bars.dead[stage] = some;
                    mbar_arrive_expect_tx(&bars.q_full[stage], bytes);
#pragma unroll
                    for (int half = 0; half < D / 64; ++half)
                        load_q_box(smem_u32(q_tiles + stage * S::Q_TILE) + half * (ROWS * 128), &map_q, half * 64, at.head, at.token, &bars.q_full[stage]);
                }
                __syncwarp();
                if (++stage == S::Q_STAGES) { stage = 0; phase ^= 1u; }
                at = ahead;
#pragma unroll
                for (int i = 0; i < ROWS / 32; ++i) shift[i] = ahead_shift[i];
            }
        } else if (warp == SUM_WARPS + 3) {
            // ---- the keys' small things: a lane has a block of 8 keys.  Pages are asked for one item ahead
            const bool old = g.a.decay != 0.f;
            const float *held = g.a.d_weights + static_cast<long long>(g.a.layer) * g.kv.n_pages * g.kv.n_kv_heads * g.kv.page_size;
            int slot = 0;
            uint32_t phase = 0;
            struct Place { int head, tok, page, n_old; } at;
            auto look_up = [&](Place &p) {
                const int j = cur.kb * KB + lane * 8, i = static_cast<int>(g.by_page.div(static_cast<uint32_t>(j)));
                p.head = cur.head;
                p.n_old = old_tokens(g, cur.b, cur.s.len, cur.s.n_q);
                p.tok = j - i * g.kv.page_size;
                p.page = j < cur.s.len ? g.a.d_pages[cur.b * g.a.pages_stride + i] : -1;
            };
            look_up(at);
            for (bool more = true; more;) {
                Place ahead = at;
                more = cur.step(g);
                if (more) look_up(ahead);
                const bool there = at.page >= 0 && at.page < g.kv.n_pages;             // (the warp that loads the keys reports pages outside the pool)
                const long long place = there ? (static_cast<long long>(at.page) * g.kv.n_kv_heads + at.head) * g.kv.page_size + at.tok : -1;
                wait_bar(&bars.meta_empty[slot], phase ^ 1u, gave_up, g.status);
                Meta &m = metas[slot];
                m.place[lane] = place;
                if (lane == 0) m.n_old = at.n_old;
                if (there && old) {
                    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(smem_u32(m.old + lane * 8)), "l"(held + place) : "memory");
                    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(smem_u32(m.old + lane * 8 + 4)), "l"(held + place + 4) : "memory");
                }
                if (EIGHT && there) asm volatile("cp.async.ca.shared.global [%0], [%1], 8;" ::"r"(smem_u32(m.exp + lane * 8)), "l"(g.kv.k_exp + place) : "memory");
                asm volatile("cp.async.mbarrier.arrive.noinc.shared.b64 [%0];" ::"r"(smem_u32(&bars.meta_full[slot])) : "memory");
                __syncwarp();
                if (lane == 0) mbar_arrive(&bars.meta_full[slot]);
                if (++slot == METAS) { slot = 0; phase ^= 1u; }
                at = ahead;
            }
            asm volatile("cp.async.wait_all;" ::: "memory");
        } else if (warp == SUM_WARPS) {
            // ---- products.  The whole warp goes through the loop; one lane issues
            const uint32_t base = __shfl_sync(0xFFFFFFFFu, tmem, 0);
            const uint64_t k_desc = smem_desc_sw128(smem_u32(tiles)), q_desc = smem_desc_sw128(smem_u32(q_tiles));
            const uint32_t id = idesc(n_cols);
            int k_stage = 0, q_stage = 0, buf = 0;
            uint32_t k_phase = 0, q_phase = 0, s_phase = 0;
            bool more = true;
            do {
                const int n = __shfl_sync(0xFFFFFFFFu, cur.units_here(), 0);
                int stages[2];
                uint32_t phases[2];
#pragma unroll
                for (int t = 0; t < 2; ++t) {
                    stages[t] = k_stage;
                    phases[t] = k_phase;
                    if (++k_stage == S::STAGES) { k_stage = 0; k_phase ^= 1u; }
                }
                for (int u = 0; u < n; ++u) {
                    wait_bar(&bars.q_full[q_stage], q_phase, gave_up, g.status);
                    const int dead = bars.dead[q_stage];
                    if (__any_sync(0xFFFFFFFFu, dead != 0)) clear_rows<D>(q_tiles + q_stage * S::Q_TILE, shifts + (dead - 1) * ROWS, rows, lane);
                    const uint64_t b = q_desc + static_cast<uint64_t>(q_stage * (S::Q_TILE >> 4));
#pragma unroll
                    for (int t = 0; t < 2; ++t) {
                        if (u == 0) wait_bar(&bars.k_full[stages[t]], phases[t], gave_up, g.status);
                        wait_bar(&bars.s_empty[t][buf], s_phase ^ 1u, gave_up, g.status);
                        tcgen05_fence_after();
                        const uint64_t a = k_desc + static_cast<uint64_t>(stages[t] * (S::TILE >> 4));
                        if (elect_one()) {
#pragma unroll
                            for (int k = 0; k < D / 16; ++k) {      // 32 bytes further along a line, or the next 64 d
                                const uint64_t off = static_cast<uint64_t>(2 * (k % 4) + (k / 4) * ((TK * 128) >> 4));
                                umma_bf16(base + (2 * t + buf) * 128, a + off, b + off, id, k ? 1u : 0u);
                            }
                            umma_commit(&bars.s_full[t][buf]);
                            if (t == 1) umma_commit(&bars.q_empty[q_stage]);
                            if (u == n - 1) umma_commit(&bars.k_empty[stages[t]]);
                        }
                        __syncwarp();
                    }
                    if (++q_stage == S::Q_STAGES) { q_stage = 0; q_phase ^= 1u; }
                    if ((buf ^= 1) == 0) s_phase ^= 1u;
                }
                more = __any_sync(0xFFFFFFFFu, cur.step(g));
            } while (more);
        }
    } else {
        // ---- sums: one or two threads per key, each with its part of the columns
        asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(S::SUM_REGS));
        const int t = warp / (4 * PER_KEY), half = (warp >> 2) % PER_KEY, key = threadIdx.x & 127;
        const int mine_cols = n_cols / PER_KEY, col = half * mine_cols;
        const uint32_t s_at = tmem + (static_cast<uint32_t>((warp & 3) * 32) << 16) + t * 256 + col;
        const bool causal = (g.a.flags & SISO_ATTN_CAUSAL) != 0u;
        float *held = g.a.d_weights + static_cast<long long>(g.a.layer) * g.kv.n_pages * g.kv.n_kv_heads * g.kv.page_size;
        int sh = 0, buf = 0;
        uint32_t sh_phase = 0, s_phase = 0;
        int slot = 0;
        uint32_t meta_phase = 0;
        for (bool more = true; more;) {
            const int n = __shfl_sync(0xFFFFFFFFu, cur.units_here(), 0), tile_first = cur.tile, j0 = cur.kb * KB + t * TK, j = j0 + key;
            const int n_q = cur.s.n_q, before = cur.s.len - n_q;
            const bool whole = FEW || cur.whole(n), began_before = cur.tile > cur.tile0;
            if (!FEW && !whole && !began_before && threadIdx.x == 0) {
                // the item's last unit begins `tiles - tile0` further on than its first
                const long long last = run_end - cur.left + (cur.s.tiles - cur.tile0);
                g.records[blockIdx.x] = Record{1, cur.b, cur.head, cur.kb, kva::cta_of(last, total, ctas) - static_cast<int>(blockIdx.x) + 1};
            }
            more = __any_sync(0xFFFFFFFFu, cur.step(g));         // (uniform, visibly: barriers and TMEM loads in the loop cost no registers then)
            wait_bar(&bars.meta_full[slot], meta_phase, gave_up, g.status);
            const Meta &meta = metas[slot];
            const bool is_old = j < meta.n_old && g.a.decay != 0.f;
            const float f = EIGHT ? g.scale_log2 * kv_scale(meta.exp[t * TK + key]) : g.scale_log2;
            float sum = 0.f;
            for (int u = 0; u < n; ++u) {
                const int tile = tile_first + u, token0 = (g.chunks == 1 ? tile : tile / g.chunks) * g.tb;
                // columns [first, last) are rows that see the key
                const int last = min(rows, (n_q - token0) * g.hb);
                const bool cut = __any_sync(0xFFFFFFFFu, last < rows || (causal && j0 + TK - 1 > before + token0));
                const int first = causal && cut ? max(0, min(j - before - token0, ROWS)) * g.hb : 0;
                const float4 *shift = reinterpret_cast<const float4 *>(shifts + sh * ROWS);
                uint64_t *const read = &bars.sh_empty[sh];
                float2 acc[2] = {make_float2(0.f, 0.f), make_float2(0.f, 0.f)};
                auto weigh = [&](auto some, const uint32_t (&r)[32], int c0) __attribute__((always_inline)) {
                    const uint32_t in = some.value ? bits_between(first - c0, last - 1 - c0) : 0u;
#pragma unroll
                    for (int x = 0; x < 32; x += 4) {
                        const float4 d = shift[(c0 + x) / 4];
                        float2 y[2] = {fma2(make_float2(__uint_as_float(r[x]), __uint_as_float(r[x + 1])), make_float2(f, f), make_float2(d.x, d.y)),
                                       fma2(make_float2(__uint_as_float(r[x + 2]), __uint_as_float(r[x + 3])), make_float2(f, f), make_float2(d.z, d.w))};
#pragma unroll
                        for (int i = 0; i < 2; ++i) {
                            if ((x / 2 + i) * S::POLY % 16 < S::POLY) y[i] = ex2_poly(y[i]);
                            else { y[i].x = kva::ex2(y[i].x); y[i].y = kva::ex2(y[i].y); }
                            if constexpr (some.value) {
                                if (!((in >> (x + 2 * i)) & 1u)) y[i].x = 0.f;
                                if (!((in >> (x + 2 * i + 1)) & 1u)) y[i].y = 0.f;
                            }
                            acc[i] = add2(acc[i], y[i]);
                        }
                    }
                };
                wait_bar(&bars.sh_full[sh], sh_phase, gave_up, g.status);
                wait_bar(&bars.s_full[t][buf], s_phase, gave_up, g.status);
                tcgen05_fence_after();
#pragma unroll 1
                for (int c = 0; c < mine_cols; c += 64) {
                    uint32_t ra[32], rb[32];
                    tmem_ld_32x32(s_at + buf * 128 + c, ra);
                    tmem_ld_32x32(s_at + buf * 128 + c + 32, rb);
                    tmem_ld_fence(ra);
                    tmem_ld_fence(rb);
                    if (c + 64 >= mine_cols) {
                        tcgen05_fence_before();
                        __syncwarp();
                        if (lane == 0) mbar_arrive(&bars.s_empty[t][buf]);
                    }
                    if (cut) {
                        weigh(Yes{}, ra, col + c);
                        weigh(Yes{}, rb, col + c + 32);
                    } else {
                        weigh(No{}, ra, col + c);
                        weigh(No{}, rb, col + c + 32);
                    }
                }
                if (++sh == SHIFTS) { sh = 0; sh_phase ^= 1u; }
                if ((buf ^= 1) == 0) s_phase ^= 1u;
                __syncwarp();
                if (lane == 0) mbar_arrive(read);
                acc[0] = add2(acc[0], acc[1]);
                sum += acc[0].x + acc[0].y;
            }
            if constexpr (PER_KEY == 2) {
                if (half == 1) bars.peer[t][key] = sum;
                asm volatile("bar.sync %0, 256;" ::"r"(1 + t) : "memory");
                if (half == 0) sum += bars.peer[t][key];
                asm volatile("bar.sync %0, 256;" ::"r"(1 + t) : "memory");
            }
            if (half == 1) {
            } else if (whole) {
                const long long place = meta.place[t * (TK / 8) + key / 8];
                if (place >= 0 && j < before + n_q) held[place + (key & 7)] = (is_old ? g.a.decay * meta.old[t * TK + key] : 0.f) + sum;
            } else {
                g.part[kva::part_place(blockIdx.x, began_before) * KB + t * TK + key] = sum;
            }
            __syncwarp();
            if (lane == 0) mbar_arrive(&bars.meta_empty[slot]);
            if (++slot == METAS) { slot = 0; meta_phase ^= 1u; }
        }
    }

    // ---- teardown
    __syncwarp();
    kva::let_copies_land(gave_up);
    tcgen05_fence_before();
    __syncthreads();
    if (warp == SUM_WARPS) {
        tcgen05_fence_after();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(512u) : "memory");
    }
}

// CTA x: the item that is recorded at CTA x, whose parts lie at place 1 of CTA x and place 0 of the next ones.  A thread per key
__global__ void __launch_bounds__(KB)
weights_join_kernel(const __grid_constant__ Args g) {
    wait_for_earlier();
    const Record rec = g.records[blockIdx.x];
    if (!rec.valid) return;
    Seq s;
    s.load(g, rec.b);
    const int j = rec.kb * KB + threadIdx.x;
    if (j >= s.len) return;
    const int i = j / g.kv.page_size, page = g.a.d_pages[rec.b * g.a.pages_stride + i];
    if (page < 0 || page >= g.kv.n_pages) return;
    float sum = 0.f;
    for (int p = 0; p < rec.n_parts; ++p) sum += g.part[kva::part_place(static_cast<int>(blockIdx.x) + p, p > 0) * KB + threadIdx.x];
    float *w = g.a.d_weights + ((static_cast<long long>(g.a.layer) * g.kv.n_pages + page) * g.kv.n_kv_heads + rec.head) * g.kv.page_size + j - i * g.kv.page_size;
    *w = (j < old_tokens(g, rec.b, s.len, s.n_q) && g.a.decay != 0.f ? g.a.decay * *w : 0.f) + sum;
}
#endif

template <int KIND, int D, bool FEW> static siso_status_t run_as(Kv *h, const Args &g, const CUtensorMap &map_q, cudaStream_t s) {
    using S = Shape<KIND, D, FEW>;
    constexpr uint32_t bit = 1u << (FEW ? 12 : 13);
    if (!(h->attr_set & bit)) {
        SISO_CUDA(cudaFuncSetAttribute(weights_kernel<KIND, D, FEW>, cudaFuncAttributeMaxDynamicSharedMemorySize, S::SMEM));
        h->attr_set |= bit;
    }
    SISO_TRY(launch_early(weights_kernel<KIND, D, FEW>, dim3(static_cast<unsigned>(g.grid)), S::THREADS, S::SMEM, s, g, h->map_k, map_q));
    return FEW ? SISO_OK : launch_early(weights_join_kernel, dim3(static_cast<unsigned>(g.grid)), KB, 0, s, g);
}
template <int KIND, int D> static siso_status_t run(Kv *h, const Args &g, bool few, const CUtensorMap &map_q, cudaStream_t s) {
    return few ? run_as<KIND, D, true>(h, g, map_q, s) : run_as<KIND, D, false>(h, g, map_q, s);
}

// up to 32 rows per kv head (kv_weights_few.cu)
siso_status_t launch_few_rows(Kv *h, const siso_weights_t *a, const int32_t *fresh, int rows, cudaStream_t s);

}  // namespace kvw

siso_status_t launch_kv_weights(Kv *h, const siso_weights_t *a, const int32_t *fresh, cudaStream_t s) {
    using namespace kvw;
    const long long rows = static_cast<long long>(a->max_q) * (a->n_heads / h->cfg.n_kv_heads);
    if (rows <= 32) return launch_few_rows(h, a, fresh, static_cast<int>(rows), s);
    Args g;
    g.fresh = fresh;
    g.kv = kv_view(h, a->layer);
    g.a = *a;
    g.group = a->n_heads / h->cfg.n_kv_heads;
    g.by_page.set(static_cast<uint32_t>(h->cfg.page_size));
    g.scale_log2 = a->scale * 1.4426950408889634f;
    g.status = h->status;
    g.box = h->box;
    g.grid = h->sm_count;
    for (g.hb = std::min(g.group, ROWS); g.group % g.hb != 0;) --g.hb;
    g.chunks = g.group / g.hb;
    g.tb = std::max(1, std::min(ROWS / g.hb, a->max_q));
    const bool few = g.chunks == 1 && a->max_q <= g.tb;
    const int dim = h->cfg.head_dim;
    // query tiles: `tb` tokens with `hb` heads, rows of 128 bytes, swizzled
    CUtensorMap map_q;
    const cuuint64_t dims[3] = {static_cast<cuuint64_t>(dim), static_cast<cuuint64_t>(a->n_heads), static_cast<cuuint64_t>(a->n_tokens)};
    const cuuint64_t strides[2] = {std::max<cuuint64_t>(a->q_stride_head * 2, 16), std::max<cuuint64_t>(a->q_stride_token * 2, 16)};
    const cuuint32_t box[3] = {64u, static_cast<cuuint32_t>(g.hb), static_cast<cuuint32_t>(g.tb)}, ones[3] = {1, 1, 1};
    using Encode = CUresult (*)(CUtensorMap *, CUtensorMapDataType, cuuint32_t, void *, const cuuint64_t *, const cuuint64_t *, const cuuint32_t *,
                                const cuuint32_t *, CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
    if (reinterpret_cast<Encode>(h->encode)(&map_q, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, const_cast<void *>(a->d_q), dims, strides, box, ones,
                                            CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_128B,
                                            CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) != CUDA_SUCCESS)
        return check_cuda(cudaErrorInvalidValue, "cuTensorMapEncodeTiled");
    const size_t records = pad256(sizeof(Record) * g.grid);
    // (the attention's, which is larger: a block that a captured call uses is never replaced by a later call's)
    static_assert(sizeof(Record) <= sizeof(kva::Record) && KB <= kva::TC_ROWS, "fits the attention's scratch");
    SISO_TRY(kva::kv_scratch(h, kva::attention_scratch(h), s));
    g.records = static_cast<Record *>(h->ws);
    g.part = reinterpret_cast<float *>(static_cast<char *>(h->ws) + records);
    const bool wide = dim == 128;
    switch (h->cfg.dtype) {
        case SISO_BF16: return wide ? run<SISO_BF16, 128>(h, g, few, map_q, s) : run<SISO_BF16, 64>(h, g, few, map_q, s);
        case SISO_E4M3: return wide ? run<SISO_E4M3, 128>(h, g, few, map_q, s) : run<SISO_E4M3, 64>(h, g, few, map_q, s);
        default: return wide ? run<SISO_I8, 128>(h, g, few, map_q, s) : run<SISO_I8, 64>(h, g, few, map_q, s);
    }
}

}  // namespace siso
