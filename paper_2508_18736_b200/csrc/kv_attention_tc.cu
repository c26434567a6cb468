// Attention of new tokens over the paged key/value cache, many rows per key/value head: prompts and their chunks.
// The formulas are in kv_attention.cu, the dealing of units to CTAs in kv_attention.cuh.
//
// With many rows the call is bound by the tensor cores and, nearly as much, by the exponentials: a tile of 128 x 128 scores takes
// 2 x 512 cycles of tcgen05.mma (d = 128) and 1024 cycles of the SM's 16 exponentials a cycle.  So a CTA works on two
// tiles of 128 rows at once: while the softmax of one runs on the CUDA cores the products of the other run on the tensor cores.
//   warps 0-7, 8-15  softmax of row tile 0, 1: a row (= TMEM lane) belongs to two threads, each with 64 of its 128 scores.  Scores from
//                    TMEM, running maximum, exponentials, probabilities as bf16 back into TMEM over the scores.  The output in
//                    TMEM is rescaled only where a maximum has grown by more than 8 (a factor 2^8, which fp32 sums and bf16
//                    probabilities bear); then by these warps.  Up to 128 rows both tiles hold the same rows, each with every
//                    other tile of keys, and are joined at the end: the alternation stays.
//   warp 16          issues the products: S_t = Q_t K^T (both from shared memory) and O_t += P_t V (P from TMEM, V as it lies, key by key:
//                    an MN-major operand)
//   warps 17, 18     fill the ring of K and V tiles by TMA, one box per run of tokens in one page
//   warp 19          zeroes what lies beyond the end in the last values of an item, and before the window in the first (bf16 caches; the
//                    widening sees to it for the others)
//   warps 20-27      8-bit caches only: turn codes into bf16 tiles, exactly (the row's scale is a power of two)
// TMEM: S_0, S_1 (128 columns each), O_0, O_1.
// Measured, 32 query heads on 8 kv heads x 128, bf16: 2048 new tokens of 33333 1000 to 1050 us in a run of seconds, 1.05 PFLOP/s; 880 us in one of
// milliseconds (tensor pipe 67 %, exponentials 70 % of the time, the clock at 1.5 GHz for power); six prompts of 129 to 903 tokens 112 us.  e4m3 in a
// window of 4096, two chunks of 1000 tokens: 166 us, where widening the codes beside the softmax makes issue the limit.
#include "kv_attention.cuh"

namespace siso {
namespace kva {
namespace tc {

using namespace umma2;

constexpr int TK = 128;
constexpr int PRODUCERS = 2;
constexpr int EXTRA = 2;               // units that an item's beginning and end cost: 4.6 us were measured, a unit takes 1.6 to 2

struct Bars {
    uint64_t q_full[2], s_full[2], p_full[2][2], o_done[2];
    uint64_t kv_full[6], kv_empty[6], landed[6], raw_full[4], raw_empty[4];
    uint32_t blocks[8];        // of unit i at i % 8: which runs of 8 keys have a page in the pool
    Run run;
    uint32_t tmem;
    int gave_up;
    unsigned long long buf[31];
    float peer[2][2][128];     // a row's maximum, or sum, on its way to the other thread of the row
};

template <int KIND, int D> struct Shape {
    static constexpr bool EIGHT = KIND != SISO_BF16;
    static constexpr int THREADS = EIGHT ? 896 : 640;
    static constexpr int Q_BYTES = 2 * 128 * D * 2;
    static constexpr int TILE = TK * D * 2;                              // a tile of K or V in bf16
    static constexpr int RAW = EIGHT ? TK * D : 0;                       // and as codes
    static constexpr int RAW_META = EIGHT ? TK : 0;                      // exponents
    static constexpr int ROOM = 232448 - static_cast<int>(sizeof(Bars)) - Q_BYTES;
    static constexpr int RAWS = EIGHT ? (D == 128 ? 2 : 4) : 0;
    static constexpr int FIT = (ROOM - RAWS * (RAW + RAW_META)) / TILE;
    static constexpr int STAGES = FIT > 6 ? 6 : FIT;
    static constexpr int SMEM = Q_BYTES + STAGES * TILE + RAWS * (RAW + RAW_META) + static_cast<int>(sizeof(Bars));
    // registers: what the CTA has at launch (96 x 640 or 72 x 896), moved to the softmax
    static constexpr int SOFTMAX_REGS = EIGHT ? 96 : 104, OTHER_REGS = EIGHT ? 40 : 64, CONVERT_REGS = 40;
    // pairs of 8 whose exponentials are taken on the FMA pipe: of d = 64 their own pipe is the limit (chunk over 33333: none 735 us,
    // two 657 us), of d = 128 (863 us; two 880 us) and of 8 bits the issue of instructions
    static constexpr int POLY = EIGHT ? 0 : (D == 64 ? 2 : 0);
    static_assert(4 * SOFTMAX_REGS + OTHER_REGS + (EIGHT ? 2 * CONVERT_REGS : 0) == (EIGHT ? 7 * 72 : 5 * 96), "register split");
};

// D fp32, A and B bf16; A from shared memory or TMEM, K-major; B K-major, or MN-major (bit 16)
template <int N, bool MN>
constexpr uint32_t IDESC = (1u << 4) | (1u << 7) | (1u << 10) | (MN ? 1u << 16 : 0u) | (static_cast<uint32_t>(N >> 3) << 17) | (static_cast<uint32_t>(128 >> 4) << 24);
// B operand that lies key by key: rows of 128 bytes (64 d) 128-byte swizzled, 8 keys 1024 bytes apart, the next 64 d after TK rows
__device__ __forceinline__ uint64_t desc_mn(uint32_t saddr) {
    uint64_t d = 0;
    d |= static_cast<uint64_t>((saddr & 0x3FFFFu) >> 4);
    d |= static_cast<uint64_t>((TK * 128) >> 4) << 16;
    d |= static_cast<uint64_t>(1024 >> 4) << 32;
    d |= static_cast<uint64_t>(1) << 46;
    d |= static_cast<uint64_t>(2) << 61;
    return d;
}
__device__ __forceinline__ bool elect_one() {
    uint32_t one;
    asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xFFFFFFFF;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(one));
    return one != 0u;
}
__device__ __forceinline__ void mma_ts(uint32_t d, uint32_t a, uint64_t b, uint32_t id, uint32_t accumulate) {
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "setp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}"
        ::"r"(d), "r"(a), "l"(b), "r"(id), "r"(accumulate) : "memory");
}
// 16 columns, complete on return
__device__ __forceinline__ void tmem_ld_32x16(uint32_t taddr, uint32_t (&r)[16]) {
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x16.b32 "
        "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];\n\t"
        "tcgen05.wait::ld.sync.aligned;"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]), "=r"(r[10]),
          "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
        : "r"(taddr) : "memory");
}
__device__ __forceinline__ void tmem_st_32x16(uint32_t taddr, const uint32_t (&r)[16]) {
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x16.b32 [%16], "
        "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15};"
        ::"r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]),
          "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]), "r"(taddr) : "memory");
}
__device__ __forceinline__ void tmem_st_32x8(uint32_t taddr, const uint32_t (&r)[8]) {
    asm volatile("tcgen05.st.sync.aligned.32x32b.x8.b32 [%8], {%0, %1, %2, %3, %4, %5, %6, %7};"
                 ::"r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(taddr) : "memory");
}
__device__ __forceinline__ void tmem_st_wait() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
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
__device__ __forceinline__ float max3(float a, float b, float c) {
    float d;
    asm("max.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(a), "f"(b), "f"(c));
    return d;
}
// 2^x for x in [-126, 127] (below: as -126) on the FMA pipe: x = n + f with n whole and f in [-1/2, 1/2], a polynomial of degree 4 for 2^f
// (largest relative error on the interval minimised numerically: 2.7e-6, a thousandth of what rounding to bf16 adds), n added to the exponent
__device__ __forceinline__ float2 ex2_poly(float2 x) {
    x.x = fmaxf(x.x, -126.f);
    x.y = fmaxf(x.y, -126.f);
    const float big = 12582912.f;                     // 1.5 2^23: adding it rounds to a whole number, which then stands in the low bits
    const float2 t = add2(x, make_float2(big, big));
    const float2 f = add2(x, fma2(t, make_float2(-1.f, -1.f), make_float2(big, big)));
    float2 y = make_float2(0.009570102207362652f, 0.009570102207362652f);
    y = fma2(y, f, make_float2(0.05591786280274391f, 0.05591786280274391f));
    y = fma2(y, f, make_float2(0.240247443318367f, 0.240247443318367f));
    y = fma2(y, f, make_float2(0.6931217908859253f, 0.6931217908859253f));
    y = fma2(y, f, make_float2(0.9999992847442627f, 0.9999992847442627f));
    y.x = __uint_as_float(__float_as_uint(y.x) + (__float_as_uint(t.x) << 23));
    y.y = __uint_as_float(__float_as_uint(y.y) + (__float_as_uint(t.y) << 23));
    return y;
}
// bits first .. last of 32, as far as there are such; every bit of the lowest four as eight
__device__ __forceinline__ uint32_t bits_between(int first, int last) {
    const uint32_t from = first <= 0 ? 0xFFFFFFFFu : first > 31 ? 0u : 0xFFFFFFFFu << first;
    return from & (last >= 31 ? 0xFFFFFFFFu : last < 0 ? 0u : 0xFFFFFFFFu >> (31 - last));
}
__device__ __forceinline__ uint32_t bits_of_blocks(uint32_t b) { return ((b & 1u) | (b & 2u) << 7 | (b & 4u) << 14 | (b & 8u) << 21) * 0xFFu; }
// Lane i of every four has pieces 0 to 3 of row i: afterwards it has piece i of rows 0 to 3
__device__ __forceinline__ void swap_piece(uint4 &keep, uint4 &give, int mask, bool upper) {      // lanes with `upper` give `keep`'s place away
    const uint4 x = upper ? keep : give;
    const uint4 y = make_uint4(__shfl_xor_sync(0xFFFFFFFFu, x.x, mask), __shfl_xor_sync(0xFFFFFFFFu, x.y, mask), __shfl_xor_sync(0xFFFFFFFFu, x.z, mask),
                               __shfl_xor_sync(0xFFFFFFFFu, x.w, mask));
    if (upper) keep = y; else give = y;
}
__device__ __forceinline__ void turn4(uint4 (&w)[4], int lane) {
    swap_piece(w[0], w[1], 1, lane & 1);
    swap_piece(w[2], w[3], 1, lane & 1);
    swap_piece(w[0], w[2], 2, lane & 2);
    swap_piece(w[1], w[3], 2, lane & 2);
}

template <int KIND, int D, bool TREE>
__global__ void __launch_bounds__(Shape<KIND, D>::THREADS, 1)
attention_many_rows_kernel(const __grid_constant__ Args g, const __grid_constant__ CUtensorMap map_k, const __grid_constant__ CUtensorMap map_v) {
    using S = Shape<KIND, D>;
    constexpr bool EIGHT = S::EIGHT;
    constexpr int STAGES = S::STAGES, RAWS = S::RAWS;
    constexpr int RB = D * (EIGHT ? 1 : 2), LINE = RB < 128 ? RB : 128;
    extern __shared__ __align__(1024) uint8_t smem[];           // all of it: nothing static, so that it begins on a boundary of the swizzle
    uint8_t *q_smem = smem, *tiles = smem + S::Q_BYTES, *raws = tiles + STAGES * S::TILE, *metas = raws + RAWS * S::RAW;
    Bars &bars = *reinterpret_cast<Bars *>(metas + RAWS * S::RAW_META);
    unsigned long long *buf = bars.buf;

    if constexpr (TREE) wait_for_earlier();                     // (launched early: its mask is often the kernel before it)
    dependents_may_start();
    const int lane = threadIdx.x & 31, warp = __shfl_sync(0xFFFFFFFFu, static_cast<int>(threadIdx.x >> 5), 0);      // (uniform)
    if (threadIdx.x == 0) {
        for (int t = 0; t < 2; ++t) { mbar_init(&bars.q_full[t], 8); mbar_init(&bars.s_full[t], 1); mbar_init(&bars.p_full[t][0], 8); mbar_init(&bars.p_full[t][1], 8); mbar_init(&bars.o_done[t], 1); }
        for (int i = 0; i < STAGES; ++i) { mbar_init(&bars.kv_full[i], EIGHT ? 8 : 1); mbar_init(&bars.kv_empty[i], 1); mbar_init(&bars.landed[i], 1); }
        for (int i = 0; i < RAWS; ++i) { mbar_init(&bars.raw_full[i], 33); mbar_init(&bars.raw_empty[i], 8); }
        bars.gave_up = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    }
    __syncthreads();
    // a tree's row tiles are often half empty: they count a sixth less, and an item's beginning and end three tiles and a third, as measured over 24 trees of 119 to 441 rows (cycles
    // of a CTA = 8514 items + 2610 full tiles + 2165 half tiles).  Not over 8 bits, where widening a key tile costs as much for few rows as for many
    constexpr bool HALF = TREE && !EIGHT;
    constexpr int W = HALF ? 6 : 1, MORE = HALF ? 20 : EXTRA;
    Cursor<TC_ROWS, TK, MORE, W, HALF> cur;
    {
        Run run;
        if (!locate<TC_ROWS, TK, MORE, W, S::THREADS, HALF>(g, run, cur, buf)) return;
        if (threadIdx.x == 0) bars.run = run;
    }
    if (warp == 16) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&bars.tmem)), "r"(512u) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    tcgen05_fence_before();
    __syncthreads();
    tcgen05_fence_after();
    const uint32_t tmem = bars.tmem;
    volatile int *gave_up = &bars.gave_up;

    if (warp >= 20) {
        if constexpr (EIGHT) {
            // ---- codes -> bf16 tiles.  8 (4) lanes share a row of 128 (64) bytes: conflict-free loads; each writes two chunks of 8 values,
            // lanes of the upper half of a row the second one first
            asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(S::CONVERT_REGS));
            constexpr int CH = RB / 16, PER = 32 / CH, MINE = TK / 8;     // chunks of a row, rows of a warp's step, rows of a warp
            const int chunk = lane % CH, r0 = (warp - 20) * MINE + lane / CH, flip = CH == 8 ? chunk >> 2 : 0;
            // rows PER further on: the same place in the swizzle, or (PER = 4) bit 6 flipped
            const int src0 = chunk_at<RB, TK>(r0, chunk), dst0 = chunk_at<2 * D, TK>(r0, 2 * chunk + flip), dst1 = chunk_at<2 * D, TK>(r0, 2 * chunk + 1 - flip);
            int stage = 0, raw = 0;
            uint32_t phase = 0, raw_phase = 0;
            do {
                const int j0 = (cur.s.tile0 + cur.tile) * TK, left = cur.s.hi - j0, before = cur.lo(g) - j0;      // rows [before, left) of the tile are there
                for (int is_v = 0; is_v < 2; ++is_v) {
                    wait_bar(&bars.raw_full[raw], raw_phase, gave_up, g.status);
                    wait_bar(&bars.kv_empty[stage], phase ^ 1u, gave_up, g.status);
                    const uint8_t *src = raws + raw * S::RAW, *exps = metas + raw * S::RAW_META + r0;
                    if (is_v && (left < TK || before > 0)) {
                        // anything may stand in the other rows: a scale of 2^-127 makes it finite, and their probabilities are zero
                        const int r = (warp - 20) * MINE + lane;
                        if (lane < MINE && (r >= left || r < before)) metas[raw * S::RAW_META + r] = 0;
                        __syncwarp();
                    }
                    uint8_t *dst = tiles + stage * S::TILE;
#pragma unroll
                    for (int i = 0; i < MINE / PER; ++i) {
                        const int x = PER == 4 ? (i & 1) << 6 : 0;
                        const uint4 w = *reinterpret_cast<const uint4 *>(src + (src0 ^ x) + i * PER * RB);
                        const CodeScale<KIND> scale(exps[i * PER]);
                        const uint32_t in[4] = {w.x, w.y, w.z, w.w};
                        uint32_t out[8];
#pragma unroll
                        for (int k = 0; k < 4; ++k) scale.widen(in[k], out[2 * k], out[2 * k + 1]);
                        const uint4 a = make_uint4(out[0], out[1], out[2], out[3]), b = make_uint4(out[4], out[5], out[6], out[7]);
                        *reinterpret_cast<uint4 *>(dst + (dst0 ^ x) + i * PER * 128) = flip ? b : a;
                        *reinterpret_cast<uint4 *>(dst + (dst1 ^ x) + i * PER * 128) = flip ? a : b;
                    }
                    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                    __syncwarp();
                    if (lane == 0) { mbar_arrive(&bars.kv_full[stage]); mbar_arrive(&bars.raw_empty[raw]); }
                    if (++stage == STAGES) { stage = 0; phase ^= 1u; }
                    if (++raw == RAWS) { raw = 0; raw_phase ^= 1u; }
                }
            } while (cur.step(g));
        }
    } else if (warp >= 16) {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(S::OTHER_REGS));
        if (warp == 19) {
            if constexpr (!EIGHT) {
                // ---- what lies beyond the end or before the window in an item's values may be anything: zeros, or 0 times NaN would reach the sums
                int stage = 0;
                uint32_t phases = 0;                          // bit i: the round that stage i's barrier is in
                do {
                    if (++stage == STAGES) stage = 0;
                    const int j0 = (cur.s.tile0 + cur.tile) * TK, left = cur.s.hi - j0, before = cur.lo(g) - j0;
                    if (left < TK || before > 0) {
                        wait_bar(&bars.landed[stage], (phases >> stage) & 1u, gave_up, g.status);
                        phases ^= 1u << stage;
                        uint8_t *dst = tiles + stage * S::TILE;
                        auto clear = [&](int from, int to) {
                            for (int x = from * (RB / 16) + lane; x < to * (RB / 16); x += 32)
                                *reinterpret_cast<uint4 *>(dst + chunk_at<RB, TK>(x / (RB / 16), x % (RB / 16))) = make_uint4(0u, 0u, 0u, 0u);
                        };
                        clear(0, before);
                        clear(max(left, 0), TK);
                        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                        __syncwarp();
                        if (lane == 0) mbar_arrive(&bars.kv_full[stage]);
                    }
                    if (++stage == STAGES) stage = 0;
                } while (cur.step(g));
            }
        } else if (warp > 16) {
            // ---- producers: K and V tiles alternate in the ring; lanes 0-15 own the tile's runs of 8 tokens
            constexpr int RING = EIGHT ? RAWS : STAGES;
            const int box_blocks = g.box / 8;
            int stage = 0, unit = 0;
            uint32_t phase = 0;
            // this lane's run of 8 tokens of a unit; the page index is asked for one unit before it is needed
            struct Place { int head, tok, page; bool wanted, edge; } at;       // edge: part of the values is zeroed, by warp 19 for bf16 caches
            auto look_up = [&](Place &p) {
                const int j0 = (cur.s.tile0 + cur.tile) * TK;
                p.head = cur.head;
                p.edge = j0 + TK > cur.s.hi || j0 < cur.lo(g);
                const int j = j0 + (lane & 15) * 8, i = static_cast<int>(g.by_page.div(static_cast<uint32_t>(j)));
                p.tok = j - i * g.kv.page_size;
                const bool wanted = lane < 16 && holds_seen(g, cur.lo(g), cur.s.hi, j);
                p.page = wanted ? g.a.d_pages[cur.b * g.a.pages_stride + i] : -1;
                p.wanted = wanted;
            };
            look_up(at);
            for (bool more = true; more; ++unit) {
                Place ahead = at;
                more = cur.step(g);
                if (more) look_up(ahead);
                const bool wanted = at.wanted, in_pool = wanted && at.page >= 0 && at.page < g.kv.n_pages;
                if (wanted && !in_pool) set_status(g.status, SISO_ERR_INVALID_ARG);
                const bool first = wanted && lane % box_blocks == 0;
                const uint32_t there = __ballot_sync(0xFFFFFFFFu, in_pool);
                const uint32_t boxes = __popc(__ballot_sync(0xFFFFFFFFu, first));
                for (int is_v = 0; is_v < 2; ++is_v) {
                    if (stage % PRODUCERS == warp - 17) {         // a stage is always filled by the same warp, so its rounds come in order
                        uint64_t *full = EIGHT ? &bars.raw_full[stage] : &bars.kv_full[stage];
                        wait_bar(EIGHT ? &bars.raw_empty[stage] : &bars.kv_empty[stage], phase ^ 1u, gave_up, g.status);
                        uint8_t *dst = EIGHT ? raws + stage * S::RAW : tiles + stage * S::TILE;
                        uint64_t *bar = !EIGHT && is_v && at.edge ? &bars.landed[stage] : full;
                        if (*gave_up == 0) {
                            if (lane == 0) {
                                if (!is_v) bars.blocks[unit & 7] = there;
                                mbar_arrive_expect_tx(bar, boxes * (g.box * RB));
                            }
                            __syncwarp();
                            if (first) {
                                // a page outside the pool is asked for at a place beyond the tensor's end, which reads as zeros
                                const int p = in_pool ? at.page : static_cast<int>(g.kv.n_pages);
#pragma unroll
                                for (int half = 0; half < RB / LINE; ++half)
                                    load_box(smem_u32(dst) + half * (TK * 128) + lane * 8 * LINE, is_v ? &map_v : &map_k, half * 64, at.head, at.tok, p, g.a.layer, bar);
                            }
                            if constexpr (EIGHT) {
                                const long long e = in_pool ? (static_cast<long long>(at.page) * g.kv.n_kv_heads + at.head) * g.kv.page_size + at.tok : 0;
                                if (lane < 16)
                                    asm volatile("cp.async.ca.shared.global [%0], [%1], 8, %2;" ::"r"(smem_u32(metas + stage * S::RAW_META + lane * 8)),
                                                 "l"((is_v ? g.kv.v_exp : g.kv.k_exp) + e), "r"(in_pool ? 8 : 0) : "memory");
                                asm volatile("cp.async.mbarrier.arrive.noinc.shared.b64 [%0];" ::"r"(smem_u32(bar)) : "memory");
                            }
                        }
                    }
                    if (++stage == RING) { stage = 0; phase ^= 1u; }
                }
                at = ahead;
            }
            if constexpr (EIGHT) asm volatile("cp.async.wait_all;" ::: "memory");
        } else {
            // ---- products.  The whole warp goes through the loop, so that addresses and descriptors stay in uniform registers; one
            // lane issues
            const uint32_t base = __shfl_sync(0xFFFFFFFFu, tmem, 0);
            const uint64_t q_desc = smem_desc_sw128(smem_u32(q_smem)), k_desc = smem_desc_sw128(smem_u32(tiles)), v_desc = desc_mn(smem_u32(tiles));
            int k_stage = 0, v_stage = 1;                   // K and V tiles alternate in the ring
            uint32_t k_phase = 0, v_phase = 0, q_phase = 0, p_phases = 0;
            auto next = [&](int &stage, uint32_t &phase) __attribute__((always_inline)) {
                stage += 2;
                if (stage >= STAGES) { stage -= STAGES; phase ^= 1u; }
            };
            auto release = [&](int stage) __attribute__((always_inline)) {
                if (elect_one()) umma_commit(&bars.kv_empty[stage]);
                __syncwarp();
            };
            auto scores = [&](int t) __attribute__((always_inline)) {                      // S_t = Q_t K^T
                const uint64_t a = q_desc + static_cast<uint64_t>(t * (S::Q_BYTES / 2 >> 4)), b = k_desc + static_cast<uint64_t>(k_stage * (S::TILE >> 4));
                if (elect_one()) {
#pragma unroll
                    for (int k = 0; k < D / 16; ++k) {      // 32 bytes further along a line, or the next 64 d
                        const uint64_t off = static_cast<uint64_t>(2 * (k % 4) + (k / 4) * ((TK * 128) >> 4));
                        umma_bf16(base + t * 128, a + off, b + off, IDESC<128, false>, k ? 1u : 0u);
                    }
                    umma_commit(&bars.s_full[t]);
                }
                __syncwarp();
            };
            auto values = [&](int t, bool fresh) __attribute__((always_inline)) {          // O_t += P_t V, or O_t = P_t V
                const uint64_t b = v_desc + static_cast<uint64_t>(v_stage * (S::TILE >> 4));
#pragma unroll
                for (int c = 0; c < 2; ++c) {               // the first 32 keys of both halves, the others: each as soon as its probabilities are there
                    wait_bar(&bars.p_full[t][c], (p_phases >> t) & 1u, gave_up, g.status);
                    tcgen05_fence_after();
                    if (elect_one()) {
#pragma unroll
                        for (int h = 0; h < 2; ++h)
#pragma unroll
                            for (int k = 2 * c; k < 2 * c + 2; ++k)
                                mma_ts(base + 256 + t * D, base + t * 128 + 64 * h + 8 * k, b + static_cast<uint64_t>((4 * h + k) * (2048 >> 4)), IDESC<D, true>,
                                       (!fresh || c > 0 || h > 0 || k > 0) ? 1u : 0u);
                        if (c == 1) umma_commit(&bars.o_done[t]);
                    }
                    __syncwarp();
                }
                p_phases ^= 1u << t;
            };
            int n;
            do {
                n = __shfl_sync(0xFFFFFFFFu, cur.tiles_here(g), 0);
                wait_bar(&bars.q_full[0], q_phase, gave_up, g.status);
                wait_bar(&bars.q_full[1], q_phase, gave_up, g.status);
                q_phase ^= 1u;
                // two tiles of rows, each with every tile of keys; or one twice, each with every other tile of keys.  (One loop for both:
                // unrolled for each it spilled, six prompts 116 us and not 108)
                const bool split = __any_sync(0xFFFFFFFFu, cur.n_q * g.group - cur.rt * TC_ROWS <= 128);
                const int ahead = split ? 2 : 1, per_tile = split ? 1 : 2;
                for (int j = -ahead; j < n; ++j) {
                    if (j >= 0) wait_bar(&bars.kv_full[v_stage], v_phase, gave_up, g.status);
                    for (int i = 0; i < per_tile; ++i) {
                        const int t = split ? j & 1 : i;
                        if (j >= 0) values(t, j < ahead);
                        if (j >= 0 && i + 1 == per_tile) {
                            release(v_stage);
                            next(v_stage, v_phase);
                        }
                        if (j + ahead < n) {
                            if (i == 0) wait_bar(&bars.kv_full[k_stage], k_phase, gave_up, g.status);
                            tcgen05_fence_after();
                            scores(t);
                            if (i + 1 == per_tile) {
                                release(k_stage);
                                next(k_stage, k_phase);
                            }
                        }
                    }
                }
            } while (cur.step(g, n));
        }
    } else {
        // ---- softmax: half of a row of one tile
        asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(S::SOFTMAX_REGS));
        const int t = warp >> 3, half = (warp >> 2) & 1, lane_row = threadIdx.x & 127;
        const uint32_t lane_at = static_cast<uint32_t>((warp & 3) * 32) << 16;
        const uint32_t s_at = tmem + lane_at + t * 128 + half * 64, o_at = tmem + lane_at + 256 + t * D + half * (D / 2);
        const bool causal = (g.a.flags & SISO_ATTN_CAUSAL) != 0u;
        // the sign of the scale goes to the queries, so that the largest product is the largest score; scale 0: queries of zeros
        const float scale = g.scale_log2 == 0.f ? 1.f : fabsf(g.scale_log2);
        float &mine_out = bars.peer[t][half][lane_row], &theirs_in = bars.peer[t][half ^ 1][lane_row];
        uint32_t tile_phase = 0;
        int unit = 0;                                                     // units of this CTA so far
        bool pending = false, split = false;                              // an item whose output is still in TMEM, in two parts
        float m = -INFINITY, l = 0.f;
        int out_token = -1, out_head = 0, out_place = -1;                 // of that item: where the row goes, or its place among the parts
        auto together = [&]() { asm volatile("bar.sync %0, 256;" ::"r"(1 + t) : "memory"); };
        auto everyone = [&]() { asm volatile("bar.sync 3, 512;" ::: "memory"); };
        auto store_item = [&](bool split_item) {
            const bool to_part = __any_sync(0xFFFFFFFFu, out_place >= 0), split = __any_sync(0xFFFFFFFFu, split_item);      // (uniform, visibly)
            wait_bar(&bars.o_done[t], tile_phase ^ 1u, gave_up, g.status);
            tcgen05_fence_after();
            mine_out = l;
            together();
            float sum = half ? theirs_in + l : l + theirs_in;             // the same sum in both threads
            float f0 = 1.f, f1 = 0.f;
            if (split) {                                                  // the rows' other tiles of keys are with the other tile
                if (t == 1) {
                    together();
                    if (half == 0) { bars.peer[1][0][lane_row] = m; bars.peer[1][1][lane_row] = sum; }
                    tcgen05_fence_before();
                    everyone();
                    everyone();                                           // until that output has been read
                    tcgen05_fence_after();
                    return;
                }
                everyone();
                tcgen05_fence_after();
                const float m1 = bars.peer[1][0][lane_row], l1 = bars.peer[1][1][lane_row], m2 = fmaxf(m, m1);
                f0 = m == -INFINITY ? 0.f : ex2(m - m2);
                f1 = m1 == -INFINITY ? 0.f : ex2(m1 - m2);
                sum = sum * f0 + l1 * f1;
                m = m2;
            }
            if (m == -INFINITY && sum == sum) sum = 0.f;                  // nothing seen (the sum may hold remainders of 2^-126)
            const float inv = inverse_of(sum);
#pragma unroll 1
            for (int c = 0; c < D / 64; ++c) {
                uint32_t r[32];
                tmem_ld_32x32(o_at + c * 32, r);
                tmem_ld_fence(r);
                if (split) {
#pragma unroll
                    for (int p = 0; p < 32; p += 16) {
                        uint32_t y[16];
                        tmem_ld_32x16(o_at + D + c * 32 + p, y);
#pragma unroll
                        for (int i = 0; i < 16; ++i)                      // (an output without tiles holds anything)
                            r[p + i] = __float_as_uint((f0 == 0.f ? 0.f : f0 * __uint_as_float(r[p + i])) + (f1 == 0.f ? 0.f : f1 * __uint_as_float(y[i])));
                    }
                }
                if constexpr (EIGHT) {                                    // d 0 2 1 3 of every four
#pragma unroll
                    for (int i = 0; i < 32; i += 4) { const uint32_t x = r[i + 1]; r[i + 1] = r[i + 2]; r[i + 2] = x; }
                }
                // four lanes turn their four pieces of 16 bytes round, so that they write 64 bytes of a row together
                if (!to_part) {
                    uint4 w[4];
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        w[i] = make_uint4(pack(__uint_as_float(r[8 * i]) * inv, __uint_as_float(r[8 * i + 1]) * inv, false),
                                          pack(__uint_as_float(r[8 * i + 2]) * inv, __uint_as_float(r[8 * i + 3]) * inv, false),
                                          pack(__uint_as_float(r[8 * i + 4]) * inv, __uint_as_float(r[8 * i + 5]) * inv, false),
                                          pack(__uint_as_float(r[8 * i + 6]) * inv, __uint_as_float(r[8 * i + 7]) * inv, false));
                    turn4(w, lane);
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const int token = __shfl_sync(0xFFFFFFFFu, out_token, (lane & ~3) + i), head = __shfl_sync(0xFFFFFFFFu, out_head, (lane & ~3) + i);
                        if (token >= 0)
                            *reinterpret_cast<uint4 *>(static_cast<__nv_bfloat16 *>(g.a.d_out) + static_cast<long long>(token) * g.a.out_stride_token +
                                                       static_cast<long long>(head) * g.a.out_stride_head + half * (D / 2) + c * 32 + (lane & 3) * 8) = w[i];
                    }
                } else {
                    // (places of neighbouring rows are neighbours; unused rows are never read, nor written)
                    const uint32_t real = __ballot_sync(0xFFFFFFFFu, out_token >= 0) >> (lane & ~3);
                    float *dst = g.part_o + static_cast<long long>(out_place - (lane & 3)) * D + half * (D / 2) + c * 32 + (lane & 3) * 4;
#pragma unroll
                    for (int p = 0; p < 2; ++p) {
                        uint4 w[4];
#pragma unroll
                        for (int i = 0; i < 4; ++i) w[i] = make_uint4(r[16 * p + 4 * i], r[16 * p + 4 * i + 1], r[16 * p + 4 * i + 2], r[16 * p + 4 * i + 3]);
                        turn4(w, lane);
#pragma unroll
                        for (int i = 0; i < 4; ++i)
                            if ((real >> i) & 1u) *reinterpret_cast<uint4 *>(dst + i * D + p * 16) = w[i];
                    }
                }
            }
            if (out_token >= 0 && half == 0) {
                if (out_place >= 0) *reinterpret_cast<float2 *>(g.part_ml + 2ll * out_place) = make_float2(m, sum);
                else if (g.a.d_lse) g.a.d_lse[static_cast<long long>(out_token) * g.a.n_heads + out_head] = lse_of(m, sum);
            }
            tcgen05_fence_before();
            if (split) everyone();
            else together();                                              // the exchange place is free again
        };
        for (bool more = true;;) {
            const int rows = cur.n_q * g.group - cur.rt * TC_ROWS;        // rows of the item from this row tile on
            const bool split_next = __any_sync(0xFFFFFFFFu, rows <= 128);      // (uniform, visibly)  one tile of rows twice, with every other tile of keys
            const int tile_row = split_next ? 0 : t * 128, in_tile = tile_row + lane_row;
            if (more) {   // the last scores of the item before have come, so its queries are no longer read.  8 (4) lanes share half a row
                const uint32_t flip = g.scale_log2 < 0.f ? 0x80008000u : 0u, keep = g.scale_log2 == 0.f ? 0u : 0xFFFFFFFFu;
                constexpr int LANES = D / 16, PER = 32 / LANES;
                uint8_t *dst = q_smem + t * (S::Q_BYTES / 2);
                const int c = half * LANES + lane % LANES, first = (warp & 3) * 32 + lane / LANES;
                uint4 x[32 / PER];
#pragma unroll
                for (int y = 0; y < 32 / PER; ++y) {
                    const int at = tile_row + first + y * PER, r = cur.rt * TC_ROWS + at;
                    x[y] = make_uint4(0u, 0u, 0u, 0u);
                    if (at < rows) {
                        const int tok = static_cast<int>(g.by_group.div(static_cast<uint32_t>(r)));
                        x[y] = *reinterpret_cast<const uint4 *>(static_cast<const __nv_bfloat16 *>(g.a.d_q) + static_cast<long long>(cur.q0 + tok) * g.a.q_stride_token +
                                                                static_cast<long long>(cur.head * g.group + r - tok * g.group) * g.a.q_stride_head + c * 8);
                    }
                }
#pragma unroll
                for (int y = 0; y < 32 / PER; ++y) {
                    uint32_t w[4] = {(x[y].x ^ flip) & keep, (x[y].y ^ flip) & keep, (x[y].z ^ flip) & keep, (x[y].w ^ flip) & keep};
                    if constexpr (EIGHT) {                            // the order in which the codes come
#pragma unroll
                        for (int k = 0; k < 4; k += 2) {
                            const uint32_t a = w[k], b = w[k + 1];
                            w[k] = __byte_perm(a, b, 0x5410);
                            w[k + 1] = __byte_perm(a, b, 0x7632);
                        }
                    }
                    *reinterpret_cast<uint4 *>(dst + chunk_at<2 * D, TK>(first + y * PER, c)) = make_uint4(w[0], w[1], w[2], w[3]);
                }
                asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                __syncwarp();
                if (lane == 0) mbar_arrive(&bars.q_full[t]);
            }
            if (pending) store_item(split);
            if (!more) break;
            pending = true;
            const int n = cur.tiles_here(g);
            const bool real = in_tile < rows;
            const int row = cur.rt * TC_ROWS + (real ? in_tile : 0);
            const int i = static_cast<int>(g.by_group.div(static_cast<uint32_t>(row))), head = cur.head * g.group + row - i * g.group;
            split = split_next;
            out_token = real ? cur.q0 + i : -1;
            out_head = head;
            out_place = cur.tile == 0 && n == cur.s.tiles ? -1 : static_cast<int>(part_place(blockIdx.x, cur.tile > 0)) * TC_ROWS + in_tile;
            int pos = real ? position(cur.len, cur.n_q, i) : cur.s.last_pos;
            const int before = cur.len - cur.n_q;                         // TREE: tokens before the new ones
            const uint32_t *mask = nullptr;
            if constexpr (TREE) {
                mask = g.mask + static_cast<long long>(cur.q0 + (real ? i : 0)) * g.mask_stride;
                if (real && g.a.window > 0) pos = position(cur.len, cur.n_q, mask_depth(g, mask, cur.n_q));
            }
            m = -INFINITY;
            l = 0.f;
            const int k0 = split ? t : 0, k_step = split ? 2 : 1;
            uint32_t next_a = 0xFFFFFFFFu, next_b = 0xFFFFFFFFu;         // TREE: the row's bits for its 64 keys of a tile, asked for one tile ahead
            auto look_at_mask = [&](int k) {
                const int at = (cur.s.tile0 + cur.tile + k) * TK - before;
                if (at + TK > 0 && k < n) {
                    next_a = mask_bits(g, mask, at + half * 64);
                    next_b = mask_bits(g, mask, at + half * 64 + 32);
                }
            };
            if constexpr (TREE) look_at_mask(k0);
            for (int k = k0; k < n; k += k_step) {
                const int j0 = (cur.s.tile0 + cur.tile + k) * TK;
                const uint32_t see_a = next_a, see_b = next_b;
                if constexpr (TREE) look_at_mask(k + k_step);
                wait_bar(&bars.s_full[t], tile_phase, gave_up, g.status);
                tcgen05_fence_after();
                uint32_t ra[32], rb[32];
                tmem_ld_32x32(s_at, ra);
                tmem_ld_32x32(s_at + 32, rb);
                const uint32_t blocks = bars.blocks[(unit + k) & 7];
                const bool cut = j0 + TK > cur.s.hi || blocks != 0xFFFFu || (causal && j0 + TK - 1 > cur.s.first_pos) || (TREE && j0 + TK > before) ||
                                 (g.a.window > 0 && j0 <= (TREE ? cur.len - 1 : cur.s.last_pos) - g.a.window);
                tmem_ld_fence(ra);
                tmem_ld_fence(rb);
                if constexpr (TREE) {
                    if (cut) {   // as below, with the row's bits for the new tokens, as one bit a key
                        const int last = cur.s.hi - 1 - j0 - half * 64;
                        const int first = g.a.window > 0 ? min(max(pos - g.a.window + 1, 0), max(before, 0)) - j0 - half * 64 : 0;
                        const uint32_t there = blocks >> (half * 8);
                        const uint32_t in_a = see_a & bits_between(first, last) & bits_of_blocks(there), in_b = see_b & bits_between(first - 32, last - 32) & bits_of_blocks(there >> 4);
#pragma unroll
                        for (int x = 0; x < 32; ++x) {
                            if (!((in_a >> x) & 1u)) ra[x] = 0xFF800000u;
                            if (!((in_b >> x) & 1u)) rb[x] = 0xFF800000u;
                        }
                    }
                } else if (cut) {       // keys that are not seen, or not there, are left out by selection: they may hold anything
                    const int last = (causal ? min(pos, cur.s.hi - 1) : cur.s.hi - 1) - j0 - half * 64;
                    const int first = g.a.window > 0 ? max(pos - g.a.window + 1, 0) - j0 - half * 64 : 0;
                    const uint32_t my_blocks = blocks >> (half * 8);
#pragma unroll
                    for (int x = 0; x < 32; ++x) {
                        if (x > last || x < first || !((my_blocks >> (x / 8)) & 1u)) ra[x] = 0xFF800000u;
                        if (32 + x > last || 32 + x < first || !((my_blocks >> (4 + x / 8)) & 1u)) rb[x] = 0xFF800000u;
                    }
                }
                float top[4] = {__uint_as_float(ra[0]), __uint_as_float(ra[1]), __uint_as_float(rb[0]), __uint_as_float(rb[1])};
#pragma unroll
                for (int x = 2; x < 32; x += 4) {
                    top[0] = max3(top[0], __uint_as_float(ra[x]), __uint_as_float(ra[x + 1]));
                    top[2] = max3(top[2], __uint_as_float(rb[x]), __uint_as_float(rb[x + 1]));
                    if (x + 2 < 32) {
                        top[1] = max3(top[1], __uint_as_float(ra[x + 2]), __uint_as_float(ra[x + 3]));
                        top[3] = max3(top[3], __uint_as_float(rb[x + 2]), __uint_as_float(rb[x + 3]));
                    }
                }
                float m2 = fmaxf(m, max3(fmaxf(top[0], top[1]), top[2], top[3]) * scale);
                uint32_t grown;
                asm volatile(
                    "{\n\t.reg .pred p, q;\n\tsetp.ne.u32 p, %2, 0;\n\t"
                    "barrier.cta.red.or.aligned.pred q, %1, 256, p;\n\tselp.u32 %0, 1, 0, q;\n\t}"
                    : "=r"(grown) : "r"(1 + t), "r"((m2 > m + 8.f || (m == -INFINITY && m2 != m)) ? 1u : 0u) : "memory");
                if (__any_sync(0xFFFFFFFFu, grown)) {                     // (uniform, visibly: the barriers in it cost no registers then)
                    mine_out = m2;
                    together();
                    m2 = fmaxf(m2, theirs_in);
                    const float corr = m == m2 ? 1.f : ex2(m - m2);
                    m = m2;
                    l *= corr;
                    if (k > k0) {
                        wait_bar(&bars.o_done[t], tile_phase ^ 1u, gave_up, g.status);
                        tcgen05_fence_after();
#pragma unroll 1
                        for (int c = 0; c < D / 2; c += 16) {         // 16 columns at a time: the scores stay in registers
                            uint32_t y[16];
                            tmem_ld_32x16(o_at + c, y);
#pragma unroll
                            for (int x = 0; x < 16; ++x) y[x] = __float_as_uint(__uint_as_float(y[x]) * corr);
                            tmem_st_32x16(o_at + c, y);
                        }
                        tmem_st_wait();
                        tcgen05_fence_before();
                    }
                    together();        // no product of this unit begins before both halves of the output are rescaled
                    tcgen05_fence_after();
                }
                const float shift = m == -INFINITY ? 0.f : -m;
                float2 sum[2] = {make_float2(0.f, 0.f), make_float2(0.f, 0.f)};
                // 16 columns of probabilities at a time; what waits for their way into TMEM waits behind the next 16
                auto weigh = [&](const uint32_t (&r)[32], int from, int at) {
                    uint32_t p[8];
#pragma unroll
                    for (int x = 0; x < 8; ++x) {
                        float2 y = fma2(make_float2(__uint_as_float(r[from + 2 * x]), __uint_as_float(r[from + 2 * x + 1])), make_float2(scale, scale), make_float2(shift, shift));
                        if ((x * S::POLY) % 8 < S::POLY) y = ex2_poly(y);
                        else { y.x = ex2(y.x); y.y = ex2(y.y); }
                        sum[x & 1] = add2(sum[x & 1], y);
                        p[x] = pack(y.x, y.y, false);
                    }
                    tmem_st_32x8(s_at + at, p);
                };
                auto bring = [&](int c) {
                    tmem_st_wait();
                    tcgen05_fence_before();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(&bars.p_full[t][c]);
                };
                weigh(ra, 0, 0);
                weigh(ra, 16, 8);
                weigh(rb, 0, 16);
                bring(0);
                weigh(rb, 16, 24);
                bring(1);
                sum[0] = add2(sum[0], sum[1]);
                l += sum[0].x + sum[0].y;
                tile_phase ^= 1u;
            }
            if (threadIdx.x == 0 && cur.tile == 0 && n < cur.s.tiles) g.records[blockIdx.x] = record_of(cur.cost(g), bars.run, cur.left, cur.b, cur.head, cur.rt, cur.s.tiles, 0);
            unit += n;
            more = cur.step(g, n);
        }
    }

    // ---- teardown
    __syncwarp();
    let_copies_land(gave_up);
    tcgen05_fence_before();
    __syncthreads();
    if (warp == 16) {
        tcgen05_fence_after();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(512u) : "memory");
    }
}

template <int KIND, int D, bool TREE> static siso_status_t run_as(Kv *h, Args &g, cudaStream_t s) {
    using S = Shape<KIND, D>;
    constexpr uint32_t bit = 1u << (TREE ? 9 : 8);
    if (!(h->attr_set & bit)) {
        SISO_CUDA(cudaFuncSetAttribute(attention_many_rows_kernel<KIND, D, TREE>, cudaFuncAttributeMaxDynamicSharedMemorySize, S::SMEM));
        h->attr_set |= bit;
    }
    if constexpr (TREE) SISO_TRY(launch_early(attention_many_rows_kernel<KIND, D, TREE>, dim3(static_cast<unsigned>(g.grid)), S::THREADS, S::SMEM, s, g, h->map_k, h->map_v));
    else attention_many_rows_kernel<KIND, D, TREE><<<g.grid, S::THREADS, S::SMEM, s>>>(g, h->map_k, h->map_v);
    SISO_CUDA(cudaGetLastError());
    return launch_join(g, TC_ROWS, D, s);
}
template <int KIND, int D> static siso_status_t run(Kv *h, Args &g, cudaStream_t s) {
    return g.mask ? run_as<KIND, D, true>(h, g, s) : run_as<KIND, D, false>(h, g, s);
}

}  // namespace tc

siso_status_t launch_many_rows(Kv *h, Args &g, cudaStream_t s) {
    const bool wide = h->cfg.head_dim == 128;
    switch (h->cfg.dtype) {
        case SISO_BF16: return wide ? tc::run<SISO_BF16, 128>(h, g, s) : tc::run<SISO_BF16, 64>(h, g, s);
        case SISO_E4M3: return wide ? tc::run<SISO_E4M3, 128>(h, g, s) : tc::run<SISO_E4M3, 64>(h, g, s);
        default: return wide ? tc::run<SISO_I8, 128>(h, g, s) : tc::run<SISO_I8, 64>(h, g, s);
    }
}

}  // namespace kva
}  // namespace siso
