// Attention of new tokens over the paged key/value cache, few rows per key/value head: single tokens of decoding and short
// runs of drafted ones.
//
// Token i of sequence b (q_len new tokens, already in the cache, kv_len tokens in all) stands at p = kv_len - q_len + i and
// sees the tokens j in [0, kv_len) with j <= p (causal) and j > p - window (window > 0):
//     s_j = scale q.k_j,  m = max s,  l = sum exp(s_j - m),  out = sum exp(s_j - m) v_j / l,  lse = m + ln l
// A row that sees nothing gives out = 0 and lse = -infinity.
//
// With few rows every byte of the cache meets few multiplications, so the call is bound by HBM: the point is to keep loads in
// flight and to spend few instructions on a byte.  One CTA per SM: four producer warps fill a ring of units (128 keys and their
// values, about 190 KB in all) by TMA, one box per run of tokens that lie in one page, and 8 warps consume it.  A unit's keys
// are split over WK groups of WM warps; a warp owns 8 NT rows and its group's keys, so up to 16 rows (WM = 1) no byte is
// read from shared memory twice and no warp waits for another inside an item.
// Matrix products are mma.sync m16n8k16 with fp32 sums: tcgen05 works on 128 rows, of which a decoding step would fill 1 to 16.
// They are taken transposed, scores^T = K Q^T and out^T = V^T P^T, so that the rows fill the 8 columns and keys and d the 16 rows.
// K fragments come straight from 16-byte shared loads: the sum over d may be taken in any order, so a lane takes 16 consecutive
// bytes of its key and the queries are laid out to match.  V fragments come through ldmatrix.trans; over 8-bit codes it hands
// a lane the pairs (key, d), (key, d + 1), (key + 1, d), (key + 1, d + 1), the fragments of an even and an odd d.  Probabilities
// change from the first product's layout to the second's by movmatrix.
// 8-bit codes of keys are turned into fp16: one conversion per two codes, exact.  The key's scale goes to its score.  Queries are brought
// into fp16's range by a power of two per row (exact but for elements below 2^-31 of the row's largest).  Codes of values are turned into
// bf16, exactly, and the value's scale goes to its probability, relative to the largest one so far: probabilities and scales of
// neighbouring tokens may lie many powers of two apart, for which fp16 has no room (a probability of 2^-40 would be zero).  bf16 costs
// nothing over i8; over e4m3 (no conversion to it) 0 to 6 %: 64 sequences of 201 to 8190 tokens 109 us either way, head size 64 73 and 77 us.
// Measured, 8 kv heads x 128, 4 query heads each, caches in HBM: 64 sequences of 4096 tokens bf16 164 us, 6.5 TB/s (8192 tokens: 6.8 TB/s);
// 201 to 8190 tokens e4m3 110 us, 5.0 TB/s, where the dependent steps of a consumer warp on a unit are the limit; one sequence of 1025 tokens
// 10.1 us, latency.  (At head size 128 the shapes of 16 and 32 rows spill 24 to 68 bytes a thread.)
#include <cuda_fp16.h>

#include "kv_attention.cuh"

namespace siso {
namespace kva {

using umma2::mbar_arrive;
using umma2::mbar_arrive_expect_tx;
using umma2::mbar_init;
using umma2::smem_u32;

constexpr int SMEM_MOST = 232448 - 512 - 1024;   // what a CTA may have, less its static part and the alignment of the ring

constexpr int PRODUCERS = 4;             // warps that fill the ring; each has its own stages

template <int KIND, int D, int WM, int NT> struct Shape {
    static constexpr bool EIGHT = KIND != SISO_BF16;
    static constexpr int WK = 8 / WM;                       // groups of warps along a unit's keys
    static constexpr int WARPS = 8;                         // consumers
    static constexpr int T = EIGHT && NT == 1 ? 256 : 128;  // keys of a unit
    static constexpr int THREADS = 32 * (WARPS + PRODUCERS);
    static constexpr int PRODUCER_REGS = 40, CONSUMER_REGS = 232;
    static_assert(WARPS * CONSUMER_REGS + PRODUCERS * PRODUCER_REGS == (WARPS + PRODUCERS) * 168, "168 registers a thread at launch");
    static constexpr int MR = 8 * NT * WM;                  // rows of a row tile
    static constexpr int NK = T / WK;                      // keys of a group
    static constexpr int RB = D * (EIGHT ? 1 : 2);          // bytes of a row
    static constexpr int CH = RB / 16;                      // 16-byte chunks of a row
    static constexpr int STAGE = 2 * T * RB;
    static constexpr int META = EIGHT ? 2 * T : 0;         // exponents
    static constexpr int MERGE_O = WARPS / 2 * 8 * NT * D;  // outputs of half the warps
    static constexpr int MERGE = (MERGE_O + WARPS / 2 * 16 * NT) * 4;
    static constexpr int FIT = (SMEM_MOST - MERGE) / (STAGE + META);
    static constexpr int STAGES = FIT > 8 ? 8 : FIT;
    static constexpr int SMEM = STAGES * (STAGE + META) + MERGE + 1024;
};

// Which of 8 keys the n-th row of a product is.  The 8 lanes of one 16-byte load read 4 chunks of rows 2i and 2i + 1: those keys have
// to lie in different halves of their lines
template <int RB> __device__ __forceinline__ int key_of(int n) { return RB == 64 ? n : ((n & 1) << 2) | (n >> 1); }

template <bool HALF> __device__ __forceinline__ void mma(float (&c)[4], const uint32_t (&a)[4], const uint32_t (&b)[2]) {
    if constexpr (HALF)
        asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                     : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b[0]), "r"(b[1]));
    else
        asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                     : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b[0]), "r"(b[1]));
}
__device__ __forceinline__ uint32_t transposed(uint32_t x) {
    uint32_t y;
    asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
    return y;
}
__device__ __forceinline__ void load_v(uint32_t addr, uint32_t (&r)[4]) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
// Codes of keys as fp16: bytes 0, 1 and 2, 3 of a word
template <int KIND> __device__ __forceinline__ void widen(uint32_t w, uint32_t &lo, uint32_t &hi) {
    if constexpr (KIND == SISO_E4M3) {
        asm("{\n\t.reg .b16 l, h;\n\tmov.b32 {l, h}, %2;\n\tcvt.rn.f16x2.e4m3x2 %0, l;\n\tcvt.rn.f16x2.e4m3x2 %1, h;\n\t}"
            : "=r"(lo), "=r"(hi) : "r"(w));
    } else {
        w ^= 0x80808080u;                                   // c + 128; beside the byte 0x64 it is the fp16 number 1024 + c + 128
        const __half2 off = __halves2half2(__ushort_as_half(0x6480), __ushort_as_half(0x6480));
        const uint32_t a = __byte_perm(w, 0x64646464u, 0x4140), b = __byte_perm(w, 0x64646464u, 0x4342);
        const __half2 x = __hsub2(*reinterpret_cast<const __half2 *>(&a), off), y = __hsub2(*reinterpret_cast<const __half2 *>(&b), off);
        lo = *reinterpret_cast<const uint32_t *>(&x);
        hi = *reinterpret_cast<const uint32_t *>(&y);
    }
}
// Codes of values as bf16, exactly: bytes 0, 2 and 1, 3 of a word.  e4m3: 2^-120 of the code, subnormal ones too (see CodeScale).  i8: the
// byte u = c + 128 as the bits of a bf16 number is u 2^-133, in the subnormal range and in the first binade above it alike; times 2^127, less 2,
// it is c 2^-6.  UP powers of two more on the probabilities make up for these factors, or most of them, so that the sums of e4m3 stay in
// the middle of fp32's range; BACK for the rest
template <int KIND> constexpr int UP = KIND == SISO_E4M3 ? 100 : 6;
template <int KIND> constexpr float BACK = KIND == SISO_E4M3 ? 1048576.f : 1.f;
template <int KIND> __device__ __forceinline__ void widen_values(uint32_t w, uint32_t &lo, uint32_t &hi) {
    if constexpr (KIND == SISO_E4M3) {
        lo = ((w << 4) & 0x07F007F0u) | ((w << 8) & 0x80008000u);
        hi = ((w >> 4) & 0x07F007F0u) | (w & 0x80008000u);
    } else {
        w ^= 0x80808080u;
        asm("fma.rn.bf16x2 %0, %1, %2, %3;" : "=r"(lo) : "r"(__byte_perm(w, 0u, 0x4240)), "r"(0x7F007F00u), "r"(0xC000C000u));
        asm("fma.rn.bf16x2 %0, %1, %2, %3;" : "=r"(hi) : "r"(__byte_perm(w, 0u, 0x4341)), "r"(0x7F007F00u), "r"(0xC000C000u));
    }
}
template <int STAGES> struct Ring {
    uint64_t full[STAGES], empty[STAGES];
    uint32_t blocks[STAGES];           // bit i: the page of keys 8 i .. 8 i + 7 of the unit is in the pool
    int gave_up;
};

template <int KIND, int D, int WM, int NT>
__global__ void __launch_bounds__(Shape<KIND, D, WM, NT>::THREADS, 1)
attention_few_rows_kernel(const __grid_constant__ Args g, const __grid_constant__ CUtensorMap map_k, const __grid_constant__ CUtensorMap map_v) {
    using S = Shape<KIND, D, WM, NT>;
    constexpr int NK = S::NK, CH = S::CH, RB = S::RB, MR = S::MR, STAGES = S::STAGES, WK = S::WK, WARPS = S::WARPS, TK = S::T;
    constexpr bool EIGHT = S::EIGHT;
    constexpr int SUB = NK < 32 ? NK : 32;                   // keys between two looks at the running maximum
    constexpr uint32_t ALL = TK == 256 ? 0xFFFFFFFFu : 0xFFFFu;       // a bit per 8 keys
    constexpr int LINE = RB < 128 ? RB : 128;                // bytes of a row that lie together
    constexpr int KT = SUB / 16, DT = D / 16;                // tiles of 16 keys, of 16 d
    extern __shared__ uint8_t smem_raw[];
    __shared__ unsigned long long buf[S::THREADS / 32 + 3];
    __shared__ Ring<STAGES> ring;
    uint8_t *smem = smem_raw + ((1024u - (smem_u32(smem_raw) & 1023u)) & 1023u);      // (an offset: the loads stay shared loads)
    float *merge_o = reinterpret_cast<float *>(smem + STAGES * S::STAGE);
    float *merge_ml = merge_o + S::MERGE_O;
    uint8_t *meta = reinterpret_cast<uint8_t *>(merge_ml + WARPS / 2 * 16 * NT);

    dependents_may_start();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    if (threadIdx.x == 0) {
        for (int i = 0; i < STAGES; ++i) { mbar_init(&ring.full[i], EIGHT ? 33 : 1); mbar_init(&ring.empty[i], 8); }      // 33: the bytes, and the lanes' exponents
        ring.gave_up = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    }
    __syncthreads();
    Run run;
    Cursor<MR, TK, 1, 2> cur;            // an item's beginning and end: half a tile
    if (!locate<MR, TK, 1, 2, S::THREADS>(g, run, cur, buf)) return;
    volatile int *gave_up = &ring.gave_up;

    // registers move from the producers to the consumers: WARPS of CONSUMER_REGS and 4 of PRODUCER_REGS make what the CTA has
    if (warp >= WARPS) {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(S::PRODUCER_REGS));
        // ---- producers: lanes 0-15 own the unit's blocks of 8 keys, lanes 16-31 of 8 values, 16 blocks at a time
        constexpr int HALVES = TK / 128;
        const int is_v = lane >> 4;
        const CUtensorMap *map = is_v ? &map_v : &map_k;
        const uint8_t *exps = is_v ? g.kv.v_exp : g.kv.k_exp;
        const int box_blocks = g.box / 8;
        int stage = 0;
        uint32_t phase = 0;
        do {
            if (stage % PRODUCERS == warp - WARPS) {         // a stage is always filled by the same warp, so its rounds come in order
                int page[HALVES], tok[HALVES];
                bool first[HALVES];
                uint32_t there = 0u, boxes = 0u;
#pragma unroll
                for (int x = 0; x < HALVES; ++x) {
                    const int blk = x * 16 + (lane & 15), j = (cur.s.tile0 + cur.tile) * TK + blk * 8;
                    const int at = static_cast<int>(g.by_page.div(static_cast<uint32_t>(j)));
                    tok[x] = j - at * g.kv.page_size;
                    page[x] = -1;
                    const bool wanted = holds_seen(g, cur.lo(g), cur.s.hi, j);
                    if (wanted) {
                        page[x] = g.a.d_pages[cur.b * g.a.pages_stride + at];
                        if (page[x] < 0 || page[x] >= g.kv.n_pages) { page[x] = -1; set_status(g.status, SISO_ERR_INVALID_ARG); }
                    }
                    first[x] = wanted && blk % box_blocks == 0;
                }
#pragma unroll
                for (int x = 0; x < HALVES; ++x) {
                    there |= (__ballot_sync(0xFFFFFFFFu, page[x] >= 0) & 0xFFFFu) << (16 * x);
                    boxes += __popc(__ballot_sync(0xFFFFFFFFu, first[x]));
                }
                wait_bar(&ring.empty[stage], phase ^ 1u, gave_up, g.status);
                if (*gave_up) break;
                uint64_t *bar = &ring.full[stage];
                if (lane == 0) {
                    ring.blocks[stage] = there;
                    mbar_arrive_expect_tx(bar, boxes * (g.box * RB));
                }
                __syncwarp();
#pragma unroll
                for (int x = 0; x < HALVES; ++x) {
                    const int blk = x * 16 + (lane & 15);
                    if (first[x]) {
                        const uint32_t dst = smem_u32(smem + stage * S::STAGE) + is_v * (TK * RB) + blk * 8 * LINE;
                        // a page outside the pool is asked for at a place beyond the tensor's end, which reads as zeros
                        const int p = page[x] < 0 ? static_cast<int>(g.kv.n_pages) : page[x];
#pragma unroll
                        for (int half = 0; half < RB / LINE; ++half)
                            load_box(dst + half * (TK * 128), map, half * 64, cur.head, tok[x], p, g.a.layer, bar);
                    }
                    if constexpr (EIGHT) {                   // 8 exponents of a page lie side by side
                        const uint32_t dst = smem_u32(meta) + stage * S::META + is_v * TK + blk * 8;
                        const long long e = page[x] < 0 ? 0 : (static_cast<long long>(page[x]) * g.kv.n_kv_heads + cur.head) * g.kv.page_size + tok[x];
                        asm volatile("cp.async.ca.shared.global [%0], [%1], 8, %2;" ::"r"(dst), "l"(exps + e), "r"(page[x] < 0 ? 0 : 8) : "memory");
                    }
                }
                if constexpr (EIGHT) asm volatile("cp.async.mbarrier.arrive.noinc.shared.b64 [%0];" ::"r"(smem_u32(bar)) : "memory");
            }
            if (++stage == STAGES) { stage = 0; phase ^= 1u; }
        } while (cur.step(g));
        if constexpr (EIGHT) asm volatile("cp.async.wait_all;" ::: "memory");
        let_copies_land(gave_up);
        return;
    }

    asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(S::CONSUMER_REGS));
    // ---- consumers: this warp's 8 NT rows over its group's keys.  A lane has keys (and d) r0 and r0 + 8 of a tile of 16, rows 2 c
    // and 2 c + 1 of a tile of 8; as a query's carrier it has row r0.
    const int kg = warp / WM, wm = warp % WM;
    const int c = lane & 3, r0 = lane >> 2;
    const bool causal = (g.a.flags & SISO_ATTN_CAUSAL) != 0u;
    // the row that this lane points ldmatrix to: bf16: keys 0-7 of two chunks of 8 d, then keys 8-15; 8 bits: keys 0-7, then 8-15
    // of a chunk of 16 d, then the next chunk
    const uint32_t v_lane = EIGHT ? chunk_at<RB, TK>(key_of<RB>(lane & 7) + (lane & 8), lane >> 4)
                                  : chunk_at<RB, TK>(key_of<RB>(lane & 7) + ((lane & 16) >> 1), (lane >> 3) & 1);
    uint32_t q[NT][D / 16][2];
    float o[NT][DT][4], m[NT][2], l[NT][2], row_scale[NT][2];
    int pos[NT][2], e_top = 0;

    // the queries of an item: 8 values of each of D / 32 pieces per lane.  bf16 cache: a lane's 16 bytes of a key hold 8 values;
    // 8-bit: 16 values, two pieces of 8
    auto fetch_q = [&]() {
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            const int row = cur.rt * MR + (wm * NT + t) * 8 + r0;
            const bool real = row < cur.n_q * g.group;
            const int i = static_cast<int>(g.by_group.div(static_cast<uint32_t>(real ? row : 0)));
            const int head = cur.head * g.group + (real ? row - i * g.group : 0);
            const __nv_bfloat16 *src = static_cast<const __nv_bfloat16 *>(g.a.d_q) + static_cast<long long>(cur.q0 + i) * g.a.q_stride_token + head * g.a.q_stride_head;
#pragma unroll
            for (int x = 0; x < D / 32; ++x) {
                const int d = EIGHT ? ((x / 2) * 4 + c) * 16 + (x & 1) * 8 : (x * 4 + c) * 8;
                const uint4 w = real ? *reinterpret_cast<const uint4 *>(src + d) : make_uint4(0u, 0u, 0u, 0u);
                q[t][2 * x][0] = w.x; q[t][2 * x][1] = w.y; q[t][2 * x + 1][0] = w.z; q[t][2 * x + 1][1] = w.w;
            }
        }
    };
    auto begin_item = [&]() {
        e_top = 0;
#pragma unroll
        for (int t = 0; t < NT; ++t) {
#pragma unroll
            for (int d = 0; d < DT; ++d) { o[t][d][0] = 0.f; o[t][d][1] = 0.f; o[t][d][2] = 0.f; o[t][d][3] = 0.f; }
            float back = 1.f;
            if constexpr (EIGHT) {
                uint32_t top = 0u;
#pragma unroll
                for (int x = 0; x < D / 16; ++x)
#pragma unroll
                    for (int i = 0; i < 2; ++i) top = max(top, max((q[t][x][i] << 16) & 0x7FFF0000u, q[t][x][i] & 0x7FFF0000u));
                top = max(top, __shfl_xor_sync(0xFFFFFFFFu, top, 1));
                top = max(top, __shfl_xor_sync(0xFFFFFFFFu, top, 2));
                const int ex = min(max(static_cast<int>(top >> 23), 16), 254);     // the row's largest value becomes 2^14 .. 2^15
                const float up = __uint_as_float(static_cast<uint32_t>(268 - ex) << 23);
                back = __uint_as_float(static_cast<uint32_t>(max(ex - 14, 1)) << 23);
#pragma unroll
                for (int x = 0; x < D / 16; ++x)
#pragma unroll
                    for (int i = 0; i < 2; ++i)
                        q[t][x][i] = pack(__uint_as_float(q[t][x][i] << 16) * up, __uint_as_float(q[t][x][i] & 0xFFFF0000u) * up, true);
            }
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int row = cur.rt * MR + (wm * NT + t) * 8 + 2 * c + h;
                pos[t][h] = row < cur.n_q * g.group ? position(cur.len, cur.n_q, static_cast<int>(g.by_group.div(static_cast<uint32_t>(row)))) : cur.s.last_pos;
                m[t][h] = -INFINITY;
                l[t][h] = 0.f;
                row_scale[t][h] = g.scale_log2 * __shfl_sync(0xFFFFFFFFu, back, (2 * c + h) * 4);
            }
        }
    };
    fetch_q();
    begin_item();
    int t_begin = cur.tile;                                  // tile at which the current part of the item began
    int stage = 0;
    uint32_t phase = 0;
    for (bool more = true; more;) {
        wait_bar(&ring.full[stage], phase, gave_up, g.status);
        uint8_t *tile = smem + stage * S::STAGE;
        const int k_first = stage * S::STAGE + chunk_at<RB, TK>(key_of<RB>(r0), c);
        const uint32_t v_first = smem_u32(tile) + TK * RB + v_lane;
        const uint8_t *mt = meta + stage * S::META;
        const int j0 = (cur.s.tile0 + cur.tile) * TK;
        const uint32_t blocks = ring.blocks[stage];
        const bool cut = j0 + TK > cur.s.hi || blocks != ALL || (causal && j0 + TK - 1 > cur.s.first_pos) ||
                         (g.a.window > 0 && j0 <= cur.s.last_pos - g.a.window);
        const int lo = cut ? cur.lo(g) : 0;
        if (cut && (j0 + TK > cur.s.hi || j0 < lo)) {    // values beyond the end or before every window may be anything: zeros, or 0 times NaN would reach the sums
            for (int x = wm * 32 + lane; x < NK * CH; x += 32 * WM) {
                const int row = kg * NK + x / CH;
                if (j0 + row >= lo && j0 + row < cur.s.hi) continue;
                *reinterpret_cast<uint4 *>(tile + TK * RB + chunk_at<RB, TK>(row, x % CH)) = make_uint4(0u, 0u, 0u, 0u);
                if (EIGHT && x % CH == 0) meta[stage * S::META + TK + row] = 0;
            }
            asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
            if constexpr (WM == 1) __syncwarp();
            else asm volatile("bar.sync %0, %1;" ::"r"(kg + 2), "n"(32 * WM) : "memory");
        }
#pragma unroll 1
        for (int n0 = kg * NK; n0 < (kg + 1) * NK; n0 += SUB) {
            float s[KT][NT][4];
#pragma unroll
            for (int i = 0; i < KT; ++i)
#pragma unroll
                for (int t = 0; t < NT; ++t) { s[i][t][0] = 0.f; s[i][t][1] = 0.f; s[i][t][2] = 0.f; s[i][t][3] = 0.f; }
#pragma unroll
            for (int a = 0; a < RB / 64; ++a) {
#pragma unroll
                for (int i = 0; i < KT; ++i) {
                    // chunk 4 a + c of keys row and row + 8: tiles start at multiples of 1024, so a only flips bits
                    const int at = ((k_first + (n0 + 16 * i) * LINE) ^ ((a & 1) << 6)) + (a >> 1) * (TK * 128);
                    const uint4 w0 = *reinterpret_cast<const uint4 *>(smem + at);
                    const uint4 w1 = *reinterpret_cast<const uint4 *>(smem + at + 8 * LINE);
                    const uint32_t x0[4] = {w0.x, w0.y, w0.z, w0.w}, x1[4] = {w1.x, w1.y, w1.z, w1.w};
                    if constexpr (!EIGHT) {
#pragma unroll
                        for (int x = 0; x < 2; ++x) {
                            const uint32_t f[4] = {x0[2 * x], x1[2 * x], x0[2 * x + 1], x1[2 * x + 1]};
#pragma unroll
                            for (int t = 0; t < NT; ++t) mma<false>(s[i][t], f, q[t][2 * a + x]);
                        }
                    } else {
#pragma unroll
                        for (int x = 0; x < 4; ++x) {
                            uint32_t f[4];
                            widen<KIND>(x0[x], f[0], f[2]);
                            widen<KIND>(x1[x], f[1], f[3]);
#pragma unroll
                            for (int t = 0; t < NT; ++t) mma<true>(s[i][t], f, q[t][4 * a + x]);
                        }
                    }
                }
            }
            // scores in powers of two; element 2 e + h of a tile: key 8 e + key_of(r0) of the 16, row 2 c + h
            uint32_t ev[KT][2];
#pragma unroll
            for (int i = 0; i < KT; ++i)
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    float f = 1.f;
                    if constexpr (EIGHT) {       // (byte 0: nothing above 2^-118, counts as zero; byte 255: infinity, then NaN)
                        const int n = n0 + 16 * i + 8 * e + key_of<RB>(r0);
                        f = __uint_as_float(static_cast<uint32_t>(mt[n]) << 23);
                        ev[i][e] = mt[TK + n];
                    }
#pragma unroll
                    for (int t = 0; t < NT; ++t)
#pragma unroll
                        for (int h = 0; h < 2; ++h) s[i][t][2 * e + h] *= EIGHT ? f * row_scale[t][h] : row_scale[t][h];
                }
            if (cut) {       // keys that are not seen, or not there, are left out by selection: they may hold anything
#pragma unroll
                for (int i = 0; i < KT; ++i)
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        const int n = n0 + 16 * i + 8 * e, j = j0 + n + key_of<RB>(r0);
                        const bool in = ((blocks >> (n / 8)) & 1u) && j < cur.s.hi;
                        if (EIGHT && !in) ev[i][e] = 0u;
#pragma unroll
                        for (int t = 0; t < NT; ++t)
#pragma unroll
                            for (int h = 0; h < 2; ++h)
                                if (!in || (causal && j > pos[t][h]) || (g.a.window > 0 && j <= pos[t][h] - g.a.window)) s[i][t][2 * e + h] = -INFINITY;
                    }
            }
            float shift[NT][2], corr[NT][2];
            bool moved = false;
#pragma unroll
            for (int t = 0; t < NT; ++t)
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    float top = fmaxf(s[0][t][h], s[0][t][2 + h]);
#pragma unroll
                    for (int i = 1; i < KT; ++i) top = fmaxf(top, fmaxf(s[i][t][h], s[i][t][2 + h]));
                    top = fmaxf(top, __shfl_xor_sync(0xFFFFFFFFu, top, 4));
                    top = fmaxf(top, __shfl_xor_sync(0xFFFFFFFFu, top, 8));
                    top = fmaxf(top, __shfl_xor_sync(0xFFFFFFFFu, top, 16));
                    const float m2 = fmaxf(m[t][h], top);
                    corr[t][h] = m[t][h] == m2 ? 1.f : ex2(m[t][h] - m2);
                    moved = moved || m[t][h] != m2;
                    m[t][h] = m2;
                    shift[t][h] = m2 == -INFINITY ? 0.f : m2;
                    l[t][h] *= corr[t][h];
                }
            if constexpr (EIGHT) {
                uint32_t e_max = max(ev[0][0], ev[0][1]);
#pragma unroll
                for (int i = 1; i < KT; ++i) e_max = max(e_max, max(ev[i][0], ev[i][1]));
                e_max = __reduce_max_sync(0xFFFFFFFFu, e_max);
                if (static_cast<int>(e_max) > e_top) {
                    const float down = ex2(static_cast<float>(e_top - static_cast<int>(e_max)));
#pragma unroll
                    for (int t = 0; t < NT; ++t) { corr[t][0] *= down; corr[t][1] *= down; }
                    moved = true;
                    e_top = static_cast<int>(e_max);
                }
            }
            if (__any_sync(0xFFFFFFFFu, moved)) {
#pragma unroll
                for (int t = 0; t < NT; ++t)
#pragma unroll
                    for (int d = 0; d < DT; ++d) { o[t][d][0] *= corr[t][0]; o[t][d][1] *= corr[t][1]; o[t][d][2] *= corr[t][0]; o[t][d][3] *= corr[t][1]; }
            }
#pragma unroll
            for (int i = 0; i < KT; ++i) {
                uint32_t p[NT][2];
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    float rel = 1.f;                      // 2^(value exponent - largest so far)
                    if constexpr (EIGHT) rel = __uint_as_float(static_cast<uint32_t>(max(127 + UP<KIND> - e_top + static_cast<int>(ev[i][e]), 0)) << 23);
#pragma unroll
                    for (int t = 0; t < NT; ++t) {
                        const float p0 = ex2(s[i][t][2 * e] - shift[t][0]), p1 = ex2(s[i][t][2 * e + 1] - shift[t][1]);
                        l[t][0] += p0;
                        l[t][1] += p1;
                        p[t][e] = transposed(EIGHT ? pack(p0 * rel, p1 * rel, false) : pack(p0, p1, false));
                    }
                }
                const uint32_t v_at = v_first + (n0 + 16 * i) * LINE;
                if constexpr (!EIGHT) {
#pragma unroll
                    for (int d = 0; d < DT; ++d) {        // keys 0-7 and 8-15 of two chunks of 8 d
                        uint32_t f[4];
                        load_v((v_at ^ (((2 * d) & 7) << 4)) + (d >> 2) * (TK * 128), f);
#pragma unroll
                        for (int t = 0; t < NT; ++t) mma<false>(o[t][d], f, p[t]);
                    }
                } else {
#pragma unroll
                    for (int d = 0; d < DT; d += 2) {     // keys 0-7 and 8-15 of two chunks of 16 d
                        uint32_t v[4], f[4];
                        load_v(v_at ^ (d << 4), v);
#pragma unroll
                        for (int x = 0; x < 2; ++x) {     // rows 0-7 of the product: even d, rows 8-15: odd d
                            widen_values<KIND>(v[2 * x], f[0], f[1]);
                            widen_values<KIND>(v[2 * x + 1], f[2], f[3]);
#pragma unroll
                            for (int t = 0; t < NT; ++t) mma<false>(o[t][d + x], f, p[t]);
                        }
                    }
                }
            }
        }
        __syncwarp();
        if (lane == 0) mbar_arrive(&ring.empty[stage]);
        if (++stage == STAGES) { stage = 0; phase ^= 1u; }
        if (__any_sync(0xFFFFFFFFu, cur.tiles_here() > 1)) {   // (uniform, visibly: the barriers further down cost no registers then)
            cur.step(g);
            continue;
        }

        // ---- end of the item, or of this CTA's part of it.  The next one's queries are on their way meanwhile
        const int t_end = cur.tile + 1;                       // tiles [t_begin, t_end) of the item were done here
        const int done_b = cur.b, done_head = cur.head, done_rt = cur.rt, done_q0 = cur.q0, done_rows = cur.n_q * g.group, done_tiles = cur.s.tiles;
        const bool whole = t_begin == 0 && t_end == done_tiles, began_before = t_begin > 0;
        const int done_left = cur.left;
        more = cur.step(g);
        t_begin = 0;
        if (more) fetch_q();
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                l[t][h] += __shfl_xor_sync(0xFFFFFFFFu, l[t][h], 4);
                l[t][h] += __shfl_xor_sync(0xFFFFFFFFu, l[t][h], 8);
                l[t][h] += __shfl_xor_sync(0xFFFFFFFFu, l[t][h], 16);
            }
        if constexpr (EIGHT) {
            const float back = kv_scale(static_cast<uint32_t>(e_top));
#pragma unroll
            for (int t = 0; t < NT; ++t)
#pragma unroll
                for (int d = 0; d < DT; ++d)
#pragma unroll
                    for (int x = 0; x < 4; ++x) o[t][d][x] = o[t][d][x] * BACK<KIND> * back;
        }
#pragma unroll 1
        for (int half = WK / 2; half >= 1; half >>= 1) { // join the groups' results, halving their number each time
            float4 *mo = reinterpret_cast<float4 *>(merge_o) + ((kg % half) * WM + wm) * (NT * DT * 32) + lane;
            float *ml = merge_ml + ((kg % half) * WM + wm) * (16 * NT) + 4 * c;
            if (kg >= half && kg < 2 * half) {
#pragma unroll
                for (int t = 0; t < NT; ++t) {
#pragma unroll
                    for (int d = 0; d < DT; ++d) mo[(t * DT + d) * 32] = make_float4(o[t][d][0], o[t][d][1], o[t][d][2], o[t][d][3]);
                    if (r0 == 0) { ml[16 * t] = m[t][0]; ml[16 * t + 1] = l[t][0]; ml[16 * t + 2] = m[t][1]; ml[16 * t + 3] = l[t][1]; }
                }
            }
            asm volatile("bar.sync 1, %0;" ::"n"(32 * WARPS) : "memory");
            if (kg < half) {
#pragma unroll
                for (int t = 0; t < NT; ++t) {
                    float mine[2], theirs[2];
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        const float m1 = ml[16 * t + 2 * h], l1 = ml[16 * t + 2 * h + 1], m2 = fmaxf(m[t][h], m1);
                        mine[h] = m[t][h] == -INFINITY ? 0.f : ex2(m[t][h] - m2);
                        theirs[h] = m1 == -INFINITY ? 0.f : ex2(m1 - m2);
                        l[t][h] = l[t][h] * mine[h] + l1 * theirs[h];
                        m[t][h] = m2;
                    }
#pragma unroll
                    for (int d = 0; d < DT; ++d) {
                        const float4 y = mo[(t * DT + d) * 32];
                        o[t][d][0] = o[t][d][0] * mine[0] + y.x * theirs[0];
                        o[t][d][1] = o[t][d][1] * mine[1] + y.y * theirs[1];
                        o[t][d][2] = o[t][d][2] * mine[0] + y.z * theirs[0];
                        o[t][d][3] = o[t][d][3] * mine[1] + y.w * theirs[1];
                    }
                }
            }
            asm volatile("bar.sync 1, %0;" ::"n"(32 * WARPS) : "memory");
        }
        if (kg == 0) {
#pragma unroll
            for (int t = 0; t < NT; ++t)
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const int in_tile = (wm * NT + t) * 8 + 2 * c + h, row = done_rt * MR + in_tile;
                    if (row >= done_rows) continue;
                    if (whole) {
                        const int i = static_cast<int>(g.by_group.div(static_cast<uint32_t>(row)));
                        const int head = done_head * g.group + row - i * g.group;
                        const float inv = inverse_of(l[t][h]);
                        __nv_bfloat16 *dst = static_cast<__nv_bfloat16 *>(g.a.d_out) + static_cast<long long>(done_q0 + i) * g.a.out_stride_token + head * g.a.out_stride_head;
#pragma unroll
                        for (int d = 0; d < DT; ++d) {
                            if constexpr (!EIGHT) {
                                dst[16 * d + r0] = __float2bfloat16_rn(o[t][d][h] * inv);
                                dst[16 * d + 8 + r0] = __float2bfloat16_rn(o[t][d][2 + h] * inv);
                            } else {
                                *reinterpret_cast<uint32_t *>(dst + 16 * d + 2 * r0) = pack(o[t][d][h] * inv, o[t][d][2 + h] * inv, false);
                            }
                        }
                        if (g.a.d_lse && r0 == 0)
                            g.a.d_lse[static_cast<long long>(done_q0 + i) * g.a.n_heads + head] = lse_of(m[t][h], l[t][h]);
                    } else {
                        const long long place = part_place(blockIdx.x, began_before) * MR + in_tile;
                        float *dst = g.part_o + place * D;
#pragma unroll
                        for (int d = 0; d < DT; ++d) {
                            if constexpr (!EIGHT) { dst[16 * d + r0] = o[t][d][h]; dst[16 * d + 8 + r0] = o[t][d][2 + h]; }
                            else *reinterpret_cast<float2 *>(dst + 16 * d + 2 * r0) = make_float2(o[t][d][h], o[t][d][2 + h]);
                        }
                        if (r0 == 0) *reinterpret_cast<float2 *>(g.part_ml + place * 2) = make_float2(m[t][h], l[t][h]);
                    }
                }
        }
        if (!whole && !began_before && threadIdx.x == 0) g.records[blockIdx.x] = record_of<2>(run, done_left, done_b, done_head, done_rt, done_tiles, t_end - 1);
        if (more) begin_item();
    }
    let_copies_land(gave_up);            // (the producers may have gone before the last wait gave up)
}

// Lets a wait of these kernels run out: a barrier that expects one arrival, and none comes
__global__ void __launch_bounds__(64) wait_timeout_kernel(int *status) {
    __shared__ uint64_t bar;
    __shared__ int abandoned;
    if (threadIdx.x == 0) {
        abandoned = 0;
        mbar_init(&bar, 1);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    __syncthreads();
    for (int i = 0; i < 3; ++i) wait_bar(&bar, 0, &abandoned, status);       // the first takes the time, the others find it given up
    let_copies_land(&abandoned);
}

// ---- joining the parts ------------------------------------------------------------------------------------------------
// CTA (x, y): the item that is recorded at CTA x, ROWS of its rows.  The parts lie at place 1 of CTA x and place 0 of the next
// ones.  8 / ROWS warps share a row: 32 lanes over d, the warps over the parts; sums are taken in the same order every time.
template <int MR, int D>
__global__ void __launch_bounds__(256)
join_kernel(const __grid_constant__ Args g) {
    constexpr int ROWS = MR / 8 < 8 ? MR / 8 : 8, WPR = 8 / ROWS;          // rows of a CTA at a time, warps of a row
    constexpr int N = D / 32;
    __shared__ float so[8][D], sml[8][2];
    wait_for_earlier();
    const Record rec = g.records[blockIdx.x];
    if (!rec.valid) return;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    int q0;
    const int n_q = seq_queries(g, rec.b, q0);
    {
        const int base = blockIdx.y * ROWS;
        const int in_tile = base + warp / WPR, part0 = warp % WPR;
        const int row = rec.row_tile * MR + in_tile;
        const bool real = row < n_q * g.group;
        float m = -INFINITY, l = 0.f, o[N];
#pragma unroll
        for (int x = 0; x < N; ++x) o[x] = 0.f;
        if (real) {
            constexpr int F = 8;                                            // parts in flight
            for (int s = part0; s < rec.n_parts; s += WPR * F) {
                float2 ml[F];
                float y[F][N];
#pragma unroll
                for (int f = 0; f < F; ++f) {
                    const int part = s + f * WPR;
                    ml[f] = make_float2(-INFINITY, 0.f);
                    if (part < rec.n_parts) {
                        const long long place = part_place(static_cast<int>(blockIdx.x) + part, part > 0) * MR + in_tile;
                        ml[f] = *reinterpret_cast<const float2 *>(g.part_ml + place * 2);
#pragma unroll
                        for (int x = 0; x < N; ++x) y[f][x] = g.part_o[place * D + x * 32 + lane];
                    }
                }
#pragma unroll
                for (int f = 0; f < F; ++f) {
                    if (ml[f].y == 0.f) continue;                            // nothing seen there (a NaN is no zero)
                    const float m2 = fmaxf(m, ml[f].x), a = m == -INFINITY ? 0.f : ex2(m - m2), b = ex2(ml[f].x - m2);
                    l = l * a + ml[f].y * b;
                    m = m2;
#pragma unroll
                    for (int x = 0; x < N; ++x) o[x] = o[x] * a + y[f][x] * b;
                }
            }
        }
        if constexpr (WPR > 1) {
            __syncthreads();
#pragma unroll
            for (int x = 0; x < N; ++x) so[warp][x * 32 + lane] = o[x];
            if (lane == 0) { sml[warp][0] = m; sml[warp][1] = l; }
            __syncthreads();
            if (part0 != 0) return;
#pragma unroll
            for (int w = 1; w < WPR; ++w) {
                const float m1 = sml[warp + w][0], l1 = sml[warp + w][1];
                if (l1 == 0.f) continue;
                const float m2 = fmaxf(m, m1), a = m == -INFINITY ? 0.f : ex2(m - m2), b = ex2(m1 - m2);
                l = l * a + l1 * b;
                m = m2;
#pragma unroll
                for (int x = 0; x < N; ++x) o[x] = o[x] * a + so[warp + w][x * 32 + lane] * b;
            }
        }
        if (!real) return;
        const int i = static_cast<int>(g.by_group.div(static_cast<uint32_t>(row))), head = rec.head * g.group + row - i * g.group;
        const float inv = inverse_of(l);
        __nv_bfloat16 *dst = static_cast<__nv_bfloat16 *>(g.a.d_out) + static_cast<long long>(q0 + i) * g.a.out_stride_token + head * g.a.out_stride_head;
#pragma unroll
        for (int x = 0; x < N; ++x) dst[x * 32 + lane] = __float2bfloat16_rn(o[x] * inv);
        if (g.a.d_lse && lane == 0)
            g.a.d_lse[static_cast<long long>(q0 + i) * g.a.n_heads + head] = lse_of(m, l);
    }
}

template <int MR, int D> static siso_status_t run_join(const Args &g, cudaStream_t s) {
    return launch_early(join_kernel<MR, D>, dim3(static_cast<unsigned>(g.grid), MR >= 64 ? MR / 8 : 8), 256, 0, s, g);
}
siso_status_t launch_join(const Args &g, int mr, int dim, cudaStream_t s) {
    switch (mr) {
        case 8: return dim == 128 ? run_join<8, 128>(g, s) : run_join<8, 64>(g, s);
        case 16: return dim == 128 ? run_join<16, 128>(g, s) : run_join<16, 64>(g, s);
        case 32: return dim == 128 ? run_join<32, 128>(g, s) : run_join<32, 64>(g, s);
        default: return dim == 128 ? run_join<TC_ROWS, 128>(g, s) : run_join<TC_ROWS, 64>(g, s);
    }
}

siso_status_t launch_wait_timeout(Kv *h, cudaStream_t s) {
    wait_timeout_kernel<<<1, 64, 0, s>>>(h->status);
    SISO_CUDA(cudaGetLastError());
    return SISO_OK;
}

siso_status_t kv_scratch(Kv *h, size_t bytes, cudaStream_t s) {
    if (bytes <= h->ws_bytes) return SISO_OK;
    if (h->ws) {                       // kernels of earlier calls may still use it, on any stream
        SISO_CUDA(cudaDeviceSynchronize());
        h->cfg.allocator.free(h->ws, h->cfg.allocator.ctx);
        h->ws = nullptr;
        h->ws_bytes = 0;
    }
    h->ws = h->cfg.allocator.alloc(bytes, s, h->cfg.allocator.ctx);
    if (!h->ws) return SISO_ERR_OOM;
    h->ws_bytes = bytes;
    return SISO_OK;
}

template <int KIND, int D, int WM, int NT> static siso_status_t run_few(Kv *h, Args &g, cudaStream_t s) {
    using S = Shape<KIND, D, WM, NT>;
    constexpr uint32_t bit = 1u << (NT == 1 ? 0 : WM);        // a handle has one type and head_dim
    if (!(h->attr_set & bit)) {
        SISO_CUDA(cudaFuncSetAttribute(attention_few_rows_kernel<KIND, D, WM, NT>, cudaFuncAttributeMaxDynamicSharedMemorySize, S::SMEM));
        h->attr_set |= bit;
    }
    attention_few_rows_kernel<KIND, D, WM, NT><<<g.grid, S::THREADS, S::SMEM, s>>>(g, h->map_k, h->map_v);
    SISO_CUDA(cudaGetLastError());
    return launch_join(g, S::MR, D, s);
}
template <int KIND, int D> static siso_status_t run_few_rows(Kv *h, Args &g, int mr, cudaStream_t s) {
    return mr == 8 ? run_few<KIND, D, 1, 1>(h, g, s) : mr == 16 ? run_few<KIND, D, 1, 2>(h, g, s) : run_few<KIND, D, 2, 2>(h, g, s);
}
template <int KIND> static siso_status_t run_few_dim(Kv *h, Args &g, int dim, int mr, cudaStream_t s) {
    return dim == 128 ? run_few_rows<KIND, 128>(h, g, mr, s) : run_few_rows<KIND, 64>(h, g, mr, s);
}

}  // namespace kva

siso_status_t launch_kv_attention(Kv *h, const siso_attention_t *a, cudaStream_t s) {
    using namespace kva;
    Args g;
    g.kv = kv_view(h, a->layer);
    g.a = *a;
    g.group = a->n_heads / h->cfg.n_kv_heads;
    g.by_page.set(static_cast<uint32_t>(h->cfg.page_size));
    g.by_group.set(static_cast<uint32_t>(g.group));
    g.scale_log2 = a->scale * 1.4426950408889634f;
    g.status = h->status;
    g.box = h->box;
    g.grid = h->sm_count;
    const int dim = h->cfg.head_dim;
    const long long rows = static_cast<long long>(a->max_q) * g.group;      // rows per key/value head of the longest chunk
    const int mr = rows <= 8 ? 8 : rows <= 16 ? 16 : rows <= 32 ? 32 : TC_ROWS;
    const size_t records = pad256(sizeof(Record) * g.grid), ml = pad256(sizeof(float) * 2 * g.grid * mr * 2);
    // sized for the widest kernel, so that a handle that has served one call serves every other without a new block
    const size_t most = records + pad256(sizeof(float) * 2 * g.grid * TC_ROWS * 2) + sizeof(float) * 2 * g.grid * TC_ROWS * static_cast<size_t>(dim);
    SISO_TRY(kv_scratch(h, most, s));
    char *ws = static_cast<char *>(h->ws);
    g.records = reinterpret_cast<Record *>(ws);
    g.part_ml = reinterpret_cast<float *>(ws + records);
    g.part_o = reinterpret_cast<float *>(ws + records + ml);
    if (mr == TC_ROWS) return launch_many_rows(h, g, s);
    switch (h->cfg.dtype) {
        case SISO_BF16: return run_few_dim<SISO_BF16>(h, g, dim, mr, s);
        case SISO_E4M3: return run_few_dim<SISO_E4M3>(h, g, dim, mr, s);
        default: return run_few_dim<SISO_I8>(h, g, dim, mr, s);
    }
}

}  // namespace siso
