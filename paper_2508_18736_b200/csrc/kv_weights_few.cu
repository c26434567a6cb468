// The weight that attention gives to each cached token, for few query rows per kv head (a step's tokens, short runs of drafted ones): up to 32.
// The formulas are in kv_weights.cu.
//
// Every key meets few multiplications, so the call is bound by HBM and the point is to spend few instructions on a byte.  As in the attention over few rows four
// producer warps fill a ring of units by TMA, one box per run of tokens in one page, and groups of warps consume it in turn; units are dealt to one CTA per SM in equal
// runs.  A warp owns 32 of a unit's keys and shares nothing with the others: scores^T = K Q^T by mma.sync m16n8k16 (rows fill the 8 columns; tcgen05's
// 128 lanes or columns would be mostly empty, and 8-bit codes would have to go through shared memory once more), exponentials, the sum over a key's rows by
// two shuffles.  What else belongs to a key (its exponent, its weight so far, where that lies) comes with the unit.  8-bit codes become fp16 in registers, exactly; queries
// are brought to fp16 with a factor per row, exactly but for elements below 2^-31 of their row's largest.
// Measured (8 kv heads x 128, 4 rows each): one token of each of 64 sequences over 201 to 8190 tokens, e4m3, 64 us (4.5 TB/s; consumers' instructions, most of them for
// the codes, and HBM are both a little over half busy); 64 x 4096 tokens of bf16 90 us (6.2 TB/s).
#include <cuda_fp16.h>

#include "kv_attention.cuh"

namespace siso {
namespace kvw {
namespace few {

using umma2::mbar_arrive;
using umma2::mbar_arrive_expect_tx;
using umma2::mbar_init;
using umma2::smem_u32;
using kva::FastDiv;
using kva::wait_bar;

constexpr int PRODUCERS = 4;             // warps that fill the ring; each has its own stages

struct Args {
    KvView kv;
    siso_weights_t a;
    const int32_t *fresh;
    FastDiv by_page, by_group;
    int group, box;
    float scale_log2;
    int *status;
};

template <int KIND, int D, int NT> struct Shape {
    static constexpr bool EIGHT = KIND != SISO_BF16;
    static constexpr int WARPS = NT > 1 ? 8 : EIGHT ? 16 : 12;      // consumers
    static constexpr int THREADS = 32 * (WARPS + PRODUCERS);
    static constexpr int T = EIGHT ? 256 : 128;             // keys of a unit
    static constexpr int NK = 32, GW = T / NK, GROUPS = WARPS / GW;      // keys of a warp, warps of a unit; groups of them take units in turn
    static constexpr int RB = D * (EIGHT ? 1 : 2), STAGE = T * RB;
    static constexpr int META = T * 4 + T / 8 * 8 + (EIGHT ? T : 0);      // weights so far, places of the blocks of 8, exponents
    static constexpr int FIT = (232448 - 1024 - 2048) / (STAGE + META);
    // a stage is always read by the same group: one that is ahead of the others must not ask for a round of a stage before the round before has come
    static constexpr int STAGES = (FIT > 12 ? 12 : FIT) / GROUPS * GROUPS;
    static constexpr int SMEM = STAGES * (STAGE + META) + 1024;
    static constexpr int AT_LAUNCH = WARPS == 8 ? 168 : WARPS == 12 ? 128 : 96, PRODUCER_REGS = WARPS == 8 ? 40 : WARPS == 12 ? 56 : 64,
                         CONSUMER_REGS = WARPS == 8 ? 232 : WARPS == 12 ? 152 : 104;
    static_assert(WARPS * CONSUMER_REGS + PRODUCERS * PRODUCER_REGS == (WARPS + PRODUCERS) * AT_LAUNCH, "registers at launch");
};
template <int STAGES> struct Ring {
    uint64_t full[STAGES], empty[STAGES];
    int gave_up;
};

__device__ __forceinline__ int seq_len(const Args &g, int b) {
    return static_cast<int>(min(static_cast<long long>(max(g.a.d_kv_len[b], 0)), static_cast<long long>(g.a.max_pages) * g.kv.page_size));
}
__device__ __forceinline__ int seq_queries(const Args &g, int b, int &q0) {
    const int n = static_cast<int>(g.a.n_tokens);
    q0 = min(max(g.a.d_cu_q[b], 0), n);
    return max(0, min(g.a.d_cu_q[b + 1], n) - q0);
}
// A unit of this CTA's run: tile of a kv head of a sequence
template <int T> struct Cursor {
    int b, head, tile, tiles, len, q0, n_q, n_old;              // n_old: tokens that have a weight already
    long long left;
    __device__ __forceinline__ void load(const Args &g) {
        n_q = seq_queries(g, b, q0);
        len = n_q > 0 ? seq_len(g, b) : 0;
        n_old = len - (g.fresh ? min(max(g.fresh[b], 0), len) : n_q);
        tiles = (len + T - 1) / T;
    }
    // to the first tile of the next kv head that has any; only called while units are left
    __device__ __forceinline__ void next_head(const Args &g) {
        tile = 0;
        if (++head == g.kv.n_kv_heads) {
            head = 0;
            do { ++b; load(g); } while (tiles == 0);
        }
    }
    __device__ __forceinline__ bool step(const Args &g) {
        if (--left <= 0) return false;
        if (++tile == tiles) next_head(g);
        return true;
    }
};
template <int T, int THREADS>
__device__ __forceinline__ bool locate(const Args &g, Cursor<T> &cur, unsigned long long *buf) {
    constexpr int W = THREADS / 32;
    unsigned long long mine = 0ull, upto = 0ull, all, total = 0ull;
    auto chunk = [&](int c0) {
        const int b = c0 + static_cast<int>(threadIdx.x);
        if (b >= g.a.n_seqs) return 0ull;
        int q0;
        return seq_queries(g, b, q0) > 0 ? static_cast<unsigned long long>((seq_len(g, b) + T - 1) / T) * g.kv.n_kv_heads : 0ull;
    };
    for (int c0 = 0; c0 < g.a.n_seqs; c0 += THREADS) {
        const unsigned long long x = chunk(c0), to = kva::cta_scan<THREADS>(x, all, buf);
        if (c0 == 0) { mine = x; upto = to; }
        total += all;
    }
    const unsigned long long n = gridDim.x, want = kva::quotient(total * blockIdx.x, n);
    cur.left = static_cast<long long>(kva::quotient(total * (blockIdx.x + 1), n) - want);
    if (cur.left <= 0) return false;
    unsigned long long base = 0ull;
    for (int c0 = 0;; c0 += THREADS) {
        if (c0 > 0) {
            mine = chunk(c0);
            upto = base + kva::cta_scan<THREADS>(mine, all, buf);
        }
        __syncthreads();
        if (threadIdx.x == 0) buf[W] = ~0ull;
        __syncthreads();
        if (want < upto && want >= upto - mine) { buf[W] = static_cast<unsigned long long>(c0 + threadIdx.x); buf[W + 1] = upto - mine; }
        __syncthreads();
        if (buf[W] != ~0ull) break;
        if (threadIdx.x == THREADS - 1) buf[0] = upto;
        __syncthreads();
        base = buf[0];
        __syncthreads();
    }
    cur.b = static_cast<int>(buf[W]);
    cur.load(g);
    const unsigned long long within = want - buf[W + 1];
    cur.head = static_cast<int>(kva::quotient(within, static_cast<unsigned long long>(cur.tiles)));
    cur.tile = static_cast<int>(within - static_cast<unsigned long long>(cur.head) * cur.tiles);
    return true;
}

// Which of 8 keys the n-th row of a product is (see the attention over few rows): the lanes of one 16-byte load lie in different halves of their lines
template <int RB> __device__ __forceinline__ int key_of(int n) { return RB == 64 ? n : ((n & 1) << 2) | (n >> 1); }
template <bool HALF> __device__ __forceinline__ void mma(float (&c)[4], const uint32_t (&a)[4], const uint32_t (&b)[2]) {
    if constexpr (HALF)
        asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                     : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b[0]), "r"(b[1]));
    else
        asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                     : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b[0]), "r"(b[1]));
}
// Codes as fp16: bytes 0, 1 and 2, 3 of a word
template <int KIND> __device__ __forceinline__ void widen(uint32_t w, uint32_t &lo, uint32_t &hi) {
    if constexpr (KIND == SISO_E4M3) {
        asm("{\n\t.reg .b16 l, h;\n\tmov.b32 {l, h}, %2;\n\tcvt.rn.f16x2.e4m3x2 %0, l;\n\tcvt.rn.f16x2.e4m3x2 %1, h;\n\t}" : "=r"(lo), "=r"(hi) : "r"(w));
    } else {
        w ^= 0x80808080u;                                   // c + 128; beside the byte 0x64 it is the fp16 number 1024 + c + 128
        const __half2 off = __halves2half2(__ushort_as_half(0x6480), __ushort_as_half(0x6480));
        const uint32_t a = __byte_perm(w, 0x64646464u, 0x4140), b = __byte_perm(w, 0x64646464u, 0x4342);
        const __half2 x = __hsub2(*reinterpret_cast<const __half2 *>(&a), off), y = __hsub2(*reinterpret_cast<const __half2 *>(&b), off);
        lo = *reinterpret_cast<const uint32_t *>(&x);
        hi = *reinterpret_cast<const uint32_t *>(&y);
    }
}

template <int KIND, int D, int NT>
__global__ void __launch_bounds__(Shape<KIND, D, NT>::THREADS, 1)
weights_few_rows_kernel(const __grid_constant__ Args g, const __grid_constant__ CUtensorMap map_k) {
    using S = Shape<KIND, D, NT>;
    constexpr bool EIGHT = S::EIGHT;
    constexpr int T = S::T, RB = S::RB, STAGES = S::STAGES, NK = S::NK, WARPS = S::WARPS, GW = S::GW, LINE = RB < 128 ? RB : 128, BLOCKS = T / 8, MR = 8 * NT;
    extern __shared__ uint8_t smem_raw[];
    __shared__ unsigned long long buf[S::THREADS / 32 + 3];
    __shared__ Ring<STAGES> ring;
    uint8_t *smem = smem_raw + ((1024u - (smem_u32(smem_raw) & 1023u)) & 1023u);      // (an offset: the loads stay shared loads)
    long long *places = reinterpret_cast<long long *>(smem + STAGES * S::STAGE);      // [STAGES][BLOCKS]: of a block's first key among the weights, or -1
    float *olds = reinterpret_cast<float *>(places + STAGES * BLOCKS);                // [STAGES][T]
    uint8_t *exps = reinterpret_cast<uint8_t *>(olds + STAGES * T);                   // [STAGES][T]

    wait_for_earlier();
    dependents_may_start();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    if (threadIdx.x == 0) {
        for (int i = 0; i < STAGES; ++i) { mbar_init(&ring.full[i], 33); mbar_init(&ring.empty[i], GW); }      // 33: the bytes, and the lanes' small things
        ring.gave_up = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    }
    __syncthreads();
    Cursor<T> cur;
    if (!locate<T, S::THREADS>(g, cur, buf)) return;
    volatile int *gave_up = &ring.gave_up;
    float *held = g.a.d_weights + static_cast<long long>(g.a.layer) * g.kv.n_pages * g.kv.n_kv_heads * g.kv.page_size;

    if (warp >= WARPS) {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(S::PRODUCER_REGS));
        // ---- producers: a lane owns a block of 8 keys of the unit (of T = 128: the first 16 lanes).  A stage is always filled by the same warp, so its
        // rounds come in order
        const int box_blocks = g.box / 8;
        const bool old = g.a.decay != 0.f;
        int stage = 0;
        uint32_t phase = 0;
        do {
            if (stage % PRODUCERS == warp - WARPS) {
                const int j = cur.tile * T + lane * 8, at = static_cast<int>(g.by_page.div(static_cast<uint32_t>(j))), tok = j - at * g.kv.page_size;
                const bool wanted = lane < BLOCKS && j < cur.len;
                int page = -1;
                if (wanted) {
                    page = g.a.d_pages[cur.b * g.a.pages_stride + at];
                    if (page < 0 || page >= g.kv.n_pages) { page = -1; set_status(g.status, SISO_ERR_INVALID_ARG); }
                }
                const bool first = page >= 0 && lane % box_blocks == 0;
                const uint32_t boxes = __popc(__ballot_sync(0xFFFFFFFFu, first));
                const long long small = (static_cast<long long>(page) * g.kv.n_kv_heads + cur.head) * g.kv.page_size + tok;
                wait_bar(&ring.empty[stage], phase ^ 1u, gave_up, g.status);
                if (*gave_up) break;
                uint64_t *bar = &ring.full[stage];
                if (lane < BLOCKS) places[stage * BLOCKS + lane] = page < 0 ? -1 : small;
                __syncwarp();
                if (lane == 0) mbar_arrive_expect_tx(bar, boxes * (g.box * RB));
                __syncwarp();
                if (first) {
                    const uint32_t dst = smem_u32(smem + stage * S::STAGE) + lane * 8 * LINE;
#pragma unroll
                    for (int half = 0; half < RB / LINE; ++half)
                        kva::load_box(dst + half * (T * 128), &map_k, half * 64, cur.head, tok, page, g.a.layer, bar);
                }
                if (page >= 0) {                             // 8 weights and exponents of a page lie side by side
                    if (old) {
                        const uint32_t dst = smem_u32(olds + stage * T + lane * 8);
                        asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(held + small) : "memory");
                        asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst + 16), "l"(held + small + 4) : "memory");
                    }
                    if constexpr (EIGHT)
                        asm volatile("cp.async.ca.shared.global [%0], [%1], 8;" ::"r"(smem_u32(exps + stage * T + lane * 8)), "l"(g.kv.k_exp + small) : "memory");
                }
                asm volatile("cp.async.mbarrier.arrive.noinc.shared.b64 [%0];" ::"r"(smem_u32(bar)) : "memory");
            }
            if (++stage == STAGES) { stage = 0; phase ^= 1u; }
        } while (cur.step(g));
        asm volatile("cp.async.wait_all;" ::: "memory");
        kva::let_copies_land(gave_up);
        return;
    }

    asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(S::CONSUMER_REGS));
    // ---- consumers.  A lane has keys r0 and r0 + 8 of a tile of 16, rows 2 c and 2 c + 1 of a tile of 8; as a query's carrier it has row r0
    const int c = lane & 3, r0 = lane >> 2;
    const bool causal = (g.a.flags & SISO_ATTN_CAUSAL) != 0u;
    struct Queries {
        uint32_t q[NT][D / 16][2];
        float lse[NT][2];
    } now, next;
    float scale[NT][2], shift[NT][2];
    int pos[NT][2];                     // the last key that a row gives anything; -1: none (its lse is -infinity, and its scores may be anything)
    // rows rt * MR .. of a kv head: 8 values of each of D / 32 pieces per lane (bf16 cache: a lane's 16 bytes of a key hold 8 values; 8-bit: 16 values, two pieces)
    auto fetch = [&](const Cursor<T> &at, int rt, Queries &x) {
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            {
                const int row = rt * MR + t * 8 + r0;
                const bool real = row < at.n_q * g.group;
                const int i = static_cast<int>(g.by_group.div(static_cast<uint32_t>(real ? row : 0))), head = at.head * g.group + (real ? row - i * g.group : 0);
                const __nv_bfloat16 *src = static_cast<const __nv_bfloat16 *>(g.a.d_q) + static_cast<long long>(at.q0 + i) * g.a.q_stride_token + head * g.a.q_stride_head;
#pragma unroll
                for (int p = 0; p < D / 32; ++p) {
                    const int d = EIGHT ? ((p / 2) * 4 + c) * 16 + (p & 1) * 8 : (p * 4 + c) * 8;
                    const uint4 w = real ? *reinterpret_cast<const uint4 *>(src + d) : make_uint4(0u, 0u, 0u, 0u);
                    x.q[t][2 * p][0] = w.x; x.q[t][2 * p][1] = w.y; x.q[t][2 * p + 1][0] = w.z; x.q[t][2 * p + 1][1] = w.w;
                }
            }
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int row = rt * MR + t * 8 + 2 * c + h, i = static_cast<int>(g.by_group.div(static_cast<uint32_t>(row)));
                x.lse[t][h] = row < at.n_q * g.group ? g.a.d_lse[static_cast<long long>(at.q0 + i) * g.a.n_heads + at.head * g.group + row - i * g.group] : -INFINITY;
            }
        }
    };
    auto take = [&](const Cursor<T> &at, int rt) {              // `now` as the products take it
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            float back = 1.f;
            if constexpr (EIGHT) {
                uint32_t top = 0u;
#pragma unroll
                for (int x = 0; x < D / 16; ++x)
#pragma unroll
                    for (int i = 0; i < 2; ++i) top = max(top, max((now.q[t][x][i] << 16) & 0x7FFF0000u, now.q[t][x][i] & 0x7FFF0000u));
                top = max(top, __shfl_xor_sync(0xFFFFFFFFu, top, 1));
                top = max(top, __shfl_xor_sync(0xFFFFFFFFu, top, 2));
                const int ex = min(max(static_cast<int>(top >> 23), 16), 254);     // the row's largest value becomes 2^14 .. 2^15
                const float up = __uint_as_float(static_cast<uint32_t>(268 - ex) << 23);
                back = __uint_as_float(static_cast<uint32_t>(max(ex - 14, 1)) << 23);
#pragma unroll
                for (int x = 0; x < D / 16; ++x)
#pragma unroll
                    for (int i = 0; i < 2; ++i)
                        now.q[t][x][i] = kva::pack(__uint_as_float(now.q[t][x][i] << 16) * up, __uint_as_float(now.q[t][x][i] & 0xFFFF0000u) * up, true);
            }
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int row = rt * MR + t * 8 + 2 * c + h;
                pos[t][h] = now.lse[t][h] == -INFINITY ? -1 : causal ? kva::position(at.len, at.n_q, static_cast<int>(g.by_group.div(static_cast<uint32_t>(row)))) : 0x7FFFFFFF;
                shift[t][h] = now.lse[t][h] == -INFINITY ? -INFINITY : now.lse[t][h] * -1.4426950408889634f;      // nothing seen, or no row: exponentials are zero
                scale[t][h] = g.scale_log2 * __shfl_sync(0xFFFFFFFFu, back, (2 * c + h) * 4);
            }
        }
    };
    int stage = warp / GW;
    uint32_t phase = 0;
    auto onward = [&]() {                                     // to this group's next unit
        for (int i = 0; i < S::GROUPS; ++i)
            if (!cur.step(g)) return false;
        stage += S::GROUPS;
        if (stage >= STAGES) { stage -= STAGES; phase ^= 1u; }
        return true;
    };
    static_assert(STAGES % S::GROUPS == 0 && STAGES > 0, "a stage is always read by the same group");
    bool more = true;
    for (int i = 0; i < warp / GW && more; ++i) more = cur.step(g);
    int b_now = -1, head_now = -1, b_next = cur.b, head_next = cur.head;      // whose queries `now` and `next` are
    if (more) fetch(cur, 0, next);
    while (more) {
        const int row_tiles = (cur.n_q * g.group + MR - 1) / MR;      // (one, unless max_q says less than there is)
        if (cur.b != b_now || cur.head != head_now) {
            if (cur.b != b_next || cur.head != head_next) fetch(cur, 0, next);
            now = next;
            take(cur, 0);
            b_now = cur.b;
            head_now = cur.head;
            Cursor<T> after = cur;                            // the next kv head's queries are on their way meanwhile
            after.left -= cur.tiles - cur.tile;
            if (after.left > 0) {
                after.next_head(g);
                fetch(after, 0, next);
                b_next = after.b;
                head_next = after.head;
            }
        }
        wait_bar(&ring.full[stage], phase, gave_up, g.status);
        const int j0 = cur.tile * T, n0 = warp % GW * NK;
        const int k_first = stage * S::STAGE + kva::chunk_at<RB, T>(key_of<RB>(r0), c) + n0 * LINE;
        float sum[2][2] = {{0.f, 0.f}, {0.f, 0.f}};           // of the keys r0 and r0 + 8 of two tiles of 16
        for (int rt = 0; rt < row_tiles; ++rt) {
            if (row_tiles > 1) {
                fetch(cur, rt, now);
                take(cur, rt);
            }
            float s[2][NT][4];
#pragma unroll
            for (int i = 0; i < 2; ++i)
#pragma unroll
                for (int t = 0; t < NT; ++t) { s[i][t][0] = 0.f; s[i][t][1] = 0.f; s[i][t][2] = 0.f; s[i][t][3] = 0.f; }
#pragma unroll
            for (int a = 0; a < RB / 64; ++a) {
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    // chunk 4 a + c of keys row and row + 8: tiles start at multiples of 1024, so a only flips bits
                    const int at = ((k_first + 16 * i * LINE) ^ ((a & 1) << 6)) + (a >> 1) * (T * 128);
                    const uint4 w0 = *reinterpret_cast<const uint4 *>(smem + at), w1 = *reinterpret_cast<const uint4 *>(smem + at + 8 * LINE);
                    const uint32_t x0[4] = {w0.x, w0.y, w0.z, w0.w}, x1[4] = {w1.x, w1.y, w1.z, w1.w};
                    if constexpr (!EIGHT) {
#pragma unroll
                        for (int x = 0; x < 2; ++x) {
                            const uint32_t f[4] = {x0[2 * x], x1[2 * x], x0[2 * x + 1], x1[2 * x + 1]};
#pragma unroll
                            for (int t = 0; t < NT; ++t) mma<false>(s[i][t], f, now.q[t][2 * a + x]);
                        }
                    } else {
#pragma unroll
                        for (int x = 0; x < 4; ++x) {
                            uint32_t f[4];
                            widen<KIND>(x0[x], f[0], f[2]);
                            widen<KIND>(x1[x], f[1], f[3]);
#pragma unroll
                            for (int t = 0; t < NT; ++t) mma<true>(s[i][t], f, now.q[t][4 * a + x]);
                        }
                    }
                }
            }
#pragma unroll
            for (int i = 0; i < 2; ++i)
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    const int n = n0 + 16 * i + 8 * e + key_of<RB>(r0);
                    // (byte 0: nothing above 2^-118, counts as zero; byte 255: infinity, then NaN)
                    const float f = EIGHT ? __uint_as_float(static_cast<uint32_t>(exps[stage * T + n]) << 23) : 1.f;
#pragma unroll
                    for (int t = 0; t < NT; ++t)
#pragma unroll
                        for (int h = 0; h < 2; ++h) {
                            const float p = kva::ex2(fmaf(s[i][t][2 * e + h], EIGHT ? f * scale[t][h] : scale[t][h], shift[t][h]));
                            sum[i][e] += j0 + n > pos[t][h] ? 0.f : p;
                        }
                }
        }
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                sum[i][e] += __shfl_xor_sync(0xFFFFFFFFu, sum[i][e], 1);
                sum[i][e] += __shfl_xor_sync(0xFFFFFFFFu, sum[i][e], 2);
            }
        {                                                     // lane c of a key's four writes key r0 + 8 (c & 1) of tile c / 2
            const int n = n0 + 8 * c + key_of<RB>(r0), j = j0 + n;
            const long long place = places[stage * BLOCKS + n / 8];
            const float given = c == 0 ? sum[0][0] : c == 1 ? sum[0][1] : c == 2 ? sum[1][0] : sum[1][1];
            if (place >= 0 && j < cur.len) {
                const float old = g.a.decay != 0.f && j < cur.n_old ? g.a.decay * olds[stage * T + n] : 0.f;
                held[place + (n & 7)] = old + given;
            }
        }
        __syncwarp();
        if (lane == 0) mbar_arrive(&ring.empty[stage]);
        more = onward();
    }
    kva::let_copies_land(gave_up);            // (the producers may have gone before the last wait gave up)
}

template <int KIND, int D, int NT> static siso_status_t run(Kv *h, const Args &g, cudaStream_t s) {
    using S = Shape<KIND, D, NT>;
    constexpr uint32_t bit = 1u << (NT == 1 ? 20 : NT == 2 ? 21 : 22);
    if (!(h->attr_set & bit)) {
        SISO_CUDA(cudaFuncSetAttribute(weights_few_rows_kernel<KIND, D, NT>, cudaFuncAttributeMaxDynamicSharedMemorySize, S::SMEM));
        h->attr_set |= bit;
    }
    return launch_early(weights_few_rows_kernel<KIND, D, NT>, dim3(static_cast<unsigned>(h->sm_count)), S::THREADS, S::SMEM, s, g, h->map_k);
}
template <int KIND> static siso_status_t run_rows(Kv *h, const Args &g, int rows, cudaStream_t s) {
    if (h->cfg.head_dim == 128) return rows <= 8 ? run<KIND, 128, 1>(h, g, s) : rows <= 16 ? run<KIND, 128, 2>(h, g, s) : run<KIND, 128, 4>(h, g, s);
    return rows <= 8 ? run<KIND, 64, 1>(h, g, s) : rows <= 16 ? run<KIND, 64, 2>(h, g, s) : run<KIND, 64, 4>(h, g, s);
}

}  // namespace few

siso_status_t launch_few_rows(Kv *h, const siso_weights_t *a, const int32_t *fresh, int rows, cudaStream_t s) {
    few::Args g;
    g.fresh = fresh;
    g.kv = kv_view(h, a->layer);
    g.a = *a;
    g.group = a->n_heads / h->cfg.n_kv_heads;
    g.by_page.set(static_cast<uint32_t>(h->cfg.page_size));
    g.by_group.set(static_cast<uint32_t>(g.group));
    g.scale_log2 = a->scale * 1.4426950408889634f;
    g.status = h->status;
    g.box = h->box;
    switch (h->cfg.dtype) {
        case SISO_BF16: return few::run_rows<SISO_BF16>(h, g, rows, s);
        case SISO_E4M3: return few::run_rows<SISO_E4M3>(h, g, rows, s);
        default: return few::run_rows<SISO_I8>(h, g, rows, s);
    }
}

}  // namespace kvw
}  // namespace siso
