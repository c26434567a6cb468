// Attention of new tokens over the paged key/value cache, few rows per key/value head: single tokens of decoding and short
// runs of drafted ones.
//
// Token i of sequence b (q_len new tokens, already in the cache, kv_len tokens in all) stands at p = kv_len - q_len + i and
// sees the tokens j in [0, kv_len) with j <= p (causal) and j > p - window (window > 0):
//     s_j = scale q.k_j,  m = max s,  l = sum exp(s_j - m),  out = sum exp(s_j - m) v_j / l,  lse = m + ln l
// A row that sees nothing gives out = 0 and lse = -infinity.
//
// With few rows every byte of the cache meets few multiplications, so the call is bound by HBM: the point is to keep loads in
// flight.  One CTA of 8 warps per SM holds a ring of units (128 keys and their values, about 190 KB in all) filled by cp.async,
// two units or more ahead.  WK = 8 / WM groups of WM warps split the unit's keys; a warp owns 16 rows and its group's keys, so up
// to 16 rows (WM = 1) no byte is read from shared memory twice and no warp waits for another inside a run of units.
// Matrix products are mma.sync m16n8k16 with fp32 sums: tcgen05 works on 128 rows, of which a decoding step would fill 1 to 16.
// K fragments come straight from 16-byte shared loads: the sum over d may be taken in any order, so a lane takes 16 consecutive
// bytes of its key and the queries are laid out to match.  V fragments come through ldmatrix.trans; over 8-bit codes it hands
// a lane the pairs (key, d), (key, d + 1), (key + 1, d), (key + 1, d + 1), which are the fragments of an even and an odd column.
// 8-bit codes are turned into fp16, not bf16: one conversion per two codes, exact.  The key's scale goes to its score, the
// value's to its probability relative to the largest one so far.  Queries are brought into fp16's range by a power of two per row
// (exact but for elements 2^-39 below the row's largest), probabilities are scaled by 2^15.
#include <cuda_fp16.h>

#include "kv_attention.cuh"

namespace siso {
namespace kva {

constexpr int THREADS = 256;
constexpr int SMEM_MOST = 232448 - 256;   // what a CTA may have, less its static part

template <int KIND, int D, int WM> struct Shape {
    static constexpr int WK = 8 / WM;                       // groups of warps along the keys
    static constexpr int MR = 16 * WM;                      // rows of a row tile
    static constexpr int NK = TK / WK;                      // keys of a group
    static constexpr bool EIGHT = KIND != SISO_BF16;
    static constexpr int RB = D * (EIGHT ? 1 : 2);          // bytes of a row
    static constexpr int CH = RB / 16;                      // 16-byte chunks of a row
    static constexpr int STAGE = 2 * TK * RB;
    static constexpr int META = TK * 4 + (EIGHT ? 2 * TK : 0);        // whether each key is there, exponents
    static constexpr int MERGE = 4 * 16 * D * 4 + 8 * 16 * 2 * 4;     // outputs, maxima and sums of half the warps
    static constexpr int FIT = (SMEM_MOST - MERGE) / (STAGE + META);
    static constexpr int STAGES = FIT > 8 ? 8 : FIT;
    static constexpr int SMEM = STAGES * (STAGE + META) + MERGE;
};

// byte offset of a 16-byte chunk in a tile of rows: neighbouring rows differ in the upper half of a 128-byte line (the 8 lanes of a
// 16-byte load read 4 chunks of 2 rows), and 8 rows of one chunk differ in all of it (ldmatrix)
template <int CH> __device__ __forceinline__ int chunk_at(int row, int chunk) {
    if constexpr (CH == 4) return row * 64 + ((chunk ^ ((row >> 1) & 3)) << 4);
    else return row * (CH * 16) + ((chunk ^ (((row & 1) << 2) | ((row >> 1) & 3))) << 4);
}
__device__ __forceinline__ void copy16(uint32_t dst, const void *src, bool take) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(take ? 16 : 0) : "memory");
}
__device__ __forceinline__ void copy8(uint32_t dst, const void *src, bool take) {
    asm volatile("cp.async.ca.shared.global [%0], [%1], 8, %2;" ::"r"(dst), "l"(src), "r"(take ? 8 : 0) : "memory");
}
template <bool HALF> __device__ __forceinline__ void mma(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
    if constexpr (HALF)
        asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                     : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
    else
        asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                     : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ void load_v(uint32_t addr, uint32_t (&r)[4]) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ uint32_t pack(float lo, float hi, bool half) {
    uint32_t r;
    if (half) asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    else asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}
// Two codes as fp16: bytes 0, 1 and 2, 3 of a word (SPLIT false), or bytes 0, 2 and 1, 3 (SPLIT true)
template <int KIND, bool SPLIT> __device__ __forceinline__ void widen(uint32_t w, uint32_t &lo, uint32_t &hi) {
    if constexpr (KIND == SISO_E4M3) {
        if constexpr (SPLIT) w = __byte_perm(w, 0u, 0x3120);
        asm("{\n\t.reg .b16 l, h;\n\tmov.b32 {l, h}, %2;\n\tcvt.rn.f16x2.e4m3x2 %0, l;\n\tcvt.rn.f16x2.e4m3x2 %1, h;\n\t}"
            : "=r"(lo), "=r"(hi) : "r"(w));
    } else {
        w ^= 0x80808080u;                                   // c + 128; beside the byte 0x64 it is the fp16 number 1024 + c + 128
        const __half2 off = __halves2half2(__ushort_as_half(0x6480), __ushort_as_half(0x6480));
        const uint32_t a = __byte_perm(w, 0x64646464u, SPLIT ? 0x4240 : 0x4140), b = __byte_perm(w, 0x64646464u, SPLIT ? 0x4341 : 0x4342);
        const __half2 x = __hsub2(*reinterpret_cast<const __half2 *>(&a), off), y = __hsub2(*reinterpret_cast<const __half2 *>(&b), off);
        lo = *reinterpret_cast<const uint32_t *>(&x);
        hi = *reinterpret_cast<const uint32_t *>(&y);
    }
}

template <int KIND, int D, int WM>
__global__ void __launch_bounds__(THREADS, 1)
attention_few_rows_kernel(const __grid_constant__ Args g) {
    using S = Shape<KIND, D, WM>;
    constexpr int NK = S::NK, CH = S::CH, RB = S::RB, MR = S::MR;
    constexpr bool EIGHT = S::EIGHT;
    constexpr int SUB = NK < 32 ? NK : 32;                   // keys between two looks at the running maximum
    constexpr int ROWS = CH / 2;                             // key rows that a thread copies per unit
    constexpr int STEP = 32 * WM / CH;                       // rows that a group copies at once
    constexpr int O_TILES = D / 8;
    extern __shared__ __align__(128) uint8_t smem[];
    uint8_t *meta = smem + S::STAGES * S::STAGE;
    float *merge_o = reinterpret_cast<float *>(meta + S::STAGES * S::META);
    float *merge_ml = merge_o + 4 * 16 * D;
    __shared__ unsigned long long buf[THREADS / 32 + 2];

    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int kg = warp / WM, wm = warp % WM;
    const int tg = threadIdx.x % (32 * WM);                  // thread of the group
    const int c = lane & 3, r0 = lane >> 2;

    long long u0, u1, total;
    int ctas;
    Cursor<MR> cur;
    if (!locate<MR, THREADS>(g, u0, u1, total, ctas, cur, buf)) return;
    Cursor<MR> ahead = cur;

    // ---- loading: page indices are fetched one unit before the copies that need them
    int pages[ROWS], exp_page = -1;
    long long ahead_u = u0;
    auto page_of = [&](int j) -> int {
        if (j >= ahead.s.hi) return -1;
        const int page = g.a.d_pages[ahead.b * g.a.pages_stride + g.by_page.div(j)];
        if (page >= 0 && page < g.kv.n_pages) return page;
        set_status(g.status, SISO_ERR_INVALID_ARG);
        return -1;
    };
    auto fetch_pages = [&]() {
        const int j0 = (ahead.s.tile0 + ahead.tile) * TK + kg * NK;
#pragma unroll
        for (int i = 0; i < ROWS; ++i) pages[i] = page_of(j0 + tg / CH + i * STEP);
        if (EIGHT && tg < NK / 4) exp_page = page_of(j0 + (tg % (NK / 8)) * 8);
    };
    auto issue = [&](int stage) {
        const int j0 = (ahead.s.tile0 + ahead.tile) * TK + kg * NK;
        const uint32_t k_dst = static_cast<uint32_t>(__cvta_generic_to_shared(smem + stage * S::STAGE));
        const uint32_t v_dst = k_dst + TK * RB;
        uint32_t *there = reinterpret_cast<uint32_t *>(meta + stage * S::META);
        const int chunk = tg % CH;
#pragma unroll
        for (int i = 0; i < ROWS; ++i) {
            const int r = kg * NK + tg / CH + i * STEP, j = j0 + tg / CH + i * STEP;
            const int page = max(pages[i], 0);
            const int t = j - static_cast<int>(g.by_page.div(j)) * g.kv.page_size;
            const long long at = (page * g.kv.stride_page + t * g.kv.stride_token + ahead.head * g.kv.stride_head) * (RB / D) + chunk * 16;
            copy16(k_dst + chunk_at<CH>(r, chunk), static_cast<const char *>(g.kv.k) + (pages[i] < 0 ? 0 : at), pages[i] >= 0);
            copy16(v_dst + chunk_at<CH>(r, chunk), static_cast<const char *>(g.kv.v) + (pages[i] < 0 ? 0 : at), pages[i] >= 0);
            if (chunk == 0) there[r] = pages[i] < 0 ? 0u : 0xFFFFFFFFu;
        }
        if (EIGHT && tg < NK / 4) {                          // 8 exponents of a page lie side by side
            const int blk = tg % (NK / 8), j = j0 + blk * 8;
            const bool is_v = tg >= NK / 8;
            const int t = j - static_cast<int>(g.by_page.div(j)) * g.kv.page_size;
            const long long at = exp_page < 0 ? 0 : (static_cast<long long>(exp_page) * g.kv.n_kv_heads + ahead.head) * g.kv.page_size + t;
            const uint32_t dst = static_cast<uint32_t>(__cvta_generic_to_shared(meta + stage * S::META)) + TK * 4 + (is_v ? TK : 0) + kg * NK + blk * 8;
            copy8(dst, (is_v ? g.kv.v_exp : g.kv.k_exp) + at, exp_page >= 0);
        }
    };
    auto load_unit = [&](int stage) {
        if (ahead_u < u1) {
            issue(stage);
            if (++ahead_u < u1) {
                if (++ahead.tile == ahead.s.tiles) ahead.next_item(g);
                fetch_pages();
            }
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
    };
    fetch_pages();
#pragma unroll 1
    for (int s = 0; s < S::STAGES - 1; ++s) load_unit(s);

    // ---- state of the row tile: this warp's 16 rows over its group's keys
    uint32_t q[D / 16][4];
    float o[O_TILES][4], m[2], l[2], row_scale[2];
    int pos[2], e_top = 0;
    long long began = u0;                                    // unit at which the current part of the item began
    bool fresh = true;
    int stage = 0;
    for (long long u = u0; u < u1; ++u) {
        if (fresh) {
            fresh = false;
            began = u;
            e_top = 0;
#pragma unroll
            for (int t = 0; t < O_TILES; ++t) { o[t][0] = 0.f; o[t][1] = 0.f; o[t][2] = 0.f; o[t][3] = 0.f; }
            uint4 raw[2][EIGHT ? D / 32 : D / 32];           // 16 bytes of each of D / 32 chunks, two rows
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int row = cur.rt * MR + wm * 16 + r0 + 8 * h;
                const bool real = row < cur.n_q * g.group;
                const int i = static_cast<int>(g.by_group.div(static_cast<uint32_t>(real ? row : 0)));
                const int head = cur.head * g.group + (real ? row - i * g.group : 0);
                pos[h] = real ? cur.len - cur.n_q + i : cur.s.last_pos;
                m[h] = -INFINITY;
                l[h] = 0.f;
                row_scale[h] = g.scale_log2;
                const __nv_bfloat16 *src = static_cast<const __nv_bfloat16 *>(g.a.d_q) + static_cast<long long>(cur.q0 + i) * g.a.q_stride_token + head * g.a.q_stride_head;
#pragma unroll
                for (int x = 0; x < D / 32; ++x) {
                    // bf16 cache: a lane's 16 bytes of a key hold 8 values; 8-bit: 16 values, two pieces of 8
                    const int d = EIGHT ? ((x / 2) * 4 + c) * 16 + (x & 1) * 8 : (x * 4 + c) * 8;
                    raw[h][x] = real ? *reinterpret_cast<const uint4 *>(src + d) : make_uint4(0u, 0u, 0u, 0u);
                }
            }
            if constexpr (EIGHT) {
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    uint32_t top = 0u;
#pragma unroll
                    for (int x = 0; x < D / 32; ++x) {
                        const uint32_t w[4] = {raw[h][x].x, raw[h][x].y, raw[h][x].z, raw[h][x].w};
#pragma unroll
                        for (int i = 0; i < 4; ++i) top = max(top, max((w[i] << 16) & 0x7FFF0000u, w[i] & 0x7FFF0000u));
                    }
                    top = max(top, __shfl_xor_sync(0xFFFFFFFFu, top, 1));
                    top = max(top, __shfl_xor_sync(0xFFFFFFFFu, top, 2));
                    const int ex = min(max(static_cast<int>(top >> 23), 16), 254);     // the row's largest value becomes 2^14 .. 2^15
                    const float up = __uint_as_float(static_cast<uint32_t>(min(127 + 14 + 127 - ex, 254)) << 23);
                    row_scale[h] *= 1.f / up;
#pragma unroll
                    for (int x = 0; x < D / 32; ++x) {
                        uint32_t w[4] = {raw[h][x].x, raw[h][x].y, raw[h][x].z, raw[h][x].w};
#pragma unroll
                        for (int i = 0; i < 4; ++i) w[i] = pack(__uint_as_float(w[i] << 16) * up, __uint_as_float(w[i] & 0xFFFF0000u) * up, true);
                        raw[h][x] = make_uint4(w[0], w[1], w[2], w[3]);
                    }
                }
            }
#pragma unroll
            for (int x = 0; x < D / 32; ++x) {
                q[2 * x][0] = raw[0][x].x; q[2 * x][2] = raw[0][x].y; q[2 * x + 1][0] = raw[0][x].z; q[2 * x + 1][2] = raw[0][x].w;
                q[2 * x][1] = raw[1][x].x; q[2 * x][3] = raw[1][x].y; q[2 * x + 1][1] = raw[1][x].z; q[2 * x + 1][3] = raw[1][x].w;
            }
        }
        asm volatile("cp.async.wait_group %0;" ::"n"(S::STAGES - 2) : "memory");
        if constexpr (WM == 1) __syncwarp();
        else asm volatile("bar.sync %0, %1;" ::"r"(kg + 1), "n"(32 * WM) : "memory");
        load_unit(stage == 0 ? S::STAGES - 1 : stage - 1);

        const uint8_t *k_tile = smem + stage * S::STAGE;
        const uint32_t v_tile = static_cast<uint32_t>(__cvta_generic_to_shared(k_tile)) + TK * RB;
        const uint8_t *mt = meta + stage * S::META;
        const int j0 = (cur.s.tile0 + cur.tile) * TK;
        const bool cut = ((g.a.flags & SISO_ATTN_CAUSAL) && j0 + TK - 1 > cur.s.first_pos) ||
                         (g.a.window > 0 && j0 <= cur.s.last_pos - g.a.window);
#pragma unroll 1
        for (int n0 = kg * NK; n0 < (kg + 1) * NK; n0 += SUB) {
            float s[SUB / 8][4];
#pragma unroll
            for (int i = 0; i < SUB / 8; ++i) { s[i][0] = 0.f; s[i][1] = 0.f; s[i][2] = 0.f; s[i][3] = 0.f; }
#pragma unroll
            for (int a = 0; a < RB / 64; ++a) {
#pragma unroll
                for (int i = 0; i < SUB / 8; ++i) {
                    const uint4 w = *reinterpret_cast<const uint4 *>(k_tile + chunk_at<CH>(n0 + 8 * i + r0, 4 * a + c));
                    if constexpr (!EIGHT) {
                        mma<false>(s[i], q[2 * a], w.x, w.y);
                        mma<false>(s[i], q[2 * a + 1], w.z, w.w);
                    } else {
                        const uint32_t ws[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
                        for (int x = 0; x < 4; ++x) {
                            uint32_t b0, b1;
                            widen<KIND, false>(ws[x], b0, b1);
                            mma<true>(s[i], q[4 * a + x], b0, b1);
                        }
                    }
                }
            }
            // scores in powers of two, masks, running maximum.  A key that is not there is left out by selection, not by adding
            // -infinity: its exponents may be anything
            float top[2] = {-INFINITY, -INFINITY};
            uint32_t ev[SUB / 8];
            uint32_t e_max = 0u;
#pragma unroll
            for (int i = 0; i < SUB / 8; ++i) {
                const int n = n0 + 8 * i + 2 * c;
                const uint2 there = *reinterpret_cast<const uint2 *>(mt + n * 4);
                float ks0 = 1.f, ks1 = 1.f;
                if constexpr (EIGHT) {
                    const uint32_t e = *reinterpret_cast<const uint16_t *>(mt + TK * 4 + n);
                    ks0 = kv_scale(e & 0xFFu);
                    ks1 = kv_scale(e >> 8);
                    ev[i] = *reinterpret_cast<const uint16_t *>(mt + TK * 5 + n) & (there.x & 0xFFu | there.y & 0xFF00u);
                    e_max = max(e_max, max(ev[i] & 0xFFu, ev[i] >> 8));
                }
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const float x0 = EIGHT ? s[i][2 * h] * ks0 * row_scale[h] : s[i][2 * h] * row_scale[h];
                    const float x1 = EIGHT ? s[i][2 * h + 1] * ks1 * row_scale[h] : s[i][2 * h + 1] * row_scale[h];
                    s[i][2 * h] = there.x ? x0 : -INFINITY;
                    s[i][2 * h + 1] = there.y ? x1 : -INFINITY;
                    if (cut) {
                        const int j = j0 + n;
                        const int last = (g.a.flags & SISO_ATTN_CAUSAL) ? pos[h] : 0x7FFFFFFF;
                        const int first = g.a.window > 0 ? pos[h] - g.a.window : -0x7FFFFFFF;
                        if (j > last || j <= first) s[i][2 * h] = -INFINITY;
                        if (j + 1 > last || j + 1 <= first) s[i][2 * h + 1] = -INFINITY;
                    }
                    top[h] = fmaxf(top[h], fmaxf(s[i][2 * h], s[i][2 * h + 1]));
                }
            }
            float shift[2], corr[2];
            bool moved = false;
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                top[h] = fmaxf(top[h], __shfl_xor_sync(0xFFFFFFFFu, top[h], 1));
                top[h] = fmaxf(top[h], __shfl_xor_sync(0xFFFFFFFFu, top[h], 2));
                const float m2 = fmaxf(m[h], top[h]);
                corr[h] = m[h] == m2 ? 1.f : ex2(m[h] - m2);
                moved = moved || m[h] != m2;
                m[h] = m2;
                shift[h] = m2 == -INFINITY ? 0.f : m2 - (EIGHT ? 15.f : 0.f);
                l[h] *= corr[h];
            }
            float rel[SUB / 8][2];                            // 2^(value exponent - largest so far)
            if constexpr (EIGHT) {
                e_max = __reduce_max_sync(0xFFFFFFFFu, e_max);
                if (static_cast<int>(e_max) > e_top) {
                    const float down = ex2(static_cast<float>(e_top - static_cast<int>(e_max)));
                    corr[0] *= down;
                    corr[1] *= down;
                    moved = true;
                    e_top = static_cast<int>(e_max);
                }
#pragma unroll
                for (int i = 0; i < SUB / 8; ++i) {
                    rel[i][0] = __uint_as_float(static_cast<uint32_t>(max(127 + static_cast<int>(ev[i] & 0xFFu) - e_top, 0)) << 23);
                    rel[i][1] = __uint_as_float(static_cast<uint32_t>(max(127 + static_cast<int>(ev[i] >> 8) - e_top, 0)) << 23);
                }
            }
            if (__any_sync(0xFFFFFFFFu, moved)) {
#pragma unroll
                for (int t = 0; t < O_TILES; ++t) { o[t][0] *= corr[0]; o[t][1] *= corr[0]; o[t][2] *= corr[1]; o[t][3] *= corr[1]; }
            }
            uint32_t p[SUB / 8][2];
#pragma unroll
            for (int i = 0; i < SUB / 8; ++i) {
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const float p0 = ex2(s[i][2 * h] - shift[h]), p1 = ex2(s[i][2 * h + 1] - shift[h]);
                    l[h] += p0 + p1;
                    p[i][h] = EIGHT ? pack(p0 * rel[i][0], p1 * rel[i][1], true) : pack(p0, p1, false);
                }
            }
#pragma unroll
            for (int k16 = 0; k16 < SUB / 16; ++k16) {
                const uint32_t a[4] = {p[2 * k16][0], p[2 * k16][1], p[2 * k16 + 1][0], p[2 * k16 + 1][1]};
                const int row = n0 + 16 * k16 + (lane & 15);
#pragma unroll
                for (int x = 0; x < CH; x += 2) {             // two chunks at once: keys 0-7 and 8-15 of each
                    uint32_t v[4];
                    load_v(v_tile + chunk_at<CH>(row, x + (lane >> 4)), v);
                    if constexpr (!EIGHT) {
                        mma<false>(o[x], a, v[0], v[1]);
                        mma<false>(o[x + 1], a, v[2], v[3]);
                    } else {
                        uint32_t e0, d0, e1, d1;
                        widen<KIND, true>(v[0], e0, d0);
                        widen<KIND, true>(v[1], e1, d1);
                        mma<true>(o[2 * x], a, e0, e1);
                        mma<true>(o[2 * x + 1], a, d0, d1);
                        widen<KIND, true>(v[2], e0, d0);
                        widen<KIND, true>(v[3], e1, d1);
                        mma<true>(o[2 * x + 2], a, e0, e1);
                        mma<true>(o[2 * x + 3], a, d0, d1);
                    }
                }
            }
        }
        if (++stage == S::STAGES) stage = 0;
        if (++cur.tile < cur.s.tiles && u + 1 < u1) continue;

        // ---- end of the item, or of this CTA's part of it: join the groups' results, halving their number each time
        fresh = true;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            l[h] += __shfl_xor_sync(0xFFFFFFFFu, l[h], 1);
            l[h] += __shfl_xor_sync(0xFFFFFFFFu, l[h], 2);
            if (EIGHT) m[h] -= 15.f;
        }
        if constexpr (EIGHT) {
            const float back = kv_scale(static_cast<uint32_t>(e_top));
#pragma unroll
            for (int t = 0; t < O_TILES; ++t) { o[t][0] *= back; o[t][1] *= back; o[t][2] *= back; o[t][3] *= back; }
        }
#pragma unroll 1
        for (int half = S::WK / 2; half >= 1; half >>= 1) {
            float4 *mo = reinterpret_cast<float4 *>(merge_o) + ((kg % half) * WM + wm) * (O_TILES * 32) + lane;
            float *ml = merge_ml + ((kg % half) * WM + wm) * 32 + 4 * r0;
            if (kg >= half && kg < 2 * half) {
#pragma unroll
                for (int t = 0; t < O_TILES; ++t) mo[t * 32] = make_float4(o[t][0], o[t][1], o[t][2], o[t][3]);
                if (c == 0) { ml[0] = m[0]; ml[1] = l[0]; ml[2] = m[1]; ml[3] = l[1]; }
            }
            __syncthreads();
            if (kg < half) {
                float mine[2], theirs[2];
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const float m1 = ml[2 * h], l1 = ml[2 * h + 1], m2 = fmaxf(m[h], m1);
                    mine[h] = m[h] == -INFINITY ? 0.f : ex2(m[h] - m2);
                    theirs[h] = m1 == -INFINITY ? 0.f : ex2(m1 - m2);
                    l[h] = l[h] * mine[h] + l1 * theirs[h];
                    m[h] = m2;
                }
#pragma unroll
                for (int t = 0; t < O_TILES; ++t) {
                    const float4 y = mo[t * 32];
                    o[t][0] = o[t][0] * mine[0] + y.x * theirs[0];
                    o[t][1] = o[t][1] * mine[0] + y.y * theirs[0];
                    o[t][2] = o[t][2] * mine[1] + y.z * theirs[1];
                    o[t][3] = o[t][3] * mine[1] + y.w * theirs[1];
                }
            }
            __syncthreads();
        }
        const int t_end = cur.tile;                           // tiles [t_end - (u + 1 - began), t_end) of the item are done here
        const int t_begin = t_end - static_cast<int>(u + 1 - began);
        const bool whole = t_begin == 0 && t_end == cur.s.tiles;
        if (kg == 0) {
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int in_tile = wm * 16 + r0 + 8 * h, row = cur.rt * MR + in_tile;
                if (row < cur.n_q * g.group) {
                    if (whole) {
                        const int i = static_cast<int>(g.by_group.div(static_cast<uint32_t>(row)));
                        const int head = cur.head * g.group + row - i * g.group;
                        const float inv = l[h] > 0.f ? 1.f / l[h] : 0.f;
                        __nv_bfloat16 *dst = static_cast<__nv_bfloat16 *>(g.a.d_out) + static_cast<long long>(cur.q0 + i) * g.a.out_stride_token + head * g.a.out_stride_head;
                        if constexpr (!EIGHT) {
#pragma unroll
                            for (int t = 0; t < O_TILES; ++t)
                                *reinterpret_cast<uint32_t *>(dst + 8 * t + 2 * c) = pack(o[t][2 * h] * inv, o[t][2 * h + 1] * inv, false);
                        } else {
#pragma unroll
                            for (int t = 0; t < O_TILES; t += 2)
                                *reinterpret_cast<uint2 *>(dst + 8 * t + 4 * c) = make_uint2(pack(o[t][2 * h] * inv, o[t + 1][2 * h] * inv, false),
                                                                                            pack(o[t][2 * h + 1] * inv, o[t + 1][2 * h + 1] * inv, false));
                        }
                        if (g.a.d_lse && c == 0)
                            g.a.d_lse[static_cast<long long>(cur.q0 + i) * g.a.n_heads + head] = l[h] > 0.f ? (m[h] + log2f(l[h])) * 0.6931471805599453f : -INFINITY;
                    } else {
                        const long long place = part_place(blockIdx.x, t_begin > 0) * MR + in_tile;
                        float *dst = g.part_o + place * D;
#pragma unroll
                        for (int t = 0; t < O_TILES; t += 2) {
                            if constexpr (!EIGHT) {
                                *reinterpret_cast<float2 *>(dst + 8 * t + 2 * c) = make_float2(o[t][2 * h], o[t][2 * h + 1]);
                                *reinterpret_cast<float2 *>(dst + 8 * t + 8 + 2 * c) = make_float2(o[t + 1][2 * h], o[t + 1][2 * h + 1]);
                            } else {
                                *reinterpret_cast<float4 *>(dst + 8 * t + 4 * c) = make_float4(o[t][2 * h], o[t + 1][2 * h], o[t][2 * h + 1], o[t + 1][2 * h + 1]);
                            }
                        }
                        if (c == 0) *reinterpret_cast<float2 *>(g.part_ml + place * 2) = make_float2(m[h], l[h]);
                    }
                }
            }
        }
        if (!whole && t_begin == 0 && threadIdx.x == 0) {
            const long long end = u + 1 + (cur.s.tiles - t_end);
            g.records[blockIdx.x] = Record{1, cur.b, cur.head, cur.rt, cta_of(end - 1, total, ctas) - static_cast<int>(blockIdx.x) + 1};
        }
        if (u + 1 < u1) cur.next_item(g);
    }
}

// ---- joining the parts ------------------------------------------------------------------------------------------------
// CTA (x, y): the item that is recorded at CTA x, MR / 8 of its rows.  The parts lie at place 1 of CTA x and place 0 of the next
// ones.  256 / (MR / 8) threads share a row: 32 lanes over d, the warps over the parts; sums are taken in the same order every time.
template <int MR, int D>
__global__ void __launch_bounds__(256)
join_kernel(const __grid_constant__ Args g) {
    constexpr int ROWS = MR / 8 < 8 ? MR / 8 : 8, WPR = 8 / ROWS;          // rows of a CTA at a time, warps of a row
    constexpr int N = D / 32;
    __shared__ float so[8][D], sml[8][2];
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const Record rec = g.records[blockIdx.x];
    if (!rec.valid) return;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    int q0;
    const int n_q = seq_queries(g, rec.b, q0);
    for (int base = blockIdx.y * (MR / 8); base < (blockIdx.y + 1) * (MR / 8); base += ROWS) {
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
                    if (ml[f].x == -INFINITY) continue;
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
            if (part0 != 0) continue;
#pragma unroll
            for (int w = 1; w < WPR; ++w) {
                const float m1 = sml[warp + w][0], l1 = sml[warp + w][1];
                if (m1 == -INFINITY) continue;
                const float m2 = fmaxf(m, m1), a = m == -INFINITY ? 0.f : ex2(m - m2), b = ex2(m1 - m2);
                l = l * a + l1 * b;
                m = m2;
#pragma unroll
                for (int x = 0; x < N; ++x) o[x] = o[x] * a + so[warp + w][x * 32 + lane] * b;
            }
        }
        if (!real) continue;
        const int i = static_cast<int>(g.by_group.div(static_cast<uint32_t>(row))), head = rec.head * g.group + row - i * g.group;
        const float inv = l > 0.f ? 1.f / l : 0.f;
        __nv_bfloat16 *dst = static_cast<__nv_bfloat16 *>(g.a.d_out) + static_cast<long long>(q0 + i) * g.a.out_stride_token + head * g.a.out_stride_head;
#pragma unroll
        for (int x = 0; x < N; ++x) dst[x * 32 + lane] = __float2bfloat16_rn(o[x] * inv);
        if (g.a.d_lse && lane == 0)
            g.a.d_lse[static_cast<long long>(q0 + i) * g.a.n_heads + head] = l > 0.f ? (m + log2f(l)) * 0.6931471805599453f : -INFINITY;
    }
}

template <int MR, int D> static siso_status_t run_join(const Args &g, cudaStream_t s) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(static_cast<unsigned>(g.grid), 8);
    cfg.blockDim = dim3(256);
    cfg.stream = s;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;       // its CTAs may be set up while the parts are still made
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    SISO_CUDA(cudaLaunchKernelEx(&cfg, join_kernel<MR, D>, g));
    SISO_CUDA(cudaGetLastError());
    return SISO_OK;
}
siso_status_t launch_join(const Args &g, int mr, int dim, cudaStream_t s) {
    if (dim == 128) return mr == 16 ? run_join<16, 128>(g, s) : mr == 32 ? run_join<32, 128>(g, s) : run_join<64, 128>(g, s);
    return mr == 16 ? run_join<16, 64>(g, s) : mr == 32 ? run_join<32, 64>(g, s) : run_join<64, 64>(g, s);
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

template <int KIND, int D, int WM> static siso_status_t run_few(Args &g, cudaStream_t s) {
    using S = Shape<KIND, D, WM>;
    // the opt-in to large shared memory is an attribute of the function on the current device; setting it again is cheap
    SISO_CUDA(cudaFuncSetAttribute(attention_few_rows_kernel<KIND, D, WM>, cudaFuncAttributeMaxDynamicSharedMemorySize, S::SMEM));
    attention_few_rows_kernel<KIND, D, WM><<<g.grid, THREADS, S::SMEM, s>>>(g);
    SISO_CUDA(cudaGetLastError());
    return launch_join(g, S::MR, D, s);
}
template <int KIND, int D> static siso_status_t run_few_wm(Args &g, int wm, cudaStream_t s) {
    return wm == 1 ? run_few<KIND, D, 1>(g, s) : wm == 2 ? run_few<KIND, D, 2>(g, s) : run_few<KIND, D, 4>(g, s);
}
template <int KIND> static siso_status_t run_few_dim(Args &g, int dim, int wm, cudaStream_t s) {
    return dim == 128 ? run_few_wm<KIND, 128>(g, wm, s) : run_few_wm<KIND, 64>(g, wm, s);
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
    g.grid = h->sm_count;
    const int dim = h->cfg.head_dim;
    const long long rows = static_cast<long long>(a->max_q) * g.group;      // rows per key/value head of the longest chunk
    const int wm = rows <= 16 ? 1 : rows <= 32 ? 2 : 4;
    const int mr = 16 * wm;
    const size_t records = pad256(sizeof(Record) * g.grid), ml = pad256(sizeof(float) * 2 * g.grid * mr * 2);
    // sized for the widest kernel, so that a handle that has served one call serves every other without a new block
    const size_t most = records + pad256(sizeof(float) * 2 * g.grid * 64 * 2) + sizeof(float) * 2 * g.grid * 64 * static_cast<size_t>(dim);
    SISO_TRY(kv_scratch(h, most, s));
    char *ws = static_cast<char *>(h->ws);
    g.records = reinterpret_cast<Record *>(ws);
    g.part_ml = reinterpret_cast<float *>(ws + records);
    g.part_o = reinterpret_cast<float *>(ws + records + ml);
    switch (h->cfg.dtype) {
        case SISO_BF16: return run_few_dim<SISO_BF16>(g, dim, wm, s);
        case SISO_E4M3: return run_few_dim<SISO_E4M3>(g, dim, wm, s);
        default: return run_few_dim<SISO_I8>(g, dim, wm, s);
    }
}

}  // namespace siso
